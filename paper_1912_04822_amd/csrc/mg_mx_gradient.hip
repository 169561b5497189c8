// Weight gradient of a linear map from the 8-bit codes of its input (formats: mg_mx.h):
//     dW[t][e] = sum over live rows m of G[m][t] X[m][e],     db[t] = sum over live rows of G[m][t].
// X is M x E codes and by far the largest operand, T (channels) is small: what bounds the kernel is
// reading the codes once.  A wavefront therefore keeps a 32 x 256 (32 x 128, 64 x 128) piece of dW in its
// accumulators and walks down the rows, 16 at a time, with v_mfma_f32_32x32x16_bf16.
//   - The sum runs over rows, so the matrix operands want 8 consecutive ROWS of one column per lane
//     while memory holds rows.  Which column of dW a matrix column stands for is free: lane c takes
//     columns 4c..4c+3, one word of codes per row, and byte j of its 8 words (one per row) is its
//     operand of the j-th of four products.  No transpose through LDS, no exchange between lanes, and
//     the results of the four products are 4 neighbouring numbers of dW.
//   - A code times its power of two is exact in bfloat16 (at most 8 significant bits); blocks whose
//     scale byte is 0 (magnitudes below 2^-120) count as zero.  A float gradient is cut into three
//     bfloat16 pieces (8 + 8 + 8 bits, exact), a half one into two, so that the products are exact and
//     only their sum, in float, rounds.
//   - Rows that are not live (past natoms[b], or past the end) are zeroed in both operands by a mask of
//     the 16 rows, so that whatever they hold counts for nothing.
//   - The rows are split over workgroups and the four wavefronts of each; partial sums are added in a
//     fixed order (LDS, then a second kernel over the workgroups' sums), so the same call gives the same
//     bits every time.
#include "mg_common.h"
#include "mg_mx.h"
#include "mg_mx_ops.h"

namespace mg {

namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kRows = 16;               // rows of one step
constexpr int kChanTile = 32;           // rows of dW per matrix product

using v4u = __attribute__((ext_vector_type(4))) uint32_t;
using v8bf = __attribute__((ext_vector_type(8))) __bf16;
using v16f = __attribute__((ext_vector_type(16))) float;

template <Num T> constexpr int kPieces = T == Num::F32 ? 3 : T == Num::F16 ? 2 : 1;

struct GradientArgs {
    const void *grad;
    uint32_t grad_stride;               // elements
    const uint8_t *codes, *scales;
    uint32_t code_pitch, scale_pitch;
    const int32_t *natoms;              // null: every row is live
    uint32_t M, N;                      // rows, rows per example
    uint32_t div_mul, div_shift;        // m / N = (umulhi(m, mul) + m) >> shift for m < 2^31
    int T, E;
    uint32_t steps, steps_per_split;
    float *partial;                     // [splits][T][code_pitch], then [splits][T] for db
    float *weight, *bias;               // written directly when there is one split
    int splits;
};

// upper halves of two floats as a pair of bfloat16 (b in the low half)
__device__ inline uint32_t pair_hi(float a, float b)
{
    return __builtin_amdgcn_perm(mx_word(a), mx_word(b), 0x07060302u);
}

// What a lane holds of a step: 8 rows of 4 Words columns, of their scales, and of CT channels.
template <int CT, int Words>
struct Step {
    uint32_t code[8][Words], scale[8];
    float g[CT][8];
    uint32_t live;
};

// CT tiles of 32 channels by 128 Words columns per wavefront.
template <Num T, Mx F, int CT, int Words>
__global__ __launch_bounds__(kThreads, 2) void gradient_kernel(GradientArgs a)
{
    using E = typename NumTraits<T>::type;
    constexpr int kCols = 128 * Words;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 31, h = lane >> 5;
    const int etile = blockIdx.x, ttile = blockIdx.y, split = blockIdx.z;

    // columns and channels past the end read the last valid ones and are not stored
    const uint32_t col = min((uint32_t)(etile * kCols + 4 * Words * c), a.code_pitch - 4 * Words);
    const uint32_t block = col / kMxBlock, shift = 8 * (block & 3);
    uint32_t code_at[8], grad_at[8], chan[CT];
    const uint32_t scale_at = 8 * h * a.scale_pitch + (block & ~3u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        code_at[i] = (8 * h + i) * a.code_pitch + col;
        grad_at[i] = (8 * h + i) * a.grad_stride;
    }
#pragma unroll
    for (int q = 0; q < CT; ++q) chan[q] = (uint32_t)min((ttile * CT + q) * kChanTile + c, a.T - 1);

    const uint32_t s0 = (uint32_t)split * a.steps_per_split;
    const uint32_t s1 = min(s0 + a.steps_per_split, a.steps);

    // the live rows of a step, one bit each
    auto mask = [&](uint32_t step) -> uint32_t {
        if (step >= s1) return 0u;
        const uint32_t m0 = step * kRows;
        if (!a.natoms) return a.M - m0 >= kRows ? 0xffffu : (1u << (a.M - m0)) - 1u;
        const uint32_t m = m0 + (lane & 15), mc = min(m, a.M - 1);
        const uint32_t b = (__umulhi(mc, a.div_mul) + mc) >> a.div_shift;
        return (uint32_t)__ballot(m < a.M && (int)(mc - b * a.N) < a.natoms[b]) & 0xffffu;
    };
    auto load = [&](uint32_t step, uint32_t live, Step<CT, Words> &r) {
        r.live = live;
        if (live == 0) return;
        const uint32_t m0 = step * kRows;
        const uint8_t *cb = a.codes + (int64_t)m0 * a.code_pitch;
        const uint8_t *sb = a.scales + (int64_t)m0 * a.scale_pitch;
        const E *gb = (const E *)a.grad + (int64_t)m0 * a.grad_stride;
        auto get = [&](int i, uint32_t ca, uint32_t sa, uint32_t ga) {
            __builtin_memcpy(r.code[i], __builtin_assume_aligned(cb + ca, 4 * Words), 4 * Words);
            r.scale[i] = *(const uint32_t *)(sb + sa);
#pragma unroll
            for (int q = 0; q < CT; ++q) r.g[q][i] = (float)gb[ga + chan[q]];
        };
        if (a.M - m0 >= kRows) {
#pragma unroll
            for (int i = 0; i < 8; ++i) get(i, code_at[i], scale_at + i * a.scale_pitch, grad_at[i]);
        } else {                            // the last step: rows past the end read the last row
            const uint32_t last = a.M - 1 - m0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t over = max((uint32_t)(8 * h + i), last) - last;
                get(i, code_at[i] - over * a.code_pitch, scale_at + i * a.scale_pitch - over * a.scale_pitch,
                    grad_at[i] - over * a.grad_stride);
            }
        }
    };

    v16f acc[CT][Words][4];
#pragma unroll
    for (int q = 0; q < CT; ++q)
#pragma unroll
        for (int w = 0; w < Words; ++w)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[q][w][j][i] = 0.0f;
    float bias[CT];
#pragma unroll
    for (int q = 0; q < CT; ++q) bias[q] = 0.0f;

    auto compute = [&](Step<CT, Words> &r) {
        if (r.live == 0) return;
        if (r.live != 0xffffu) {
            const uint32_t mine = r.live >> (8 * h);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool on = (mine >> i) & 1u;
                r.scale[i] = on ? r.scale[i] : 0u;          // times code 0: e4m3 codes can be NaN
#pragma unroll
                for (int w = 0; w < Words; ++w) r.code[i][w] = on ? r.code[i][w] : 0u;
#pragma unroll
                for (int q = 0; q < CT; ++q) r.g[q][i] = on ? r.g[q][i] : 0.0f;
            }
        }
        v8bf gp[CT][kPieces<T>];
#pragma unroll
        for (int q = 0; q < CT; ++q) {
            float rest[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                rest[i] = r.g[q][i];
                bias[q] += rest[i];
            }
#pragma unroll
            for (int p = 0; p < kPieces<T>; ++p) {
                const v4u w = {pair_hi(rest[1], rest[0]), pair_hi(rest[3], rest[2]), pair_hi(rest[5], rest[4]),
                               pair_hi(rest[7], rest[6])};
                gp[q][p] = __builtin_bit_cast(v8bf, w);
                if (p + 1 < kPieces<T>) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) rest[i] -= mx_bits(mx_word(rest[i]) & 0xffff0000u);
                }
            }
        }
        float s[8], off[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[i] = mx_bits(((r.scale[i] >> shift) & 255u) << 23);       // S = 255: infinity, times code 0
            off[i] = -128.0f * s[i];
        }
#pragma unroll
        for (int w = 0; w < Words; ++w) {
            // this lane's 8 rows of 4 columns, as 4 operands
            float x[4][8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (F == Mx::INT8) {
                    // bytes as q + 128, which one conversion takes; (q + 128) s - 128 s = q s is exact
                    const uint32_t u = r.code[i][w] ^ 0x80808080u;
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j][i] = fmaf((float)((u >> (8 * j)) & 255u), s[i], off[i]);
                } else {
                    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.code[i][w], false);
                    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.code[i][w], true);
                    x[0][i] = lo[0] * s[i];
                    x[1][i] = lo[1] * s[i];
                    x[2][i] = hi[0] * s[i];
                    x[3][i] = hi[1] * s[i];
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const v4u v = {pair_hi(x[j][1], x[j][0]), pair_hi(x[j][3], x[j][2]), pair_hi(x[j][5], x[j][4]),
                               pair_hi(x[j][7], x[j][6])};
                const v8bf xb = __builtin_bit_cast(v8bf, v);
#pragma unroll
                for (int q = 0; q < CT; ++q)
#pragma unroll
                    for (int p = 0; p < kPieces<T>; ++p)
                        acc[q][w][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(gp[q][p], xb, acc[q][w][j], 0, 0, 0);
            }
        }
    };

    {
        uint32_t step = s0 + wave;
        uint32_t live = mask(step), ahead = mask(step + kWaves);
        Step<CT, Words> now, next;
        load(step, live, now);
        for (; step < s1; step += kWaves) {
            load(step + kWaves, ahead, next);
            ahead = mask(step + 2 * kWaves);
            compute(now);
            now = next;
        }
    }

    // The wavefronts' sums, one tile of 32 channels by 128 columns at a time, through LDS as [wavefront]
    // [accumulator row][lane] of 4 columns: the upper four hand theirs to the lower four, those lay out
    // theirs, and every wavefront adds up and stores two accumulator rows.
    __shared__ float4 sums[kWaves / 2][16][64];
    __shared__ float bsum[kWaves][32];
    const int64_t weights = (int64_t)a.T * a.code_pitch;
#pragma unroll
    for (int q = 0; q < CT; ++q) {
        const int t0 = (ttile * CT + q) * kChanTile;
        const float b = bias[q] + __shfl_xor(bias[q], 32);
        if (q) __syncthreads();
        if (h == 0) bsum[wave][c] = b;
#pragma unroll
        for (int w = 0; w < Words; ++w) {
            if (w) __syncthreads();
            if (wave >= kWaves / 2) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    sums[wave - kWaves / 2][i][lane] =
                        make_float4(acc[q][w][0][i], acc[q][w][1][i], acc[q][w][2][i], acc[q][w][3][i]);
            }
            __syncthreads();
            if (wave < kWaves / 2) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float4 o = sums[wave][i][lane];
                    sums[wave][i][lane] = make_float4(acc[q][w][0][i] + o.x, acc[q][w][1][i] + o.y,
                                                      acc[q][w][2][i] + o.z, acc[q][w][3][i] + o.w);
                }
            }
            __syncthreads();
            if (w == 0 && etile == 0 && threadIdx.x < 32 && t0 + (int)threadIdx.x < a.T) {
                const int t = t0 + threadIdx.x;
                float v = 0.0f;
#pragma unroll
                for (int k = 0; k < kWaves; ++k) v += bsum[k][threadIdx.x];
                if (a.splits > 1) a.partial[(int64_t)a.splits * weights + (int64_t)split * a.T + t] = v;
                else if (a.bias) a.bias[t] = v;
            }
#pragma unroll
            for (int k = 0; k < 16 / kWaves; ++k) {
                const int i = 16 / kWaves * wave + k;
                const int t = t0 + 8 * (i >> 2) + 4 * h + (i & 3);
                const int e = etile * kCols + 4 * Words * c + 4 * w;
                float4 v = sums[0][i][lane];
#pragma unroll
                for (int o = 1; o < kWaves / 2; ++o) {
                    const float4 x = sums[o][i][lane];
                    v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
                }
                if (t >= a.T || e >= a.E) continue;
                if (a.splits == 1) {
                    float *to = a.weight + (int64_t)t * a.E + e;
                    to[0] = v.x;
                    if (e + 1 < a.E) to[1] = v.y;
                    if (e + 2 < a.E) to[2] = v.z;
                    if (e + 3 < a.E) to[3] = v.w;
                } else {
                    *(float4 *)(a.partial + (int64_t)split * weights + (int64_t)t * a.code_pitch + e) = v;
                }
            }
        }
    }
}

// Adds the splits' sums: 32 lanes hold 128 neighbouring numbers of one channel's row, 32 groups of lanes
// take every 32nd split.  One more workgroup per channel adds up db[t].
constexpr int kSumThreads = 1024, kSumGroups = kSumThreads / 32;

__global__ __launch_bounds__(kSumThreads) void gradient_sum_kernel(GradientArgs a)
{
    __shared__ float4 part[kSumGroups][32];
    const int64_t weights = (int64_t)a.T * a.code_pitch;
    const int t = blockIdx.y;
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const bool is_bias = blockIdx.x == gridDim.x - 1;
    const int e = blockIdx.x * 128 + 4 * x;
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (is_bias) {
        const float *from = a.partial + (int64_t)a.splits * weights + t;
        for (int s = threadIdx.x; s < a.splits; s += kSumThreads) v.x += from[(int64_t)s * a.T];
#pragma unroll
        for (int n = 16; n >= 1; n >>= 1) v.x += __shfl_xor(v.x, n);     // the same sum in all 32 lanes
    } else if (e < a.E) {
        const float *from = a.partial + (int64_t)t * a.code_pitch + e;
#pragma unroll 4
        for (int s = y; s < a.splits; s += kSumGroups) {
            const float4 o = *(const float4 *)(from + (int64_t)s * weights);
            v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        }
    }
    part[y][x] = v;
#pragma unroll
    for (int n = kSumGroups / 2; n >= 1; n >>= 1) {
        __syncthreads();
        if (y < n) {
            const float4 o = part[y + n][x];
            v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
            part[y][x] = v;
        }
    }
    if (y != 0) return;
    if (is_bias) {
        if (x == 0 && a.bias) a.bias[t] = v.x;
        return;
    }
    float *to = a.weight + (int64_t)t * a.E + e;
    if (e < a.E) to[0] = v.x;
    if (e + 1 < a.E) to[1] = v.y;
    if (e + 2 < a.E) to[2] = v.z;
    if (e + 3 < a.E) to[3] = v.w;
}

// Two tiles of channels share a pass over the codes where there are that many channels; else a wavefront
// takes 256 columns, so that it meets the gradients half as often.
int channel_tiles(int64_t T) { return T > kChanTile ? 2 : 1; }
int column_words(int64_t T, int64_t pitch) { return T <= kChanTile && pitch > 128 ? 2 : 1; }

int64_t gradient_tiles(int64_t T, int64_t pitch)
{
    const int64_t cols = 128 * column_words(T, pitch), chans = kChanTile * channel_tiles(T);
    return ((pitch + cols - 1) / cols) * ((T + chans - 1) / chans);
}

// Enough workgroups to fill the chip, but at least kLeastSteps steps of 16 rows per wavefront, as every split
// costs a write and a read of T x E sums.
constexpr int kWantGroups = 256, kLeastSteps = 2;
int gradient_splits(int64_t M, int64_t T, int64_t E)
{
    const int64_t steps = (M + kRows - 1) / kRows;
    const int64_t tiles = gradient_tiles(T, mx_blocks(E) * kMxBlock);
    const int64_t want = (kWantGroups + tiles - 1) / tiles;
    const int64_t most = (steps + kLeastSteps * kWaves - 1) / (kLeastSteps * kWaves);
    return (int)std::max<int64_t>(1, std::min(want, most));
}

template <Num T, Mx F, int CT, int Words>
hipError_t gradient_run(const GradientArgs &a, hipStream_t stream)
{
    const dim3 grid((a.code_pitch + 128 * Words - 1) / (128 * Words), (a.T + kChanTile * CT - 1) / (kChanTile * CT),
                    a.splits);
    hipLaunchKernelGGL((gradient_kernel<T, F, CT, Words>), grid, dim3(kThreads), 0, stream, a);
    if (a.splits > 1) {
        const dim3 sum((a.code_pitch + 127) / 128 + 1, a.T);
        hipLaunchKernelGGL(gradient_sum_kernel, sum, dim3(kSumThreads), 0, stream, a);
    }
    return hipGetLastError();
}

template <Num T, Mx F>
hipError_t gradient_typed(const GradientArgs &a, hipStream_t stream)
{
    if (channel_tiles(a.T) == 2) return gradient_run<T, F, 2, 1>(a, stream);
    if (column_words(a.T, a.code_pitch) == 2) return gradient_run<T, F, 1, 2>(a, stream);
    return gradient_run<T, F, 1, 1>(a, stream);
}

}  // namespace

size_t mx_gradient_workspace(int64_t M, int64_t T, int64_t E)
{
    const int splits = gradient_splits(M, T, E);
    return splits == 1 ? 0 : (size_t)splits * T * (mx_blocks(E) * kMxBlock + 1) * sizeof(float);
}

hipError_t launch_mx_gradient(Mx f, Num t, int B, int N, int T, int E, const void *grad, int64_t grad_stride,
                              const uint8_t *codes, const uint8_t *scales, const int32_t *natoms, float *weight,
                              float *bias, void *workspace, hipStream_t stream)
{
    GradientArgs a = {};
    a.grad = grad; a.grad_stride = (uint32_t)grad_stride; a.codes = codes; a.scales = scales;
    a.code_pitch = (uint32_t)mx_code_pitch(f, E); a.scale_pitch = (uint32_t)mx_scale_pitch(E);
    a.natoms = natoms; a.M = (uint32_t)((int64_t)B * N); a.N = (uint32_t)N; a.T = T; a.E = E;
    while ((1ull << a.div_shift) < a.N) ++a.div_shift;
    a.div_mul = (uint32_t)(((1ull << 32) * ((1ull << a.div_shift) - a.N)) / a.N + 1);
    a.splits = gradient_splits(a.M, T, E);
    a.steps = (a.M + kRows - 1) / kRows;
    a.steps_per_split = (a.steps + a.splits - 1) / a.splits;
    a.partial = (float *)workspace; a.weight = weight; a.bias = bias;
#define MG_CASE(TT, FF) if (t == Num::TT && f == Mx::FF) return gradient_typed<Num::TT, Mx::FF>(a, stream)
    MG_CASE(F32, INT8); MG_CASE(F16, INT8); MG_CASE(BF16, INT8);
    MG_CASE(F32, E4M3); MG_CASE(F16, E4M3); MG_CASE(BF16, E4M3);
#undef MG_CASE
    return hipErrorInvalidValue;
}

}  // namespace mg
