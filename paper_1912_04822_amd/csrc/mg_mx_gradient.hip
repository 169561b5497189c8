// Weight gradient of a linear map from the 8-bit codes of its input (formats: mg_mx.h):
//     dW[t][e] = sum over live rows m of G[m][t] X[m][e],     db[t] = sum over live rows of G[m][t].
// X is M x E codes and by far the largest operand, T (channels) is small: what bounds the kernel is
// reading the codes once.  A wavefront therefore keeps a 32 x 128 piece of dW in its accumulators and
// walks down the rows, 16 at a time, with v_mfma_f32_32x32x16_bf16.
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

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kRows = 16;               // rows of one step
constexpr int kColTile = 128;           // columns of dW per wavefront
constexpr int kChanTile = 32;           // rows of dW per matrix product

using v4u = __attribute__((ext_vector_type(4))) uint32_t;
using v8bf = __attribute__((ext_vector_type(8))) __bf16;
using v16f = __attribute__((ext_vector_type(16))) float;

template <Num T> constexpr int kPieces = T == Num::F32 ? 3 : T == Num::F16 ? 2 : 1;

struct GradientArgs {
    const void *grad;
    int64_t grad_stride;                // elements
    const uint8_t *codes, *scales;
    uint32_t code_pitch, scale_pitch;
    const int32_t *natoms;              // null: every row is live
    uint32_t M, N;                      // rows, rows per example
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

template <Num T, Mx F, int CT>
struct Step {
    uint32_t code[8], scale[8];
    float g[CT][8];
    uint32_t live;
};

template <Num T, Mx F, int CT>
__global__ __launch_bounds__(kThreads) void gradient_kernel(GradientArgs a)
{
    using E = typename NumTraits<T>::type;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 31, h = lane >> 5;
    const int etile = blockIdx.x, ttile = blockIdx.y, split = blockIdx.z;

    // columns and channels past the end read the last valid ones and are not stored
    const uint32_t col = min((uint32_t)(etile * kColTile + 4 * c), a.code_pitch - 4);
    const uint32_t swd = min((uint32_t)etile * 4, a.scale_pitch - 4);
    const int shift = 8 * (int)((col / kMxBlock) & 3);
    uint32_t chan[CT];
#pragma unroll
    for (int q = 0; q < CT; ++q) chan[q] = (uint32_t)min((ttile * CT + q) * kChanTile + c, a.T - 1);

    const uint32_t s0 = (uint32_t)split * a.steps_per_split;
    const uint32_t s1 = min(s0 + a.steps_per_split, a.steps);

    auto load = [&](uint32_t step, Step<T, F, CT> &r) {
        const uint32_t m0 = step * kRows;
        uint32_t live;
        if (a.natoms) {
            const uint32_t m = m0 + (lane & 15);
            const uint32_t mc = min(m, a.M - 1);
            const uint32_t b = mc / a.N;
            live = (uint32_t)__ballot(m < a.M && (int)(mc - b * a.N) < a.natoms[b]) & 0xffffu;
        } else {
            live = a.M - m0 >= kRows ? 0xffffu : (1u << (a.M - m0)) - 1u;
        }
        r.live = live;
        if (live == 0) return;
        const uint8_t *cb = a.codes + (int64_t)m0 * a.code_pitch;
        const uint8_t *sb = a.scales + (int64_t)m0 * a.scale_pitch;
        const E *gb = (const E *)a.grad + (int64_t)m0 * a.grad_stride;
        const uint32_t last = min(a.M - 1 - m0, (uint32_t)kRows - 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t row = min((uint32_t)(8 * h + i), last);
            r.code[i] = *(const uint32_t *)(cb + row * a.code_pitch + col);
            r.scale[i] = *(const uint32_t *)(sb + row * a.scale_pitch + swd);
#pragma unroll
            for (int q = 0; q < CT; ++q) r.g[q][i] = (float)gb[row * a.grad_stride + chan[q]];
        }
    };

    v16f acc[CT][4];
#pragma unroll
    for (int q = 0; q < CT; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[q][j][i] = 0.0f;
    float bias[CT];
#pragma unroll
    for (int q = 0; q < CT; ++q) bias[q] = 0.0f;

    auto compute = [&](Step<T, F, CT> &r) {
        if (r.live == 0) return;
        if (r.live != 0xffffu) {
            const uint32_t mine = r.live >> (8 * h);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool on = (mine >> i) & 1u;
                r.code[i] = on ? r.code[i] : 0u;
                r.scale[i] = on ? r.scale[i] : 0u;
#pragma unroll
                for (int q = 0; q < CT; ++q) r.g[q][i] = on ? r.g[q][i] : 0.0f;
            }
        }
        // this lane's 8 rows of 4 columns, as 4 operands
        float x[4][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = mx_bits(((r.scale[i] >> shift) & 255u) << 23);      // S = 255: infinity, times code 0
            if constexpr (F == Mx::INT8) {
                // bytes as q + 128, which one conversion takes; (q + 128) s - 128 s = q s is exact
                const uint32_t u = r.code[i] ^ 0x80808080u;
                const float off = -128.0f * s;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j][i] = fmaf((float)((u >> (8 * j)) & 255u), s, off);
            } else {
                const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.code[i], false);
                const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.code[i], true);
                x[0][i] = lo[0] * s;
                x[1][i] = lo[1] * s;
                x[2][i] = hi[0] * s;
                x[3][i] = hi[1] * s;
            }
        }
        v8bf xb[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const v4u w = {pair_hi(x[j][1], x[j][0]), pair_hi(x[j][3], x[j][2]), pair_hi(x[j][5], x[j][4]),
                           pair_hi(x[j][7], x[j][6])};
            xb[j] = __builtin_bit_cast(v8bf, w);
        }
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
                const v8bf gb = __builtin_bit_cast(v8bf, w);
                if (p + 1 < kPieces<T>) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) rest[i] -= mx_bits(mx_word(rest[i]) & 0xffff0000u);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[q][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(gb, xb[j], acc[q][j], 0, 0, 0);
            }
        }
    };

    uint32_t step = s0 + wave;
    if (step < s1) {
        Step<T, F, CT> now, next;
        load(step, now);
        for (; step < s1; step += kWaves) {
            const bool more = step + kWaves < s1;
            if (more) load(step + kWaves, next);
            compute(now);
            if (more) now = next;
        }
    }

    // the four wavefronts' sums: [wave][16 accumulator rows][64 lanes] of 4 columns, one channel tile at
    // a time; wavefront w adds up and stores accumulator rows 4w..4w+3
    __shared__ float4 sums[kWaves][16][64];
    __shared__ float bsum[kWaves][32];
    const int64_t weights = (int64_t)a.T * a.code_pitch;
#pragma unroll
    for (int q = 0; q < CT; ++q) {
        if (q) __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i)
            sums[wave][i][lane] = make_float4(acc[q][0][i], acc[q][1][i], acc[q][2][i], acc[q][3][i]);
        if (etile == 0) {
            const float b = bias[q] + __shfl_xor(bias[q], 32);
            if (h == 0) bsum[wave][c] = b;
        }
        __syncthreads();
        const int t0 = (ttile * CT + q) * kChanTile;
        if (etile == 0 && threadIdx.x < 32 && t0 + (int)threadIdx.x < a.T) {
            const int t = t0 + threadIdx.x;
            const float b = (bsum[0][threadIdx.x] + bsum[1][threadIdx.x]) + (bsum[2][threadIdx.x] + bsum[3][threadIdx.x]);
            if (a.splits == 1) {
                if (a.bias) a.bias[t] = b;
            } else {
                a.partial[(int64_t)a.splits * weights + (int64_t)split * a.T + t] = b;
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = 4 * wave + k;
            const int t = t0 + 8 * (i >> 2) + 4 * h + (i & 3);
            const int e = etile * kColTile + 4 * c;
            float4 v = sums[0][i][lane];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) {
                const float4 o = sums[w][i][lane];
                v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
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

// Adds the splits' sums: 32 lanes hold 128 neighbouring numbers of one channel's row, 8 groups of lanes
// take every eighth split.  One more workgroup per channel adds up db[t] (every 256th split a lane).
__global__ __launch_bounds__(256) void gradient_sum_kernel(GradientArgs a)
{
    const int64_t weights = (int64_t)a.T * a.code_pitch;
    const int t = blockIdx.y;
    if (blockIdx.x == gridDim.x - 1) {
        __shared__ float total[256];
        const float *from = a.partial + (int64_t)a.splits * weights + t;
        float v = 0.0f;
        for (int s = threadIdx.x; s < a.splits; s += 256) v += from[(int64_t)s * a.T];
        total[threadIdx.x] = v;
        __syncthreads();
#pragma unroll
        for (int n = 128; n >= 1; n >>= 1) {
            if ((int)threadIdx.x < n) total[threadIdx.x] += total[threadIdx.x + n];
            __syncthreads();
        }
        if (threadIdx.x == 0 && a.bias) a.bias[t] = total[0];
        return;
    }
    __shared__ float4 part[8][32];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int e = blockIdx.x * 128 + 4 * x;
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (e < (int)a.code_pitch) {
        const float *from = a.partial + (int64_t)t * a.code_pitch + e;
#pragma unroll 4
        for (int s = y; s < a.splits; s += 8) {
            const float4 o = *(const float4 *)(from + (int64_t)s * weights);
            v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        }
    }
    part[y][x] = v;
    __syncthreads();
    if (y == 0) {
#pragma unroll
        for (int k = 1; k < 8; ++k) {
            const float4 o = part[k][x];
            v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        }
        float *to = a.weight + (int64_t)t * a.E + e;
        if (e < a.E) to[0] = v.x;
        if (e + 1 < a.E) to[1] = v.y;
        if (e + 2 < a.E) to[2] = v.z;
        if (e + 3 < a.E) to[3] = v.w;
    }
}

// Enough workgroups to fill the chip (256 compute units, two to three of 4 wavefronts each), but at
// least 4 steps of 16 rows per wavefront, as every split costs a write and a read of T x E sums.
int gradient_splits(int64_t M, int64_t T, int64_t E)
{
    const int64_t steps = (M + kRows - 1) / kRows;
    const int64_t tiles = ((mx_blocks(E) * kMxBlock + kColTile - 1) / kColTile) * ((T + kChanTile - 1) / kChanTile);
    const int64_t want = (768 + tiles - 1) / tiles, most = (steps + 4 * kWaves - 1) / (4 * kWaves);
    return (int)std::max<int64_t>(1, std::min(want, most));
}

template <Num T, Mx F>
hipError_t gradient_typed(GradientArgs a, hipStream_t stream)
{
    const dim3 grid((a.code_pitch + kColTile - 1) / kColTile, (a.T + kChanTile - 1) / kChanTile, a.splits);
    hipLaunchKernelGGL((gradient_kernel<T, F, 1>), grid, dim3(kThreads), 0, stream, a);
    if (a.splits > 1) {
        const dim3 sum((a.code_pitch + 127) / 128 + 1, a.T);
        hipLaunchKernelGGL(gradient_sum_kernel, sum, dim3(256), 0, stream, a);
    }
    return hipGetLastError();
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
    a.grad = grad; a.grad_stride = grad_stride; a.codes = codes; a.scales = scales;
    a.code_pitch = (uint32_t)mx_code_pitch(f, E); a.scale_pitch = (uint32_t)mx_scale_pitch(E);
    a.natoms = natoms; a.M = (uint32_t)((int64_t)B * N); a.N = (uint32_t)N; a.T = T; a.E = E;
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
