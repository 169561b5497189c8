// Weight gradient of a linear map from the 8-bit codes of its input (formats: mg_mx.h):
//     dW[t][e] = sum over live rows m of G[m][t] X[m][e],     db[t] = sum over live rows of G[m][t].
// X is M x E codes and by far the largest operand, T (channels) is small: the kernel is bound by reading the
// codes once and by taking them apart.  A wavefront keeps a piece of dW, 32 channels by 128 columns (up to 16
// channels: 16 by 256), in its accumulators and walks down the rows, 32 at a time, with
// v_mfma_f32_16x16x32_bf16.
//   - The sum runs over rows, so the matrix operands want 8 consecutive ROWS of one column per lane
//     while memory holds rows.  Which column of dW a matrix column stands for is free: lane c takes
//     columns 8c..8c+7 (16c..), 8 (16) bytes of codes a row, and byte j of its 8 rows is its operand of the
//     j-th of 8 (16) products.  No transpose through LDS, and the results of the products are neighbouring
//     numbers of dW.  Channels likewise: a lane loads 2 neighbours of a row for 2 operands.
//   - A wavefront can have 63 loads under way: loads are as wide as can be, 17 a step, and the scales come in
//     one word per lane and go to the lanes that need them by an exchange.  (24 loads per 16 rows: 19.5 and 39
//     us below.)
//   - A code times its power of two is exact in bfloat16 (at most 8 significant bits); int8 blocks whose
//     scale byte is 0 (magnitudes below 2^-120) count as zero.  A float gradient is cut into three
//     bfloat16 pieces (8 + 8 + 8 bits, exact), a half one into two, so that the products are exact and
//     only their sum, in float, rounds.  bfloat16 ends at 2^-133: what of a number lies below it is lost.
//   - Rows that are not live (past natoms[b], or past the end) are zeroed in both operands by a mask of
//     the 32 rows, so that whatever they hold counts for nothing.
//   - The rows are split over workgroups and the eight wavefronts of each; partial sums are added in a
//     fixed order (LDS, then a second kernel over the workgroups' sums), so the same call gives the same
//     bits every time.
// Measured (both kernels, back to back): 102000 x 256 int8, 28 channels of float 15.3 us (38 MB: 2.5 TB/s; the
// first kernel 14, 3 to 4 steps a wavefront and their vector instructions, 5 a code); 96000 live of 128000 x
// 1000 e4m3, 28 of bfloat16 27 us (110 MB: 4.1 TB/s); 512000 x 256 e4m3 29.5 us (5.6 TB/s).
#include <type_traits>

#include "mg_common.h"
#include "mg_mx.h"
#include "mg_mx_ops.h"

namespace mg {

namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kRows = 32;               // rows of one step
constexpr int kDepth = 2;               // steps a wavefront holds: one it works on, the rest under way

using v8bf = __attribute__((ext_vector_type(8))) __bf16;
using v4f = __attribute__((ext_vector_type(4))) float;

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

// Bytes j and j + 1 (j = 0 or 2) of a word of e4m3 codes, times a scale, as a pair of bfloat16: exact, and NaN
// for the scale of byte 255 (checked for every code and scale).
__device__ inline uint32_t scaled_pair(uint32_t codes, float scale, int j)
{
    return j == 0 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false))
                  : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true));
}

// What a lane holds of a step: 8 rows of 4 Words columns and of Q channels; one word of scales, which its
// wavefront exchanges.
template <Num T, int Q, int Words>
struct Step {
    uint32_t code[8][Words], scale;
    typename NumTraits<T>::type g[8][Q];
    uint32_t live;
};

// 16 Q channels by 64 Words columns per wavefront.
template <Num T, Mx F, int Q, int Words>
__global__ __launch_bounds__(kThreads, 2) void gradient_kernel(GradientArgs a)
{
    using E = typename NumTraits<T>::type;
    constexpr int kCols = 64 * Words;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    // Tiles of the same rows run on the same XCD (workgroup number modulo 8), whose L2 gives them the gradients
    // and scales they share: 33.0 -> 28.0 us with 8 tiles, 17.5 -> 16.6 with 2 (sizes as above).
    const int etiles = gridDim.x, ttiles = gridDim.y, total = etiles * ttiles * gridDim.z;
    const int number = blockIdx.x + etiles * (blockIdx.y + ttiles * blockIdx.z), xcd = number % 8;
    const int id = xcd * (total / 8) + min(xcd, total % 8) + number / 8;
    const int etile = id % etiles, ttile = id / etiles % ttiles, split = id / (etiles * ttiles);

    // Columns past the end read the last valid ones and are not stored.  Lane c of an operand stands for
    // channels first .. first + Q - 1: the last lanes overlap the ones before where Q does not divide T.
    const uint32_t col = min((uint32_t)(etile * kCols + 4 * Words * c), a.code_pitch - 4 * Words);
    const uint32_t block = col / kMxBlock, shift = 8 * (block & 3);
    auto first_channel = [&](int lane16) { return min((ttile * 16 + lane16) * Q, a.T - Q); };
    const uint32_t first = (uint32_t)first_channel(c);
    uint32_t code_at[8], grad_at[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t row = min((uint32_t)(8 * g + i), a.M - 1);
        code_at[i] = row * a.code_pitch + col;
        grad_at[i] = row * a.grad_stride + first;
    }
    // lane l fetches scale word l / 32 of the tile's columns of row l % 32; lane (c, g) needs that of its
    // column in rows 8 g + i
    const uint32_t word0 = etile * kCols / (4 * kMxBlock), word = word0 + (Words == 4 ? lane >> 5 : 0);
    const uint32_t scale_at = min((uint32_t)(lane & 31), a.M - 1) * a.scale_pitch + min(4 * word, a.scale_pitch - 4);
    const int scale_from = 4 * (8 * g + (Words == 4 ? 32 * (int)((block >> 2) - word0) : 0));

    const uint32_t s0 = (uint32_t)split * a.steps_per_split;
    const uint32_t s1 = min(s0 + a.steps_per_split, a.steps);

    // the live rows of a step, one bit each
    auto mask = [&](uint32_t step) -> uint32_t {
        if (step >= s1) return 0u;
        const uint32_t m0 = step * kRows;
        const uint32_t rows = min(a.M - m0, (uint32_t)kRows);
        if (!a.natoms) return 0xffffffffu >> (kRows - rows);
        uint32_t b = (__umulhi(m0, a.div_mul) + m0) >> a.div_shift, from = m0 - b * a.N, live = 0;
        for (uint32_t done = 0; done < rows; ++b, from = 0) {
            const uint32_t run = min(a.N - from, rows - done);      // of example b
            const int left = min(max(max(a.natoms[b], 0) - (int)from, 0), (int)run);
            if (left > 0) live |= (0xffffffffu >> (kRows - left)) << done;
            done += run;
        }
        return live;
    };
    // No branch lies around the loads: the compiler counts those under way, and where their number depends on
    // the path it waits for all of them.  The last step takes the last 32 rows (its mask says which are new),
    // a step without live rows takes the workgroup's first rows again, which are near.
    const uint32_t most = a.M > kRows ? a.M - kRows : 0u;
    auto load = [&](uint32_t step, uint32_t live, Step<T, Q, Words> &r) {
        const uint32_t want = (live ? step : s0) * kRows, m0 = min(want, most);
        r.live = live ? live << (want - m0) : 0u;
        const uint8_t *cb = a.codes + (int64_t)m0 * a.code_pitch;
        const uint8_t *sb = a.scales + (int64_t)m0 * a.scale_pitch;
        const E *gb = (const E *)a.grad + (int64_t)m0 * a.grad_stride;
        r.scale = *(const uint32_t *)(sb + scale_at);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            __builtin_memcpy(r.code[i], __builtin_assume_aligned(cb + code_at[i], 4 * Words), 4 * Words);
            __builtin_memcpy(r.g[i], gb + grad_at[i], sizeof r.g[i]);
        }
    };

    v4f acc[Q][Words][4];
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int w = 0; w < Words; ++w)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[q][w][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    float bias[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) bias[q] = 0.0f;

    auto compute = [&](Step<T, Q, Words> &r, auto careful) {
        if (r.live == 0) return;
        float s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t w = (uint32_t)__builtin_amdgcn_ds_bpermute(scale_from + 4 * i, (int)r.scale);
            s[i] = mx_bits(((w >> shift) & 255u) << 23);
            if (F == Mx::INT8) s[i] = fmaf(s[i], 0.0f, s[i]);   // S = 255: infinity made NaN (e4m3: read as a scale)
        }
        if (r.live != 0xffffffffu) {
            const uint32_t mine = r.live >> (8 * g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool on = (mine >> i) & 1u;
                s[i] = on ? s[i] : 0.0f;                        // times code 0: e4m3 codes can be NaN
#pragma unroll
                for (int w = 0; w < Words; ++w) r.code[i][w] = on ? r.code[i][w] : 0u;
#pragma unroll
                for (int q = 0; q < Q; ++q) r.g[i][q] = on ? r.g[i][q] : (E)0.0f;
            }
        }
        v8bf gp[Q][kPieces<T>];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            float rest[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                rest[i] = (float)r.g[i][q];
                if (etile == 0) bias[q] += rest[i];
            }
#pragma unroll
            for (int p = 0; p < kPieces<T>; ++p) {
                const v4u w = {pair_hi(rest[1], rest[0]), pair_hi(rest[3], rest[2]), pair_hi(rest[5], rest[4]),
                               pair_hi(rest[7], rest[6])};
                gp[q][p] = __builtin_bit_cast(v8bf, w);
                if (p + 1 < kPieces<T>) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float more = rest[i] - mx_bits(mx_word(rest[i]) & 0xffff0000u);
                        rest[i] = careful && __builtin_isinf(rest[i]) ? 0.0f : more;
                    }
                }
            }
        }
#pragma unroll
        for (int w = 0; w < Words; ++w) {
            // this lane's 8 rows of 4 columns, as 4 operands
            v4u x[4];
            if constexpr (F == Mx::INT8) {
#pragma unroll
                for (int i = 0; i < 8; i += 2)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        x[j][i / 2] = pair_hi((float)(int)(int8_t)(r.code[i + 1][w] >> (8 * j)) * s[i + 1],
                                              (float)(int)(int8_t)(r.code[i][w] >> (8 * j)) * s[i]);
            } else {
                // two columns of a row at a time, then two rows of each
#pragma unroll
                for (int i = 0; i < 8; i += 2)
#pragma unroll
                    for (int j = 0; j < 4; j += 2) {
                        const uint32_t u = scaled_pair(r.code[i][w], s[i], j), v = scaled_pair(r.code[i + 1][w], s[i + 1], j);
                        x[j][i / 2] = __builtin_amdgcn_perm(v, u, 0x05040100u);
                        x[j + 1][i / 2] = __builtin_amdgcn_perm(v, u, 0x07060302u);
                    }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const v8bf xb = __builtin_bit_cast(v8bf, x[j]);
#pragma unroll
                for (int q = 0; q < Q; ++q)
#pragma unroll
                    for (int p = 0; p < kPieces<T>; ++p)
                        acc[q][w][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(gp[q][p], xb, acc[q][w][j], 0, 0, 0);
            }
        }
    };

    Step<T, Q, Words> ring[kDepth];
    uint32_t ahead = mask(s0 + wave);
    {
#pragma unroll
        for (int d = 0; d < kDepth - 1; ++d) {
            const uint32_t step = s0 + wave + d * kWaves, live = ahead;
            ahead = mask(step + kWaves);
            load(step, live, ring[d]);
        }
        for (uint32_t step0 = s0 + wave;; step0 += kDepth * kWaves) {
#pragma unroll
            for (int d = 0; d < kDepth; ++d) {
                const uint32_t step = step0 + d * kWaves, live = ahead;
                if (step >= s1) goto done;
                ahead = mask(step + kDepth * kWaves);
                load(step + (kDepth - 1) * kWaves, live, ring[(d + kDepth - 1) % kDepth]);
                compute(ring[d], std::false_type{});
            }
        }
    }
done:

    // An infinity in a gradient of several pieces leaves NaN in the pieces after its first and makes its channel's
    // sums NaN in every column.  A wavefront that finds one walks its rows once more, and there an infinity is whole
    // in its first piece.  (Looked for in the walk above it costs 15.4 -> 15.7 us at 102000 x 256 x 28 floats and
    // 22.9 -> 23.6 at 32640 x 512 x 100; without either 15.4 and 22.6.)
    if constexpr (kPieces<T> > 1) {
        float any = 0.0f;
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) any = __builtin_elementwise_maximum(any, acc[q][0][0][i]);
        if (__builtin_amdgcn_ballot_w64(__builtin_isnan(any)) != 0) {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                bias[q] = 0.0f;
#pragma unroll
                for (int w = 0; w < Words; ++w)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[q][w][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            }
#pragma unroll 1
            for (uint32_t step = s0 + wave; step < s1; step += kWaves) {
                Step<T, Q, Words> r;
                load(step, mask(step), r);
                compute(r, std::true_type{});
            }
        }
    }

    // The wavefronts' sums, 16 of a lane's channels at a time, through LDS as [wavefront][item][lane] of 4
    // columns, an item being one of a lane's four accumulator rows and one of its words; the wavefronts share
    // the items out, add them up and store them.
    constexpr int kItems = 4 * Words;
    __shared__ float4 sums[kWaves][kItems][64];
    __shared__ float bsum[kWaves][16];
    const int64_t weights = (int64_t)a.T * a.code_pitch;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        if (q) __syncthreads();
        float b = bias[q];
        b += __shfl_xor(b, 16);
        b += __shfl_xor(b, 32);
        if (g == 0) bsum[wave][c] = b;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int w = 0; w < Words; ++w)
                sums[wave][i * Words + w][lane] =
                    make_float4(acc[q][w][0][i], acc[q][w][1][i], acc[q][w][2][i], acc[q][w][3][i]);
        __syncthreads();
        if (etile == 0 && threadIdx.x < 16) {
            const int own = (ttile * 16 + (int)threadIdx.x) * Q, t = first_channel(threadIdx.x) + q;
            if (t >= own && own < a.T) {
                float v = 0.0f;
#pragma unroll
                for (int o = 0; o < kWaves; ++o) v += bsum[o][threadIdx.x];
                if (a.splits > 1) a.partial[(int64_t)a.splits * weights + (int64_t)split * a.T + t] = v;
                else if (a.bias) a.bias[t] = v;
            }
        }
        for (int item = wave; item < kItems; item += kWaves) {
            const int row = 4 * g + item / Words, own = (ttile * 16 + row) * Q, t = first_channel(row) + q;
            const int e = etile * kCols + 4 * Words * c + 4 * (item % Words);
            if (t < own || own >= a.T || e >= a.E) continue;    // a channel is stored by the first lane that has it
            float4 v = sums[0][item][lane];
#pragma unroll
            for (int o = 1; o < kWaves; ++o) {
                const float4 x = sums[o][item][lane];
                v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
            }
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

// Channels a lane takes (of the gradient, in one load) and words of codes: what leaves room for two wavefronts
// per SIMD (241 registers).  32 channels by 256 columns with one wavefront per SIMD: 20.9 us where this takes
// 17.3, 31.7 where it takes 33; 64 by 64: 22.5 against 22.6 at 100 channels, and registers in scratch.
int lane_channels(int64_t T) { return T > 16 ? 2 : 1; }
int lane_words(int64_t T, int64_t pitch) { return T > 16 ? 2 : pitch > 64 ? 4 : 1; }

int64_t gradient_tiles(int64_t T, int64_t pitch)
{
    const int64_t cols = 64 * lane_words(T, pitch), chans = 16 * lane_channels(T);
    return ((pitch + cols - 1) / cols) * ((T + chans - 1) / chans);
}

// A workgroup per compute unit (512: 24.0 instead of 17.4 us, 192: 18.9), but at least a step of 32 rows per
// wavefront (4 steps: 14.2 instead of 9.1 us at 2040 rows), as every split costs a write and a read of T x E
// sums.
constexpr int kWantGroups = 256;
int gradient_splits(int64_t M, int64_t T, int64_t E)
{
    const int64_t steps = (M + kRows - 1) / kRows;
    const int64_t tiles = gradient_tiles(T, mx_blocks(E) * kMxBlock);
    const int64_t want = (kWantGroups + tiles - 1) / tiles, most = (steps + kWaves - 1) / kWaves;
    return (int)std::max<int64_t>(1, std::min(want, most));
}

template <Num T, Mx F, int Q, int Words>
hipError_t gradient_run(const GradientArgs &a, hipStream_t stream)
{
    const dim3 grid((a.code_pitch + 64 * Words - 1) / (64 * Words), (a.T + 16 * Q - 1) / (16 * Q), a.splits);
    hipLaunchKernelGGL((gradient_kernel<T, F, Q, Words>), grid, dim3(kThreads), 0, stream, a);
    if (a.splits > 1) {
        const dim3 sum((a.code_pitch + 127) / 128 + 1, a.T);
        hipLaunchKernelGGL(gradient_sum_kernel, sum, dim3(kSumThreads), 0, stream, a);
    }
    return hipGetLastError();
}

template <Num T, Mx F>
hipError_t gradient_typed(const GradientArgs &a, hipStream_t stream)
{
    const int words = lane_words(a.T, a.code_pitch);
    if (lane_channels(a.T) == 2) return gradient_run<T, F, 2, 2>(a, stream);
    return words == 4 ? gradient_run<T, F, 1, 4>(a, stream) : gradient_run<T, F, 1, 1>(a, stream);
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
