// Products of matrices in 4 bits (e2m1 elements, formats: mg_mx.h):
//     C[m][n] = sum_k A[m][k] B[n][k] + bias[n]
// with v_mfma_scale_f32_16x16x128_f8f6f4.  An operand of that instruction is 32 consecutive k of one row
// per lane (row = lane % 16, group of 32 = lane / 16) with that lane's scale byte: exactly a block of the
// format, so 16 bytes of codes and one byte of scales go from memory to the matrix cores as they lie.
// Products of elements and scales are exact; sums are in float.
//
// The operands are given as (B, A), so a lane's four results are 4 neighbouring n of one row m of C.
#include <type_traits>

#include "mg_common.h"
#include "mg_mx.h"
#include "mg_mx_ops.h"

namespace mg {

namespace {

using v4u = __attribute__((ext_vector_type(4))) uint32_t;
using v8i = __attribute__((ext_vector_type(8))) int;
using v4f = __attribute__((ext_vector_type(4))) float;

constexpr int kE2m1 = 4;                // the instruction's code for the element type

struct ProductArgs {
    const void *a;                      // codes, or plain numbers
    const uint8_t *a_scales;
    int64_t a_stride;                   // plain numbers: elements from row to row
    const uint8_t *b, *b_scales;
    uint32_t pitch, scale_pitch;        // of codes and scales, the same on both sides
    int M, N, K, blocks;                // blocks of 32 in a row
    const float *bias;
    void *c;
    int64_t c_stride;
};

struct Operand {
    v4u code;
    int scale;
};

__device__ inline v4f product(const Operand &b, const Operand &a, v4f c)
{
    const v8i x = {(int)b.code[0], (int)b.code[1], (int)b.code[2], (int)b.code[3], 0, 0, 0, 0};
    const v8i y = {(int)a.code[0], (int)a.code[1], (int)a.code[2], (int)a.code[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, kE2m1, kE2m1, 0, b.scale, 0, a.scale);
}

// Block `blk` of a row of codes; past the row's end zeros at scale 1.
__device__ inline Operand load_block(const uint8_t *codes, const uint8_t *scales, const ProductArgs &p,
                                     uint32_t row, int blk)
{
    Operand o;
    const bool in = blk < p.blocks;
    const int at = in ? blk : 0;
    o.code = *(const v4u *)(codes + (int64_t)row * p.pitch + 16 * at);
    o.scale = scales[(int64_t)row * p.scale_pitch + at];
    if (!in) {
        o.code = v4u{0, 0, 0, 0};
        o.scale = 127;
    }
    return o;
}

template <Num T> __device__ inline void widen16(v4u w, float *f)        // 16 bytes of plain numbers
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (T == Num::F32) {
            f[i] = mx_bits(w[i]);
        } else if constexpr (T == Num::BF16) {
            f[2 * i] = mx_bits(w[i] << 16);
            f[2 * i + 1] = mx_bits(w[i] & 0xffff0000u);
        } else {
            f[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)w[i]);
            f[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i] >> 16));
        }
    }
}

// Block `blk` of a row of plain numbers, taken to e2m1 in this lane.
template <Num T>
__device__ inline Operand quantise_block(const ProductArgs &p, uint32_t row, int blk)
{
    using E = typename NumTraits<T>::type;
    constexpr int P = 16 / NumTraits<T>::bytes;
    float f[kMxBlock];
    const E *x = (const E *)p.a + (int64_t)row * p.a_stride + blk * kMxBlock;
    const int left = p.K - blk * kMxBlock;
    if (left >= kMxBlock) {
#pragma unroll
        for (int i = 0; i < kMxBlock / P; ++i) {
            v4u w;
            __builtin_memcpy(&w, x + i * P, 16);
            widen16<T>(w, f + i * P);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kMxBlock; ++i) f[i] = i < left ? (float)x[i] : 0.0f;
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kMxBlock; ++i) m = max(m, mx_word(f[i]) & 0x7fffffffu);
    const uint32_t s = mx_shared<Mx::E2M1>(m);
    const float inv = mx_inverse(s);
    Operand o;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = s == 255u ? 0.0f : f[8 * k + i] * inv;
        uint32_t w = mx_encode_pair<0>(0u, y[0], y[1]);
        w = mx_encode_pair<1>(w, y[2], y[3]);
        w = mx_encode_pair<2>(w, y[4], y[5]);
        o.code[k] = mx_encode_pair<3>(w, y[6], y[7]);
    }
    o.scale = left > 0 ? (int)s : 127;
    return o;
}

// Four neighbouring results of row m.
template <Num T>
__device__ inline void store_results(const ProductArgs &p, int m, int n, v4f v)
{
    using E = typename NumTraits<T>::type;
    if (m >= p.M || n >= p.N) return;
    E *to = (E *)p.c + (int64_t)m * p.c_stride + n;
    E e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float b = p.bias && n + i < p.N ? p.bias[n + i] : 0.0f;
        e[i] = (E)(v[i] + b);
    }
    if (n + 4 <= p.N) {
        __builtin_memcpy(to, e, sizeof e);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < p.N) to[i] = e[i];
    }
}

// Operands straight from memory.  A wavefront holds RM x RN tiles of 16 x 16; the KW wavefronts of a
// group share a tile and split k between them (their sums meet in LDS), the others lie along m.
template <Num T, bool Plain, int RM, int RN, int Waves, int KW>
__global__ __launch_bounds__(64 * Waves) void product_kernel(ProductArgs p)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int kw = wave % KW, mw = wave / KW;
    const int m0 = (blockIdx.x * (Waves / KW) + mw) * RM * 16, n0 = blockIdx.y * RN * 16;

    v4f acc[RM][RN];
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
        for (int j = 0; j < RN; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    uint32_t arow[RM], brow[RN];
#pragma unroll
    for (int i = 0; i < RM; ++i) arow[i] = min(m0 + 16 * i + r, p.M - 1);
#pragma unroll
    for (int j = 0; j < RN; ++j) brow[j] = min(n0 + 16 * j + r, p.N - 1);

    for (int k = kw * 4; k < p.blocks; k += KW * 4) {
        Operand a[RM], b[RN];
#pragma unroll
        for (int i = 0; i < RM; ++i) {
            if constexpr (Plain) a[i] = quantise_block<T>(p, arow[i], k + g);
            else a[i] = load_block((const uint8_t *)p.a, p.a_scales, p, arow[i], k + g);
        }
#pragma unroll
        for (int j = 0; j < RN; ++j) b[j] = load_block(p.b, p.b_scales, p, brow[j], k + g);
#pragma unroll
        for (int i = 0; i < RM; ++i)
#pragma unroll
            for (int j = 0; j < RN; ++j) acc[i][j] = product(b[j], a[i], acc[i][j]);
    }

    if constexpr (KW > 1) {
        __shared__ v4f sums[Waves][RM * RN][64];
#pragma unroll
        for (int i = 0; i < RM; ++i)
#pragma unroll
            for (int j = 0; j < RN; ++j) sums[wave][i * RN + j][lane] = acc[i][j];
        __syncthreads();
        if (kw != 0) return;
#pragma unroll
        for (int i = 0; i < RM; ++i)
#pragma unroll
            for (int j = 0; j < RN; ++j)
#pragma unroll
                for (int w = 1; w < KW; ++w) acc[i][j] += sums[wave + w][i * RN + j][lane];
    }
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
        for (int j = 0; j < RN; ++j) store_results<T>(p, m0 + 16 * i + r, n0 + 16 * j + 4 * g, acc[i][j]);
}

template <Num T, bool Plain, int RM, int RN, int Waves, int KW>
hipError_t direct(const ProductArgs &p, hipStream_t stream)
{
    const int rows = Waves / KW * RM * 16;
    const dim3 grid((p.M + rows - 1) / rows, (p.N + RN * 16 - 1) / (RN * 16));
    hipLaunchKernelGGL((product_kernel<T, Plain, RM, RN, Waves, KW>), grid, dim3(64 * Waves), 0, stream, p);
    return hipGetLastError();
}

// Large products: a workgroup of 4 wavefronts makes a 256 x 256 tile of C, each wavefront 128 x 128 of it
// (8 x 8 tiles of 16 x 16 in 256 accumulator registers, one wavefront per SIMD).  Codes go through LDS, where
// every byte is read by two wavefronts: per 128 k a wavefront issues 64 products (1024 cycles of its matrix
// core) for 16 operands of 1 KB.
//   - Two buffers of 128 k.  While a step's products run, the next step's operands are read from LDS and the
//     codes of the step after that are on their way from memory to registers; they are written to LDS at the
//     end of the step, before its one barrier.
//   - A row's 64 bytes of a step lie in LDS as four pieces of 16, piece c at place c ^ (row / 4) % 4: the 16
//     rows that a quarter of a wavefront reads at once then cover all banks.
//   - Scales are taken for four steps at a time (16 bytes of a row); three byte permutes turn them into one
//     register that holds a lane's scale of each of the four steps, which the instruction picks by its
//     operand selector.
// Codes past the end of k are zeros with scale 0 (a power of two), rows past M or N repeat the last one and
// are not stored.
constexpr int kTile = 256;

__device__ inline uint32_t tile_place(uint32_t row, uint32_t piece) { return row * 4 + (piece ^ ((row >> 2) & 3)); }

template <int Step> __device__ inline v4f product_step(v4u b, v4u a, v4f c, int sb, int sa)
{
    const v8i x = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    const v8i y = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, kE2m1, kE2m1, Step, sb, Step, sa);
}

// Byte g of each of four words.
__device__ inline int scale_bytes(v4u w, uint32_t pick)
{
    const uint32_t lo = __builtin_amdgcn_perm(w[1], w[0], pick), hi = __builtin_amdgcn_perm(w[3], w[2], pick);
    return (int)__builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

struct TileStage {
    v4u a[4], b[4];
};

template <Num T>
__global__ __launch_bounds__(256, 1) void product_tile_kernel(ProductArgs p, int mtiles, int ntiles)
{
    __shared__ v4u lds_a[2][kTile * 4], lds_b[2][kTile * 4], lds_sa[kTile], lds_sb[kTile];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int wm = wave >> 1, wn = wave & 1;

    // tiles in runs of 8 along m, and every XCD (workgroup number modulo 8) on a run of its own
    const int total = mtiles * ntiles;
    int id = blockIdx.x;
    {
        const int per = total / 8, extra = total % 8, xcd = id % 8;
        id = xcd * per + min(xcd, extra) + id / 8;
    }
    const int band = id / (8 * ntiles), rows = min(8, mtiles - band * 8);
    const int in = id - band * 8 * ntiles;
    const int m0 = (band * 8 + in % rows) * kTile, n0 = (in / rows) * kTile;

    const int steps = (p.blocks + 3) / 4;
    const uint8_t *codes_a = (const uint8_t *)p.a;
    uint32_t row_a[4], row_b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = (tid >> 2) + 64 * i;
        row_a[i] = (uint32_t)min(m0 + row, p.M - 1);
        row_b[i] = (uint32_t)min(n0 + row, p.N - 1);
    }
    const int piece = tid & 3;

    auto fetch = [&](int step, TileStage &s) {
        const int blk = step * 4 + piece;
        const bool in_row = blk < p.blocks;
        const int64_t at = in_row ? 16 * blk : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s.a[i] = *(const v4u *)(codes_a + (int64_t)row_a[i] * p.pitch + at);
            s.b[i] = *(const v4u *)(p.b + (int64_t)row_b[i] * p.pitch + at);
        }
        if (!in_row) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s.a[i] = s.b[i] = v4u{0, 0, 0, 0};
        }
    };
    auto put = [&](int buffer, const TileStage &s) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t at = tile_place((tid >> 2) + 64 * i, piece);
            lds_a[buffer][at] = s.a[i];
            lds_b[buffer][at] = s.b[i];
        }
    };
    auto fetch_scales = [&](int step, v4u &sa, v4u &sb) {       // of steps step .. step + 3
        const uint8_t *a = p.a_scales + (int64_t)min(m0 + tid, p.M - 1) * p.scale_pitch + step * 4;
        const uint8_t *b = p.b_scales + (int64_t)min(n0 + tid, p.N - 1) * p.scale_pitch + step * 4;
        if (step * 4 + 16 <= p.blocks) {
            __builtin_memcpy(&sa, a, 16);
            __builtin_memcpy(&sb, b, 16);
        } else {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int left = p.blocks - (step + w) * 4;     // blocks of this word
                const uint32_t mask = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
                sa[w] = left > 0 ? *(const uint32_t *)(a + 4 * w) & mask : 0u;
                sb[w] = left > 0 ? *(const uint32_t *)(b + 4 * w) & mask : 0u;
            }
        }
    };

    const uint32_t lane_at = tile_place(r, g);
    struct Operands {
        v4u a[8], b[8];
    };
    auto read = [&](int buffer, Operands &o) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            o.a[i] = lds_a[buffer][(wm * 8 + i) * 64 + lane_at];
            o.b[i] = lds_b[buffer][(wn * 8 + i) * 64 + lane_at];
        }
    };

    v4f acc[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    const uint32_t pick = (uint32_t)g | (uint32_t)(4 + g) << 8 | 0x0c0c0000u;
    int sa[8], sb[8];
    TileStage stage;
    Operands now;
    v4u fa, fb;
    fetch(0, stage);
    fetch_scales(0, fa, fb);
    put(0, stage);
    lds_sa[tid] = fa;
    lds_sb[tid] = fb;
    fetch(min(1, steps - 1), stage);
    __syncthreads();
    read(0, now);
    for (int step0 = 0; step0 < steps; step0 += 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sa[i] = scale_bytes(lds_sa[wm * 128 + 16 * i + r], pick);
            sb[i] = scale_bytes(lds_sb[wn * 128 + 16 * i + r], pick);
        }
        fetch_scales(min(step0 + 4, steps - 1), fa, fb);
        auto one = [&](auto which) {
            constexpr int W = decltype(which)::value;
            const int step = step0 + W;
            if (step >= steps) return;
            put((W + 1) & 1, stage);                    // step + 1, whose buffer was read two steps ago
            fetch(min(step + 2, steps - 1), stage);
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    acc[i][j] = product_step<W>(now.b[j], now.a[i], acc[i][j], sb[j], sa[i]);
            if (W == 3) {
                lds_sa[tid] = fa;
                lds_sb[tid] = fb;
            }
            __syncthreads();
            read((W + 1) & 1, now);
        };
        one(std::integral_constant<int, 0>{});
        one(std::integral_constant<int, 1>{});
        one(std::integral_constant<int, 2>{});
        one(std::integral_constant<int, 3>{});
    }

#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            store_results<T>(p, m0 + wm * 128 + 16 * i + r, n0 + wn * 128 + 16 * j + 4 * g, acc[i][j]);
}

template <Num T>
hipError_t tiled(const ProductArgs &p, hipStream_t stream)
{
    const int mtiles = (p.M + kTile - 1) / kTile, ntiles = (p.N + kTile - 1) / kTile;
    hipLaunchKernelGGL((product_tile_kernel<T>), dim3(mtiles * ntiles), dim3(256), 0, stream, p, mtiles, ntiles);
    return hipGetLastError();
}

template <Num T>
hipError_t product_typed(const ProductArgs &p, hipStream_t stream)
{
    if (p.M <= 64) return direct<T, false, 1, 1, 4, 4>(p, stream);
    if (p.N <= 32) return direct<T, false, 2, 2, 4, 1>(p, stream);
    if ((int64_t)((p.M + kTile - 1) / kTile) * ((p.N + kTile - 1) / kTile) >= 64) return tiled<T>(p, stream);
    return direct<T, false, 4, 4, 4, 1>(p, stream);
}

ProductArgs arguments(int M, int N, int K, const void *a, const uint8_t *a_scales, int64_t a_stride,
                      const uint8_t *b, const uint8_t *b_scales, const float *bias, void *c, int64_t c_stride)
{
    ProductArgs p;
    p.a = a; p.a_scales = a_scales; p.a_stride = a_stride; p.b = b; p.b_scales = b_scales;
    p.pitch = (uint32_t)mx_code_pitch(Mx::E2M1, K); p.scale_pitch = (uint32_t)mx_scale_pitch(K);
    p.M = M; p.N = N; p.K = K; p.blocks = (int)mx_blocks(K);
    p.bias = bias; p.c = c; p.c_stride = c_stride;
    return p;
}

// One pass over the plain rows where they are read about once: few columns of C (each workgroup of rows
// quantises its rows for all of them), or so few rows that quantising them again costs nothing.
bool linear_fused(int M, int N) { return N <= 64 || M <= 16; }

}  // namespace

hipError_t launch_mx4_product(Num out, int M, int N, int K, const uint8_t *a_codes, const uint8_t *a_scales,
                              const uint8_t *b_codes, const uint8_t *b_scales, const float *bias, void *c,
                              int64_t c_stride, hipStream_t stream)
{
    const ProductArgs p = arguments(M, N, K, a_codes, a_scales, 0, b_codes, b_scales, bias, c, c_stride);
    switch (out) {
    case Num::F32: return product_typed<Num::F32>(p, stream);
    case Num::F16: return product_typed<Num::F16>(p, stream);
    case Num::BF16: return product_typed<Num::BF16>(p, stream);
    }
    return hipErrorInvalidValue;
}

size_t mx4_linear_workspace(int M, int N, int K)
{
    if (linear_fused(M, N)) return 0;
    return (size_t)M * (mx_code_pitch(Mx::E2M1, K) + mx_scale_pitch(K));
}

namespace {

template <Num T>
hipError_t linear_typed(const ProductArgs &p, void *workspace, hipStream_t stream)
{
    if (linear_fused(p.M, p.N)) {
        if (p.M <= 64) return direct<T, true, 1, 1, 4, 4>(p, stream);
        if (p.N <= 32) return direct<T, true, 2, 2, 4, 1>(p, stream);
        return direct<T, true, 2, 4, 4, 1>(p, stream);
    }
    uint8_t *codes = (uint8_t *)workspace, *scales = codes + (int64_t)p.M * p.pitch;
    const hipError_t e = launch_mx_pack(Mx::E2M1, T, p.M, p.K, p.a, p.a_stride, codes, scales, stream);
    if (e != hipSuccess) return e;
    ProductArgs q = p;
    q.a = codes;
    q.a_scales = scales;
    return product_typed<T>(q, stream);
}

}  // namespace

hipError_t launch_mx4_linear(Num t, int M, int N, int K, const void *x, int64_t x_stride, const uint8_t *w_codes,
                             const uint8_t *w_scales, const float *bias, void *c, int64_t c_stride, void *workspace,
                             hipStream_t stream)
{
    const ProductArgs p = arguments(M, N, K, x, nullptr, x_stride, w_codes, w_scales, bias, c, c_stride);
    switch (t) {
    case Num::F32: return linear_typed<Num::F32>(p, workspace, stream);
    case Num::F16: return linear_typed<Num::F16>(p, workspace, stream);
    case Num::BF16: return linear_typed<Num::BF16>(p, workspace, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace mg
