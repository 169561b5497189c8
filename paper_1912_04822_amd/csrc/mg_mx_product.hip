// Products of matrices in 4 bits (e2m1 elements, formats: mg_mx.h):
//     C[m][n] = sum_k A[m][k] B[n][k] + bias[n]
// with v_mfma_scale_f32_16x16x128_f8f6f4.  An operand of that instruction is 32 consecutive k of one row
// per lane (row = lane % 16, group of 32 = lane / 16) with that lane's scale byte: exactly a block of the
// format, so 16 bytes of codes and one byte of scales go from memory to the matrix cores as they lie.
// Products of elements and scales are exact; sums are in float.
//
// The operands are given as (B, A), so a lane's four results are 4 neighbouring n of one row m of C.
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

template <Num T>
hipError_t product_typed(const ProductArgs &p, hipStream_t stream)
{
    if (p.M <= 64) return direct<T, false, 1, 1, 4, 4>(p, stream);
    if (p.N <= 32) return direct<T, false, 2, 2, 4, 1>(p, stream);
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
