// Numbers into the codes of a microscaled format, and back (layout and rounding: mg_mx.h).
//
// One lane holds 16 bytes of plain numbers (4 floats or 8 halves), so 8 or 4 neighbouring lanes hold a
// block: its largest magnitude is three or two exchanges within a row of lanes (DPP, no LDS), and both
// the plain numbers and the codes are moved in runs that are contiguous over the wavefront.  Magnitudes
// are compared as unsigned words, where a NaN is larger than everything: a block that is not finite is
// found by its maximum alone.  Both directions are bound by memory: a number is read or written once and
// meets about a dozen instructions.  Measured (medians of launches), with a copy at 5.1 TB/s (read and written):
// 155 million floats to int8 in 127 us and back in 99 (6.1 and 7.8 TB/s of their 0.78 GB), 22 million bfloat16
// to e4m3 in 12.8 and back in 12.4 (5.3), 128000 odd rows of 509 halves to e2m1 in 44 (3.8) and back in 26.5 (6.2).
#include "mg_common.h"
#include "mg_mx.h"

namespace mg {

namespace {

constexpr int kThreads = 256;

__device__ inline void store16(void *p, v4u v) { __builtin_memcpy(p, &v, 16); }

// A tensor that is larger than the memory-side cache is not found there by whoever comes next: it is read or
// written past the caches (137 -> 119 and 131 -> 110 us for 0.62 GB of floats), aligned as it must be for that.
// Smaller ones are not: what was just produced is still there, and what is restored is read again at once.
bool streamed(const void *p, int64_t rows, int64_t row_stride, int64_t cols, int bytes)
{
    return rows * cols * bytes > kMemoryCacheBytes && ((uintptr_t)p & 15) == 0 &&
           (rows == 1 || row_stride * bytes % 16 == 0);
}

template <Num T> __device__ inline v4u narrow(const float *f)
{
    v4u w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (T == Num::F32) {
            w[i] = mx_word(f[i]);
        } else {
            using H = typename NumTraits<T>::type;
            w[i] = (uint32_t)__builtin_bit_cast(uint16_t, (H)f[2 * i]) |
                   (uint32_t)__builtin_bit_cast(uint16_t, (H)f[2 * i + 1]) << 16;
        }
    }
    return w;
}

// Blocks are counted along the scale rows, whose length is a multiple of four: those past a row's last
// block only clear their shared byte.
template <Num T, Mx F, int Unroll, bool Stream>
__global__ __launch_bounds__(kThreads) void pack_kernel(const unsigned char *x, int64_t row_stride,
                                                        int64_t cols, uint32_t blocks, uint32_t pitch,
                                                        uint32_t total, uint8_t *codes, uint8_t *scales)
{
    constexpr int P = kPerLane<T>, L = kMxBlock / P;
    constexpr uint32_t kBlocks = kThreads / L;              // blocks a workgroup takes at a time
    const uint32_t first = (blockIdx.x + blockIdx.y * gridDim.x) * (kBlocks * Unroll) + threadIdx.x / L;
    const int sub = threadIdx.x % L;
    v4u raw[Unroll];
    uint32_t at[Unroll], blk[Unroll];
    uint32_t row[Unroll];
#pragma unroll
    for (int u = 0; u < Unroll; ++u) {
        const uint32_t g = first + u * kBlocks;
        at[u] = g;
        row[u] = pitch >= total ? 0u : g / pitch;           // one row: no division
        blk[u] = g - row[u] * pitch;
        raw[u] = v4u{0, 0, 0, 0};
        if (g < total && blk[u] < blocks) {
            const int64_t c = (int64_t)blk[u] * kMxBlock + sub * P;
            const unsigned char *p = x + (int64_t)row[u] * row_stride * NumTraits<T>::bytes;
            if (Stream && c + P <= cols) raw[u] = __builtin_nontemporal_load((const v4u *)(p + c * NumTraits<T>::bytes));
            else raw[u] = load_row<T>(p, c, cols);
        }
    }
#pragma unroll
    for (int u = 0; u < Unroll; ++u) {
        float f[P];
        widen<T>(raw[u], f);
        const uint32_t s = scale_block<F, T>(f);
        if (at[u] >= total) continue;
        if (sub == 0) scales[at[u]] = blk[u] < blocks ? (uint8_t)s : (uint8_t)0;
        if (blk[u] >= blocks) continue;
        const int64_t to = ((int64_t)row[u] * blocks + blk[u]) * L + sub;       // in units of P elements
        if constexpr (F == Mx::E2M1) {
            const uint32_t w = encode_e2m1<T>(f);
            if constexpr (P == 8) ((uint32_t *)codes)[to] = w;
            else ((uint16_t *)codes)[to] = (uint16_t)w;
        } else if constexpr (P == 8) {
            ((uint2 *)codes)[to] = make_uint2(mx_encode4<F>(f), mx_encode4<F>(f + 4));
        } else {
            ((uint32_t *)codes)[to] = mx_encode4<F>(f);
        }
    }
}

// Elements of one word: four of 8 bits.
template <Mx F> __device__ inline void decode4(uint32_t w, float *f)
{
    if constexpr (F == Mx::INT8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = (float)(int)(int8_t)(w >> (8 * i));
    } else {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
        const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        f[0] = lo[0]; f[1] = lo[1]; f[2] = hi[0]; f[3] = hi[1];
    }
}

template <Num T, Mx F, int Unroll, bool Stream>
__global__ __launch_bounds__(kThreads) void unpack_kernel(const uint8_t *codes, const uint8_t *scales,
                                                          int64_t cols, uint32_t blocks, uint32_t pitch,
                                                          uint32_t total, unsigned char *x,
                                                          int64_t row_stride)
{
    constexpr int P = kPerLane<T>, L = kMxBlock / P;
    constexpr uint32_t kBlocks = kThreads / L;
    const uint32_t first = (blockIdx.x + blockIdx.y * gridDim.x) * (kBlocks * Unroll) + threadIdx.x / L;
    const int sub = threadIdx.x % L;
    uint32_t w[Unroll][2], row[Unroll], blk[Unroll];
    int s[Unroll];
#pragma unroll
    for (int u = 0; u < Unroll; ++u) {
        const uint32_t g = first + u * kBlocks;             // blocks are counted without padding here
        row[u] = blocks >= total ? 0u : g / blocks;
        blk[u] = g - row[u] * blocks;
        w[u][0] = w[u][1] = 0;
        s[u] = 0;
        if (g < total) {
            const int64_t from = (int64_t)g * L + sub;
            s[u] = scales[(int64_t)row[u] * pitch + blk[u]];
            if constexpr (F == Mx::E2M1 && P == 4) {
                w[u][0] = ((const uint16_t *)codes)[from];
            } else if constexpr (F == Mx::E2M1 || P == 4) {
                w[u][0] = ((const uint32_t *)codes)[from];
            } else {
                const uint2 v = ((const uint2 *)codes)[from];
                w[u][0] = v.x;
                w[u][1] = v.y;
            }
        }
    }
#pragma unroll
    for (int u = 0; u < Unroll; ++u) {
        if (first + u * kBlocks >= total) continue;
        float f[8];
        if constexpr (F == Mx::E2M1) {
            const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u][0], 1.0f, 0);
            const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u][0], 1.0f, 1);
            f[0] = a[0]; f[1] = a[1]; f[2] = b[0]; f[3] = b[1];
            if constexpr (P == 8) {
                const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u][0], 1.0f, 2);
                const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u][0], 1.0f, 3);
                f[4] = c[0]; f[5] = c[1]; f[6] = d[0]; f[7] = d[1];
            }
        } else {
            decode4<F>(w[u][0], f);
            if constexpr (P == 8) decode4<F>(w[u][1], f + 4);
        }
        const float scale = mx_power((uint32_t)s[u]);       // a NaN scale or e4m3's NaN codes make a NaN
        constexpr float top = T == Num::F16 ? 65504.0f : T == Num::BF16 ? 0x1.fep127f : 0x1.fffffep127f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            // the bounds that hand a NaN on (fminf and fmaxf would make it finite)
            f[i] = __builtin_elementwise_minimum(__builtin_elementwise_maximum(f[i] * scale, -top), top);
        }
        const v4u out = narrow<T>(f);
        const int64_t c = (int64_t)blk[u] * kMxBlock + sub * P;
        unsigned char *p = x + ((int64_t)row[u] * row_stride + c) * NumTraits<T>::bytes;
        if (c + P <= cols) {
            if constexpr (Stream) __builtin_nontemporal_store(out, (v4u *)p);
            else store16(p, out);
        } else if (c < cols) {
            using E = typename NumTraits<T>::type;
            E e[P];
            __builtin_memcpy(e, &out, 16);
#pragma unroll
            for (int i = 0; i < P; ++i)
                if (c + i < cols) ((E *)p)[i] = e[i];
        }
    }
}

constexpr int kUnroll = 4;

// A launch counts the threads along x in 32 bits: 2^24 workgroups, which floats in 2^31 - 127 blocks or more take,
// are one too many.
dim3 grid(uint32_t groups) { return groups < (1u << 24) ? dim3(groups) : dim3((groups + 1) / 2, 2); }

template <Num T, Mx F>
hipError_t pack_typed(int64_t rows, int64_t cols, const void *x, int64_t row_stride, uint8_t *codes,
                      uint8_t *scales, hipStream_t stream)
{
    const uint32_t blocks = (uint32_t)mx_blocks(cols), pitch = (uint32_t)mx_scale_pitch(cols);
    const uint32_t total = (uint32_t)(rows * pitch);
    constexpr uint32_t per = kThreads / (kMxBlock / kPerLane<T>) * kUnroll;
    const auto kernel = streamed(x, rows, row_stride, cols, NumTraits<T>::bytes) ? pack_kernel<T, F, kUnroll, true>
                                                                                : pack_kernel<T, F, kUnroll, false>;
    hipLaunchKernelGGL(kernel, grid((total + per - 1) / per), dim3(kThreads), 0, stream, (const unsigned char *)x,
                       row_stride, cols, blocks, pitch, total, codes, scales);
    return hipGetLastError();
}

template <Num T, Mx F>
hipError_t unpack_typed(int64_t rows, int64_t cols, const uint8_t *codes, const uint8_t *scales, void *x,
                        int64_t row_stride, hipStream_t stream)
{
    const uint32_t blocks = (uint32_t)mx_blocks(cols), pitch = (uint32_t)mx_scale_pitch(cols);
    const uint32_t total = (uint32_t)(rows * blocks);
    constexpr uint32_t per = kThreads / (kMxBlock / kPerLane<T>) * kUnroll;
    const auto kernel = streamed(x, rows, row_stride, cols, NumTraits<T>::bytes) ? unpack_kernel<T, F, kUnroll, true>
                                                                                : unpack_kernel<T, F, kUnroll, false>;
    hipLaunchKernelGGL(kernel, grid((total + per - 1) / per), dim3(kThreads), 0, stream, codes, scales, cols, blocks,
                       pitch, total, (unsigned char *)x, row_stride);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_pack(Mx f, Num t, int64_t rows, int64_t cols, const void *x, int64_t row_stride,
                          uint8_t *codes, uint8_t *scales, hipStream_t stream)
{
#define MG_CASE(TT, FF) if (t == Num::TT && f == Mx::FF) \
        return pack_typed<Num::TT, Mx::FF>(rows, cols, x, row_stride, codes, scales, stream)
    MG_CASE(F32, INT8); MG_CASE(F32, E4M3); MG_CASE(F32, E2M1);
    MG_CASE(F16, INT8); MG_CASE(F16, E4M3); MG_CASE(F16, E2M1);
    MG_CASE(BF16, INT8); MG_CASE(BF16, E4M3); MG_CASE(BF16, E2M1);
#undef MG_CASE
    return hipErrorInvalidValue;
}

hipError_t launch_mx_unpack(Mx f, Num t, int64_t rows, int64_t cols, const uint8_t *codes,
                            const uint8_t *scales, void *x, int64_t row_stride, hipStream_t stream)
{
#define MG_CASE(TT, FF) if (t == Num::TT && f == Mx::FF) \
        return unpack_typed<Num::TT, Mx::FF>(rows, cols, codes, scales, x, row_stride, stream)
    MG_CASE(F32, INT8); MG_CASE(F32, E4M3); MG_CASE(F32, E2M1);
    MG_CASE(F16, INT8); MG_CASE(F16, E4M3); MG_CASE(F16, E2M1);
    MG_CASE(BF16, INT8); MG_CASE(BF16, E4M3); MG_CASE(BF16, E2M1);
#undef MG_CASE
    return hipErrorInvalidValue;
}

}  // namespace mg
