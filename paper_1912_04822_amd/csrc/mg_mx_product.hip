// Products of matrices in 4 bits (e2m1 elements, formats: mg_mx.h):
//     C[m][n] = sum_k A[m][k] B[n][k] + bias[n]
// with v_mfma_scale_f32_16x16x128_f8f6f4 and 32x32x64.  An operand of these is 32 consecutive k of one row per
// lane (row = lane % 16 or 32, group of 32 = lane / 16 or 32) with that lane's scale byte: exactly a block of
// the format, so 16 bytes of codes and one byte of scales go from memory to the matrix cores as they lie.
// Products of elements and scales are exact; sums are in float.
//
// The operands are given as (B, A), so a lane's four results are 4 neighbouring n of one row m of C.
//
// Measured: 16320 x 4096 x 4096 into bfloat16 149 us (3.7 PFLOP/s; of it 29 us for a quarter of k and about 33
// that do not depend on k: 134 MB of results, four rounds of workgroups; 185 us in a loop of nothing else);
// 2040 x 509 x 1000 7.4; plain rows of 102000 x 256 floats to 28 columns 23.4 (116 MB: 5.0 TB/s); one row by
// 4096 x 4096 6.0 (8.9 MB of weights).
#include <type_traits>

#include "mg_common.h"
#include "mg_mx.h"
#include "mg_mx_ops.h"

namespace mg {

namespace {

using v8i = __attribute__((ext_vector_type(8))) int;
using v4f = __attribute__((ext_vector_type(4))) float;
using v16f = __attribute__((ext_vector_type(16))) float;

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
            widen<T>(w, f + i * P);
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

__device__ inline v4f load_bias(const ProductArgs &p, int n)
{
    v4f b = {0.0f, 0.0f, 0.0f, 0.0f};
    if (p.bias) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < p.N) b[i] = p.bias[n + i];
    }
    return b;
}

// Four neighbouring results of row m.
template <Num T>
__device__ inline void store_results(const ProductArgs &p, int m, int n, v4f v)
{
    using E = typename NumTraits<T>::type;
    if (m >= p.M || n >= p.N) return;
    E *to = (E *)p.c + (int64_t)m * p.c_stride + n;
    const E e[4] = {(E)v[0], (E)v[1], (E)v[2], (E)v[3]};
    if (n + 4 <= p.N) {
        __builtin_memcpy(to, e, sizeof e);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < p.N) to[i] = e[i];
    }
}

// Operands straight from memory.  A wavefront holds RM x RN tiles of 16 x 16; the KW wavefronts of a
// group share a tile and split k between them (their sums meet in LDS), the others lie along m.  Two steps'
// operands are asked for at a time.  Plain numbers are read by the lane that wants them, 128 bytes of a row in
// 16-byte loads; read as they lie by neighbouring lanes and exchanged through LDS they take 26.0 instead of 28.7
// us from memory at 102000 x 256 floats, but 20.6 instead of 13.9 at 8000 x 1000 and 14.2 instead of 12.8 at 8000
// x 1024 by 64 columns.
template <Num T, bool Plain, int RM, int RN, int Waves, int KW>
__global__ __launch_bounds__(64 * Waves) void product_kernel(ProductArgs p)
{
    constexpr int U = 2;
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

    for (int k = kw * 4; k < p.blocks; k += U * KW * 4) {
        Operand a[U][RM], b[U][RN];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < RN; ++j) b[u][j] = load_block(p.b, p.b_scales, p, brow[j], k + u * KW * 4 + g);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < RM; ++i) {
                if constexpr (Plain) a[u][i] = quantise_block<T>(p, arow[i], k + u * KW * 4 + g);
                else a[u][i] = load_block((const uint8_t *)p.a, p.a_scales, p, arow[i], k + u * KW * 4 + g);
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < RM; ++i)
#pragma unroll
                for (int j = 0; j < RN; ++j) acc[i][j] = product(b[u][j], a[u][i], acc[i][j]);
    }

    if constexpr (KW > 1) {
        // the sums of a group in LDS; every wavefront of it adds up and stores its share of the tiles
        __shared__ v4f sums[Waves][RM * RN][64];
#pragma unroll
        for (int i = 0; i < RM; ++i)
#pragma unroll
            for (int j = 0; j < RN; ++j) sums[wave][i * RN + j][lane] = acc[i][j];
        __syncthreads();
        for (int tile = kw; tile < RM * RN; tile += KW) {
            v4f v = sums[mw * KW][tile][lane];
#pragma unroll
            for (int w = 1; w < KW; ++w) v += sums[mw * KW + w][tile][lane];
            const int n = n0 + 16 * (tile % RN) + 4 * g;
            store_results<T>(p, m0 + 16 * (tile / RN) + r, n, v + load_bias(p, n));
        }
    } else {
#pragma unroll
        for (int j = 0; j < RN; ++j) {
            const v4f bias = load_bias(p, n0 + 16 * j + 4 * g);
#pragma unroll
            for (int i = 0; i < RM; ++i) store_results<T>(p, m0 + 16 * i + r, n0 + 16 * j + 4 * g, acc[i][j] + bias);
        }
    }
}

template <Num T, bool Plain, int RM, int RN, int Waves, int KW>
hipError_t direct(const ProductArgs &p, hipStream_t stream)
{
    const int rows = Waves / KW * RM * 16;
    const dim3 grid((p.M + rows - 1) / rows, (p.N + RN * 16 - 1) / (RN * 16));
    hipLaunchKernelGGL((product_kernel<T, Plain, RM, RN, Waves, KW>), grid, dim3(64 * Waves), 0, stream, p);
    return hipGetLastError();
}

// Large products: a workgroup of 4 wavefronts makes a square tile of C, each wavefront a quarter of it as WT x WT
// tiles of 32 x 32, with v_mfma_scale_f32_32x32x64_f8f6f4: from registers alone it reaches 9.0 PFLOP/s (6.3 with
// random codes, where the chip lowers its clock), the 16 x 16 x 128 form 5.6 (4.9).  Codes go through LDS, where
// every byte is read by two wavefronts.  WT = 4, 256 x 256 in 256 accumulator registers, one wavefront per SIMD:
// per 128 k a wavefront issues 32 products (1024 cycles of its matrix core) for 16 operands of 1 KB.  WT = 2,
// 128 x 128, two workgroups to a compute unit: twice the reads of LDS per product, for products that are too
// small to fill the chip with large tiles.
//   - Two buffers of 256 k, whole lines of 128 bytes a row (64 bytes at a time ask the caches for twice as
//     much: 170 against 165 us at 16320 x 4096 x 4096).  Codes go from memory to LDS without passing
//     registers, two steps of 128 k ahead, and from LDS to registers one step ahead, while the products of
//     the step before run.
//   - A row's 128 bytes lie in LDS as eight pieces of 16, piece c at place c ^ (row / 2) % 8: the 16 rows that a
//     quarter of a wavefront reads at once then cover all banks.
//   - Scales are taken for four steps at a time (16 bytes of a row); three byte permutes turn them into one
//     register that holds a lane's scale of each of the four steps, which the instruction picks by its
//     operand selector.
// Past the end of k the codes of A are zeros and the scales powers of two; rows past M or N repeat the last
// one and are not stored.

__device__ inline uint32_t tile_place(uint32_t row, uint32_t piece) { return row * 8 + (piece ^ ((row >> 1) & 7)); }

template <int Step> __device__ inline v16f product_step(v4u b, v4u a, v16f c, int sb, int sa)
{
    const v8i x = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    const v8i y = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, kE2m1, kE2m1, Step, sb, Step, sa);
}

// The byte that `pick` names of each of four words.
__device__ inline int scale_bytes(v4u w, uint32_t pick)
{
    const uint32_t lo = __builtin_amdgcn_perm(w[1], w[0], pick), hi = __builtin_amdgcn_perm(w[3], w[2], pick);
    return (int)__builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

// 16 bytes per lane from memory (a common base, an offset per lane) to LDS, where they lie one lane after the
// other.  Written as an instruction because the compiler would wait for every load under way before each read
// of LDS (223 against 209 us, before the steps that followed); nothing is returned to registers, and wait_loads
// and the barrier stand before the first read of what was loaded.  The address in LDS goes by m0, which is put
// back.
__device__ inline void load_to_lds(const uint8_t *base, uint32_t offset, uint32_t lds)
{
    uint32_t m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "v"(offset), "s"(base), "s"(lds) : "memory");
}
__device__ inline void load_word_to_lds(const float *base, uint32_t offset, uint32_t lds)       // 4 bytes per lane
{
    uint32_t m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "v"(offset), "s"(base), "s"(lds) : "memory");
}
__device__ inline uint32_t lds_address(const v4u *p)
{
    return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p);
}

// Waits until at most N of this wavefront's loads are under way, and for its LDS accesses.
template <int N> __device__ inline void wait_loads()
{
    __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (N >> 4) << 14);
}

template <Num T, int WT>
__global__ __launch_bounds__(256, WT == 4 ? 1 : 2) void product_tile_kernel(ProductArgs p, int mtiles, int ntiles)
{
    constexpr int kTile = 64 * WT;
    constexpr int kBuffer = kTile * 16;                     // 16-byte pieces of a buffer: codes of A, then of B
    constexpr int kLoads = 4 * WT;                          // a wavefront's loads of a buffer, 8 rows each
    // then 16 bytes of scales for every row of A and B, and the bias
    __shared__ v4u lds[2 * kBuffer + 2 * kTile + kTile / 4];
    v4u *const lds_s = lds + 2 * kBuffer, *const lds_bias = lds_s + 2 * kTile;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 31, h = lane >> 5;                 // an operand: row r, the h-th 32 of its 64 k
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
    const uint8_t *const base_a = (const uint8_t *)p.a + (int64_t)m0 * p.pitch;
    const uint8_t *const base_b = p.b + (int64_t)n0 * p.pitch;
    const uint32_t piece = (lane & 7) ^ (4 * (wave & 1) + (lane >> 4));     // see tile_place: row / 2 modulo 8
    uint32_t off[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int row = (4 * (i % (2 * WT)) + wave) * 8 + (lane >> 3);
        off[i] = (uint32_t)min(row, (i < 2 * WT ? p.M - m0 : p.N - n0) - 1) * p.pitch + 16 * piece;
    }
    const uint32_t put = lds_address(lds) + wave * 1024;
    auto fetch = [&](int pair, int buffer, int which, uint32_t back) {      // 8 rows of A, or (from 2 WT on) of B
        load_to_lds((which < 2 * WT ? base_a : base_b) + pair * 128, off[which] - back,
                    put + buffer * kBuffer * 16 + which * 4096);
    };
    // pieces past a row's end are not read: the lane takes the pair's first piece, which its row has
    auto past_end = [&](int pair) { return pair * 8 + (int)piece < p.blocks ? 0u : 16 * piece; };
    auto fetch_scales = [&](int step) {                     // of steps step .. step + 3
#pragma unroll
        for (int i = 0; i < WT / 2; ++i) {
            const int unit = 4 * i + wave;                  // 64 rows of A, or (from WT on) of B
            const bool of_b = unit >= WT;
            const uint8_t *base = of_b ? p.b_scales + (int64_t)n0 * p.scale_pitch : p.a_scales + (int64_t)m0 * p.scale_pitch;
            const int row = (of_b ? unit - WT : unit) * 64 + lane;
            const uint32_t at = (uint32_t)min(row, (of_b ? p.N - n0 : p.M - m0) - 1) * p.scale_pitch;
            if (step * 4 + 16 <= p.blocks) {
                load_to_lds(base + step * 4, at, lds_address(lds_s) + unit * 1024);
                continue;
            }
            v4u s;                                          // a row's end: bytes past it become zeros
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int left = p.blocks - (step + w) * 4; // blocks of this word
                const uint32_t mask = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
                s[w] = left > 0 ? *(const uint32_t *)(base + at + (step + w) * 4) & mask : 0u;
            }
            lds_s[unit * 64 + lane] = s;
        }
    };

    uint32_t lane_at[2][2];                                 // [step of the pair][first or second 64 k]
#pragma unroll
    for (int o = 0; o < 2; ++o)
#pragma unroll
        for (int k = 0; k < 2; ++k) lane_at[o][k] = tile_place(r, 4 * o + 2 * k + h);
    struct Operands {
        v4u a[2][WT], b[2][WT];
    };
    auto read = [&](int step, int which, Operands &to) {    // one of 4 WT, those of the first 64 k first
        const v4u *from = lds + (step >> 1 & 1) * kBuffer;
        const int k = which / (2 * WT), i = which % WT, o = step & 1;
        if (which / WT & 1) to.a[k][i] = from[(wm * WT + i) * 256 + lane_at[o][k]];
        else to.b[k][i] = from[kTile * 8 + (wn * WT + i) * 256 + lane_at[o][k]];
    };
    const uint32_t pick = (uint32_t)h | (uint32_t)(4 + h) << 8 | 0x0c0c0000u;
    struct Scales {
        int a[2][WT], b[2][WT];
    };
    auto read_scales = [&](int i, Scales &s) {              // one of the WT rows of tiles
        const v4u a = lds_s[(wm * WT + i) * 32 + r], b = lds_s[kTile + (wn * WT + i) * 32 + r];
        s.a[0][i] = scale_bytes(a, pick);
        s.b[0][i] = scale_bytes(b, pick);
        s.a[1][i] = scale_bytes(a, pick + 0x0202u);
        s.b[1][i] = scale_bytes(b, pick + 0x0202u);
    };

    v16f acc[WT][WT];
#pragma unroll
    for (int i = 0; i < WT; ++i)
#pragma unroll
        for (int j = 0; j < WT; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.0f;

    Scales scales, later;
    Operands even, odd;
    const int last_pair = (steps - 1) >> 1;
    if (wave < WT) {
        if (p.bias)
            load_word_to_lds(p.bias + n0, 4 * (uint32_t)min(wave * 64 + lane, p.N - n0 - 1), lds_address(lds_bias) + wave * 256);
        else
            ((float *)lds_bias)[wave * 64 + lane] = 0.0f;
    }
    fetch_scales(0);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int pair = min(q, last_pair);
        const uint32_t back = past_end(pair);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) fetch(pair, q, i, back);
    }
    wait_loads<kLoads>();
    __builtin_amdgcn_s_barrier();
#pragma unroll
    for (int q = 0; q < 4 * WT; ++q) read(0, q, even);
#pragma unroll
    for (int i = 0; i < WT; ++i) read_scales(i, later);

    for (int step0 = 0; step0 < steps; step0 += 4) {
        scales = later;
        // One step.  Between its products the next step's operands are read.  At the barrier of the second
        // step of a pair every wavefront has this pair's operands in registers and the next pair's codes in
        // LDS, and the pair after that is asked for (the last pair again where there is none: nothing reads
        // it).  The order is pinned: a wavefront issues one instruction at a time, and everything else has to
        // fit between two products.
        auto one = [&](auto which) {
            constexpr int W = decltype(which)::value;
            const int step = step0 + W;
            if (step >= steps) return;
            Operands &now = W & 1 ? odd : even, &next = W & 1 ? even : odd;
            int ahead = 0;
            uint32_t back = 0;
            if constexpr (W & 1) {
                wait_loads<0>();
                __builtin_amdgcn_s_barrier();
                if (W == 1 && step + 3 < steps) fetch_scales(step + 3);
                ahead = min((step >> 1) + 2, last_pair);
                back = past_end(ahead);
            }
            if (step * 4 + 4 > p.blocks) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const bool in_row = step * 4 + 2 * k + h < p.blocks;
#pragma unroll
                    for (int i = 0; i < WT; ++i) now.a[k][i] = in_row ? now.a[k][i] : v4u{0, 0, 0, 0};
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            constexpr int kProducts = 2 * WT * WT, kReads = 4 * WT, kLate = kProducts / 4;
#pragma unroll
            for (int t = 0; t < kProducts; ++t) {
                const int k = t / (WT * WT), i = t / WT % WT, j = t % WT;
                acc[i][j] = product_step<W>(now.b[k][j], now.a[k][i], acc[i][j], scales.b[k][j], scales.a[k][i]);
                if constexpr (W & 1) {
                    if (t < kLoads) fetch(ahead, W >> 1, t, back);
                    if (WT == 4 ? t >= kLate && t < kLate + kReads : true) read(W + 1, WT == 4 ? t - kLate : t, next);
                    if (W == 3 && t >= kProducts - WT) read_scales(t - (kProducts - WT), later);
                } else if (t < kReads) {
                    read(W + 1, t, next);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        one(std::integral_constant<int, 0>{});
        one(std::integral_constant<int, 1>{});
        one(std::integral_constant<int, 2>{});
        one(std::integral_constant<int, 3>{});
    }

    // A wavefront turns its results, already of their type, through LDS, 32 rows of 32 WT at a time (rows 16 bytes
    // further apart for the banks), and stores 16 bytes per lane, rows at a stretch.  A part of C that is full goes
    // past the caches where its rows begin with a line: 4096 x 4096 x 1024 into bfloat16 takes 17 us so and 24 with
    // ordinary stores, 32 and 37 together with a kernel that reads the result.  Where rows share lines, only a
    // result that the memory-side cache does not hold does: 8000 x 1004 x 500 into floats 11.5 us with ordinary
    // stores and 14.7 past the caches, 100000 x 1000 x 1000 179 and 160.  Kept short: a small product runs through
    // this code once, and waits for it to come from memory (2040 x 509 x 1000 7.4 us; with a choice of stores also
    // at the edges 7.7).
    using E = typename NumTraits<T>::type;
    constexpr int P = 16 / NumTraits<T>::bytes, kLanes = 32 * WT / P, kRows = 64 / kLanes;
    constexpr int kPitch = 32 * WT * sizeof(E) + 16;
    const int at_m = m0 + wm * 32 * WT, at_n = n0 + wn * 32 * WT;
    const uintptr_t c_bits = (uintptr_t)p.c | (uintptr_t)(p.c_stride * sizeof(E));
    const bool past = (c_bits & ((int64_t)p.M * p.N * (int)sizeof(E) > kMemoryCacheBytes ? 15 : 127)) == 0;
    const bool inside = past && at_m + 32 * WT <= p.M && at_n + 32 * WT <= p.N;
    wait_loads<0>();
    __builtin_amdgcn_s_barrier();
    uint8_t *const mine = (uint8_t *)(lds + wave * (kBuffer / 2));
    const float *const bias = (const float *)lds_bias + wn * 32 * WT;
    const int part = lane % kLanes, first = lane / kLanes, n = at_n + P * part;
#pragma unroll
    for (int i = 0; i < WT; ++i) {
#pragma unroll
        for (int j = 0; j < WT; ++j) {
            if constexpr (WT == 4) asm volatile("" : "+a"(acc[i][j]));  // it stays in its accumulators until here
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = 32 * j + 8 * q + 4 * h;
                const v4f b = *(const v4f *)(bias + c);
                E e[4];
#pragma unroll
                for (int d = 0; d < 4; ++d) e[d] = (E)(acc[i][j][4 * q + d] + b[d]);
                __builtin_memcpy(mine + r * kPitch + c * sizeof(E), e, sizeof(e));
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const uint8_t *const from = mine + first * kPitch + 16 * part;
        const int m = at_m + 32 * i + first;
        E *const to = (E *)p.c + (int64_t)m * p.c_stride + n;
        if (inside) {
#pragma unroll
            for (int t = 0; t < 32; t += kRows)
                __builtin_nontemporal_store(*(const v4u *)(from + t * kPitch), (v4u *)(to + t * p.c_stride));
        } else {
#pragma unroll 1
            for (int t0 = 0; t0 < 32; t0 += 4 * kRows) {
                v4u v[4];
#pragma unroll
                for (int s = 0; s < 4; ++s) v[s] = *(const v4u *)(from + (t0 + s * kRows) * kPitch);
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int t = t0 + s * kRows;
                    if (m + t >= p.M) continue;
                    if (n + P <= p.N) {
                        __builtin_memcpy(to + t * p.c_stride, &v[s], 16);
                        continue;
                    }
                    E e[P];
                    __builtin_memcpy(e, &v[s], 16);
#pragma unroll
                    for (int d = 0; d < P; ++d)
                        if (n + d < p.N) to[t * p.c_stride + d] = e[d];
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

template <Num T, int WT>
hipError_t tiled(const ProductArgs &p, hipStream_t stream)
{
    const int tile = 64 * WT, mtiles = (p.M + tile - 1) / tile, ntiles = (p.N + tile - 1) / tile;
    hipLaunchKernelGGL((product_tile_kernel<T, WT>), dim3(mtiles * ntiles), dim3(256), 0, stream, p, mtiles, ntiles);
    return hipGetLastError();
}

// 16 x 16 tiles of C
int64_t small_tiles(int M, int N) { return (int64_t)((M + 15) / 16) * ((N + 15) / 16); }

// Which kernel.  Microseconds measured back to back, float results:
//   - up to 512 tiles of 16 x 16 the chip has room for a workgroup each (1 x 8192 or 300 x 400): a
//     workgroup per tile, its wavefronts share k.  300 x 300 x 512: 3.4, with 32 x 32 tiles 4.4, 128 x 128 6.7.
//   - up to 1536, or 4096 where k is one step, unless k is very long: 32 x 32 tiles.  8000 x 28 x 2048: 6.4
//     (16 x 16 9.7, 128 x 128 9.8), x 4096: 9.9 against 12.9; 300 x 2048 x 512: 7.9 against 6.9; 300 x 1000 x
//     4096: 17.7 against 13.3.
//   - beyond, tiles of 128 or 256 through LDS, by how many rounds of workgroups they take and what a round
//     costs (us, K in numbers): 11 + 0.0075 K for 256 tiles of 256, 4 + 0.0045 K for 512 of 128.
//     2040 x 2048 x 2048: 10.8 with 128, 22.5 with 256; 8000 x 2048 x 4096: 48.7 with 128, 44.7 with 256.
template <Num T>
hipError_t product_typed(const ProductArgs &p, hipStream_t stream)
{
    const int64_t small = small_tiles(p.M, p.N);
    if (small <= 512) return direct<T, false, 1, 1, 4, 4>(p, stream);
    if (small <= (p.K <= 128 ? 4096 : 1536) && small * p.K <= 4500000) return direct<T, false, 2, 2, 4, 4>(p, stream);
    const int64_t large = (int64_t)((p.M + 255) / 256) * ((p.N + 255) / 256);
    const int64_t mid = (int64_t)((p.M + 127) / 128) * ((p.N + 127) / 128);
    const double cost_large = (double)((large + 255) / 256) * (11.0 + 0.0075 * p.K);
    const double cost_mid = std::max(1.0, (double)mid / 512) * (4.0 + 0.0045 * p.K);
    return cost_large < cost_mid ? tiled<T, 4>(p, stream) : tiled<T, 2>(p, stream);
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

// The plain rows are taken to codes where they are multiplied as long as that is not done too often (every
// workgroup of columns does it again) and the operands need not be shared through LDS; else once, into a
// workspace.  Measured (us, float rows, fused against packed): 100 x 28 x 256 4.0 / 7, 100000 x 28 x 1024 86 /
// 107, 8000 x 64 x 1024 11.6 / 13.9, 32000 x 64 x 1024 34 / 32, 2040 x 1024 x 64 7.6 / 8.9 (bfloat16), 8000 x
// 256 x 256 11.9 / 11.3, 8000 x 128 x 1024 19.4 / 15.2, 100 x 4096 x 4096 26 / 16.5 (bfloat16).
bool linear_fused(int M, int N, int K)
{
    const int64_t small = small_tiles(M, N);
    return N <= 32 || small <= 512 || small * K <= (N <= 64 ? 8000000 : 2000000);
}

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
    if (linear_fused(M, N, K)) return 0;
    return (size_t)M * (mx_code_pitch(Mx::E2M1, K) + mx_scale_pitch(K));
}

namespace {

template <Num T>
hipError_t linear_typed(const ProductArgs &p, void *workspace, hipStream_t stream)
{
    if (linear_fused(p.M, p.N, p.K)) {
        // as above: a workgroup per 16 x 16 tile while there are few, with eight wavefronts along a long k (1 x
        // 4096 x 4096 bfloat16: 6.9 against 8.2); else 64 rows by all of 32 or 64 columns, or 16 rows with the
        // wavefronts along k where it is long (8000 x 64 x 1024: 11.6 against 18.9; x 256: 6.0 against 7.2)
        if (small_tiles(p.M, p.N) <= 512)
            return p.K >= 2048 ? direct<T, true, 1, 1, 8, 8>(p, stream) : direct<T, true, 1, 1, 4, 4>(p, stream);
        if (p.K >= 1024) return direct<T, true, 1, 4, 4, 4>(p, stream);
        return p.N <= 32 ? direct<T, true, 1, 2, 4, 1>(p, stream) : direct<T, true, 1, 4, 4, 1>(p, stream);
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
