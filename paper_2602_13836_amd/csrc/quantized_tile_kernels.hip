// The product of several hidden rows (bfloat16) with an embedding in 8 bits (quantized_rows.h) on the matrix cores, through LDS:
//     out[r, j] = < U[row(j), :], h[r, :] >
// U travels as the bytes it is -- from memory to LDS, from LDS to registers -- and is widened to bfloat16 in front of the matrix
// instruction that takes it (v_cvt_scalef32_pk_bf16_fp8: two codes times a power of two per instruction, exact).
//
// A 16-byte unit of U is 16 values, the operands of two steps of v_mfma_f32_32x32x16_bf16, which take 8 values per lane: so the
// lanes of k-group g read unit 2 q + g of 32 values' worth, use its first half in one step and its second in the next, and h's fragments
// are read to match: in which order a step takes the reduction's elements does not matter as long as both operands agree.
//
// The scales of a tile's rows are brought to LDS once, a byte each.  A row with a NaN scale is remembered and its results are made NaN at
// the end (the conversion takes a scale's exponent bits for a number).
//
// Two main loops, as in the bfloat16 kernels: the ring for up to 64 hidden rows, where the one pass over U bounds the product, and the
// loop of wavefronts that take turns for more, where the matrix cores do.  Measured, 4096 elements: 32 hidden rows by 65536 tokens 48 us
// (5.6 TB/s), 64 by 65536 49, 64 by 128256 112 (4.7 TB/s), 512 by 151936 560 (1.14 PFLOP/s; a
// library product of the same sizes in bfloat16, U twice as large, 698).  Sources are named by 32-bit offsets where these reach, else
// (FAR) by addresses.
#include "quantized_rows.h"
#include "sv_launch.h"

#include "memory_to_lds.h"
#include "tile_epilogue.h"

#include <type_traits>

namespace sv {

namespace {

constexpr int kXcds = 8;
constexpr size_t kLdsBytes = 160 * 1024;

__device__ __forceinline__ bf16x8_t widen_8(uint32_t lo, uint32_t hi, float scale) {
    u32x4 v;
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
    return __builtin_bit_cast(bf16x8_t, v);
}

// bytes of LDS per row of U for its scales: the bytes, and a word that is not zero if one of them is NaN (which also spreads rows over banks)
__host__ __device__ inline int scale_row_bytes(int units) { return (units + 31) / 32 * 4 + 4; }

// where a tile lies
struct Tile {
    int rt;                  // tile of hidden rows
    int64_t first, end;      // items
    int64_t slot;            // of its XCD: consecutive slots are the hidden-row tiles of one item tile
    int tn;                  // items of a tile
    bool any;
};
template <int TM, int TN>
__device__ __forceinline__ Tile find_tile(const QuantizedArgs& a, int balance_cus) {
    Tile t;
    const int64_t n_items = a.n_items_dev ? (int64_t)*a.n_items_dev : a.n_items;
    t.tn = TN;
    if (balance_cus > 0 && n_items > 0) {        // the smallest multiple of 32 with which the list takes as many rounds of workgroups as with TN
        const int64_t rounds = (n_items + (int64_t)TN * balance_cus - 1) / ((int64_t)TN * balance_cus);
        const int64_t lanes32 = (int64_t)32 * balance_cus * rounds;
        t.tn = (int)(32 * ((n_items + lanes32 - 1) / lanes32));
    }
    const int RT = (a.rows + TM - 1) / TM;
    t.slot = blockIdx.x / kXcds;
    t.rt = (int)(t.slot % RT);
    const int64_t it = (t.slot / RT) * kXcds + (blockIdx.x % kXcds);
    t.first = it * t.tn;
    t.end = min(t.first + t.tn, n_items);
    t.any = t.first < n_items;
    return t;
}

// The scales of the tile's rows of U into LDS, a thread per row.  (Rows past the tile's end repeat its last.)
__device__ __forceinline__ void bring_scales(const QuantizedArgs& a, const Tile& t, int rows, unsigned char* lds) {
    const int stride = scale_row_bytes(a.units), words = stride / 4 - 1, blocks = (a.units + 7) / 8;
    for (int i = threadIdx.x; i < rows; i += blockDim.x) {
        const int64_t item = min(t.first + i, t.end - 1);
        const uint32_t* s = reinterpret_cast<const uint32_t*>(a.u_scales + (a.idx ? (int64_t)a.idx[item] : item) * a.ldus);
        uint32_t* to = reinterpret_cast<uint32_t*>(lds + i * stride);
        uint32_t nan = 0u;
        for (int w = 0; w < words; ++w) {
            const uint32_t v = s[w];
            to[w] = v;
#pragma unroll
            for (int b = 0; b < 4; ++b) nan |= w * 4 + b < blocks && ((v >> (8 * b)) & 255u) == 255u ? 1u : 0u;
        }
        to[words] = nan;
    }
}

// element e of the 32 x 32 block (m, n): hidden row 8 (e / 4) + 4 (lane / 32) + e % 4, item lane % 32
template <int WM, int WN>
__device__ __forceinline__ void store_product(const QuantizedArgs& a, const Tile& t, const f32x16_t (&acc)[WM][WN], int row0, int64_t item0,
                                              const unsigned char* scales, int item_in_tile) {
    const int lane = threadIdx.x & 63;
    const int stride = scale_row_bytes(a.units);
#pragma unroll
    for (int n = 0; n < WN; ++n) {
        const int64_t item = item0 + 32 * n + (lane & 31);
        if (item >= t.end) continue;
        const bool nan = *reinterpret_cast<const uint32_t*>(scales + (item_in_tile + 32 * n + (lane & 31)) * stride + stride - 4) != 0u;
#pragma unroll
        for (int m = 0; m < WM; ++m)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int r = row0 + 32 * m + 8 * (e >> 2) + (e & 3) + 4 * (lane >> 5);
                if (r < a.rows) a.out[(int64_t)r * a.out_row_stride + item] = nan ? __builtin_nanf("") : acc[m][n][e];
            }
    }
}

// ---- Up to 64 hidden rows, and short lists of more: TM = 32 WM of them and TN = 32 WN GN items; KS wavefronts share each group of 32 WN items and split every
// slice of 128 values between them (what a wavefront reads of h from LDS is for more items then: with 64 items a wavefront instead of 32, half
// as much), their sums being added up at the end.  A ring of D stages in LDS, D - 1 slices on their way, one barrier per slice: behind
// it everybody has slice s and nobody reads slice s - 1 any more, whose stage takes slice s + D - 1.  Rows of 128 bytes (h's slice as
// two halves), the 16-byte unit u of row r at place u ^ ((r >> 1) & 7).
template <int WM, int WN, int GN, int KS, int D>
struct Ring {
    static constexpr int kWaves = GN * KS, TM = 32 * WM, TN = 32 * WN * GN, kStage = TN * 128 + TM * 256, kPass = 8 * kWaves;
    static constexpr int LB = (TN + kPass - 1) / kPass, LX = 2 * TM / kPass;      // requests per wavefront and slice, 8 rows of 128 bytes each
    static constexpr size_t kBytes = (size_t)D * kStage;
    static_assert(LX * kPass == 2 * TM && kWaves % 2 == 0 && D >= 3, "whole requests for h, a constant swizzle per lane");
    static_assert(kBytes >= (size_t)kWaves * WM * WN * 4096, "the ring holds the wavefronts' sums");
};
template <int WM, int WN, int GN, int KS, int D, bool FAR>
__global__ __launch_bounds__(64 * GN * KS) void quantized_ring_kernel(const QuantizedArgs a, const int balance_cus) {
    using R = Ring<WM, WN, GN, KS, D>;
    constexpr int TM = R::TM, TN = R::TN, kStage = R::kStage, kPass = R::kPass, LB = R::LB, LX = R::LX;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];     // [D][TN rows of U, TM rows of h twice], scales
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
    // its group of items, and its part of every slice (a SIMD's wavefronts, w and w + 4, are of groups 0 and 2 or 1 and 3 of four: in
    // a tile of 160 items each SIMD has 64 or 96 to multiply with, none 128)
    const int wc = wave / KS, kh = wave % KS;
    const Tile t = find_tile<TM, TN>(a, balance_cus);
    if (!t.any) return;
    const int units = a.units, nk = (units + 7) / 8;
    // (workgroups walk the reduction from different slices on: rows a power of two apart put the same offset on the same memory channels)
    const int step = nk % 37 ? 37 : 41, rot = nk >= 8 && !a.plain_order ? (int)((t.slot * step) % nk) : 0;
    auto eff = [&](int s) { const int e = min(s, nk - 1) + rot; return e >= nk ? e - nk : e; };
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const int l8 = lane >> 3;
    const int unit = (lane & 7) ^ ((4 * (wave & 1) + (l8 >> 1)) & 7);
    const char* const base_x = a.h + (int64_t)t.rt * TM * a.ldh;
    const char* const base_u = reinterpret_cast<const char*>(a.idx ? a.U : a.U + t.first * a.ldu);
    LaneSource<FAR> src_x[LX], src_u[LB];
#pragma unroll
    for (int i = 0; i < LX; ++i) {
        const int q = wave + R::kWaves * i, row = 8 * (q % (TM / 8)) + l8, half = q / (TM / 8);
        src_x[i].set(base_x, min(t.rt * TM + row, a.rows - 1) - t.rt * TM, a.ldh, (uint32_t)(half * 128 + unit * 16));
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        const int64_t item = min(t.first + kPass * i + 8 * wave + l8, t.end - 1);
        src_u[i].set(base_u, a.idx ? (int64_t)a.idx[item] : item - t.first, a.ldu, (uint32_t)unit * 16u);
    }
    const i32x4_t buf_x = buffer_of(base_x), buf_u = buffer_of(base_u);
    unsigned char* const scales = smem + R::kBytes;
    const int stride = scale_row_bytes(units);
    f32x16_t acc[WM][WN];
#pragma unroll
    for (int m = 0; m < WM; ++m)
#pragma unroll
        for (int n = 0; n < WN; ++n)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[m][n][e] = 0.f;
    // The slice is four groups of 32 values, two steps each: this wavefront's are groups q0 .. q0 + NQ - 1, steps k0 .. k0 + NK - 1 of them.
    constexpr int NQ = KS >= 4 ? 1 : 4 / KS, NK = KS >= 8 ? 1 : 2;
    static_assert(KS == 2 || KS == 4 || KS == 8, "eight steps");
    const int q0 = KS == 8 ? kh >> 1 : kh * NQ, k0 = KS == 8 ? kh & 1 : 0;
    const int swz = (lane >> 1) & 7;
    const int fx0 = TN * 128 + (lane & 31) * 128 + ((((2 * g) ^ swz) * 16) ^ ((4 * (q0 & 1) + k0) * 16)) + (q0 >> 1) * TM * 128;
    const int fu0 = (wc * 32 * WN + (lane & 31)) * 128 + (((g ^ swz) * 16) ^ (q0 * 32));
    // What lies past the tile's width is neither requested nor multiplied.
    const int my_items = __builtin_amdgcn_readfirstlane(t.tn - wc * 32 * WN);
    const bool none = my_items <= 0;
    const unsigned char* const my_scales = scales + (wc * 32 * WN + (lane & 31)) * stride;
    auto walk = [&](auto mine, auto some) {
        constexpr int MINE = decltype(mine)::value;
        auto request = [&](int s, int stage) {
            const int e = eff(s);
            const uint32_t at = lds0 + (uint32_t)(stage * kStage + wave * 1024);
            const bool cut_u = e * 8 + unit >= units;
#pragma unroll
            for (int i = 0; i + 1 < MINE; i += 2)
                bring<kPass * 128>(src_u[i], src_u[i + 1], cut_u, cut_u, buf_u, (int64_t)e * 128, at + (uint32_t)(i * kPass * 128));
            if constexpr (MINE % 2 == 1) bring(src_u[MINE - 1], cut_u, buf_u, (int64_t)e * 128, at + (uint32_t)((MINE - 1) * kPass * 128));
#pragma unroll
            for (int i = 0; i < LX; ++i) {
                const int half = (wave + R::kWaves * i) / (TM / 8);
                bring(src_x[i], e * 16 + half * 8 + unit >= 2 * units, buf_x, (int64_t)e * 256, at + (uint32_t)(TN * 128 + i * kPass * 128));
            }
        };
#pragma unroll
        for (int i = 0; i < D - 1; ++i) request(i, i);
        bring_scales(a, t, TN, scales);
        int st = 0;
        for (int s = 0; s < nk; ++s) {
            // (lgkmcnt: this wavefront's own reads of slice s - 1, and its scales, are done too)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((D - 2) * (LX + MINE)) : "memory");
            request(s + D - 1, st == 0 ? D - 1 : st - 1);
            if (!none) {                                             // (uniform; the same barriers)
                const unsigned char* base = smem + (size_t)st * kStage;
                float scale[WN];
#pragma unroll
                for (int n = 0; n < WN; ++n) scale[n] = __uint_as_float((uint32_t)my_scales[32 * n * stride + eff(s)] << 23);
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    u32x4 raw[WN];
#pragma unroll
                    for (int n = 0; n < WN; ++n) raw[n] = *reinterpret_cast<const u32x4*>(base + (fu0 ^ (q * 32)) + 32 * n * 128);
#pragma unroll
                    for (int k = 0; k < NK; ++k) {
                        bf16x8_t f[WM];
#pragma unroll
                        for (int m = 0; m < WM; ++m)
                            f[m] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(
                                base + (fx0 ^ ((4 * (q & 1) + k) * 16)) + (q >> 1) * TM * 128 + 32 * m * 128));
#pragma unroll
                        for (int n = 0; n < WN; ++n) {
                            if (decltype(some)::value && 32 * n >= my_items) break;              // uniform
                            const uint32_t lo = NK == 1 && k0 ? raw[n][2] : raw[n][2 * k], hi = NK == 1 && k0 ? raw[n][3] : raw[n][2 * k + 1];
                            const bf16x8_t b = widen_8(lo, hi, scale[n]);
#pragma unroll
                            for (int m = 0; m < WM; ++m) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[m], b, acc[m][n], 0, 0, 0);
                        }
                    }
                }
            }
            st = st == D - 1 ? 0 : st + 1;
        }
    };
    const int live = (t.tn - 8 * wave + kPass - 1) / kPass;          // requests for U: 0 .. LB
    auto of_width = [&](auto some) {
        if (LB >= 4 && live >= 4) walk(std::integral_constant<int, (LB < 4 ? LB : 4)>{}, some);
        else if (LB >= 3 && live == 3) walk(std::integral_constant<int, (LB < 3 ? LB : 3)>{}, some);
        else if (LB >= 2 && live >= 2) walk(std::integral_constant<int, (LB < 2 ? LB : 2)>{}, some);
        else if (live >= 1) walk(std::integral_constant<int, 1>{}, some);
        else walk(std::integral_constant<int, 0>{}, some);
    };
    if (WN > 1 && my_items < 32 * WN) of_width(std::bool_constant<(WN > 1)>{});
    else of_width(std::false_type{});
    // Everybody has read its last slice, and nothing is on its way into the ring any more (slices past the end: requested, never
    // read): the wavefronts' sums go there, [part][group][value][lane], and each of the KS adds up and stores its share of the group's.
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    constexpr int kValues = WM * WN * 16, kShare = kValues / KS;
    float* const sums = reinterpret_cast<float*>(smem);
    if (!none) {
#pragma unroll
        for (int m = 0; m < WM; ++m)
#pragma unroll
            for (int n = 0; n < WN; ++n)
#pragma unroll
                for (int e = 0; e < 16; ++e) sums[((kh * GN + wc) * kValues + (m * WN + n) * 16 + e) * 64 + lane] = acc[m][n][e];
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (none) return;
#pragma unroll 4
    for (int i = 0; i < kShare; ++i) {
        const int v = kh * kShare + i, e = v % 16, n = v / 16 % WN, m = v / (16 * WN);
        float sum = sums[(wc * kValues + v) * 64 + lane];
#pragma unroll
        for (int k = 1; k < KS; ++k) sum += sums[((k * GN + wc) * kValues + v) * 64 + lane];
        const int in_tile = wc * 32 * WN + 32 * n + (lane & 31);
        const int64_t item = t.first + in_tile;
        const int r = t.rt * TM + 32 * m + 8 * (e >> 2) + (e & 3) + 4 * (lane >> 5);
        if (item < t.end && r < a.rows)
            a.out[(int64_t)r * a.out_row_stride + item] =
                *reinterpret_cast<const uint32_t*>(scales + in_tile * stride + stride - 4) != 0u ? __builtin_nanf("") : sum;
    }
}

// ---- More hidden rows: two wavefronts share a SIMD and take turns, a barrier ending every turn: while one multiplies a 16-value step (nothing
// but its MFMAs), the other does its memory work -- widens U's fragment of the step it multiplies next, reads h's fragments of the one
// after, and every other step U's 16 bytes for two steps, and asks for what a later slice needs -- and waits for none of it: what it
// reads is there at the end of its following multiply turn.  The second group (wavefronts 4 .. 7; w and w + 4 share a SIMD) is one turn
// behind the first.
//   Slice s is 64 values: h's 128 bytes of it, and half of the 128 bytes that U's block s / 2 takes.  Two stages each.  A wavefront's requests, in
//   order: at the start U of block 0, h of slices 0 and 1; in slice s: (s even) U of block s / 2 + 1 in turns 0 and 1, h of slice
//   s + 2 in turn 3, into the stage that slice s has been read from.  At the end of its multiply turn 2 h of slice s + 1 has to be there and, for
//   odd s, U of block (s + 1) / 2: even s leaves the LB requests for U outstanding, odd s none.
constexpr int kWaves = 8;
template <int WM, int WN>
constexpr size_t turns_bytes() { return (size_t)2 * (64 * WM + 128 * WN) * 128; }
template <int WM, int WN, bool FAR>
__global__ __launch_bounds__(64 * kWaves) void quantized_turns_kernel(const QuantizedArgs a) {
    constexpr int GN = 4, TM = 64 * WM, TN = 128 * WN, kXStage = TM * 128, kUStage = TN * 128;
    constexpr int LX = TM / 64, LB = TN / 64, LB0 = (LB / 2 + 1) / 2 * 2;
    static_assert(LX % 2 == 0 && LB % 2 == 0, "requests go in pairs");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];     // [2][TN rows of U], [2][TM rows of h], scales
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
    const int wr = wave / GN, wc = wave % GN;
    const Tile t = find_tile<TM, TN>(a, 0);
    if (!t.any) return;
    const int units = a.units, blocks = (units + 7) / 8, nk = 2 * blocks;
    const int RT = (a.rows + TM - 1) / TM, step = RT == 1 ? (blocks % 37 ? 37 : 41) : 1;
    const int rot = blocks >= 8 && !a.plain_order ? (int)((t.slot * step) % blocks) : 0;
    auto eff = [&](int b) { const int e = min(b, blocks - 1) + rot; return e >= blocks ? e - blocks : e; };
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const uint32_t lds_u = lds0 + (uint32_t)wave * 1024u, lds_x = lds_u + 2u * kUStage;
    const int l8 = lane >> 3;
    const int unit = (lane & 7) ^ ((4 * (wave & 1) + (l8 >> 1)) & 7);
    const char* const base_x = a.h + (int64_t)t.rt * TM * a.ldh;
    const char* const base_u = reinterpret_cast<const char*>(a.idx ? a.U : a.U + t.first * a.ldu);
    LaneSource<FAR> src_x[LX], src_u[LB];
#pragma unroll
    for (int i = 0; i < LX; ++i) {
        const int row = t.rt * TM + 64 * i + 8 * wave + l8;
        src_x[i].set(base_x, min(row, a.rows - 1) - t.rt * TM, a.ldh, (uint32_t)unit * 16u);
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        const int64_t item = min(t.first + 64 * i + 8 * wave + l8, t.end - 1);
        src_u[i].set(base_u, a.idx ? (int64_t)a.idx[item] : item - t.first, a.ldu, (uint32_t)unit * 16u);
    }
    const i32x4_t buf_x = buffer_of(base_x), buf_u = buffer_of(base_u);
    auto request_x = [&](int s) {
        const int e = 2 * eff(s >> 1) + (s & 1);
        const bool cut = e * 8 + unit >= 2 * units;
#pragma unroll
        for (int i = 0; i < LX; i += 2)
            bring<8192>(src_x[i], src_x[i + 1], cut, cut, buf_x, (int64_t)e * 128, lds_x + (uint32_t)((s & 1) * kXStage + i * 8192));
    };
    auto request_u = [&](int b, int lo, int hi) {
        const int e = eff(b);
        const bool cut = e * 8 + unit >= units;
#pragma unroll
        for (int i = 0; i < LB; i += 2)
            if (i >= lo && i < hi)
                bring<8192>(src_u[i], src_u[i + 1], cut, cut, buf_u, (int64_t)e * 128, lds_u + (uint32_t)((b & 1) * kUStage + i * 8192));
    };
    unsigned char* const scales = smem + turns_bytes<WM, WN>();
    const int stride = scale_row_bytes(units);
    f32x16_t acc[WM][WN];
#pragma unroll
    for (int m = 0; m < WM; ++m)
#pragma unroll
        for (int n = 0; n < WN; ++n)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[m][n][e] = 0.f;
    const int swz = (lane >> 1) & 7;
    const int fx0 = 2 * kUStage + (wr * 32 * WM + (lane & 31)) * 128 + ((2 * g) ^ swz) * 16;
    const int fu0 = (wc * 32 * WN + (lane & 31)) * 128 + (g ^ swz) * 16;
    const unsigned char* const my_scales = scales + (wc * 32 * WN + (lane & 31)) * stride;
    bf16x8_t fx[2][WM], fu[WN];
    u32x4 raw[2][WN];
    float scale[WN], next_scale[WN];
    auto read_x = [&](int stage, int m, bf16x8_t (&F)[WM]) {          // h's fragments of step m of the slice in `stage`
        const unsigned char* p = smem + ((fx0 ^ ((4 * (m >> 1) + (m & 1)) * 16)) + stage * kXStage);
#pragma unroll
        for (int i = 0; i < WM; ++i) F[i] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(p + 32 * i * 128));
    };
    auto read_u = [&](int stage, int q, u32x4 (&F)[WN]) {             // U's 16 bytes of the q-th 32 values of the block in `stage`
        const unsigned char* p = smem + ((fu0 ^ (q * 32)) + stage * kUStage);
#pragma unroll
        for (int n = 0; n < WN; ++n) F[n] = *reinterpret_cast<const u32x4*>(p + 32 * n * 128);
    };
    auto read_scales = [&](int b, float (&S)[WN]) {
        const int e = eff(b);
#pragma unroll
        for (int n = 0; n < WN; ++n) S[n] = __uint_as_float((uint32_t)my_scales[32 * n * stride + e] << 23);
    };
    const bool second = wave >= 4;
    auto turn_ends = [&]() { asm volatile("s_barrier" ::: "memory"); };
    request_u(0, 0, LB);
    request_x(0);
    request_x(1);
    bring_scales(a, t, TN, scales);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LX) : "memory");
    turn_ends();
    read_x(0, 0, fx[0]);
    read_u(0, 0, raw[0]);
    read_scales(0, scale);
    __builtin_amdgcn_s_waitcnt(0xC07F);
    if (second) turn_ends();               // the second group starts one turn later ...
    const int live = __builtin_amdgcn_readfirstlane((a.rows - (t.rt * TM + wr * 32 * WM) + 31) / 32);     // its groups of 32 hidden rows that are any
    auto walk = [&](auto some) {
        for (int s0 = 0; s0 < nk; s0 += 2) {
            static_for<0, 2>([&](auto hc) {
                constexpr int h = decltype(hc)::value;               // which half of the block
                const int b = s0 >> 1, su = b & 1;
                static_for<0, 4>([&](auto mc) {
                    constexpr int m = decltype(mc)::value;
                    // memory turn
#pragma unroll
                    for (int n = 0; n < WN; ++n) fu[n] = widen_8(raw[m >> 1][n][2 * (m & 1)], raw[m >> 1][n][2 * (m & 1) + 1], scale[n]);
                    if constexpr (m < 3) read_x(h, m + 1, fx[(m + 1) & 1]);
                    else read_x(h ^ 1, 0, fx[0]);
                    if constexpr (m == 1) read_u(su, 2 * h + 1, raw[1]);
                    if constexpr (m == 3) {
                        if constexpr (h == 0) {
                            read_u(su, 2, raw[0]);
                        } else {
                            read_u(su ^ 1, 0, raw[0]);
                            read_scales(b + 1, next_scale);
                        }
                    }
                    if constexpr (h == 0 && m == 0) request_u(b + 1, 0, LB0);
                    if constexpr (h == 0 && m == 1) request_u(b + 1, LB0, LB);
                    if constexpr (m == 3) request_x(s0 + h + 2);
                    if constexpr (m == 2) {
                        __builtin_amdgcn_s_waitcnt(0xC07F);          // the slice's last reads: done before this turn ends
                        if (second) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(h == 0 ? LB : 0) : "memory");
                    }
                    turn_ends();
                    // multiply turn
                    __builtin_amdgcn_s_setprio(1);
#pragma unroll
                    for (int i = 0; i < WM; ++i) {
                        if (decltype(some)::value && i >= live) break;           // uniform
#pragma unroll
                        for (int n = 0; n < WN; ++n)
                            acc[i][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[m & 1][i], fu[n], acc[i][n], 0, 0, 0);
                    }
                    __builtin_amdgcn_s_setprio(0);
                    __builtin_amdgcn_sched_barrier(0);
                    __builtin_amdgcn_s_waitcnt(0xC07F);              // lgkmcnt(0): what the last memory turn read is there
                    if constexpr (m == 2) {
                        if (!second) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(h == 0 ? LB : 0) : "memory");
                    }
                    turn_ends();
                    if constexpr (h == 1 && m == 3) {
#pragma unroll
                        for (int n = 0; n < WN; ++n) scale[n] = next_scale[n];
                    }
                });
            });
        }
    };
    if (live >= WM) walk(std::false_type{});
    else walk(std::true_type{});           // (the same turns, and as many)
    if (!second) turn_ends();              // ... and the first ends one turn earlier: the same count for all
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                 // (slices past the end: requested, never read)
    turn_ends();
    store_product<WM, WN>(a, t, acc, t.rt * TM + wr * 32 * WM, t.first + wc * 32 * WN, scales, wc * 32 * WN);
}

// 32-bit offsets reach: from a tile's first row for a whole matrix, from the matrix itself for rows by list
bool near(const QuantizedArgs& a) {
    constexpr int64_t kSpan = (int64_t)kBufferBytes;
    if (256 * a.ldh > kSpan || 256 * a.ldu > kSpan) return false;
    return a.idx == nullptr || a.u_rows <= kSpan / a.ldu;
}

template <class F>
hipError_t opt_in(F* kernel) {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLdsBytes);
}

// the rings: tiles of 32, 64, 128 and 256 items, by 32 or 64 hidden rows (and 96, by 128 items)
template <int WM, int TN>
struct RingOf;
template <int WM>
struct RingOf<WM, 32> { static constexpr int WN = 1, GN = 1, KS = 8, D = WM == 1 ? 8 : 6; };
template <int WM>
struct RingOf<WM, 64> { static constexpr int WN = 1, GN = 2, KS = 4, D = 6; };
template <int WM>
struct RingOf<WM, 128> { static constexpr int WN = 2, GN = 2, KS = 4, D = WM == 1 ? 6 : 4; };
template <int WM>
struct RingOf<WM, 256> { static constexpr int WN = 2, GN = 4, KS = 2, D = 3; };
template <>
struct RingOf<3, 128> { static constexpr int WN = 1, GN = 4, KS = 2, D = 3; };
template <int WM, int TN, bool FAR>
constexpr auto ring_kernel() {
    using P = RingOf<WM, TN>;
    return &quantized_ring_kernel<WM, P::WN, P::GN, P::KS, P::D, FAR>;
}
template <int WM, int TN>
size_t ring_lds(const QuantizedArgs& a) {
    using P = RingOf<WM, TN>;
    return Ring<WM, P::WN, P::GN, P::KS, P::D>::kBytes + (size_t)TN * scale_row_bytes(a.units);
}
template <int WM, int WN>
bool turns_fit(const QuantizedArgs& a) { return turns_bytes<WM, WN>() + (size_t)128 * WN * scale_row_bytes(a.units) <= kLdsBytes; }

// workgroups: item tiles of every XCD rounded up, times tiles of hidden rows
template <class K>
hipError_t launch(K kernel_near, K kernel_far, const QuantizedArgs& a, int tm, int tn, int balance_cus, int threads, size_t lds, hipStream_t stream) {
    const int64_t RT = (a.rows + tm - 1) / tm;
    int64_t IT = (a.n_items + tn - 1) / tn;
    if (balance_cus > 0) IT = (IT + balance_cus - 1) / balance_cus * balance_cus;
    const int64_t bx = (IT + kXcds - 1) / kXcds * RT * kXcds;
    if (bx * threads >= (int64_t)1 << 32) return hipErrorInvalidValue;      // (the runtime would take the low 32 bits)
    K kernel = near(a) ? kernel_near : kernel_far;
    if constexpr (std::is_same<K, void (*)(QuantizedArgs, int)>::value)
        hipLaunchKernelGGL(kernel, dim3((unsigned)bx), dim3(threads), lds, stream, a, balance_cus);
    else
        hipLaunchKernelGGL(kernel, dim3((unsigned)bx), dim3(threads), lds, stream, a);
    return hipGetLastError();
}
template <int TN>
hipError_t launch_ring(const QuantizedArgs& a, int balance_cus, hipStream_t stream) {
    using K = void (*)(QuantizedArgs, int);
    // (more rows than 64: in tiles of 64)
    return a.rows <= 32 ? launch<K>(ring_kernel<1, TN, false>(), ring_kernel<1, TN, true>(), a, 32, TN, balance_cus, 512, ring_lds<1, TN>(a), stream)
                        : launch<K>(ring_kernel<2, TN, false>(), ring_kernel<2, TN, true>(), a, 64, TN, balance_cus, 512, ring_lds<2, TN>(a), stream);
}
template <int WM, int WN>
hipError_t launch_turns(const QuantizedArgs& a, hipStream_t stream) {
    return launch<void (*)(QuantizedArgs)>(&quantized_turns_kernel<WM, WN, false>, &quantized_turns_kernel<WM, WN, true>, a, 64 * WM, 128 * WN, 0,
                                           64 * kWaves, turns_bytes<WM, WN>() + (size_t)128 * WN * scale_row_bytes(a.units), stream);
}

}  // namespace

hipError_t configure_quantized_tile_lds() {
    hipError_t e = hipSuccess;
    auto both = [&](auto* near_kernel, auto* far_kernel) {
        if (e == hipSuccess) e = opt_in(near_kernel);
        if (e == hipSuccess) e = opt_in(far_kernel);
    };
    both(ring_kernel<1, 32, false>(), ring_kernel<1, 32, true>());
    both(ring_kernel<1, 64, false>(), ring_kernel<1, 64, true>());
    both(ring_kernel<1, 128, false>(), ring_kernel<1, 128, true>());
    both(ring_kernel<1, 256, false>(), ring_kernel<1, 256, true>());
    both(ring_kernel<2, 32, false>(), ring_kernel<2, 32, true>());
    both(ring_kernel<2, 64, false>(), ring_kernel<2, 64, true>());
    both(ring_kernel<2, 128, false>(), ring_kernel<2, 128, true>());
    both(ring_kernel<2, 256, false>(), ring_kernel<2, 256, true>());
    both(ring_kernel<3, 128, false>(), ring_kernel<3, 128, true>());
    both(&quantized_turns_kernel<2, 1, false>, &quantized_turns_kernel<2, 1, true>);
    both(&quantized_turns_kernel<2, 2, false>, &quantized_turns_kernel<2, 2, true>);
    both(&quantized_turns_kernel<4, 2, false>, &quantized_turns_kernel<4, 2, true>);
    return e;
}

// True if one of these kernels can: the scales of a tile's rows have to fit into LDS beside its slices.
bool quantized_tile_supported(const QuantizedArgs& a) {
    return a.rows > 64 ? turns_fit<4, 2>(a) : ring_lds<2, 64>(a) <= kLdsBytes && ring_lds<2, 128>(a) <= kLdsBytes && ring_lds<1, 128>(a) <= kLdsBytes;
}

hipError_t launch_quantized_tile(const QuantizedArgs& a, hipStream_t stream) {
    DeviceInfo di;
    const hipError_t e = device_info(&di);
    if (e != hipSuccess) return e;
    if (a.rows <= 64) {
        // The narrowest tiles that fill no more than a round.  4096 elements, 48 hidden rows: 8192 items 16.4 us in tiles of 32, 18.5 of 64, 23.7 of 128; 16384
        // 29.3, 19.6, 23.9 and (256) 24.5; 32768 54.6, 35.9, 28.6 and 29.2; 40000 67.9, 51.5, 48.1 and 33.7.
        const int64_t cus = di.cus;
        if (a.n_items <= 32 * cus) return launch_ring<32>(a, 0, stream);
        if (a.n_items <= 64 * cus) return launch_ring<64>(a, 0, stream);
        // (from 8192 elements on, the scales of 256 items do not fit beside their slices: more rounds of 128)
        if (a.n_items <= 128 * cus || ring_lds<2, 256>(a) > kLdsBytes) return launch_ring<128>(a, 0, stream);
        return launch_ring<256>(a, di.cus, stream);
    }
    // Lists so short that tiles of 64 hidden rows by 64 or 128 items, or 96 by 128, fill no more than a round of workgroups: the ring, which
    // splits the slices among its wavefronts, is done with 4096 elements in 18 to 21, 27 to 30 and 36 to 37 us, the alternating loop in 43
    // to 52 whatever the list's length.  (In a second round it takes as long again: 96 rows x 65536 items, 74 us and 67.)
    auto one_round = [&](int tm, int tn) { return ((int64_t)a.rows + tm - 1) / tm * ((a.n_items + tn - 1) / tn) <= di.cus; };
    if (ring_lds<2, 128>(a) <= kLdsBytes && ring_lds<3, 128>(a) <= kLdsBytes) {
        if (one_round(64, 64)) return launch_ring<64>(a, 0, stream);
        if (one_round(64, 128)) return launch_ring<128>(a, 0, stream);
        if (one_round(96, 128))
            return launch<void (*)(QuantizedArgs, int)>(ring_kernel<3, 128, false>(), ring_kernel<3, 128, true>(), a, 96, 128, 0, 512,
                                                        ring_lds<3, 128>(a), stream);
    }
    switch (tile_shape(a.rows, a.n_items, di.cus, false)) {
        case TILE_128x128: return launch_turns<2, 1>(a, stream);
        case TILE_128x256: return launch_turns<2, 2>(a, stream);
        default: return launch_turns<4, 2>(a, stream);
    }
}

}  // namespace sv
