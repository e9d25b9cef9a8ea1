// chunk_common.hpp -- what the kernels on chunks of new tokens share: arguments,
// the search for a workgroup's sequence, and the operands of their matrix products.
//
// A chunk's query heads of one KV head are its rows: row r of sequence b is query
// head h*G + r % G of new token r / G (G query heads per KV head), at position
// p = seq_len[b] + r / G.
//
// Scores q . k_hat with k_hat = s c + z per group of 32 dims, on
// v_mfma_f32_16x16x32_f16, whose 32-element depth is one group.  The codes c enter as
// fp16 denormals (value c 2^-24, the code's own bits; see key_unit), exactly; their
// group sums are weighted by 2^15 s in fp32.  A row of q is scaled by the power of two 2^e that
// brings its largest element to [2^13, 2^14), exactly, so that all terms have the unit
// 2^(e-9):
//   sum_g (2^15 s_g) (2^-24 sum_d c_d q_d 2^e) + sum_g z_g (2^(e-9) sum_d q_d)
// The second sum is one more product of the same kind over the token's eight
// metadata halfs as they lie in the page ({s, z} of four groups), against the row's
// group sums as fp16 high and low parts (2^-22 relative).  So a logit's error is fp32's;
// keys rounded to fp16 would move logits by 4e-4 (keys N(0, 1), four channels
// times 10), and the normalizers with them.
#pragma once

#include <utility>

#include "internal.hpp"

namespace dkv {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr float kChunkLog2e = 1.4426950408889634f;
constexpr float kChunkLog2eRest = 1.925963034e-08f;  // log2(e) less that
constexpr float kChunkLn2 = 0.6931471805599453f;
constexpr float kLowest = -1e30f;  // a running max before the first key (finite: no inf - inf; below all scores)

// The operands are named once more after the product: the compiler would otherwise place a result over an
// operand that ends there, and what the hardware does then is not relied on.
__device__ __forceinline__ f4 mfma_k32(h8 a, h8 b, f4 c)
{
    f4 d = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    asm("" : "+v"(d) : "v"(a), "v"(b));
    return d;
}
__device__ __forceinline__ f4 mfma_k16(h4 a, h4 b, f4 c)
{
    f4 d = __builtin_amdgcn_mfma_f32_16x16x16f16(a, b, c, 0, 0, 0);
    asm("" : "+v"(d) : "v"(a), "v"(b));
    return d;
}

// ---- loads -----------------------------------------------------------------------
// Through a buffer resource: a uniform base and 32-bit offsets.  (With 64-bit addresses the
// compiler keeps one per lane and piece of a page across the loops.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t span(const void* base, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
// The lane number where the compiler cannot see that it is the same every time: what is worked out
// from it is worked out there, not kept in registers across a loop that has none to spare.
__device__ __forceinline__ int fresh(int lane)
{
    asm volatile("" : "+v"(lane));
    return lane;
}
template <int BYTES>  // 4, 8 or 16
__device__ __forceinline__ auto fetch(__amdgpu_buffer_rsrc_t r, int lane_offset, int offset)
{
    if constexpr (BYTES == 16) return __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(r, lane_offset, offset, 0));
    else if constexpr (BYTES == 8) return __builtin_bit_cast(u2, __builtin_amdgcn_raw_buffer_load_b64(r, lane_offset, offset, 0));
    else return (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(r, lane_offset, offset, 0);
}

// ---- a table's sections ------------------------------------------------------------
// Section lengths as the kernels use them: no length leads out of the table's row.  The high section's
// pages are at most its slots, the low section's at most those that the high one leaves.
struct SecLens {
    int hi, lo;
};
template <int LI>
__device__ __forceinline__ SecLens section_lens(const ChunkArgs& a, int t)
{
    constexpr unsigned Th = kLayoutFmts[LI].hi.T, Tl = kLayoutFmts[LI].lo.T;
    const unsigned P = (unsigned)a.p_max;
    const unsigned hi = (unsigned)max(a.len[2 * t], 0), lo = (unsigned)max(a.len[2 * t + 1], 0);
    const unsigned ph = min((hi + Th - 1) / Th, P), pl = min((lo + Tl - 1) / Tl, P - ph);
    return SecLens{(int)min(hi, ph * Th), (int)min(lo, pl * Tl)};
}

// ---- the sequence and row block of a workgroup --------------------------------
struct SeqBlock {
    int b, n;        // sequence, its new tokens (0: none of this launch's)
    int blk;         // row block inside the sequence
    long long row0;  // its first token row
};

// New tokens of sequence b, clamped to [0, max_new].
__device__ __forceinline__ int new_tokens(const ChunkArgs& a, int b)
{
    const int n = a.new_len[b];
    return n < 0 ? 0 : (n > a.max_new ? a.max_new : n);
}

// Number of row blocks that this launch takes of a sequence of n new tokens: those
// whose rows lie in [lo, hi].
__device__ __forceinline__ int chunk_blocks(int n, int G, int rows, int lo, int hi)
{
    const long long r = (long long)n * G;
    return r < lo || r > hi ? 0 : (int)((r + rows - 1) / rows);
}

// Block number `want` in sequence order.  Every wave finds it by itself: 64 lengths at
// a time, two prefix sums.  Lengths are clamped to [0, max_new] and to total_new rows.
__device__ __forceinline__ SeqBlock find_block(const ChunkArgs& a, int want, int rows, int lo, int hi)
{
    SeqBlock s{-1, 0, 0, 0};
    const int lane = lane_id();
    const int G = a.Hq / a.Hkv;
    long long row = 0;
    int blocks = 0;
    for (int b0 = 0; b0 < a.B; b0 += kWave) {
        const int b = b0 + lane;
        int n = b < a.B ? new_tokens(a, b) : 0;
        const long long before = row + (wave_incl_scan_wide(n) - n);
        const long long room = a.total_new - before;
        if (n > room) n = room > 0 ? (int)room : 0;
        const int nb = chunk_blocks(n, G, rows, lo, hi);
        const int incl = wave_incl_scan(nb);
        const unsigned long long past = __ballot(blocks + incl > want);
        if (past) {
            const int l = __builtin_ctzll(past);
            s.b = b0 + l;
            s.n = __builtin_amdgcn_readlane(n, l);
            s.blk = want - blocks - __builtin_amdgcn_readlane(incl - nb, l);
            s.row0 = read_lane<long long>(before, l);
            return s;
        }
        blocks += __builtin_amdgcn_readlane(incl, kWave - 1);
        row = read_lane<long long>(before + n, kWave - 1);
    }
    return s;
}

// The first 64 sequences', a lane each: asked for before a workgroup knows its sequence, they are there
// when it does (a step's single tokens of up to 64 sequences: 1 us of 47).
__device__ __forceinline__ int first_tokens(const ChunkArgs& a)
{
    const int lane = lane_id();
    return lane < a.B ? new_tokens(a, lane) : 0;
}
// First row and length of sequence s.b (clamped as there); every wave by itself, its lanes each adding
// every 64th sequence's, so that no load waits for another.
__device__ __forceinline__ void sequence_rows(const ChunkArgs& a, SeqBlock& s, int first_n)
{
    const int lane = lane_id();
    long long sum = lane < s.b ? first_n : 0;
#pragma unroll 4
    for (int i = lane + kWave; i < s.b; i += kWave) sum += new_tokens(a, i);
    const int n = s.b < kWave ? __builtin_amdgcn_readlane(first_n, s.b) : new_tokens(a, s.b);
    s.row0 = read_lane<long long>(wave_incl_scan_wide(sum), kWave - 1);
    const long long room = a.total_new - s.row0;
    s.n = n <= room ? n : (room > 0 ? (int)room : 0);
}

// ---- split rows, joined inside the launch -----------------------------------------
// A row block whose steps are split over workgroups: each writes its rows' states {acc[kD], max,
// sum} to its slot with agent-scope stores (through to memory: the workgroups may be on
// different XCDs), and the one that arrives last reads them all back.
// Sixteen bytes of a state with agent scope (cache policy bit 4 is sc1: past the XCD's L2).
__device__ __forceinline__ void put_quad(__amdgpu_buffer_rsrc_t r, int lane_offset, int offset, f4 x)
{
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, x), r, lane_offset, offset, 16);
}
__device__ __forceinline__ f4 get_quad(__amdgpu_buffer_rsrc_t r, int lane_offset, int offset)
{
    return __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(r, lane_offset, offset, 16));
}
// After the workgroup's stores: whether it is the last of `splits` (uniform).
__device__ __forceinline__ bool split_last(unsigned long long* word, int splits, int* lds_flag)
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) *lds_flag = arrive_count(word, call_tag()) == (unsigned long long)splits;
    __syncthreads();
    return *lds_flag != 0;
}

// ---- operands ---------------------------------------------------------------------
// max and sum over the four 16-lane rows, in every row
__device__ __forceinline__ float rows_max(float v)
{
    auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
    x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ __forceinline__ float rows_sum(float v)
{
    auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

// eight key codes (8 bits: two dwords; 4 bits: one) -> fp16 denormals in order.  Codes of 4 bits stand four
// bits higher, 2^-20 c: a matrix product aligns its terms by their exponents alone and cuts them off 2^-24
// below, so small denormals would lose what their leading zeros take (4e-5 of a probability, measured).
template <int KB>
constexpr float key_unit() { return KB == 4 ? 1.0f / 16 : 1.0f; }
__device__ __forceinline__ h8 key_codes8(uint32_t lo, uint32_t hi)
{
    u4 r;
    r[0] = __builtin_amdgcn_perm(0u, lo, 0x0C010C00u);
    r[1] = __builtin_amdgcn_perm(0u, lo, 0x0C030C02u);
    r[2] = __builtin_amdgcn_perm(0u, hi, 0x0C010C00u);
    r[3] = __builtin_amdgcn_perm(0u, hi, 0x0C030C02u);
    return __builtin_bit_cast(h8, r);
}
__device__ __forceinline__ h8 key_codes4(uint32_t w)
{
    const uint32_t even = (w << 4) & 0xF0F0F0F0u, odd = w & 0xF0F0F0F0u;
    u4 r;
    r[0] = __builtin_amdgcn_perm(odd, even, 0x0C040C00u);
    r[1] = __builtin_amdgcn_perm(odd, even, 0x0C050C01u);
    r[2] = __builtin_amdgcn_perm(odd, even, 0x0C060C02u);
    r[3] = __builtin_amdgcn_perm(odd, even, 0x0C070C03u);
    return __builtin_bit_cast(h8, r);
}

// A row of q (this lane's eight dims of each group, lanes l, l + 16, l + 32, l + 48 hold the
// row): its operands scaled by 2^e, the group sums' operand, and 2^(9-e).
struct RowOperands {
    h8 q[kNG];
    h8 sums;      // row-quarter 0: {0, hi_g} pairs, quarter 1: {0, lo_g}, else 0
    float unit;   // 2^(9-e)
};
__device__ __forceinline__ RowOperands row_operands(const u4 (&x)[kNG], int quarter)
{
    RowOperands o;
    uint32_t top = 0;
#pragma unroll
    for (int g = 0; g < kNG; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t m = x[g][i] & 0x7fff7fffu;
            const uint32_t a = m & 0xffffu, b = m >> 16;
            top = top > a ? top : a;
            top = top > b ? top : b;
        }
    {
        uint32_t v = (uint32_t)__shfl_xor((int)top, 16);
        top = top > v ? top : v;
        v = (uint32_t)__shfl_xor((int)top, 32);
        top = top > v ? top : v;
    }
    int e = 28 - (int)(top >> 10);
    e = e > 15 ? 15 : e;  // (an infinite or NaN row: -3)
    const _Float16 up = __builtin_bit_cast(_Float16, (unsigned short)((e + 15) << 10));
    o.unit = __uint_as_float((uint32_t)(127 + 9 - e) << 23);
    const h2 up2 = {up, up};
    u4 sums = {0, 0, 0, 0};
#pragma unroll
    for (int g = 0; g < kNG; ++g) {
        u4 y;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const h2 v = __builtin_bit_cast(h2, (uint32_t)x[g][i]) * up2;
            s += (float)v.x + (float)v.y;
            y[i] = __builtin_bit_cast(uint32_t, v);
        }
        o.q[g] = __builtin_bit_cast(h8, y);
        s = rows_sum(s) * 0x1p-9f;
        const _Float16 hi = (_Float16)s;
        const _Float16 lo = (_Float16)(s - (float)hi);
        const uint32_t bits = __builtin_bit_cast(unsigned short, quarter == 0 ? hi : lo);
        sums[g] = quarter < 2 ? bits << 16 : 0u;
    }
    o.sums = __builtin_bit_cast(h8, sums);
    return o;
}

// ---- the forms of a score --------------------------------------------------------
// sm_scale q.k capped by cap tanh(x / cap), with slope (c - p) added, in natural units (a slope or
// a normalizer times log2(e) would be rounded where a score is still far from its row's
// largest: 2^-24 of biases of 40 and more).
struct ScoreForm {
    float cap_in, cap;  // 2 log2(e) / cap; 0: no cap
    float slope;        // 0: none
};
__device__ __forceinline__ float formed(float x, const ScoreForm& f, float away)
{
    if (f.cap_in != 0.0f) {
        // With t = 2 log2(e) x / cap: below |x| = 5/8 cap x + x t^2 Q(t^2), Q a Chebyshev fit of degree 4
        // (2^-23 of the result: 1 - 2 / (1 + exp) alone would leave 2^-23 of the cap, 10^-6 of a score's
        // probability at caps of 30); above it, where a wave has any, 1 - 2 e / (1 + e), e = 2^-|t|.
        const float t = x * f.cap_in, u = t * t;
        float y = __builtin_fmaf(u, -1.5262884e-7f, 4.3717801e-6f);
        y = __builtin_fmaf(y, u, -9.3320843e-5f);
        y = __builtin_fmaf(y, u, 1.9235463e-3f);
        y = __builtin_fmaf(y, u, -4.0037747e-2f);
        y = __builtin_fmaf(x, u * y, x);
        if (!(fabsf(t) < 1.8f)) {
            const float e = __builtin_amdgcn_exp2f(-fabsf(t));
            y = __builtin_copysignf(__builtin_fmaf(-f.cap, 2.0f * e * __builtin_amdgcn_rcpf(1.0f + e), f.cap), x);
        }
        x = y;
    }
    return __builtin_fmaf(-f.slope, away, x);
}

}  // namespace dkv
