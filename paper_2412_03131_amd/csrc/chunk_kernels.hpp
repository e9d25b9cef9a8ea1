// chunk_kernels.hpp -- attention and scores of chunks of new tokens over the
// differentiated paged cache, templated on the page layout (k_chunk_l<n>.hip).
#pragma once

#include "chunk_common.hpp"

namespace dkv {

// A step is 32 tokens: two tiles of 16.  Row m of tile t is token slot
//   pages of 16 tokens: slot m of the step's page t;
//   pages of 32 tokens and the chunk's own tokens: slot 8 (m / 4) + 4 t + m % 4,
// so that the tokens of result rows 4 quarter .. + 3 of both tiles are, for a lane, whole bytes
// of a dimension's value codes.
template <int T>
__device__ __forceinline__ int step_slot(int t, int m)
{
    return T == 16 ? m : 8 * (m >> 2) + 4 * t + (m & 3);
}

// ---- pages through LDS ------------------------------------------------------------
// A wave stages a step's pages in a slot of its own with loads that have an LDS destination: the
// page's bytes as they lie, 1 KB a load, no registers held while they are in flight.  The
// buffer resource ends with the bytes that are needed (beyond, the loads fetch nothing).
template <int KB, int VB, int T, bool MOD>
struct Staged {
    static constexpr SecOffsets O = sec_offsets(KvFmt{KB, VB, T});
    static constexpr int need = MOD ? O.used : O.sc;
    static constexpr int loads = (need + 1023) / 1024;
    static constexpr int page = loads * 1024;
    static constexpr int slot = (T == 16 ? 2 : 1) * page;
};

template <int NEED>
__device__ __forceinline__ void stage_page(uint8_t* lds, const uint8_t* pg, int lane)
{
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(__attribute__((address_space(3))) void*)lds);
    const unsigned long long base = (unsigned long long)pg;
    const u4 rs = {(uint32_t)base, (uint32_t)(base >> 32) & 0xffffu, (uint32_t)NEED, 0x00020000u};
#pragma unroll
    for (int i = 0; i < (NEED + 1023) / 1024; ++i)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(at + 1024 * i),
                     "v"(lane * 16), "s"(rs), "s"(1024 * i)
                     : "memory");
}
// One KB of a page (piece i), by one wave.
__device__ __forceinline__ void stage_piece(uint8_t* lds, const uint8_t* pg, int need, int i, int lane)
{
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(__attribute__((address_space(3))) void*)lds) + 1024 * i;
    const unsigned long long base = (unsigned long long)pg;
    const u4 rs = {(uint32_t)base, (uint32_t)(base >> 32) & 0xffffu, (uint32_t)need, 0x00020000u};
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(at), "v"(lane * 16), "s"(rs),
                 "s"(1024 * i)
                 : "memory");
}
// Four rows of 256 bytes, `stride` bytes apart from `base` on, rows beyond `last` read as the last.
__device__ __forceinline__ void stage_rows(uint8_t* lds, const void* base, int stride, int row, int last, int lane)
{
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(__attribute__((address_space(3))) void*)lds);
    const unsigned long long b = (unsigned long long)base;
    const u4 rs = {(uint32_t)b, (uint32_t)(b >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at),
                 "v"(min(row + (lane >> 4), last) * stride + (lane & 15) * 16), "s"(rs)
                 : "memory");
}
// (the wave's only vector loads in flight are its slot's)
__device__ __forceinline__ void staged_ready() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// Keeps the reads of a slot where they are written: all of a step's at once need more registers than
// four waves per SIMD have.
__device__ __forceinline__ void keep_order() { asm volatile("" ::: "memory"); }
__device__ __forceinline__ void staged_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// What a lane (column c = lane % 16, quarter = lane / 16) takes of a step.
template <int KB>
struct TileKeys {
    uint32_t kc[kNG][KB / 4];  // key codes of token m = c, its quarter of each group
    u4 km;                     // its {s, z} of four groups
    int4 pos;                  // positions of the quarter's four tokens
};
// Of one group of its values (dims 32 g .. + 31: two 16-dim tiles).
template <int VB, int T>
struct GroupValues {
    static constexpr int kPieces = T == 16 ? 2 : 1;  // value code pieces per dim: one per page
    uint32_t vc[kPieces][2];      // value codes of dims 32 g + 16 d + c, the quarter's tokens
    u4 vm[2];                     // {s, z} of the quarter's four tokens
};

template <int VB, int T>
__device__ __forceinline__ uint32_t load_value_codes(const uint8_t* p)
{
    constexpr int bytes = (T == 16 ? 4 : 8) * VB / 8;
    if constexpr (bytes == 4) return *reinterpret_cast<const uint32_t*>(p);
    else if constexpr (bytes == 2) return *reinterpret_cast<const uint16_t*>(p);
    else return *p;
}

template <int KB, int VB, int T, bool MOD>
__device__ __forceinline__ void load_keys(TileKeys<KB>& r, const uint8_t* slot_, int t, int c, int quarter)
{
    constexpr SecOffsets O = sec_offsets(KvFmt{KB, VB, T});
    const uint8_t* pg = slot_ + (T == 16 ? t * Staged<KB, VB, T, MOD>::page : 0);
    const int slot = step_slot<T>(t, c);
#pragma unroll
    for (int g = 0; g < kNG; ++g) {
        if constexpr (KB == 8) {
            const u2 v = *reinterpret_cast<const u2*>(pg + O.kc + ((2 * g + (quarter >> 1)) * T + slot) * 16 + (quarter & 1) * 8);
            r.kc[g][0] = v[0];
            r.kc[g][1] = v[1];
        } else {
            r.kc[g][0] = *reinterpret_cast<const uint32_t*>(pg + O.kc + (g * T + slot) * 16 + quarter * 4);
        }
    }
    r.km = *reinterpret_cast<const u4*>(pg + O.km + slot * 16);
    if constexpr (MOD) r.pos = *reinterpret_cast<const int4*>(pg + O.pos + step_slot<T>(t, 4 * quarter) * 4);
}

template <int KB, int VB, int T, bool MOD>
__device__ __forceinline__ void load_values(GroupValues<VB, T>& r, const uint8_t* slot_, int g, int c, int quarter)
{
    constexpr SecOffsets O = sec_offsets(KvFmt{KB, VB, T});
    constexpr int row = T * VB / 8, piece = (T == 16 ? 4 : 8) * VB / 8;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const uint8_t* pg = slot_ + (T == 16 ? t * Staged<KB, VB, T, MOD>::page : 0);
        r.vm[t] = *reinterpret_cast<const u4*>(pg + O.vm + (g * T + step_slot<T>(t, 4 * quarter)) * 4);
        if (t < GroupValues<VB, T>::kPieces) {
#pragma unroll
            for (int d = 0; d < 2; ++d)
                r.vc[t < GroupValues<VB, T>::kPieces ? t : 0][d] =
                    load_value_codes<VB, T>(pg + O.vc + (32 * g + 16 * d + c) * row + quarter * piece);
        }
    }
}

// Four value codes of a tile (the low 4 VB bits of w) -> half of s c + z as fp16 pairs of tokens
// (0, 2) and (1, 3), z given halved.  A code is read as 1024 + c (its bits under the exponent of
// 1024, exact), the second pair as 1024 + 2^VB c; two packed steps give c / 2 and (s c + z) / 2, the
// only rounding (2^-11: values N(0, 1) of a kept token, far below their own quantization).  Halves,
// because s c + z of a group's largest code can round past the largest finite fp16: infinite are
// then only those that are (a limit per pair would also hide NaN); sums of cached values are doubled once.
// With a second part, as the weights have, results are as exact as a 32-bit computation's rounded once, not 1.15 to
// 1.25 times as far off; but the conversions are most of the few-row kernel's work: 64 single tokens over 1k-4k
// take 46 us so and 68 with two parts, one token of 16 sequences over 32k 108 and 156, parts of eight prompts 419
// and 471, 2048 tokens over 8192 913 and 1044.
template <int VB>
__device__ __forceinline__ void value_pairs(uint32_t w, h2 s02, h2 z02, h2 s13, h2 z13, uint32_t& p02, uint32_t& p13)
{
    const h2 half = {(_Float16)0.5f, (_Float16)0.5f}, m512 = {(_Float16)-512.0f, (_Float16)-512.0f};
    h2 y02, y13;
    if constexpr (VB == 8) {
        y02 = __builtin_elementwise_fma(__builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, 0x04020400u)), half, m512);
        y13 = __builtin_elementwise_fma(__builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030401u)), half, m512);
    } else {
        constexpr uint32_t m = ((1u << VB) - 1) * 0x00010001u;
        const uint32_t x = VB == 4 ? __builtin_amdgcn_perm(0u, w, 0x0C010C00u) : (w | (w << (16 - 2 * VB)));
        const h2 inv = {(_Float16)(0.5f / (1 << VB)), (_Float16)(0.5f / (1 << VB))};
        const h2 off = {(_Float16)(-512.0f / (1 << VB)), (_Float16)(-512.0f / (1 << VB))};
        y02 = __builtin_elementwise_fma(__builtin_bit_cast(h2, (x & m) | 0x64006400u), half, m512);
        y13 = __builtin_elementwise_fma(__builtin_bit_cast(h2, (x & (m << VB)) | 0x64006400u), inv, off);
    }
    p02 = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(s02, y02, z02));
    p13 = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(s13, y13, z13));
}

// The rows a wave works on: 16 RT of them, column c of tile rt is row 16 rt + c of its block.
// Their queries' operands are read from LDS, where the workgroup's waves share them: five
// registers of four a tile would not fit beside the rest.
template <int RT>
struct RowsLds {
    h8 q[RT][kNG][kWave];
    h8 sums[RT][kWave];
};
template <int RT>
struct Rows {
    float unit[RT];   // logit = unit * product sum (log2 units, natural ones with a score form)
    int p[RT];        // position in the sequence
    ScoreForm form[RT];
    float m[RT], l[RT];  // (m: raise_max)
    f4 acc[RT][8];    // O^T: dims 16 dt + 4 quarter + r of row c
};

// One step's scores against the running softmax: sums x[rt][t][r] of tokens (t, 4 quarter + r), a
// logit being unit * x, -> weights 2^(logit - m), with m the running max less 7: a weight enters its
// product as fp16, whose denormals end at 2^-24, so the offset keeps what is 2^-32 of the largest (without it
// everything below 2^-25 was lost from the sums of values, yet counted in the normalizer).  The running max is
// raised only when a logit passes it by 8 (weights up to 2^15; m is rounded, the product it is taken from is not:
// logits up to 2^22 leave them below 2^16).  before() is called where it is, before anything is scaled.
constexpr float kWeightBits = 7.0f, kRaiseBits = 8.0f;
template <int RT, typename F>
__device__ __forceinline__ void raise_max(Rows<RT>& R, const float (&unit)[RT], const float (&x)[RT][2][4], F&& before)
{
    float top[RT];
    bool raise = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        top[rt] = max3(max3(x[rt][0][0], x[rt][0][1], x[rt][0][2]), x[rt][0][3], max3(x[rt][1][0], x[rt][1][1], x[rt][1][2]));
        top[rt] = max3(top[rt], x[rt][1][3], kLowest) * unit[rt];
        raise |= top[rt] > R.m[rt] + (kWeightBits + kRaiseBits);
    }
    if (!__any(raise)) return;
    before();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        top[rt] = fmaxf(R.m[rt], rows_max(top[rt]) - kWeightBits);
        const float f = __builtin_amdgcn_exp2f(R.m[rt] - top[rt]);
        R.m[rt] = top[rt];
        R.l[rt] *= f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) R.acc[rt][dt] *= f;
    }
}
__device__ __forceinline__ float weight(float x, float unit, float m)
{
    return __builtin_amdgcn_exp2f(__builtin_fmaf(x, unit, -m));
}
// weights as fp16 pairs (0, 2), (1, 3) of both tiles
__device__ __forceinline__ h8 pack_weights(const float (&w)[2][4])
{
    u4 bits;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const h2 a = {(_Float16)w[t][0], (_Float16)w[t][2]}, b = {(_Float16)w[t][1], (_Float16)w[t][3]};
        bits[2 * t] = __builtin_bit_cast(uint32_t, a);
        bits[2 * t + 1] = __builtin_bit_cast(uint32_t, b);
    }
    return __builtin_bit_cast(h8, bits);
}
// What the rounding left of them: two parts hold a weight to 2^-22, or to 2^-32 of its row's largest where that
// is more (raise_max).  Weights enter all kernels whole, so a token's precision does not go by which kernel or
// how many row tiles its neighbours in a call ask for.  The results' error against 64 bits is then the
// values' and their own rounding alone, 1.15 to 1.25 times a 32-bit computation's rounded once; with
// weights rounded once it was up to 1.5 times.  The second products take 2 us of 46 for 64 single tokens over
// 1k-4k, 2 % with two row tiles, 15 % in chunk_tiles (257-512 tokens for each of 8 sequences over 0-8192: 367 ->
// 421 us, 2048 tokens over 8192 at 64 / 8 heads: 791 -> 935).
__device__ __forceinline__ h8 pack_rest(const float (&w)[2][4], h8 P)
{
    float rest[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) rest[t][r] = w[t][r] - (float)P[4 * t + 2 * (r & 1) + (r >> 1)];
    return pack_weights(rest);
}
template <int RT>
__device__ __forceinline__ void softmax_step(Rows<RT>& R, const float (&unit)[RT], float (&x)[RT][2][4], h8 (&P)[RT])
{
    raise_max<RT>(R, unit, x, [] {});
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float sum = 0.0f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += x[rt][t][r] = weight(x[rt][t][r], unit[rt], R.m[rt]);
        R.l[rt] += sum;
        P[rt] = pack_weights(x[rt]);
    }
}

// ---- cached values that are not finite ------------------------------------------------
// An infinite or NaN s c + z reaches every row of a matrix product (0 * inf is NaN), which is right while every row sees
// every cached token: only a window hides some.  In windowed calls every step's {s, z} are looked at; a group
// with one that is not finite (or twice the largest half) enters the products as 0, and a piece that met one adds
// its s c + z in fp32 at the end (odd_four), each logit computed anew.
template <int VB>
__device__ __forceinline__ bool odd_group(uint32_t sz)
{
    const h2 m = __builtin_bit_cast(h2, sz);
    return !(fabsf(__builtin_fmaf((float)m.x, (float)((1 << VB) - 1), (float)m.y)) < 131008.0f);
}
// A row (of the chunk's, of table t) and the cached steps u0 .. u1 - 1 that its piece went over.
struct OddRow {
    const ChunkArgs* args;
    int t, row, u0, u1;
    long long row0;  // the sequence's first token row
    float m;         // the row's running max
};
template <int KB, int VB, int T>
__device__ __forceinline__ void odd_section(f4& o, const ChunkArgs& a, const int32_t* table, bool high, int len, int u0, int u1,
                                            const uint16_t* q, int p, const ScoreForm& form, float m, int d)
{
    constexpr SecOffsets O = sec_offsets(KvFmt{KB, VB, T});
#pragma unroll 1
    for (int token = 32 * max(u0, 0); token < min(32 * u1, len); ++token) {
        const int slot = token % T, id = table[high ? token / T : a.p_max - 1 - token / T];
        if ((unsigned long long)(unsigned)id >= (unsigned long long)a.num_pages) continue;
        const uint8_t* pg = a.pool + (long long)id * a.page_bytes;
        const uint32_t sz = *reinterpret_cast<const uint32_t*>(pg + O.vm + ((d >> 5) * T + slot) * 4);
        const int away = p - *reinterpret_cast<const int32_t*>(pg + O.pos + 4 * slot);
        if (!odd_group<VB>(sz) || away >= a.window) continue;
        float x = 0.0f;
#pragma unroll 1
        for (int i = 0; i < kD; ++i) {
            const int code = KB == 8 ? pg[O.kc + ((i >> 4) * T + slot) * 16 + (i & 15)]
                                     : pg[O.kc + ((i >> 5) * T + slot) * 16 + ((i & 31) >> 1)] >> (4 * (i & 1)) & 15;
            const h2 k = *reinterpret_cast<const h2*>(pg + O.km + slot * 16 + (i >> 5) * 4);
            x = __builtin_fmaf(h2f(q[i]), __builtin_fmaf((float)k.x, (float)code, (float)k.y), x);
        }
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(formed(x * a.scale, form, (float)away), kChunkLog2e, -m));
        const h2 v = __builtin_bit_cast(h2, sz);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int byte = pg[O.vc + (d + i) * (T * VB / 8) + slot * VB / 8];
            o[i] += w * __builtin_fmaf((float)v.x, (float)(byte >> (slot * VB % 8) & ((1 << VB) - 1)), (float)v.y);
        }
    }
}
// The sums o of four dims d .. of one group, with what odd groups add.  A function of its own that reads the launch's
// arguments itself: inlined, or given them, it took registers from the loops (drafted tokens 34.6 -> 38 us).
template <int LI>
__device__ __noinline__ f4 odd_four(f4 o, OddRow r, int d)
{
    constexpr KvFmt hi = kLayoutFmts[LI].hi, lo = kLayoutFmts[LI].lo;
    const ChunkArgs& a = *r.args;
    const int G = a.Hq / a.Hkv, b = r.t / a.Hkv, j = r.row / G, hq = (r.t - b * a.Hkv) * G + r.row - j * G;
    const SecLens len = section_lens<LI>(a, r.t);
    const int s_hi = (len.hi + 31) >> 5, p = a.seq_len[b] + j;
    const int32_t* table = a.page_table + (long long)r.t * a.p_max;
    const uint16_t* q = a.q + (r.row0 + j) * a.q_stride + hq * kD;
    const ScoreForm form{a.cap_in, a.cap, a.slopes ? a.slopes[hq] : 0.0f};
    odd_section<hi.kb, hi.vb, hi.T>(o, a, table, true, len.hi, r.u0, r.u1, q, p, form, r.m, d);
    odd_section<lo.kb, lo.vb, lo.T>(o, a, table, false, len.lo, r.u0 - s_hi, r.u1 - s_hi, q, p, form, r.m, d);
    return o;
}
// The launch's arguments where they lie.
__device__ __forceinline__ const ChunkArgs* chunk_args() { return (const ChunkArgs*)__builtin_amdgcn_kernarg_segment_ptr(); }

// A step of cached tokens in the wave's slot; those with index >= left (in the step, by token) and
// those of tile t where bit t of `bad` is set (a page ID outside the pool) do not exist.
// next() is called once the slot has been read.  Whether the step has odd groups (uniform).
template <int KB, int VB, int T, int RT, bool MOD, typename F>
__device__ __forceinline__ bool cached_step(Rows<RT>& R, const RowsLds<RT>& Q, uint8_t* slot, int left, uint32_t bad,
                                            const ChunkArgs& a, int lane, F&& next)
{
    const int c = lane & 15, quarter = lane >> 4;
    float x[RT][2][4];
    const h4 pick0 = {(_Float16)(quarter == 0 ? 0x1p15f * key_unit<KB>() : 0.0f), (_Float16)0.0f, (_Float16)0.0f, (_Float16)0.0f};
    const h4 pick1 = {(_Float16)0.0f, (_Float16)0.0f, (_Float16)(quarter == 0 ? 0x1p15f * key_unit<KB>() : 0.0f), (_Float16)0.0f};
    const f4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        keep_order();
        TileKeys<KB> raw;
        load_keys<KB, VB, T, MOD>(raw, slot, t, c, quarter);
        const h8 meta = __builtin_bit_cast(h8, raw.km);
        const h4 m01 = {meta[0], meta[1], meta[2], meta[3]}, m23 = {meta[4], meta[5], meta[6], meta[7]};
        // 2^15 s (times the codes' unit) of the quarter's four tokens, per group: a product with a unit vector
        f4 s[kNG];
        s[0] = mfma_k16(m01, pick0, zero);
        s[1] = mfma_k16(m01, pick1, zero);
        s[2] = mfma_k16(m23, pick0, zero);
        s[3] = mfma_k16(m23, pick1, zero);
        h8 k[kNG];
#pragma unroll
        for (int g = 0; g < kNG; ++g) {
            if constexpr (KB == 8) k[g] = key_codes8(raw.kc[g][0], raw.kc[g][1]);
            else k[g] = key_codes4(raw.kc[g][0]);
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            f4 sum = mfma_k32(meta, Q.sums[rt][16 * quarter + c], zero);
#pragma unroll
            for (int g = 0; g < kNG; ++g) {
                const f4 part = mfma_k32(k[g], Q.q[rt][g][16 * quarter + c], zero);
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[r] = __builtin_fmaf(s[g][r], part[r], sum[r]);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) x[rt][t][r] = MOD ? sum[r] * R.unit[rt] : sum[r];
        }
        if constexpr (MOD) {
            const int pos[4] = {raw.pos.x, raw.pos.y, raw.pos.z, raw.pos.w};
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int away = R.p[rt] - pos[r];
                    const float y = formed(x[rt][t][r], R.form[rt], (float)away);
                    x[rt][t][r] = away < a.window ? y : -INFINITY;
                }
        }
    }
    bool odd = false;
    if (MOD && a.window != INT32_MAX) {  // a lane looks at {s, z} of two tokens and one group
        constexpr SecOffsets O = sec_offsets(KvFmt{KB, VB, T});
        uint8_t* at = slot + O.vm + (T == 16 ? (lane >> 5) * Staged<KB, VB, T, MOD>::page + 8 * (lane & 31) : 8 * lane);
        const int token = T == 16 ? 16 * (lane >> 5) + 2 * (lane & 7) : 2 * (lane & 15);
        const u2 sz = *reinterpret_cast<const u2*>(at);
        const bool in = !((bad >> (T == 16 ? lane >> 5 : 0)) & 1);
        const bool odd0 = odd_group<VB>(sz[0]) && token < left && in, odd1 = odd_group<VB>(sz[1]) && token + 1 < left && in;
        odd = __any(odd0 || odd1);
        if (__builtin_expect(odd, 0)) *reinterpret_cast<u2*>(at) = u2{odd0 ? 0u : sz[0], odd1 ? 0u : sz[1]};
    }
    uint32_t keep[2] = {0xfu, 0xfu};  // which of the quarter's tokens exist
    const bool whole = left >= 32 && bad == 0;
    if (!whole) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            keep[t] = 0;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool there = (T == 16 ? 16 * t : 0) + step_slot<T>(t, 4 * quarter + r) < left && !((bad >> t) & 1);
                if (there) keep[t] |= 1u << r;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) x[rt][t][r] = there ? x[rt][t][r] : -INFINITY;
            }
        }
    }
    h8 P[RT];
    float unit[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) unit[rt] = MOD ? kChunkLog2e : R.unit[rt];
    softmax_step<RT>(R, unit, x, P);
    h8 rest[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) rest[rt] = pack_rest(x[rt], P[rt]);
#pragma unroll
    for (int g = 0; g < kNG; ++g) {
        keep_order();
        GroupValues<VB, T> val;
        load_values<KB, VB, T, MOD>(val, slot, g, c, quarter);
        if (g == kNG - 1) {
            staged_read();
            next();
        }
        h2 s02[2], z02[2], s13[2], z13[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const u4 m = val.vm[t];
            s02[t] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(m[2], m[0], 0x05040100u));
            z02[t] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(m[2], m[0], 0x07060302u)) * (_Float16)0.5f;
            s13[t] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(m[3], m[1], 0x05040100u));
            z13[t] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(m[3], m[1], 0x07060302u)) * (_Float16)0.5f;
        }
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            const int dt = 2 * g + d;
            u4 v;
            uint32_t p, q;
            value_pairs<VB>(val.vc[0][d], s02[0], z02[0], s13[0], z13[0], p, q);
            v[0] = p;
            v[1] = q;
            value_pairs<VB>(T == 16 ? val.vc[GroupValues<VB, T>::kPieces - 1][d] : val.vc[0][d] >> (4 * VB), s02[1], z02[1],
                            s13[1], z13[1], p, q);
            v[2] = p;
            v[3] = q;
            if (!whole) {  // nothing behind a section's end reaches the sums
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    v[2 * t] &= (keep[t] & 1 ? 0xffffu : 0u) | (keep[t] & 4 ? 0xffff0000u : 0u);
                    v[2 * t + 1] &= (keep[t] & 2 ? 0xffffu : 0u) | (keep[t] & 8 ? 0xffff0000u : 0u);
                }
            }
            const h8 V = __builtin_bit_cast(h8, v);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) R.acc[rt][dt] = mfma_k32(V, P[rt], R.acc[rt][dt]);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) R.acc[rt][dt] = mfma_k32(V, rest[rt], R.acc[rt][dt]);
        }
    }
    return odd;
}

// An infinite or NaN own value must not reach the rows that do not see its token (0 * inf in a matrix
// product): it enters the product as 0 and is added here to those that do.  x: the step's weights.
template <int RT>
__device__ __forceinline__ void odd_values(Rows<RT>& R, const float (&x)[RT][2][4], const uint16_t* v, int i0, int n, int first,
                                           const ChunkArgs& a, int c, int quarter)
{
#pragma unroll 1
    for (int token = 0; token < 32 && i0 + token < n; ++token) {
        float p[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            p[rt] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float pi = __shfl(x[rt][i >> 2][i & 3], c + 16 * (token >> 3));
                p[rt] = (token & 7) == i ? pi : p[rt];
            }
        }
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint32_t w = v[(long long)(i0 + token) * a.v_stride + 16 * dt + 4 * quarter + r];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const int away = R.p[rt] - first - (i0 + token);
                    if ((w & 0x7c00u) == 0x7c00u && away >= 0 && away < a.window) R.acc[rt][dt][r] += p[rt] * h2f(w);
                }
            }
    }
}

// A step of the chunk's own tokens i0 .. i0 + 31 of n, keys at k, values at v (strides in halfs).
// first: position of token 0.
template <int RT, bool MOD>
__device__ __forceinline__ void own_step(Rows<RT>& R, const RowsLds<RT>& Q, const uint16_t* k, const uint16_t* v, int i0, int n, int first,
                                         const ChunkArgs& a, int c, int quarter)
{
    float x[RT][2][4];
    const f4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int i = min(i0 + step_slot<32>(t, c), n - 1);
        const uint16_t* row = k + (long long)i * a.k_stride + quarter * 8;
        u4 raw[kNG];
#pragma unroll
        for (int g = 0; g < kNG; ++g) raw[g] = *reinterpret_cast<const u4*>(row + g * kG);
        f4 sum[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) sum[rt] = zero;
#pragma unroll
        for (int g = 0; g < kNG; ++g) {
            const h8 kk = __builtin_bit_cast(h8, raw[g]);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) sum[rt] = mfma_k32(kk, Q.q[rt][g][16 * quarter + c], sum[rt]);
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int token = i0 + step_slot<32>(t, 4 * quarter + r);
                const int away = R.p[rt] - first - token;
                float y = sum[rt][r] * 0x1p-9f;
                if constexpr (MOD) y = formed(y * R.unit[rt], R.form[rt], (float)away);
                x[rt][t][r] = away >= 0 && away < a.window ? y : -INFINITY;
            }
    }
    h8 P[RT];
    float unit[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) unit[rt] = MOD ? kChunkLog2e : R.unit[rt];
    softmax_step<RT>(R, unit, x, P);
    h8 rest[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) rest[rt] = pack_rest(x[rt], P[rt]);
    // values: the quarter's eight tokens of dims 16 dt + c
    bool odd = false;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
        uint32_t b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int token = i0 + 8 * quarter + i;
            uint32_t w = v[(long long)min(token, n - 1) * a.v_stride + 16 * dt + c];
            const bool bad = (w & 0x7c00u) == 0x7c00u;
            odd |= bad && token < n;
            b[i] = bad || token >= n ? 0u : w;
        }
        // tokens (0, 2), (1, 3) of both tiles, as the weights
        const u4 w = {b[0] | b[2] << 16, b[1] | b[3] << 16, b[4] | b[6] << 16, b[5] | b[7] << 16};
        const h8 V = __builtin_bit_cast(h8, w);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) R.acc[rt][dt] = mfma_k32(V, P[rt], R.acc[rt][dt]);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) R.acc[rt][dt] = mfma_k32(V, rest[rt], R.acc[rt][dt]);
    }
    if (__any(odd)) odd_values<RT>(R, x, v, i0, n, first, a, c, quarter);
}

// ---- attention: few rows, tokens split over waves and workgroups ------------------------
//
// A workgroup takes 16 RT rows of one (sequence, KV head) and its share of the table's steps
// (high pages, low pages, the chunk's own tokens), its four waves every fourth step each.  A
// wave has the transposed result O^T, so the scores of a step come out with a lane's values in
// one row and go into the second product as they lie: no exchange between lanes but the rare raise of
// the running max.  A wave's next step is staged in LDS as soon as the one before has been read from
// there; with four waves per SIMD (two with two row tiles) the others' work covers the rest of its way.
// Bound: 64 sequences' single tokens over 1k-4k (8 KV heads, K8V4 / K4V2, 144 MB of pages) take 46 us, 3.2 TB/s
// against 4.9 of a copy, one token of 16 sequences over 32k with a cap and slopes 109 us at 3.6 TB/s: VALU issue
// (dequantization) and the longest tables' pieces; calls of few tables the chain lengths - page IDs -
// pages - states (12 us over 600 tokens).
constexpr int kChunkWaves = 4;

// The piece of workgroup blockIdx.x: tables in order, a table's row blocks, a block's pieces.  All blocks
// of a table have about one piece per `quantum` steps, the quantum such that all pieces together (a
// table's last is half a quantum on average) are kRowPieces at most, and at least a step for each wave.
constexpr int kRowTables = 1024;  // (more are not split)
struct RowPiece {
    int table, blk, split, splits, block;
};
__device__ __forceinline__ int piece_quantum(const ChunkArgs& a, int total, int blocks)
{
    return max((total + a.pieces - 1) / max(a.pieces - blocks / 2, a.pieces / 4), kChunkWaves);
}
// No block has more than half the root of its steps: the pieces' states are read by one workgroup, which
// takes about as long for four of them as a wave for a step.  (One sequence, 8 KV heads, one token over 8192:
// 96 us with as many pieces as there can be, 26 with the root of the steps, 23 with half of it; over 32768 302,
// 56, 38; eight tokens for each of four over 8192: 47, 34, 30.)
__device__ __forceinline__ int block_pieces(int steps, int quantum)
{
    return min((steps + quantum - 1) / quantum, (int)(0.5f * __builtin_sqrtf((float)steps)) + 1);
}
// A table's row blocks and the steps of each.
template <int LI>
__device__ __forceinline__ void row_steps(const ChunkArgs& a, int rows, int t, int& steps, int& nb)
{
    const SecLens len = section_lens<LI>(a, t);
    const int n = new_tokens(a, t / a.Hkv);
    nb = chunk_blocks(n, a.Hq / a.Hkv, rows, a.rows_lo, a.rows_hi);
    // (at most 2^18, so that the sums of 4096 blocks stay below 2^31: a longer table's pieces are longer)
    steps = min(((len.hi + 31) >> 5) + ((len.lo + 31) >> 5) + ((n + 31) >> 5), 1 << 18);
    steps &= -(int)(nb > 0);  // (a mask: the lengths' loads do not wait for the new tokens')
}
template <int LI>
__device__ __forceinline__ RowPiece row_piece(const ChunkArgs& a, int rows, long long* lds)
{
    const int tables = a.B * a.Hkv, me = (int)blockIdx.x;
    if (tables <= kWave) {  // a lane per table, every wave by itself
        const int lane = lane_id();
        int steps = 0, nb = 0;
        if (lane < tables) row_steps<LI>(a, rows, lane, steps, nb);
        const int total = __builtin_amdgcn_readlane(wave_incl_scan(nb * steps), kWave - 1);
        const int blocks = wave_incl_scan(nb);
        const int quantum = piece_quantum(a, total, __builtin_amdgcn_readlane(blocks, kWave - 1));
        const int each = block_pieces(steps, quantum);
        const int end = wave_incl_scan(nb * each);
        const unsigned long long past = __ballot(end > me);
        if (!past) return RowPiece{-1, 0, 0, 0, 0};
        const int l = __builtin_ctzll(past);
        const int e = __builtin_amdgcn_readlane(each, l), k = me - __builtin_amdgcn_readlane(end - nb * each, l), blk = k / e;
        return RowPiece{l, blk, k - blk * e, e, __builtin_amdgcn_readlane(blocks - nb, l) + blk};
    }
    constexpr int kPer = kRowTables / (kChunkWaves * kWave);
    int steps[kPer], nb[kPer], sum = 0, count = 0;
    const int t0 = (int)threadIdx.x * kPer;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        steps[i] = nb[i] = 0;
        if (t0 + i < tables) row_steps<LI>(a, rows, t0 + i, steps[i], nb[i]);
        sum += nb[i] * steps[i];
        count += nb[i];
    }
    long long both;
    const long long before = block_excl_scan<long long>(((long long)count << 32) | sum, lds, &both);
    const int quantum = piece_quantum(a, (int)(both & 0xffffffff), (int)(both >> 32));
    int pieces = 0, block = (int)(before >> 32);
#pragma unroll
    for (int i = 0; i < kPer; ++i) pieces += nb[i] * block_pieces(steps[i], quantum);
    long long all, at = block_excl_scan<long long>(pieces, lds, &all);
    if (me >= all) return RowPiece{-1, 0, 0, 0, 0};
    int* found = reinterpret_cast<int*>(lds);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int each = block_pieces(steps[i], quantum);
        const long long next = at + nb[i] * each;
        if (me >= at && me < next) {
            const int k = me - (int)at, blk = k / each;
            found[0] = t0 + i;
            found[1] = blk;
            found[2] = k - blk * each;
            found[3] = each;
            found[4] = block + blk;
        }
        at = next;
        block += nb[i];
    }
    __syncthreads();
    const RowPiece p{__builtin_amdgcn_readfirstlane(found[0]), __builtin_amdgcn_readfirstlane(found[1]),
                     __builtin_amdgcn_readfirstlane(found[2]), __builtin_amdgcn_readfirstlane(found[3]),
                     __builtin_amdgcn_readfirstlane(found[4])};
    __syncthreads();
    return p;
}

template <int LI, int RT, bool MOD>
__global__ __launch_bounds__(kChunkWaves * kWave, RT == 1 ? (LI == 1 ? 3 : 4) : 2) void chunk_rows(ChunkArgs a)
{
    constexpr KvFmt hi = kLayoutFmts[LI].hi, lo = kLayoutFmts[LI].lo;
    constexpr int kRows = 16 * RT;
    constexpr int kSlot = Staged<hi.kb, hi.vb, hi.T, MOD>::slot > Staged<lo.kb, lo.vb, lo.T, MOD>::slot
                              ? Staged<hi.kb, hi.vb, hi.T, MOD>::slot
                              : Staged<lo.kb, lo.vb, lo.T, MOD>::slot;
    union Shared {
        uint8_t slot[kChunkWaves][kSlot];
        struct {
            float acc[kChunkWaves][16][kD + 4];
            float ml[kChunkWaves][2][16];
            int last;
        } merge;
        long long find[kChunkWaves];
    };
    __shared__ __align__(1024) Shared lds;
    __shared__ RowsLds<RT> Q;
    __shared__ int odd_waves[kChunkWaves], odd_at[3];  // (the table and the piece's cached steps, kept out of the registers)
    const int lane = lane_id(), wave = wave_index();
    const int c = lane & 15, quarter = lane >> 4;
    const int G = a.Hq / a.Hkv;
    // Which piece of which row block: every block has as many pieces as its table's steps want.
    SeqBlock sb;
    int h, split, splits;
    long long slot_no;   // the block's number (its arrival word)
    long long part_no;   // its first piece's state
    const int first_n = first_tokens(a);
    if (a.splits == 1) {  // none is split
        const int item = (int)blockIdx.x / a.Hkv;
        h = (int)blockIdx.x - item * a.Hkv;
        if (a.one_block) {
            sb.b = item;
            sb.blk = 0;
            sequence_rows(a, sb, first_n);
            if (chunk_blocks(sb.n, G, kRows, a.rows_lo, a.rows_hi) == 0) return;
        } else {
            sb = find_block(a, item, kRows, a.rows_lo, a.rows_hi);
            if (sb.b < 0) return;
        }
        split = 0;
        splits = 1;
        slot_no = part_no = 0;
    } else {
        const RowPiece p = row_piece<LI>(a, kRows, lds.find);
        if (p.table < 0 || p.block >= a.blocks) return;  // (the second: lengths that do not sum to total_new)
        sb.b = p.table / a.Hkv;
        h = p.table - sb.b * a.Hkv;
        sb.blk = p.blk;
        split = p.split;
        splits = p.splits;
        slot_no = p.block;
        part_no = (int)blockIdx.x - split;
        sequence_rows(a, sb, first_n);
        if (sb.blk * kRows >= sb.n * G) return;  // (lengths that do not sum to total_new)
    }
    const int first = a.seq_len[sb.b];
    const int rows = sb.n * G, r0 = sb.blk * kRows;
    // the queries' loads first, then the table's lengths and first pages, whose loads follow each other
    u4 x[RT][kNG];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = min(r0 + 16 * rt + c, rows - 1);
        const int j = row / G, hq = h * G + row - j * G;
        const uint16_t* q = a.q + (sb.row0 + j) * a.q_stride + hq * kD + quarter * 8;
#pragma unroll
        for (int g = 0; g < kNG; ++g) x[rt][g] = *reinterpret_cast<const u4*>(q + g * kG);
    }
    const int t = sb.b * a.Hkv + h;
    const SecLens len = section_lens<LI>(a, t);
    const int len_hi = len.hi, len_lo = len.lo;
    const int last = min(r0 + kRows, rows) - 1;
    const int own = last / G + 1;  // tokens of the chunk that some row sees
    const int s_hi = (len_hi + 31) >> 5, s_lo = (len_lo + 31) >> 5, s_own = (own + 31) >> 5;
    const int steps = s_hi + s_lo + s_own;
    const int begin = (int)((long long)steps * split / splits), end = (int)((long long)steps * (split + 1) / splits);
    const int32_t* table = a.page_table + (long long)t * a.p_max;

    // a step's page, IDs outside the pool read as page 0 (and count no token)
    auto page_id = [&](int u, int part) {
        const bool high = u < s_hi;
        const int T = high ? hi.T : lo.T, len = high ? len_hi : len_lo;
        const int i = min(T == 16 ? 2 * (high ? u : u - s_hi) + part : (high ? u : u - s_hi), (len + T - 1) / T - 1);
        return __builtin_amdgcn_readfirstlane(table[high ? i : a.p_max - 1 - i]);
    };
    auto outside = [&](int id) { return (unsigned long long)(unsigned)id >= (unsigned long long)a.num_pages; };
    using Hi = Staged<hi.kb, hi.vb, hi.T, MOD>;
    using Lo = Staged<lo.kb, lo.vb, lo.T, MOD>;
    uint8_t* slot = lds.slot[wave];
    uint32_t bad = 0;  // of the staged step
    auto stage = [&](int u, int id0, int id1) {
        const bool o0 = outside(id0), o1 = outside(id1);
        const uint8_t* p0 = a.pool + (long long)(o0 ? 0 : id0) * a.page_bytes;
        const uint8_t* p1 = a.pool + (long long)(o1 ? 0 : id1) * a.page_bytes;
        if (u < s_hi) {
            stage_page<Hi::need>(slot, p0, lane);
            if (hi.T == 16) stage_page<Hi::need>(slot + Hi::page, p1, lane);
        } else {
            stage_page<Lo::need>(slot, p0, lane);
            if (lo.T == 16) stage_page<Lo::need>(slot + Lo::page, p1, lane);
        }
        const bool two = u < s_hi ? hi.T == 16 : lo.T == 16;
        bad = two ? (o0 ? 1u : 0u) | (o1 ? 2u : 0u) : (o0 ? 3u : 0u);
    };
    const int cached = min(end, s_hi + s_lo);
    int u = begin + wave;
    int n0 = 0, n1 = 0;
    if (u < cached) {
        n0 = page_id(u, 0);
        n1 = page_id(u, 1);
    }
    Rows<RT> R;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = min(r0 + 16 * rt + c, rows - 1);
        const int j = row / G, hq = h * G + row - j * G;
        const RowOperands o = row_operands(x[rt], quarter);
        if (wave == 0) {
#pragma unroll
            for (int g = 0; g < kNG; ++g) Q.q[rt][g][lane] = o.q[g];
            Q.sums[rt][lane] = o.sums;
        }
        R.unit[rt] = o.unit * a.scale;
        R.p[rt] = first + j;
        R.form[rt] = ScoreForm{a.cap_in, a.cap, MOD && a.slopes ? a.slopes[hq] : 0.0f};
        R.m[rt] = kLowest;
        R.l[rt] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) R.acc[rt][dt] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    if (MOD && threadIdx.x == 0) {
        odd_at[0] = t;
        odd_at[1] = begin;
        odd_at[2] = cached;
    }
    __syncthreads();
    if (u < cached) stage(u, n0, n1);
    bool odd = false;  // whether the wave met odd groups
    {
        while (u < cached) {
            const int next = u + kChunkWaves;
            if (next < cached) {
                n0 = page_id(next, 0);
                n1 = page_id(next, 1);
            }
            const uint32_t b = bad;
            auto ahead = [&]() {
                if (next < cached) stage(next, n0, n1);
            };
            staged_ready();
            if (u < s_hi) odd |= cached_step<hi.kb, hi.vb, hi.T, RT, MOD>(R, Q, slot, len_hi - 32 * u, b, a, fresh(lane), ahead);
            else odd |= cached_step<lo.kb, lo.vb, lo.T, RT, MOD>(R, Q, slot, len_lo - 32 * (u - s_hi), b, a, fresh(lane), ahead);
            u = next;
        }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) R.acc[rt][dt] *= 2.0f;  // (value_pairs)
    {
        const uint16_t* k = a.k + sb.row0 * a.k_stride + h * kD;
        const uint16_t* v = a.v + sb.row0 * a.v_stride + h * kD;
        for (int s = max(begin - s_hi - s_lo, 0) + wave; s < end - s_hi - s_lo; s += kChunkWaves)
            own_step<RT, MOD>(R, Q, k, v, 32 * s, own, first, a, c, quarter);
    }

    // the waves' states, 16 rows at a time: 16 threads a row, eight dims each
    const int row = threadIdx.x >> 4, d = (threadIdx.x & 15) * 8;
    auto part_of = [&](int k) {
        return span(a.part + (part_no + k) * kRows * kChunkPart, kRows * kChunkPart * 4);
    };
    auto write = [&](int at, const float (&o)[8], float m, float sum) {
        if (at >= rows) return;
        const int j = at / G, hq = h * G + at - j * G;
        const long long row_q = (sb.row0 + j) * a.Hq + hq;
        const float inv = 1.0f / sum;
        h8 r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = (_Float16)(o[i] * inv);
        *reinterpret_cast<h8*>(a.out + row_q * kD + d) = r;
        if (a.lse && d == 0) a.lse[row_q] = kChunkLn2 * (m + __builtin_amdgcn_logf(sum));
    };
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        if (MOD && lane == 0) odd_waves[wave] = odd;
        __syncthreads();
        const float l = rows_sum(R.l[rt]);
        if (quarter == 0) {
            lds.merge.ml[wave][0][c] = R.m[rt];
            lds.merge.ml[wave][1][c] = l;
        }
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<f4*>(&lds.merge.acc[wave][c][16 * dt + 4 * quarter]) = R.acc[rt][dt];
        __syncthreads();
        float m = kLowest, sum = 0.0f, o[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kChunkWaves; ++w) m = fmaxf(m, lds.merge.ml[w][0][row]);
#pragma unroll
        for (int w = 0; w < kChunkWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(lds.merge.ml[w][0][row] - m);
            sum += f * lds.merge.ml[w][1][row];
            const f4 x = *reinterpret_cast<const f4*>(&lds.merge.acc[w][row][d]);
            const f4 y = *reinterpret_cast<const f4*>(&lds.merge.acc[w][row][d + 4]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[i] += f * x[i];
                o[i + 4] += f * y[i];
            }
        }
        if (MOD && __builtin_expect(odd_waves[0] | odd_waves[1] | odd_waves[2] | odd_waves[3], 0)) {
            const OddRow r{chunk_args(), odd_at[0], min(r0 + 16 * rt + row, rows - 1), odd_at[1], odd_at[2], sb.row0, m};
            const f4 x = odd_four<LI>(f4{o[0], o[1], o[2], o[3]}, r, d), y = odd_four<LI>(f4{o[4], o[5], o[6], o[7]}, r, d + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[i] = x[i];
                o[i + 4] = y[i];
            }
        }
        if (splits == 1) {
            write(r0 + 16 * rt + row, o, m, sum);
        } else if (r0 + 16 * rt + row < rows) {
            const __amdgpu_buffer_rsrc_t to = part_of(split);
            const int at = (16 * rt + row) * kChunkPart * 4;
            put_quad(to, at + d * 4, 0, f4{o[0], o[1], o[2], o[3]});
            put_quad(to, at + d * 4, 16, f4{o[4], o[5], o[6], o[7]});
            if (d == 0) put_quad(to, at, kD * 4, f4{m, sum, 0.0f, 0.0f});
        }
    }
    if (splits == 1 || !split_last(a.arrive + slot_no, splits, &lds.merge.last)) return;
    // the last of the block's workgroups joins their states, in order
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        if (r0 + 16 * rt + row >= rows) continue;
        float m = kLowest, sum = 0.0f;
        f4 x = {0.0f, 0.0f, 0.0f, 0.0f}, y = x;
        constexpr int kAhead = 4;  // states whose loads are in flight together
        for (int k = 0; k < splits; k += kAhead) {
            f4 ml[kAhead], px[kAhead], py[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const __amdgpu_buffer_rsrc_t from = part_of(min(k + i, splits - 1));
                const int at = (16 * rt + row) * kChunkPart * 4;
                ml[i] = get_quad(from, at, kD * 4);
                px[i] = get_quad(from, at + d * 4, 0);
                py[i] = get_quad(from, at + d * 4, 16);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (k + i >= splits) continue;
                const float top = fmaxf(m, ml[i][0]);
                const float f = __builtin_amdgcn_exp2f(m - top), g = __builtin_amdgcn_exp2f(ml[i][0] - top);
                m = top;
                sum = sum * f + ml[i][1] * g;
                x = x * f + px[i] * g;
                y = y * f + py[i] * g;
            }
        }
        const float o[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        write(r0 + 16 * rt + row, o, m, sum);
    }
}

// ---- attention: many rows, pages dequantized once for a workgroup -----------------------------
//
// A workgroup takes 256 rows of one (sequence, KV head), 32 per wave, and goes over the table's
// steps together: each step's 32 tokens are turned into matrix operands once, by all eight
// waves (one key and one value operand of a lane each), and read from LDS by all of them: keys
// as exact codes with their scales in 32 bits beside them, values dequantized to fp16.  Raw pages
// arrive in one of two slots by loads with an LDS destination, asked for two steps ahead; operands lie
// in one of three buffers: a step's scores are computed from one while the step before's weights meet
// their values from another and the next one is made.
// The blocks of all tables end to end are cut into equal shares, one per CU: with a workgroup per block the
// longest ones set the time (257-512 tokens for each of 8 sequences over 0-8192: 546 us, with shares 377).
// Bound by issue: that case takes 419 us at 160 GFLOP, 2048 tokens over 8192 at 64 / 8 heads 913 us, 499
// TFLOP/s (an 8192^3 fp16 library product 1137), the weights' second products not counted.
constexpr int kTileWaves = 8;
constexpr int kTileRows = kTileWaves * 32;
static_assert(kTileRows == kChunkRows, "row blocks of the plan");

constexpr int kStepUnits = 64;  // work units of a step

struct TileBuf {
    h8 k[2][kNG][kWave];     // [tile][group][lane]
    h8 v[8][kWave];          // [16-dim tile][lane]
    h8 meta[2][16];          // [tile][token] {s, z} of four groups
    float s[2][kNG][16];     // 2^15 s times the codes' unit (own tokens: 2^-9, their products are sums of halfs)
    int pos[2][16];
    uint32_t odd[kTileWaves];  // own values that are not finite, by the wave that met them
};

// The staged pages of a step (slot) into operands: wave w makes the key operand of tile w / 4, group
// w % 4, and the value operand of dims 16 w ..; wave 0 the metadata.  Tokens with index >= left and
// those of tile t where bit t of `bad` is set do not exist.  Odd groups are left at 0 and noted in *odd
// (null: not looked for).
template <int KB, int VB, int T, bool MOD>
__device__ __forceinline__ void tile_put(TileBuf& b, const uint8_t* slot_, int left, uint32_t bad, int* odd, int wave, int lane)
{
    constexpr SecOffsets O = sec_offsets(KvFmt{KB, VB, T});
    constexpr int page = T == 16 ? Staged<KB, VB, T, MOD>::page : 0;  // from one tile's page to the other's
    const int c = lane & 15, quarter = lane >> 4;
    {
        const int t = wave >> 2, g = wave & 3;
        const uint8_t* pg = slot_ + t * page;
        const int slot = step_slot<T>(t, c);
        if constexpr (KB == 8) {
            const u2 v = *reinterpret_cast<const u2*>(pg + O.kc + ((2 * g + (quarter >> 1)) * T + slot) * 16 + (quarter & 1) * 8);
            b.k[t][g][lane] = key_codes8(v[0], v[1]);
        } else {
            b.k[t][g][lane] = key_codes4(*reinterpret_cast<const uint32_t*>(pg + O.kc + (g * T + slot) * 16 + quarter * 4));
        }
    }
    constexpr int row = T * VB / 8, piece = (T == 16 ? 4 : 8) * VB / 8;
    const int at = O.vc + (16 * wave + c) * row + quarter * piece;
    uint32_t codes[2];
    codes[0] = load_value_codes<VB, T>(slot_ + at);
    codes[1] = T == 16 ? load_value_codes<VB, T>(slot_ + page + at) : codes[0] >> (4 * VB);
    u4 v;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const u4 m = *reinterpret_cast<const u4*>(slot_ + t * page + O.vm + ((wave >> 1) * T + step_slot<T>(t, 4 * quarter)) * 4);
        uint32_t p, q;
        value_pairs<VB>(codes[t], __builtin_bit_cast(h2, __builtin_amdgcn_perm(m[2], m[0], 0x05040100u)),
                        __builtin_bit_cast(h2, __builtin_amdgcn_perm(m[2], m[0], 0x07060302u)) * (_Float16)0.5f,
                        __builtin_bit_cast(h2, __builtin_amdgcn_perm(m[3], m[1], 0x05040100u)),
                        __builtin_bit_cast(h2, __builtin_amdgcn_perm(m[3], m[1], 0x07060302u)) * (_Float16)0.5f, p, q);
        v[2 * t] = p;
        v[2 * t + 1] = q;
    }
    if (left < 32 || bad) {  // nothing behind a section's end reaches the sums
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            auto none = [&](int i) {
                return (T == 16 ? 16 * t : 0) + step_slot<T>(t, 4 * quarter + i) >= left || ((bad >> t) & 1);
            };
            v[2 * t] &= (none(0) ? 0u : 0xffffu) | (none(2) ? 0u : 0xffff0000u);
            v[2 * t + 1] &= (none(1) ? 0u : 0xffffu) | (none(3) ? 0u : 0xffff0000u);
        }
    }
    if (MOD && odd) {  // (a lane looks at one token's {s, z} of the wave's group)
        const int token = lane & 31;
        const uint32_t sz = *reinterpret_cast<const uint32_t*>(slot_ + (T == 16 ? (token >> 4) * page : 0) + O.vm +
                                                               ((wave >> 1) * T + token % T) * 4);
        if (__builtin_expect(__any(odd_group<VB>(sz) && token < left && !((bad >> (T == 16 ? token >> 4 : 0)) & 1)), 0)) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const u4 m = *reinterpret_cast<const u4*>(slot_ + t * page + O.vm + ((wave >> 1) * T + step_slot<T>(t, 4 * quarter)) * 4);
                v[2 * t] &= (odd_group<VB>(m[0]) ? 0u : 0xffffu) | (odd_group<VB>(m[2]) ? 0u : 0xffff0000u);
                v[2 * t + 1] &= (odd_group<VB>(m[1]) ? 0u : 0xffffu) | (odd_group<VB>(m[3]) ? 0u : 0xffff0000u);
            }
            if (lane == 0) *odd = 1;
        }
    }
    b.v[wave][lane] = __builtin_bit_cast(h8, v);
    if (wave == 0 && lane < 32) {
        const uint8_t* pg = slot_ + quarter * page;
        const int slot = step_slot<T>(quarter, c);
        const h8 m = *reinterpret_cast<const h8*>(pg + O.km + slot * 16);
        b.meta[quarter][c] = m;
#pragma unroll
        for (int g = 0; g < kNG; ++g) b.s[quarter][g][c] = 0x1p15f * key_unit<KB>() * (float)m[2 * g];
        if constexpr (MOD) b.pos[quarter][c] = *reinterpret_cast<const int32_t*>(pg + O.pos + slot * 4);
    }
}

// The same of own tokens, staged as 32 rows of keys, then 32 of values; the first `left` exist, the
// first is at position pos0.
constexpr int kOwnSlot = 2 * 32 * kD * 2;
__device__ __forceinline__ void tile_put_own(TileBuf& b, const uint8_t* slot, int left, int pos0, int wave, int lane)
{
    const int c = lane & 15, quarter = lane >> 4;
    b.k[wave >> 2][wave & 3][lane] =
        *reinterpret_cast<const h8*>(slot + step_slot<32>(wave >> 2, c) * 256 + (wave & 3) * 64 + quarter * 16);
    const uint16_t* values = reinterpret_cast<const uint16_t*>(slot + kOwnSlot / 2) + 16 * wave + c;
    uint32_t w[8];
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int token = 8 * quarter + e;
        w[e] = values[token * kD];
        const bool none = token >= left, bad = (w[e] & 0x7c00u) == 0x7c00u;
        odd |= bad && !none;
        w[e] = bad || none ? 0u : w[e];
    }
    b.v[wave][lane] = __builtin_bit_cast(h8, u4{w[0] | w[2] << 16, w[1] | w[3] << 16, w[4] | w[6] << 16, w[5] | w[7] << 16});
    const unsigned long long any = __ballot(odd);
    if (lane == 0) b.odd[wave] = any != 0;
    if (wave == 0 && lane < 32) {
        b.meta[quarter][c] = __builtin_bit_cast(h8, u4{0, 0, 0, 0});
#pragma unroll
        for (int g = 0; g < kNG; ++g) b.s[quarter][g][c] = 0x1p-9f;
        b.pos[quarter][c] = pos0 + step_slot<32>(quarter, c);
    }
}

// Nothing is scheduled across.  The step is written in the order it is to be issued: left to itself the
// compiler, short of registers, puts every product right before its use and waits for it.
__device__ __forceinline__ void phase() { __builtin_amdgcn_sched_barrier(0); }
// x is computed before the next phase.
__device__ __forceinline__ void by_now(float& x) { asm volatile("" : "+v"(x)); }

// The sums x[rt][t][r] of a staged step: token (t, 4 quarter + r) against rows 16 rt + c.  Units of a
// tile's group: while one's products are issued, the additions of the one before run beside
// them and the operands of the one after the next are read.
template <int RT>
__device__ __forceinline__ void tile_sums(const TileBuf& b, const h8 (&q)[RT][kNG], const h8 (&sums)[RT], float (&x)[RT][2][4],
                                          int lane)
{
    const int c = lane & 15, quarter = lane >> 4;
    const f4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int kUnits = 2 * kNG;
    h8 k[kUnits], meta[2];
    f4 s[kUnits], sum[2][RT], part[kUnits][RT];
    auto read = [&](int i) {
        k[i] = b.k[i / kNG][i % kNG][lane];
        s[i] = *reinterpret_cast<const f4*>(&b.s[i / kNG][i % kNG][4 * quarter]);
    };
    meta[0] = b.meta[0][c];
    read(0);
    read(1);
    phase();
#pragma unroll
    for (int i = 0; i <= kUnits; ++i) {
        const int t = i / kNG;
        if (i % kNG == 0 && i < kUnits) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) sum[t][rt] = mfma_k32(meta[t], sums[rt], zero);
        }
        if (i < kUnits) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) part[i][rt] = mfma_k32(k[i], q[rt][i % kNG], zero);
        }
        if (i + 2 < kUnits) read(i + 2);
        if (i + 2 == kNG) meta[1] = b.meta[1][c];
        if (i > 0) {
            const int e = i - 1;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                {
                    float y = __builtin_fmaf(s[e][r], part[e][rt][r], sum[e / kNG][rt][r]);
                    by_now(y);
                    sum[e / kNG][rt][r] = y;
                }
        }
        phase();
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) x[rt][t][r] = sum[t][rt][r];
}

template <int LI, bool MOD>
__global__ __launch_bounds__(kTileWaves * kWave, 2) void chunk_tiles(ChunkArgs a)
{
    constexpr KvFmt hi = kLayoutFmts[LI].hi, lo = kLayoutFmts[LI].lo;
    constexpr int RT = 2;
    using Hi = Staged<hi.kb, hi.vb, hi.T, MOD>;
    using Lo = Staged<lo.kb, lo.vb, lo.T, MOD>;
    constexpr int kPages = Hi::slot > Lo::slot ? Hi::slot : Lo::slot, kSlot = kPages > kOwnSlot ? kPages : kOwnSlot;
    struct Shared {
        uint8_t slots[2][kSlot];  // (first: the loads that write there take 16-bit addresses)
        TileBuf bufs[3];
        long long scan[kTileWaves];
        long long found_at;
        int found, last, odd;
    };
    __shared__ __align__(1024) Shared sh;
    auto& slots = sh.slots;
    auto& bufs = sh.bufs;
    const int lane = lane_id(), wave = wave_index();
    const int c = lane & 15, quarter = lane >> 4;
    const int G = a.Hq / a.Hkv;

    // The work of all tables end to end, cut into equal shares
    const int own_units = 2 * kTileRows / G;  // of one block's own tokens more than the block before has
    const int tables = a.B * a.Hkv, chunk = (tables + kTileWaves * kWave - 1) / (kTileWaves * kWave);
    const int t0 = min((int)threadIdx.x * chunk, tables), t1 = min(t0 + chunk, tables);
    auto blocks_units = [&](int t, int& nb) -> long long {  // units of a block's cached steps; blocks
        const int n = new_tokens(a, t / a.Hkv);
        nb = chunk_blocks(n, G, kTileRows, a.rows_lo, a.rows_hi);
        const SecLens len = section_lens<LI>(a, t);
        return nb ? (long long)(((len.hi + 31) >> 5) + ((len.lo + 31) >> 5)) * kStepUnits : 0;
    };
    auto units_to = [&](long long cached, int nb) { return nb * cached + (long long)own_units * nb * (nb + 1) / 2; };
    long long mine = 0;
    for (int t = t0; t < t1; ++t) {
        int nb;
        const long long cached = blocks_units(t, nb);
        mine += units_to(cached, nb);
    }
    long long total;
    const long long mine_from = block_excl_scan_wide(mine, sh.scan, &total);
    // a share has at least eight steps (its fixed cost is about as much)
    const long long quantum = max((total + gridDim.x - 1) / gridDim.x, 8ll * kStepUnits);
    // consecutive shares on one XCD (workgroups go round over the eight): they read the same tables
    const int per_xcd = ((int)gridDim.x + 7) >> 3;
    const int share = gridDim.x % 8 == 0 ? ((int)blockIdx.x & 7) * per_xcd + ((int)blockIdx.x >> 3) : (int)blockIdx.x;
    const long long start = share * quantum, stop = min(total, start + quantum);
    if (start >= total) return;
    const int first_n = first_tokens(a);
    int piece = 0;
    // One piece: units cur .. piece_end of the row block of head h that has from .. to
    auto tile_piece = [&](const SeqBlock& sb, int h, long long from, long long to, long long cur, long long piece_end) {
    const int first = a.seq_len[sb.b];
    const int rows = sb.n * G, r0 = sb.blk * kTileRows + wave * 32;  // the wave's first row
    if (sb.blk * kTileRows >= rows) return;
    h8 q[RT][kNG], sums[RT];
    Rows<RT> R;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = min(r0 + 16 * rt + c, rows - 1);
        const int j = row / G, hq = h * G + row - j * G;
        const uint16_t* p = a.q + (sb.row0 + j) * a.q_stride + hq * kD + quarter * 8;
        u4 x[kNG];
#pragma unroll
        for (int g = 0; g < kNG; ++g) x[g] = *reinterpret_cast<const u4*>(p + g * kG);
        const RowOperands o = row_operands(x, quarter);
#pragma unroll
        for (int g = 0; g < kNG; ++g) q[rt][g] = o.q[g];
        sums[rt] = o.sums;
        R.unit[rt] = o.unit * a.scale;
        R.p[rt] = first + j;
        R.form[rt] = ScoreForm{a.cap_in, a.cap, MOD && a.slopes ? a.slopes[hq] : 0.0f};
        R.m[rt] = kLowest;
        R.l[rt] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) R.acc[rt][dt] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int t = sb.b * a.Hkv + h;
    const SecLens len = section_lens<LI>(a, t);
    const int len_hi = len.hi, len_lo = len.lo;
    const int own = (min((sb.blk + 1) * kTileRows, rows) - 1) / G + 1;  // own tokens that some row sees
    const bool idle = r0 >= rows;                                        // a wave without rows only helps
    const int j_first = min(r0, rows - 1) / G;  // the wave's first position
    const int s_hi = (len_hi + 31) >> 5, s_lo = (len_lo + 31) >> 5, s_own = (own + 31) >> 5;
    // units -> steps: the own steps share the block's units behind the cached ones'
    auto step_of = [&](long long x) -> int {
        const long long before_own = (long long)(s_hi + s_lo) * kStepUnits;
        if (x < before_own) return (int)(x / kStepUnits);
        return s_hi + s_lo + (int)((x - before_own) * s_own / (to - from - before_own));
    };
    const int begin = step_of(cur - from), end = step_of(piece_end - from);
    const bool whole = cur == from && piece_end == to;
    const int32_t* table = a.page_table + (long long)t * a.p_max;
    const uint16_t* ok = a.k + sb.row0 * a.k_stride + h * kD;
    const uint16_t* ov = a.v + sb.row0 * a.v_stride + h * kD;

    // lane l: the pages of step id_step + l (-1: outside the pool, reads as page 0 and counts no token)
    int id_step = begin, ids0 = 0, ids1 = 0;
    auto fetch_ids = [&](int from) {
        id_step = from;
        const int u = min(from + lane, s_hi + s_lo - 1);
        const bool high = u < s_hi;
        const int T = high ? hi.T : lo.T, len = high ? len_hi : len_lo, k = high ? u : u - s_hi;
        const int last = (len + T - 1) / T - 1, i0 = T == 16 ? 2 * k : k, i1 = T == 16 ? min(i0 + 1, last) : i0;
        ids0 = table[high ? i0 : a.p_max - 1 - i0];
        ids1 = table[high ? i1 : a.p_max - 1 - i1];
        ids0 = (unsigned long long)(unsigned)ids0 < (unsigned long long)a.num_pages ? ids0 : -1;
        ids1 = (unsigned long long)(unsigned)ids1 < (unsigned long long)a.num_pages ? ids1 : -1;
    };
    if (begin < min(end, s_hi + s_lo)) fetch_ids(begin);
    // step u's pages (or own rows) on their way into a slot, 1 KB pieces over the waves; which of its
    // tiles lie outside the pool
    auto load = [&](int u, uint8_t* slot) -> uint32_t {
        if (u >= s_hi + s_lo) {
            const int i0 = 32 * (u - s_hi - s_lo);
            stage_rows(slot + wave * 1024, ok + (long long)i0 * a.k_stride, 2 * (int)a.k_stride, 4 * wave, own - 1 - i0, fresh(lane));
            stage_rows(slot + kOwnSlot / 2 + wave * 1024, ov + (long long)i0 * a.v_stride, 2 * (int)a.v_stride, 4 * wave,
                       own - 1 - i0, fresh(lane));
            return 0;
        }
        if (u >= id_step + kWave) fetch_ids(u);
        const int id0 = __builtin_amdgcn_readlane(ids0, u - id_step), id1 = __builtin_amdgcn_readlane(ids1, u - id_step);
        const bool high = u < s_hi, two = high ? hi.T == 16 : lo.T == 16;
        const int loads = high ? Hi::loads : Lo::loads, need = high ? Hi::need : Lo::need;
        for (int i = wave; i < (two ? 2 : 1) * loads; i += kTileWaves) {
            const int part = i >= loads ? 1 : 0, id = part ? id1 : id0;
            stage_piece(slot + part * loads * 1024, a.pool + (long long)(id < 0 ? 0 : id) * a.page_bytes, need, i - part * loads,
                        fresh(lane));
        }
        return two ? (id0 < 0 ? 1u : 0u) | (id1 < 0 ? 2u : 0u) : (id0 < 0 ? 3u : 0u);
    };
    int* const odd_word = MOD && a.window != INT32_MAX ? &sh.odd : nullptr;
    auto put = [&](int u, TileBuf& b, const uint8_t* slot, uint32_t bad) {
        if (u < s_hi) tile_put<hi.kb, hi.vb, hi.T, MOD>(b, slot, len_hi - 32 * u, bad, odd_word, wave, fresh(lane));
        else if (u < s_hi + s_lo) tile_put<lo.kb, lo.vb, lo.T, MOD>(b, slot, len_lo - 32 * (u - s_hi), bad, odd_word, wave, fresh(lane));
        else tile_put_own(b, slot, own - 32 * (u - s_hi - s_lo), first + 32 * (u - s_hi - s_lo), wave, fresh(lane));
    };
    // steps begin, begin + 1 on their way; `bad` of the step that is computed, the next and the one after
    uint32_t now_bad = begin < end ? load(begin, slots[0]) : 0, next_bad = begin + 1 < end ? load(begin + 1, slots[1]) : 0;
    uint32_t last_bad = 0;
    if (MOD && threadIdx.x == 0) sh.odd = 0;
    staged_ready();
    __syncthreads();
    if (begin < end) put(begin, bufs[0], slots[0], now_bad);
    bufs[2].v[wave][lane] = __builtin_bit_cast(h8, u4{0, 0, 0, 0});  // "before" the first step
    h8 P[RT], rest[RT];  // the weights of the step before, whose values are still to be added
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) P[rt] = rest[rt] = __builtin_bit_cast(h8, u4{0, 0, 0, 0});
    auto add_values = [&](const TileBuf& b) {
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            const h8 V = b.v[dt][lane];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) R.acc[rt][dt] = mfma_k32(V, P[rt], R.acc[rt][dt]);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) R.acc[rt][dt] = mfma_k32(V, rest[rt], R.acc[rt][dt]);
        }
    };
    int at = 0;  // buffer of the step
    __syncthreads();
    // a step, of cached tokens or (own) of the chunk's
    auto step = [&](int u, auto own_) {
        constexpr bool mine = decltype(own_)::value;
        const TileBuf& b = bufs[at];
        const TileBuf& before = bufs[at == 0 ? 2 : at - 1];
        TileBuf& after = bufs[at == 2 ? 0 : at + 1];
        const int i0 = 32 * (u - s_hi - s_lo);
        // the slot of the step after the next is free: its step (this one) has been put
        if (u + 2 < end) last_bad = load(u + 2, slots[(u - begin) & 1]);
        if (!idle) {
            const int T = u < s_hi ? hi.T : lo.T;
            const int left = mine ? 32 : (u < s_hi ? len_hi - 32 * u : len_lo - 32 * (u - s_hi));
            // logits with a score form, -inf where a row does not see a token
            auto hide = [&](float (&x)[RT][2][4]) {
                if (MOD || (mine && i0 + 31 > j_first)) {
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt) {
                        const int4 ps = *reinterpret_cast<const int4*>(&b.pos[tt][4 * quarter]);
                        const int pos[4] = {ps.x, ps.y, ps.z, ps.w};
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const int away = R.p[rt] - pos[r];
                                const float y = MOD ? formed(x[rt][tt][r] * R.unit[rt], R.form[rt], (float)away) : x[rt][tt][r];
                                x[rt][tt][r] = (away >= 0 || !mine) && away < a.window ? y : -INFINITY;
                            }
                    }
                }
                if (!mine && (left < 32 || now_bad)) {
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int token = T == 16 ? 16 * tt + 4 * quarter + r : step_slot<32>(tt, 4 * quarter + r);
                            const bool there = token < left && !((now_bad >> tt) & 1);
#pragma unroll
                            for (int rt = 0; rt < RT; ++rt) x[rt][tt][r] = there ? x[rt][tt][r] : -INFINITY;
                        }
                }
            };
            float unit[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) unit[rt] = MOD ? kChunkLog2e : R.unit[rt];
            {
                // the values of the step before beside this step's exponentials
                float x[RT][2][4];
                tile_sums<RT>(b, q, sums, x, lane);
                h8 V[8];
                V[0] = before.v[0][lane];
                V[1] = before.v[1][lane];
                phase();
                hide(x);
                raise_max<RT>(R, unit, x, [&] {  // (the step before still has the old max)
                    add_values(before);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) P[rt] = rest[rt] = __builtin_bit_cast(h8, u4{0, 0, 0, 0});
                });
                phase();
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) R.acc[rt][dt] = mfma_k32(V[dt], P[rt], R.acc[rt][dt]);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) R.acc[rt][dt] = mfma_k32(V[dt], rest[rt], R.acc[rt][dt]);
                    if (dt + 2 < 8) V[dt + 2] = before.v[dt + 2][lane];
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {  // a score of each row tile
                        float& w = x[rt][dt >> 2][dt & 3];
                        w = weight(w, unit[rt], R.m[rt]);
                        R.l[rt] += w;
                        by_now(w);
                        by_now(R.l[rt]);
                    }
                    phase();
                }
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    P[rt] = pack_weights(x[rt]);
                    rest[rt] = pack_rest(x[rt], P[rt]);
                }
            }
            if constexpr (mine) {
                uint32_t odd = 0;
#pragma unroll
                for (int w = 0; w < kTileWaves; ++w) odd |= b.odd[w];
                if (odd) {  // (the weights once more: kept until here they cost registers in every step)
                    float x[RT][2][4];
                    tile_sums<RT>(b, q, sums, x, lane);
                    hide(x);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                x[rt][tt][r] = weight(x[rt][tt][r], unit[rt], R.m[rt]);
                    odd_values<RT>(R, x, ov, i0, own, first, a, c, quarter);
                }
            }
        }
        if (u + 1 < end) put(u + 1, after, slots[(u + 1 - begin) & 1], next_bad);
        at = at == 2 ? 0 : at + 1;
        now_bad = next_bad;
        next_bad = last_bad;
        staged_ready();
        __syncthreads();
    };
    for (int u = begin; u < min(end, s_hi + s_lo); ++u) step(u, std::false_type{});
    if (!idle) {
        add_values(bufs[at == 0 ? 2 : at - 1]);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            P[rt] = rest[rt] = __builtin_bit_cast(h8, u4{0, 0, 0, 0});
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) R.acc[rt][dt] *= 2.0f;  // (value_pairs)
        }
    }
    if (end > s_hi + s_lo) {
        for (int u = max(begin, s_hi + s_lo); u < end; ++u) step(u, std::true_type{});
        if (!idle) add_values(bufs[at == 0 ? 2 : at - 1]);
    }
    // A wave's part of a piece's state in the workspace: its accumulators lane by lane (1 KB each), then max and sum
    // of its rows.  A share's first piece has slot 0, the others slot 1, whose last one is read by others.
    constexpr int kWavePart = RT * 8 * 1024 + RT * 128;
    static_assert(kTileWaves * kWavePart <= kTileRows * kChunkPart * 4, "a piece's room in the workspace");
    auto part_of = [&](int k, bool first_piece) {
        return span(reinterpret_cast<uint8_t*>(a.part + (2ll * k + (first_piece ? 0 : 1)) * kTileRows * kChunkPart) +
                        wave * kWavePart,
                    kWavePart);
    };
    if (MOD && !idle && __builtin_expect(__builtin_amdgcn_readfirstlane(sh.odd), 0)) {
        // (the sums wait in the workspace: beside them there are no registers for this)
        const __amdgpu_buffer_rsrc_t room = part_of(share, piece == 0);
#pragma unroll
        for (int i = 0; i < RT * 8; ++i) put_quad(room, lane * 16, i * 1024, R.acc[i / 8][i % 8]);
        staged_ready();
#pragma unroll 1
        for (int i = 0; i < RT * 8; ++i) {
            const OddRow r{chunk_args(), t, min(r0 + 2 * (i & 8) + c, rows - 1), begin, min(end, s_hi + s_lo), sb.row0,
                           i < 8 ? R.m[0] : R.m[1]};
            put_quad(room, lane * 16, i * 1024, odd_four<LI>(get_quad(room, lane * 16, i * 1024), r, 16 * (i & 7) + 4 * quarter));
        }
        staged_ready();
#pragma unroll
        for (int i = 0; i < RT * 8; ++i) R.acc[i / 8][i % 8] = get_quad(room, lane * 16, i * 1024);
    }

    float l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) l[rt] = rows_sum(R.l[rt]);
    auto write = [&](int rt) {
        const int at = r0 + 16 * rt + c;
        if (at >= rows) return;
        const int j = at / G, hq = h * G + at - j * G;
        const long long row_q = (sb.row0 + j) * a.Hq + hq;
        const float inv = 1.0f / l[rt];
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            h4 r;
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = (_Float16)(R.acc[rt][dt][i] * inv);
            *reinterpret_cast<h4*>(a.out + row_q * kD + 16 * dt + 4 * quarter) = r;
        }
        if (a.lse && quarter == 0) a.lse[row_q] = kChunkLn2 * (R.m[rt] + __builtin_amdgcn_logf(l[rt]));
    };
    if (whole) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) write(rt);
        return;
    }
    // Cut by a share's end: the pieces' states are joined by the last of them, in order.  A share has at most
    // two pieces of cut blocks, its first (slot 0) and its last (slot 1, if it is not also the first);
    // the block's word is that of the share where it begins.
    const int k0 = (int)(from / quantum), k1 = (int)((to - 1) / quantum);
    {
        const __amdgpu_buffer_rsrc_t out = part_of(share, piece == 0);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) put_quad(out, lane * 16, (rt * 8 + dt) * 1024, R.acc[rt][dt]);
            if (quarter == 0)
                __builtin_amdgcn_raw_buffer_store_b64(u2{__float_as_uint(R.m[rt]), __float_as_uint(l[rt])}, out, c * 8,
                                                      RT * 8 * 1024 + rt * 128, 16);
        }
    }
    if (!split_last(a.arrive + k0, k1 - k0 + 1, &sh.last)) return;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        R.m[rt] = kLowest;
        l[rt] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) R.acc[rt][dt] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    for (int k = k0; k <= k1; ++k) {
        const __amdgpu_buffer_rsrc_t in = part_of(k, k > k0 || from == k0 * quantum);
        f4 o[RT][8];
        u2 ml[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            ml[rt] = __builtin_bit_cast(u2, __builtin_amdgcn_raw_buffer_load_b64(in, c * 8, RT * 8 * 1024 + rt * 128, 16));
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) o[rt][dt] = get_quad(in, lane * 16, (rt * 8 + dt) * 1024);
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const float m = __uint_as_float(ml[rt][0]), top = fmaxf(R.m[rt], m);
            const float f = __builtin_amdgcn_exp2f(R.m[rt] - top), g = __builtin_amdgcn_exp2f(m - top);
            R.m[rt] = top;
            l[rt] = l[rt] * f + __uint_as_float(ml[rt][1]) * g;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) R.acc[rt][dt] = R.acc[rt][dt] * f + o[rt][dt] * g;
        }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) write(rt);
    };
    for (long long cur = start; cur < stop; ++piece) {
        // the table that has unit `cur`
        __syncthreads();
        if (cur >= mine_from && cur < mine_from + mine) {
            long long at = mine_from;
            for (int t = t0; t < t1; ++t) {
                int nb;
                const long long cached = blocks_units(t, nb);
                const long long next = at + units_to(cached, nb);
                if (cur < next) {
                    sh.found = t;
                    sh.found_at = at;
                    break;
                }
                at = next;
            }
        }
        __syncthreads();
        const int t = __builtin_amdgcn_readfirstlane(sh.found);
        const long long table_at = read_lane<long long>(sh.found_at, 0);
        int nb;
        const long long cached = blocks_units(t, nb);
        int blk = 0;
        {
            int above = nb - 1;  // the last block that starts at or before cur
            while (blk < above) {
                const int mid = (blk + above + 1) >> 1;
                if (table_at + units_to(cached, mid) <= cur) blk = mid;
                else above = mid - 1;
            }
        }
        const long long from = table_at + units_to(cached, blk), to = table_at + units_to(cached, blk + 1);
        const long long piece_end = min(stop, to);
        SeqBlock sb;
        sb.b = t / a.Hkv;
        sb.blk = blk;
        sequence_rows(a, sb, first_n);
        tile_piece(sb, t - sb.b * a.Hkv, from, to, cur, piece_end);
        cur = piece_end;
    }
}

// ---- scores ---------------------------------------------------------------------------------
//
// A wave takes 32 tokens of a table (or of the chunk's own), their keys in registers as matrix
// operands, and goes over all rows of the sequence in sets of 16, whose queries pass through LDS for
// the workgroup's eight waves.  A set is either 16 positions of one query head (the maximum over the
// heads is taken between one set's results and the next's, in a lane) or 4 positions of four heads
// (between a lane's four results): the second where four divides the heads.  One exp2 serves all
// heads of a position.  Short chunks have a kernel of their own (chunk_scores_short); the sets of a longer one
// pass four at a time, the blocks of all tables cut into equal shares, two per CU (364 us without shares, 190
// with them, 155 with queries loaded straight to where the products read them: 257-512 tokens for each of 8
// sequences over 0-8192, 77 GFLOP, 498 TFLOP/s).  Bound by issue: two products, eight additions in fp32 and a
// maximum for 64 scores of a group.
//
// Queries stay unscaled here: a token's scales are in registers, in fp32, and take the 2^24 of
// the codes themselves; the unit of the sums is 2^-5, so that a group's sum of 32 halfs fits one.
constexpr int kScoreWaves = 8, kScoreTiles = 2;
constexpr int kScoreTokens = 16 * kScoreTiles;               // per wave
constexpr int kScoreBlock = kScoreTokens * kScoreWaves;      // per workgroup pass
constexpr int kScorePass = 4;                                // sets per pass of a long chunk
constexpr int kScoreSets = 3 * kScorePass;                   // in LDS
constexpr int kShortSets = 4;                                // of a short chunk, of four positions and heads
__device__ __forceinline__ bool score_short(int n, int G) { return (n + 3) / 4 * ((G + 3) >> 2) <= kShortSets; }

struct ScoreSet {
    h8 q[kNG][kWave];
    h8 sums[kWave];
    float lse[16];    // log2 units (natural ones with a score form); +inf: no such row
    float slope[16];
};

// One set on its way, by one wave: row m = c is at `offset` bytes from `base`; its queries go straight to
// where the products read them (a load with an LDS destination puts lane l's 16 bytes at l).
__device__ __forceinline__ void score_load(ScoreSet& s, const void* base, int offset, int quarter)
{
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(__attribute__((address_space(3))) void*)&s.q[0][0]);
    const unsigned long long p = (unsigned long long)base;
    const u4 rs = {(uint32_t)p, (uint32_t)(p >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
#pragma unroll
    for (int g = 0; g < kNG; ++g)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(at + g * 1024),
                     "v"(offset + quarter * 16), "s"(rs), "s"(g * 2 * kG)
                     : "memory");
}
// ... and arrived: the group sums beside them, by the same wave.
__device__ __forceinline__ void score_sums(ScoreSet& s, float lse, float slope, int c, int quarter, int lane)
{
    u4 sums;
    const h2 one = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
    for (int g = 0; g < kNG; ++g) {
        const u4 x = __builtin_bit_cast(u4, s.q[g][lane]);
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) t = __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, (uint32_t)x[i]), one, t, false);
        t = rows_sum(t) * 0x1p-5f;
        const _Float16 hi = (_Float16)t;
        const _Float16 lo = (_Float16)(t - (float)hi);
        const uint32_t bits = __builtin_bit_cast(unsigned short, quarter == 0 ? hi : lo);
        sums[g] = quarter < 2 ? bits << 16 : 0u;
    }
    s.sums[lane] = __builtin_bit_cast(h8, sums);
    if (quarter == 0) {
        s.lse[c] = lse;
        s.slope[c] = slope;
    }
}

// A score's probability.  In natural units the whole powers of two are split off before the product with
// log2(e) is rounded: 2^-24 of it alone would be 10^-6 of a probability of e^-20.
template <bool MOD>
__device__ __forceinline__ float probability(float x)
{
    if constexpr (!MOD) return __builtin_amdgcn_exp2f(x);
    x = fmaxf(x, -150.0f);
    const float whole = __builtin_rintf(x * kChunkLog2e);
    const float rest = __builtin_fmaf(x, kChunkLog2eRest, __builtin_fmaf(x, kChunkLog2e, -whole));
    return __builtin_ldexpf(__builtin_amdgcn_exp2f(rest), (int)whole);
}

// One set against a wave's tokens: the running maxima over the heads, of position p (+ 4 r) and tokens
// 16 kt + c, in log2 units (natural ones with a score form).
template <bool FOUR, bool MOD>
__device__ __forceinline__ void score_use(const ScoreSet& S, const ChunkArgs& a, const h8 (&K)[kScoreTiles][kNG],
                                          const h8 (&meta)[kScoreTiles], const float (&s)[kScoreTiles][kNG],
                                          const int (&pos)[kScoreTiles], int p, float (&top)[kScoreTiles][FOUR ? 1 : 4], int quarter,
                                          int lane)
{
    const f4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    const f4 lse = *reinterpret_cast<const f4*>(&S.lse[4 * quarter]);
    f4 slope = zero;
    if constexpr (MOD) slope = *reinterpret_cast<const f4*>(&S.slope[4 * quarter]);
    h8 q[kNG];
#pragma unroll
    for (int g = 0; g < kNG; ++g) q[g] = S.q[g][lane];
    const h8 qs = S.sums[lane];
    const float unit = a.scale * 32.0f;
    // a group's products beside the additions of the one before
    f4 sum[kScoreTiles], part[kNG][kScoreTiles];
    phase();
#pragma unroll
    for (int kt = 0; kt < kScoreTiles; ++kt) sum[kt] = mfma_k32(qs, meta[kt], zero);
#pragma unroll
    for (int g = 0; g <= kNG; ++g) {
        if (g < kNG) {
#pragma unroll
            for (int kt = 0; kt < kScoreTiles; ++kt) part[g][kt] = mfma_k32(q[g], K[kt][g], zero);
        }
        if (g > 0) {
#pragma unroll
            for (int kt = 0; kt < kScoreTiles; ++kt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float y = __builtin_fmaf(s[kt][g - 1], part[g - 1][kt][r], sum[kt][r]);
                    by_now(y);
                    sum[kt][r] = y;
                }
        }
        phase();
    }
#pragma unroll
    for (int kt = 0; kt < kScoreTiles; ++kt) {
        float x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if constexpr (MOD) {
                const int away = p + (FOUR ? 0 : 4 * r) - pos[kt];
                const float y = formed(sum[kt][r] * unit, ScoreForm{a.cap_in, a.cap, slope[r]}, (float)away) - lse[r];
                x[r] = away < a.window ? y : -INFINITY;
            } else {
                x[r] = __builtin_fmaf(sum[kt][r], unit, -lse[r]);
            }
        }
        if constexpr (FOUR) {
            top[kt][0] = max3(max3(top[kt][0], x[0], x[1]), x[2], x[3]);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) top[kt][r] = fmaxf(top[kt][r], x[r]);
        }
    }
}

template <int LI, bool FOUR, bool MOD>
__global__ __launch_bounds__(kScoreWaves * kWave, 4) void chunk_scores(ChunkArgs a)
{
    constexpr KvFmt hi = kLayoutFmts[LI].hi, lo = kLayoutFmts[LI].lo;
    __shared__ ScoreSet sets[kScoreSets];
    __shared__ long long scan[kScoreWaves], found_at;
    __shared__ int found, last;
    const int lane = lane_id(), wave = wave_index();
    const int c = lane & 15, quarter = lane >> 4;
    const int G = a.Hq / a.Hkv;
    constexpr int kPos = FOUR ? 4 : 16;
    const int HS = FOUR ? (G + 3) >> 2 : G;             // sets of a position tile

    // The work of all tables end to end, cut into equal shares.  A block of 256 tokens costs its sets and
    // as much as kBlockUnits more for its keys; the own tokens' block i begins at its first position's set.
    constexpr int kBlockUnits = 8;
    const int own_step = kScoreBlock / kPos * HS;
    struct Table {
        int n, all, b_hi, b_lo, own;  // new tokens, sets, blocks
    };
    auto takes = [&](int n) { return n > 0 && (a.all_lengths || !score_short(n, G)); };
    auto table_of = [&](int t) {
        const int n = new_tokens(a, t / a.Hkv);
        Table x{n, (n + kPos - 1) / kPos * HS, 0, 0, 0};
        if (takes(n)) {
            const SecLens len = section_lens<LI>(a, t);
            x.b_hi = (len.hi + kScoreBlock - 1) / kScoreBlock;
            x.b_lo = (len.lo + kScoreBlock - 1) / kScoreBlock;
            x.own = (n + kScoreBlock - 1) / kScoreBlock;
        }
        return x;
    };
    auto units_to = [&](const Table& x, int blocks) -> long long {
        const long long cached = min(blocks, x.b_hi + x.b_lo), own = blocks - cached;
        return (cached + own) * (x.all + kBlockUnits) - own * (own - 1) / 2 * own_step;
    };
    const int tables = a.B * a.Hkv, chunk = (tables + kScoreWaves * kWave - 1) / (kScoreWaves * kWave);
    const int t0 = min((int)threadIdx.x * chunk, tables), t1 = min(t0 + chunk, tables);
    long long mine = 0;
    for (int t = t0; t < t1; ++t) {
        const Table x = table_of(t);
        mine += units_to(x, x.b_hi + x.b_lo + x.own);
    }
    long long total_units;
    const long long mine_from = block_excl_scan_wide(mine, scan, &total_units);
    const long long quantum = max((total_units + gridDim.x - 1) / gridDim.x, 2ll * kBlockUnits);
    // consecutive shares on one XCD: they read the same tables
    const int share = gridDim.x % 8 == 0 ? ((int)blockIdx.x & 7) * ((int)gridDim.x >> 3) + ((int)blockIdx.x >> 3) : (int)blockIdx.x;
    const long long start = share * quantum, stop = min(total_units, start + quantum);
    const int first_n = first_tokens(a);
    int piece = 0;
    for (long long cur = start; cur < stop;) {
    // the table that has unit `cur`
    __syncthreads();
    if (cur >= mine_from && cur < mine_from + mine) {
        long long at = mine_from;
        for (int t = t0; t < t1; ++t) {
            const Table x = table_of(t);
            const long long next = at + units_to(x, x.b_hi + x.b_lo + x.own);
            if (cur < next) {
                found = t;
                found_at = at;
                break;
            }
            at = next;
        }
    }
    __syncthreads();
    const int t = __builtin_amdgcn_readfirstlane(found);
    const long long table_at = read_lane<long long>(found_at, 0);
    const Table tb = table_of(t);
    const int blocks = tb.b_hi + tb.b_lo + tb.own;
    int blk = 0;
    for (int above = blocks - 1; blk < above;) {  // the last block that starts at or before cur
        const int mid = (blk + above + 1) >> 1;
        if (table_at + units_to(tb, mid) <= cur) blk = mid;
        else above = mid - 1;
    }
    SeqBlock sb;
    sb.b = t / a.Hkv;
    sequence_rows(a, sb, first_n);
    const int n = sb.n, h = t - sb.b * a.Hkv;
    const int first = a.seq_len[sb.b];
    const SecLens lens = section_lens<LI>(a, t);
    const int len_hi = lens.hi, len_lo = lens.lo;
    const int b_hi = tb.b_hi, b_lo = tb.b_lo;
    const int all = (n + kPos - 1) / kPos * HS;
    const int32_t* table = a.page_table + (long long)t * a.p_max;
    // set i on its way into LDS; its rows' normalizers and slopes (row c's)
    float row_lse = 0.0f, row_slope = 0.0f;
    auto load_set = [&](int i, ScoreSet& S) {
        const int ln = fresh(lane), c = ln & 15;
        const int pt = i / HS, hs = i - pt * HS, j0 = kPos * pt;
        const int j = j0 + (FOUR ? c >> 2 : 4 * (c & 3) + (c >> 2)), g = FOUR ? 4 * hs + (c & 3) : hs;
        const bool there = j < n && g < G;
        const int jj = there ? j : j0, hq = h * G + (there ? g : 0);
        score_load(S, a.q + (sb.row0 + j0) * a.q_stride, 2 * ((jj - j0) * (int)a.q_stride + hq * kD), ln >> 4);
        row_lse = there ? a.lse_in[(sb.row0 + jj) * a.Hq + hq] * (MOD ? 1.0f : kChunkLog2e) : INFINITY;
        if constexpr (MOD) row_slope = a.slopes ? a.slopes[hq] : 0.0f;
    };
    for (; blk < blocks && cur < stop; ++blk, ++piece) {
        const long long from = table_at + units_to(tb, blk), to = table_at + units_to(tb, blk + 1);
        const long long piece_from = cur, piece_end = min(stop, to);
        cur = piece_end;
        if (!takes(n)) continue;  // (lengths that do not sum to total_new)
        const int sec = blk < b_hi ? 0 : (blk < b_hi + b_lo ? 1 : 2);
        const int len = sec == 0 ? len_hi : (sec == 1 ? len_lo : n);
        const int tok0 = (blk - (sec == 0 ? 0 : (sec == 1 ? b_hi : b_hi + b_lo))) * kScoreBlock + wave * kScoreTokens;
        const bool idle = tok0 >= len;
        h8 K[kScoreTiles][kNG], meta[kScoreTiles];
        float s[kScoreTiles][kNG];
        int pos[kScoreTiles];
        float* where = nullptr;  // the score of token (tile = quarter, c), which lanes of quarters 0 and 1 finish
        int where_pos = 0;
        float old = 0.0f;
        const int token = tok0 + lane;
        if (!idle && sec == 2) {
#pragma unroll
            for (int kt = 0; kt < kScoreTiles; ++kt) {
                const uint16_t* row = a.k + (sb.row0 + min(tok0 + 16 * kt + c, n - 1)) * a.k_stride + h * kD + quarter * 8;
#pragma unroll
                for (int g = 0; g < kNG; ++g) {
                    K[kt][g] = *reinterpret_cast<const h8*>(row + g * kG);
                    s[kt][g] = 0x1p-5f;
                }
                meta[kt] = __builtin_bit_cast(h8, u4{0, 0, 0, 0});
                pos[kt] = first + tok0 + 16 * kt + c;
            }
            if (token < n && quarter < kScoreTiles) where = a.score + (sb.row0 + token) * a.Hkv + h;
            where_pos = first + token;
        } else if (!idle) {
            auto take = [&](auto kb, auto vb, auto tt) {
                constexpr int KB = decltype(kb)::value, VB = decltype(vb)::value, T = decltype(tt)::value;
                constexpr SecOffsets O = sec_offsets(KvFmt{KB, VB, T});
                constexpr int kPer = T / 16;  // tiles of a page
                constexpr int kIds = kScoreTiles / kPer;
                int id[kIds];
#pragma unroll
                for (int i = 0; i < kIds; ++i) {
                    const int page = min(tok0 / T + i, (len - 1) / T);
                    id[i] = __builtin_amdgcn_readfirstlane(table[sec == 0 ? page : a.p_max - 1 - page]);
                }
                int mine = id[0];
#pragma unroll
                for (int i = 1; i < kIds; ++i) mine = quarter / kPer == i ? id[i] : mine;
                {
                    // (an ID outside the pool reads page 0; its tokens' scores are not written)
                    const bool ok = (unsigned long long)(unsigned)mine < (unsigned long long)a.num_pages;
                    uint8_t* pg = a.pool_rw + (long long)(ok ? mine : 0) * a.page_bytes;
                    const int slot = 16 * (quarter % kPer) + c;
                    where_pos = *reinterpret_cast<const int32_t*>(pg + O.pos + slot * 4);
                    old = *reinterpret_cast<const float*>(pg + O.sc + slot * 4);
                    if (token < len && ok && quarter < kScoreTiles) where = reinterpret_cast<float*>(pg + O.sc + slot * 4);
                }
#pragma unroll
                for (int kt = 0; kt < kScoreTiles; ++kt) {
                    const int i = id[kt / kPer];
                    const bool ok = (unsigned long long)(unsigned)i < (unsigned long long)a.num_pages;
                    const __amdgpu_buffer_rsrc_t r = span(a.pool + (long long)(ok ? i : 0) * a.page_bytes, O.used);
                    const int slot = 16 * (kt % kPer) + c;
#pragma unroll
                    for (int g = 0; g < kNG; ++g) {
                        if constexpr (KB == 8) {
                            const u2 v = fetch<8>(r, ((quarter >> 1) * T + slot) * 16 + (quarter & 1) * 8, O.kc + 2 * g * T * 16);
                            K[kt][g] = key_codes8(v[0], v[1]);
                        } else {
                            K[kt][g] = key_codes4(fetch<4>(r, slot * 16 + quarter * 4, O.kc + g * T * 16));
                        }
                    }
                    meta[kt] = __builtin_bit_cast(h8, fetch<16>(r, slot * 16, O.km));
                    if constexpr (MOD) pos[kt] = (int)fetch<4>(r, slot * 4, O.pos);
                }
#pragma unroll
                for (int kt = 0; kt < kScoreTiles; ++kt)
#pragma unroll
                    for (int g = 0; g < kNG; ++g) s[kt][g] = 0x1p19f * key_unit<KB>() * (float)meta[kt][2 * g];
            };
            using std::integral_constant;
            if (sec == 0) take(integral_constant<int, hi.kb>{}, integral_constant<int, hi.vb>{}, integral_constant<int, hi.T>{});
            else take(integral_constant<int, lo.kb>{}, integral_constant<int, lo.vb>{}, integral_constant<int, lo.T>{});
        }
        float total[kScoreTiles] = {0.0f, 0.0f};
        constexpr int kTops = FOUR ? 1 : 4;
        float top[kScoreTiles][kTops];
        auto use = [&](int i, const ScoreSet& S) {
            const int pt = i / HS, hs = i - pt * HS;
            if (hs == 0) {
#pragma unroll
                for (int kt = 0; kt < kScoreTiles; ++kt)
#pragma unroll
                    for (int r = 0; r < kTops; ++r) top[kt][r] = -INFINITY;
            }
            const int j = kPos * pt + quarter;  // (+ 4 r with sixteen positions)
            score_use<FOUR, MOD>(S, a, K, meta, s, pos, first + j, top, quarter, lane);
            if (hs == HS - 1) {
#pragma unroll
                for (int kt = 0; kt < kScoreTiles; ++kt)
#pragma unroll
                    for (int r = 0; r < kTops; ++r) {
                        const float p = probability<MOD>(top[kt][r]);
                        // the chunk's own tokens are seen from their own positions on
                        total[kt] += sec != 2 || j + 4 * r >= tok0 + 16 * kt + c ? p : 0.0f;
                    }
            }
        };
        {
            // (own tokens: from the first tile that sees one of the workgroup's)
            const int low = sec == 2 ? (tok0 - wave * kScoreTokens) / kPos * HS : 0;
            // (cuts lie between position tiles: the maximum over the heads is not divided)
            auto cut = [&](long long units) { return low + (int)(max(units - kBlockUnits, 0ll) / HS) * HS; };
            // (never past the rows that are there, also where lengths do not sum to total_new)
            const int begin = cut(piece_from - from), end = piece_end == to ? all : min(cut(piece_end - from), all);
            // passes of kScorePass sets through three thirds of LDS: one is used, the next one's sums are
            // made, the one after is on its way (each set by one wave)
            const bool makes = wave < kScorePass;
            __syncthreads();
            if (makes && begin + wave < end) {
                load_set(begin + wave, sets[wave]);
                staged_ready();
                score_sums(sets[wave], row_lse, row_slope, c, quarter, lane);
            }
            if (makes && begin + kScorePass + wave < end) load_set(begin + kScorePass + wave, sets[kScorePass + wave]);
            staged_ready();
            __syncthreads();
            int third = 0;
            for (int i0 = begin; i0 < end; i0 += kScorePass) {
                const int second = third == 2 ? 0 : third + 1, next = second == 2 ? 0 : second + 1;
                if (makes && i0 + kScorePass + wave < end)
                    score_sums(sets[second * kScorePass + wave], row_lse, row_slope, c, quarter, lane);
                if (makes && i0 + 2 * kScorePass + wave < end)
                    load_set(i0 + 2 * kScorePass + wave, sets[next * kScorePass + wave]);
                if (!idle)
                    for (int i = i0; i < min(i0 + kScorePass, end); ++i) use(i, sets[third * kScorePass + i - i0]);
                third = second;
                staged_ready();
                __syncthreads();
            }
        }
        float x = xsum4(total[0], total[1], 0.0f, 0.0f);  // quarter r: tile r's
        if (piece_from != from || piece_end != to) {
                // cut by a share's end: the pieces' sums are added by the last of them, in order (slots and
                // words as in chunk_tiles)
                auto part_of = [&](int k, bool first_piece) {
                    return a.part + (2ll * k + (first_piece ? 0 : 1)) * kScoreBlock + wave * kScoreTokens + (lane & 31);
                };
                const int k0 = (int)(from / quantum), k1 = (int)((to - 1) / quantum);
                if (lane < kScoreTokens) __hip_atomic_store(part_of(share, piece == 0), x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                if (!split_last(a.arrive + k0, k1 - k0 + 1, &last)) continue;
                x = 0.0f;
                for (int k = k0; k <= k1; ++k)
                    x += __hip_atomic_load(part_of(k, k > k0 || from == k0 * quantum), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        if (where) {
            const int received = max(first + n - where_pos, 1);
            *where = sec == 2 ? x / (float)received : old + (x - (float)n * old) / (float)received;
        }
    }
    }
}

// The short chunks: at most kShortSets sets of four positions and heads, staged once for a workgroup's share
// of its table.  Each wave takes every eighth step of 32 tokens, the keys' half of its pages by way of LDS as
// in chunk_rows, the next step's on its way while one is computed.  Bound by memory.
// (4 query heads per KV head, 64 sequences over 2048 tokens, here / in passes of a longer chunk: 4 tokens 23 / 23 us,
// 8 26 / 60, 16 32 / 66.  Room for eight sets leaves one workgroup a CU less: 16 tokens 43, 32 tokens 60 / 88.)
template <int LI, bool MOD>
__global__ __launch_bounds__(kScoreWaves * kWave, 4) void chunk_scores_short(ChunkArgs a)
{
    constexpr KvFmt hi = kLayoutFmts[LI].hi, lo = kLayoutFmts[LI].lo;
    constexpr SecOffsets Oh = sec_offsets(hi), Ol = sec_offsets(lo);
    constexpr int kHi = (Oh.vc + 1023) / 1024 * 1024, kLo = (Ol.vc + 1023) / 1024 * 1024;  // a page's room
    constexpr int kSlot = (hi.T == 16 ? 2 : 1) * kHi > (lo.T == 16 ? 2 : 1) * kLo ? (hi.T == 16 ? 2 : 1) * kHi
                                                                                 : (lo.T == 16 ? 2 : 1) * kLo;
    struct Shared {
        uint8_t slot[kScoreWaves][kSlot];
        ScoreSet sets[kShortSets];
    };
    __shared__ __align__(1024) Shared sh;
    const int lane = lane_id(), wave = wave_index();
    const int c = lane & 15, quarter = lane >> 4;
    const int G = a.Hq / a.Hkv, HS = (G + 3) >> 2;
    const int item = (int)blockIdx.x / a.Hkv, h = (int)blockIdx.x - item * a.Hkv;
    SeqBlock sb;
    sb.b = item / a.splits;
    const int share = item - sb.b * a.splits;
    const int t = sb.b * a.Hkv + h;
    const SecLens len = section_lens<LI>(a, t);
    const int first = a.seq_len[sb.b], len_hi = len.hi, len_lo = len.lo;
    sequence_rows(a, sb, first_tokens(a));
    const int n = sb.n;
    if (n == 0 || !score_short(n, G)) return;
    const int s_hi = (len_hi + 31) >> 5, s_lo = (len_lo + 31) >> 5, steps = s_hi + s_lo + 1;  // (the last: own tokens)
    const int shares = min(a.splits, (steps + kScoreWaves - 1) / kScoreWaves);
    if (share >= shares) return;
    const int begin = (int)((long long)steps * share / shares), end = (int)((long long)steps * (share + 1) / shares);
    const int32_t* table = a.page_table + (long long)t * a.p_max;
    uint8_t* slot = sh.slot[wave];

    auto page_id = [&](int u, int part) {
        const bool high = u < s_hi;
        const int T = high ? hi.T : lo.T, len = high ? len_hi : len_lo, k = high ? u : u - s_hi;
        const int i = min(T == 16 ? 2 * k + part : k, (len + T - 1) / T - 1);
        const int id = __builtin_amdgcn_readfirstlane(table[high ? i : a.p_max - 1 - i]);
        return (unsigned long long)(unsigned)id < (unsigned long long)a.num_pages ? id : -1;  // (outside: reads page 0)
    };
    // the staged step: this lane's token (tile = quarter, c; quarters 0 and 1), its score and position
    float* where = nullptr;
    float old = 0.0f;
    int where_pos = 0;
    int pos[kScoreTiles] = {0, 0};
    auto stage = [&](int u, int id0, int id1) {
        const bool high = u < s_hi;
        const uint8_t* p0 = a.pool + (long long)(id0 < 0 ? 0 : id0) * a.page_bytes;
        const uint8_t* p1 = a.pool + (long long)(id1 < 0 ? 0 : id1) * a.page_bytes;
        if (high) {
            stage_page<Oh.vc>(slot, p0, lane);
            if (hi.T == 16) stage_page<Oh.vc>(slot + kHi, p1, lane);
        } else {
            stage_page<Ol.vc>(slot, p0, lane);
            if (lo.T == 16) stage_page<Ol.vc>(slot + kLo, p1, lane);
        }
        const bool two = high ? hi.T == 16 : lo.T == 16;
        const int tile = quarter & 1, id = two && tile ? id1 : id0;
        uint8_t* pg = a.pool_rw + (long long)(id < 0 ? 0 : id) * a.page_bytes;
        const int sl = two ? c : 16 * tile + c;
        where_pos = *reinterpret_cast<const int32_t*>(pg + (high ? Oh.pos : Ol.pos) + 4 * sl);
        float* at = reinterpret_cast<float*>(pg + (high ? Oh.sc : Ol.sc) + 4 * sl);
        old = *at;
        const int left = high ? len_hi - 32 * u : len_lo - 32 * (u - s_hi);
        where = quarter < 2 && id >= 0 && 16 * tile + c < left ? at : nullptr;
    };
    const int cached = min(end, s_hi + s_lo);
    int u = begin + wave;
    if (u < cached) stage(u, page_id(u, 0), page_id(u, 1));

    const int all = (n + 3) / 4 * HS;
    if (wave < all) {
        const int pt = wave / HS, hs = wave - pt * HS, j = 4 * pt + (c >> 2), g = 4 * hs + (c & 3);
        const bool there = j < n && g < G;
        const int jj = there ? j : 4 * pt, hq = h * G + (there ? g : 0);
        const long long row = sb.row0 + jj;
        const uint16_t* q = a.q + row * a.q_stride + hq * kD + quarter * 8;
        u4 x[kNG];
#pragma unroll
        for (int g4 = 0; g4 < kNG; ++g4) x[g4] = *reinterpret_cast<const u4*>(q + g4 * kG);
        const float lse = there ? a.lse_in[row * a.Hq + hq] * (MOD ? 1.0f : kChunkLog2e) : INFINITY;
        const float slope = MOD && a.slopes ? a.slopes[hq] : 0.0f;
        ScoreSet& S = sh.sets[wave];
#pragma unroll
        for (int g4 = 0; g4 < kNG; ++g4) S.q[g4][lane] = __builtin_bit_cast(h8, x[g4]);
        score_sums(S, lse, slope, c, quarter, lane);
    }
    __syncthreads();

    // a step's sums over all queries: quarter 0's for tile 0, quarter 1's for tile 1
    auto received = [&](const h8 (&K)[kScoreTiles][kNG], const h8 (&meta)[kScoreTiles], const float (&s)[kScoreTiles][kNG], int own) {
        float total[kScoreTiles] = {0.0f, 0.0f}, top[kScoreTiles][1];
        for (int i = 0; i < all; ++i) {
            const int pt = i / HS, hs = i - pt * HS, j = 4 * pt + quarter;
            if (hs == 0) top[0][0] = top[1][0] = -INFINITY;
            score_use<true, MOD>(sh.sets[i], a, K, meta, s, pos, first + j, top, quarter, lane);
            if (hs == HS - 1) {
#pragma unroll
                for (int kt = 0; kt < kScoreTiles; ++kt) {
                    const float p = probability<MOD>(top[kt][0]);
                    total[kt] += own < 0 || j >= own + 16 * kt + c ? p : 0.0f;
                }
            }
        }
        return xsum4(total[0], total[1], 0.0f, 0.0f);
    };
    int n0 = 0, n1 = 0;
    while (u < cached) {
        const int next = u + kScoreWaves;
        if (next < cached) {
            n0 = page_id(next, 0);
            n1 = page_id(next, 1);
        }
        staged_ready();
        h8 K[kScoreTiles][kNG], meta[kScoreTiles];
        float s[kScoreTiles][kNG];
        auto take = [&](auto kb, auto vb, auto tt, int page) {
            constexpr int KB = decltype(kb)::value, VB = decltype(vb)::value, T = decltype(tt)::value;
            constexpr SecOffsets O = sec_offsets(KvFmt{KB, VB, T});
#pragma unroll
            for (int kt = 0; kt < kScoreTiles; ++kt) {
                const uint8_t* pg = slot + (T == 16 ? kt * page : 0);
                const int sl = T == 16 ? c : 16 * kt + c;
#pragma unroll
                for (int g = 0; g < kNG; ++g) {
                    if constexpr (KB == 8) {
                        const u2 v = *reinterpret_cast<const u2*>(pg + O.kc + ((2 * g + (quarter >> 1)) * T + sl) * 16 + (quarter & 1) * 8);
                        K[kt][g] = key_codes8(v[0], v[1]);
                    } else {
                        K[kt][g] = key_codes4(*reinterpret_cast<const uint32_t*>(pg + O.kc + (g * T + sl) * 16 + quarter * 4));
                    }
                }
                meta[kt] = *reinterpret_cast<const h8*>(pg + O.km + sl * 16);
#pragma unroll
                for (int g = 0; g < kNG; ++g) s[kt][g] = 0x1p19f * key_unit<KB>() * (float)meta[kt][2 * g];
            }
        };
        using std::integral_constant;
        if (u < s_hi) take(integral_constant<int, hi.kb>{}, integral_constant<int, hi.vb>{}, integral_constant<int, hi.T>{}, kHi);
        else take(integral_constant<int, lo.kb>{}, integral_constant<int, lo.vb>{}, integral_constant<int, lo.T>{}, kLo);
        float* at = where;
        const float before = old;
        const int at_pos = where_pos;
        if constexpr (MOD) {  // every quarter's lane c needs the positions of its two tokens
            pos[0] = __shfl(at_pos, c);
            pos[1] = __shfl(at_pos, 16 + c);
        }
        staged_read();
        if (next < cached) stage(next, n0, n1);
        const float x = received(K, meta, s, -1);
        if (at) *at = before + (x - (float)n * before) / (float)max(first + n - at_pos, 1);
        u = next;
    }
    if (u == s_hi + s_lo && u < end) {  // (one wave of one share) the chunk's own tokens, at most 16
        h8 K[kScoreTiles][kNG], meta[kScoreTiles];
        float s[kScoreTiles][kNG];
#pragma unroll
        for (int kt = 0; kt < kScoreTiles; ++kt) {
            const uint16_t* row = a.k + (sb.row0 + min(16 * kt + c, n - 1)) * a.k_stride + h * kD + quarter * 8;
#pragma unroll
            for (int g = 0; g < kNG; ++g) {
                K[kt][g] = *reinterpret_cast<const h8*>(row + g * kG);
                s[kt][g] = 0x1p-5f;
            }
            meta[kt] = __builtin_bit_cast(h8, u4{0, 0, 0, 0});
            pos[kt] = first + 16 * kt + c;
        }
        const float x = received(K, meta, s, 0);
        if (lane < n) a.score[(sb.row0 + lane) * a.Hkv + h] = x / (float)(n - lane);
    }
}

}  // namespace dkv

// Kernel entry points of layout n: which = 0 scores (sets of 16 positions), 4 (of 4 positions and
// heads), 5 (of short chunks), 1 / 2 attention of few rows with that many row tiles, 3 of many.
#define DKV_CHUNK_KERNELS(LI)                                                                                  \
    const void* chunk_kernel_l##LI(int which, bool mod)                                                        \
    {                                                                                                          \
        switch (which) {                                                                                       \
        case 0: return mod ? (const void*)chunk_scores<LI, false, true> : (const void*)chunk_scores<LI, false, false>; \
        case 4: return mod ? (const void*)chunk_scores<LI, true, true> : (const void*)chunk_scores<LI, true, false>; \
        case 5: return mod ? (const void*)chunk_scores_short<LI, true> : (const void*)chunk_scores_short<LI, false>; \
        case 1: return mod ? (const void*)chunk_rows<LI, 1, true> : (const void*)chunk_rows<LI, 1, false>;     \
        case 2: return mod ? (const void*)chunk_rows<LI, 2, true> : (const void*)chunk_rows<LI, 2, false>;     \
        case 3: return mod ? (const void*)chunk_tiles<LI, true> : (const void*)chunk_tiles<LI, false>;         \
        default: return nullptr;                                                                               \
        }                                                                                                      \
    }
