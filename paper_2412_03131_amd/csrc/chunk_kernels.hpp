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

// What a lane (column c = lane % 16, quarter = lane / 16) holds of a step.
template <int KB, int VB, int T>
struct StepRaw {
    static constexpr int kPieces = T == 16 ? 2 : 1;  // value code pieces per dim: one per page
    uint32_t kc[2][kNG][KB / 4];  // key codes of token m = c, its quarter of each group
    u4 km[2];                     // its {s, z} of four groups
    uint32_t vc[kPieces][8];      // value codes of dims 16 dt + c, the quarter's tokens
    u4 vm[2][kNG];                // {s, z} of the quarter's four tokens, per group
    int4 pos[2];                  // their positions
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
__device__ __forceinline__ void load_step(StepRaw<KB, VB, T>& r, const uint8_t* pg0, const uint8_t* pg1, int c, int quarter)
{
    constexpr SecOffsets O = sec_offsets(KvFmt{KB, VB, T});
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const uint8_t* pg = T == 16 && t == 1 ? pg1 : pg0;
        const int slot = step_slot<T>(t, c);
#pragma unroll
        for (int g = 0; g < kNG; ++g) {
            if constexpr (KB == 8) {
                const u2 v = *reinterpret_cast<const u2*>(pg + O.kc + ((2 * g + (quarter >> 1)) * T + slot) * 16 + (quarter & 1) * 8);
                r.kc[t][g][0] = v[0];
                r.kc[t][g][1] = v[1];
            } else {
                r.kc[t][g][0] = *reinterpret_cast<const uint32_t*>(pg + O.kc + (g * T + slot) * 16 + quarter * 4);
            }
        }
        r.km[t] = *reinterpret_cast<const u4*>(pg + O.km + slot * 16);
        const int first = step_slot<T>(t, 4 * quarter);
#pragma unroll
        for (int g = 0; g < kNG; ++g) r.vm[t][g] = *reinterpret_cast<const u4*>(pg + O.vm + (g * T + first) * 4);
        if constexpr (MOD) r.pos[t] = *reinterpret_cast<const int4*>(pg + O.pos + first * 4);
        if (t < StepRaw<KB, VB, T>::kPieces) {
            constexpr int row = T * VB / 8, piece = (T == 16 ? 4 : 8) * VB / 8;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt)
                r.vc[t < StepRaw<KB, VB, T>::kPieces ? t : 0][dt] =
                    load_value_codes<VB, T>(pg + O.vc + (16 * dt + c) * row + quarter * piece);
        }
    }
}

// Four value codes of a tile (the low 4 VB bits of w) -> s c + z as fp16 pairs of tokens
// (0, 2) and (1, 3).  A code is read as 1024 + c (its bits under the exponent of
// 1024, exact), the second pair as 1024 + 2^VB c; two packed steps give c and s c + z, the
// only rounding (2^-11: values N(0, 1) of a kept token, far below their own quantization).
template <int VB>
__device__ __forceinline__ void value_pairs(uint32_t w, h2 s02, h2 z02, h2 s13, h2 z13, uint32_t& p02, uint32_t& p13)
{
    const h2 m1024 = {(_Float16)-1024.0f, (_Float16)-1024.0f};
    h2 y02, y13;
    if constexpr (VB == 8) {
        y02 = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, 0x04020400u)) + m1024;
        y13 = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030401u)) + m1024;
    } else {
        constexpr uint32_t m = ((1u << VB) - 1) * 0x00010001u;
        const uint32_t x = VB == 4 ? __builtin_amdgcn_perm(0u, w, 0x0C010C00u) : (w | (w << (16 - 2 * VB)));
        const h2 inv = {(_Float16)(1.0f / (1 << VB)), (_Float16)(1.0f / (1 << VB))};
        const h2 off = {(_Float16)(-1024.0f / (1 << VB)), (_Float16)(-1024.0f / (1 << VB))};
        y02 = __builtin_bit_cast(h2, (x & m) | 0x64006400u) + m1024;
        y13 = __builtin_elementwise_fma(__builtin_bit_cast(h2, (x & (m << VB)) | 0x64006400u), inv, off);
    }
    p02 = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(s02, y02, z02));
    p13 = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(s13, y13, z13));
}

// The rows a wave works on: 16 RT of them, column c of tile rt is row 16 rt + c of its block.
template <int RT>
struct Rows {
    h8 q[RT][kNG];
    h8 sums[RT];
    float unit[RT];   // logit = unit * product sum (log2 units, or natural ones with a cap)
    int p[RT];        // position in the sequence
    ScoreForm form[RT];
    float m[RT], l[RT];
    f4 acc[RT][8];    // O^T: dims 16 dt + 4 quarter + r of row c
};

// One step's scores against the running softmax: logits x[rt][t][r] of tokens (t, 4 quarter + r)
// -> weights 2^(x - m) as fp16 pairs (0, 2), (1, 3) of both tiles.  The running max is raised
// only when a logit passes it by 8 (weights up to 2^8).
template <int RT>
__device__ __forceinline__ void softmax_step(Rows<RT>& R, float (&x)[RT][2][4], h8 (&P)[RT])
{
    bool raise = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float top = x[rt][0][0];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, x[rt][t][r]);
        raise |= top > R.m[rt] + 8.0f;
    }
    if (__any(raise)) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float top = x[rt][0][0];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, x[rt][t][r]);
            top = fmaxf(R.m[rt], rows_max(top));
            const float f = __builtin_amdgcn_exp2f(R.m[rt] - top);
            R.m[rt] = top;
            R.l[rt] *= f;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) R.acc[rt][dt] *= f;
        }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        u4 bits;
        float sum = 0.0f;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float w[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                w[r] = __builtin_amdgcn_exp2f(x[rt][t][r] - R.m[rt]);
                x[rt][t][r] = w[r];
                sum += w[r];
            }
            const h2 a = {(_Float16)w[0], (_Float16)w[2]}, b = {(_Float16)w[1], (_Float16)w[3]};
            bits[2 * t] = __builtin_bit_cast(uint32_t, a);
            bits[2 * t + 1] = __builtin_bit_cast(uint32_t, b);
        }
        R.l[rt] += sum;
        P[rt] = __builtin_bit_cast(h8, bits);
    }
}

// A step of cached tokens; those with index >= left (in the step, by token) and those of tile t where
// bit t of `bad` is set (a page ID outside the pool) do not exist.
template <int KB, int VB, int T, int RT, bool MOD>
__device__ __forceinline__ void cached_step(Rows<RT>& R, const StepRaw<KB, VB, T>& raw, int left, uint32_t bad,
                                            const ChunkArgs& a, int quarter)
{
    float x[RT][2][4];
    const h4 pick0 = {(_Float16)(quarter == 0 ? 32768.0f : 0.0f), (_Float16)0.0f, (_Float16)0.0f, (_Float16)0.0f};
    const h4 pick1 = {(_Float16)0.0f, (_Float16)0.0f, (_Float16)(quarter == 0 ? 32768.0f : 0.0f), (_Float16)0.0f};
    const f4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const h8 meta = __builtin_bit_cast(h8, raw.km[t]);
        const h4 m01 = {meta[0], meta[1], meta[2], meta[3]}, m23 = {meta[4], meta[5], meta[6], meta[7]};
        // 2^15 s of the quarter's four tokens, per group: a product with a unit vector
        f4 s[kNG];
        s[0] = mfma_k16(m01, pick0, zero);
        s[1] = mfma_k16(m01, pick1, zero);
        s[2] = mfma_k16(m23, pick0, zero);
        s[3] = mfma_k16(m23, pick1, zero);
        h8 k[kNG];
#pragma unroll
        for (int g = 0; g < kNG; ++g) {
            if constexpr (KB == 8) k[g] = key_codes8(raw.kc[t][g][0], raw.kc[t][g][1]);
            else k[g] = key_codes4(raw.kc[t][g][0]);
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            f4 sum = mfma_k32(meta, R.sums[rt], zero);
#pragma unroll
            for (int g = 0; g < kNG; ++g) {
                const f4 part = mfma_k32(k[g], R.q[rt][g], zero);
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[r] = __builtin_fmaf(s[g][r], part[r], sum[r]);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) x[rt][t][r] = sum[r] * R.unit[rt];
        }
        if constexpr (MOD) {
            const int pos[4] = {raw.pos[t].x, raw.pos[t].y, raw.pos[t].z, raw.pos[t].w};
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
    softmax_step<RT>(R, x, P);
#pragma unroll
    for (int g = 0; g < kNG; ++g) {
        h2 s02[2], z02[2], s13[2], z13[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            u4 m = raw.vm[t][g];
            if (!whole) {  // nothing behind a section's end reaches the sums
#pragma unroll
                for (int r = 0; r < 4; ++r) m[r] = (keep[t] >> r) & 1 ? m[r] : 0u;
            }
            s02[t] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(m[2], m[0], 0x05040100u));
            z02[t] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(m[2], m[0], 0x07060302u));
            s13[t] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(m[3], m[1], 0x05040100u));
            z13[t] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(m[3], m[1], 0x07060302u));
        }
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            const int dt = 2 * g + d;
            u4 v;
            uint32_t p, q;
            value_pairs<VB>(raw.vc[0][dt], s02[0], z02[0], s13[0], z13[0], p, q);
            v[0] = p;
            v[1] = q;
            value_pairs<VB>(T == 16 ? raw.vc[StepRaw<KB, VB, T>::kPieces - 1][dt] : raw.vc[0][dt] >> (4 * VB), s02[1], z02[1],
                            s13[1], z13[1], p, q);
            v[2] = p;
            v[3] = q;
            const h8 V = __builtin_bit_cast(h8, v);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) R.acc[rt][dt] = mfma_k32(V, P[rt], R.acc[rt][dt]);
        }
    }
}

// A step of the chunk's own tokens i0 .. i0 + 31 of n, keys at k, values at v (strides in halfs).
// first: position of token 0.
template <int RT, bool MOD>
__device__ __forceinline__ void own_step(Rows<RT>& R, const uint16_t* k, const uint16_t* v, int i0, int n, int first,
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
            const h8 kk = pair_order(raw[g]);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) sum[rt] = mfma_k32(kk, R.q[rt][g], sum[rt]);
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int token = i0 + step_slot<32>(t, 4 * quarter + r);
                const int away = R.p[rt] - first - token;
                float y = sum[rt][r] * (R.unit[rt] * 0x1p-9f);
                if constexpr (MOD) y = formed(y, R.form[rt], (float)away);
                x[rt][t][r] = away >= 0 && away < a.window ? y : -INFINITY;
            }
    }
    h8 P[RT];
    softmax_step<RT>(R, x, P);
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
    }
    // An infinite or NaN value must not reach the rows that do not see its token (0 * inf in a matrix
    // product): it entered as 0 above and is added here to those that do.
    if (__any(odd)) {
        for (int token = 0; token < 32 && i0 + token < n; ++token)
#pragma unroll
            for (int dt = 0; dt < 8; ++dt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t w = v[(long long)(i0 + token) * a.v_stride + 16 * dt + 4 * quarter + r];
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        float p = 0.0f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float pi = __shfl(x[rt][i >> 2][i & 3], c + 16 * (token >> 3));
                            p = (token & 7) == i ? pi : p;
                        }
                        const int away = R.p[rt] - first - (i0 + token);
                        if ((w & 0x7c00u) == 0x7c00u && away >= 0 && away < a.window) R.acc[rt][dt][r] += p * h2f(w);
                    }
                }
    }
}

// ---- attention: few rows, tokens split over waves and workgroups ------------------------
//
// A workgroup takes 16 RT rows of one (sequence, KV head) and its share of the table's steps
// (high pages, low pages, the chunk's own tokens), its four waves every fourth step each.  A
// wave holds its rows' queries as matrix operands and the transposed result O^T, so the
// scores of a step come out with a lane's values in one row and go into the second product as
// they lie: no exchange between lanes but the rare raise of the running max.  Pages go from memory
// to registers; a step's loads are in flight while the one before is computed.
constexpr int kChunkWaves = 4;

template <int LI, int RT, bool MOD>
__global__ __launch_bounds__(kChunkWaves * kWave, RT == 1 ? 2 : 1) void chunk_rows(ChunkArgs a)
{
    constexpr KvFmt hi = kLayoutFmts[LI].hi, lo = kLayoutFmts[LI].lo;
    constexpr int kRows = 16 * RT;
    __shared__ float lds_acc[kChunkWaves][16][kD + 4];
    __shared__ float lds_ml[kChunkWaves][2][16];
    set_fp16_saturate();
    const int lane = lane_id(), wave = wave_index();
    const int c = lane & 15, quarter = lane >> 4;
    const int G = a.Hq / a.Hkv;
    const int item = (int)blockIdx.x / a.splits, split = (int)blockIdx.x - item * a.splits;
    const int h = item % a.Hkv;
    const SeqBlock sb = find_block(a, item / a.Hkv, kRows, a.rows_lo, a.rows_hi);
    if (sb.b < 0) return;
    const int first = a.seq_len[sb.b];
    const int rows = sb.n * G, r0 = sb.blk * kRows;
    Rows<RT> R;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = min(r0 + 16 * rt + c, rows - 1);
        const int j = row / G, hq = h * G + row - j * G;
        const uint16_t* q = a.q + (sb.row0 + j) * a.q_stride + hq * kD + quarter * 8;
        u4 x[kNG];
#pragma unroll
        for (int g = 0; g < kNG; ++g) x[g] = *reinterpret_cast<const u4*>(q + g * kG);
        const RowOperands o = row_operands(x, quarter);
#pragma unroll
        for (int g = 0; g < kNG; ++g) R.q[rt][g] = o.q[g];
        R.sums[rt] = o.sums;
        R.unit[rt] = o.unit * a.scale;
        R.p[rt] = first + j;
        R.form[rt] = ScoreForm{a.cap_in, a.cap_out, MOD && a.slopes ? a.slopes[hq] * kChunkLog2e : 0.0f};
        R.m[rt] = kLowest;
        R.l[rt] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) R.acc[rt][dt] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int t = sb.b * a.Hkv + h;
    const int len_hi = a.len[2 * t], len_lo = a.len[2 * t + 1];
    const int last = min(r0 + kRows, rows) - 1;
    const int own = last / G + 1;  // tokens of the chunk that some row sees
    const int s_hi = (len_hi + 31) >> 5, s_lo = (len_lo + 31) >> 5, s_own = (own + 31) >> 5;
    const int steps = s_hi + s_lo + s_own;
    const int begin = (int)((long long)steps * split / a.splits), end = (int)((long long)steps * (split + 1) / a.splits);
    const int32_t* table = a.page_table + (long long)t * a.p_max;

    auto section = [&](auto kb, auto vb, auto tt, int sec, int from, int to, int len) {
        constexpr int KB = decltype(kb)::value, VB = decltype(vb)::value, T = decltype(tt)::value;
        const int pages = (len + T - 1) / T;
        // a step's page IDs; one outside the pool reads page 0 and counts no token
        auto page = [&](int k, bool& ok) {
            const int i = min(k, pages - 1);
            const int id = table[sec == 0 ? i : a.p_max - 1 - i];
            ok = (unsigned long long)(unsigned)id < (unsigned long long)a.num_pages;
            return a.pool + (long long)(ok ? id : 0) * a.page_bytes;
        };
        StepRaw<KB, VB, T> raw;
        for (int s = from + wave; s < to; s += kChunkWaves) {
            bool ok0, ok1 = true;
            const uint8_t* p0 = page(T == 16 ? 2 * s : s, ok0);
            const uint8_t* p1 = T == 16 ? page(2 * s + 1, ok1) : p0;
            load_step<KB, VB, T, MOD>(raw, p0, p1, c, quarter);
            const uint32_t bad = T == 16 ? (ok0 ? 0u : 1u) | (ok1 ? 0u : 2u) : (ok0 ? 0u : 3u);
            cached_step<KB, VB, T, RT, MOD>(R, raw, len - 32 * s, bad, a, quarter);
        }
    };
    using std::integral_constant;
    if (begin < s_hi)
        section(integral_constant<int, hi.kb>{}, integral_constant<int, hi.vb>{}, integral_constant<int, hi.T>{}, 0, begin,
                min(end, s_hi), len_hi);
    if (end > s_hi && begin < s_hi + s_lo)
        section(integral_constant<int, lo.kb>{}, integral_constant<int, lo.vb>{}, integral_constant<int, lo.T>{}, 1,
                max(begin - s_hi, 0), min(end - s_hi, s_lo), len_lo);
    {
        const uint16_t* k = a.k + sb.row0 * a.k_stride + h * kD;
        const uint16_t* v = a.v + sb.row0 * a.v_stride + h * kD;
        for (int s = max(begin - s_hi - s_lo, 0) + wave; s < end - s_hi - s_lo; s += kChunkWaves)
            own_step<RT, MOD>(R, k, v, 32 * s, own, first, a, c, quarter);
    }

    // the waves' states, 16 rows at a time
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float l = rows_sum(R.l[rt]);
        if (quarter == 0) {
            lds_ml[wave][0][c] = R.m[rt];
            lds_ml[wave][1][c] = l;
        }
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<f4*>(&lds_acc[wave][c][16 * dt + 4 * quarter]) = R.acc[rt][dt];
        __syncthreads();
        // 16 threads a row, eight dims each
        const int row = threadIdx.x >> 4, d = (threadIdx.x & 15) * 8;
        const int at = r0 + 16 * rt + row;
        float m = kLowest, sum = 0.0f, o[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kChunkWaves; ++w) m = fmaxf(m, lds_ml[w][0][row]);
#pragma unroll
        for (int w = 0; w < kChunkWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(lds_ml[w][0][row] - m);
            sum += f * lds_ml[w][1][row];
            const f4 x = *reinterpret_cast<const f4*>(&lds_acc[w][row][d]), y = *reinterpret_cast<const f4*>(&lds_acc[w][row][d + 4]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[i] += f * x[i];
                o[i + 4] += f * y[i];
            }
        }
        if (at < rows) {
            const int j = at / G, hq = h * G + at - j * G;
            const long long row_q = (sb.row0 + j) * a.Hq + hq;
            if (a.splits == 1) {
                const float inv = 1.0f / sum;
                h8 r;
#pragma unroll
                for (int i = 0; i < 8; ++i) r[i] = (_Float16)(o[i] * inv);
                *reinterpret_cast<h8*>(a.out + row_q * kD + d) = r;
                if (a.lse && (threadIdx.x & 15) == 0) a.lse[row_q] = kChunkLn2 * (m + __builtin_amdgcn_logf(sum));
            } else {
                float* part = a.part + (row_q * a.splits + split) * kChunkPart;
                *reinterpret_cast<f4*>(part + d) = f4{o[0], o[1], o[2], o[3]};
                *reinterpret_cast<f4*>(part + d + 4) = f4{o[4], o[5], o[6], o[7]};
                if ((threadIdx.x & 15) == 0) {
                    part[kD] = m;
                    part[kD + 1] = sum;
                }
            }
        }
        __syncthreads();
    }
}

// ---- scores ---------------------------------------------------------------------------------
//
// A wave takes 64 tokens of a table (or of the chunk's own), their keys in registers as matrix
// operands, and goes over all rows of the sequence: tiles of 16 positions, one query head after
// another, so that the maximum over the heads is between registers of one lane and one exp2
// serves all heads of a position.  A tile's queries pass through LDS for the workgroup's four waves.
// Position i of a tile is its row 4 (i % 4) + i / 4: a chunk of up to four positions needs
// only the first of a lane's four results.
constexpr int kScoreTokens = 64;                             // per wave
constexpr int kScoreBlock = kScoreTokens * kChunkWaves;      // per workgroup pass

template <int LI, bool MOD>
__global__ __launch_bounds__(kChunkWaves * kWave, 2) void chunk_scores(ChunkArgs a)
{
    constexpr KvFmt hi = kLayoutFmts[LI].hi, lo = kLayoutFmts[LI].lo;
    __shared__ __align__(16) h8 lds_q[2][kNG][kWave];   // one head's operands: [group][lane]
    __shared__ __align__(16) h8 lds_sum[2][kWave];
    __shared__ __align__(16) float lds_unit[2][16], lds_lse[2][16];
    const int lane = lane_id(), wave = wave_index();
    const int c = lane & 15, quarter = lane >> 4;
    const int G = a.Hq / a.Hkv;
    const int t = (int)blockIdx.x / a.shares, share = (int)blockIdx.x - t * a.shares;
    const int b = t / a.Hkv, h = t - b * a.Hkv;
    int n = 0;
    long long row0 = 0;
    if (a.max_new == 1 && a.total_new == a.B) {
        n = 1;
        row0 = b;
    } else {
        for (int b0 = 0; b0 <= b; b0 += kWave) {
            const int i = b0 + lane;
            int x = i <= b ? a.new_len[i] : 0;
            x = x < 0 ? 0 : (x > a.max_new ? a.max_new : x);
            const int incl = wave_incl_scan(x);
            const int lb = min(b - b0, kWave - 1);
            n = __builtin_amdgcn_readlane(x, lb);
            row0 += __builtin_amdgcn_readlane(incl, lb) - (b0 + kWave > b ? n : 0);
        }
        const long long room = a.total_new - row0;
        if (n > room) n = room > 0 ? (int)room : 0;
    }
    if (n == 0) return;
    const int first = a.seq_len[b];
    const int len_hi = a.len[2 * t], len_lo = a.len[2 * t + 1];
    const int b_hi = (len_hi + kScoreBlock - 1) / kScoreBlock, b_lo = (len_lo + kScoreBlock - 1) / kScoreBlock;
    const int blocks = b_hi + b_lo + (n + kScoreBlock - 1) / kScoreBlock;
    const int32_t* table = a.page_table + (long long)t * a.p_max;
    const f4 zero = {0.0f, 0.0f, 0.0f, 0.0f};

    for (int blk = share; blk < blocks; blk += a.shares) {
        const int sec = blk < b_hi ? 0 : (blk < b_hi + b_lo ? 1 : 2);
        const int len = sec == 0 ? len_hi : (sec == 1 ? len_lo : n);
        const int tok0 = (blk - (sec == 0 ? 0 : (sec == 1 ? b_hi : b_hi + b_lo))) * kScoreBlock + wave * kScoreTokens;
        h8 K[4][kNG];
        float s[4][kNG];
        h8 meta[4];
        int pos[4];
        float* where[4];
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
            const int token = tok0 + 16 * kt + c;
            where[kt] = nullptr;
            if (sec == 2) {
                const uint16_t* row = a.k + (row0 + min(token, n - 1)) * a.k_stride + h * kD + quarter * 8;
#pragma unroll
                for (int g = 0; g < kNG; ++g) {
                    K[kt][g] = pair_order(*reinterpret_cast<const u4*>(row + g * kG));
                    s[kt][g] = 0x1p-9f;
                }
                meta[kt] = __builtin_bit_cast(h8, u4{0, 0, 0, 0});
                pos[kt] = first + token;
                if (token < n && quarter == 0) where[kt] = a.score + (row0 + token) * a.Hkv + h;
                continue;
            }
            auto take = [&](auto kb, auto vb, auto tt) {
                constexpr int KB = decltype(kb)::value, VB = decltype(vb)::value, T = decltype(tt)::value;
                constexpr SecOffsets O = sec_offsets(KvFmt{KB, VB, T});
                const int tk = min(token, len - 1), page = tk / T, slot = tk - page * T;
                const int id = table[sec == 0 ? page : a.p_max - 1 - page];
                const bool ok = (unsigned long long)(unsigned)id < (unsigned long long)a.num_pages;
                uint8_t* pg = a.pool_rw + (long long)(ok ? id : 0) * a.page_bytes;
#pragma unroll
                for (int g = 0; g < kNG; ++g) {
                    if constexpr (KB == 8) {
                        const u2 v = *reinterpret_cast<const u2*>(pg + O.kc + ((2 * g + (quarter >> 1)) * T + slot) * 16 + (quarter & 1) * 8);
                        K[kt][g] = key_codes8(v[0], v[1]);
                    } else {
                        K[kt][g] = key_codes4(*reinterpret_cast<const uint32_t*>(pg + O.kc + (g * T + slot) * 16 + quarter * 4));
                    }
                }
                meta[kt] = *reinterpret_cast<const h8*>(pg + O.km + slot * 16);
#pragma unroll
                for (int g = 0; g < kNG; ++g) s[kt][g] = 32768.0f * (float)meta[kt][2 * g];
                pos[kt] = *reinterpret_cast<const int32_t*>(pg + O.pos + slot * 4);
                if (token < len && quarter == 0 && ok) where[kt] = reinterpret_cast<float*>(pg + O.sc + slot * 4);
            };
            using std::integral_constant;
            if (sec == 0) take(integral_constant<int, hi.kb>{}, integral_constant<int, hi.vb>{}, integral_constant<int, hi.T>{});
            else take(integral_constant<int, lo.kb>{}, integral_constant<int, lo.vb>{}, integral_constant<int, lo.T>{});
        }
        float total[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        // the chunk's own tokens are seen from their own positions on
        const int p_begin = sec == 2 ? (tok0 - wave * kScoreTokens) / 16 : 0;
        const int p_tiles = (n + 15) / 16;
        for (int pt = p_begin; pt < p_tiles; ++pt) {
            float top[4][4];
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int r = 0; r < 4; ++r) top[kt][r] = -INFINITY;
            for (int g0 = 0; g0 < G; ++g0) {
                const int buf = g0 & 1;
                const int hq = h * G + g0;
                __syncthreads();
                if (wave == 0) {
                    // row m = c of the tile is position 16 pt + 4 (c % 4) + c / 4
                    const int j = 16 * pt + 4 * (c & 3) + (c >> 2);
                    const uint16_t* q = a.q + (row0 + min(j, n - 1)) * a.q_stride + hq * kD + quarter * 8;
                    u4 x[kNG];
#pragma unroll
                    for (int g = 0; g < kNG; ++g) x[g] = *reinterpret_cast<const u4*>(q + g * kG);
                    const RowOperands o = row_operands(x, quarter);
#pragma unroll
                    for (int g = 0; g < kNG; ++g) lds_q[buf][g][lane] = o.q[g];
                    lds_sum[buf][lane] = o.sums;
                    if (quarter == 0) {
                        lds_unit[buf][c] = o.unit * a.scale;
                        lds_lse[buf][c] = j < n ? a.lse_in[(row0 + j) * a.Hq + hq] * kChunkLog2e : INFINITY;
                    }
                }
                __syncthreads();
                const f4 unit = *reinterpret_cast<const f4*>(&lds_unit[buf][4 * quarter]);
                const f4 lse = *reinterpret_cast<const f4*>(&lds_lse[buf][4 * quarter]);
                const ScoreForm form{a.cap_in, a.cap_out, MOD && a.slopes ? a.slopes[hq] * kChunkLog2e : 0.0f};
                h8 q[kNG];
#pragma unroll
                for (int g = 0; g < kNG; ++g) q[g] = lds_q[buf][g][lane];
                const h8 qs = lds_sum[buf][lane];
#pragma unroll
                for (int kt = 0; kt < 4; ++kt) {
                    f4 sum = mfma_k32(qs, meta[kt], zero);
#pragma unroll
                    for (int g = 0; g < kNG; ++g) {
                        const f4 part = mfma_k32(q[g], K[kt][g], zero);
#pragma unroll
                        for (int r = 0; r < 4; ++r) sum[r] = __builtin_fmaf(s[kt][g], part[r], sum[r]);
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float x;
                        if constexpr (MOD) {
                            const int away = first + 16 * pt + 4 * r + quarter - pos[kt];
                            x = formed(sum[r] * unit[r], form, (float)away) - lse[r];
                            x = away < a.window ? x : -INFINITY;
                        } else {
                            x = __builtin_fmaf(sum[r], unit[r], -lse[r]);
                        }
                        top[kt][r] = fmaxf(top[kt][r], x);
                    }
                }
            }
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int away = first + 16 * pt + 4 * r + quarter - pos[kt];
                    total[kt] += away >= 0 || sec != 2 ? __builtin_amdgcn_exp2f(top[kt][r]) : 0.0f;
                }
        }
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
            const float x = rows_sum(total[kt]);
            if (where[kt]) {
                if (sec == 2) {
                    *where[kt] = x / (float)(first + n - pos[kt]);
                } else {
                    const float old = *where[kt];
                    const int received = max(first + n - pos[kt], 1);
                    *where[kt] = old + (x - (float)n * old) / (float)received;
                }
            }
        }
    }
}

}  // namespace dkv

// Kernel entry points of layout n: which = 0 scores, 1 / 2 / 4 attention with that many row tiles.
#define DKV_CHUNK_KERNELS(LI)                                                                                  \
    const void* chunk_kernel_l##LI(int which, bool mod)                                                        \
    {                                                                                                          \
        switch (which) {                                                                                       \
        case 0: return mod ? (const void*)chunk_scores<LI, true> : (const void*)chunk_scores<LI, false>;       \
        case 1: return mod ? (const void*)chunk_rows<LI, 1, true> : (const void*)chunk_rows<LI, 1, false>;     \
        case 2: return mod ? (const void*)chunk_rows<LI, 2, true> : (const void*)chunk_rows<LI, 2, false>;     \
        case 4: return mod ? (const void*)chunk_rows<LI, 4, true> : (const void*)chunk_rows<LI, 4, false>;     \
        default: return nullptr;                                                                               \
        }                                                                                                      \
    }
