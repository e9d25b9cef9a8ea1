// k_block_attn.hip -- attention of new tokens over the uniform 8-bit cache, its tail and themselves.
//
// A sequence's query heads of one KV head are its rows: row r is query head h G + r % G of new token r / G, at
// position L + r / G.  Positions are cut in tiles of 32: the tiles below L / 32 are the cache's
// blocks, the others are fp16 rows (the tail's up to L, the call's own behind it).  A key at c is seen
// from p >= c if p - c < window or c < sinks.
//
// Scores come from v_mfma_f32_16x16x32_f16 with the keys as A operand (codes / 32 are fp16 values, exactly; the
// block's scale multiplies the fp32 sum), so a lane's eight scores of a tile lie in one row; their weights go into the
// second product as they lie, in two fp16 parts (2^-22), with the values as A operand.
// A value block's scale s enters the weights: u = exp2(x + log2 s - R) for a row's reference R, so that the
// products of all blocks add up as they are, and the normalizer takes u / s.  R is twelve below the
// largest exponent so far, which the next ones may pass by three before R is raised: fp16 (to 2^16, in steps of 2^-24 at
// its lower end) then holds 2^-37 of the largest weight.
#include "block_common.hpp"

namespace dkv {

namespace {

constexpr float kRefBelow = 12.0f, kRefRoom = 15.0f;  // log2 units

// The tiles that a sequence's new tokens see, in order: [0, sb) and [w0, last].
struct Tiles {
    int sb, w0, last;
    __device__ __forceinline__ int count() const { return sb + last + 1 - w0; }
    __device__ __forceinline__ int at(int step) const { return step < sb ? step : w0 + step - sb; }
};
__device__ __forceinline__ Tiles tiles_of(const BlockAttnArgs& a, int n, int L)
{
    Tiles t;
    t.last = (L + n - 1) / kBT;
    const int sb = a.sinks / kBT + (a.sinks % kBT != 0);
    t.sb = min(sb, t.last + 1);
    t.w0 = max(t.sb, max(0, L + 1 - a.window) / kBT);
    return t;
}

// ---- fp16 rows as operands -------------------------------------------------------------
// A tile of fp16 rows in LDS (16 KB): keys [2: token / 16][4: s = 2 i + w][4: r][16: token % 16][8 dims], dims
// (4 i + r) 16 + 8 w ..; values [4: u][2: j][4: r][16: dim][8 tokens], both as a block's codes are taken.  Tokens from
// `end` on are zero, and so are values that are not finite (0 * inf would reach the rows that do
// not see them): their tokens' bits go into *odd.
constexpr int kRowTileBytes = 4 * kBlockSide;

struct RowSource {
    const uint16_t* tail[2];  // keys, values: rows of positions % 32
    const uint16_t* own[2];   // rows of position L
    long long stride[2];
    int L, end;               // positions below L from the tail, up to end from the call
};
__device__ __forceinline__ const uint16_t* row_of(const RowSource& s, int side, int pos)
{
    return pos < s.L ? s.tail[side] + (pos & (kBT - 1)) * kD : s.own[side] + (long long)(pos - s.L) * s.stride[side];
}
// Pieces of a tile: keys 512 (token, 16 bytes), values 128 (r, four dims).
__device__ __forceinline__ void stage_key(const RowSource& s, int pos0, uint8_t* lds, int piece)
{
    const int c = piece & 15, token = piece >> 4;  // c: dims 8 c ..
    u4 x = {0, 0, 0, 0};
    if (pos0 + token < s.end) x = *reinterpret_cast<const u4*>(row_of(s, 0, pos0 + token) + c * 8);
    const int step = (c >> 3) * 2 + (c & 1), r = (c >> 1) & 3;
    *reinterpret_cast<u4*>(lds + (token >> 4) * 4096 + step * 1024 + r * 256 + (token & 15) * 16) = x;
}
__device__ __forceinline__ void stage_value(const RowSource& s, int pos0, uint8_t* lds, int piece, uint32_t* odd)
{
    const int dq = piece & 31, r = piece >> 5;  // dims 4 dq ..
    u2 x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int token = (e >> 2) * 16 + 4 * r + (e & 3);
        x[e] = u2{0, 0};
        if (pos0 + token < s.end) x[e] = *reinterpret_cast<const u2*>(row_of(s, 1, pos0 + token) + dq * 4);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t m0 = x[e][0] & 0x7fff7fffu, m1 = x[e][1] & 0x7fff7fffu;
        const bool bad = (m0 & 0xffffu) >= 0x7c00u || (m0 >> 16) >= 0x7c00u || (m1 & 0xffffu) >= 0x7c00u || (m1 >> 16) >= 0x7c00u;
        if (bad) {
            atomicOr(odd, 1u << ((e >> 2) * 16 + 4 * r + (e & 3)));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if ((x[e][i] & 0x7c00u) == 0x7c00u) x[e][i] &= 0xffff0000u;
                if ((x[e][i] & 0x7c000000u) == 0x7c000000u) x[e][i] &= 0xffffu;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        u4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            y[e] = __builtin_amdgcn_perm(x[2 * e + 1][i >> 1], x[2 * e][i >> 1], i & 1 ? 0x07060302u : 0x05040100u);
        const int dim = dq * 4 + i;
        *reinterpret_cast<u4*>(lds + 8192 + (dim >> 5) * 2048 + ((dim >> 4) & 1) * 1024 + r * 256 + (dim & 15) * 16) = y;
    }
}

// ---- few rows: a workgroup on 16 rows -------------------------------------------------
// Eight waves on the tiles of a piece, one tile each at a time; their states meet in LDS.  All (sequence, KV head, 16
// rows) are laid end to end by their tiles and cut into equal pieces, one for each workgroup; one that is
// split has its pieces' states joined by the last to arrive.
constexpr int kRowWaves = 8;
constexpr int kRowStart = 2;    // a 16-row block's start, in tiles
constexpr int kStaged = 4;      // tiles of fp16 rows in LDS at once

struct RowState {               // of a wave: lane = r * 16 + row
    f4 acc[8];                  // [u * 2 + j]: dims u 32 + j 16 + 4 r ..
    float ref, sum;             // reference (the same in all four lanes of a row), the lane's part of the normalizer
};

struct RowLds {
    union {
        uint8_t rows[kStaged * kRowTileBytes];
        float state[kRowWaves][16][kChunkPart];
    };
    float ref[kRowWaves][16], sum[kRowWaves][16];
    uint32_t odd[kStaged];
    int last;
};

// One tile's scores (natural units with a form, else log2) -> weights into the values' product.
struct RowTile {
    float ks;       // of the fp32 product: a code's unit, scales, without a form log2(e)
    float add;      // log2 of the values' scale (natural units with a form)
    float rs;       // 1 / the values' scale
    int pos0;
    bool whole;     // all rows see all 32 tokens
    int end;        // tokens from here on are not there
};

template <bool MOD>
__device__ __forceinline__ void row_weights(const BlockAttnArgs& a, const RowTile& t, const f4 (&s)[2], int p, const ScoreForm& form,
                                            RowState& st, h8& hi, h8& lo, float (&u)[8])
{
    const int r = lane_id() >> 4;
    float y[8], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = t.pos0 + (i >> 2) * 16 + 4 * r + (i & 3);
        if constexpr (MOD) {
            y[i] = formed(s[i >> 2][i & 3] * t.ks, form, (float)(p - c)) + t.add;
        } else {
            y[i] = __builtin_fmaf(s[i >> 2][i & 3], t.ks, t.add);
        }
        if (!t.whole) {
            const bool seen = c <= p && c < t.end && (p - c < a.window || c < a.sinks);
            y[i] = seen ? y[i] : -INFINITY;
        }
        top = fmaxf(top, y[i]);
    }
    constexpr float unit = MOD ? kChunkLn2 : 1.0f;
    if (__any(top > st.ref + kRefRoom * unit)) {
        const float now = rows_max(top);
        const float ref = now > st.ref + kRefRoom * unit ? now - kRefBelow * unit : st.ref;
        const float f = __builtin_amdgcn_exp2f((st.ref - ref) * (MOD ? kChunkLog2e : 1.0f));
        st.ref = ref;
        st.sum *= f;
#pragma unroll
        for (int i = 0; i < 8; ++i) st.acc[i] *= f;
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        u[i] = __builtin_amdgcn_exp2f(MOD ? (y[i] - st.ref) * kChunkLog2e : y[i] - st.ref);
        sum += u[i];
        hi[i] = (_Float16)u[i];
        lo[i] = (_Float16)(u[i] - (float)hi[i]);
    }
    st.sum = __builtin_fmaf(sum, t.rs, st.sum);
}

template <int FMT, bool MOD>
__global__ __launch_bounds__(64 * kRowWaves, 4) void block_rows(BlockAttnArgs a)
{
    __shared__ RowLds lds;
    const int lane = lane_id(), wave = wave_index(), r = lane >> 4, col = lane & 15;
    const auto loads = [&](int b, int& n, int& L) {
        n = a.new_len[b];
        L = seq_tokens(a, b);
    };
    // units of a sequence: 16-row blocks times their tiles and start
    const auto units = [&](int n, int L) {
        return n > 0 ? (long long)a.Hkv * (((long long)n * a.G + 15) / 16) * (tiles_of(a, n, L).count() + kRowStart) : 0LL;
    };
    const long long all = find_item(a.B, a.total_new, a.max_new, INT64_MAX, loads, units).items;
    long long share = (all + a.shares - 1) / a.shares;
    share = share < 16 ? 16 : share;
    long long x = (long long)blockIdx.x * share;
    const long long x_end = min(x + share, all);

    while (x < x_end) {
        const SeqItem sq = find_item(a.B, a.total_new, a.max_new, x, loads, units);
        if (sq.b < 0) break;
        const Tiles tl = tiles_of(a, sq.n, sq.L);
        const int steps = tl.count(), blk_units = steps + kRowStart;
        const int blocks = (int)(((long long)sq.n * a.G + 15) / 16);
        // 16-row block of the sequence: KV head major
        long long which = (x - sq.item0) / blk_units;
        const long long seq_end = sq.item0 + (long long)a.Hkv * blocks * blk_units;
        for (; x < x_end && x < seq_end; ++which) {
            const long long t0 = sq.item0 + which * blk_units;  // the block's first unit
            const int h = (int)(which / blocks), row_first = (int)(which - (long long)h * blocks) * 16;
            const int s0 = (int)max(x - t0 - kRowStart, 0LL);
            const int s1 = (int)(min(x_end, t0 + blk_units) - t0) - kRowStart;
            x = min(x_end, t0 + blk_units);
            if (s1 <= s0) continue;

            // this lane's row
            const int rows = (int)min((long long)sq.n * a.G - row_first, 16LL);
            const int row = row_first + min(col, rows - 1), token = row / a.G, hq = h * a.G + row % a.G, p = sq.L + token;
            h8 q[4];
            {
                const uint16_t* at = a.q + (sq.row0 + token) * a.q_stride + (long long)hq * kD;
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const h8*>(at + ((i >> 1) * 4 + r) * 16 + (i & 1) * 8);
            }
            ScoreForm form{0.0f, 0.0f, 0.0f};
            if constexpr (MOD) form = ScoreForm{a.cap_in, a.cap, a.slopes ? a.slopes[hq] : 0.0f};
            const int p_lo = sq.L + row_first / a.G, p_hi = sq.L + (row_first + rows - 1) / a.G;
            RowState st;
#pragma unroll
            for (int i = 0; i < 8; ++i) st.acc[i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
            st.ref = kLowest;
            st.sum = 0.0f;

            // steps of the cache's blocks, then those of fp16 rows
            const int blocks_held = sq.L / kBT;
            const int coded = blocks_held <= tl.sb ? min(blocks_held, tl.sb)
                                                   : min(max(blocks_held - tl.w0, 0) + tl.sb, steps);
            const int c1 = min(s1, coded);
            for (int base = s0; base < c1; base += kRowWaves * kWave) {
                // this wave's next 64 tiles: block IDs and scales, a lane each
                const int mine = base + wave + lane * kRowWaves;
                int id = -1;
                float ks = 0.0f, vs = 1.0f;
                if (mine < c1) id = block_id(a, sq.b, tl.at(mine));
                if (id >= 0) {
                    const float* sc = a.scale + ((long long)id * a.Hkv + h) * 2;
                    ks = sc[0];
                    vs = sc[1] * kCodeUnit;
                }
                const float rs = vs > 0.0f && vs < INFINITY ? 1.0f / vs : 1.0f;
                const float add = __builtin_amdgcn_logf(vs) * (MOD ? kChunkLn2 : 1.0f);
                ks *= kCodeUnit * a.scale_x;
                const int here = min(kWave, (c1 - base - wave + kRowWaves - 1) / kRowWaves);
                for (int i = 0; i < here; ++i) {
                    const int bid = __builtin_amdgcn_readlane(id, i);
                    if (bid < 0) continue;
                    RowTile t;
                    t.ks = read_lane_f(ks, i);
                    t.add = read_lane_f(add, i);
                    t.rs = read_lane_f(rs, i);
                    t.pos0 = tl.at(base + wave + i * kRowWaves) * kBT;
                    t.end = INT32_MAX;
                    t.whole = t.pos0 + kBT - 1 <= p_lo && (p_hi - t.pos0 < a.window || t.pos0 + kBT <= a.sinks);
                    const auto src = span(a.pool + ((long long)bid * a.Hkv + h) * kBlockBytes, kBlockBytes);
                    f4 s[2] = {f4{0.0f, 0.0f, 0.0f, 0.0f}, f4{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                        for (int i2 = 0; i2 < 2; ++i2) {
                            const u4 w = fetch<16>(src, lane * 16, (tt * 2 + i2) * 1024);
                            s[tt] = mfma_k32(codes8<FMT>(w[0], w[1]), q[i2 * 2], s[tt]);
                            s[tt] = mfma_k32(codes8<FMT>(w[2], w[3]), q[i2 * 2 + 1], s[tt]);
                        }
                    h8 hi, lo;
                    float u[8];
                    row_weights<MOD>(a, t, s, p, form, st, hi, lo, u);
#pragma unroll
                    for (int uu = 0; uu < 4; ++uu) {
                        const u4 w = fetch<16>(src, lane * 16, kBlockSide + uu * 1024);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const h8 v = codes8<FMT>(w[2 * j], w[2 * j + 1]);
                            st.acc[uu * 2 + j] = mfma_k32(v, hi, st.acc[uu * 2 + j]);
                            st.acc[uu * 2 + j] = mfma_k32(v, lo, st.acc[uu * 2 + j]);
                        }
                    }
                }
            }

            const int f0 = max(s0, coded);
            if (f0 < s1) {
                const uint16_t* tail = tail_rows(a, sq.b, h);
                const RowSource src{{tail, tail + kBlockSide},
                                    {a.k + sq.row0 * a.k_stride + h * kD, a.v + sq.row0 * a.v_stride + h * kD},
                                    {a.k_stride, a.v_stride}, sq.L, sq.L + sq.n};
                for (int base = f0; base < s1; base += kStaged) {
                    const int here = min(kStaged, s1 - base);
                    __syncthreads();
                    if (threadIdx.x < kStaged) lds.odd[threadIdx.x] = 0;
                    __syncthreads();
                    for (int piece = threadIdx.x; piece < here * 512; piece += 64 * kRowWaves)
                        stage_key(src, tl.at(base + piece / 512) * kBT, lds.rows + piece / 512 * kRowTileBytes, piece & 511);
                    for (int piece = threadIdx.x; piece < here * 128; piece += 64 * kRowWaves)
                        stage_value(src, tl.at(base + piece / 128) * kBT, lds.rows + piece / 128 * kRowTileBytes, piece & 127,
                                    &lds.odd[piece / 128]);
                    __syncthreads();
                    if (wave < here) {
                        const uint8_t* tile = lds.rows + wave * kRowTileBytes;
                        RowTile t;
                        t.ks = a.scale_x;
                        t.add = 0.0f;
                        t.rs = 1.0f;
                        t.pos0 = tl.at(base + wave) * kBT;
                        t.end = sq.L + sq.n;
                        t.whole = t.pos0 + kBT - 1 <= p_lo && (p_hi - t.pos0 < a.window || t.pos0 + kBT <= a.sinks);
                        f4 s[2] = {f4{0.0f, 0.0f, 0.0f, 0.0f}, f4{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
                        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                s[tt] = mfma_k32(*reinterpret_cast<const h8*>(tile + tt * 4096 + i * 1024 + lane * 16), q[i], s[tt]);
                        h8 hi, lo;
                        float u[8];
                        row_weights<MOD>(a, t, s, p, form, st, hi, lo, u);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const h8 v = *reinterpret_cast<const h8*>(tile + 8192 + i * 1024 + lane * 16);
                            st.acc[i] = mfma_k32(v, hi, st.acc[i]);
                            st.acc[i] = mfma_k32(v, lo, st.acc[i]);
                        }
                        // values that are not finite, to the rows that see their token
                        for (uint32_t odd = __builtin_amdgcn_readfirstlane(lds.odd[wave]); odd; odd &= odd - 1) {
                            const int token_odd = __builtin_ctz(odd), c = t.pos0 + token_odd;
                            const int from = ((token_odd & 15) >> 2) * 16 + col, reg = (token_odd >> 4) * 4 + (token_odd & 3);
                            float w = 0.0f;
#pragma unroll
                            for (int i = 0; i < 8; ++i) w = i == reg ? u[i] : w;
                            w = __shfl(w, from);
                            const bool seen = c <= p && (p - c < a.window || c < a.sinks);
                            const uint16_t* vr = row_of(src, 1, c);
#pragma unroll
                            for (int i = 0; i < 8; ++i)
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const float v = h2f(vr[(i >> 1) * 32 + (i & 1) * 16 + 4 * r + j]);
                                    if (seen && !(fabsf(v) < INFINITY)) st.acc[i][j] = __builtin_fmaf(w, v, st.acc[i][j]);
                                }
                        }
                    }
                }
            }

            // the waves' states
            st.sum = rows_sum(st.sum);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) *reinterpret_cast<f4*>(&lds.state[wave][col][(i >> 1) * 32 + (i & 1) * 16 + 4 * r]) = st.acc[i];
            if (r == 0) {
                lds.ref[wave][col] = st.ref;
                lds.sum[wave][col] = st.sum;
            }
            __syncthreads();
            const int my_row = threadIdx.x >> 5, dim = (threadIdx.x & 31) * 4;
            constexpr float to_log2 = MOD ? kChunkLog2e : 1.0f;
            float ref = kLowest, sum = 0.0f;
            f4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < kRowWaves; ++w) ref = fmaxf(ref, lds.ref[w][my_row]);
#pragma unroll
            for (int w = 0; w < kRowWaves; ++w) {
                const float f = __builtin_amdgcn_exp2f((lds.ref[w][my_row] - ref) * to_log2);
                sum = __builtin_fmaf(lds.sum[w][my_row], f, sum);
                acc += *reinterpret_cast<const f4*>(&lds.state[w][my_row][dim]) * f;
            }
            const auto finish = [&]() {
                if (my_row < rows) {
                    const int orow = row_first + my_row, otoken = orow / a.G, ohq = h * a.G + orow % a.G;
                    const long long at = (sq.row0 + otoken) * a.Hq + ohq;
                    const float inv = 1.0f / sum;
                    h4 y;
#pragma unroll
                    for (int j = 0; j < 4; ++j) y[j] = (_Float16)(acc[j] * inv);
                    *reinterpret_cast<h4*>(a.out + at * kD + dim) = y;
                    if (a.lse && dim == 0) a.lse[at] = MOD ? ref + __logf(sum) : (ref + __log2f(sum)) * kChunkLn2;
                }
            };
            const long long first_share = (t0 + kRowStart) / share, last_share = (t0 + blk_units - 1) / share;
            if (first_share == last_share) {
                finish();
                __syncthreads();
                continue;
            }
            // split: slot 1 of the share where the block starts, slot 0 of the others
            const auto slot = [&](long long sh) {
                return span(a.part + (sh * 2 + (sh == first_share ? 1 : 0)) * 16 * kChunkPart, 16 * kChunkPart * 4);
            };
            {
                const auto to = slot(blockIdx.x);
                put_quad(to, (my_row * kChunkPart + dim) * 4, 0, acc);
                if (dim == 0) put_quad(to, (my_row * kChunkPart + kD) * 4, 0, f4{ref, sum, 0.0f, 0.0f});
            }
            if (split_last(a.arrive + first_share, (int)(last_share - first_share) + 1, &lds.last)) {
                ref = kLowest;
                for (long long sh = first_share; sh <= last_share; ++sh)
                    ref = fmaxf(ref, get_quad(slot(sh), (my_row * kChunkPart + kD) * 4, 0)[0]);
                sum = 0.0f;
                acc = f4{0.0f, 0.0f, 0.0f, 0.0f};
                for (long long sh = first_share; sh <= last_share; ++sh) {
                    const auto from = slot(sh);
                    const f4 m = get_quad(from, (my_row * kChunkPart + kD) * 4, 0), part = get_quad(from, (my_row * kChunkPart + dim) * 4, 0);
                    const float f = __builtin_amdgcn_exp2f((m[0] - ref) * to_log2);
                    sum = __builtin_fmaf(m[1], f, sum);
                    acc += part * f;
                }
                finish();
            }
            __syncthreads();
        }
    }
}

}  // namespace

hipError_t launch_block_attention(const BlockAttnArgs& args, int format, bool mod, hipStream_t st)
{
    BlockAttnArgs a = args;
    a.shares = kBlockRowShares;
    void (*kernel)(BlockAttnArgs) = format == kE4m3 ? (mod ? block_rows<kE4m3, true> : block_rows<kE4m3, false>)
                                                    : (mod ? block_rows<kInt8, true> : block_rows<kInt8, false>);
    return launch1(kernel, kBlockRowShares, 64 * kRowWaves, st, a);
}

}  // namespace dkv
