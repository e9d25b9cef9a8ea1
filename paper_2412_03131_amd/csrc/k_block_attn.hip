// k_block_attn.hip -- attention of new tokens over the uniform 8-bit cache, its tail and themselves.
//
// A sequence's query heads of one KV head are its rows: row r is query head h G + r % G of new token r / G, at
// position L + r / G.  Positions are cut in tiles of 32: the tiles below L / 32 are the cache's
// blocks, the others are fp16 rows (the tail's up to L, the call's own behind it).  A key at c is seen
// from p >= c if p - c < window or c < sinks.
//
// Keys are the first product's A operand (codes / 32 are fp16 values, exactly; the block's scale multiplies the fp32 sum),
// so a lane's scores of a tile lie in one row; their weights go into the second product as they lie, in two fp16 parts
// (2^-22), with the values as A operand.  Sequences of few rows go to block_rows, the others to block_tiles.
// A value block's scale s enters the weights: u = exp2(x + log2 s - R) for a row's reference R, so that the
// products of all blocks add up as they are, and the normalizer takes u / s.  R is twelve below the
// largest exponent so far, which the next ones may pass by three before R is raised: fp16 (to 2^16, in steps of 2^-24 at
// its lower end) then holds 2^-37 of the largest weight.
#include "block_common.hpp"

namespace dkv {

namespace {

constexpr float kRefBelow = 12.0f, kRefRoom = 15.0f;  // log2 units

// ---- fp16 rows as operands -------------------------------------------------------------
// A tile of fp16 rows in LDS (16 KB): keys [2: token / 16][4: s = 2 i + w][4: r][16: token % 16][8 dims], dims
// (4 i + r) 16 + 8 w ..; values [4: u][2: j][4: r][16: dim][8 tokens], both as a block's codes are taken.  Tokens from
// `end` on are zero, and so are values that are not finite (0 * inf would reach the rows that do
// not see them): put_value returns their tokens' bits, and their products follow one by one.
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
// Pieces of a tile: keys 512 (token, eight dims), values 128 (r, four dims of r's eight tokens).
__device__ __forceinline__ void put_key(u4 x, uint8_t* lds, int piece)
{
    const int c = piece & 15, token = piece >> 4;  // c: dims 8 c ..
    const int step = (c >> 3) * 2 + (c & 1), r = (c >> 1) & 3;
    *reinterpret_cast<u4*>(lds + (token >> 4) * 4096 + step * 1024 + r * 256 + (token & 15) * 16) = x;
}
// Returns the bits of the tokens with values that are not finite among the wave's pieces.
__device__ __forceinline__ uint32_t put_value(u2 (&x)[8], uint8_t* values, int piece)
{
    const int dq = piece & 31, r = piece >> 5;  // dims 4 dq ..
    uint32_t bad = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            // (an exponent of ones: adding one there carries into the sign's place)
            const uint32_t full = ((x[e][i] & 0x7fff7fffu) + 0x04000400u) & 0x80008000u;
            bad |= full ? 1u << ((e >> 2) * 16 + 4 * r + (e & 3)) : 0u;
        }
    }
    uint32_t odd = 0;
    if (__any(bad != 0)) {
        odd = wave_or_u32(bad);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
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
        *reinterpret_cast<u4*>(values + (dim >> 5) * 2048 + ((dim >> 4) & 1) * 1024 + r * 256 + (dim & 15) * 16) = y;
    }
    return odd;
}
__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b)  // of two unsigned halves each
{
    typedef unsigned short us2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b)));
}
__device__ __forceinline__ u4 key_piece(const RowSource& s, int pos0, int piece)
{
    const int pos = pos0 + (piece >> 4);
    return pos < s.end ? *reinterpret_cast<const u4*>(row_of(s, 0, pos) + (piece & 15) * 8) : u4{0, 0, 0, 0};
}
__device__ __forceinline__ u2 value_piece(const RowSource& s, int pos0, int piece, int e)
{
    const int pos = pos0 + (e >> 2) * 16 + 4 * (piece >> 5) + (e & 3);
    return pos < s.end ? *reinterpret_cast<const u2*>(row_of(s, 1, pos) + (piece & 31) * 4) : u2{0, 0};
}

// A value that all lanes have alike, where the compiler has computed it in vector registers (quotients).
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// ---- scores to weights ----------------------------------------------------------------
// One tile's scores (natural units with a form, else log2) -> weights for the values' product.
struct TileScale {
    float ks;       // of the fp32 product: a code's unit, scales, without a form log2(e)
    float add;      // log2 of the values' scale (natural units with a form)
    float rs;       // 1 / the values' scale
    bool nan;       // a scale is NaN
};
struct TileView {
    int pos0, end;  // tokens from position `end` on are not there
    bool whole;     // all rows see all 32 tokens
};
// The steps whose tiles all rows at p_lo .. p_hi see whole: below `sinks`, or from `first` on, up to `last`.
struct TileRange {
    int sinks, first, last;
    __device__ __forceinline__ bool whole(int step) const { return (step < sinks || step >= first) && step <= last; }
};
__device__ __forceinline__ TileRange tile_range(const BlockAttnArgs& a, const Tiles& tl, int p_lo, int p_hi)
{
    TileRange r;
    r.sinks = min(a.sinks / kBT, tl.sb);
    // tiles that start behind p_hi - window, and those that end at p_lo or before
    const int from = (p_hi - a.window + kBT) >> 5, to = (p_lo + 1) / kBT - 1;
    r.first = tl.sb + max(0, from - tl.w0);
    r.last = to < tl.sb ? to : (to < tl.w0 ? tl.sb - 1 : to - tl.w0 + tl.sb);
    return r;
}
__device__ __forceinline__ float pairs_max(float v)  // over lanes l, l + 32
{
    auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ __forceinline__ float pairs_sum(float v)
{
    auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}

// N products of a lane (8: tiles of 16 rows, token (i / 4) 16 + 4 r + i % 4; 16: tiles of 32, token 8 (i / 4) + 4 half +
// i % 4) become weights in two steps: here forms, masks and the row's reference, with which acc, its sums of values, are raised.
// Hidden tokens' products become -inf at once, so that all tiles go one way from there.
template <bool MOD, int N, typename Acc, int A>
__device__ __forceinline__ void raise(const BlockAttnArgs& a, TileScale& t, const TileView& w, float (&y)[N], int p,
                                      const ScoreForm& form, Acc (&acc)[A], float& ref, float& sum)
{
    constexpr float unit = MOD ? kChunkLn2 : 1.0f;
    const int group = N == 8 ? lane_id() >> 4 : lane_id() >> 5;
    if (t.nan && __builtin_isnan(t.ks)) {  // (keys that read NaN, to the rows that see one of their tokens)
        t.ks = 1.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = __builtin_nanf("");
    }
    if constexpr (MOD) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = w.pos0 + (i >> 2) * (N == 8 ? 16 : 8) + 4 * group + (i & 3);
            y[i] = formed(y[i] * t.ks, form, (float)(p - c));
        }
    }
    if (!w.whole) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = w.pos0 + (i >> 2) * (N == 8 ? 16 : 8) + 4 * group + (i & 3);
            const bool seen = c <= p && c < w.end && (p - c < a.window || c < a.sinks);
            y[i] = seen ? y[i] : -INFINITY;
        }
    }
    float top = max3(y[0], y[1], y[2]);
#pragma unroll
    for (int i = 3; i + 1 < N; i += 2) top = max3(top, y[i], y[i + 1]);
    top = fmaxf(top, y[N - 1]);
    top = MOD ? top + t.add : __builtin_fmaf(top, t.ks, t.add);
    if (__any(top > ref + kRefRoom * unit)) {
        const float now = N == 8 ? rows_max(top) : pairs_max(top);
        const float up = now > ref + kRefRoom * unit ? now - kRefBelow * unit : ref;
        const float f = __builtin_amdgcn_exp2f((ref - up) * (MOD ? kChunkLog2e : 1.0f));
        ref = up;
        sum *= f;
#pragma unroll
        for (int i = 0; i < A; ++i) acc[i] *= f;
    }
}
// ... and here the exponents of 2.
template <bool MOD, int N>
__device__ __forceinline__ void exponents(const TileScale& t, float (&y)[N], float ref)
{
    const float less = t.add - ref;
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = MOD ? (y[i] + less) * kChunkLog2e : __builtin_fmaf(y[i], t.ks, less);
}
// Values that read NaN, to the rows that see one of their tokens: a NaN among a row's weights, behind their sum, reaches all of its
// sums of values and not its normalizer.
template <int N>
__device__ __forceinline__ void spoil(const BlockAttnArgs& a, const TileView& w, float (&y)[N], int p)
{
    if (w.whole || p - (w.pos0 + kBT - 1) < a.window || w.pos0 < a.sinks) y[0] = __builtin_nanf("");
}
// Weights as two fp16 parts, four at a time.
struct Parts {
    h8 hi, lo;
};
__device__ __forceinline__ Parts parts(float a, float b, float c, float d, float e, float f, float g, float h)
{
    const float u[8] = {a, b, c, d, e, f, g, h};
    u4 hi, lo;
    float minus = -1.0f;  // (hidden: a product that takes the half as it is, where a subtraction would convert it first)
    asm("" : "+s"(minus));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const h2 top = {(_Float16)u[2 * i], (_Float16)u[2 * i + 1]};
        hi[i] = __builtin_bit_cast(uint32_t, top);
        asm("" : "+v"(hi[i]));  // (else each half is converted once more by itself)
        const h2 back = __builtin_bit_cast(h2, (uint32_t)hi[i]);
        const h2 rest = {(_Float16)__builtin_fmaf((float)back.x, minus, u[2 * i]), (_Float16)__builtin_fmaf((float)back.y, minus, u[2 * i + 1])};
        lo[i] = __builtin_bit_cast(uint32_t, rest);
    }
    return Parts{__builtin_bit_cast(h8, hi), __builtin_bit_cast(h8, lo)};
}

// 64 steps of the cache from `first` on (below `end`), a lane each: their block's ID (-1: none), and its scales.
__device__ __forceinline__ int step_id(const BlockAttnArgs& a, const Tiles& tl, int b, int first, int end)
{
    const int step = first + lane_id();
    return step < end ? block_id(a, b, tl.at(step)) : -1;
}
struct StepScales {
    float ks, add, rs;
    unsigned long long nan;
    __device__ __forceinline__ TileScale at(int i) const
    {
        return TileScale{read_lane_f(ks, i), read_lane_f(add, i), read_lane_f(rs, i), ((nan >> i) & 1) != 0};
    }
};
template <bool MOD>
__device__ __forceinline__ StepScales step_scales(const BlockAttnArgs& a, int id, int h)
{
    float ks = 1.0f, vs = 1.0f;
    if (id >= 0) {
        const float* sc = a.scale + ((long long)id * a.Hkv + h) * 2;
        ks = sc[0];
        vs = sc[1];
    }
    StepScales s;
    vs *= kCodeUnit;
    s.nan = __ballot(__builtin_isnan(ks + vs));
    vs = __builtin_isnan(vs) ? kCodeUnit : vs;
    s.ks = ks * kCodeUnit * a.scale_x;
    s.add = __builtin_amdgcn_logf(vs) * (MOD ? kChunkLn2 : 1.0f);
    s.rs = vs > 0.0f && vs < INFINITY ? 1.0f / vs : 1.0f;
    return s;
}

__device__ __forceinline__ RowSource row_source(const BlockAttnArgs& a, const SeqItem& sq, int h)
{
    const uint16_t* tail = tail_rows(a, sq.b, h);
    return RowSource{{tail, tail + kBlockSide},
                     {a.k + sq.row0 * a.k_stride + h * kD, a.v + sq.row0 * a.v_stride + h * kD},
                     {a.k_stride, a.v_stride}, sq.L, sq.L + sq.n};
}
__device__ __forceinline__ auto lengths_of(const BlockAttnArgs& a)
{
    return [&a](int b, int& n, int& L) {
        n = a.new_len[b];
        L = seq_tokens(a, b);
    };
}
// Steps whose tiles are blocks of the cache: they come first.
__device__ __forceinline__ int coded_steps(const Tiles& tl, int L)
{
    const int held = L / kBT;
    return held <= tl.sb ? held : min(max(held - tl.w0, 0) + tl.sb, tl.count());
}

// ---- few rows: a wave on 16 rows ---------------------------------------------------------
// All (sequence, KV head, 16 rows) are laid end to end by their tiles and cut into equal pieces, one for each wave that the
// device holds; a block of rows that is split has its pieces' states joined by the last to arrive.  Waves of a SIMD do not run
// alike (the older is served first), so none waits for another: with pieces of eight waves that met in LDS, 64 ragged requests
// took 102 us, half of it at barriers.
//
// Bound by memory where there are many sequences.  A wave asks for a tile's keys again as soon as their codes are operands, and for
// its values likewise, so 8 KB of the next tile are always on their way.  64 single tokens over 1024 .. 4096, 32 / 8 heads: 73 us,
// 345 MB at 4.7 TB/s; two tiles ahead gained nothing, two row tiles for a wave took 41 us instead of 28 (24 requests' drafts over a
// window of 2048).
constexpr int kRowWaves = 4;    // of a workgroup
constexpr int kRowStart = 3;    // units of a block's start, in tiles of the cache
constexpr int kRowTile = 4;     // and of a tile of fp16 rows
constexpr int kQuads = 4;      // quads of a lane in a join
// Least units of a piece.  A block's pieces grow in number with its length, and one wave joins them all: short contexts want small
// pieces, lone long ones large ones.  (us with 6 / 12 / 24 / 48, one token, 32 / 8 heads) over 600 13.6 / 16.8 / 23.4 / 36.8, over 4096
// 28 / 22 / 27 / 40, over 32768 211 / 56 / 60 / 74; 64 tokens over 2560 69.9 / 69.9 / 71.0 / 98.
constexpr int kRowShare = 6;

template <int FMT, bool MOD>
__global__ __launch_bounds__(64 * kRowWaves, 2) void block_rows(BlockAttnArgs a)
{
    __shared__ uint8_t staged[kRowWaves][2 * kBlockSide];  // a wave's tile of fp16 values
    const int lane = lane_id(), wave = wave_index(), r = lane >> 4, col = lane & 15;
    // units of a sequence: those of its blocks of rows
    const auto block_units = [&](const Tiles& tl, int L) {
        const int coded = coded_steps(tl, L);
        return coded + (tl.count() - coded) * kRowTile + kRowStart;
    };
    const auto units = [&](int n, int L) {
        return n > 0 && n * a.G <= a.few_rows ? (long long)a.Hkv * ((n * a.G + 15) / 16) * block_units(tiles_of(a, n, L), L) : 0LL;
    };
    SeqScan scan(a.B, a.max_new, a.total_new, lengths_of(a), units);
    const long long all = scan.total();
    const int shares = (int)gridDim.x * kRowWaves;
    const long long share = max((all + shares - 1) / shares, (long long)kRowShare);
    // (workgroup i runs on XCD i % 8: pieces that follow each other share an L2)
    const int me = ((int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3)) * kRowWaves + wave;
    long long x = me * share;
    const long long x_end = min(x + share, all);

    while (x < x_end) {
        const SeqItem sq = scan.find(x);
        if (sq.b < 0) break;
        const Tiles tl = tiles_of(a, sq.n, sq.L);
        const int steps = tl.count(), coded = coded_steps(tl, sq.L), blk_units = block_units(tl, sq.L);
        const int blocks = (sq.n * a.G + 15) / 16;
        // steps that start before unit u of a block
        const auto step_at = [&](long long u) {
            const int v = (int)u - kRowStart;
            return v <= coded ? max(v, 0) : coded + (v - coded + kRowTile - 1) / kRowTile;
        };
        // block of the sequence: KV head major
        int which = uniform((int)((x - sq.item0) / blk_units));
        for (; x < x_end && which < a.Hkv * blocks; ++which) {
            const long long t0 = sq.item0 + (long long)which * blk_units;  // the block's first unit
            const int h = which / blocks, row_first = (which - h * blocks) * 16;
            const int s0 = uniform(step_at(x - t0)), s1 = uniform(step_at(min(x_end - t0, (long long)blk_units)));
            x = min(x_end, t0 + blk_units);
            if (s1 <= s0) continue;

            // this lane's row
            const int rows = min(sq.n * a.G - row_first, 16);
            const int row = row_first + min(col, rows - 1), token = row / a.G, hq = h * a.G + row % a.G, p = sq.L + token;
            const long long out_row = (sq.row0 + token) * a.Hq + hq;
            h8 q[4];
            {
                const uint16_t* at = a.q + (sq.row0 + token) * a.q_stride + (long long)hq * kD;
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const h8*>(at + ((i >> 1) * 4 + r) * 16 + (i & 1) * 8);
            }
            ScoreForm form{0.0f, 0.0f, 0.0f};
            if constexpr (MOD) form = ScoreForm{a.cap_in, a.cap, a.slopes ? a.slopes[hq] : 0.0f};
            const TileRange range = tile_range(a, tl, sq.L + row_first / a.G, sq.L + (row_first + rows - 1) / a.G);
            f4 acc[8];  // [u * 2 + j]: dims u 32 + j 16 + 4 r ..
            float ref = kLowest, sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
            // a tile's products -> weights
            const auto weigh = [&](const f4 (&s)[2], TileScale ts, int step, int end, float (&y)[8]) {
                TileView view{0, end, range.whole(step)};
                if (!view.whole || MOD) view.pos0 = tl.at(step) * kBT;
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = s[j >> 2][j & 3];
                raise<MOD>(a, ts, view, y, p, form, acc, ref, sum);
                exponents<MOD>(ts, y, ref);
                float total = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    y[j] = __builtin_amdgcn_exp2f(y[j]);
                    total += y[j];
                }
                sum = __builtin_fmaf(total, ts.rs, sum);
                if (ts.nan) spoil(a, view, y, p);
                return parts(y[0], y[1], y[2], y[3], y[4], y[5], y[6], y[7]);
            };

            // the cache's blocks
            const int c1 = min(s1, coded);
            for (int base = s0; base < c1; base += kWave) {
                const int id = step_id(a, tl, sq.b, base, c1);
                unsigned long long todo = __ballot(id >= 0);
                if (!todo) continue;
                int i = __builtin_ctzll(todo);
                const auto block = [&](int at) {
                    return span(a.pool + ((long long)__builtin_amdgcn_readlane(id, at) * a.Hkv + h) * kBlockBytes, kBlockBytes);
                };
                auto src = block(i);
                u4 k[4], v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) k[j] = fetch<16>(src, lane * 16, j * 1024);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = fetch<16>(src, lane * 16, kBlockSide + j * 1024);
                const StepScales scales = step_scales<MOD>(a, id, h);
                while (todo) {
                    todo &= todo - 1;
                    const int next = todo ? __builtin_ctzll(todo) : i;
                    src = block(next);
                    f4 s[2] = {f4{0.0f, 0.0f, 0.0f, 0.0f}, f4{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        s[j >> 2] = mfma_k32(codes8<FMT>(k[j >> 1][(j & 1) * 2], k[j >> 1][(j & 1) * 2 + 1]), q[j & 3], s[j >> 2]);
                    if (todo) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) k[j] = fetch<16>(src, lane * 16, j * 1024);
                    }
                    float y[8];
                    const Parts w = weigh(s, scales.at(i), base + i, INT32_MAX, y);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const h8 x8 = codes8<FMT>(v[j >> 1][(j & 1) * 2], v[j >> 1][(j & 1) * 2 + 1]);
                        acc[j] = mfma_k32(x8, w.hi, acc[j]);
                        acc[j] = mfma_k32(x8, w.lo, acc[j]);
                    }
                    if (todo) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] = fetch<16>(src, lane * 16, kBlockSide + j * 1024);
                    }
                    i = next;
                }
            }

            // rows in fp16: keys straight from their rows, values through LDS
#pragma unroll 1
            for (int step = max(s0, coded); step < s1; ++step) {
                const RowSource src = row_source(a, sq, h);
                const int pos0 = tl.at(step) * kBT;
                h8 k[8];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint16_t* at = row_of(src, 0, min(pos0 + j * 16 + col, src.end - 1)) + r * 16;
#pragma unroll
                    for (int i = 0; i < 4; ++i) k[j * 4 + i] = *reinterpret_cast<const h8*>(at + (i >> 1) * 64 + (i & 1) * 8);
                }
                uint32_t odd = 0;
                wave_lds_sync();  // (the last tile's values are read)
#pragma unroll 1
                for (int piece = lane; piece < 128; piece += kWave) {
                    u2 v8[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v8[e] = value_piece(src, pos0, piece, e);
                    odd |= put_value(v8, staged[wave], piece);
                }
                wave_lds_sync();
                f4 s[2] = {f4{0.0f, 0.0f, 0.0f, 0.0f}, f4{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j >> 2] = mfma_k32(k[j], q[j & 3], s[j >> 2]);
                float y[8];
                const Parts w = weigh(s, TileScale{a.scale_x, 0.0f, 1.0f, false}, step, src.end, y);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const h8 x8 = *reinterpret_cast<const h8*>(staged[wave] + j * 1024 + lane * 16);
                    acc[j] = mfma_k32(x8, w.hi, acc[j]);
                    acc[j] = mfma_k32(x8, w.lo, acc[j]);
                }
                // values that are not finite, to the rows that see their token
                for (odd = __builtin_amdgcn_readfirstlane(odd); odd; odd &= odd - 1) {
                    const int tok = __builtin_ctz(odd), c = pos0 + tok;
                    const int reg = (tok >> 4) * 4 + (tok & 3);
                    float wt = 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) wt = j == reg ? y[j] : wt;
                    wt = __shfl(wt, ((tok & 15) >> 2) * 16 + col);
                    const bool seen = c <= p && (p - c < a.window || c < a.sinks);
                    const uint16_t* vr = row_of(src, 1, c) + 4 * r;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const u2 w2 = *reinterpret_cast<const u2*>(vr + (j >> 1) * 32 + (j & 1) * 16);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float v1 = h2f((w2[e >> 1] >> ((e & 1) * 16)) & 0xffffu);
                            if (seen && !(fabsf(v1) < INFINITY)) acc[j][e] = __builtin_fmaf(wt, v1, acc[j][e]);
                        }
                    }
                }
            }

            constexpr float to_log2 = MOD ? kChunkLog2e : 1.0f;
            sum = rows_sum(sum);
            const int last_unit = steps > coded ? coded + (steps - 1 - coded) * kRowTile : steps - 1;
            const int first_share = uniform((int)((t0 + kRowStart) / share)), last_share = uniform((int)((t0 + kRowStart + last_unit) / share));
            if (first_share == last_share) {
                const float inv = 1.0f / sum;
                if (col < rows) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        h4 y;
#pragma unroll
                        for (int j = 0; j < 4; ++j) y[j] = (_Float16)(acc[i][j] * inv);
                        *reinterpret_cast<h4*>(a.out + out_row * kD + (i >> 1) * 32 + (i & 1) * 16 + 4 * r) = y;
                    }
                    if (a.lse && r == 0) a.lse[out_row] = MOD ? ref + __logf(sum) : (ref + __log2f(sum)) * kChunkLn2;
                }
                continue;
            }
            // split: slot 1 of the share where the block starts, slot 0 of the others.  A state: rows of sums, then a quad
            // {reference, sum, -, -} per row.
            const auto slot = [&](int sh) {
                return span(a.part + ((long long)sh * 2 + (sh == first_share ? 1 : 0)) * kRowPart, kRowPart * 4);
            };
            if (col < rows) {
                const auto to = slot(me);
#pragma unroll
                for (int i = 0; i < 8; ++i) put_quad(to, col * (kD * 4) + r * 16, (i >> 1) * 128 + (i & 1) * 64, acc[i]);
                if (r == 0) put_quad(to, 16 * kD * 4 + col * 16, 0, f4{ref, sum, 0.0f, 0.0f});
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            int arrived = 0;
            if (lane == 0) arrived = (int)arrive_count(a.arrive + first_share, call_tag());
            if (__builtin_amdgcn_readfirstlane(arrived) != last_share - first_share + 1) continue;
            // All of the block's pieces, in order: first every row's reference and normalizer (a lane a row), then the sums, a lane
            // a quad of dims of several rows, four pieces' asked for at once.
            const int my_row = min(lane, rows - 1);
            float top = kLowest, total = 0.0f;
#pragma unroll 1
            for (int sh = first_share; sh <= last_share; sh += 8) {
                f4 m[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) m[i] = get_quad(slot(min(sh + i, last_share)), 16 * kD * 4 + my_row * 16, 0);
                float up = top;
#pragma unroll
                for (int i = 0; i < 8; ++i) up = fmaxf(up, m[i][0]);
                total *= __builtin_amdgcn_exp2f((top - up) * to_log2);
                top = up;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (sh + i <= last_share) total = __builtin_fmaf(m[i][1], __builtin_amdgcn_exp2f((m[i][0] - top) * to_log2), total);
            }
            if (a.lse && lane < rows) {
                const int orow = row_first + lane;
                a.lse[(sq.row0 + orow / a.G) * a.Hq + h * a.G + orow % a.G] = MOD ? top + __logf(total) : (top + __log2f(total)) * kChunkLn2;
            }
#pragma unroll 1
            for (int first = 0; first < rows * 32; first += kQuads * kWave) {
                f4 out[kQuads];
                float up[kQuads];
                int at[kQuads];
#pragma unroll
                for (int i = 0; i < kQuads; ++i) {
                    at[i] = min(first + i * kWave + lane, rows * 32 - 1);
                    up[i] = __shfl(top, at[i] >> 5);
                    out[i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
                }
#pragma unroll 1
                for (int sh = first_share; sh <= last_share; sh += 4) {
                    f4 part[kQuads][4];
                    float m[kQuads][4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const auto from = slot(min(sh + j, last_share));
#pragma unroll
                        for (int i = 0; i < kQuads; ++i) {
                            m[i][j] = get_one(from, 16 * kD * 4 + (at[i] >> 5) * 16, 0);
                            part[i][j] = get_quad(from, at[i] * 16, 0);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (sh + j <= last_share) {
#pragma unroll
                            for (int i = 0; i < kQuads; ++i) out[i] += part[i][j] * __builtin_amdgcn_exp2f((m[i][j] - up[i]) * to_log2);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < kQuads; ++i) {
                    const float inv = 1.0f / __shfl(total, at[i] >> 5);
                    if (first + i * kWave + lane >= rows * 32) continue;
                    const int orow = row_first + (at[i] >> 5);
                    h4 y;
#pragma unroll
                    for (int j = 0; j < 4; ++j) y[j] = (_Float16)(out[i][j] * inv);
                    *reinterpret_cast<h4*>(a.out + ((sq.row0 + orow / a.G) * a.Hq + h * a.G + orow % a.G) * kD + (at[i] & 31) * 4) = y;
                }
            }
        }
    }
}

// ---- many rows: a workgroup on 128 rows -------------------------------------------------
// Four waves of 32 rows each go over the same tiles.  A tile is brought into LDS once, as fp16 operands (a block's
// codes are converted on the way), one step ahead of its use, and its loads are asked for a step before that.
// v_mfma_f32_32x32x16_f16: A lane l holds row l % 32, k 8 (l / 32) .. + 7, B the same with columns, C lane l in register i row
// 8 (i / 4) + i % 4 + 4 (l / 32) of column l % 32.
//
// All (sequence, KV head, 128 rows) are laid end to end and cut into equal shares, one for each workgroup; shares that follow
// each other run on one XCD, so that its L2 serves their tiles.
//
// Bound by issue, the matrix products before the rest: 2048 tokens over 8192, 64 / 8 heads, take 899 us, 689 TFLOP/s of the two
// products (867 to 970 us from card to card); the weights' second part adds half as many again (weights rounded once: 770 us, where
// this took 932).  A cap takes 1299 us where a call without takes 869, slopes 1107, both 1395.  A third wave on a SIMD does not fit
// its registers (spilled: 1117 us).
constexpr int kTileWaves = 4;
// Least units of a share (us with 8 / 16 / 32, one sequence): 512 tokens alone, 32 / 8 heads, 39 / 49 / 75; 300 tokens over 8192, 4 / 1
// heads, 70 / 58 / 69, whose blocks are cut into some 33 pieces with 8; of longer parts the same.
constexpr int kTileShare = 8;

typedef float f16v __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f16v mfma_32(h8 a, h8 b, f16v c)
{
    f16v d = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    asm("" : "+v"(d) : "v"(a), "v"(b));
    return d;
}

struct TileLds {
    uint8_t rows[2][kRowTileBytes];
    uint32_t odd[2][kTileWaves];
    int last;
};
template <int FMT, bool MOD>
__global__ __launch_bounds__(64 * kTileWaves, 2) void block_tiles(BlockAttnArgs a)
{
    __shared__ TileLds lds;
    const int lane = lane_id(), wave = wave_index(), half = lane >> 5, col = lane & 31;
    const auto units = [&](int n, int L) {
        if (n <= 0 || n * a.G <= a.few_rows) return 0LL;
        const TileUnits u = tile_units(a, n, L);
        return a.Hkv * u.upto(u.blocks);
    };
    SeqScan scan(a.B, a.max_new, a.total_new, lengths_of(a), units);
    const long long all = scan.total();
    const long long share = max((all + gridDim.x - 1) / gridDim.x, (long long)kTileShare);
    // A CU's two workgroups share its SIMDs, which serve the older wave first: the later one took 1.4 times as long, the last third of
    // that alone.  So its waves go first in every second step (one prompt's 2048 tokens over 8192, 64 / 8 heads: 932 -> 903 us).
    const bool late = blockIdx.x >= gridDim.x / 2;
    // (workgroup i runs on XCD i % 8)
    const int me = (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
    long long x = (long long)me * share;
    const long long x_end = min(x + share, all);

    while (x < x_end) {
        const SeqItem sq = scan.find(x);
        if (sq.b < 0) break;
        const TileUnits tu = tile_units(a, sq.n, sq.L);
        const long long head_units = tu.upto(tu.blocks);
        int h = uniform((int)((x - sq.item0) / head_units)), blk;
        {
            const long long y = x - sq.item0 - h * head_units;
            int lo = 0, hi = tu.blocks - 1;  // the last block that starts at y or before
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (tu.upto(mid) <= y) lo = mid;
                else hi = mid - 1;
            }
            blk = lo;
        }
        for (; x < x_end && h < a.Hkv;) {
            // the block's tiles, and this share's of them
            const long long t0 = sq.item0 + h * head_units + tu.upto(blk), t1 = sq.item0 + h * head_units + tu.upto(blk + 1);
            const int row_first = blk * kTileRows, rows = min(sq.n * a.G - row_first, kTileRows);
            const int my_h = h, j0 = row_first / a.G, j1 = (row_first + rows - 1) / a.G;
            const Tiles tl = tiles_of(a, j1 - j0 + 1, sq.L + j0);
            const int steps = tl.count();
            // (a block's units and its tiles differ: unit y of w stands for its first tiles up to y steps / w)
            const auto step_at = [&](long long y) { return (int)((y - t0) * steps / (t1 - t0)); };
            const int s0 = uniform(step_at(x)), s1 = uniform(step_at(min(x_end, t1)));
            x = min(x_end, t1);
            if (++blk == tu.blocks) blk = 0, ++h;
            if (s1 <= s0) continue;

            const int wrow = row_first + wave * 32, wrows = min(max(sq.n * a.G - wrow, 0), 32);  // the wave's
            const int row = min(wrow + col, sq.n * a.G - 1), token = row / a.G, hq = my_h * a.G + row % a.G, p = sq.L + token;
            const int p_lo = sq.L + wrow / a.G, p_hi = wrows ? sq.L + (wrow + wrows - 1) / a.G : -1;
            h8 q[8];  // [2 s + rr], s = 2 i + w: dims (4 i + 2 rr + half) 16 + 8 w ..
            {
                const uint16_t* at = a.q + (sq.row0 + token) * a.q_stride + (long long)hq * kD;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    q[i] = *reinterpret_cast<const h8*>(at + ((i >> 2) * 4 + (i & 1) * 2 + half) * 16 + ((i >> 1) & 1) * 8);
            }
            ScoreForm form{0.0f, 0.0f, 0.0f};
            if constexpr (MOD) form = ScoreForm{a.cap_in, a.cap, a.slopes ? a.slopes[hq] : 0.0f};
            f16v acc[4];  // dims u 32 + 8 (i / 4) + 4 half + i % 4
            float ref = kLowest, sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[i][j] = 0.0f;

            const int coded = coded_steps(tl, sq.L);
            const TileRange range = tile_range(a, tl, p_lo, p_hi);
            const uint32_t at_k = (col >> 4) * 4096 + half * 256 + (col & 15) * 16, at_v = 8192 + (col >> 4) * 1024 + half * 256 + (col & 15) * 16;
            f16v sc;     // a tile's products
            float y[16]; // its exponents, then weights
            h8 x[8];     // operands: asked for together (the scheduler would wait for each by itself)
            const auto read_keys = [&](int buf) {
                const uint8_t* tile = lds.rows[buf] + at_k;
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const h8*>(tile + (i >> 1) * 1024 + (i & 1) * 512);
            };
            const auto scores = [&]() {
#pragma unroll
                for (int j = 0; j < 16; ++j) sc[j] = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) sc = mfma_32(x[i], q[i], sc);
            };
            // A tile in LDS.  Its values are asked for beside its products.
            const auto tile_step = [&](int buf, TileScale ts, int s, int end) {
                if (late) {
                    if (s & 1) __builtin_amdgcn_s_setprio(1);
                    else __builtin_amdgcn_s_setprio(0);
                }
                TileView view{0, end, range.whole(s)};
                if (!view.whole || MOD) view.pos0 = tl.at(s) * kBT;
                read_keys(buf);
                __builtin_amdgcn_sched_barrier(0);
                scores();
                const uint8_t* tile = lds.rows[buf] + at_v;
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const h8*>(tile + (i & 3) * 2048 + (i >> 2) * 512);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < 16; ++j) y[j] = sc[j];
                raise<MOD>(a, ts, view, y, p, form, acc, ref, sum);
                exponents<MOD>(ts, y, ref);
                float total[2] = {0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    y[j] = __builtin_amdgcn_exp2f(y[j]);
                    total[j & 1] += y[j];
                }
                sum = __builtin_fmaf(total[0] + total[1], ts.rs, sum);
                if (ts.nan) spoil(a, view, y, p);
                const Parts w0 = parts(y[0], y[1], y[2], y[3], y[8], y[9], y[10], y[11]);
#pragma unroll
                for (int u = 0; u < 4; ++u) acc[u] = mfma_32(x[u], w0.hi, acc[u]);
#pragma unroll
                for (int u = 0; u < 4; ++u) acc[u] = mfma_32(x[u], w0.lo, acc[u]);
                const Parts w1 = parts(y[4], y[5], y[6], y[7], y[12], y[13], y[14], y[15]);
#pragma unroll
                for (int u = 0; u < 4; ++u) acc[u] = mfma_32(x[4 + u], w1.hi, acc[u]);
#pragma unroll
                for (int u = 0; u < 4; ++u) acc[u] = mfma_32(x[4 + u], w1.lo, acc[u]);
            };

            // the cache's blocks: a block's loads are asked for a step before it is written to LDS, and that two steps before its
            // values' use
            const int c1 = min(s1, coded);
            for (int base = s0; base < c1; base += kWave) {
                const int id = step_id(a, tl, sq.b, base, c1);
                const StepScales scales = step_scales<MOD>(a, id, my_h);
                unsigned long long todo = __ballot(id >= 0), loaded = todo;
                if (!todo) continue;
                u4 raw_k, raw_v;
                const auto load = [&]() {
                    if (!loaded) return;
                    const int now = __builtin_amdgcn_readlane(id, __builtin_ctzll(loaded));
                    loaded &= loaded - 1;
                    const auto from = span(a.pool + ((long long)now * a.Hkv + my_h) * kBlockBytes, kBlockBytes);
                    raw_k = fetch<16>(from, threadIdx.x * 16, 0);
                    raw_v = fetch<16>(from, threadIdx.x * 16, kBlockSide);
                };
                const auto store = [&](int buf) {
                    const int piece = threadIdx.x, c = (piece >> 4) & 7;
                    uint8_t* k = lds.rows[buf] + (piece >> 7) * 4096 + (c >> 2) * 2048 + (c & 3) * 256 + (piece & 15) * 16;
                    *reinterpret_cast<h8*>(k) = codes8<FMT>(raw_k[0], raw_k[1]);
                    *reinterpret_cast<h8*>(k + 1024) = codes8<FMT>(raw_k[2], raw_k[3]);
                    uint8_t* v = lds.rows[buf] + 8192 + (piece >> 6) * 2048 + ((piece >> 4) & 3) * 256 + (piece & 15) * 16;
                    *reinterpret_cast<h8*>(v) = codes8<FMT>(raw_v[0], raw_v[1]);
                    *reinterpret_cast<h8*>(v + 1024) = codes8<FMT>(raw_v[2], raw_v[3]);
                };
                load();
                store(0);
                load();
                __syncthreads();
                for (int buf = 0; todo; buf ^= 1) {
                    const int i = __builtin_ctzll(todo);
                    todo &= todo - 1;
                    if (todo) store(buf ^ 1);
                    load();
                    tile_step(buf, scales.at(i), base + i, INT32_MAX);
                    __syncthreads();
                }
            }

            // rows in fp16
            if (max(s0, coded) < s1) {
                const RowSource src = row_source(a, sq, my_h);
                // keys: two pieces (token, eight dims) of a thread; values: r = the wave, two dims of a lane
                u4 kx[2];
                uint32_t vx[8];
                const int k_lane = (threadIdx.x >> 4) * (int)a.k_stride * 2 + (threadIdx.x & 15) * 16;
                const auto load = [&](int s) {
                    const int pos0 = tl.at(s) * kBT;
                    if (pos0 >= src.L) {  // the call's own rows alone: rows behind the last lie outside the span and read zero
                        const int n = min(src.end - pos0, kBT);
                        const auto kr = span(src.own[0] + (long long)(pos0 - src.L) * a.k_stride, (uint32_t)((n - 1) * (int)a.k_stride * 2 + kD * 2));
                        const auto vr = span(src.own[1] + (long long)(pos0 - src.L) * a.v_stride, (uint32_t)((n - 1) * (int)a.v_stride * 2 + kD * 2));
#pragma unroll
                        for (int i = 0; i < 2; ++i) kx[i] = fetch<16>(kr, k_lane, i * 16 * (int)a.k_stride * 2);
#pragma unroll
                        for (int e = 0; e < 8; ++e) vx[e] = fetch<4>(vr, lane * 4, ((e >> 2) * 16 + 4 * wave + (e & 3)) * (int)a.v_stride * 2);
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i) kx[i] = key_piece(src, pos0, i * 256 + threadIdx.x);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int pos = pos0 + (e >> 2) * 16 + 4 * wave + (e & 3);
                            vx[e] = pos < src.end ? *reinterpret_cast<const uint32_t*>(row_of(src, 1, pos) + lane * 2) : 0u;
                        }
                    }
                };
                const auto store = [&](int buf) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) put_key(kx[i], lds.rows[buf], i * 256 + threadIdx.x);
                    uint32_t top = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) top = pk_max(top, vx[e] & 0x7fff7fffu);
                    uint32_t odd = 0;
                    if (__any((top & 0xffffu) >= 0x7c00u || top >= 0x7c000000u)) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const bool bad = (vx[e] & 0x7c00u) == 0x7c00u || (vx[e] & 0x7c000000u) == 0x7c000000u;
                            if (__any(bad)) odd |= 1u << ((e >> 2) * 16 + 4 * wave + (e & 3));
                            if ((vx[e] & 0x7c00u) == 0x7c00u) vx[e] &= 0xffff0000u;
                            if ((vx[e] & 0x7c000000u) == 0x7c000000u) vx[e] &= 0xffffu;
                        }
                    }
                    if (lane == 0) lds.odd[buf][wave] = odd;
                    uint8_t* to = lds.rows[buf] + 8192 + (lane >> 4) * 2048 + ((lane >> 3) & 1) * 1024 + wave * 256 + (lane & 7) * 32;
                    u4 y[2];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        y[0][e] = __builtin_amdgcn_perm(vx[2 * e + 1], vx[2 * e], 0x05040100u);
                        y[1][e] = __builtin_amdgcn_perm(vx[2 * e + 1], vx[2 * e], 0x07060302u);
                    }
                    *reinterpret_cast<u4*>(to) = y[0];
                    *reinterpret_cast<u4*>(to + 16) = y[1];
                };
                const int f0 = max(s0, coded);
                load(f0);
                store(0);
                if (f0 + 1 < s1) load(f0 + 1);
                __syncthreads();
                int buf = 0;
                for (int s = f0; s < s1; ++s, buf ^= 1) {
                    if (s + 1 < s1) store(buf ^ 1);
                    if (s + 2 < s1) load(s + 2);
                    tile_step(buf, TileScale{a.scale_x, 0.0f, 1.0f, false}, s, src.end);
                    // values that are not finite, to the rows that see their token
                    for (uint32_t odd = __builtin_amdgcn_readfirstlane(lds.odd[buf][0] | lds.odd[buf][1] | lds.odd[buf][2] | lds.odd[buf][3]); odd; odd &= odd - 1) {
                        const int tok = __builtin_ctz(odd), c = tl.at(s) * kBT + tok;
                        const int at = ((tok >> 2) & 1) * 32 + col, reg = (tok >> 3) * 4 + (tok & 3);
                        float wt = 0.0f;
#pragma unroll
                        for (int j = 0; j < 16; ++j) wt = j == reg ? y[j] : wt;
                        wt = __shfl(wt, at);
                        const bool seen = c <= p && (p - c < a.window || c < a.sinks);
                        const uint16_t* vr = row_of(src, 1, c);
#pragma unroll
                        for (int u = 0; u < 4; ++u)
#pragma unroll
                            for (int j = 0; j < 16; ++j) {
                                const float v1 = h2f(vr[u * 32 + 8 * (j >> 2) + 4 * half + (j & 3)]);
                                if (seen && !(fabsf(v1) < INFINITY)) acc[u][j] = __builtin_fmaf(wt, v1, acc[u][j]);
                            }
                    }
                    __syncthreads();
                }
            }

            sum = pairs_sum(sum);
            constexpr float to_log2 = MOD ? kChunkLog2e : 1.0f;
            // the first and last share that has a tile of this block
            const auto share_of = [&](int s) {  // of step s: that of the first unit behind it
                const long long w = t1 - t0;
                // the least unit y with (y + 1) steps / w > s
                const long long y = ((long long)(s + 1) * w + steps - 1) / steps - 1;
                return (int)((t0 + y) / share);
            };
            const int first_share = uniform(share_of(0)), last_share = uniform(share_of(steps - 1));
            // (where a share has less units than a tile stands for, it may have no tile)
            const auto has = [&](int sh) {
                return share * steps >= t1 - t0 || step_at(min((sh + 1) * share, t1)) > step_at(max(sh * share, t0));
            };
            bool whole = first_share == last_share;
            if (!whole) {
                int pieces = last_share - first_share + 1;
                if (share * steps < t1 - t0) {
                    pieces = 0;
                    for (int sh = first_share; sh <= last_share; ++sh) pieces += has(sh) ? 1 : 0;
                }
                const auto slot = [&](int sh) {
                    return span(a.tile_part + (long long)(sh * 2 + (sh == first_share ? 1 : 0)) * kTilePart + wave * (kTilePart / kTileWaves), kTilePart / kTileWaves * 4);
                };
                {
                    const auto to = slot(me);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        put_quad(to, lane * 16, i * 1024, f4{acc[i >> 2][(i & 3) * 4], acc[i >> 2][(i & 3) * 4 + 1], acc[i >> 2][(i & 3) * 4 + 2], acc[i >> 2][(i & 3) * 4 + 3]});
                    put_quad(to, lane * 16, 16 * 1024, f4{ref, sum, 0.0f, 0.0f});
                }
                whole = split_last(a.tile_arrive + first_share, pieces, &lds.last);
                if (whole) {
                    // All pieces in order: references and normalizers first, then the sums, eight quads of four pieces asked
                    // for at once.
                    ref = kLowest, sum = 0.0f;
#pragma unroll 1
                    for (int sh = first_share; sh <= last_share; sh += 8) {
                        f4 m[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) m[i] = get_quad(slot(min(sh + i, last_share)), lane * 16, 16 * 1024);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            if (sh + i <= last_share && has(sh + i)) {
                                const float up = fmaxf(ref, m[i][0]);
                                sum = __builtin_fmaf(m[i][1], __builtin_amdgcn_exp2f((m[i][0] - up) * to_log2), sum * __builtin_amdgcn_exp2f((ref - up) * to_log2));
                                ref = up;
                            }
                        }
                    }
#pragma unroll
                    for (int u = 0; u < 4; u += 2) {
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int j = 0; j < 16; ++j) acc[u + i][j] = 0.0f;
#pragma unroll 1
                        for (int sh = first_share; sh <= last_share; sh += 4) {
                            f4 part[4][8], m[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const auto from = slot(min(sh + k, last_share));
                                m[k] = get_quad(from, lane * 16, 16 * 1024);
#pragma unroll
                                for (int i = 0; i < 8; ++i) part[k][i] = get_quad(from, lane * 16, (u * 4 + i) * 1024);
                            }
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                if (sh + k <= last_share && has(sh + k)) {
                                    const float f = __builtin_amdgcn_exp2f((m[k][0] - ref) * to_log2);
#pragma unroll
                                    for (int i = 0; i < 8; ++i)
#pragma unroll
                                        for (int j = 0; j < 4; ++j)
                                            acc[u + (i >> 2)][(i & 3) * 4 + j] = __builtin_fmaf(part[k][i][j], f, acc[u + (i >> 2)][(i & 3) * 4 + j]);
                                }
                            }
                        }
                    }
                }
            }
            if (whole && col < wrows) {
                const long long at = (sq.row0 + token) * a.Hq + hq;
                const float inv = 1.0f / sum;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    h4 y;
#pragma unroll
                    for (int j = 0; j < 4; ++j) y[j] = (_Float16)(acc[i >> 2][(i & 3) * 4 + j] * inv);
                    *reinterpret_cast<h4*>(a.out + at * kD + (i >> 2) * 32 + (i & 3) * 8 + 4 * half) = y;
                }
                if (a.lse && half == 0) a.lse[at] = MOD ? ref + __logf(sum) : (ref + __log2f(sum)) * kChunkLn2;
            }
            __syncthreads();
        }
    }
}

}  // namespace

hipError_t launch_block_attention(const BlockAttnArgs& a, int format, bool mod, hipStream_t st)
{
    // (sequences of many rows there are none, or no others)
    if ((long long)a.max_new * a.G > a.few_rows) {
        void (*kernel)(BlockAttnArgs) = format == kE4m3 ? (mod ? block_tiles<kE4m3, true> : block_tiles<kE4m3, false>)
                                                        : (mod ? block_tiles<kInt8, true> : block_tiles<kInt8, false>);
        BlockAttnArgs t = a;
        if (a.B == 1) t.few_rows = 0;  // (a lone sequence is this kernel's, also where it has less rows than max_new says)
        const hipError_t e = launch1(kernel, kBlockTileShares, 64 * kTileWaves, st, t);
        if (e != hipSuccess || a.B == 1) return e;
    }
    void (*kernel)(BlockAttnArgs) = format == kE4m3 ? (mod ? block_rows<kE4m3, true> : block_rows<kE4m3, false>)
                                                    : (mod ? block_rows<kInt8, true> : block_rows<kInt8, false>);
    return launch1(kernel, kBlockRowShares / kRowWaves, 64 * kRowWaves, st, a);
}

}  // namespace dkv
