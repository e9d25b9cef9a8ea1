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
// Pieces of a tile: keys 512 (token, eight dims), values 128 (r, four dims of r's eight tokens).
__device__ __forceinline__ void put_key(u4 x, uint8_t* lds, int piece)
{
    const int c = piece & 15, token = piece >> 4;  // c: dims 8 c ..
    const int step = (c >> 3) * 2 + (c & 1), r = (c >> 1) & 3;
    *reinterpret_cast<u4*>(lds + (token >> 4) * 4096 + step * 1024 + r * 256 + (token & 15) * 16) = x;
}
// Returns the bits of the tokens with values that are not finite among the wave's pieces.
__device__ __forceinline__ uint32_t put_value(u2 (&x)[8], uint8_t* lds, int piece)
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
        *reinterpret_cast<u4*>(lds + 8192 + (dim >> 5) * 2048 + ((dim >> 4) & 1) * 1024 + r * 256 + (dim & 15) * 16) = y;
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

// ---- scores to weights ----------------------------------------------------------------
// One tile's scores (natural units with a form, else log2) -> weights for the values' product.
struct TileScale {
    float ks;       // of the fp32 product: a code's unit, scales, without a form log2(e)
    float add;      // log2 of the values' scale (natural units with a form)
    float rs;       // 1 / the values' scale
};
struct TileView {
    int pos0, end;  // tokens from position `end` on are not there
    bool whole;     // all rows see all 32 tokens
};
// A tile for rows at p_lo .. p_hi: whether all of them see all of it, and whether none sees any of it.
__device__ __forceinline__ bool all_seen(const BlockAttnArgs& a, int pos0, int p_lo, int p_hi)
{
    return pos0 + kBT - 1 <= p_lo && (p_hi - pos0 < a.window || pos0 + kBT <= a.sinks);
}
__device__ __forceinline__ bool none_seen(const BlockAttnArgs& a, int pos0, int p_lo, int p_hi)
{
    return pos0 > p_hi || (p_lo - (pos0 + kBT - 1) >= a.window && pos0 >= a.sinks);
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
// i % 4) become weights; acc are the row's sums of values, raised with its reference.  Hidden tokens' products become -inf
// at once, so that all tiles go one way from there.
template <bool MOD, int N, typename Acc, int A>
__device__ __forceinline__ void weights(const BlockAttnArgs& a, TileScale t, const TileView& w, float (&y)[N], int p,
                                        const ScoreForm& form, Acc (&acc)[A], float& ref, float& sum)
{
    constexpr float unit = MOD ? kChunkLn2 : 1.0f;
    const int group = N == 8 ? lane_id() >> 4 : lane_id() >> 5;
    if (__builtin_isnan(t.ks + t.add)) {  // (uniform: a block that reads NaN, to the rows that see one of its tokens)
        t.ks = 1.0f, t.add = 0.0f;
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
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; i += 2) top = max3(top, y[i], y[i + 1]);
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
    const float less = t.add - ref;
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = __builtin_amdgcn_exp2f(MOD ? (y[i] + less) * kChunkLog2e : __builtin_fmaf(y[i], t.ks, less));
    float total = y[0];
#pragma unroll
    for (int i = 1; i < N; ++i) total += y[i];
    sum = __builtin_fmaf(total, t.rs, sum);
}
// Eight weights as two fp16 parts.
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
        const h2 rest = {(_Float16)__builtin_fmaf((float)top.x, minus, u[2 * i]), (_Float16)__builtin_fmaf((float)top.y, minus, u[2 * i + 1])};
        lo[i] = __builtin_bit_cast(uint32_t, rest);
    }
    return Parts{__builtin_bit_cast(h8, hi), __builtin_bit_cast(h8, lo)};
}

// Block IDs and scales of 64 steps of a wave, a lane each (step = first + lane * stride < end); those whose block is there.
struct StepList {
    int id;
    TileScale scale;
    unsigned long long there;
};
template <bool MOD>
__device__ __forceinline__ StepList list_steps(const BlockAttnArgs& a, const Tiles& tl, int b, int h, int first, int stride, int end)
{
    StepList s;
    const int step = first + lane_id() * stride;
    s.id = step < end ? block_id(a, b, tl.at(step)) : -1;
    s.there = __ballot(s.id >= 0);
    float ks = 1.0f, vs = 1.0f;
    if (s.id >= 0) {
        const float* sc = a.scale + ((long long)s.id * a.Hkv + h) * 2;
        ks = sc[0];
        vs = sc[1];
    }
    vs *= kCodeUnit;
    s.scale.ks = ks * kCodeUnit * a.scale_x;
    s.scale.add = __builtin_amdgcn_logf(vs) * (MOD ? kChunkLn2 : 1.0f);
    s.scale.rs = vs > 0.0f && vs < INFINITY ? 1.0f / vs : 1.0f;  // (a NaN scale: see weights)
    return s;
}
__device__ __forceinline__ TileScale scale_of(const StepList& s, int i)
{
    return TileScale{read_lane_f(s.scale.ks, i), read_lane_f(s.scale.add, i), read_lane_f(s.scale.rs, i)};
}

__device__ __forceinline__ RowSource row_source(const BlockAttnArgs& a, const SeqItem& sq, int h)
{
    const uint16_t* tail = tail_rows(a, sq.b, h);
    return RowSource{{tail, tail + kBlockSide},
                     {a.k + sq.row0 * a.k_stride + h * kD, a.v + sq.row0 * a.v_stride + h * kD},
                     {a.k_stride, a.v_stride}, sq.L, sq.L + sq.n};
}
// Steps whose tiles are blocks of the cache: they come first.
__device__ __forceinline__ int coded_steps(const Tiles& tl, int L)
{
    const int held = L / kBT;
    return held <= tl.sb ? held : min(max(held - tl.w0, 0) + tl.sb, tl.count());
}

// ---- few rows: a workgroup on 16 rows -------------------------------------------------
// Eight waves on the tiles of a piece, one tile each at a time; their states meet in LDS.  All (sequence, KV head, 16
// rows) are laid end to end by their tiles and cut into equal pieces, one for each workgroup; one that is
// split has its pieces' states joined by the last to arrive.
//
// Bound by memory.  A wave asks for a tile's keys again as soon as their codes are operands, and for its values likewise, so 8 KB
// of the next tile are always on their way.
constexpr int kRowWaves = 8;
constexpr int kRowStart = 2;    // a 16-row block's start, in tiles
constexpr int kRowShare = 16;  // least units of a piece: two tiles a wave
constexpr int kStaged = 4;      // tiles of fp16 rows in LDS at once

struct RowLds {
    union {
        uint8_t rows[kStaged * kRowTileBytes];
        float state[kRowWaves][16][kChunkPart];
    };
    float ref[kRowWaves][16], sum[kRowWaves][16];
    uint32_t odd[kStaged];
    int last;
};

template <int FMT, bool MOD>
__global__ __launch_bounds__(64 * kRowWaves, 4) void block_rows(BlockAttnArgs a)
{
    __shared__ RowLds lds;
    const int lane = lane_id(), wave = wave_index(), r = lane >> 4, col = lane & 15;
    const int first_n = lane < a.B ? a.new_len[lane] : 0, first_L = lane < a.B ? seq_tokens(a, lane) : 0;
    const auto loads = [&](int b, int& n, int& L) {
        n = b < kWave ? first_n : a.new_len[b];
        L = b < kWave ? first_L : seq_tokens(a, b);
    };
    // units of a sequence: 16-row blocks times their tiles and start
    const auto units = [&](int n, int L) {
        return n > 0 && n * a.G <= a.few_rows ? (long long)a.Hkv * ((n * a.G + 15) / 16) * (tiles_of(a, n, L).count() + kRowStart) : 0LL;
    };
    const long long all = find_item(a.B, a.total_new, a.max_new, INT64_MAX, loads, units).items;
    long long share = (all + gridDim.x - 1) / gridDim.x;
    share = share < kRowShare ? kRowShare : share;
    long long x = (long long)blockIdx.x * share;
    const long long x_end = min(x + share, all);

    while (x < x_end) {
        const SeqItem sq = find_item(a.B, a.total_new, a.max_new, x, loads, units);
        if (sq.b < 0) break;
        const Tiles tl = tiles_of(a, sq.n, sq.L);
        const int blk_units = tl.count() + kRowStart, coded = coded_steps(tl, sq.L);
        const int blocks = (sq.n * a.G + 15) / 16;
        // 16-row block of the sequence: KV head major
        int which = (int)((x - sq.item0) / blk_units);
        for (; x < x_end && which < a.Hkv * blocks; ++which) {
            const long long t0 = sq.item0 + (long long)which * blk_units;  // the block's first unit
            const int h = which / blocks, row_first = (which - h * blocks) * 16;
            const int s0 = (int)max(x - t0 - kRowStart, 0LL);
            const int s1 = (int)(min(x_end, t0 + blk_units) - t0) - kRowStart;
            x = min(x_end, t0 + blk_units);
            if (s1 <= s0) continue;

            // this lane's row
            const int rows = min(sq.n * a.G - row_first, 16);
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
            f4 acc[8];  // [u * 2 + j]: dims u 32 + j 16 + 4 r ..
            float ref = kLowest, sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = f4{0.0f, 0.0f, 0.0f, 0.0f};

            // steps of the cache's blocks, then those of fp16 rows
            const int c1 = min(s1, coded);
            for (int base = s0 + wave; base < c1; base += kRowWaves * kWave) {
                const StepList list = list_steps<MOD>(a, tl, sq.b, h, base, kRowWaves, c1);
                unsigned long long todo = list.there;
                if (!todo) continue;
                int i = __builtin_ctzll(todo);
                const auto block = [&](int at) {
                    const int id = __builtin_amdgcn_readlane(list.id, at);
                    return span(a.pool + ((long long)id * a.Hkv + h) * kBlockBytes, kBlockBytes);
                };
                auto src = block(i);
                u4 k[4], v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) k[j] = fetch<16>(src, lane * 16, j * 1024);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = fetch<16>(src, lane * 16, kBlockSide + j * 1024);
                while (todo) {
                    todo &= todo - 1;
                    const int next = todo ? __builtin_ctzll(todo) : i;
                    const TileScale ts = scale_of(list, i);
                    TileView view{tl.at(base + i * kRowWaves) * kBT, INT32_MAX, false};
                    view.whole = all_seen(a, view.pos0, p_lo, p_hi);
                    src = block(next);
                    f4 s[2] = {f4{0.0f, 0.0f, 0.0f, 0.0f}, f4{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[j >> 1] = mfma_k32(codes8<FMT>(k[j][0], k[j][1]), q[(j & 1) * 2], s[j >> 1]);
                        s[j >> 1] = mfma_k32(codes8<FMT>(k[j][2], k[j][3]), q[(j & 1) * 2 + 1], s[j >> 1]);
                    }
                    if (todo) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) k[j] = fetch<16>(src, lane * 16, j * 1024);
                    }
                    float y[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) y[j] = s[j >> 2][j & 3];
                    weights<MOD>(a, ts, view, y, p, form, acc, ref, sum);
                    const Parts w = parts(y[0], y[1], y[2], y[3], y[4], y[5], y[6], y[7]);
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

            for (int base = max(s0, coded); base < s1; base += kStaged) {
                const RowSource src = row_source(a, sq, h);
                const int here = min(kStaged, s1 - base);
                __syncthreads();
                if (threadIdx.x < kStaged) lds.odd[threadIdx.x] = 0;
                __syncthreads();
#pragma unroll 1
                for (int piece = threadIdx.x; piece < here * 512; piece += 64 * kRowWaves) {
                    const int t = piece / 512;
                    put_key(key_piece(src, tl.at(base + t) * kBT, piece & 511), lds.rows + t * kRowTileBytes, piece & 511);
                }
#pragma unroll 1
                for (int piece = threadIdx.x; piece < here * 128; piece += 64 * kRowWaves) {
                    const int t = piece / 128;
                    u2 v8[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v8[e] = value_piece(src, tl.at(base + t) * kBT, piece & 127, e);
                    const uint32_t odd = put_value(v8, lds.rows + t * kRowTileBytes, piece & 127);
                    if (odd && lane == 0) atomicOr(&lds.odd[t], odd);
                }
                __syncthreads();
                if (wave < here) {
                    const uint8_t* tile = lds.rows + wave * kRowTileBytes;
                    TileView view{tl.at(base + wave) * kBT, sq.L + sq.n, false};
                    view.whole = all_seen(a, view.pos0, p_lo, p_hi);
                    f4 s[2] = {f4{0.0f, 0.0f, 0.0f, 0.0f}, f4{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        s[j >> 2] = mfma_k32(*reinterpret_cast<const h8*>(tile + j * 1024 + lane * 16), q[j & 3], s[j >> 2]);
                    float y[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) y[j] = s[j >> 2][j & 3];
                    weights<MOD>(a, TileScale{a.scale_x, 0.0f, 1.0f}, view, y, p, form, acc, ref, sum);
                    const Parts w = parts(y[0], y[1], y[2], y[3], y[4], y[5], y[6], y[7]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const h8 x8 = *reinterpret_cast<const h8*>(tile + 8192 + j * 1024 + lane * 16);
                        acc[j] = mfma_k32(x8, w.hi, acc[j]);
                        acc[j] = mfma_k32(x8, w.lo, acc[j]);
                    }
                    // values that are not finite, to the rows that see their token
                    for (uint32_t odd = __builtin_amdgcn_readfirstlane(lds.odd[wave]); odd; odd &= odd - 1) {
                        const int tok = __builtin_ctz(odd), c = view.pos0 + tok;
                        const int from = ((tok & 15) >> 2) * 16 + col, reg = (tok >> 4) * 4 + (tok & 3);
                        float wt = 0.0f;
#pragma unroll
                        for (int j = 0; j < 8; ++j) wt = j == reg ? y[j] : wt;
                        wt = __shfl(wt, from);
                        const bool seen = c <= p && (p - c < a.window || c < a.sinks);
                        const uint16_t* vr = row_of(src, 1, c);
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const float v1 = h2f(vr[(j >> 3) * 32 + ((j >> 2) & 1) * 16 + 4 * r + (j & 3)]);
                            if (seen && !(fabsf(v1) < INFINITY)) acc[j >> 2][j & 3] = __builtin_fmaf(wt, v1, acc[j >> 2][j & 3]);
                        }
                    }
                }
            }

            // the waves' states
            sum = rows_sum(sum);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) *reinterpret_cast<f4*>(&lds.state[wave][col][(i >> 1) * 32 + (i & 1) * 16 + 4 * r]) = acc[i];
            if (r == 0) {
                lds.ref[wave][col] = ref;
                lds.sum[wave][col] = sum;
            }
            __syncthreads();
            const int my_row = threadIdx.x >> 5, dim = (threadIdx.x & 31) * 4;
            constexpr float to_log2 = MOD ? kChunkLog2e : 1.0f;
            ref = kLowest, sum = 0.0f;
            f4 out = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < kRowWaves; ++w) ref = fmaxf(ref, lds.ref[w][my_row]);
#pragma unroll
            for (int w = 0; w < kRowWaves; ++w) {
                const float f = __builtin_amdgcn_exp2f((lds.ref[w][my_row] - ref) * to_log2);
                sum = __builtin_fmaf(lds.sum[w][my_row], f, sum);
                out += *reinterpret_cast<const f4*>(&lds.state[w][my_row][dim]) * f;
            }
            const long long first_share = (t0 + kRowStart) / share, last_share = (t0 + blk_units - 1) / share;
            bool whole = first_share == last_share;
            if (!whole) {
                // split: slot 1 of the share where the block starts, slot 0 of the others
                const auto slot = [&](long long sh) {
                    return span(a.part + (sh * 2 + (sh == first_share ? 1 : 0)) * 16 * kChunkPart, 16 * kChunkPart * 4);
                };
                const int at = my_row * kChunkPart * 4;
                {
                    const auto to = slot(blockIdx.x);
                    put_quad(to, at + dim * 4, 0, out);
                    if (dim == 0) put_quad(to, at + kD * 4, 0, f4{ref, sum, 0.0f, 0.0f});
                }
                whole = split_last(a.arrive + first_share, (int)(last_share - first_share) + 1, &lds.last);
                if (whole) {
                    ref = kLowest, sum = 0.0f;
                    out = f4{0.0f, 0.0f, 0.0f, 0.0f};
                    for (long long sh = first_share; sh <= last_share; ++sh) ref = fmaxf(ref, get_quad(slot(sh), at + kD * 4, 0)[0]);
                    for (long long sh = first_share; sh <= last_share; ++sh) {
                        const auto from = slot(sh);
                        const f4 m = get_quad(from, at + kD * 4, 0), part = get_quad(from, at + dim * 4, 0);
                        const float f = __builtin_amdgcn_exp2f((m[0] - ref) * to_log2);
                        sum = __builtin_fmaf(m[1], f, sum);
                        out += part * f;
                    }
                }
            }
            if (whole && my_row < rows) {
                const int orow = row_first + my_row, otoken = orow / a.G, ohq = h * a.G + orow % a.G;
                const long long at = (sq.row0 + otoken) * a.Hq + ohq;
                const float inv = 1.0f / sum;
                h4 y;
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = (_Float16)(out[j] * inv);
                *reinterpret_cast<h4*>(a.out + at * kD + dim) = y;
                if (a.lse && dim == 0) a.lse[at] = MOD ? ref + __logf(sum) : (ref + __log2f(sum)) * kChunkLn2;
            }
            __syncthreads();
        }
    }
}

// ---- many rows: a workgroup on 128 rows -------------------------------------------------
// Four waves of 32 rows each go over the same tiles.  A tile is brought into LDS once, as fp16 operands (a block's
// codes are converted on the way), one step ahead of its use: its loads are asked for before a step's products and
// written behind them.  v_mfma_f32_32x32x16_f16: A lane l holds row l % 32, k 8 (l / 32) .. + 7, B the same with columns, C
// lane l in register i row 8 (i / 4) + i % 4 + 4 (l / 32) of column l % 32.
//
// All (sequence, KV head, 128 rows) are laid end to end and cut into equal shares, one for each workgroup; shares that follow
// each other run on one XCD, so that its L2 serves their tiles.
constexpr int kTileRows = 128, kTileWaves = 4;
constexpr int kTileShare = 16; // least units of a share
constexpr int kTileStart = 4;  // a 128-row block's start, in tiles

typedef float f16v __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f16v mfma_32(h8 a, h8 b, f16v c)
{
    f16v d = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    asm("" : "+v"(d) : "v"(a), "v"(b));
    return d;
}

// Units of a sequence's 128-row blocks up to block t: each counts about as many as it has tiles.  They grow with the rows'
// positions until the window is full; between its ends a sum of that shape in closed form stands for them.
struct TileUnits {
    int blocks, full;        // 128-row blocks; from `full` on all have as many tiles
    long long first, most;   // units of block 0, of those from `full` on
    __device__ __forceinline__ long long upto(long long t) const
    {
        const long long g = t < full ? t : full;
        return first * g + (most - first) * g * (g - 1) / (2 * (long long)max(full, 1)) + most * (t - g);
    }
};
__device__ __forceinline__ TileUnits tile_units(const BlockAttnArgs& a, int n, int L)
{
    TileUnits u;
    u.blocks = (n * a.G + kTileRows - 1) / kTileRows;
    const int step = (kTileRows + a.G - 1) / a.G;  // tokens of a block, about
    u.first = tiles_of(a, min(n, step), L).count() + kTileStart;
    const int last = max(0, n - step);
    const int late = a.window < L + last ? max(0, min(last, a.window - L)) : last;
    u.full = late / step;
    u.most = max((long long)tiles_of(a, min(n - late, step), L + late).count() + kTileStart, u.first);
    return u;
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
    const auto loads = [&](int b, int& n, int& L) {
        n = a.new_len[b];
        L = seq_tokens(a, b);
    };
    const auto units = [&](int n, int L) {
        if (n <= 0 || n * a.G <= a.few_rows) return 0LL;
        const TileUnits u = tile_units(a, n, L);
        return a.Hkv * u.upto(u.blocks);
    };
    const long long all = find_item(a.B, a.total_new, a.max_new, INT64_MAX, loads, units).items;
    long long share = (all + gridDim.x - 1) / gridDim.x;
    share = share < kTileShare ? kTileShare : share;
    // (workgroup i runs on XCD i % 8)
    const int me = (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
    long long x = (long long)me * share;
    const long long x_end = min(x + share, all);

    while (x < x_end) {
        const SeqItem sq = find_item(a.B, a.total_new, a.max_new, x, loads, units);
        if (sq.b < 0) break;
        const TileUnits tu = tile_units(a, sq.n, sq.L);
        const long long head_units = tu.upto(tu.blocks);
        int h = (int)((x - sq.item0) / head_units), blk;
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
            const int s0 = step_at(x), s1 = step_at(min(x_end, t1));
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
            // A tile in LDS: scores, weights, values.  (Its operands are asked for together: the scheduler would
            // wait for each by itself.)
            const uint32_t at_k = (col >> 4) * 4096 + half * 256 + (col & 15) * 16, at_v = 8192 + (col >> 4) * 1024 + half * 256 + (col & 15) * 16;
            float y[16];
            const auto tile_step = [&](const uint8_t* tile, const TileScale& ts, const TileView& view) {
                h8 x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const h8*>(tile + at_k + (i >> 1) * 1024 + (i & 1) * 512);
                __builtin_amdgcn_sched_barrier(0);
                f16v sc;
#pragma unroll
                for (int j = 0; j < 16; ++j) sc[j] = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) sc = mfma_32(x[i], q[i], sc);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const h8*>(tile + at_v + (i >> 1) * 2048 + (i & 1) * 512);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < 16; ++j) y[j] = sc[j];
                weights<MOD>(a, ts, view, y, p, form, acc, ref, sum);
                const Parts w[2] = {parts(y[0], y[1], y[2], y[3], y[8], y[9], y[10], y[11]),
                                    parts(y[4], y[5], y[6], y[7], y[12], y[13], y[14], y[15])};
#pragma unroll
                for (int k = 0; k < 2; ++k) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) acc[u] = mfma_32(x[2 * u + k], w[k].hi, acc[u]);
#pragma unroll
                    for (int u = 0; u < 4; ++u) acc[u] = mfma_32(x[2 * u + k], w[k].lo, acc[u]);
                }
            };

            // the cache's blocks: a block's loads are asked for a step before it is written to LDS, and that a step before its use
            const int c1 = min(s1, coded);
            for (int base = s0; base < c1; base += kWave) {
                const StepList list = list_steps<MOD>(a, tl, sq.b, my_h, base, 1, c1);
                unsigned long long todo = list.there, loaded = todo;
                if (!todo) continue;
                u4 raw_k, raw_v;
                const auto load = [&]() {
                    if (!loaded) return;
                    const int id = __builtin_amdgcn_readlane(list.id, __builtin_ctzll(loaded));
                    loaded &= loaded - 1;
                    const auto from = span(a.pool + ((long long)id * a.Hkv + my_h) * kBlockBytes, kBlockBytes);
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
                    TileView view{tl.at(base + i) * kBT, INT32_MAX, false};
                    if (!none_seen(a, view.pos0, p_lo, p_hi)) {
                        view.whole = all_seen(a, view.pos0, p_lo, p_hi);
                        tile_step(lds.rows[buf], scale_of(list, i), view);
                    }
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
                load(max(s0, coded));
                store(0);
                if (max(s0, coded) + 1 < s1) load(max(s0, coded) + 1);
                __syncthreads();
                int buf = 0;
                for (int s = max(s0, coded); s < s1; ++s, buf ^= 1) {
                    if (s + 1 < s1) store(buf ^ 1);
                    if (s + 2 < s1) load(s + 2);
                    TileView view{tl.at(s) * kBT, src.end, false};
                    if (!none_seen(a, view.pos0, p_lo, p_hi)) {
                        view.whole = all_seen(a, view.pos0, p_lo, p_hi);
                        tile_step(lds.rows[buf], TileScale{a.scale_x, 0.0f, 1.0f}, view);
                        // values that are not finite, to the rows that see their token
                        for (uint32_t odd = __builtin_amdgcn_readfirstlane(lds.odd[buf][0] | lds.odd[buf][1] | lds.odd[buf][2] | lds.odd[buf][3]); odd; odd &= odd - 1) {
                            const int tok = __builtin_ctz(odd), c = view.pos0 + tok;
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
            const int first_share = share_of(0), last_share = share_of(steps - 1);
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
                    float top = kLowest;
                    for (int sh = first_share; sh <= last_share; ++sh)
                        if (has(sh)) top = fmaxf(top, get_quad(slot(sh), lane * 16, 16 * 1024)[0]);
                    ref = top, sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 16; ++j) acc[i][j] = 0.0f;
                    for (int sh = first_share; sh <= last_share; ++sh) {
                        if (!has(sh)) continue;
                        const auto from_slot = slot(sh);
                        const f4 m = get_quad(from_slot, lane * 16, 16 * 1024);
                        const float f = __builtin_amdgcn_exp2f((m[0] - ref) * to_log2);
                        sum = __builtin_fmaf(m[1], f, sum);
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const f4 part = get_quad(from_slot, lane * 16, i * 1024);
#pragma unroll
                            for (int j = 0; j < 4; ++j) acc[i >> 2][(i & 3) * 4 + j] = __builtin_fmaf(part[j], f, acc[i >> 2][(i & 3) * 4 + j]);
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
        const hipError_t e = launch1(kernel, kBlockTileShares, 64 * kTileWaves, st, a);
        if (e != hipSuccess || a.B == 1) return e;
    }
    void (*kernel)(BlockAttnArgs) = format == kE4m3 ? (mod ? block_rows<kE4m3, true> : block_rows<kE4m3, false>)
                                                    : (mod ? block_rows<kInt8, true> : block_rows<kInt8, false>);
    return launch1(kernel, kBlockRowShares, 64 * kRowWaves, st, a);
}

}  // namespace dkv
