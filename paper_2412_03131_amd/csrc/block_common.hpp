// block_common.hpp -- the uniform 8-bit cache: arguments, conversions of its codes, and the operand tiles
// of its fp16 rows.
//
// A cache of whole blocks of 32 positions: per block and KV head 128 x 32 key codes and as many value codes, a
// scale for each side; the positions behind a sequence's last whole block lie in its tail as fp16 rows.  The
// bytes of a block lie as the matrix products take them, so that a lane's operands are whole 16-byte pieces:
//   keys    [2: token / 16][8: dim / 16][16: token % 16][16: dim % 16].  With lane = r * 16 + key and chunk 4 i + r, a
//           wave's load i of a half is 1024 bytes in lane order.
//   values  [4: u = dim / 32][4: r][16: dim % 16][2: dim / 16 % 2][8: e], e < 4 token 4 r + e, e >= 4 token 12 + 4 r + e.
//           Scores come out of their product (keys as A operand) with tokens 4 r .. 4 r + 3 of each half in the lanes
//           of r, and go into the next one (values as A operand, depth 32) as they lie; load u is 1024 bytes in
//           lane order again and holds two tiles of 16 dims.
#pragma once

#include "block_units.hpp"
#include "chunk_common.hpp"

namespace dkv {

constexpr int kBlockSide = kBT * kD;          // bytes of a block's keys (or values) of one KV head
constexpr int kBlockBytes = 2 * kBlockSide;
enum BlockFmt { kE4m3 = 0, kInt8 = 1 };
constexpr float kCodeUnit = 32.0f;            // codes enter products as code / 32: at most 14 and 4

// ---- conversions -------------------------------------------------------------------
// Four codes -> four fp16 values code / 32, exactly.  e4m3: the conversion's scale is a power of two.  Integers:
// 128 + code in the low bits of 32.0 (whose last place is 1/32), less 36.
template <int FMT>
__device__ __forceinline__ u2 codes4(uint32_t w)
{
    u2 r;
    if constexpr (FMT == kE4m3) {
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f / kCodeUnit, false));
        r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f / kCodeUnit, true));
    } else {
        const uint32_t x = w ^ 0x80808080u;
        const h2 off = {(_Float16)-36.0f, (_Float16)-36.0f};
        r[0] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x50505050u, x, 0x04010400u)) + off);
        r[1] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x50505050u, x, 0x04030402u)) + off);
    }
    return r;
}
template <int FMT>
__device__ __forceinline__ h8 codes8(uint32_t lo, uint32_t hi)
{
    const u2 a = codes4<FMT>(lo), b = codes4<FMT>(hi);
    return __builtin_bit_cast(h8, u4{a[0], a[1], b[0], b[1]});
}

__device__ __forceinline__ float read_lane_f(float x, int l)  // l uniform
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), l));
}

// ---- the cache --------------------------------------------------------------------------
// Block ID of a sequence's block, -1 where it is none of the pool's.
__device__ __forceinline__ int block_id(const BlockCacheArgs& c, int b, int tile)
{
    const int id = tile < c.width ? c.table[(long long)b * c.width + tile] : -1;
    return id >= 0 && id < c.num_blocks ? id : -1;
}
__device__ __forceinline__ int seq_tokens(const BlockCacheArgs& c, int b)
{
    const int L = c.seq_len[b];
    return L < 0 ? 0 : (L > c.max_len ? c.max_len : L);
}
// Tail rows of (sequence, KV head): 32 rows of keys, 32 of values.
__device__ __forceinline__ const uint16_t* tail_rows(const BlockCacheArgs& c, int b, int h)
{
    return c.tail + ((long long)b * c.Hkv + h) * (2 * kBlockSide);
}

// One number of a state with agent scope, as get_quad.
__device__ __forceinline__ float get_one(__amdgpu_buffer_rsrc_t r, int lane_offset, int offset)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_raw_buffer_load_b32(r, lane_offset, offset, 16));
}

// ---- the item of a wave ----------------------------------------------------------------
// Sequences in order, each with a number of items; a wave finds the one that holds a given item, 64 sequences at a time
// (a lane a sequence).  The last 64 are kept from one search to the next: a call of up to 64 sequences reads their
// lengths once.  In larger ones four 64s' lengths are asked for at once, and where each 64 (or a few of them) starts is kept, a
// lane each, so that a search reads one 64 again (attention of 4096 sequences' single tokens over 128, 8 / 1 heads:
// 99 -> 74 us; of 1024 over 64, 32 / 8 heads: 56 -> 49).  Loads(b, n, L) gives a sequence's rows and tokens, unclamped; rows are
// clamped to [0, most] and to those left of `total`.  Items(n, L): a sequence's items.
struct SeqItem {
    int b, n, L;          // b < 0: there is none
    long long row0;       // the sequence's first row
    long long item0;      // and first item
};
template <typename Loads, typename Items>
struct SeqScan {
    int B, most;
    long long rows;
    Loads loads;
    Items items;
    bool bad = false;                // some length lay outside its range
    int base = -1, n, L;             // the lanes' sequences: base + lane; rows and tokens
    long long before, incl, count;   // rows before the lane's sequence; items up to its end; its items
    long long row_end, item_end;     // behind the 64
    int stride;                      // 64s from one kept start to the next
    long long row_at, item_at;       // the lane's start: rows and items before it

    __device__ __forceinline__ SeqScan(int B_, int most_, long long rows_, Loads l, Items i) : B(B_), most(most_), rows(rows_), loads(l), items(i) {}
    __device__ __forceinline__ void load(int from, long long row, long long item)
    {
        int n0 = 0, L0 = 0;
        if (from + lane_id() < B) loads(from + lane_id(), n0, L0);
        take(from, n0, L0, row, item);
    }
    __device__ __forceinline__ void take(int from, int n0, int L0, long long row, long long item)
    {
        base = from;
        n = n0;
        L = L0;
        const int b = base + lane_id();
        bad = bad || __ballot(n < 0 || n > most) != 0;
        n = n < 0 ? 0 : (n > most ? most : n);
        before = row + (wave_incl_scan_wide(n) - n);
        const long long room = rows - before;
        bad = bad || __ballot(n > room && n > 0) != 0;
        if (n > room) n = room > 0 ? (int)room : 0;
        count = b < B ? items(n, L) : 0;
        incl = item + wave_incl_scan_wide(count);
        row_end = read_lane<long long>(before + n, kWave - 1);
        item_end = read_lane<long long>(incl, kWave - 1);
    }
    // All sequences' items.
    __device__ __forceinline__ long long total()
    {
        constexpr int kAtOnce = 4;
        stride = (B - 1) / (kWave * kWave) + 1;
        row_at = 0;
        item_at = INT64_MAX;
        row_end = item_end = 0;
        int kept = 0, left = 0;
        for (int from = 0; from < B; from += kAtOnce * kWave) {
            int n4[kAtOnce], L4[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const int b = from + i * kWave + lane_id();
                n4[i] = L4[i] = 0;
                if (b < B) loads(b, n4[i], L4[i]);
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                if (from + i * kWave >= B) break;
                if (left == 0) {
                    if (lane_id() == kept) row_at = row_end, item_at = item_end;
                    ++kept;
                    left = stride;
                }
                --left;
                take(from + i * kWave, n4[i], L4[i], row_end, item_end);
            }
        }
        return item_end;
    }
    // The sequence that holds item `want` (after total()).
    __device__ __forceinline__ SeqItem find(long long want)
    {
        if (want < read_lane<long long>(incl - count, 0) || want >= item_end) {
            const int at = __popcll(__ballot(item_at <= want)) - 1;  // the last that starts at `want` or before
            load(at * stride * kWave, read_lane<long long>(row_at, at), read_lane<long long>(item_at, at));
        }
        while (want >= item_end && base + kWave < B) load(base + kWave, row_end, item_end);
        SeqItem s{-1, 0, 0, 0, 0};
        const unsigned long long past = __ballot(incl > want);
        if (past) {
            const int l = __builtin_ctzll(past);
            s.b = base + l;
            s.n = __builtin_amdgcn_readlane(n, l);
            s.L = __builtin_amdgcn_readlane(L, l);
            s.row0 = read_lane<long long>(before, l);
            s.item0 = read_lane<long long>(incl - count, l);
        }
        return s;
    }
};

}  // namespace dkv
