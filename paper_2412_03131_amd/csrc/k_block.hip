// k_block.hip -- writing the uniform 8-bit cache, and reading it back.
//
// Per block of 32 positions, KV head and side, with amax the largest |x| of its 32 x 128 values:
//   e4m3      s = 2^e, e the least with amax <= 448 * 2^e; code = x / s to the nearest e4m3 value (ties to even)
//   integers  s = amax / 127 rounded up to eight significant bits; code = x / s to the nearest integer
// and s = 1 where amax = 0.  Scales of few bits make every code exactly what the definition says: x / s is exact
// for a power of two; for eight bits a quotient of an fp16 value lies on a tie between two codes, or at least 2^-12 from
// one (x and s (n + 1/2) are both multiples of 2^-4 of s's last place), which fp32 tells apart.
// A block with a value that is not finite gets the scale NaN and codes 0.
//
// Bound by memory, with few rows by a chain of loads.  A wave takes one block of one side and KV head, all of it in registers, so
// the maximum needs no second read and no workgroup waits for another: 32768 tokens of 8 KV heads are appended in 46 us (201 MB at
// 4.3 TB/s; 37 where the last-level cache still holds the rows), 16 sequences of 32701 read back in 647 us (3.2 GB at 5.0 TB/s).
#include "block_common.hpp"

namespace dkv {

namespace {

constexpr float kSnap = 1536.0f;        // 1.5 * 2^10: added and taken away, a number below 128 is left in steps of 2^-13
constexpr float kToInt = 12582912.0f;   // 1.5 * 2^23: the sum's low byte is the nearest integer's

// Largest of a wave's 16-bit magnitudes.
__device__ __forceinline__ uint32_t wave_top(uint32_t x)
{
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const uint32_t y = (uint32_t)__shfl_xor((int)x, o);
        x = x > y ? x : y;
    }
    return x;
}
__device__ __forceinline__ uint32_t top_of(uint32_t top, u4 x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = x[i] & 0x7fffu, b = (x[i] >> 16) & 0x7fffu;
        top = top > a ? top : a;
        top = top > b ? top : b;
    }
    return top;
}

struct Scale {
    float s, inv;  // the scale and its inverse (integers: rounded; no code is taken from it but within 2^-17)
    bool fine;     // all values were finite
};
template <int FMT>
__device__ __forceinline__ Scale block_scale(uint32_t top)
{
    Scale r{1.0f, 1.0f, top < 0x7c00u};
    const float amax = h2f(top);
    if (top != 0 && r.fine) {
        uint32_t u;
        if constexpr (FMT == kE4m3) {
            // amax = m 2^x, 1 <= m < 2; 448 = 1.75 * 2^8
            u = __float_as_uint(amax);
            u = (u & 0x7f800000u) - (8u << 23) + ((u & 0x7fffffu) > 0x600000u ? 1u << 23 : 0u);
        } else {
            u = (__float_as_uint(amax / 127.0f) + 0xffffu) & 0xffff0000u;
        }
        r.s = __uint_as_float(u);
        r.inv = 1.0f / r.s;
    }
    return r;
}
template <int FMT>
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d, float inv)
{
    if constexpr (FMT == kE4m3) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
    } else {
        const float x[4] = {a, b, c, d};
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = __float_as_uint((__builtin_fmaf(x[i], inv, kSnap) - kSnap) + kToInt);
        const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(u[3], u[2], 0x0C0C0400u);
        return lo | (hi << 16);
    }
}

// Row of a position: in the tail below L, else among the call's rows.
struct Source {
    const uint16_t* tail;  // 32 rows of kD
    const uint16_t* rows;  // row of position L
    long long stride;
    int L;
};
__device__ __forceinline__ const uint16_t* row_at(const Source& s, int pos)
{
    return pos < s.L ? s.tail + (pos & (kBT - 1)) * kD : s.rows + (long long)(pos - s.L) * s.stride;
}

// A whole block of keys: lane = token % 8 * 8 + chunk of 16 dims.
template <int FMT>
__device__ __forceinline__ float put_keys(const Source& src, int first, uint8_t* to)
{
    const int lane = lane_id(), c = lane & 7, t = lane >> 3;
    u4 x[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint16_t* row = row_at(src, first + t + 8 * i) + c * 16;
        x[i][0] = *reinterpret_cast<const u4*>(row);
        x[i][1] = *reinterpret_cast<const u4*>(row + 8);
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = top_of(top_of(top, x[i][0]), x[i][1]);
    const Scale s = block_scale<FMT>(wave_top(top));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int token = t + 8 * i;
        u4 w = {0, 0, 0, 0};
        if (s.fine) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const u4 v = x[i][j >> 1];
                const uint32_t a = v[(j & 1) * 2], b = v[(j & 1) * 2 + 1];
                w[j] = code4<FMT>(h2f(a & 0xffffu), h2f(a >> 16), h2f(b & 0xffffu), h2f(b >> 16), s.inv);
            }
        }
        *reinterpret_cast<u4*>(to + (token >> 4) * 2048 + c * 256 + (token & 15) * 16) = w;
    }
    return s.fine ? s.s : __builtin_nanf("");
}

// From the lane whose number differs by two.
__device__ __forceinline__ u2 pair_swap(u2 x) { return u2{dpp_u32<0x4E, 0xF>(x[0]), dpp_u32<0x4E, 0xF>(x[1])}; }

// A whole block of values: lane = r * 16 + group of eight dims, which takes the eight tokens of r.
template <int FMT>
__device__ __forceinline__ float put_values(const Source& src, int first, uint8_t* to)
{
    const int lane = lane_id(), dg = lane & 15, r = lane >> 4;
    u4 x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = *reinterpret_cast<const u4*>(row_at(src, first + (e >> 2) * 16 + 4 * r + (e & 3)) + dg * 8);
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = top_of(top, x[e]);
    const Scale s = block_scale<FMT>(wave_top(top));
    u2 w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        w[i] = u2{0, 0};
        if (s.fine) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = h2f((x[e][i >> 1] >> ((i & 1) * 16)) & 0xffffu);
            w[i][0] = code4<FMT>(f[0], f[1], f[2], f[3], s.inv);
            w[i][1] = code4<FMT>(f[4], f[5], f[6], f[7], s.inv);
        }
    }
    // lanes dg and dg ^ 2 have the two halves of eight 16-byte pieces: the lower one takes the first four
    const bool upper = (dg & 2) != 0;
    uint8_t* at = to + (dg >> 2) * 1024 + r * 256 + (dg & 1) * 128 + (upper ? 64 : 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u2 mine = upper ? w[4 + i] : w[i], theirs = pair_swap(upper ? w[i] : w[4 + i]);
        *reinterpret_cast<u4*>(at + i * 16) = upper ? u4{theirs[0], theirs[1], mine[0], mine[1]} : u4{mine[0], mine[1], theirs[0], theirs[1]};
    }
    return s.fine ? s.s : __builtin_nanf("");
}

// One wave per (sequence, span of 32 positions, KV head, side).  A sequence's spans are the blocks that it fills; the
// first of them (or the sequence, if it fills none) also moves the rows that stay into the tail, after it has
// read those that were there.
template <int FMT>
__global__ __launch_bounds__(256) void block_append(BlockAppendArgs a)
{
    bool over = false;  // of the lane's sequences, some has more tokens than a sequence may
    const auto loads = [&](int b, int& n, int& L) {
        n = a.new_len[b];
        L = a.seq_len[b];
        over = over || L < 0 || L > a.max_len || (n > 0 && n > a.max_len - L);
    };
    const auto spans = [&](int n, int L) { return n > 0 ? max((long long)((L + (long long)n) / kBT - L / kBT), 1LL) : 0LL; };
    SeqScan scan(a.B, a.max_new, a.total_new, loads, spans);
    const long long jobs = scan.total() * 2 * a.Hkv;
    // a call with lengths out of their range changes nothing
    if (scan.bad || __any(over)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            if (scan.bad) atomicOr(a.status, (unsigned)DIFFKV_ST_BAD_INPUT);
            else atomicOr(a.status, (unsigned)DIFFKV_ST_TABLE_OVERFLOW);
        }
        return;
    }
    const int lane = lane_id();
    for (long long job = (long long)blockIdx.x * 4 + wave_index(); job < jobs; job += (long long)gridDim.x * 4) {
        const long long want = job / (2 * a.Hkv);
        const int side = (int)(job - want * (2 * a.Hkv)) / a.Hkv, h = (int)(job % a.Hkv);
        const SeqItem s = scan.find(want);
        const int first = s.L / kBT, whole = (s.L + s.n) / kBT - first, i = (int)(want - s.item0);
        uint16_t* tail = a.tail + (((long long)s.b * a.Hkv + h) * 2 + side) * kBlockSide;
        const Source src{tail, a.in[side] + s.row0 * a.in_stride[side] + h * kD, a.in_stride[side], s.L};
        if (i < whole) {
            const int id = block_id(a, s.b, first + i);
            if (id >= 0) {
                uint8_t* to = a.pool + (((long long)id * a.Hkv + h) * 2 + side) * kBlockSide;
                const int pos = (first + i) * kBT;
                const float scale = side == 0 ? put_keys<FMT>(src, pos, to) : put_values<FMT>(src, pos, to);
                if (lane == 0) a.scale[((long long)id * a.Hkv + h) * 2 + side] = scale;
            }
        }
        if (i == 0) {
            // (the tail's old rows are read: nothing below goes before that)
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            const int end = s.L + s.n, from = max(s.L, (first + whole) * kBT);
            for (int p = from + (lane >> 4); p < end; p += 4)
                *reinterpret_cast<u4*>(tail + (p & (kBT - 1)) * kD + (lane & 15) * 8) =
                    *reinterpret_cast<const u4*>(row_at(src, p) + (lane & 15) * 8);
        }
    }
}

// ---- reading back ------------------------------------------------------------------------
// Codes times their scale, exact in fp32, rounded once; beyond the largest fp16 that one.
template <int FMT>
__device__ __forceinline__ uint32_t value2(uint32_t w, int at, float s)
{
    float a, b;
    if constexpr (FMT == kE4m3) {
        typedef float f2 __attribute__((ext_vector_type(2)));
        const f2 x = at ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
        a = x.x * s;
        b = x.y * s;
    } else {
        a = (float)((int)(w << (at ? 8 : 24)) >> 24) * s;
        b = (float)((int)(w << (at ? 0 : 16)) >> 24) * s;
    }
    a = __builtin_isnan(a) ? a : fminf(fmaxf(a, -65504.0f), 65504.0f);
    b = __builtin_isnan(b) ? b : fminf(fmaxf(b, -65504.0f), 65504.0f);
    return f2h_rne(a) | (f2h_rne(b) << 16);
}

// One wave per (sequence, span of 32 positions that its range meets, KV head, side).
template <int FMT>
__global__ __launch_bounds__(256) void block_read(BlockReadArgs a)
{
    const auto loads = [&](int b, int& n, int& L) {
        n = a.count[b];
        L = a.start[b];
    };
    // (a range's first and last position in 64 bits: any start is allowed)
    const auto spans = [&](int n, int L) { return n > 0 ? (((long long)L + n - 1) >> 5) - ((long long)L >> 5) + 1 : 0LL; };
    SeqScan scan(a.B, a.max_count, a.total, loads, spans);
    const long long jobs = scan.total() * 2 * a.Hkv;
    const int lane = lane_id();
    for (long long job = (long long)blockIdx.x * 4 + wave_index(); job < jobs; job += (long long)gridDim.x * 4) {
        const long long want = job / (2 * a.Hkv);
        const int side = (int)(job - want * (2 * a.Hkv)) / a.Hkv, h = (int)(job % a.Hkv);
        const SeqItem s = scan.find(want);
        const int held = seq_tokens(a, s.b);
        const long long tile = ((long long)s.L >> 5) + (want - s.item0), pos0 = tile * kBT;
        const long long lo = s.L, hi = (long long)s.L + s.n;
        uint16_t* out = a.out[side] + s.row0 * a.out_stride[side] + h * kD;
        const auto put = [&](int token, int dim, u4 w) {
            const long long p = pos0 + token;
            if (p >= lo && p < hi) *reinterpret_cast<u4*>(out + (p - lo) * a.out_stride[side] + dim) = w;
        };
        const bool inside = tile >= 0 && tile < held / kBT;
        const int id = inside ? block_id(a, s.b, (int)tile) : -1;
        if (id >= 0) {
            const uint8_t* from = a.pool + (((long long)id * a.Hkv + h) * 2 + side) * kBlockSide;
            const float scale = a.scale[((long long)id * a.Hkv + h) * 2 + side];
            if (side == 0) {
                // lane: eight dims of a token, so that 16 lanes write a whole row
                const int c = lane & 15, t = lane >> 4;
                u2 w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int token = t + 4 * i;
                    w[i] = *reinterpret_cast<const u2*>(from + (token >> 4) * 2048 + (c >> 1) * 256 + (token & 15) * 16 + (c & 1) * 8);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    put(t + 4 * i, c * 8, u4{value2<FMT>(w[i][0], 0, scale), value2<FMT>(w[i][0], 1, scale), value2<FMT>(w[i][1], 0, scale), value2<FMT>(w[i][1], 1, scale)});
            } else {
                const int dg = lane & 15, r = lane >> 4;
                const bool upper = (dg & 2) != 0;
                const uint8_t* at = from + (dg >> 2) * 1024 + r * 256 + (dg & 1) * 128 + (upper ? 64 : 0);
                u2 w[8];  // dim i: tokens 0 .. 7 of r; lanes dg and dg ^ 2 read half of both's pieces each
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const u4 x = *reinterpret_cast<const u4*>(at + i * 16);
                    const u2 lo = {x[0], x[1]}, hi = {x[2], x[3]}, theirs = pair_swap(upper ? lo : hi);
                    w[i] = upper ? theirs : lo;
                    w[4 + i] = upper ? hi : theirs;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    u4 y;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        // the two dims' codes of token e side by side
                        const uint32_t x = ((w[2 * i][e >> 2] >> (8 * (e & 3))) & 0xffu) | (((w[2 * i + 1][e >> 2] >> (8 * (e & 3))) & 0xffu) << 8);
                        y[i] = value2<FMT>(x, 0, scale);
                    }
                    put((e >> 2) * 16 + 4 * r + (e & 3), dg * 8, y);
                }
            }
        } else {
            const bool tail = tile == held / kBT;
            const uint16_t* from = tail_rows(a, s.b, h) + side * kBlockSide;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int token = (lane >> 4) + 4 * i, dim = (lane & 15) * 8;
                u4 w = {0, 0, 0, 0};
                if (tail && pos0 + token < held) w = *reinterpret_cast<const u4*>(from + token * kD + dim);
                put(token, dim, w);
            }
        }
    }
}

// Enough waves for every job of the call, but no more workgroups than keep the device busy (eight for each CU).
unsigned grid_of(long long jobs)
{
    const long long groups = (jobs + 3) / 4;
    return (unsigned)(groups < 1 ? 1 : (groups > 2048 ? 2048 : groups));
}

}  // namespace

hipError_t launch_block_append(const BlockAppendArgs& a, int format, hipStream_t st)
{
    // spans: one for each 32 rows and one or two more per sequence that has rows
    const long long seqs = a.B < a.total_new ? a.B : a.total_new;
    const unsigned grid = grid_of((a.total_new / kBT + seqs) * 2 * a.Hkv);
    return launch1(format == kE4m3 ? block_append<kE4m3> : block_append<kInt8>, grid, 256, st, a);
}

hipError_t launch_block_read(const BlockReadArgs& a, int format, hipStream_t st)
{
    const long long seqs = a.B < a.total ? a.B : a.total;
    const unsigned grid = grid_of((a.total / kBT + 2 * seqs) * 2 * a.Hkv);
    return launch1(format == kE4m3 ? block_read<kE4m3> : block_read<kInt8>, grid, 256, st, a);
}

}  // namespace dkv
