// k_chunk.hip -- host side of the chunk attention and score kernels (chunk_kernels.hpp,
// instantiated per page layout in k_chunk_l<n>.hip): which of them takes which sequences, the workspace.
#include "chunk_common.hpp"

namespace dkv {

static const void* chunk_kernel(int li, int which, bool mod)
{
    switch (li) {
    case 0: return chunk_kernel_l0(which, mod);
    case 1: return chunk_kernel_l1(which, mod);
    case 2: return chunk_kernel_l2(which, mod);
    case 3: return chunk_kernel_l3(which, mod);
    default: return nullptr;
    }
}

static long long align256(long long x) { return (x + 255) & ~255ll; }

ChunkPlan chunk_plan(long long B, long long Hq, long long Hkv, long long total_new)
{
    ChunkPlan p{};
    const long long G = Hq / Hkv, rows = total_new * G;
    const long long seqs = B < total_new ? B : total_new;
    auto clamp = [](long long x, long long lo, long long hi) { return x < lo ? lo : (x > hi ? hi : x); };
    p.few_rows = total_new * Hq <= kChunkFewTotal && rows > kChunkFewRows ? rows : kChunkFewRows;
    auto blocks_of = [&](long long n) {  // (in blocks of 32: two each)
        return Hkv * clamp(rows / 16 + 2 * n, 0, n * ((p.few_rows + 31) / 32 * 2));
    };
    p.few_blocks = blocks_of(seqs);
    p.few_split = B * Hkv < kRowPieces;
    // Room for the states of the largest batch up to this one that is split, and not by the rows: a workspace
    // for many sequences and rows serves calls of fewer.
    // (row_piece makes at most kRowPieces and one per block of them, of 16 rows; of 32 half as many)
    const long long split = clamp((kRowPieces - 1) / Hkv, 0, seqs);
    p.few_part = split > 0 ? (kRowPieces + blocks_of(split)) * 16 * kChunkPart : 0;
    p.bytes = align256((p.few_blocks + kTileShares) * 8) + align256(p.few_part * 4) +
              (rows > p.few_rows ? 2ll * kTileShares * kChunkRows * kChunkPart * 4 : 0);
    return p;
}

hipError_t launch_chunk_attention(const ChunkArgs& args, const ChunkPlan& plan, bool mod, hipStream_t st)
{
    const long long G = args.Hq / args.Hkv, rows = args.max_new * G;
    const long long seqs = args.B < args.total_new ? args.B : args.total_new;
    unsigned long long* arrive = args.arrive;
    float* part = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(arrive) + align256((plan.few_blocks + kTileShares) * 8));
    auto launch = [&](ChunkArgs& a, int which, long long grid, int threads) {
        const void* kern = chunk_kernel(a.layout, which, mod);
        if (!kern || grid < 1 || grid > UINT32_MAX / threads) return hipErrorInvalidValue;
        void* kargs[] = {&a};
        return hipLaunchKernel(kern, dim3((unsigned)grid), dim3((unsigned)threads), kargs, 0, st);
    };
    if (rows > plan.few_rows) {
        ChunkArgs a = args;
        // With room for the longest chunk in every sequence all lengths are that one, or the rows are padded:
        // these take all sequences then, and no second launch (4-5 us) looks for shorter ones.
        const bool all = args.total_new == (long long)args.B * args.max_new;
        a.rows_lo = all ? 1 : 17;
        a.rows_hi = INT32_MAX;
        a.arrive = arrive + plan.few_blocks;
        a.part = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(part) + align256(plan.few_part * 4));
        const hipError_t e = launch(a, 3, kTileShares, kTileThreads);
        if (e != hipSuccess || all) return e;
    }
    // Few rows: all sequences if none is longer, else those of one block of 16 rows
    ChunkArgs a = args;
    a.rows_lo = 1;
    a.rows_hi = rows > plan.few_rows ? 16 : (int)plan.few_rows;
    a.part = part;
    // Two row tiles share a step's dequantization (20 rows for each of 64 sequences over 2048 tokens 55 us, with
    // one tile 62; 64 rows 104 and 123; 128 rows for 4 over 8192 53 and 62; only 32 rows for 4 31 and 29)
    const int rt = rows > 16 && rows <= plan.few_rows ? 2 : 1;
    a.splits = plan.few_split ? 0 : 1;
    a.blocks = (int)(plan.few_blocks < INT32_MAX ? plan.few_blocks : INT32_MAX);
    a.pieces = kRowPieces / rt;  // (a CU holds half as many workgroups with two row tiles)
    const long long per = 16 * rt, most = rows < a.rows_hi ? rows : a.rows_hi;
    const long long whole = args.total_new * G / per + seqs, each = seqs * ((most + per - 1) / per);
    const long long blocks = (whole < each ? whole : each) * a.Hkv;
    if (!plan.few_split) {
        // (256 sequences' single tokens over 100-1000, 32 / 8 heads: 53 us, 54 where each workgroup searches; 1500 of 4 / 1
        // over 100-600 36 and 44)
        a.one_block = most <= per;
        return launch(a, rt, a.one_block ? (long long)a.B * a.Hkv : blocks, 4 * kWave);
    }
    // a piece has at least a step for each of its four waves, a table at most a step per page and its own
    const long long pieces = blocks * ((a.p_max + 2 + (a.max_new + 31) / 32 + 3) / 4), cap = a.pieces + blocks;
    return launch(a, rt, pieces < cap ? pieces : cap, 4 * kWave);
}

hipError_t launch_chunk_scores(const ChunkArgs& args, bool mod, hipStream_t st)
{
    ChunkArgs a = args;
    const long long G = a.Hq / a.Hkv, T = (long long)a.B * a.Hkv;
    const bool longs = ((long long)a.max_new + 3) / 4 * ((G + 3) / 4) > 4;
    if (longs) {
        // four heads a set where four divides them (8 x 256 tokens over 4096, sets of four heads and positions /
        // of sixteen positions: 4 query heads per KV head 100 / 109 us, 3 100 / 95, 5 160 / 128, 6 159 / 144, 7 165 / 164)
        const void* kern = chunk_kernel(a.layout, G % 4 == 0 ? 4 : 0, mod);
        if (!kern) return hipErrorInvalidValue;
        // (as for attention: one length, or padded rows)
        a.all_lengths = a.total_new == (long long)a.B * a.max_new;
        void* kargs[] = {&a};
        const hipError_t e = hipLaunchKernel(kern, dim3(kScoreShares), dim3(8 * kWave), kargs, 0, st);
        if (e != hipSuccess || a.all_lengths) return e;
    }
    const void* kern = chunk_kernel(a.layout, 5, mod);
    if (!kern) return hipErrorInvalidValue;
    // about 1024 workgroups, a step for each of their waves
    const long long most = (a.p_max / 2 + 2 + 7) / 8;
    long long shares = (1024 + T - 1) / T;
    if (shares > most) shares = most;
    a.splits = (int)(shares < 1 ? 1 : shares);
    const long long grid = T * a.splits;
    if (grid > UINT32_MAX / (8 * kWave)) return hipErrorInvalidValue;
    void* kargs[] = {&a};
    return hipLaunchKernel(kern, dim3((unsigned)grid), dim3(8 * kWave), kargs, 0, st);
}

}  // namespace dkv
