// k_chunk.hip -- host side of the chunk attention and score kernels (chunk_kernels.hpp,
// instantiated per page layout in k_chunk_l<n>.hip), and the join of split rows.
#include "chunk_common.hpp"

namespace dkv {

// Joins the partial states of a row's splits: one wave per (token, query head), two dims a lane.
__global__ __launch_bounds__(256) void chunk_join(ChunkArgs a)
{
    set_fp16_saturate();
    const long long row = (long long)blockIdx.x * 4 + wave_index();
    if (row >= a.total_new * a.Hq) return;
    const int lane = lane_id();
    const float* part = a.part + row * a.splits * kChunkPart;
    float m = kLowest, sum = 0.0f, o0 = 0.0f, o1 = 0.0f;
    for (int s = 0; s < a.splits; ++s) m = fmaxf(m, part[s * kChunkPart + kD]);
    for (int s = 0; s < a.splits; ++s) {
        const float f = __builtin_amdgcn_exp2f(part[s * kChunkPart + kD] - m);
        sum += f * part[s * kChunkPart + kD + 1];
        o0 += f * part[s * kChunkPart + 2 * lane];
        o1 += f * part[s * kChunkPart + 2 * lane + 1];
    }
    const float inv = 1.0f / sum;
    const h2 r = {(_Float16)(o0 * inv), (_Float16)(o1 * inv)};
    *reinterpret_cast<h2*>(a.out + row * kD + 2 * lane) = r;
    if (a.lse && lane == 0) a.lse[row] = kChunkLn2 * (m + __builtin_amdgcn_logf(sum));
}

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

// Workgroups per row block: about 1024 in all, no more than the longest table there can be has
// steps of 32 tokens for their waves, at most 64.
int chunk_splits(long long B, long long Hq, long long Hkv, long long total_new, long long p_max)
{
    const long long G = Hq / Hkv;
    const long long seqs = B < total_new ? B : total_new;
    const long long items = Hkv * (seqs + total_new * G / 64);
    const long long most = p_max / 8 + 1;
    long long s = items > 0 ? 1024 / items : 1;
    if (s > most) s = most;
    if (s > 64) s = 64;
    return (int)(s < 1 ? 1 : s);
}

hipError_t launch_chunk_attention(const ChunkArgs& args, bool mod, hipStream_t st)
{
    ChunkArgs a = args;
    const long long G = a.Hq / a.Hkv;
    const long long rows = a.max_new * G;
    const int rt = rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
    const void* kern = chunk_kernel(a.layout, rt, mod);
    if (!kern) return hipErrorInvalidValue;
    a.rows_lo = 1;
    a.rows_hi = INT32_MAX;
    // row blocks: at most one more than whole ones per sequence, and as many as the longest has
    const long long per = 16 * rt, seqs = a.B < a.total_new ? a.B : a.total_new;
    long long blocks = a.total_new * G / per + seqs;
    const long long other = seqs * ((rows + per - 1) / per);
    if (other < blocks) blocks = other;
    const long long grid = blocks * a.Hkv * a.splits;
    if (grid < 1 || grid > INT32_MAX) return hipErrorInvalidValue;
    void* kargs[] = {&a};
    hipError_t e = hipLaunchKernel(kern, dim3((unsigned)grid), dim3(4 * kWave), kargs, 0, st);
    if (e != hipSuccess || a.splits == 1) return e;
    return launch1(chunk_join, (unsigned)((a.total_new * a.Hq + 3) / 4), 256, st, a);
}

hipError_t launch_chunk_scores(const ChunkArgs& args, bool mod, hipStream_t st)
{
    ChunkArgs a = args;
    const void* kern = chunk_kernel(a.layout, 0, mod);
    if (!kern) return hipErrorInvalidValue;
    const long long T = (long long)a.B * a.Hkv;
    const long long most = (long long)a.p_max * 16 / 256 + 3 + (a.max_new + 255) / 256;
    long long shares = (4096 + T - 1) / T;
    if (shares > most) shares = most;
    a.shares = (int)shares;
    const long long grid = T * shares;
    if (grid < 1 || grid > INT32_MAX) return hipErrorInvalidValue;
    void* kargs[] = {&a};
    return hipLaunchKernel(kern, dim3((unsigned)grid), dim3(4 * kWave), kargs, 0, st);
}

}  // namespace dkv
