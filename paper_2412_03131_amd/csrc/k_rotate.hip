// k_rotate.hip -- rotary positions of queries and keys.
//
// Pair i of a head's first rot_dim dims (i, i + rot_dim/2 in the half style, 2i, 2i + 1 in the
// interleaved one) is turned by pos * freq[i] and scaled:
//   a' = m (a cos t - b sin t), b' = m (b cos t + a sin t);
// the other dims pass.  The angle is taken in 64 bits as turns and reduced to [-1/2, 1/2]
// before the 32-bit sine and cosine: positions of 10^5 times one radian have no digits left
// for it in 32 bits.  fp32 products, one rounding to fp16.
//
// Bound by memory (each value is read and written once): 32767 rows of 48 heads take 159 us, 5.05 TB/s
// (a copy of that size 154).  A lane owns the eight pairs of a
// 16-dim unit and goes over heads, so their sines and cosines, which cost more than
// the rest, serve all of them.
#include "chunk_common.hpp"

namespace dkv {

namespace {

constexpr double kTurns = 0.15915494309189533577;  // 1 / 2 pi

// A wave takes one row's heads, eight at a time: lane = head * 8 + unit.  `waves` per row share them.
__global__ __launch_bounds__(256) void rotate_rows(RotateArgs a, int waves_per_row)
{
    for (long long w = (long long)blockIdx.x * 4 + wave_index(); w < a.rows * waves_per_row; w += (long long)gridDim.x * 4) {
        const long long row = w / waves_per_row;
        const int lane = lane_id(), unit = lane & 7;
        const int half = a.rot_dim >> 1, pairs = half >> 3;  // units that turn
        float cs[8], sn[8];
        const bool turns = unit < pairs;
        if (turns) {
            const double p = (double)a.pos[row];
            const f4 f0 = *reinterpret_cast<const f4*>(a.freq + unit * 8), f1 = *reinterpret_cast<const f4*>(a.freq + unit * 8 + 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                double x = p * ((double)(i < 4 ? f0[i & 3] : f1[i & 3]) * kTurns);
                x -= __builtin_rint(x);
                const float r = (float)x;
                sn[i] = a.scale * __builtin_amdgcn_sinf(r);
                cs[i] = a.scale * __builtin_amdgcn_cosf(r);
            }
        }
        const int heads = a.heads[0] + a.heads[1];
        for (int head = (int)(w - row * waves_per_row) * 8 + (lane >> 3); head < heads; head += waves_per_row * 8) {
            const int which = head >= a.heads[0] ? 1 : 0;
            const int hh = head - (which ? a.heads[0] : 0);
            const uint16_t* in = a.in[which] + row * a.in_stride[which] + hh * kD;
            uint16_t* out = a.out[which] + row * a.out_stride[which] + hh * kD;
            // dims of the unit's two 16-byte pieces
            const int d0 = a.style == 0 && turns ? unit * 8 : unit * 16;
            const int d1 = a.style == 0 && turns ? half + unit * 8 : unit * 16 + 8;
            if (!turns && in == out) continue;
            h8 x = *reinterpret_cast<const h8*>(in + d0), y = *reinterpret_cast<const h8*>(in + d1);
            if (turns) {
                if (a.style == 0) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float p = (float)x[i], q = (float)y[i];
                        x[i] = (_Float16)(p * cs[i] - q * sn[i]);
                        y[i] = (_Float16)(q * cs[i] + p * sn[i]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float p = (float)x[2 * i], q = (float)x[2 * i + 1];
                        x[2 * i] = (_Float16)(p * cs[i] - q * sn[i]);
                        x[2 * i + 1] = (_Float16)(q * cs[i] + p * sn[i]);
                        p = (float)y[2 * i], q = (float)y[2 * i + 1];
                        y[2 * i] = (_Float16)(p * cs[i + 4] - q * sn[i + 4]);
                        y[2 * i + 1] = (_Float16)(q * cs[i + 4] + p * sn[i + 4]);
                    }
                }
            }
            *reinterpret_cast<h8*>(out + d0) = x;
            *reinterpret_cast<h8*>(out + d1) = y;
        }
    }
}

// Sum over the eight lanes of a head, in all of them (fixed order: neighbours, then pairs, then fours).
__device__ __forceinline__ float head_sum(float x)
{
    x += __uint_as_float(dpp_u32<0xB1, 0xF>(__float_as_uint(x)));   // quad_perm 1, 0, 3, 2
    x += __uint_as_float(dpp_u32<0x4E, 0xF>(__float_as_uint(x)));   // quad_perm 2, 3, 0, 1
    x += __uint_as_float(dpp_u32<0x141, 0xF>(__float_as_uint(x)));  // row_half_mirror: 7 - lane of eight
    return x;
}

// The same with each head over its root mean square first, times its side's weights w: a head is whole in its eight lanes'
// registers, so the row is still read once.  Queries, then keys; a side's weights enter the cosines and sines, once per row:
//   a' = m (a (w_a cos) - b (w_b sin)), b' = m (b (w_b cos) + a (w_a sin)), m = 1 / sqrt(mean + eps).
// Bound by memory as the rotation: 32767 rows of 48 heads take 158 us (weights read for every head: 175).
__global__ __launch_bounds__(256) void norm_rotate_rows(RotateArgs a, int waves_per_row)
{
    for (long long w = (long long)blockIdx.x * 4 + wave_index(); w < a.rows * waves_per_row; w += (long long)gridDim.x * 4) {
        const long long row = w / waves_per_row;
        const int lane = lane_id(), unit = lane & 7, part = (int)(w - row * waves_per_row);
        const int half = a.rot_dim >> 1, pairs = half >> 3;  // units that turn
        const bool turns = unit < pairs, halves = a.style == 0;
        // dims of the unit's two 16-byte pieces x, y; pair k is (x[k], y[k]), or neighbours of x, then of y
        const int d0 = halves && turns ? unit * 8 : unit * 16;
        const int d1 = halves && turns ? half + unit * 8 : unit * 16 + 8;
        float cs[8], sn[8];
        if (turns) {
            const double p = (double)a.pos[row];
            const f4 f0 = *reinterpret_cast<const f4*>(a.freq + unit * 8), f1 = *reinterpret_cast<const f4*>(a.freq + unit * 8 + 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                double x = p * ((double)(i < 4 ? f0[i & 3] : f1[i & 3]) * kTurns);
                x -= __builtin_rint(x);
                const float r = (float)x;
                sn[i] = a.scale * __builtin_amdgcn_sinf(r);
                cs[i] = a.scale * __builtin_amdgcn_cosf(r);
            }
        }
        for (int which = 0; which < 2; ++which) {
            if (part * 8 >= a.heads[which]) continue;
            float wa[8], wb[8];  // of the pairs' first and second dims
            {
                const f4 one = {1.0f, 1.0f, 1.0f, 1.0f};
                const float* weight = a.weight[which];
                f4 v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = weight ? *reinterpret_cast<const f4*>(weight + (i < 2 ? d0 : d1) + (i & 1) * 4) : one;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    wa[i] = halves || !turns ? v[i >> 2][i & 3] : v[i >> 1][(i & 1) * 2];
                    wb[i] = halves || !turns ? v[2 + (i >> 2)][i & 3] : v[i >> 1][(i & 1) * 2 + 1];
                }
            }
            float ac[8], as[8], bc[8], bs[8];  // a weight's cosine and sine
            if (turns) {
#pragma unroll
                for (int i = 0; i < 8; ++i) ac[i] = wa[i] * cs[i], as[i] = wa[i] * sn[i], bc[i] = wb[i] * cs[i], bs[i] = wb[i] * sn[i];
            }
            for (int head = part * 8 + (lane >> 3); head < a.heads[which]; head += waves_per_row * 8) {
                const uint16_t* in = a.in[which] + row * a.in_stride[which] + head * kD;
                uint16_t* out = a.out[which] + row * a.out_stride[which] + head * kD;
                h8 x = *reinterpret_cast<const h8*>(in + d0), y = *reinterpret_cast<const h8*>(in + d1);
                float p[8], q[8], sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[i] = (float)x[i];
                    q[i] = (float)y[i];
                    sum = __builtin_fmaf(p[i], p[i], sum);
                    sum = __builtin_fmaf(q[i], q[i], sum);
                }
                const float m = __builtin_amdgcn_rsqf(head_sum(sum) * (1.0f / kD) + a.eps);
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] *= m, q[i] *= m;
                if (!turns) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = (_Float16)(p[i] * wa[i]), y[i] = (_Float16)(q[i] * wb[i]);
                } else if (halves) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[i] = (_Float16)(p[i] * ac[i] - q[i] * bs[i]);
                        y[i] = (_Float16)(q[i] * bc[i] + p[i] * as[i]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x[2 * i] = (_Float16)(p[2 * i] * ac[i] - p[2 * i + 1] * bs[i]);
                        x[2 * i + 1] = (_Float16)(p[2 * i + 1] * bc[i] + p[2 * i] * as[i]);
                        y[2 * i] = (_Float16)(q[2 * i] * ac[i + 4] - q[2 * i + 1] * bs[i + 4]);
                        y[2 * i + 1] = (_Float16)(q[2 * i + 1] * bc[i + 4] + q[2 * i] * as[i + 4]);
                    }
                }
                *reinterpret_cast<h8*>(out + d0) = x;
                *reinterpret_cast<h8*>(out + d1) = y;
            }
        }
    }
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& args, hipStream_t st)
{
    RotateArgs a = args;
    const int heads = a.heads[0] + a.heads[1];
    // as many waves per row as there are groups of eight heads while that leaves the device idle
    const int groups = (heads + 7) / 8;
    long long per = 8192 / a.rows;
    int waves = per < 1 ? 1 : (per < groups ? (int)per : groups);
    // (a launch has less than 2^32 threads: more rows than that go round)
    const long long most = 1 << 22, grid = (a.rows * waves + 3) / 4 < most ? (a.rows * waves + 3) / 4 : most;
    void* kargs[] = {&a, &waves};
    const void* kernel = a.norm ? reinterpret_cast<const void*>(norm_rotate_rows) : reinterpret_cast<const void*>(rotate_rows);
    return hipLaunchKernel(kernel, dim3((unsigned)grid), dim3(256), kargs, 0, st);
}

}  // namespace dkv
