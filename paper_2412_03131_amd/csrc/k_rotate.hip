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
    return hipLaunchKernel(reinterpret_cast<const void*>(rotate_rows), dim3((unsigned)grid), dim3(256), kargs, 0, st);
}

}  // namespace dkv
