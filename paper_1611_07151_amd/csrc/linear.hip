// Matrix product of rows with bias, activation and residual: out[r][j] = act(sum_k in[r][k] w[j][k] + b[j]) + residual[r][j].
#include "nhwc_common.h"

#include <algorithm>

namespace sq {
namespace {

constexpr int kTile = 64, kStep = 16;

// 64 x 64 results per workgroup of 256 threads, 4 x 4 per thread, fp32 sums of fp32 products.
template <typename TI, typename TO, int ACT> __global__ __launch_bounds__(256) void linear_kernel(LinearArgs p, long long tiles_j, long long tiles)
{
    __shared__ float xs[kStep][kTile + 4], ws[kStep][kTile + 4];
    const int t = threadIdx.x, tr = t >> 4, tj = t & 15;
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const long long r0 = tile / tiles_j * kTile, j0 = tile % tiles_j * kTile;
        float acc[4][4] = {};
        for (int k0 = 0; k0 < p.Cin; k0 += kStep) {
            __syncthreads();
            for (int i = t; i < kTile * kStep; i += 256) {
                const int k = i % kStep, row = i / kStep;
                const bool kin = k0 + k < p.Cin;
                xs[k][row] = kin && r0 + row < p.rows ? to_f32(((const TI *)p.in)[(r0 + row) * p.ld_in + k0 + k]) : 0.f;
                ws[k][row] = kin && j0 + row < p.Cout ? to_f32(((const TI *)p.w)[(j0 + row) * p.Cin + k0 + k]) : 0.f;
            }
            __syncthreads();
            for (int k = 0; k < kStep; ++k)
                for (int a = 0; a < 4; ++a)
                    for (int b = 0; b < 4; ++b) acc[a][b] += xs[k][tr * 4 + a] * ws[k][tj * 4 + b];
        }
        for (int a = 0; a < 4; ++a)
            for (int b = 0; b < 4; ++b) {
                const long long r = r0 + tr * 4 + a, j = j0 + tj * 4 + b;
                if (r >= p.rows || j >= p.Cout) continue;
                float v = activate<ACT>(acc[a][b] + (p.b ? p.b[j] : 0.f));
                if (p.residual) v += to_f32(((const TO *)p.residual)[r * p.ld_res + j]);
                ((TO *)p.out)[r * p.ld_out + j] = from_f32<TO>(v);
            }
    }
}

template <typename TI, typename TO, int ACT> int launch(const LinearArgs &p)
{
    const long long tj = (p.Cout + kTile - 1) / kTile, tiles = tj * ((p.rows + kTile - 1) / kTile);
    const LaunchScope prof("linear", linear_flops(p), linear_bytes(p), 0.0);
    hipLaunchKernelGGL((linear_kernel<TI, TO, ACT>), dim3((unsigned)std::min<long long>(tiles, 1 << 20)), dim3(256), 0, current_stream(), p, tj, tiles);
    return check_launch();
}

template <typename TI, typename TO> int by_act(const LinearArgs &p)
{
    switch (p.act) {
        case SQ_ACT_NONE: return launch<TI, TO, SQ_ACT_NONE>(p);
        case SQ_ACT_RELU: return launch<TI, TO, SQ_ACT_RELU>(p);
        case SQ_ACT_SILU: return launch<TI, TO, SQ_ACT_SILU>(p);
        default: return launch<TI, TO, SQ_ACT_GELU>(p);
    }
}

}  // namespace

size_t linear_workspace_bytes(int, int, int, int) { return 0; }

int linear(const LinearArgs &p)
{
    if (p.in_dtype == SQ_F32) return by_act<float, float>(p);
    return p.out_dtype == SQ_F32 ? by_act<bf16_t, float>(p) : by_act<bf16_t, bf16_t>(p);
}

}  // namespace sq
