// Group norm with an activation on channels-last maps.
#include "nhwc_common.h"

#include <algorithm>

namespace sq {
namespace {

struct NormArgs {
    const void *in;
    void *out;
    const float *gamma, *beta;
    int N, C, G;
    long long HW, ld_in, ld_out;
    float eps;
};

__device__ float block_sum(float v, float *s)
{
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    return s[0] + s[1] + s[2] + s[3];
}

// One workgroup per image and group, which it reads three times: mean, squared deviation, result.
template <typename T, int ACT> __global__ __launch_bounds__(256) void group_norm_kernel(NormArgs p)
{
    __shared__ float s[4];
    const int cg = p.C / p.G, n = blockIdx.x / p.G, g = blockIdx.x % p.G;
    const T *in = (const T *)p.in + n * p.HW * p.ld_in + g * cg;
    T *out = (T *)p.out + n * p.HW * p.ld_out + g * cg;
    const long long m = p.HW * cg;
    float sum = 0.f, sq = 0.f;
    for (long long i = threadIdx.x; i < m; i += 256) sum += to_f32(in[i / cg * p.ld_in + i % cg]);
    const float mean = block_sum(sum, s) / (float)m;
    for (long long i = threadIdx.x; i < m; i += 256) {
        const float d = to_f32(in[i / cg * p.ld_in + i % cg]) - mean;
        sq += d * d;
    }
    const float inv = 1.f / sqrtf(block_sum(sq, s) / (float)m + p.eps);
    for (long long i = threadIdx.x; i < m; i += 256) {
        const int c = (int)(i % cg);
        const float d = (to_f32(in[i / cg * p.ld_in + c]) - mean) * inv;
        const float v = d * (p.gamma ? p.gamma[g * cg + c] : 1.f) + (p.beta ? p.beta[g * cg + c] : 0.f);
        out[i / cg * p.ld_out + c] = from_f32<T>(activate<ACT>(v));
    }
}

template <typename T, int ACT> int launch(const NormArgs &p)
{
    const double values = (double)p.N * p.HW * p.C;
    const LaunchScope prof("group_norm", 10.0 * values, 2.0 * sizeof(T) * values, 0.0);
    hipLaunchKernelGGL((group_norm_kernel<T, ACT>), dim3((unsigned)p.N * p.G), dim3(256), 0, current_stream(), p);
    return check_launch();
}

template <typename T> int by_act(const NormArgs &p, int act)
{
    switch (act) {
        case SQ_ACT_NONE: return launch<T, SQ_ACT_NONE>(p);
        case SQ_ACT_RELU: return launch<T, SQ_ACT_RELU>(p);
        case SQ_ACT_SILU: return launch<T, SQ_ACT_SILU>(p);
        default: return launch<T, SQ_ACT_GELU>(p);
    }
}

}  // namespace

size_t nhwc_group_norm_workspace_bytes(int, int, long long, int) { return 0; }

int nhwc_group_norm(const void *in, void *out, int dtype, const float *gamma, const float *beta, int N, int C, long long HW, int G,
                    float eps, int act, long long ld_in, long long ld_out, void *, size_t)
{
    const NormArgs p{in, out, gamma, beta, N, C, G, HW, ld_in, ld_out, eps};
    return dtype == SQ_F32 ? by_act<float>(p, act) : by_act<bf16_t>(p, act);
}

}  // namespace sq
