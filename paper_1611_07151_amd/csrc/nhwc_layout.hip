// NCHW maps to channels-last rows and back: a transposition of each image's [C][HW] matrix with a conversion on the way.
#include "nhwc_common.h"

#include <algorithm>

namespace sq {
namespace {

constexpr int kTile = 64;

// n matrices [rows][cols] (row stride ld_in, matrix stride img_in) -> [cols][rows] (ld_out, img_out).
template <typename TI, typename TO>
__global__ __launch_bounds__(256) void transpose_kernel(const TI *in, TO *out, long long rows, long long cols, long long ld_in,
                                                        long long img_in, long long ld_out, long long img_out,
                                                        long long tiles_r, long long tiles_c, long long tiles)
{
    __shared__ float tile[kTile][kTile + 1];
    const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
    for (long long t = blockIdx.x; t < tiles; t += gridDim.x) {
        const long long c0 = t % tiles_c * kTile, q = t / tiles_c;
        const long long r0 = q % tiles_r * kTile, n = q / tiles_r;
        const TI *src = in + n * img_in;
        TO *dst = out + n * img_out;
        for (int i = ty; i < kTile; i += 4)
            if (r0 + i < rows && c0 + tx < cols) tile[i][tx] = to_f32(src[(r0 + i) * ld_in + c0 + tx]);
        __syncthreads();
        for (int i = ty; i < kTile; i += 4)
            if (c0 + i < cols && r0 + tx < rows) dst[(c0 + i) * ld_out + r0 + tx] = from_f32<TO>(tile[tx][i]);
        __syncthreads();
    }
}

template <typename TI, typename TO>
int transpose(const char *name, const void *in, void *out, int N, long long rows, long long cols, long long ld_in, long long img_in,
              long long ld_out, long long img_out)
{
    const long long tr = (rows + kTile - 1) / kTile, tc = (cols + kTile - 1) / kTile, tiles = tr * tc * N;
    const LaunchScope prof(name, 0.0, (double)N * rows * cols * (sizeof(TI) + sizeof(TO)), 0.0);
    hipLaunchKernelGGL((transpose_kernel<TI, TO>), dim3((unsigned)std::min<long long>(tiles, 1 << 20)), dim3(256), 0, current_stream(),
                       (const TI *)in, (TO *)out, rows, cols, ld_in, img_in, ld_out, img_out, tr, tc, tiles);
    return check_launch();
}

template <typename... A> int by_types(int ti, int to, A... a)
{
    if (ti == SQ_F32) return to == SQ_F32 ? transpose<float, float>(a...) : transpose<float, bf16_t>(a...);
    return to == SQ_F32 ? transpose<bf16_t, float>(a...) : transpose<bf16_t, bf16_t>(a...);
}

}  // namespace

int nhwc_pack(const void *in, int in_dtype, void *out, int out_dtype, int N, int C, long long HW, long long ld)
{
    return by_types(in_dtype, out_dtype, "nhwc_pack", in, out, N, (long long)C, HW, HW, C * HW, ld, HW * ld);
}

int nhwc_unpack(const void *in, int in_dtype, void *out, int out_dtype, int N, int C, long long HW, long long ld, int out_channels)
{
    return by_types(in_dtype, out_dtype, "nhwc_unpack", in, out, N, HW, (long long)C, ld, HW * ld, HW, out_channels * HW);
}

}  // namespace sq
