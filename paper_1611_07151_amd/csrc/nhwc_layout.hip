// NCHW maps to channels-last rows and back: a transposition of each image's [layers][pixels] matrix with a conversion on the
// way.  Bound by memory: 64 x 55 x 55 x 128 fp32 to bf16 in 34 us (4.4 TB/s), fp32 back to NCHW in 48 us (4.1 TB/s); in 24 and 32 us
// with the same maps again, part of which then lies in the memory-side cache; one map of 13 x 13 x 512 in 3.8 us, which is the launch.
#include "nhwc_common.h"

#include <algorithm>

namespace sq {
namespace {

// Per image a matrix of `rows` rows of `cols` values (dense within a row, ld_in from row to row) becomes one of `cols` rows.
struct TransposeArgs {
    const void *in;
    void *out;
    long long rows, cols, ld_in, img_in, ld_out, img_out;
    long long tiles_r, tiles_c;     // per image
};

template <typename T> constexpr int kPer = 16 / (int)sizeof(T);

// 16 bytes of a row at any address, of which `have` values exist
template <typename T> __device__ __forceinline__ void load_piece(const T *p, long long have, float (&v)[kPer<T>])
{
    T raw[kPer<T>];
    if (have >= kPer<T>) {
        __builtin_memcpy(raw, p, 16);
    } else {
#pragma unroll
        for (int i = 0; i < kPer<T>; ++i) raw[i] = i < have ? p[i] : T(0);
    }
#pragma unroll
    for (int i = 0; i < kPer<T>; ++i) v[i] = to_f32(raw[i]);
}
template <typename T> __device__ __forceinline__ void store_piece(T *p, long long have, const float (&v)[kPer<T>])
{
    T raw[kPer<T>];
#pragma unroll
    for (int i = 0; i < kPer<T>; ++i) raw[i] = from_f32<T>(v[i]);
    if (have >= kPer<T>) {
        __builtin_memcpy(p, raw, 16);
    } else {
#pragma unroll
        for (int i = 0; i < kPer<T>; ++i)
            if (i < have) p[i] = raw[i];
    }
}

// R x C values per workgroup of 256 threads through LDS as fp32.  Both sides move 16 bytes a lane, along the rows of the input
// and along the rows of the output.
template <typename TI, typename TO, int R, int C> __global__ __launch_bounds__(256) void transpose_kernel(TransposeArgs p)
{
    constexpr int ni = kPer<TI>, no = kPer<TO>, kPitch = C + 1;
    constexpr int LI = C / ni, LO = R / no;      // lanes along a row
    constexpr int KI = R * LI / 256, KO = C * LO / 256;
    static_assert(KI * 256 == R * LI && KO * 256 == C * LO, "whole turns");
    __shared__ float tile[R * kPitch];
    // neighbours along the rows of the output, which share its cache lines, follow each other on one XCD
    const unsigned q = gridDim.x >> 3, rest = gridDim.x & 7, xcd = blockIdx.x & 7;
    const unsigned t = (xcd < rest ? xcd * (q + 1) : rest * (q + 1) + (xcd - rest) * q) + (blockIdx.x >> 3);
    const unsigned per = (unsigned)(p.tiles_r * p.tiles_c), in_image = t % per;
    const long long n = t / per, r0 = (long long)(in_image % (unsigned)p.tiles_r) * R, c0 = (long long)(in_image / (unsigned)p.tiles_r) * C;
    const TI *in = (const TI *)p.in + n * p.img_in;
    TO *out = (TO *)p.out + n * p.img_out;
    {
        const int c = threadIdx.x % LI * ni, r = threadIdx.x / LI;
        float v[KI][ni];
#pragma unroll
        for (int k = 0; k < KI; ++k) {
            const long long row = r0 + r + k * (256 / LI);
            if (row < p.rows && c0 + c < p.cols) load_piece(in + row * p.ld_in + c0 + c, p.cols - c0 - c, v[k]);
        }
#pragma unroll
        for (int k = 0; k < KI; ++k)
#pragma unroll
            for (int i = 0; i < ni; ++i) tile[(r + k * (256 / LI)) * kPitch + c + i] = v[k][i];
    }
    __syncthreads();
    const int r = threadIdx.x % LO * no, c = threadIdx.x / LO;
#pragma unroll
    for (int k = 0; k < KO; ++k) {
        const long long row = c0 + c + k * (256 / LO);
        if (row >= p.cols || r0 + r >= p.rows) continue;
        float v[no];
#pragma unroll
        for (int i = 0; i < no; ++i) v[i] = tile[(r + i) * kPitch + c + k * (256 / LO)];
        store_piece(out + row * p.ld_out + r0 + r, p.rows - r0 - r, v);
    }
}

template <typename TI, typename TO, int R, int C> int launch(const char *name, TransposeArgs p, int N)
{
    p.tiles_r = (p.rows + R - 1) / R;
    p.tiles_c = (p.cols + C - 1) / C;
    const long long tiles = p.tiles_r * p.tiles_c;
    if (!one_launch((double)tiles, 256)) return SQ_ERR_UNSUPPORTED;
    const int most = images_in_one_launch(N, (double)tiles, 256);
    for (long long n = 0; n < N; n += most) {
        const int images = (int)std::min<long long>(most, N - n);
        const LaunchScope prof(name, 0.0, (double)images * p.rows * p.cols * (sizeof(TI) + sizeof(TO)), 0.0);
        hipLaunchKernelGGL((transpose_kernel<TI, TO, R, C>), dim3((unsigned)(tiles * images)), dim3(256), 0, current_stream(), p);
        if (const int rc = check_launch()) return rc;
        p.in = (const TI *)p.in + p.img_in * images;
        p.out = (TO *)p.out + p.img_out * images;
    }
    return SQ_OK;
}

// 64 layers x 64 pixels; 32 x 128 where that leaves less of the tiles empty (96 layers, fp32 to bfloat16: 123 -> 101 us for 64 maps
// of 111 x 111), 16 x 256 up to 16 layers (3 layers, 64 maps of 224 x 224 fp32: 55 -> 19 us in, 53 -> 18 us back).
template <typename TI, typename TO, bool PACK> int transpose(const char *name, const TransposeArgs &p, int N, long long layers)
{
    if (layers <= 16) return PACK ? launch<TI, TO, 16, 256>(name, p, N) : launch<TI, TO, 256, 16>(name, p, N);
    const long long by64 = (layers + 63) / 64 * 64, by32 = (layers + 31) / 32 * 32;
    if (by64 > by32 + by32 / 8) return PACK ? launch<TI, TO, 32, 128>(name, p, N) : launch<TI, TO, 128, 32>(name, p, N);
    return launch<TI, TO, 64, 64>(name, p, N);
}

template <bool PACK> int by_types(int ti, int to, const char *name, const TransposeArgs &p, int N, long long layers)
{
    if (ti == SQ_F32) return to == SQ_F32 ? transpose<float, float, PACK>(name, p, N, layers) : transpose<float, bf16_t, PACK>(name, p, N, layers);
    return to == SQ_F32 ? transpose<bf16_t, float, PACK>(name, p, N, layers) : transpose<bf16_t, bf16_t, PACK>(name, p, N, layers);
}

}  // namespace

bool nhwc_layout_register_kernels()
{
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, (const void *)transpose_kernel<float, float, 64, 64>) == hipSuccess;
}

int nhwc_pack(const void *in, int in_dtype, void *out, int out_dtype, int N, int C, long long HW, long long ld)
{
    return by_types<true>(in_dtype, out_dtype, "nhwc_pack", TransposeArgs{in, out, C, HW, HW, C * HW, ld, HW * ld, 0, 0}, N, C);
}

int nhwc_unpack(const void *in, int in_dtype, void *out, int out_dtype, int N, int C, long long HW, long long ld, int out_channels)
{
    return by_types<false>(in_dtype, out_dtype, "nhwc_unpack", TransposeArgs{in, out, HW, C, ld, HW * ld, HW, out_channels * HW, 0, 0}, N, C);
}

}  // namespace sq
