// Rows in microscaled 4-bit floating point (blocks of 32 values of a row with a power of two in common, elements of one sign, two exponent
// and one mantissa bits) and the matrix product of such rows: out[r][j] = act(sum_k X[r][k] W[j][k] + b[j]) + residual[r][j].
#include "linear_common.h"

#include <algorithm>
#include <cmath>

namespace sq {
namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));

// ---- packed rows ------------------------------------------------------------------------------------------------------
// A chunk is 256 values of a row: eight blocks, 128 bytes of codes.  Rows are filled up to whole chunks with zeros.
//   scales  [groups of 32 rows][chunks][2][32] words: the word of half h and row r % 32 has the scales of blocks h, 2 + h, 4 + h and
//           6 + h of the chunk, a byte each.  The 256 bytes of a group and chunk are what a wavefront of the product reads at once, one
//           word a lane, and each of its four instructions of 64 k takes the next byte of that word.
//   codes   [rows][chunks][128 bytes]: two values a byte, the earlier one in the lower half
// Scales come first, so that both parts begin at multiples of 256 bytes and 128 bytes of codes at whole lines.
struct Packed {
    const uint32_t *scales;
    const uint8_t *codes;
};
__host__ __device__ inline int chunks_of(int Cin) { return (int)(((unsigned)Cin + 255) / 256); }
__host__ __device__ inline int groups_of(int rows) { return (int)(((unsigned)rows + 31) / 32); }
size_t scale_bytes(int rows, int Cin) { return (size_t)groups_of(rows) * chunks_of(Cin) * 256; }
Packed packed_at(const void *buffer, int rows, int Cin)
{
    return Packed{(const uint32_t *)buffer, (const uint8_t *)buffer + scale_bytes(rows, Cin)};
}

// The scale's code (exponent + 127) of a block whose largest magnitude has this bit pattern: the power of two of that magnitude less the 2
// of the largest element, 0 where that is no longer a normal number, 255 (NaN) where a value is infinite or NaN.
__device__ __forceinline__ uint32_t scale_code(uint32_t most)
{
    return most >= 0x7f800000u ? 255u : most < 0x01000000u ? 0u : (most >> 23) - 2u;
}
// The power of two as the conversion instructions take it (they look at its exponent bits; 2^-127 is no normal number).
__device__ __forceinline__ float scale_value(uint32_t code) { return __builtin_bit_cast(float, code ? code << 23 : 0x00400000u); }

// Eight values of a block: magnitudes, and the codes for a scale.  The conversion instructions divide by the scale and round to nearest
// even, to 6 at most (as measured on every border and beside it, in both types, down to scales of 2^-127).
template <typename TI> struct Eight;
template <> struct Eight<float> {
    float v[8];
    __device__ __forceinline__ uint32_t most() const
    {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu);
        return m;
    }
    __device__ __forceinline__ uint32_t codes(float scale) const
    {
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
    }
};
template <> struct Eight<bf16_t> {
    bf16_t v[8];
    __device__ __forceinline__ uint32_t most() const
    {
        const u32x4_t w = __builtin_bit_cast(u32x4_t, v);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) m = max(m, max(w[i] << 16 & 0x7fffffffu, w[i] & 0x7fff0000u));
        return m;
    }
    __device__ __forceinline__ uint32_t codes(float scale) const
    {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        Vec<bf16x2, 4> w;
        __builtin_memcpy(&w, v, sizeof(w));
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, w.v[0], scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, w.v[1], scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, w.v[2], scale, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, w.v[3], scale, 3);
    }
};
// Values k to k + 7 of a row of Cin values, zeros behind its end.
template <typename TI> __device__ __forceinline__ Eight<TI> eight_at(const TI *row, int k, int Cin)
{
    Eight<TI> e;
    if (k + 8 <= Cin) {
        __builtin_memcpy(&e, row + k, sizeof(e));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = k + i < Cin ? row[k + i] : TI(0);
    }
    return e;
}

// A workgroup packs one chunk of 32 rows: four lanes take a block, eight values each, a wavefront two rows at a time, four times over.  The
// scales go through LDS, so that their 256 bytes leave in one store.
template <typename TI> __global__ __launch_bounds__(256) void mx_pack_kernel(const TI *in, long long ld, int rows, int Cin, int chunks, uint32_t *scales, uint8_t *codes)
{
    __shared__ uint8_t sc[256];
    const int group = blockIdx.x / (unsigned)chunks, chunk = blockIdx.x - (unsigned)group * chunks;
    const int part = threadIdx.x & 31, k = chunk * 256 + part * 8;
    const unsigned first = (unsigned)group * 32 + (threadIdx.x >> 5);       // then every eighth row
    Eight<TI> e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned r = min(first + 8 * i, (unsigned)rows - 1);
        e[i] = eight_at(in + (long long)r * ld, k, Cin);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned r = first + 8 * i;
        uint32_t most = e[i].most();
        most = max(most, (uint32_t)__builtin_amdgcn_mov_dpp((int)most, 0xB1, 0xf, 0xf, true));      // lanes 1 0 3 2
        most = max(most, (uint32_t)__builtin_amdgcn_mov_dpp((int)most, 0x4E, 0xf, 0xf, true));      // lanes 2 3 0 1
        const uint32_t code = scale_code(most);
        if (r < (unsigned)rows) *(uint32_t *)(codes + ((long long)r * chunks + chunk) * 128 + part * 4) = code == 255 ? 0 : e[i].codes(scale_value(code));
        const int block = part >> 2;
        if ((part & 3) == 0) sc[((block & 1) * 32 + (r & 31)) * 4 + (block >> 1)] = (uint8_t)code;
    }
    __syncthreads();
    if (threadIdx.x < 64) scales[(long long)blockIdx.x * 64 + threadIdx.x] = ((const uint32_t *)sc)[threadIdx.x];
}

// A thread gives eight values back.
template <typename TO> __global__ __launch_bounds__(256) void mx_unpack_kernel(Packed p, TO *out, long long ld, int rows, int Cin, int chunks, int eights)
{
    const unsigned long long e = blockIdx.x * 256ull + threadIdx.x;
    const unsigned long long r = e / (unsigned)eights;
    if (r >= (unsigned)rows) return;
    const int part = (int)(e - r * (unsigned)eights), chunk = part >> 5, block = part >> 2 & 7;
    const uint32_t word = p.scales[((long long)(r >> 5) * chunks + chunk) * 64 + (block & 1) * 32 + (r & 31)];
    const uint32_t c = *(const uint32_t *)(p.codes + ((long long)r * chunks + chunk) * 128 + (part & 31) * 4);
    const int code = word >> (block >> 1) * 8 & 255;
    Vec<TO, 8> v;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // twice the element: 0 1 2 3 4 6 8 12
        const float twice = (float)(0xC8643210u >> ((c >> 4 * i & 7) * 4) & 15);
        const float x = __builtin_ldexpf(c >> 4 * i & 8 ? -twice : twice, code - 128);
        v.v[i] = from_f32<TO>(code == 255 ? __builtin_nanf("") : x);
    }
    TO *at = out + (long long)r * ld + part * 8;
    if (part * 8 + 8 <= Cin) {
        __builtin_memcpy(at, &v, sizeof(v));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (part * 8 + i < Cin) at[i] = v.v[i];
    }
}

// ---- the product -------------------------------------------------------------------------------------------------------
struct MxArgs {
    LinearArgs p;           // in, w, Cin and their ld are not looked at
    Packed x, w;
    int chunks;             // of a row
    int share;              // of the chunks: a workgroup's
};

__device__ __forceinline__ i32x8_t wide(u32x4_t v)
{
    const i32x4_t a = __builtin_bit_cast(i32x4_t, v);
    return __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);       // 4-bit operands are four registers
}

// Few results: a workgroup makes 16 layers of 16 rows; its wavefronts share out the chunks, each holding the 16 x 16 sums, and add up through
// LDS, in order of wavefronts.  Operands go from memory straight into the lanes of v_mfma_scale_f32_16x16x128_f8f6f4: lane l takes
// block l / 16 of row l % 16, 16 bytes, and its scale.
template <typename TO, int MAXW> __global__ __launch_bounds__(64 * MAXW) void mx_wave_kernel(MxArgs a, int tiles_r, int tiles_j)
{
    constexpr int kRow = 20;
    __shared__ float red[MAXW * 16 * kRow];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    const int l16 = lane & 15, q = lane >> 4;
    int tr, tj;
    tile_at(blockIdx.x, tiles_r * tiles_j, tiles_r, tiles_j, tr, tj);
    const int r0 = tr * 16, j0 = tj * 16;
    const long long r = row_at(r0, l16, a.p.rows), j = row_at(j0, l16, a.p.Cout);
    const uint8_t *const xc = a.x.codes + r * a.chunks * 128 + q * 16, *const wc = a.w.codes + j * a.chunks * 128 + q * 16;
    const uint32_t *const xs = a.x.scales + (r >> 5) * a.chunks * 64 + (q & 1) * 32 + (r & 31), *const ws = a.w.scales + (j >> 5) * a.chunks * 64 + (q & 1) * 32 + (j & 31);
    const int shift = (q >> 1) * 8;
    f32x4_t acc = {};
    auto chunks = [&](auto count, int c) {
        constexpr int S = decltype(count)::value;
        u32x4_t x[S][2], w[S][2];
        uint32_t sx[S], sw[S];
#pragma unroll
        for (int i = 0; i < S; ++i) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                w[i][t] = *(const u32x4_t *)(wc + (c + i) * 128ll + t * 64);
                x[i][t] = *(const u32x4_t *)(xc + (c + i) * 128ll + t * 64);
            }
            sw[i] = ws[(c + i) * 64ll];
            sx[i] = xs[(c + i) * 64ll];
        }
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int bw = (int)(sw[i] >> shift), bx = (int)(sx[i] >> shift);
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w[i][0]), wide(x[i][0]), acc, 4, 4, 0, bw, 0, bx);
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w[i][1]), wide(x[i][1]), acc, 4, 4, 2, bw, 2, bx);
        }
    };
    int at = (int)((long long)a.chunks * wave / nw);
    const int end = (int)((long long)a.chunks * (wave + 1) / nw);
    for (; at + 4 <= end; at += 4) chunks(std::integral_constant<int, 4>{}, at);
    for (; at < end; ++at) chunks(std::integral_constant<int, 1>{}, at);
    *(f32x4_t *)&red[(wave * 16 + l16) * kRow + q * 4] = acc;
    __syncthreads();
    if (threadIdx.x < 64) {
        const int row = threadIdx.x >> 2, jj = (threadIdx.x & 3) * 4;
        f32x4_t s = *(const f32x4_t *)&red[row * kRow + jj];
        for (int n = 1; n < nw; ++n) s += *(const f32x4_t *)&red[(n * 16 + row) * kRow + jj];
        float v[4] = {s[0], s[1], s[2], s[3]};
        if (row_in(r0, row, a.p.rows)) finish<TO>(a.p, (long long)r0 + row, j0 + jj, a.p.Cout - j0 - jj, v);
    }
}

template <typename TO> int launch_wave(const MxArgs &a)
{
    const int tr = (a.p.rows - 1) / 16 + 1, tj = (a.p.Cout - 1) / 16 + 1, waves = std::min(a.chunks, 16);
    if (!one_launch((double)tr * tj, 64 * waves)) return SQ_ERR_UNSUPPORTED;
    const LaunchScope prof("mx_wave", linear_flops(a.p), 0);
    hipLaunchKernelGGL((mx_wave_kernel<TO, 16>), dim3((unsigned)tr * tj), dim3(64 * waves), 0, current_stream(), a, tr, tj);
    return check_launch();
}

}  // namespace

size_t mxfp4_packed_bytes(int rows, int Cin) { return scale_bytes(rows, Cin) + (size_t)rows * chunks_of(Cin) * 128; }

int mxfp4_pack(const void *in, int in_dtype, void *out, int rows, int Cin, long long ld)
{
    const int chunks = chunks_of(Cin);
    const double blocks = (double)groups_of(rows) * chunks;
    if (!one_launch(blocks, 256)) return SQ_ERR_UNSUPPORTED;
    const Packed p = packed_at(out, rows, Cin);
    const LaunchScope prof("mx_pack", 0, (in_dtype == SQ_F32 ? 4.0 : 2.0) * rows * Cin + (double)mxfp4_packed_bytes(rows, Cin));
    auto go = [&](auto kernel, auto *from) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, current_stream(), from, ld, rows, Cin, chunks, (uint32_t *)p.scales, (uint8_t *)p.codes);
    };
    if (in_dtype == SQ_F32) go(mx_pack_kernel<float>, (const float *)in);
    else go(mx_pack_kernel<bf16_t>, (const bf16_t *)in);
    return check_launch();
}

int mxfp4_unpack(const void *in, void *out, int out_dtype, int rows, int Cin, long long ld)
{
    const int chunks = chunks_of(Cin), eights = (Cin - 1) / 8 + 1;
    const double blocks = std::ceil((double)rows * eights / 256);
    if (!one_launch(blocks, 256)) return SQ_ERR_UNSUPPORTED;
    const Packed p = packed_at(in, rows, Cin);
    const LaunchScope prof("mx_unpack", 0, (out_dtype == SQ_F32 ? 4.0 : 2.0) * rows * Cin + (double)mxfp4_packed_bytes(rows, Cin));
    auto go = [&](auto kernel, auto *to) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, current_stream(), p, to, ld, rows, Cin, chunks, eights); };
    if (out_dtype == SQ_F32) go(mx_unpack_kernel<float>, (float *)out);
    else go(mx_unpack_kernel<bf16_t>, (bf16_t *)out);
    return check_launch();
}

size_t mxfp4_linear_workspace_bytes(int rows, int Cin, int Cout, int in_dtype)
{
    (void)Cout;
    return in_dtype == SQ_MXFP4 ? 0 : align_up(mxfp4_packed_bytes(rows, Cin), 256);
}

int mxfp4_linear(const LinearArgs &p)
{
    MxArgs a{};
    a.p = p;
    a.chunks = a.share = chunks_of(p.Cin);
    a.w = packed_at(p.w, p.Cout, p.Cin);
    if (!one_launch(((p.rows - 1) / 16 + 1.0) * ((p.Cout - 1) / 16 + 1.0), 1024)) return SQ_ERR_UNSUPPORTED;
    const void *x = p.in;
    if (p.in_dtype != SQ_MXFP4) {
        if (const int rc = mxfp4_pack(p.in, p.in_dtype, p.workspace, p.rows, p.Cin, p.ld_in)) return rc;
        x = p.workspace;
    }
    a.x = packed_at(x, p.rows, p.Cin);
    return p.out_dtype == SQ_F32 ? launch_wave<float>(a) : launch_wave<bf16_t>(a);
}

bool mxfp4_register_kernels()
{
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, (const void *)mx_pack_kernel<float>) == hipSuccess;
}

}  // namespace sq
