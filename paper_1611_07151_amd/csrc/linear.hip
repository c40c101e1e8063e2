// Matrix product of rows with bias, activation and residual: out[r][j] = act(sum_k in[r][k] w[j][k] + b[j]) + residual[r][j].
#include "nhwc_common.h"

#include <algorithm>

namespace sq {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

__device__ __forceinline__ float activate_by(float v, int act)
{
    switch (act) {      // the same for the whole launch
        case SQ_ACT_RELU: return activate<SQ_ACT_RELU>(v);
        case SQ_ACT_SILU: return activate<SQ_ACT_SILU>(v);
        case SQ_ACT_GELU: return activate<SQ_ACT_GELU>(v);
        default: return v;
    }
}

template <typename T, int n> struct Vec {
    T v[n];
};
// row first + i where there is one, else the last row (its results are not written)
__device__ __forceinline__ long long row_at(int first, int i, int rows) { return min((unsigned)first + i, (unsigned)rows - 1); }
__device__ __forceinline__ bool row_in(int first, int i, int rows) { return (unsigned)first + i < (unsigned)rows; }

// n values at any address their type allows (global memory takes unaligned wide loads and stores)
template <int n, typename T> __device__ __forceinline__ Vec<T, n> load_n(const T *p)
{
    Vec<T, n> r;
    __builtin_memcpy(&r, p, sizeof(r));
    return r;
}

// Bias, activation and residual of n neighbouring results of one row, of which the first `have` exist.
template <typename TO, int n> __device__ __forceinline__ void finish(const LinearArgs &p, long long r, int j, int have, float (&v)[n])
{
    if (have <= 0) return;
    TO *out = (TO *)p.out + r * p.ld_out + j;
    const TO *res = (const TO *)p.residual + r * p.ld_res + j;
    if (have >= n) {
        if (p.b) {
            const Vec<float, n> b = load_n<n>(p.b + j);
#pragma unroll
            for (int i = 0; i < n; ++i) v[i] += b.v[i];
        }
        if (p.act != SQ_ACT_NONE) {
#pragma unroll
            for (int i = 0; i < n; ++i) v[i] = activate_by(v[i], p.act);
        }
        if (p.residual) {
            const Vec<TO, n> q = load_n<n>(res);
#pragma unroll
            for (int i = 0; i < n; ++i) v[i] += to_f32(q.v[i]);
        }
        Vec<TO, n> o;
#pragma unroll
        for (int i = 0; i < n; ++i) o.v[i] = from_f32<TO>(v[i]);
        __builtin_memcpy(out, &o, sizeof(o));
        return;
    }
#pragma unroll
    for (int i = 0; i < n; ++i)
        if (i < have) {
            float s = activate_by(p.b ? v[i] + p.b[j + i] : v[i], p.act);
            if (p.residual) s += to_f32(res[i]);
            out[i] = from_f32<TO>(s);
        }
}

// 16 bytes of a row from k on, of which `have` values exist (the rest zero).
template <typename TI> __device__ __forceinline__ u32x4_t load16_tail(const TI *p, int have)
{
    constexpr int n = 16 / sizeof(TI);
    Vec<TI, n> r;
#pragma unroll
    for (int i = 0; i < n; ++i) r.v[i] = i < have ? p[i] : TI(0);
    return __builtin_bit_cast(u32x4_t, r);
}
template <typename TI> __device__ __forceinline__ u32x4_t load16(const TI *p)
{
    return __builtin_bit_cast(u32x4_t, load_n<16 / (int)sizeof(TI)>(p));
}

// ---- few results: wavefronts that share out the sum ---------------------------------------------------------------
// A workgroup makes CT layers of RT rows; its wavefronts share out k in pieces of 64 bytes of a row ("steps"), each
// holding the whole RT x CT block of sums in registers, and add up through LDS, in order of wavefronts.  Operands go
// from memory straight into the lanes of v_mfma_f32_16x16x32_bf16 / _16x16x4_f32: lane l takes 16 bytes of row l % 16 at
// piece l / 16 of the step (fp32: value i of every lane's four is one instruction; both operands number k alike).
template <typename TI, typename TO, int RT, int CT, int MAXW>
__global__ __launch_bounds__(64 * MAXW) void linear_wave_kernel(LinearArgs p, int tiles_j, long long tiles)
{
    constexpr int RB = RT / 16, CB = CT / 16, kStep = 64 / (int)sizeof(TI), kPiece = 16 / (int)sizeof(TI), kRow = CT + 4;
    constexpr int kMost = 16 / (RB + CB) ? 16 / (RB + CB) : 1;       // steps whose loads fly together
    __shared__ float red[MAXW * RT * kRow];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
    const int l16 = lane & 15, piece = lane >> 4;
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int r0 = (int)(tile / tiles_j) * RT, j0 = (int)(tile % tiles_j) * CT;
        const TI *xr[RB], *wr[CB];
#pragma unroll
        for (int i = 0; i < RB; ++i) xr[i] = (const TI *)p.in + row_at(r0, 16 * i + l16, p.rows) * p.ld_in + piece * kPiece;
#pragma unroll
        for (int i = 0; i < CB; ++i) wr[i] = (const TI *)p.w + row_at(j0, 16 * i + l16, p.Cout) * p.Cin + piece * kPiece;
        f32x4_t acc[CB][RB] = {};
        auto multiply = [&](const u32x4_t (&a)[CB], const u32x4_t (&b)[RB]) {
#pragma unroll
            for (int c = 0; c < CB; ++c)
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    if constexpr (sizeof(TI) == 2) {
                        acc[c][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[c]), __builtin_bit_cast(bf16x8, b[r]), acc[c][r], 0, 0, 0);
                    } else {
                        const f32x4_t af = __builtin_bit_cast(f32x4_t, a[c]), bf = __builtin_bit_cast(f32x4_t, b[r]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[c][r] = __builtin_amdgcn_mfma_f32_16x16x4f32(af[i], bf[i], acc[c][r], 0, 0, 0);
                    }
                }
        };
        auto steps = [&](auto count, int k) {
            constexpr int S = decltype(count)::value;
            u32x4_t a[S][CB], b[S][RB];
#pragma unroll
            for (int s = 0; s < S; ++s) {
#pragma unroll
                for (int c = 0; c < CB; ++c) a[s][c] = load16(wr[c] + k + s * kStep);
#pragma unroll
                for (int r = 0; r < RB; ++r) b[s][r] = load16(xr[r] + k + s * kStep);
            }
#pragma unroll
            for (int s = 0; s < S; ++s) multiply(a[s], b[s]);
        };
        const int whole = p.Cin / kStep;
        int at = (int)((long long)whole * wave / nw);
        const int end = (int)((long long)whole * (wave + 1) / nw);
        for (; at + kMost <= end; at += kMost) steps(std::integral_constant<int, kMost>{}, at * kStep);
        if constexpr (kMost >= 8)
            if (at + 4 <= end) { steps(std::integral_constant<int, 4>{}, at * kStep); at += 4; }
        if constexpr (kMost >= 4)
            if (at + 2 <= end) { steps(std::integral_constant<int, 2>{}, at * kStep); at += 2; }
        for (; at < end; ++at) steps(std::integral_constant<int, 1>{}, at * kStep);
        if (wave == nw - 1 && whole * kStep < p.Cin) {
            const int k = whole * kStep, have = p.Cin - k - piece * kPiece;
            u32x4_t a[CB], b[RB];
#pragma unroll
            for (int c = 0; c < CB; ++c) a[c] = load16_tail(wr[c] + k, have);
#pragma unroll
            for (int r = 0; r < RB; ++r) b[r] = load16_tail(xr[r] + k, have);
            multiply(a, b);
        }
        // lane holds, of row l16 of every block of rows, four neighbouring layers of every block of layers
        __syncthreads();
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int r = 0; r < RB; ++r) *(f32x4_t *)&red[(wave * RT + r * 16 + l16) * kRow + c * 16 + piece * 4] = acc[c][r];
        __syncthreads();
        for (int e = threadIdx.x; e < RT * CT / 4; e += blockDim.x) {
            const int r = e / (CT / 4), j = e % (CT / 4) * 4;
            f32x4_t s = *(const f32x4_t *)&red[r * kRow + j];
            for (int q = 1; q < nw; ++q) s += *(const f32x4_t *)&red[(q * RT + r) * kRow + j];
            float v[4] = {s[0], s[1], s[2], s[3]};
            if (row_in(r0, r, p.rows)) finish<TO>(p, (long long)r0 + r, j0 + j, p.Cout - j0 - j, v);
        }
    }
}

// ---- many results: tiles through LDS ------------------------------------------------------------------------------
// Rows and layers of the b-th tile: neighbouring workgroups of one XCD take a band of eight row tiles, row tile fastest,
// so that what one of its L2 holds is eight row tiles and a few layer tiles.
__device__ __forceinline__ void tile_at(int b, int tiles, int tiles_r, int tiles_j, int &tr, int &tj)
{
    const int q = tiles >> 3, rest = tiles & 7, xcd = b & 7;
    b = (xcd < rest ? xcd * (q + 1) : rest * (q + 1) + (xcd - rest) * q) + (b >> 3);
    const int band = b / (8 * tiles_j), in_band = b - band * 8 * tiles_j;
    const int high = min(8, tiles_r - band * 8);
    tj = in_band / high;
    tr = band * 8 + in_band - tj * high;
}

// A wavefront's 32 rows x 32*NJ layers (in order j-block, then the accumulator's registers), through its own part of
// LDS, out row by row.
template <typename TO, int NJ> __device__ __forceinline__ void write_rows(const LinearArgs &p, float *buf, const f32x16_t (&acc)[NJ], int r0, int j0, int lane)
{
    constexpr int kRow = 32 * NJ + 4, n = 16 / (int)sizeof(TO), kLanes = 32 * NJ / n, kPer = 64 / kLanes;
#pragma unroll
    for (int c = 0; c < NJ; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4_t v = {acc[c][4 * q], acc[c][4 * q + 1], acc[c][4 * q + 2], acc[c][4 * q + 3]};
            *(f32x4_t *)&buf[(lane & 31) * kRow + c * 32 + q * 8 + (lane >> 5) * 4] = v;
        }
    __builtin_amdgcn_wave_barrier();
    const int j = lane % kLanes * n;
    for (int i = lane / kLanes; i < 32; i += kPer) {
        float v[n];
#pragma unroll
        for (int e = 0; e < n; e += 4) *(f32x4_t *)&v[e] = *(const f32x4_t *)&buf[i * kRow + j + e];
        if (row_in(r0, i, p.rows)) finish<TO>(p, (long long)r0 + i, j0 + j, p.Cout - j0 - j, v);
    }
    __builtin_amdgcn_wave_barrier();
}

// bfloat16: BM rows x BN layers per workgroup of WR x WC wavefronts, v_mfma_f32_32x32x16_bf16 with the kernels as the
// first operand.  64 values of k per step; a row's 128 bytes lie as eight 16-byte pieces, piece q of row r at place
// q ^ (r & 7), so that the 32 rows a read takes at one k spread over all banks.  Two images of the step in LDS: the
// next one is loaded (memory to LDS directly) while this one is multiplied.
template <typename TO, int BM, int BN, int WR, int WC> __device__ __forceinline__ void linear_tile_bf16(const LinearArgs &p, int tiles_r, int tiles_j)
{
    constexpr int NW = WR * WC, XB = BM / WR / 32, JB = BN / WC / 32;
    constexpr int XI = BM / 8 / NW, JI = BN / 8 / NW;       // loads of 8 rows per wavefront
    __shared__ u32x4_t lds0[(BM + BN) * 8];
    __shared__ u32x4_t lds1[(BM + BN) * 8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tr, tj;
    tile_at(blockIdx.x, tiles_r * tiles_j, tiles_r, tiles_j, tr, tj);
    const int r0 = tr * BM, j0 = tj * BN;
    const int piece = (lane & 7) ^ (lane >> 3);
    // per load the lane's row and piece as a 32-bit offset from the tile's first row; k moves in the uniform offset
    const auto xr = __builtin_amdgcn_make_buffer_rsrc((void *)((const bf16_t *)p.in + r0 * p.ld_in), 0, 0xffffffffu, 0x00020000);
    const auto wr = __builtin_amdgcn_make_buffer_rsrc((void *)((const bf16_t *)p.w + (long long)j0 * p.Cin), 0, 0xffffffffu, 0x00020000);
    uint32_t xo[XI], wo[JI];
#pragma unroll
    for (int i = 0; i < XI; ++i) xo[i] = (uint32_t)(row_at(r0, (wave * XI + i) * 8 + (lane >> 3), p.rows) - r0) * (uint32_t)(2 * p.ld_in) + piece * 16;
#pragma unroll
    for (int i = 0; i < JI; ++i) wo[i] = (uint32_t)(row_at(j0, (wave * JI + i) * 8 + (lane >> 3), p.Cout) - j0) * (uint32_t)(2 * p.Cin) + piece * 16;
    auto fetch = [&](u32x4_t *to, int k) {
        u32x4_t *xto = to + wave * XI * 64, *wto = to + BM * 8 + wave * JI * 64;
#pragma unroll
        for (int i = 0; i < XI; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xr, (__attribute__((address_space(3))) void *)(xto + i * 64), 16, xo[i], 2 * k, 0, 0);
#pragma unroll
        for (int i = 0; i < JI; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (__attribute__((address_space(3))) void *)(wto + i * 64), 16, wo[i], 2 * k, 0, 0);
    };
    const int xrow = wave / WC * (XB * 32) + (lane & 31), wrow = BM + wave % WC * (JB * 32) + (lane & 31);
    f32x16_t acc[XB][JB] = {};
    auto multiply = [&](const u32x4_t *from) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int place = (2 * s + (lane >> 5)) ^ (lane & 7);
            bf16x8 x[XB], w[JB];
#pragma unroll
            for (int i = 0; i < JB; ++i) w[i] = __builtin_bit_cast(bf16x8, from[(wrow + 32 * i) * 8 + place]);
#pragma unroll
            for (int i = 0; i < XB; ++i) x[i] = __builtin_bit_cast(bf16x8, from[(xrow + 32 * i) * 8 + place]);
#pragma unroll
            for (int i = 0; i < XB; ++i)
#pragma unroll
                for (int c = 0; c < JB; ++c) acc[i][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[c], x[i], acc[i][c], 0, 0, 0);
        }
    };
    auto arrive = [&]() {
        __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    // the part of k behind the last whole step goes first, through registers, with zeros behind its end
    const int whole = p.Cin & ~63;
    if (whole < p.Cin) {
        const int have = p.Cin - whole - piece * 8;
        const bf16_t *x = (const bf16_t *)p.in + r0 * p.ld_in + whole, *w = (const bf16_t *)p.w + (long long)j0 * p.Cin + whole;
#pragma unroll 1
        for (int i = 0; i < XI; ++i) lds1[(wave * XI + i) * 64 + lane] = load16_tail((const bf16_t *)((const char *)x + xo[i]), have);
#pragma unroll 1
        for (int i = 0; i < JI; ++i) lds1[BM * 8 + (wave * JI + i) * 64 + lane] = load16_tail((const bf16_t *)((const char *)w + wo[i]), have);
    } else {
        fetch(lds0, 0);
    }
    for (int k = whole < p.Cin ? -128 : 0;; k += 128) {
        if (k >= 0) {
            arrive();
            if (k + 64 < whole) fetch(lds1, k + 64);
            multiply(lds0);
            if (k + 64 >= whole) break;
        }
        arrive();
        if (k + 128 < whole) fetch(lds0, k + 128);
        multiply(lds1);
        if (k + 128 >= whole) break;
    }
    __syncthreads();
    constexpr int kBuf = 32 * (32 * JB + 4);
    static_assert(kBuf * 4 * (NW / 2) <= (BM + BN) * 128, "the exchange areas of half of the wavefronts fit an image");
    float *buf = wave < NW / 2 ? (float *)lds0 + wave * kBuf : (float *)lds1 + (wave - NW / 2) * kBuf;
#pragma unroll
    for (int i = 0; i < XB; ++i)
        write_rows<TO, JB>(p, buf, acc[i], r0 + wave / WC * (XB * 32) + 32 * i, j0 + wave % WC * (JB * 32), lane);
}

template <typename TO, int BM, int BN, int WR, int WC>
__global__ __launch_bounds__(64 * WR *WC) void linear_tile_bf16_kernel(LinearArgs p, int tiles_r, int tiles_j)
{
    linear_tile_bf16<TO, BM, BN, WR, WC>(p, tiles_r, tiles_j);
}

// ---- which of them ------------------------------------------------------------------------------------------------
template <typename TI, typename TO, int RT, int CT, int MAXW> int launch_wave(const LinearArgs &p, int waves)
{
    const int tj = (p.Cout - 1) / CT + 1;
    const long long tiles = (long long)tj * ((p.rows - 1) / RT + 1);
    const LaunchScope prof("linear_wave", linear_flops(p), linear_bytes(p));
    hipLaunchKernelGGL((linear_wave_kernel<TI, TO, RT, CT, MAXW>), dim3((unsigned)std::min<long long>(tiles, 1 << 20)), dim3(64 * std::min(waves, MAXW)), 0,
                       current_stream(), p, tj, tiles);
    return check_launch();
}

template <typename TO, int BM, int BN, int WR, int WC> int launch_tile_bf16(const LinearArgs &p)
{
    const int tr = (p.rows - 1) / BM + 1, tj = (p.Cout - 1) / BN + 1;
    const LaunchScope prof("linear_tile", linear_flops(p), linear_bytes(p));
    hipLaunchKernelGGL((linear_tile_bf16_kernel<TO, BM, BN, WR, WC>), dim3((unsigned)(tr * tj)), dim3(64 * WR * WC), 0, current_stream(), p, tr, tj);
    return check_launch();
}

template <typename TI, typename TO> int by_size(const LinearArgs &p)
{
    if constexpr (sizeof(TI) == 2) {
        const bool direct = p.Cin % 8 == 0 && p.ld_in % 8 == 0 && ((uintptr_t)p.in & 15) == 0 && ((uintptr_t)p.w & 15) == 0 &&
                            p.ld_in < (1 << 22) && p.Cin < (1 << 22);      // a tile's rows within 32-bit offsets
        if (direct && linear_flops(p) > 4e9) {
            const long long big = (long long)((p.rows - 1) / 256 + 1) * ((p.Cout - 1) / 256 + 1);
            if (big >= 200) return launch_tile_bf16<TO, 256, 256, 2, 4>(p);
            return launch_tile_bf16<TO, 128, 128, 2, 2>(p);
        }
    }
    const int steps = (int)(p.Cin * sizeof(TI) / 64) + 1;
    if (p.rows <= 16) return launch_wave<TI, TO, 16, 16, 16>(p, std::max(1, steps));
    const long long t64 = (long long)((p.rows - 1) / 64 + 1) * ((p.Cout - 1) / 64 + 1);
    if (t64 >= 200) return launch_wave<TI, TO, 64, 64, 8>(p, std::max(1, steps / 4));
    return launch_wave<TI, TO, 32, 32, 8>(p, std::max(1, steps / 2));
}

}  // namespace

size_t linear_workspace_bytes(int, int, int, int) { return 0; }

int linear(const LinearArgs &p)
{
    if (p.in_dtype == SQ_F32) return by_size<float, float>(p);
    return p.out_dtype == SQ_F32 ? by_size<bf16_t, float>(p) : by_size<bf16_t, bf16_t>(p);
}

}  // namespace sq
