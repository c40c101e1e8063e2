// Matrix product of rows with bias, activation and residual: out[r][j] = act(sum_k in[r][k] w[j][k] + b[j]) + residual[r][j].
#include "nhwc_common.h"

#include <algorithm>
#include <cmath>

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

// A lane's place in a row.  ODD: bfloat16 rows that may begin between words; 16 bytes at such an address in lanes of sixteen rows take four
// times as long to load as at a whole word's, so the words that hold them are loaded, none beyond, and shifted (8 x 1111 x 2000 7.4 -> 5.8
// us; not in the tiles, whose eight lanes take 128 bytes of a row: 1000 x 1111 x 2000 18.9 -> 20.0).
template <typename TI, bool ODD> struct Row {
    struct Loaded {
        u32x4_t v;
        uint32_t behind[ODD ? 1 : 0];
    };
    const TI *p;
    uint32_t shift;
    __device__ __forceinline__ void set(const TI *at)
    {
        shift = ODD ? ((uint32_t)(uintptr_t)at & 2) * 8 : 0;
        p = ODD ? (const TI *)((uintptr_t)at & ~(uintptr_t)3) : at;
    }
    __device__ __forceinline__ Loaded load(int k) const
    {
        Loaded l;
        if constexpr (ODD) {
            const uint32_t *const words = (const uint32_t *)(p + k);
            __builtin_memcpy(&l.v, words, 16);
            l.behind[0] = words[shift ? 4 : 3];
        } else {
            l.v = load16(p + k);
        }
        return l;
    }
    __device__ __forceinline__ u32x4_t whole(const Loaded &l) const
    {
        if constexpr (ODD) {
            const uint32_t a = l.v[0], b = l.v[1], c = l.v[2], d = l.v[3];
            return u32x4_t{__builtin_amdgcn_alignbit(b, a, shift), __builtin_amdgcn_alignbit(c, b, shift), __builtin_amdgcn_alignbit(d, c, shift),
                           __builtin_amdgcn_alignbit(l.behind[0], d, shift)};
        } else {
            return l.v;
        }
    }
    __device__ __forceinline__ u32x4_t tail(int k, int have) const { return load16_tail(p + k + (ODD ? (int)(shift / 16) : 0), have); }
};

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

// The y-th workgroup of a tile takes the y-th share of k; with more than one, what it writes is its share's sums, each share
// its own [rows][ld_out] in the workspace, which linear_join_kernel adds up.
template <typename TI, typename TO> __device__ __forceinline__ void take_share(LinearArgs &p)
{
    const int first = blockIdx.y * p.share;
    p.in = (const TI *)p.in + first;
    p.w = (const TI *)p.w + first;
    p.out = (TO *)p.out + (long long)blockIdx.y * p.rows * p.ld_out;
    p.Cin = blockIdx.y + 1 < gridDim.y ? p.share : p.Cin - first;      // the last also what is left of k
}

// ---- few results: wavefronts that share out the sum ---------------------------------------------------------------
// A workgroup makes CT layers of RT rows; its wavefronts share out k in pieces of 64 bytes of a row ("steps"), each
// holding the whole RT x CT block of sums in registers, and add up through LDS, in order of wavefronts.  Operands go
// from memory straight into the lanes of v_mfma_f32_16x16x32_bf16 / _16x16x4_f32: lane l takes 16 bytes of row l % 16 at
// piece l / 16 of the step (fp32: value i of every lane's four is one instruction; both operands number k alike).
// Bound by reading the kernels, and for small ones by the latency of one round of loads: 8 rows by 4096 x 4096 bf16 kernels take
// 9.5 us (3.5 TB/s, launch included; fp32 15.9, 4.2 TB/s; one compute unit reads one block of 16 layers), one row by 512 x 1000
// fp32 4.2 us.  Loads of the next steps held before the products of these changed nothing (fp32 15.9 -> 16.1).
template <typename TI, typename TO, int RT, int CT, int MAXW, bool ODD>
__global__ __launch_bounds__(64 * MAXW) void linear_wave_kernel(LinearArgs p, int tiles_r, int tiles_j)
{
    constexpr int RB = RT / 16, CB = CT / 16, kStep = 64 / (int)sizeof(TI), kPiece = 16 / (int)sizeof(TI), kRow = CT + 4;
    constexpr int kMost = 16 / (RB + CB) ? 16 / (RB + CB) : 1;       // steps whose loads fly together
    __shared__ float red[MAXW * RT * kRow];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
    const int l16 = lane & 15, piece = lane >> 4;
    int tr, tj;
    tile_at(blockIdx.x, tiles_r * tiles_j, tiles_r, tiles_j, tr, tj);
    const int r0 = tr * RT, j0 = tj * CT;
    Row<TI, ODD> xr[RB], wr[CB];
#pragma unroll
    for (int i = 0; i < RB; ++i) xr[i].set((const TI *)p.in + row_at(r0, 16 * i + l16, p.rows) * p.ld_in + piece * kPiece);
#pragma unroll
    for (int i = 0; i < CB; ++i) wr[i].set((const TI *)p.w + row_at(j0, 16 * i + l16, p.Cout) * p.ld_w + piece * kPiece);
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
        typename Row<TI, ODD>::Loaded a[S][CB], b[S][RB];
#pragma unroll
        for (int s = 0; s < S; ++s) {
#pragma unroll
            for (int c = 0; c < CB; ++c) a[s][c] = wr[c].load(k + s * kStep);
#pragma unroll
            for (int r = 0; r < RB; ++r) b[s][r] = xr[r].load(k + s * kStep);
        }
#pragma unroll
        for (int s = 0; s < S; ++s) {
            u32x4_t w[CB], x[RB];
#pragma unroll
            for (int c = 0; c < CB; ++c) w[c] = wr[c].whole(a[s][c]);
#pragma unroll
            for (int r = 0; r < RB; ++r) x[r] = xr[r].whole(b[s][r]);
            multiply(w, x);
        }
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
        for (int c = 0; c < CB; ++c) a[c] = wr[c].tail(k, have);
#pragma unroll
        for (int r = 0; r < RB; ++r) b[r] = xr[r].tail(k, have);
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

// ---- many results: tiles through LDS ------------------------------------------------------------------------------
// The results of a wavefront, 32 * XB rows from r0 on and 32 * JB layers from j0 on, out through its own part of LDS, 32 rows at
// a time: the accumulators hold a row's layers spread over registers and lanes, LDS gives them back row by row, so that
// the residual is read and the result written in whole lines.  A lane's layers are the same in every row: its bias is loaded
// once, and the residual one block of 32 rows ahead.
template <typename TO, int XB, int JB> __device__ __forceinline__ void write_rows(const LinearArgs &p, float *buf, const f32x16_t (&acc)[XB][JB], int r0, int j0, int lane)
{
    constexpr int kRow = 32 * JB + 4, n = 16 / (int)sizeof(TO), kLanes = 32 * JB / n, kPer = 64 / kLanes, kTurns = 32 / kPer;
    const int j = lane % kLanes * n, row = lane / kLanes;
    auto stage = [&](int x) {
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int c = 0; c < JB; ++c)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4_t v = {acc[x][c][4 * q], acc[x][c][4 * q + 1], acc[x][c][4 * q + 2], acc[x][c][4 * q + 3]};
                *(f32x4_t *)&buf[(lane & 31) * kRow + c * 32 + q * 8 + (lane >> 5) * 4] = v;
            }
        __builtin_amdgcn_wave_barrier();
    };
    auto staged = [&](int t, float (&v)[n]) {
#pragma unroll
        for (int e = 0; e < n; e += 4) *(f32x4_t *)&v[e] = *(const f32x4_t *)&buf[(row + t * kPer) * kRow + j + e];
    };
    if (!row_in(r0, 32 * XB - 1, p.rows) || !row_in(j0, 32 * JB - 1, p.Cout)) {     // the edge of the output
#pragma unroll
        for (int x = 0; x < XB; ++x) {
            stage(x);
#pragma unroll 1
            for (int t = 0; t < kTurns; ++t) {
                float v[n];
                staged(t, v);
                const int i = 32 * x + row + t * kPer;
                if (row_in(r0, i, p.rows)) finish<TO>(p, (long long)r0 + i, j0 + j, p.Cout - j0 - j, v);
            }
        }
        return;
    }
    float bias[n];
#pragma unroll
    for (int e = 0; e < n; ++e) bias[e] = 0.f;
    if (p.b) {
        const Vec<float, n> b = load_n<n>(p.b + j0 + j);
#pragma unroll
        for (int e = 0; e < n; ++e) bias[e] = b.v[e];
    }
    const TO *res = (const TO *)p.residual + (r0 + row) * p.ld_res + j0 + j;
    TO *out = (TO *)p.out + (r0 + row) * p.ld_out + j0 + j;
    Vec<TO, n> ahead[kTurns];
    auto load = [&](int x) {
        if (p.residual)
#pragma unroll
            for (int t = 0; t < kTurns; ++t) ahead[t] = load_n<n>(res + (32 * x + t * kPer) * p.ld_res);
    };
    auto blocks = [&](auto act) {
        load(0);
#pragma unroll
        for (int x = 0; x < XB; ++x) {
            stage(x);
            float v[kTurns][n];
#pragma unroll
            for (int t = 0; t < kTurns; ++t) {
                staged(t, v[t]);
#pragma unroll
                for (int e = 0; e < n; ++e) v[t][e] = activate<decltype(act)::value>(v[t][e] + bias[e]);
                if (p.residual)
#pragma unroll
                    for (int e = 0; e < n; ++e) v[t][e] += to_f32(ahead[t].v[e]);
            }
            if (x + 1 < XB) load(x + 1);
#pragma unroll
            for (int t = 0; t < kTurns; ++t) {
                Vec<TO, n> o;
#pragma unroll
                for (int e = 0; e < n; ++e) o.v[e] = from_f32<TO>(v[t][e]);
                __builtin_memcpy(out + (32 * x + t * kPer) * p.ld_out, &o, sizeof(o));
            }
        }
    };
    switch (p.act) {
        case SQ_ACT_RELU: blocks(std::integral_constant<int, SQ_ACT_RELU>{}); break;
        case SQ_ACT_SILU: blocks(std::integral_constant<int, SQ_ACT_SILU>{}); break;
        case SQ_ACT_GELU: blocks(std::integral_constant<int, SQ_ACT_GELU>{}); break;
        default: blocks(std::integral_constant<int, SQ_ACT_NONE>{});
    }
}

// bfloat16: BM rows x BN layers per workgroup of WR x WC wavefronts, v_mfma_f32_32x32x16_bf16 with the kernels as the
// first operand.  64 values of k per step; a row's 128 bytes lie as eight 16-byte pieces, piece q of row r at place
// q ^ (r / 2 % 8), so that any 16 neighbouring rows a read takes at one k cover the 64 banks once (with q ^ (r % 8) half of the
// cycles of every read were conflicts).  NS images of a step in LDS, loaded from memory directly; up to NS steps are on
// their way or in use.
// Bound by the matrix unit, which a large product keeps busy two thirds of the cycles at the clock that its power leaves (1.8 GHz):
// 8192^3 in 796 us (1381 TFLOP/s); 16224 x 4096 x 4096 in 402 us (1354), with GELU and residual 463.  What is left is one
// barrier a step and the time it takes the wavefronts to come out of it.
// KS teams of WR x WC wavefronts share out k for results that are too few to fill the chip with tiles, where what bounds a
// tile is the latency of its steps: 128 x 4096 x 4096 19.8 -> 14.8 us, 729 x 1536 x 384 9.5 -> 7.7 (64 x 64 tiles, two teams).
// p.Cin / 64 has to be a multiple of KS.
template <typename TO, int BM, int BN, int WR, int WC, int NS, int KS>
__global__ __launch_bounds__(64 * WR *WC *KS, (BM + BN) * 128 * NS * KS <= 80 * 1024 ? 2 : 1) void linear_tile_bf16_kernel(LinearArgs p, int tiles_r, int tiles_j)
{
    constexpr int NW = WR * WC, XB = BM / WR / 32, JB = BN / WC / 32, kImage = (BM + BN) * 8;
    constexpr int XI = BM / 8 / NW, JI = BN / 8 / NW, NI = XI + JI;       // loads of 8 rows per wavefront
    __shared__ u32x4_t all[KS * NS * kImage];
    const int lane = threadIdx.x & 63, team = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * NW)), wave = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) % NW);
    u32x4_t *const lds = all + team * NS * kImage;
    int tr, tj;
    tile_at(blockIdx.x, tiles_r * tiles_j, tiles_r, tiles_j, tr, tj);
    take_share<bf16_t, TO>(p);
    const int r0 = tr * BM, j0 = tj * BN;
    // Loads 0 to XI - 1 of a wavefront are rows of the input, the others of the kernels; load i takes rows 8 g to 8 g + 7, the
    // lane's row is lane / 8 and its place lane % 8.  Per load the lane's row and piece are a 32-bit offset from the
    // tile's first row; k moves in the uniform offset.
    auto piece = [&](int i) { return (lane & 7) ^ (((wave * (i < XI ? XI : JI) + (i < XI ? i : i - XI)) & 1) * 4 + (lane >> 4)); };
    // the team's share of the whole steps, the same number for each
    const int whole = p.Cin / 64 / KS, tail = p.Cin % 64, k0 = 64 * whole * team;
    const bf16_t *const x0 = (const bf16_t *)p.in + r0 * p.ld_in + k0, *const w0 = (const bf16_t *)p.w + j0 * p.ld_w + k0;
    const u32x4_t xr = {(uint32_t)(uintptr_t)x0, (uint32_t)((uintptr_t)x0 >> 32), 0xffffffffu, 0x00020000u};
    const u32x4_t wr = {(uint32_t)(uintptr_t)w0, (uint32_t)((uintptr_t)w0 >> 32), 0xffffffffu, 0x00020000u};
    uint32_t off[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i)
        off[i] = i < XI ? (uint32_t)(row_at(r0, (wave * XI + i) * 8 + (lane >> 3), p.rows) - r0) * (uint32_t)(2 * p.ld_in) + piece(i) * 16
                        : (uint32_t)(row_at(j0, (wave * JI + i - XI) * 8 + (lane >> 3), p.Cout) - j0) * (uint32_t)(2 * p.ld_w) + piece(i) * 16;
    auto place_of = [&](int i) { return i < XI ? (wave * XI + i) * 64 : BM * 8 + (wave * JI + i - XI) * 64; };
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4_t *)all) + team * (uint32_t)(NS * kImage * 16);
    // Load i of the step at k into an image.  As an instruction of its own, because the compiler would let every later read of
    // LDS wait for it; `arrive` is what orders them.  m0 is set before each: nothing else in this kernel reads it (gfx950's
    // LDS instructions do not).
    auto fetch = [&](int img, int k, int i) {
        __asm__ volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds"
                         :: "v"(off[i]), "s"(i < XI ? xr : wr), "s"(2 * k), "s"(lds0 + 16 * (uint32_t)(img * kImage + place_of(i))));
    };
    const int xrow = wave / WC * (XB * 32) + (lane & 31), wrow = BM + wave % WC * (JB * 32) + (lane & 31);
    f32x16_t acc[XB][JB] = {};
    // Until all but the loads of the `younger` youngest steps have landed, and every wavefront is here: a wavefront waits for
    // its own loads and for its reads of LDS, the barrier for those of the others.
    auto arrive = [&](auto younger, bool all) {
        if (decltype(younger)::value > 0 && !all) __asm__ volatile("s_waitcnt vmcnt(%0)" :: "n"(decltype(younger)::value * NI) : "memory");
        else __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __asm__ volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    // Step s lies in image s % NS.  The part of k behind the last whole step goes first, through registers, with zeros behind
    // its end, as step -1 in the last image.
    if (tail) {         // by the last team; the others' share of it is zeros.  A piece is whole or behind the end (Cin is a multiple of 8).
        u32x4_t rest[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i)
            rest[i] = team == KS - 1 && piece(i) * 8 < tail ? load16((const bf16_t *)((const char *)((i < XI ? x0 : w0) + 64 * whole) + off[i])) : u32x4_t{};
#pragma unroll
        for (int i = 0; i < NI; ++i) lds[(NS - 1) * kImage + place_of(i) + lane] = rest[i];
    }
#pragma unroll
    for (int s = 0; s < NS; ++s)
        if (s < (tail ? min(whole, NS - 1) : whole)) {
#pragma unroll
            for (int i = 0; i < NI; ++i) fetch(s, 64 * s, i);
        }
    // Four parts of 16 k per step; the operands of a part are read while the part before is multiplied.  Before the last part,
    // whose operands are in registers by then, every wavefront is done with the image: it takes step s + NS, and the
    // first operands of step s + 1 are read under the last part's products.
    bf16x8 x[2][XB], w[2][JB];
    auto read = [&](const u32x4_t *from, int q) {
        const int place = (2 * q + (lane >> 5)) ^ ((lane >> 1) & 7);
#pragma unroll
        for (int i = 0; i < JB; ++i) w[q & 1][i] = __builtin_bit_cast(bf16x8, from[(wrow + 32 * i) * 8 + place]);
#pragma unroll
        for (int i = 0; i < XB; ++i) x[q & 1][i] = __builtin_bit_cast(bf16x8, from[(xrow + 32 * i) * 8 + place]);
    };
    // with half of the loads of a step spread over the products: issued at once they hold the wavefront up while the unit
    // that takes them works through 64 bytes a cycle
    auto multiply = [&](int q, bool load, int to, int k, int half) {
#pragma unroll
        for (int m = 0; m < XB * JB; ++m) {
            if (half >= 0) {
                if (load) {
#pragma unroll
                    for (int i = 0; i < NI / 2; ++i)
                        if (i * XB * JB / (NI / 2) == m) fetch(to, k, half * (NI / 2) + i);
                }
            }
            if (m == 0) __builtin_amdgcn_s_setprio(1);
            acc[m / JB][m % JB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[q & 1][m % JB], x[q & 1][m / JB], acc[m / JB][m % JB], 0, 0, 0);
            if (half >= 0) __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
    };
    int img = tail ? NS - 1 : 0;
    arrive(std::integral_constant<int, NS - 1>{}, tail || whole < NS);
    read(lds + img * kImage, 0);
    const int first = tail ? -1 : 0;
    for (int s = first; s < whole; ++s) {
        const u32x4_t *const from = lds + img * kImage;
        const int next = img == NS - 1 ? 0 : img + 1, last = img == 0 ? NS - 1 : img - 1;
        read(from, 1);
        multiply(0, s > first && s - 1 + NS < whole, last, 64 * (s - 1 + NS), 1);
        read(from, 2);
        multiply(1, false, 0, 0, -1);
        read(from, 3);
        multiply(2, false, 0, 0, -1);
        if (s + 1 < whole) {
            arrive(std::integral_constant<int, NS - 2>{}, s + NS > whole);
            read(lds + next * kImage, 0);
        }
        multiply(3, s + NS < whole, img, 64 * (s + NS), 0);
        img = next;
    }
    __syncthreads();
    if constexpr (KS > 1) {     // the first team adds the others' sums, in their order
        constexpr int kSums = XB * JB * 4 * 64;     // 16-byte pieces of a wavefront
        static_assert(kSums * NW <= NS * kImage, "a team's sums fit its images");
        if (team > 0) {
#pragma unroll
            for (int m = 0; m < XB * JB; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4_t v = {acc[m / JB][m % JB][4 * q], acc[m / JB][m % JB][4 * q + 1], acc[m / JB][m % JB][4 * q + 2], acc[m / JB][m % JB][4 * q + 3]};
                    ((f32x4_t *)lds)[wave * kSums + (m * 4 + q) * 64 + lane] = v;
                }
        }
        __syncthreads();
        if (team > 0) return;
#pragma unroll
        for (int t = 1; t < KS; ++t)
#pragma unroll
            for (int m = 0; m < XB * JB; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4_t v = ((const f32x4_t *)(all + t * NS * kImage))[wave * kSums + (m * 4 + q) * 64 + lane];
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[m / JB][m % JB][4 * q + e] += v[e];
                }
    }
    constexpr int kBuf = 32 * (32 * JB + 4);
    static_assert(kBuf * 4 * NW <= NS * kImage * 16, "the wavefronts' exchange areas fit the images");
    write_rows<TO, XB, JB>(p, (float *)all + wave * kBuf, acc, r0 + wave / WC * (XB * 32), j0 + wave % WC * (JB * 32), lane);
}

// The same tiles through registers: operands that memory-to-LDS loads cannot take (rows at any address, any number of
// layers) and fp32.  A step is 128 bytes of a row, PF of them on their way in registers, two images in LDS.  KS teams as above,
// of any number of steps (fp32: 729 x 1536 x 384 34 -> 24 us, 1024^3 25 -> 19; tiles of 32 rows where there are no more, 17 x 4000 x 4000
// in shares of k 23.4 -> 20.6; bf16 gained nothing, its unaligned loads are the
// bound).
//
// fp32 products run on the bf16 instructions: every operand is the sum of three bfloat16 values, x = h + m + l with h its
// upper half, m = round(x - h) and l = x - h - m, all three exact (24 bits in pieces of at most 8), and of the nine products the
// six down to 2^-16 of the largest are summed: m l, l m and l l are together below 2^-22 of the term, with the sign of
// chance, where each addition in fp32 loses up to 2^-24 of a whole sum.  Six instructions of 16 k cost 192 cycles of the
// matrix unit where fp32 ones take 512.  Every term keeps its own accuracy whatever lies beside it; only operands below
// 2^-110 lose bits (their l falls below what a bfloat16 can hold).
// An infinity has no such form (inf - inf).  It, a NaN, or sums that overflow leave a sum that is not finite; the tile is then
// made once more from the operands as they are, on the fp32 instructions, and those results that were not finite take its values.
// (Rounded upper parts would do for ordinary numbers, but a rounded operand can change its kind: the largest numbers
// become infinities and the smallest zeros, whose products with a zero or an infinity are NaN.)  With a NaN in every tile 1024^3 takes
// 43 us instead of 22, 10816 x 2048 x 2048 1200 instead of 454.
//
// Bound by the matrix unit and the vector instructions of the splitting beside it: 10816 x 2048 x 2048 fp32 with GELU and residual in
// 454 us (200 TFLOP/s; the fp32 instructions reach 154 in a large library product), 8192 x 4096 x 4096 in 1250 us (220); bf16 rows at
// any address 2001^3 in 33 us (486 TFLOP/s), 14301 x 1649 x 2808 in 224 us (590).
template <typename TI> struct Image;
template <> struct Image<bf16_t> {
    static constexpr int kStep = 64, kPlanes = 1;
    // 16-byte piece q of row r
    static __device__ __forceinline__ int at(int r, int q) { return r * 8 + (q ^ ((r >> 1) & 7)); }
};
template <> struct Image<float> {
    static constexpr int kStep = 32, kPlanes = 3;
    // 16-byte piece q of row r in one of the planes: two rows share 128 bytes
    static __device__ __forceinline__ int at(int r, int q) { return (r >> 1) * 8 + (((r & 1) * 4 + q) ^ ((r >> 2) & 3)); }
};

__device__ __forceinline__ uint32_t bf16_pair(float a, float b)
{
    uint32_t v;     // written out: the compiler would round `a` a second time where it is wanted as fp32 again
    __asm__("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(v) : "v"(a), "v"(b));
    return v;
}
__device__ __forceinline__ void split_pair(float a, float b, uint32_t &h, uint32_t &m, uint32_t &l)
{
    const uint32_t ua = __builtin_bit_cast(uint32_t, a), ub = __builtin_bit_cast(uint32_t, b);
    h = __builtin_amdgcn_perm(ub, ua, 0x07060302);
    a -= __builtin_bit_cast(float, ua & 0xffff0000u);
    b -= __builtin_bit_cast(float, ub & 0xffff0000u);
    m = bf16_pair(a, b);
    l = bf16_pair(a - __builtin_bit_cast(float, m << 16), b - __builtin_bit_cast(float, m & 0xffff0000u));
}

template <typename TI, typename TO, int BM, int BN, int WR, int WC, int PF, int KS>
__global__ __launch_bounds__(64 * WR *WC *KS) void linear_tile_kernel(LinearArgs p, int tiles_r, int tiles_j)
{
    using I = Image<TI>;
    constexpr int NW = WR * WC, XB = BM / WR / 32, JB = BN / WC / 32, kRows = BM + BN, kStep = I::kStep;
    constexpr int kPlane = kRows * 8 / (sizeof(TI) == 4 ? 2 : 1), kImage = kPlane * I::kPlanes;       // in 16-byte pieces
    constexpr int NP = kRows * 8 / (64 * NW), kPiece = 16 / (int)sizeof(TI), kSub = kStep / 16;
    static_assert(NP * 64 * NW == kRows * 8 && BM * 8 % (64 * NW) == 0, "whole pieces per thread");
    constexpr int kBuf = 32 * (32 * JB + 4);
    static_assert(kBuf * 4 * NW <= kImage * 32, "the wavefronts' exchange areas fit the images");
    __shared__ u32x4_t all[KS * 2 * kImage];
    const int lane = threadIdx.x & 63, team = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * NW)), wave = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) % NW);
    u32x4_t *const lds = all + team * 2 * kImage;
    int tr, tj;
    tile_at(blockIdx.x, tiles_r * tiles_j, tiles_r, tiles_j, tr, tj);
    take_share<TI, TO>(p);
    const int r0 = tr * BM, j0 = tj * BN;
    // KS teams share out the whole steps evenly; what is left of them and the part step are for the last team
    const int whole = p.Cin / kStep / KS, left = whole * KS * kStep, k0 = whole * kStep * team;
    // thread t of a team takes piece t % 8 of rows t / 8 + i * (threads / 8): BM rows of the input, then BN of the kernels
    const int q = threadIdx.x & 7, row = (threadIdx.x % (64 * NW)) >> 3;
    const TI *src[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int r = row + i * 8 * NW;
        src[i] = (i * 8 * NW < BM ? (const TI *)p.in + row_at(r0, r, p.rows) * p.ld_in : (const TI *)p.w + row_at(j0, r - BM, p.Cout) * p.ld_w) + q * kPiece + k0;
    }
    auto fetch = [&](u32x4_t (&to)[NP], int k) {
#pragma unroll
        for (int i = 0; i < NP; ++i) to[i] = load16(src[i] + k);
    };
    const int xrow = wave / WC * (XB * 32) + (lane & 31), wrow = BM + wave % WC * (JB * 32) + (lane & 31);
    f32x16_t acc[XB][JB];
    // the sums of all of k; plain: on the fp32 instructions, a row's 128 bytes in LDS as in a bfloat16 image
    auto sums = [&](auto plain) {
        constexpr bool kPlain = decltype(plain)::value;
        using Raw = Image<bf16_t>;
        static_assert(kRows * 8 <= kImage, "a step's operands fit an image as they are");
        auto store = [&](const u32x4_t (&from)[NP], u32x4_t *to) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int r = row + i * 8 * NW;
                if constexpr (sizeof(TI) == 2 || kPlain) {
                    to[Raw::at(r, q)] = from[i];
                } else {
                    const f32x4_t v = __builtin_bit_cast(f32x4_t, from[i]);
                    uint2 *at = (uint2 *)(to + I::at(r, q >> 1)) + (q & 1);
                    uint2 h, m, l;
                    split_pair(v[0], v[1], h.x, m.x, l.x);
                    split_pair(v[2], v[3], h.y, m.y, l.y);
                    at[0] = h;
                    at[2 * kPlane] = m;
                    at[4 * kPlane] = l;
                }
            }
        };
        auto multiply = [&](const u32x4_t *from) {
            if constexpr (kPlain) {
#pragma unroll 1
                for (int s = 0; s < 4; ++s) {       // a lane's 16 bytes of either operand are four instructions' values
                    f32x4_t x[XB], w[JB];
#pragma unroll
                    for (int i = 0; i < JB; ++i) w[i] = __builtin_bit_cast(f32x4_t, from[Raw::at(wrow + 32 * i, 2 * s + (lane >> 5))]);
#pragma unroll
                    for (int i = 0; i < XB; ++i) x[i] = __builtin_bit_cast(f32x4_t, from[Raw::at(xrow + 32 * i, 2 * s + (lane >> 5))]);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int i = 0; i < XB; ++i)
#pragma unroll
                            for (int c = 0; c < JB; ++c) acc[i][c] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[c][e], x[i][e], acc[i][c], 0, 0, 0);
                }
            } else {
                constexpr int NPL = I::kPlanes;
#pragma unroll
                for (int s = 0; s < kSub; ++s) {
                    bf16x8 x[NPL][XB], w[NPL][JB];
#pragma unroll
                    for (int n = 0; n < NPL; ++n) {
#pragma unroll
                        for (int i = 0; i < JB; ++i) w[n][i] = __builtin_bit_cast(bf16x8, from[n * kPlane + I::at(wrow + 32 * i, 2 * s + (lane >> 5))]);
#pragma unroll
                        for (int i = 0; i < XB; ++i) x[n][i] = __builtin_bit_cast(bf16x8, from[n * kPlane + I::at(xrow + 32 * i, 2 * s + (lane >> 5))]);
                    }
                    // the smallest products first
#pragma unroll
                    for (int n = NPL - 1; n >= 0; --n)
#pragma unroll
                        for (int a = 0; a <= n; ++a)
#pragma unroll
                            for (int i = 0; i < XB; ++i)
#pragma unroll
                                for (int c = 0; c < JB; ++c) acc[i][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[a][c], x[n - a][i], acc[i][c], 0, 0, 0);
                }
            }
        };
#pragma unroll
        for (int i = 0; i < XB; ++i)
#pragma unroll
            for (int c = 0; c < JB; ++c) acc[i][c] = f32x16_t{};
        // Image s % 2 holds step s, ring entry s % PF what is to become step s; loads behind the last step take it again.
        u32x4_t ring[PF][NP];
#pragma unroll
        for (int i = 0; i < PF; ++i)
            if (whole) fetch(ring[i], min(i, whole - 1) * kStep);
        __syncthreads();
#pragma unroll 1
        for (int k = left; k < p.Cin; k += kStep) {     // at most KS of them, first; zeros behind the end and for the other teams
            u32x4_t rest[NP];
            const int have = team == KS - 1 ? p.Cin - k - q * kPiece : 0;
#pragma unroll
            for (int i = 0; i < NP; ++i) rest[i] = load16_tail(src[i] + k - k0, have);
            store(rest, lds);
            __syncthreads();
            multiply(lds);
            __syncthreads();
        }
        if (whole) {
            auto step = [&](int s, u32x4_t (&next)[NP]) {
                store(next, lds + (s + 1) % 2 * kImage);
                fetch(next, min(s + 1 + PF, whole - 1) * kStep);
                multiply(lds + s % 2 * kImage);
                if constexpr (XB * JB > 1 && !kPlain) {     // larger tiles: the loads go out between the products, not before them (3 to 6 %)
                    constexpr int M = XB * JB * kSub * (sizeof(TI) == 2 ? 1 : 6);
                    __builtin_amdgcn_sched_group_barrier(0x008, M / 4, 0);
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x008, (M / 2 + NP - 1) / NP, 0);
                    }
                }
                __syncthreads();
            };
            store(ring[0], lds);
            fetch(ring[0], min(PF, whole - 1) * kStep);
            __syncthreads();
            int s = 0;
            for (; s + PF < whole; s += PF)
#pragma unroll
                for (int u = 0; u < PF; ++u) step(s + u, ring[(u + 1) % PF]);
#pragma unroll
            for (int u = 0; u < PF - 1; ++u)
                if (s + 1 < whole) step(s++, ring[(u + 1) % PF]);
            multiply(lds + s % 2 * kImage);
            __syncthreads();
        }
    };
    // the first team adds the others' sums to its own, in their order
    constexpr int kSums = XB * JB * 4 * 64;         // 16-byte pieces of a wavefront
    static_assert(KS == 1 || kSums * NW <= 2 * kImage, "a team's sums fit its images");
    auto add_up = [&]() {
        if constexpr (KS > 1) {
            if (team > 0) {
#pragma unroll
                for (int m = 0; m < XB * JB * 4; ++m) {
                    const f32x16_t &v = acc[m / 4 / JB][m / 4 % JB];
                    const f32x4_t part = {v[m % 4 * 4], v[m % 4 * 4 + 1], v[m % 4 * 4 + 2], v[m % 4 * 4 + 3]};
                    ((f32x4_t *)lds)[wave * kSums + m * 64 + lane] = part;
                }
            }
            __syncthreads();
            if (team == 0) {
#pragma unroll
                for (int t = 1; t < KS; ++t)
#pragma unroll
                    for (int m = 0; m < XB * JB * 4; ++m) {
                        const f32x4_t part = ((const f32x4_t *)(all + t * 2 * kImage))[wave * kSums + m * 64 + lane];
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[m / 4 / JB][m / 4 % JB][m % 4 * 4 + e] += part[e];
                    }
            }
            __syncthreads();
        }
    };
    sums(std::false_type{});
    add_up();
    if constexpr (sizeof(TI) == 4) {
        int odd = 0;
        if (team == 0) {
#pragma unroll
            for (int i = 0; i < XB; ++i)
#pragma unroll
                for (int c = 0; c < JB; ++c)
#pragma unroll
                    for (int e = 0; e < 16; ++e) odd |= !__builtin_isfinite(acc[i][c][e]);
        }
        if (__syncthreads_or(odd)) {
            f32x16_t fine[XB][JB];
#pragma unroll
            for (int i = 0; i < XB; ++i)
#pragma unroll
                for (int c = 0; c < JB; ++c) fine[i][c] = acc[i][c];
            sums(std::true_type{});
            add_up();
#pragma unroll
            for (int i = 0; i < XB; ++i)
#pragma unroll
                for (int c = 0; c < JB; ++c)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[i][c][e] = __builtin_isfinite(fine[i][c][e]) ? fine[i][c][e] : acc[i][c][e];
        }
    }
    if (team > 0) return;
    write_rows<TO, XB, JB>(p, (float *)all + wave * kBuf, acc, r0 + wave / WC * (XB * 32), j0 + wave % WC * (JB * 32), lane);
}

// ---- the shares' sums ----------------------------------------------------------------------------------------------
// A thread adds up four neighbouring results of a row, in order of the shares, and finishes them.  In LinearArgs `in` is the
// shares' sums in rows of ld_in, a multiple of four.  Bound by its launch.
constexpr int kMostShares = 16;
template <typename TO> __global__ __launch_bounds__(256) void linear_join_kernel(LinearArgs p)
{
    const unsigned quads = (unsigned)(p.Cout - 1) / 4 + 1, e = blockIdx.x * 256 + threadIdx.x, r = e / quads;
    if (r >= (unsigned)p.rows) return;
    const int j = (int)(e - r * quads) * 4;
    const float *at = (const float *)p.in + r * p.ld_in + j;
    const long long part = p.rows * p.ld_in;
    // every load before the first sum
    f32x4_t of[kMostShares];
#pragma unroll
    for (int i = 0; i < kMostShares; ++i)
        if (i < p.shares) of[i] = *(const f32x4_t *)(at + i * part);
    const bool full = j + 4 <= p.Cout;
    Vec<float, 4> b = {};
    Vec<TO, 4> res = {};
    if (full && p.b) b = load_n<4>(p.b + j);
    if (full && p.residual) res = load_n<4>((const TO *)p.residual + r * p.ld_res + j);
    f32x4_t s = of[0];
#pragma unroll
    for (int i = 1; i < kMostShares; ++i)
        if (i < p.shares) s += of[i];
    float v[4] = {s[0], s[1], s[2], s[3]};
    if (!full) return finish<TO>(p, r, j, p.Cout - j, v);
    Vec<TO, 4> o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float y = activate_by(v[i] + b.v[i], p.act);
        o.v[i] = from_f32<TO>(p.residual ? y + to_f32(res.v[i]) : y);
    }
    __builtin_memcpy((TO *)p.out + r * p.ld_out + j, &o, sizeof(o));
}

// ---- which of them ------------------------------------------------------------------------------------------------
template <typename TI, typename TO, int RT, int CT, int MAXW, bool ODD> int launch_wave(const LinearArgs &p, int waves)
{
    const int tr = (p.rows - 1) / RT + 1, tj = (p.Cout - 1) / CT + 1;
    if (!one_launch((double)tr * tj, 64 * waves)) return SQ_ERR_UNSUPPORTED;
    const LaunchScope prof("linear_wave", linear_flops(p), linear_bytes(p));
    hipLaunchKernelGGL((linear_wave_kernel<TI, TO, RT, CT, MAXW, ODD>), dim3((unsigned)tr * tj), dim3(64 * waves), 0, current_stream(), p, tr, tj);
    return check_launch();
}

template <typename TO, int BM, int BN, int WR, int WC, int NS, int KS = 1> int launch_tile_bf16(const LinearArgs &p)
{
    const int tr = (p.rows - 1) / BM + 1, tj = (p.Cout - 1) / BN + 1;
    if (!one_launch((double)tr * tj, 64 * WR * WC * KS)) return SQ_ERR_UNSUPPORTED;
    const LaunchScope prof("linear_tile_bf16", linear_flops(p), linear_bytes(p));
    hipLaunchKernelGGL((linear_tile_bf16_kernel<TO, BM, BN, WR, WC, NS, KS>), dim3((unsigned)tr * tj, p.shares), dim3(64 * WR * WC * KS), 0, current_stream(), p, tr, tj);
    return check_launch();
}

template <typename TI, typename TO, int BM, int BN, int WR, int WC, int PF, int KS = 1> int launch_tile(const LinearArgs &p)
{
    const int tr = (p.rows - 1) / BM + 1, tj = (p.Cout - 1) / BN + 1;
    if (!one_launch((double)tr * tj, 64 * WR * WC * KS)) return SQ_ERR_UNSUPPORTED;
    const LaunchScope prof("linear_tile", linear_flops(p), linear_bytes(p), (sizeof(TI) == 4 ? 6.0 : 1.0) * linear_flops(p));
    hipLaunchKernelGGL((linear_tile_kernel<TI, TO, BM, BN, WR, WC, PF, KS>), dim3((unsigned)tr * tj, p.shares), dim3(64 * WR * WC * KS), 0, current_stream(), p, tr, tj);
    return check_launch();
}

// Microseconds of a tiling, from what it measured (products of 128 to 8192 rows, layers and results): `fixed` for filling the
// pipeline and writing the results, `step` for 128 bytes of k when `slots` workgroups share the chip, `alone` when each
// has a compute unit to itself.  `threads` of a workgroup.
struct Tiling { int BM, BN, slots; double fixed, step, alone; int teams, threads; };
double tiling_us(const Tiling &t, const LinearArgs &p, int Cin, int shares)
{
    const long long tiles = (long long)((p.rows - 1) / t.BM + 1) * ((p.Cout - 1) / t.BN + 1) * shares;
    const int unit = p.in_dtype == SQ_F32 ? 32 : 64, whole = Cin / unit, steps = (Cin - 1) / unit + 1;
    // fp32: the steps that teams cannot share evenly and the part step come one at a time
    const int odd = p.in_dtype == SQ_F32 ? whole % t.teams + (Cin % unit != 0) : 0;
    // full rounds of the chip, and a last one with fewer to a compute unit
    auto round = [&](double step, double part) { return t.fixed + step * steps + part * odd; };
    const long long full = tiles / t.slots, rest = tiles % t.slots;
    const int each = (int)((rest + 255) / 256), most = t.slots / 256;
    return full * round(t.step, 1.0) + (rest ? round(most == 1 ? t.alone : t.alone + (t.step - t.alone) * (each - 1) / (most - 1), each == 1 ? 2.0 : 1.0) : 0.0);
}
const Tiling kF32[] = {{64, 64, 768, 3.0, 1.25, 0.6, 1, 256}, {128, 128, 256, 4.5, 1.36, 1.2, 1, 512}, {256, 128, 256, 8.5, 2.45, 2.1, 1, 512},
                       {64, 64, 256, 3.5, 0.55, 0.43, 2, 512}, {32, 128, 256, 3.5, 0.66, 0.54, 2, 512}};
const Tiling kDirect[] = {{64, 64, 512, 1.9, 0.4, 0.29, 1, 256},  {128, 128, 256, 2.5, 0.57, 0.5, 1, 512},  {128, 128, 512, 4.4, 1.0, 0.75, 1, 256},
                          {256, 256, 256, 9.0, 1.5, 1.25, 1, 512}, {64, 64, 256, 2.5, 0.22, 0.19, 2, 512}, {128, 64, 256, 3.5, 0.32, 0.3, 2, 512}};
const Tiling kAny[] = {{64, 64, 1024, 2.0, 1.45, 0.45, 1, 256}, {128, 128, 512, 4.0, 1.8, 0.85, 1, 512}};

// How a product is made: by wavefronts in blocks of 16 x 16 or 32 x 32, or by a tiling, with k in shares of `share` values.
enum { kWave16 = -1, kWave32 = -2 };
struct Plan { int which, share, shares; };
// Wavefronts of a workgroup that share out a sum of `steps` times 128 bytes.
int wave_count(int which, int steps) { return which == kWave16 ? std::min(2 * steps, 16) : std::min(steps, 8); }
double blocks_of(const LinearArgs &p, int rows, int layers) { return ((p.rows - 1) / rows + 1.0) * ((p.Cout - 1) / layers + 1.0); }

// Few results: the wavefronts, in blocks of 16 x 16 up to 2^16 results, a short sum or 16 rows, else 32 x 32 (us, 16 / 32: 586 x
// 1952 x 64 bf16 5.4 / 7.8, 99 x 3088 x 80 7.0 / 10.9; 45 x 1792 x 3520 12.9 / 9.5, 3458 x 2016 x 56 13.1 / 8.2).  Tiles through LDS
// from as many results on as they need to fill the chip: bf16 2^16 where two teams can share k (us, wavefronts / tiles: 32 x 4096 x
// 4096 19.0 / 13.6, 64 x 1024 x 1024 6.7 / 5.8; 300 x 2048 x 300 10.2 / 10.0), else 2^18 (461 x 64 x 2752 7.8 / 3.8; 1959 x 3224 x 72
// 11.9 / 17.8), 2^16 too where rows lie at any address (300 x 2049 x 300 27.7 / 16.1, 905 x 193 x 704 11.1 / 5.1; 129 x 2657 x 416
// 16.1 / 18.1), by estimate for fp32 (3506 x 416 x 1096 58 / 27, 1024^3 35 / 19, 729 x 1536 x 384 26.5 / 23.7; 300 x 2048 x 300 17.5 /
// 27.8, 64 x 4096 x 4096 34 / 52).
// Where one workgroup's way through k leaves the chip idle, tiles in shares of k and a second launch that adds them up (3.8 us and
// the sums' bytes), if that is to save 8 % (us, without / with: 300 x 4000 x 1000 fp32 50.5 / 26.6, 24 x 3691 x 3000 bf16 24.9 /
// 11.7, 17 x 4096 x 4096 14.2 / 10.2; 42 x 728 x 7032 fp32 14.4 / 14.5, 64 x 1280 x 3712 bf16 7.0 / 8.8, 40 x 2500 x 150 6.2 / 9.1).
// What has more threads than a launch takes is passed over; where nothing is left the launch refuses.
Plan plan_of(const LinearArgs &p, bool direct)
{
    const bool f32 = p.in_dtype == SQ_F32;
    const double results = (double)p.rows * p.Cout;
    const int unit = f32 ? 32 : 64, steps = (p.Cin - 1) / unit + 1;
    const bool teams = direct && p.Cin / 64 % 2 == 0 && p.Cin >= 256;       // two teams share k evenly
    const Tiling *const all = f32 ? kF32 : direct ? kDirect : kAny;
    const int n = f32 ? 5 : direct ? (teams ? 6 : 4) : 2;
    Plan best{0, p.Cin, 1};
    double us = HUGE_VAL;
    for (int i = 0; i < n; ++i) {
        if (!one_launch(blocks_of(p, all[i].BM, all[i].BN), all[i].threads)) continue;
        const double t = tiling_us(all[i], p, p.Cin, 1);
        if (t < us) us = t, best.which = i;
    }
    // the wavefronts: us for 1000 of k, of a block by itself and of a full chip's 256 (30 products); bf16 rows that begin
    // between words take more
    const bool small = p.rows <= 16 || results <= 65536 || steps <= 2;
    const int B = small ? 16 : 32, which = small ? kWave16 : kWave32;
    const double blocks = blocks_of(p, B, B);
    const bool far = ((double)p.rows + p.Cout) * p.Cin > 2e6;       // rows of blocks read kernels and input again: from beyond an XCD's cache
    const double one = small ? (f32 ? 2.0 : p.Cin % 2 == 0 ? 1.0 : 1.6) : (f32 ? 7.3 : 3.3);
    const double all256 = !small ? one : p.rows <= 16 ? (f32 ? 3.0 : 1.35 * one) : f32 ? (far ? 4.3 : 2.7) : 1.6 * one;
    const double waves = 4.0 + std::max(std::ceil(blocks / 256) * one, blocks / 256 * all256) * p.Cin * 1e-3;
    const double many = direct && !teams ? 1 << 18 : 1 << 16;
    if (one_launch(blocks, 64 * wave_count(which, steps)) && (p.rows <= 16 || results <= many || (f32 && (waves < us || (steps <= 2 && results < 1 << 20)))))
        us = waves, best.which = which;
    us *= 0.92;
    if (steps < 16 || us < 3.8 + 1.9) return best;
    for (int i = 0; i < n; ++i) {
        const Tiling &t = all[i];
        const double tiles = blocks_of(p, t.BM, t.BN);
        const int units = p.Cin / (unit * t.teams);
        for (int want = 2; want <= kMostShares && tiles * want <= 512; ++want) {
            const int share = ((units - 1) / want + 1) * unit * t.teams, shares = (units * unit * t.teams - 1) / share + 1;
            if (shares != want) continue;
            const double join = 3.8 + results * shares * 8.0 / 5e6, cost = tiling_us(t, p, std::max(share, p.Cin - (shares - 1) * share), shares) + join;
            if (cost < us) us = cost, best = Plan{i, share, shares};
        }
    }
    return best;
}

// Memory-to-LDS loads: whole 16-byte pieces, a tile's rows within 32-bit offsets.
bool direct_loads(int in_dtype, int Cin, long long ld_in, bool aligned)
{
    return in_dtype == SQ_BF16 && Cin % 8 == 0 && ld_in % 8 == 0 && aligned && ld_in < (1 << 22) && Cin < (1 << 22);
}
// Whether bfloat16 rows may begin between words.
bool between_words(const LinearArgs &p) { return p.in_dtype == SQ_BF16 && ((p.Cin | p.ld_in) % 2 || (((uintptr_t)p.in | (uintptr_t)p.w) & 3)); }
// Rows of the shares' sums begin at whole lines.
long long share_row(int Cout) { return ((long long)Cout + 31) / 32 * 32; }

template <typename TI, typename TO> int launch_tiling(const LinearArgs &p, int which, bool direct)
{
    if constexpr (sizeof(TI) == 4) {
        switch (which) {
            case 0: return launch_tile<TI, TO, 64, 64, 2, 2, 2>(p);
            case 1: return launch_tile<TI, TO, 128, 128, 2, 4, 1>(p);
            case 2: return launch_tile<TI, TO, 256, 128, 4, 2, 1>(p);
            case 3: return launch_tile<TI, TO, 64, 64, 2, 2, 2, 2>(p);
            default: return launch_tile<TI, TO, 32, 128, 1, 4, 2, 2>(p);
        }
    } else if (direct) {
        switch (which) {
            case 0: return launch_tile_bf16<TO, 64, 64, 2, 2, 4>(p);
            case 1: return launch_tile_bf16<TO, 128, 128, 2, 4, 4>(p);
            case 2: return launch_tile_bf16<TO, 128, 128, 2, 2, 2>(p);
            case 3: return launch_tile_bf16<TO, 256, 256, 2, 4, 2>(p);
            case 4: return launch_tile_bf16<TO, 64, 64, 2, 2, 4, 2>(p);
            default: return launch_tile_bf16<TO, 128, 64, 2, 2, 3, 2>(p);
        }
    } else {
        return which == 0 ? launch_tile<TI, TO, 64, 64, 2, 2, 2>(p) : launch_tile<TI, TO, 128, 128, 2, 4, 1>(p);
    }
}

template <typename TI, typename TO> int by_size(LinearArgs p)
{
    const bool direct = direct_loads(p.in_dtype, p.Cin, p.ld_in, (((uintptr_t)p.in | (uintptr_t)p.w) & 15) == 0);
    const Plan plan = plan_of(p, direct);
    p.ld_w = p.Cin;
    p.share = plan.share, p.shares = plan.shares;
    const int waves = wave_count(plan.which, (p.Cin - 1) / (128 / (int)sizeof(TI)) + 1);
    if (plan.which == kWave16) {
        if constexpr (sizeof(TI) == 2)
            if (between_words(p)) return launch_wave<TI, TO, 16, 16, 16, true>(p, waves);
        return launch_wave<TI, TO, 16, 16, 16, false>(p, waves);
    }
    if (plan.which == kWave32) return launch_wave<TI, TO, 32, 32, 8, false>(p, waves);
    if (plan.shares == 1) return launch_tiling<TI, TO>(p, plan.which, direct);
    LinearArgs part = p;
    part.b = nullptr, part.residual = nullptr, part.act = SQ_ACT_NONE;
    part.out = p.workspace, part.out_dtype = SQ_F32, part.ld_out = share_row(p.Cout);
    if (const int rc = launch_tiling<TI, float>(part, plan.which, direct)) return rc;
    p.in = p.workspace, p.ld_in = part.ld_out;
    const unsigned threads = (unsigned)p.rows * ((unsigned)(p.Cout - 1) / 4 + 1);       // at most 512 tiles' results
    const LaunchScope prof("linear_join", 0, 4.0 * plan.shares * p.rows * p.Cout + (sizeof(TO) * (p.residual ? 2.0 : 1.0)) * p.rows * p.Cout);
    hipLaunchKernelGGL((linear_join_kernel<TO>), dim3((threads - 1) / 256 + 1), dim3(256), 0, current_stream(), p);
    return check_launch();
}

}  // namespace

bool linear_register_kernels()
{
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, (const void *)linear_wave_kernel<float, float, 16, 16, 16, false>) == hipSuccess;
}

size_t linear_workspace_bytes(int rows, int Cin, int Cout, int in_dtype, long long ld_in, bool aligned)
{
    LinearArgs p{};
    p.rows = rows, p.Cin = Cin, p.Cout = Cout, p.in_dtype = in_dtype;
    const int shares = plan_of(p, direct_loads(in_dtype, Cin, ld_in, aligned)).shares;
    return shares == 1 ? 0 : (size_t)shares * rows * share_row(Cout) * sizeof(float);
}

int linear(const LinearArgs &p)
{
    if (p.in_dtype == SQ_F32) return by_size<float, float>(p);
    return p.out_dtype == SQ_F32 ? by_size<bf16_t, float>(p) : by_size<bf16_t, bf16_t>(p);
}

}  // namespace sq
