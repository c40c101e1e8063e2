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
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        Vec<uint32_t, 4> w;
        __builtin_memcpy(&w, v, sizeof(w));
        u16x2 m = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t magnitudes = w.v[i] & 0x7fff7fffu;
            m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, magnitudes));
        }
        return (uint32_t)max(m.x, m.y) << 16;
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
// Values k to k + 7 of a row of Cin values, zeros behind its end; whole: all are there.
template <typename TI> __device__ __forceinline__ Eight<TI> eight_at(const TI *row, int k, int Cin, bool whole)
{
    Eight<TI> e;
    if (whole || k <= Cin - 8) {         // (k + 8 may pass 32 bits)
        __builtin_memcpy(&e, row + k, sizeof(e));
    } else {
        Vec<TI, 8> v = {};
        if (k < Cin) v = load_some<8>(row + k, Cin - k);
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = k + i < Cin ? v.v[i] : TI(0);
    }
    return e;
}

// A workgroup packs one chunk of 32 rows: four lanes take a block, eight values each, a wavefront two rows at a time, four times over.  The
// scales go through LDS, so that their 256 bytes leave in one store.  Bound by memory: 16224 x 4096 bf16 in 29 us (168 MB, 5.9 TB/s).
template <typename TI> __global__ __launch_bounds__(256) void mx_pack_kernel(const TI *in, long long ld, int rows, int Cin, int chunks, uint32_t *scales, uint8_t *codes)
{
    __shared__ uint8_t sc[256];
    const int group = blockIdx.x / (unsigned)chunks, chunk = blockIdx.x - (unsigned)group * chunks;
    const int part = threadIdx.x & 31, k = chunk * 256 + part * 8;
    const unsigned first = (unsigned)group * 32 + (threadIdx.x >> 5);       // then every eighth row
    Eight<TI> e[4];
    auto load = [&](auto whole) {
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = eight_at(in + (long long)min(first + 8 * i, (unsigned)rows - 1) * ld, k, Cin, decltype(whole)::value);
    };
    if ((long long)chunk * 256 + 256 <= Cin) load(std::true_type{});
    else load(std::false_type{});
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

// A thread gives eight values back.  Bound by memory as well: packing 46656 x 384 fp32 values and giving them back takes 40 us (162 MB).
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
    if (part * 8 <= Cin - 8) {          // (the sum may pass 32 bits)
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
};

__device__ __forceinline__ i32x8_t wide(u32x4_t v)
{
    const i32x4_t a = __builtin_bit_cast(i32x4_t, v);
    return __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);       // 4-bit operands are four registers
}

// Few results: a workgroup makes 16 layers of 16 rows; its wavefronts share out the chunks, each holding the 16 x 16 sums, and add up through
// LDS, in order of wavefronts.  Operands go from memory straight into the lanes of v_mfma_scale_f32_16x16x128_f8f6f4: lane l takes
// block l / 16 of row l % 16, 16 bytes, and its scale.  TX: float or bf16_t, rows that are packed on the way: the 32 values of a block
// are a lane's own, so that it finds their largest and converts them without the others.
// Bound by the latency of a round of loads, and with rows packed on the way by the vector instructions for that: 8 rows by 4096 x 4096 packed
// 4.7 us, as they are 7.1; 1 row by 512 x 1000 fp32 3.6.
template <typename TX, typename TO, int MAXW> __global__ __launch_bounds__(64 * MAXW) void mx_wave_kernel(MxArgs a, int tiles_r, int tiles_j)
{
    constexpr bool kRaw = !std::is_same<TX, uint8_t>::value;
    constexpr int kRow = 20, kMost = kRaw ? 1 : 4;        // chunks whose loads fly together
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
        uint32_t sx[S][2], sw[S];
#pragma unroll
        for (int i = 0; i < S; ++i) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                w[i][t] = *(const u32x4_t *)(wc + (c + i) * 128ll + t * 64);
                if constexpr (!kRaw) x[i][t] = *(const u32x4_t *)(xc + (c + i) * 128ll + t * 64);
            }
            sw[i] = ws[(c + i) * 64ll] >> shift;
            if constexpr (!kRaw) sx[i][0] = xs[(c + i) * 64ll] >> shift, sx[i][1] = sx[i][0] >> 16;
        }
        if constexpr (kRaw) {
            Eight<TX> e[S][2][4];
            auto load = [&](auto whole) {
#pragma unroll
                for (int i = 0; i < S; ++i)
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int n = 0; n < 4; ++n) e[i][t][n] = eight_at((const TX *)a.p.in + r * a.p.ld_in, (c + i) * 256 + t * 128 + q * 32 + n * 8, a.p.Cin, decltype(whole)::value);
            };
            if ((c + S) * 256ll <= a.p.Cin) load(std::true_type{});
            else load(std::false_type{});
#pragma unroll
            for (int i = 0; i < S; ++i)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    uint32_t most = 0;
#pragma unroll
                    for (int n = 0; n < 4; ++n) most = max(most, e[i][t][n].most());
                    const uint32_t code = scale_code(most);
                    sx[i][t] = code;
#pragma unroll
                    for (int n = 0; n < 4; ++n) x[i][t][n] = e[i][t][n].codes(scale_value(code));      // (a NaN scale makes NaN of any code)
                }
        }
#pragma unroll
        for (int i = 0; i < S; ++i) {
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w[i][0]), wide(x[i][0]), acc, 4, 4, 0, (int)sw[i], 0, (int)sx[i][0]);
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w[i][1]), wide(x[i][1]), acc, 4, 4, 2, (int)sw[i], 0, (int)sx[i][1]);
        }
    };
    int at = (int)((long long)a.chunks * wave / nw);
    const int end = (int)((long long)a.chunks * (wave + 1) / nw);
    for (; at + kMost <= end; at += kMost) chunks(std::integral_constant<int, kMost>{}, at);
    if constexpr (kMost > 1)
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

// Many results: BM rows x BN layers per workgroup of WR x WC wavefronts, v_mfma_scale_f32_32x32x64_f8f6f4 with the kernels as the first
// operand.  A step is a chunk of both operands: 128 bytes of codes a row, which lie in LDS as eight 16-byte pieces, piece q of row r at
// place q ^ (r / 2 % 8) (any 16 neighbouring rows read at one k cover the banks once), and behind them 256 bytes of scales for each 32
// rows as they are in memory.  NS images of a step in LDS, loaded from memory directly.
// Bound by LDS and the matrix unit together (by count 2077 and 2048 cycles a step of the 256 x 256 tile; a step takes 1.5 us): 8192^3 in 249 us
// (4410 TFLOP/s), 16224 x 4096 x 4096 in 141 to 155, with GELU and residual 185 to 198.  Four wavefronts of 128 x 128 results read a third
// less and were no faster.
template <typename TO, int BM, int BN, int WR, int WC, int NS>
__global__ __launch_bounds__(64 * WR *WC, (BM + BN) * 136 * NS <= 80 * 1024 ? 2 : 1) void mx_tile_kernel(MxArgs a, int tiles_r, int tiles_j)
{
    constexpr int NW = WR * WC, XB = BM / WR / 32, JB = BN / WC / 32, kGroups = (BM + BN) / 32, kScales = (BM + BN) * 8, kImage = kScales + kGroups * 16;
    constexpr int XI = BM / 8 / NW, JI = BN / 8 / NW, NI = XI + JI, SI = (kGroups + NW - 1) / NW, NL = NI + SI;     // loads of a wavefront: of 8 rows, of scales
    __shared__ u32x4_t lds[NS * kImage];
    const LinearArgs &p = a.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tr, tj;
    tile_at(blockIdx.x, tiles_r * tiles_j, tiles_r, tiles_j, tr, tj);
    const int r0 = tr * BM, j0 = tj * BN;
    const int steps = a.chunks;
    const uint32_t row_bytes = (uint32_t)a.chunks * 128;
    const uint8_t *const x0 = a.x.codes + (long long)r0 * row_bytes, *const w0 = a.w.codes + (long long)j0 * row_bytes;
    const uint32_t *const xs0 = a.x.scales + (long long)(r0 >> 5) * a.chunks * 64, *const ws0 = a.w.scales + (long long)(j0 >> 5) * a.chunks * 64;
    // A buffer's third word is its size: 0 for the steps behind the last one, whose loads then fetch nothing but are waited for like the
    // others, so that the loop has no branches.
    auto resource = [](const void *at, uint32_t size) {
        return u32x4_t{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)at),
                       (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)((uintptr_t)at >> 32)), size, 0x00020000u};
    };
    // Loads 0 to XI - 1 are rows of the input, up to NI of the kernels, the rest scales; a load of rows takes rows 8 g to 8 g + 7, the lane's row
    // is lane / 8 and its place lane % 8.
    uint32_t off[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int g = i < XI ? wave * XI + i : wave * JI + i - XI, row = g * 8 + (lane >> 3), piece = (lane & 7) ^ ((g & 1) * 4 + (lane >> 4));
        off[i] = (uint32_t)(i < XI ? row_at(r0, row, p.rows) - r0 : row_at(j0, row, p.Cout) - j0) * row_bytes + piece * 16;
    }
    const int groups_x = groups_of(p.rows) - (r0 >> 5), groups_w = groups_of(p.Cout) - (j0 >> 5);
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4_t *)lds);
    // Load i of step s into an image.  As instructions of their own, because the compiler would let every later read of LDS wait for
    // them; `arrive` is what orders them.  m0 is set before each: nothing else in this kernel reads it.
    const uint32_t *scale_at[SI];
    uint32_t scale_place[SI];
#pragma unroll
    for (int i = 0; i < SI; ++i) {
        const int g = min(wave * SI + i, kGroups - 1);          // the last group more than once where they do not come out even
        // rows behind the last group take its scales
        const int at = g < BM / 32 ? min(g, groups_x - 1) : min(g - BM / 32, groups_w - 1);
        scale_at[i] = (g < BM / 32 ? xs0 : ws0) + (long long)at * a.chunks * 64;
        scale_place[i] = kScales + g * 16;
    }
    const uint32_t lane4 = lane * 4;
    auto fetch = [&](int img, int s, int i) {
        const uint32_t size = __builtin_amdgcn_readfirstlane(s < steps ? 0xffffffffu : 0u);
        if (i < NI) {
            const int place = i < XI ? (wave * XI + i) * 64 : BM * 8 + (wave * JI + i - XI) * 64;
            __asm__ volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds"
                             :: "v"(off[i]), "s"(resource(i < XI ? x0 : w0, size)), "s"(s * 128), "s"(lds0 + 16 * (uint32_t)(img * kImage + place)));
        } else {
            __asm__ volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dword %0, %1, %2 offen lds"
                             :: "v"(lane4), "s"(resource(scale_at[i - NI], size)), "s"(s * 256), "s"(lds0 + 16 * (uint32_t)(img * kImage + scale_place[i - NI])));
        }
    };
    const int xrow = wave / WC * (XB * 32) + (lane & 31), wrow = BM + wave % WC * (JB * 32) + (lane & 31);
    f32x16_t acc[XB][JB] = {};
    // Until all but the youngest `younger` loads have landed, and every wavefront is here.
    auto arrive = [&](auto younger) {
        __asm__ volatile("s_waitcnt vmcnt(%0)" :: "n"(decltype(younger)::value) : "memory");
        __asm__ volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    constexpr int kHalf = NL / 2;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < (s < NS - 1 ? NL : kHalf); ++i) fetch(s, s, i);
    // Four parts of 64 k per step; the operands of a part are read while the part before is multiplied.  Before the last part, whose operands
    // are in registers by then, every wavefront is done with the image: it takes step s + NS, and the first operands and the scales
    // of step s + 1 are read under the last part's products.
    u32x4_t x[2][XB], w[2][JB];
    int sx[2][XB], sw[2][JB];
    auto read = [&](const u32x4_t *from, int q) {
        const int place = (2 * q + (lane >> 5)) ^ ((lane >> 1) & 7);
#pragma unroll
        for (int i = 0; i < JB; ++i) w[q & 1][i] = from[(wrow + 32 * i) * 8 + place];
#pragma unroll
        for (int i = 0; i < XB; ++i) x[q & 1][i] = from[(xrow + 32 * i) * 8 + place];
    };
    auto read_scales = [&](const u32x4_t *from) {
        const int *const at = (const int *)(from + kScales) + lane;
#pragma unroll
        for (int i = 0; i < JB; ++i) sw[1][i] = at[(BM / 32 + wave % WC * JB + i) * 64];
#pragma unroll
        for (int i = 0; i < XB; ++i) sx[1][i] = at[(wave / WC * XB + i) * 64];
    };
    // with `count` loads of step s spread over the products
    auto multiply = [&](auto part, int to, int s, int first, int count) {
        constexpr int q = decltype(part)::value;
#pragma unroll
        for (int m = 0; m < XB * JB; ++m) {
#pragma unroll
            for (int i = 0; i < count; ++i)
                if (i * XB * JB / count == m) fetch(to, s, first + i);
            if (m == 0) __builtin_amdgcn_s_setprio(1);
            acc[m / JB][m % JB] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(w[q & 1][m % JB]), wide(x[q & 1][m / JB]), acc[m / JB][m % JB], 4, 4, q, sw[0][m % JB], q,
                                                                                sx[0][m / JB]);
            if (count) __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
    };
    using std::integral_constant;
    int img = 0;
    arrive(integral_constant<int, (NS - 2) * NL + kHalf>{});
    read(lds, 0);
    read_scales(lds);
#pragma unroll 1
    for (int s = 0; s < steps; ++s) {
        const u32x4_t *const from = lds + img * kImage;
        const int next = img == NS - 1 ? 0 : img + 1, last = img == 0 ? NS - 1 : img - 1;
#pragma unroll
        for (int i = 0; i < JB; ++i) sw[0][i] = sw[1][i];
#pragma unroll
        for (int i = 0; i < XB; ++i) sx[0][i] = sx[1][i];
        read(from, 1);
        multiply(integral_constant<int, 0>{}, last, s - 1 + NS, kHalf, NL - kHalf);
        read(from, 2);
        multiply(integral_constant<int, 1>{}, 0, 0, 0, 0);
        read(from, 3);
        multiply(integral_constant<int, 2>{}, 0, 0, 0, 0);
        arrive(integral_constant<int, (NS - 2) * NL>{});
        read(lds + next * kImage, 0);
        read_scales(lds + next * kImage);
        multiply(integral_constant<int, 3>{}, img, s + NS, 0, kHalf);
        img = next;
    }
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");        // loads that fetch nothing write LDS all the same
    __syncthreads();
    constexpr int kBuf = 32 * (32 * JB + 4);
    static_assert(kBuf * 4 * NW <= NS * kImage * 16, "the wavefronts' exchange areas fit the images");
    write_rows<TO, XB, JB>(p, (float *)lds + wave * kBuf, acc, r0 + wave / WC * (XB * 32), j0 + wave % WC * (JB * 32), lane);
}

// Bytes that a product cannot do without: its packed operands (or the rows as they are), results and residual.
double mx_bytes(const MxArgs &a)
{
    const double so = a.p.out_dtype == SQ_F32 ? 4.0 : 2.0, rows = a.x.codes ? (double)mxfp4_packed_bytes(a.p.rows, a.p.Cin) : (a.p.in_dtype == SQ_F32 ? 4.0 : 2.0) * a.p.rows * a.p.Cin;
    return rows + (double)mxfp4_packed_bytes(a.p.Cout, a.p.Cin) + so * a.p.rows * a.p.Cout * (a.p.residual ? 2 : 1) + 4.0 * a.p.Cout;
}
template <typename TX, typename TO> int launch_wave(const MxArgs &a)
{
    const int tr = (a.p.rows - 1) / 16 + 1, tj = (a.p.Cout - 1) / 16 + 1, waves = std::min(a.chunks, 16);
    if (!one_launch((double)tr * tj, 64 * waves)) return SQ_ERR_UNSUPPORTED;
    const LaunchScope prof("mx_wave", linear_flops(a.p), mx_bytes(a));
    hipLaunchKernelGGL((mx_wave_kernel<TX, TO, 16>), dim3((unsigned)tr * tj), dim3(64 * waves), 0, current_stream(), a, tr, tj);
    return check_launch();
}

template <typename TO, int BM, int BN, int WR, int WC, int NS> int launch_tile(const MxArgs &a)
{
    const int tr = (a.p.rows - 1) / BM + 1, tj = (a.p.Cout - 1) / BN + 1;
    if (!one_launch((double)tr * tj, 64 * WR * WC)) return SQ_ERR_UNSUPPORTED;
    const LaunchScope prof("mx_tile", linear_flops(a.p), mx_bytes(a));
    hipLaunchKernelGGL((mx_tile_kernel<TO, BM, BN, WR, WC, NS>), dim3((unsigned)tr * tj), dim3(64 * WR * WC), 0, current_stream(), a, tr, tj);
    return check_launch();
}

// Microseconds of a tiling: `fixed` for filling the pipeline and writing the results, `step` for a chunk of k when `slots` workgroups share
// the chip, `alone` when each has a compute unit to itself; from what it measured on products of 40 to 16224 rows.
struct Tiling { int BM, BN, slots; double fixed, step, alone; int threads; };
const Tiling kTilings[] = {{64, 64, 512, 1.2, 0.44, 0.31, 256}, {128, 64, 512, 1.9, 0.7, 0.35, 256}, {128, 128, 512, 2.6, 1.1, 0.44, 256}, {256, 256, 256, 4.0, 1.8, 1.1, 512}};
double tiling_us(const Tiling &t, int rows, int Cout, int chunks)
{
    const long long tiles = (long long)((rows - 1) / t.BM + 1) * ((Cout - 1) / t.BN + 1), full = tiles / t.slots, rest = tiles % t.slots;
    return full * (t.fixed + t.step * chunks) + (rest ? t.fixed + (rest > 256 ? t.step : t.alone) * chunks : 0.0);
}
double blocks_of(int rows, int Cout, int R, int C) { return ((rows - 1) / R + 1.0) * ((Cout - 1) / C + 1.0); }

// How a product is made: by wavefronts in blocks of 16 x 16 (rows not packed before as they are, where they are few), or by a tiling.
// Rows given as they are: packing them in every block of 16 layers again costs 0.17 us for 256 blocks and chunk, a launch that packs them
// first 2.3 us on the GPU and 5 on the host, counted as 4 (us, in the product / before it: 1 x 512 x 1000 fp32 3.6 / 5.4, 8 x 4096 x 4096
// bf16 7.2 / 7.4); up to 16 chunks a block, so that no block packs for longer than that launch takes.  Packed rows take the same form, so that they give the same bits.
// What has more threads than a launch takes, or rows too long for the tiles' 32-bit offsets, is passed over.
enum { kWaves = -1, kNone = -2 };
constexpr double kRawChunks = 16, kPackFirst = 4.0;
struct Plan { int which; bool raw; };
Plan plan_of(int rows, int Cin, int Cout)
{
    const int chunks = chunks_of(Cin);
    Plan plan{kNone, false};
    double us = HUGE_VAL;
    const double blocks = blocks_of(rows, Cout, 16, 16);
    if (one_launch(blocks, 64 * std::min(chunks, 16))) {
        const double some = chunks * std::max(1.0, blocks / 256);
        plan.which = kWaves, plan.raw = some <= kRawChunks;
        us = std::max(0.5, 0.22 * some) + 0.3 + (plan.raw ? 0.17 * some : kPackFirst);
    }
    if (rows <= 16 || chunks >= 1 << 15) return plan;
    for (int i = 0; i < 4; ++i) {
        const Tiling &t = kTilings[i];
        if (!one_launch(blocks_of(rows, Cout, t.BM, t.BN), t.threads)) continue;
        const double tu = tiling_us(t, rows, Cout, chunks) + kPackFirst;
        if (tu < us) us = tu, plan = Plan{i, false};
    }
    return plan;
}
template <typename TO> int by_size(const MxArgs &a, int which)
{
    switch (which) {
        case kWaves: return launch_wave<uint8_t, TO>(a);
        case 0: return launch_tile<TO, 64, 64, 2, 2, 4>(a);
        case 1: return launch_tile<TO, 128, 64, 2, 2, 3>(a);
        case 2: return launch_tile<TO, 128, 128, 2, 2, 2>(a);
        default: return launch_tile<TO, 256, 256, 2, 4, 2>(a);
    }
}
template <typename TX> int raw_rows(const MxArgs &a) { return a.p.out_dtype == SQ_F32 ? launch_wave<TX, float>(a) : launch_wave<TX, bf16_t>(a); }

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

static size_t need_of(const Plan &plan, int rows, int Cin, int in_dtype) { return in_dtype == SQ_MXFP4 || plan.raw ? 0 : mxfp4_packed_bytes(rows, Cin); }

size_t mxfp4_linear_workspace_bytes(int rows, int Cin, int Cout, int in_dtype)
{
    return need_of(plan_of(rows, Cin, Cout), rows, Cin, in_dtype);
}

int mxfp4_linear(const LinearArgs &p, size_t workspace_bytes)
{
    MxArgs a{};
    a.p = p;
    a.chunks = chunks_of(p.Cin);
    a.w = packed_at(p.w, p.Cout, p.Cin);
    const Plan plan = plan_of(p.rows, p.Cin, p.Cout);
    if (!enough_workspace(need_of(plan, p.rows, p.Cin, p.in_dtype), p.workspace, workspace_bytes)) return SQ_ERR_WORKSPACE;
    if (plan.which == kNone) return SQ_ERR_UNSUPPORTED;
    if (plan.raw && p.in_dtype != SQ_MXFP4) return p.in_dtype == SQ_F32 ? raw_rows<float>(a) : raw_rows<bf16_t>(a);
    const void *x = p.in;
    if (p.in_dtype != SQ_MXFP4) {
        if (const int rc = mxfp4_pack(p.in, p.in_dtype, p.workspace, p.rows, p.Cin, p.ld_in)) return rc;
        x = p.workspace;
    }
    a.x = packed_at(x, p.rows, p.Cin);
    return p.out_dtype == SQ_F32 ? by_size<float>(a, plan.which) : by_size<bf16_t>(a, plan.which);
}

extern "C" int sq_tune_mxfp4_linear_plan(int rows, int Cin, int Cout, int *plan)
{
    if (!plan || rows <= 0 || Cin <= 0 || Cout <= 0) return SQ_ERR_SHAPE;
    const Plan of = plan_of(rows, Cin, Cout);
    if (of.which == kNone) return SQ_ERR_UNSUPPORTED;
    plan[0] = of.which < 0 ? 16 : kTilings[of.which].BM, plan[1] = of.which < 0 ? 16 : kTilings[of.which].BN, plan[2] = of.raw;
    return SQ_OK;
}

bool mxfp4_register_kernels()
{
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, (const void *)mx_pack_kernel<float>) == hipSuccess;
}

}  // namespace sq
