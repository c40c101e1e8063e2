// Attention of the rows of one map (queries) to the rows of another (an encoder's states):
//   out[n][i][h] = sum_j p_j v[n][j][h'] / sum_j p_j,  p_j = exp(scale q[n][i][h] . k[n][j][h'])  over the states j that the query sees,
// h' = the head of the states that head h shares with its neighbours.  Zeros where a query sees none.
#include "linear_common.h"

#include <algorithm>
#include <cmath>

namespace sq {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896341f;

// What a row's exponents were taken against, in base two, and their sum.
struct PartSum {
    double base;
    float total;
};

// The heads of the queries that share a head of the states are further rows to it: row r is query r / group, head r % group of them.
struct CrossParams {
    CrossArgs a;
    int group, rows;        // rows of an image and head of the states
    int tiles;              // of rows
    int share, shares;      // of the states: one workgroup's, and how many
    float c;                // |scale| log2 e, or 1 where the scale is 0
    uint32_t keep, flip;    // bits of q that stay (none where the scale is 0), sign bits that turn q into -q where it is below 0
    float *part_o;          // [share][image, head, row][part_ld] and
    PartSum *part_ml;       // [share][image, head, row], where shares > 1
    int part_ld;
};

// 16 bytes of a head's D values from value d on; behind the last its last ones again, as rows behind the last state are the last one again:
// what multiplies them are zeros of the query or of the exponentials, and what they give is not written (they are finite wherever the
// state itself is).  EVEN: heads of whole pieces.  The others are loaded from where all 16 bytes are the head's own and moved into place
// by `placed`, so that no load waits for another, and heads of less than 16 bytes one value at a time.  bfloat16 values may begin between
// words: the words that hold them are loaded, none beyond (16 bytes at such an address take four times as long), and `placed` shifts them too.
template <bool EVEN, typename T> struct Piece {
    u32x4_t v;
};
template <> struct Piece<false, bf16_t> {
    u32x4_t v;
    uint32_t behind;        // the word behind, where the values begin between words
};
template <typename T> __device__ __forceinline__ uint32_t between_words(const T *p) { return (uint32_t)(uintptr_t)p >> 1 & 1; }
template <bool EVEN, typename T> __device__ __forceinline__ Piece<EVEN, T> loaded(const T *head, int d, int D)
{
    constexpr int n = 16 / (int)sizeof(T);
    Piece<EVEN, T> r;
    if constexpr (!EVEN && sizeof(T) == 2) {
        r.behind = 0;
        if (D >= n) {
            const T *const at = head + min(d, D - n);
            const bool between = (uintptr_t)at & 2;
            const uint32_t *const words = (const uint32_t *)((uintptr_t)at & ~(uintptr_t)3);
            __builtin_memcpy(&r.v, words, 16);
            r.behind = words[between ? 4 : 3];
            return r;
        }
    }
    r.v = EVEN || D >= n ? __builtin_bit_cast(u32x4_t, load_n<n>(head + min(d, D - n))) : __builtin_bit_cast(u32x4_t, load_some<n>(head, D));
    return r;
}
// With zeros behind the last value.  odd: whether the head begins between words.
template <bool EVEN, typename T> __device__ __forceinline__ u32x4_t placed(const Piece<EVEN, T> &piece, int d, int D, bool odd)
{
    constexpr int n = 16 / (int)sizeof(T);
    u32x4_t v = piece.v;
    if (EVEN) {
        if (d >= D) v = u32x4_t{};
        return v;
    }
    if constexpr (!EVEN && sizeof(T) == 2) {
        const uint32_t shift = D >= n && (odd ^ (min(d, D - n) & 1)) ? 16 : 0;
        v = u32x4_t{__builtin_amdgcn_alignbit(v[1], v[0], shift), __builtin_amdgcn_alignbit(v[2], v[1], shift), __builtin_amdgcn_alignbit(v[3], v[2], shift),
                    __builtin_amdgcn_alignbit(piece.behind, v[3], shift)};
    }
    if (D < n) {
        Vec<T, n> r = __builtin_bit_cast(Vec<T, n>, v);
#pragma unroll
        for (int i = 0; i < n; ++i) r.v[i] = d + i < D ? r.v[i] : T(0);
        return __builtin_bit_cast(u32x4_t, r);
    }
    const int away = max(d - (D - n), 0) * (int)sizeof(T);      // bytes
    if (away >= 16) v = u32x4_t{};
    if (away & 8) v = u32x4_t{v[2], v[3], 0, 0};
    if (away & 4) v = u32x4_t{v[1], v[2], v[3], 0};
    if (sizeof(T) == 2 && (away & 2))
        v = u32x4_t{__builtin_amdgcn_alignbit(v[1], v[0], 16), __builtin_amdgcn_alignbit(v[2], v[1], 16), __builtin_amdgcn_alignbit(v[3], v[2], 16), v[3] >> 16};
    return v;
}

__device__ __forceinline__ float other_half(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? r[0] : r[1]);
}
// maximum over the lanes that are 16 and 32 apart
__device__ __forceinline__ float over_quarters(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    const uint32_t a = r[0], b = r[1];          // (a bit cast of a vector's element itself would take element 0)
    v = fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
    return fmaxf(v, other_half(v));
}
// maximum of three, NaN counting for nothing (written out: fmaxf first passes each operand through an instruction of its own)
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    __asm__("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// Results of matrix instructions are read by instructions the compiler does not look into: until the last of them has been written.
template <typename V> __device__ __forceinline__ void settled(V &v) { __asm__ volatile("s_nop 15\n\ts_nop 3" : "+v"(v)); }
__device__ __forceinline__ uint32_t bf16_two(float a, float b)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}

// the sum of two bfloat16 values and c in fp32
__device__ __forceinline__ float add_two(uint32_t two, float c)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), bf16x2{(__bf16)1.f, (__bf16)1.f}, c, false);
}

template <typename T> __device__ __forceinline__ void row_of(const CrossParams &p, int image, int head, int r, const T *&q, const uint8_t *&mask, T *&out)
{
    const int i = (int)((unsigned)r / (unsigned)p.group), g = r - i * p.group;
    const long long at = (long long)image * p.a.Lq + i;
    const int h = (head * p.group + g) * p.a.D;
    q = (const T *)p.a.q + at * p.a.ld_q + h;
    out = (T *)p.a.out + at * p.a.ld_out + h;
    mask = p.a.mask ? p.a.mask + image * p.a.mask_image + i * p.a.mask_row : nullptr;
}

// What a row's exponents may be taken against: a scaled score of any size, held within fp32's range, or -infinity where no state has been
// seen.  The exponentials' sum is about one at least and 2^43 at most (2^30 states, 2^13 each).  A score past the range leaves a sum that is
// zero or infinite, and one so far out, from about 2^26 on, that its product with c is rounded by several powers of two may leave a sum that
// is too small for the bits of its products with small values, or too large: by that the row is known.
__device__ __forceinline__ float in_range(float score) { return fminf(fmaxf(score, -__FLT_MAX__), __FLT_MAX__); }
__device__ __forceinline__ bool beyond(float base, float total) { return base != -HUGE_VALF && !(total > 0x1p-8f && total < 0x1p60f); }

__device__ __forceinline__ float lane_of(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }

// A row whose sums 32 bits do not hold (of scores, or of values too large to be added up), or into whose sums a hidden value that is not finite has gone as 0 * it: a wavefront makes it again
// from the states it sees, lane by lane of the head's values, with scores and sums in 64 bits, which hold every product and sum of fp32
// values.  area: the sums over the head's values to go with `total`, their mean where they are the result.
template <typename T, int DP> __device__ __forceinline__ void row_again(const CrossParams &p, int image, int head, int r, int first, int end, float *area, double &base, float &total)
{
    constexpr int E = (DP + 63) / 64;
    const int lane = threadIdx.x & 63, D = p.a.D;
    const T *q;
    const uint8_t *mask;
    T *unused;
    row_of<T>(p, image, head, r, q, mask, unused);
    const T *const k0 = (const T *)p.a.k + (long long)image * p.a.Lk * p.a.ld_k + head * D, *const v0 = (const T *)p.a.v + (long long)image * p.a.Lk * p.a.ld_v + head * D;
    float qv[E];
    double sum[E] = {}, m = -HUGE_VAL, l = 0.0;
    bool odd = false, sees = false;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        qv[e] = lane + 64 * e < D ? (p.keep ? to_f32(q[lane + 64 * e]) : 0.f) * (p.flip ? -1.f : 1.f) : 0.f;
        odd |= !__builtin_isfinite(qv[e]);
    }
    odd = __any(odd);
    // 64 states at a time: a lane each for the scores, then the lanes of the head's values
    for (int j0 = first; j0 < end; j0 += 64) {
        const int j = min(j0 + lane, end - 1);
        const bool seen = j0 + lane < end && (!mask || mask[j]);
        if (!__any(seen)) continue;
        sees = true;
        if (odd) l = __builtin_nan("");
        if (l != l) break;          // and so is the result
        double dot = 0.0;
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll 1
            for (int d = 0; d < 64 && 64 * e + d < D; d += 8) {
                float k[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) k[i] = to_f32(k0[j * p.a.ld_k + min(64 * e + d + i, D - 1)]);       // behind the head times the zeros of the query
#pragma unroll
                for (int i = 0; i < 8; ++i) dot = __builtin_fma((double)lane_of(qv[e], d + i), (double)k[i], dot);
            }
        double up = seen ? dot : -HUGE_VAL;
        for (int x = 32; x; x >>= 1) up = fmax(up, __shfl_xor(up, x));
        up = fmax(up, m);
        const float shrink = m == -HUGE_VAL ? 0.f : __builtin_amdgcn_exp2f((float)((m - up) * p.c));
        const float w = !seen || dot == -HUGE_VAL ? 0.f : __builtin_amdgcn_exp2f((float)((dot - up) * p.c));
        m = up;
        double all = w;
        for (int x = 32; x; x >>= 1) all += __shfl_xor(all, x);
        l = l * shrink + all;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int d = min(lane + 64 * e, D - 1);
            sum[e] *= shrink;
#pragma unroll 1
            for (int i = 0; i < 64 && j0 + i < end; i += 8) {
                float v[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] = to_f32(v0[min(j0 + i + x, end - 1) * p.a.ld_v + d]);
#pragma unroll
                for (int x = 0; x < 8; ++x) sum[e] = __builtin_fma((double)lane_of(w, i + x), lane_of(w, i + x) == 0.f ? 0.0 : (double)v[x], sum[e]);
            }
        }
    }
    // a share's sums are brought below the largest value by a power of two
    double by = 0.0;
    base = -HUGE_VAL, total = 0.f;
    if (sees && !(l > 0.0)) {
        by = __builtin_nan(""), base = 0.0, total = __builtin_nanf("");
    } else if (sees) {
        const int power = p.shares > 1 ? (int)__builtin_amdgcn_logf((float)l) + 1 : 0;
        by = p.shares > 1 ? __builtin_ldexp(1.0, -power) : 1.0 / l;
        base = m * p.c + power, total = p.shares > 1 ? (float)(l * by) : 1.f;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (lane + 64 * e < DP) area[lane + 64 * e] = (float)(sum[e] * by);
    __builtin_amdgcn_wave_barrier();
}
// Whether everything is finite in a head's states first to end - 1, looked through by a wavefront.  Rows that are not right because a state is not
// finite, which no mask hides, stay as they are: all rows made again would take a thousand times the call's time.
template <typename T> __device__ __forceinline__ bool finite_states(const CrossParams &p, int image, int head, int first, int end)
{
    const T *const k0 = (const T *)p.a.k + (long long)image * p.a.Lk * p.a.ld_k + head * p.a.D, *const v0 = (const T *)p.a.v + (long long)image * p.a.Lk * p.a.ld_v + head * p.a.D;
    bool odd = false;
    for (int d = threadIdx.x & 63; d < p.a.D; d += 64)
        for (int j = first; j < end; ++j) odd |= !__builtin_isfinite(to_f32(k0[j * p.a.ld_k + d])) | !__builtin_isfinite(to_f32(v0[j * p.a.ld_v + d]));
    return !__any(odd);
}

// Four neighbouring sums of a row from d on, out as results or as a share's sums.
template <typename T> __device__ __forceinline__ void put4(const CrossParams &p, T *out, long long part, int d, const float (&v)[4], float total, float inverse)
{
    if (p.shares > 1) {
        if (total != 0.f && d < p.part_ld) *(f32x4_t *)(p.part_o + part * p.part_ld + d) = f32x4_t{v[0], v[1], v[2], v[3]};
        return;
    }
    if (d >= p.a.D) return;
    Vec<T, 4> o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o.v[e] = from_f32<T>(total == 0.f ? 0.f : v[e] * inverse);
    store_some<4>(out + d, o, p.a.D - d);
}

// ---- tiles ------------------------------------------------------------------------------------------------------------
// A workgroup of four wavefronts takes 128 rows, each wavefront 32, and goes over the states in tiles of KT, two images of which lie in
// LDS.  Scores are formed transposed, states x rows, so that a lane holds scores of one row alone (lane % 32): its maximum and sum are sums
// within the lane and over the two halves.  The scores' places in the accumulators are, as they are, the second operand of the
// product with the transposed values: lane half h has states 8 i + 4 h to 8 i + 4 h + 3, and the values' lanes take the same ones.
// fp32 heads of up to 128 run on the bfloat16 instructions, every operand as the sum of three bfloat16 values (x = h + m + l, exact; of the nine
// products the six down to 2^-16 of the largest, the smallest first), each a plane of its own in LDS or registers (4 x 3025 x 729 in 8 heads of
// 64: 160 us on the fp32 instructions, 115 so).  Wider ones run on the fp32 instructions: two images of the planes take 126 KB of LDS at 160
// values, which would fit and has not been made, and 212 KB at 256, which does not.
// bf16: the exponentials are rounded to bfloat16, half a step or 2^-8 each, as the matrix instruction takes them, and it is the rounded ones that
// are added up, so that a row's weights add up to one.  Against 64 bits results are off by 2.0e-3 to 2.3e-3 of their size so, 1.5e-3 to
// 1.7e-3 with fp32 exponentials (of that nearly all the rounding of the result itself).  Exponentials in two pieces would take half as
// many matrix instructions again, and five vector instructions more for two scores, where both bound the kernel.
// Bound by the vector instructions of the exponentials beside the matrix unit: bf16, 16 heads of 64, 16 images of 3025 queries to 4096
// states 880 to 1010 us (800 to 920 TFLOP/s, matrix unit 42 % busy), 4 images in heads of 128 420 to 470 (860 to 960).  Sums by additions instead of
// the two-value instruction need more registers than there are (spills: 1280 us for 960).
template <typename T, int DP> struct Tile {
    static constexpr bool kF32 = sizeof(T) == 4, kSplit = kF32 && DP <= 128;
    static constexpr int KT = kF32 ? 32 : 64, PL = kSplit ? 3 : 1, P = kF32 && !kSplit ? DP / 4 : DP / 8;     // states, planes, 16-byte pieces of a row in LDS
    // Workgroups to a compute unit, with 32 or 64 rows to a wavefront.
    static constexpr int kFit[2] = {DP <= 32 || (DP <= 64 && !kF32) ? 3 : DP <= 96 || (DP <= 128 && !kF32) ? 2 : 1, 2};
    // Pieces from one state to the next: keys in odd steps (a column of pieces covers all banks), values in steps of 4 modulo 8 (the four
    // states of a transposed read lie apart; fp32 ones are read as they lie).
    static constexpr int SK = P + 1, SV = kF32 && !kSplit ? P : P % 8 == 4 ? P : P + 4;
};

// How far scores may pass what the exponents are taken against: in base two, and a lane's sum over a tile.
constexpr float kHeadroom = 8.f, kFar = 8192.f;

template <typename T, int DP, int RB, bool EVEN> __global__ __launch_bounds__(256, (Tile<T, DP>::kFit[RB - 1])) void cross_tile_kernel(CrossParams p)
{
    using Form = Tile<T, DP>;
    constexpr bool kSplit = Form::kSplit, kPlain = Form::kF32 && !kSplit;
    // P: pieces of a row in memory, PT: in LDS
    constexpr int KT = Form::KT, PL = Form::PL, PT = Form::P, SK = Form::SK, SV = Form::SV, n = 16 / (int)sizeof(T), P = DP / n;
    constexpr int kValues = PL * KT * SK, kImage = kValues + PL * KT * SV, NP = KT * P / 256, KB = KT / 32, DB = DP / 32;
    static_assert(KT * P % 256 == 0, "whole pieces per thread");
    __shared__ u32x4_t lds[2 * kImage];
    __shared__ __attribute__((aligned(16))) float biases[2][KT];         // of the states of an image: 0, or -infinity for what no row sees
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    // neighbouring workgroups of an XCD take the row tiles of one image and head
    const unsigned all = gridDim.x, xcd = blockIdx.x & 7;
    const unsigned b = (xcd < all % 8 ? xcd * (all / 8 + 1) : all % 8 * (all / 8 + 1) + (xcd - all % 8) * (all / 8)) + (blockIdx.x >> 3);
    const unsigned share = b % (unsigned)p.shares, bt = b / (unsigned)p.shares;
    const int tile = (int)(bt % (unsigned)p.tiles), ih = (int)(bt / (unsigned)p.tiles), image = ih / p.a.kv_heads, head = ih - image * p.a.kv_heads;
    const int D = p.a.D;
    const int len = p.a.lengths ? min(max(p.a.lengths[image], 0), p.a.Lk) : p.a.Lk;
    const int first = min((long long)share * p.share, (long long)len), end = min(((long long)share + 1) * p.share, (long long)len);

    const int row0 = tile * (128 * RB) + wave * (32 * RB) + (lane & 31);
    const uint8_t *mask[RB];
    u32x4_t q[RB][PL][PT / 2];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const T *qrow;
        T *out;
        row_of<T>(p, image, head, min(row0 + 32 * r, p.rows - 1), qrow, mask[r], out);
        // pieces of a lane: 2 t + half, or for planes the two that make up that one of bfloat16 values
        auto value = [&](int i) { return kSplit ? (2 * (i / 2) + half) * 8 + i % 2 * 4 : (2 * i + half) * n; };
        Piece<EVEN, T> nq[P / 2];
#pragma unroll
        for (int i = 0; i < P / 2; ++i) nq[i] = loaded<EVEN>(qrow, value(i), D);
#pragma unroll
        for (int i = 0; i < P / 2; ++i) {
            u32x4_t v = placed(nq[i], value(i), D, between_words(qrow));
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (v[e] & p.keep) ^ p.flip;
            if constexpr (kSplit) {
                const f32x4_t f = __builtin_bit_cast(f32x4_t, v);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    uint32_t h, m, l;
                    split_pair(f[2 * e], f[2 * e + 1], h, m, l);
                    q[r][0][i / 2][i % 2 * 2 + e] = h, q[r][1][i / 2][i % 2 * 2 + e] = m, q[r][2][i / 2][i % 2 * 2 + e] = l;
                }
            } else {
                q[r][0][i] = v;
            }
        }
    }
    const T *const k0 = (const T *)p.a.k + (long long)image * p.a.Lk * p.a.ld_k + head * D, *const v0 = (const T *)p.a.v + (long long)image * p.a.Lk * p.a.ld_v + head * D;
    // What hides states from every row, a mask by states or the end of them, is what the scores start from.  (A key there that is not finite
    // makes the row's sums NaN, and the row is made again.)
    const bool by_state = p.a.mask && p.a.mask_row == 0, by_pair = RB == 1 && p.a.mask && p.a.mask_row != 0;      // (wider blocks are not launched for these)
    const uint8_t *const shared = by_state ? p.a.mask + image * p.a.mask_image : nullptr;
    uint32_t seen = 0;
    // A thread's pieces are those at e % P of the states e / P of a tile, e = threadIdx.x + 256 i, the same in every tile.
    Piece<EVEN, T> nk[NP], nv[NP];
    uint32_t odd = 0;           // bits 2 i and 2 i + 1: whether their rows begin between words
    long long step_k[NP], step_v[NP];
    if (EVEN)
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int e = threadIdx.x + i * 256, d = min(e % P * n, D - n);
            step_k[i] = e / P * p.a.ld_k + d, step_v[i] = e / P * p.a.ld_v + d;
        }
    // Whether a tile's biases are written: wide blocks, whose registers are all taken, write them only where they are looked at (16 x 3025 x
    // 4096 in 16 heads of 64 998 -> 987 us); the others have no use for the test (fp32 4 x 3025 x 729 117 -> 121).
    auto some_hidden_at = [&](int at) { return RB == 1 || p.a.mask || at + KT > end; };
    auto fetch = [&](int at) {
        if (some_hidden_at(at) && threadIdx.x < KT) seen = at + (int)threadIdx.x < end && (!by_state || shared[at + threadIdx.x]);
        const T *const kt = k0 + at * p.a.ld_k, *const vt = v0 + at * p.a.ld_v;
        if (EVEN && at + KT <= end) {
#pragma unroll
            for (int i = 0; i < NP; ++i) nk[i].v = __builtin_bit_cast(u32x4_t, load_n<n>(kt + step_k[i])), nv[i].v = __builtin_bit_cast(u32x4_t, load_n<n>(vt + step_v[i]));
        } else {        // states behind the last are the last one again
            odd = 0;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int e = threadIdx.x + i * 256, j = min(e / P, end - 1 - at), d = e % P * n;
                const T *const kj = kt + j * p.a.ld_k, *const vj = vt + j * p.a.ld_v;
                nk[i] = loaded<EVEN>(kj, d, D);
                nv[i] = loaded<EVEN>(vj, d, D);
                odd |= between_words(kj) << 2 * i | between_words(vj) << (2 * i + 1);
            }
        }
    };
    auto store = [&](int image_of, int at) {
        u32x4_t *const to = lds + image_of * kImage;
        if (some_hidden_at(at) && threadIdx.x < KT) biases[image_of][threadIdx.x] = seen ? 0.f : -HUGE_VALF;
        if constexpr (!EVEN)
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int d = (int)(threadIdx.x + i * 256) % P * n;
                nk[i].v = placed(nk[i], d, D, odd >> 2 * i & 1);
                nv[i].v = placed(nv[i], d, D, odd >> (2 * i + 1) & 1);
            }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int e = threadIdx.x + i * 256, j = e / P, d = e % P;
            if constexpr (kSplit) {
                auto planes = [&](u32x4_t v, uint2 *at, int plane) {
                    const f32x4_t f = __builtin_bit_cast(f32x4_t, v);
                    uint2 h, m, l;
                    split_pair(f[0], f[1], h.x, m.x, l.x);
                    split_pair(f[2], f[3], h.y, m.y, l.y);
                    at[0] = h, at[2 * plane] = m, at[4 * plane] = l;
                };
                planes(nk[i].v, (uint2 *)(to + j * SK) + d, KT * SK);
                planes(nv[i].v, (uint2 *)(to + kValues + j * SV) + d, KT * SV);
            } else {
                to[j * SK + d] = nk[i].v;
                to[kValues + j * SV + d] = nv[i].v;
            }
        }
    };
    // (Zeros that the compiler does not know: a constant would be the one that the scores start from too, and keep that one in registers.)
    float zero = 0.f;
    __asm__ volatile("" : "+v"(zero));
    f32x16_t o[RB][DB];
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[r][d][i] = zero;
    float base[RB], total[RB];      // what the exponents are taken against, in base two, and their sum
#pragma unroll
    for (int r = 0; r < RB; ++r) base[r] = -HUGE_VALF, total[r] = 0.f;
    if (first < end) {
        fetch(first);
        store(0, first);
    }
    __syncthreads();
    int img = 0;
    // some_hidden: whether some states may be; where that is a constant, the others' way has neither the tests nor the registers for it
    auto tile_of = [&](int at, auto some_hidden) __attribute__((always_inline)) {
        const bool hidden = some_hidden;
        const bool more = at + KT < end;
        if (more) fetch(at + KT);
        uint32_t bytes[RB][KB * 4];
        if (hidden && by_pair) {
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int i = 0; i < KB * 4; ++i) {
                    const int j = at + i * 8 + half * 4;
                    if (at + KT <= end) __builtin_memcpy(&bytes[r][i], mask[r] + j, 4);
                    else bytes[r][i] = __builtin_bit_cast(uint32_t, load_some<4>(mask[r] + min(j, end - 1), end - min(j, end - 1)));
                }
        }
        const u32x4_t *const keys = lds + img * kImage, *const values = keys + kValues;
        __builtin_amdgcn_s_setprio(1);
        f32x16_t s[RB][KB];
        u32x4_t pt[RB][PL][kPlain ? 1 : KT / 16];         // their exponentials: bfloat16 pairs, or as they are
        f32x16_t pf[kPlain ? RB : 1];
        float part[RB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            f32x16_t start = {};
            if (hidden) {
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const f32x4_t of = *(const f32x4_t *)&biases[img][kb * 32 + i * 2 + half * 4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) start[i + e] = of[e];
                }
            }
#pragma unroll
            for (int r = 0; r < RB; ++r) s[r][kb] = start;
#pragma unroll
            for (int t = 0; t < PT / 2; ++t) {
                u32x4_t k[PL];
#pragma unroll
                for (int a = 0; a < PL; ++a) k[a] = keys[(a * KT + kb * 32 + (lane & 31)) * SK + 2 * t + half];
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    if constexpr (kPlain) {
                        const f32x4_t kf = __builtin_bit_cast(f32x4_t, k[0]), qf = __builtin_bit_cast(f32x4_t, q[r][0][t]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[r][kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qf[e], s[r][kb], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int sum = PL - 1; sum >= 0; --sum)
#pragma unroll
                            for (int a = 0; a <= sum; ++a)
                                s[r][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k[a]), __builtin_bit_cast(bf16x8, q[r][sum - a][t]), s[r][kb], 0, 0, 0);
                    }
                }
            }
        }
        uint32_t seen_of[RB] = {};
        if (hidden && by_pair) {
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int i = 0; i < KB * 4; ++i) seen_of[r] |= bytes[r][i];
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[r][kb][i] = bytes[r][kb * 4 + i / 4] >> i % 4 * 8 & 255 ? s[r][kb][i] : -HUGE_VALF;
        }
        // The exponents are taken against the base as it stands.  Only where there is none yet, or where a sum shows that scores have passed
        // it by far, is the tile's maximum looked for, and only where that raises a base are they taken again (a row that sees nothing goes
        // no further: 4 x 3025 queries x 4096 states of which one image hides all 280 us for 373, all the first half 266 for 308).
        __builtin_amdgcn_s_setprio(0);
        auto exponents = [&](int r) {
            const float off = base[r] == -HUGE_VALF ? 0.f : base[r];
            part[r] = 0.f;
            auto p_of = [&](int i) { return __builtin_amdgcn_exp2f(__builtin_fmaf(s[r][i / 16][i % 16], p.c, -off)); };
            if constexpr (kPlain) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    pf[r][i] = p_of(i);
                    part[r] += pf[r][i];
                }
            } else {
#pragma unroll
                for (int t = 0; t < KT / 16; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float a = p_of(t * 8 + 2 * e), b = p_of(t * 8 + 2 * e + 1);
                        if constexpr (kSplit) {
                            uint32_t h, m, l;
                            split_pair(a, b, h, m, l);
                            pt[r][0][t][e] = h, pt[r][1][t][e] = m, pt[r][2][t][e] = l;
                            part[r] += a + b;
                        } else {
                            pt[r][0][t][e] = bf16_two(a, b);
                            part[r] = add_two(pt[r][0][t][e], part[r]);
                        }
                    }
            }
        };
        bool far = false;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            exponents(r);
            far |= part[r] > kFar || base[r] == -HUGE_VALF;
        }
        if (__any(far)) {
            // whether a row sees any state of this tile, which its scores may not tell where all are -infinity
            bool some = true, raise = false;
            float raised[RB];
            if (hidden && by_state) some = __any(biases[img][lane & (KT - 1)] == 0.f);
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                if (hidden && by_pair) some = (seen_of[r] | __shfl_xor(seen_of[r], 32)) != 0;
                float top = s[r][0][0];
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[r][kb][i]);
                top *= p.c;
                raised[r] = some ? fmaxf(base[r], in_range(fmaxf(top, other_half(top)))) : base[r];
                raise |= raised[r] != base[r];
            }
            if (__any(raise))
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    const float shrink = base[r] == -HUGE_VALF ? 0.f : __builtin_amdgcn_exp2f(base[r] - raised[r]);
                    total[r] *= shrink;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[r][d][i] *= shrink;
                    base[r] = raised[r];
                    exponents(r);
                }
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) total[r] += part[r];
        __builtin_amdgcn_s_setprio(1);
        if constexpr (kPlain) {
            const float *const vf = (const float *)values;
#pragma unroll
            for (int i = 0; i < 16; ++i)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const float v = vf[(i / 4 * 8 + half * 4 + i % 4) * SV * 4 + d * 32 + (lane & 31)];
#pragma unroll
                    for (int r = 0; r < RB; ++r) o[r][d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, pf[r][i], o[r][d], 0, 0, 0);
                }
        } else {
            typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
#pragma unroll
            for (int t = 0; t < KT / 16; ++t) {
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    bf16x8 vt[PL];
#pragma unroll
                    for (int a = 0; a < PL; ++a) {
                        // sixteen lanes read four states of sixteen neighbouring values, a lane four of them, and get a column each
                        const char *const from = (const char *)(values + (a * KT + t * 16 + half * 4 + (lane & 15) / 4) * SV) + d * 64 + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
                        const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)from), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(from + 8 * SV * 16));
                        const auto both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                        vt[a] = __builtin_bit_cast(bf16x8, both);
                    }
#pragma unroll
                    for (int r = 0; r < RB; ++r)
#pragma unroll
                        for (int sum = PL - 1; sum >= 0; --sum)
#pragma unroll
                            for (int a = 0; a <= sum; ++a)
                                o[r][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vt[a], __builtin_bit_cast(bf16x8, pt[r][sum - a][t]), o[r][d], 0, 0, 0);
                }
            }
        }
        __builtin_amdgcn_s_setprio(0);
        img ^= 1;
        if (more) store(img, at + KT);
        __syncthreads();
    };
    int at = first;
    if constexpr (sizeof(T) == 2 && DP <= 128) {
        if (!p.a.mask)
            for (; at + KT <= end; at += KT) tile_of(at, std::false_type{});
        for (; at < end; at += KT) tile_of(at, std::true_type{});
    } else {        // (in wider heads there are no registers for two ways)
        for (; at < end; at += KT) tile_of(at, p.a.mask || at + KT > end);
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        total[r] += other_half(total[r]);
        const int row = row0 + 32 * r;
        double base_of = base[r];
        const bool lost = beyond(base[r], total[r]);
        float zeros[2] = {};        // NaN where a sum is not finite
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) zeros[i & 1] = __builtin_fmaf(o[r][d][i], 0.f, zeros[i & 1]);
        const uint64_t lanes = __ballot((lost || !(zeros[0] + zeros[1] == 0.f)) && row < p.rows);
        uint32_t again = (uint32_t)lanes | (uint32_t)(lanes >> 32);
        if (__builtin_expect(again != 0, 0)) {
            if (!p.a.mask && !finite_states<T>(p, image, head, first, end)) {
                if (lost) total[r] = __builtin_nanf("");
                again = 0;
            }
            float *const area = (float *)lds + wave * DP;
            static_assert(4 * DP * 4 <= 2 * kImage * 16, "the areas fit");
            while (again) {
                const int which = __builtin_ctz(again);
                again &= again - 1;
                double m;
                float l;
                row_again<T, DP>(p, image, head, row - (lane & 31) + which, first, end, area, m, l);
                if ((lane & 31) == which) {
                    base_of = m, total[r] = l;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[r][d][i] = area[d * 32 + i / 4 * 8 + half * 4 + i % 4];
                }
                __builtin_amdgcn_wave_barrier();
            }
        }
        if (row >= p.rows) continue;
        const long long part = ((long long)share * p.a.N * p.a.kv_heads + ih) * p.rows + row;
        if (p.shares > 1 && half == 0) p.part_ml[part] = PartSum{base_of, total[r]};
        const T *qrow;
        const uint8_t *unused;
        T *out;
        row_of<T>(p, image, head, row, qrow, unused, out);
        const float inverse = 1.f / total[r];
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const float v[4] = {o[r][d][i], o[r][d][i + 1], o[r][d][i + 2], o[r][d][i + 3]};
                put4<T>(p, out, part, d * 32 + i * 2 + half * 4, v, total[r], inverse);
            }
    }
}

// ---- few rows ----------------------------------------------------------------------------------------------------------
// A workgroup takes 16 rows, its wavefronts share out the states in chunks of KC, each with sums of its own for all 16 rows, which are
// added up through LDS in the end.  Keys go from memory straight into the lanes of the 16 x 16 instructions (lane l takes 16 bytes of key
// l % 16 at piece l / 16), and the next chunk's are on their way as soon as these are multiplied.  Scores lie transposed as above: lane l
// has states 4 (l / 16) to 4 (l / 16) + 3 of row l % 16.
//   bf16: values go through the wavefront's part of LDS, which gives them back transposed
//   fp32: an instruction takes one state of each four, and value e of each four of a head, so that lanes load 16 bytes of neighbouring values
// Bound by memory where states are many (8 queries to 16384 states of 8 heads of 128: 114 us, 4.7 TB/s), else by the latency of a turn of
// loads and of the joining (1 query to 729 states of 8 heads of 64: 8.1 us).
template <typename T> struct Chunk;
template <> struct Chunk<bf16_t> {
    static constexpr int KC = 32;
};
template <> struct Chunk<float> {
    static constexpr int KC = 16;
};
template <typename T, int DP, int NW, bool EVEN> __global__ __launch_bounds__(64 * NW) void cross_wave_kernel(CrossParams p)
{
    constexpr bool kF32 = sizeof(T) == 4;
    constexpr int KC = Chunk<T>::KC, n = 16 / (int)sizeof(T), P = DP / n, KB = KC / 16;
    constexpr int SV = P % 8 == 4 ? P : P + 4;      // bf16: pieces from one state to the next in LDS
    constexpr int NV = kF32 ? 4 * ((DP + 63) / 64) : KC * P / 64, DB = kF32 ? (DP + 63) / 64 * 4 : DP / 16;
    constexpr int kRow = DP + 4;                                    // of a wavefront's sums
    constexpr int kArea = kF32 ? 0 : KC * SV, kRoom = kArea > 4 * kRow ? NW * kArea : NW * 4 * kRow;        // 16 bytes: of a wavefront's values; in all
    __shared__ u32x4_t lds[kRoom];
    __shared__ float bases[NW][16], totals[NW][16];
    __shared__ int again[16], some_again;
    __shared__ PartSum made[16];        // of the rows that are made again
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, quarter = lane >> 4;
    const unsigned share = blockIdx.x % (unsigned)p.shares, bt = blockIdx.x / (unsigned)p.shares;
    const int tile = (int)(bt % (unsigned)p.tiles), ih = (int)(bt / (unsigned)p.tiles), image = ih / p.a.kv_heads, head = ih - image * p.a.kv_heads;
    const int D = p.a.D;
    const int len = p.a.lengths ? min(max(p.a.lengths[image], 0), p.a.Lk) : p.a.Lk;
    const int first = min((long long)share * p.share, (long long)len), end = min(((long long)share + 1) * p.share, (long long)len);
    const int row = tile * 16 + l16;
    const T *qrow;
    const uint8_t *mask;
    T *out;
    row_of<T>(p, image, head, min(row, p.rows - 1), qrow, mask, out);
    u32x4_t q[P / 4];
    Piece<EVEN, T> nq[P / 4];
#pragma unroll
    for (int t = 0; t < P / 4; ++t) nq[t] = loaded<EVEN>(qrow, (4 * t + quarter) * n, D);
    const T *const k0 = (const T *)p.a.k + (long long)image * p.a.Lk * p.a.ld_k + head * D, *const v0 = (const T *)p.a.v + (long long)image * p.a.Lk * p.a.ld_v + head * D;
    Piece<EVEN, T> nk[KB][P / 4], nv[NV];
    uint32_t bytes[KB];                 // of the mask
    uint32_t odd_k = 0, odd_v = 0;      // bit i: whether the i-th row begins between words
    auto fetch_keys = [&](int at) {
        odd_k = 0;
        if (mask)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                const int j = at + kb * 16 + quarter * 4, there = min(j, end - 1);
                if (at + KC <= end) __builtin_memcpy(&bytes[kb], mask + j, 4);
                else bytes[kb] = __builtin_bit_cast(uint32_t, load_some<4>(mask + there, end - there));
            }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const T *const kj = k0 + min(at + kb * 16 + l16, end - 1) * p.a.ld_k;
#pragma unroll
            for (int t = 0; t < P / 4; ++t) nk[kb][t] = loaded<EVEN>(kj, (4 * t + quarter) * n, D);
            odd_k |= between_words(kj) << kb;
        }
    };
    // bf16: piece e % P of state e / P, e = lane + 64 i; fp32: values 64 (i / 4) + 4 (lane % 16) on of state 4 (lane / 16) + i % 4
    auto value_state = [&](int i) { return kF32 ? 4 * quarter + i % 4 : (lane + 64 * i) / P; };
    auto value_at = [&](int i) { return kF32 ? i / 4 * 64 + 4 * l16 : (lane + 64 * i) % P * n; };
    auto fetch_values = [&](int at) {
        odd_v = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const T *const vj = v0 + min(at + value_state(i), end - 1) * p.a.ld_v;
            nv[i] = loaded<EVEN>(vj, value_at(i), D);
            odd_v |= between_words(vj) << i;
        }
    };
    f32x4_t o[DB] = {};
    // scores above `limit` raise the base
    float base = -HUGE_VALF, limit = -HUGE_VALF, total = 0.f;
    int at = first + wave * KC;
    uint32_t sees = !mask && at < end;
    if (at < end) {
        fetch_keys(at);
        fetch_values(at);
    }
#pragma unroll
    for (int t = 0; t < P / 4; ++t) {
        q[t] = placed(nq[t], (4 * t + quarter) * n, D, between_words(qrow));
#pragma unroll
        for (int e = 0; e < 4; ++e) q[t][e] = (q[t][e] & p.keep) ^ p.flip;
    }
    u32x4_t *const area = lds + wave * kArea;
    for (; at < end; at += NW * KC) {
        const bool more = at + NW * KC < end;
        f32x4_t s[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            s[kb] = f32x4_t{};
#pragma unroll
            for (int t = 0; t < P / 4; ++t) {
                const u32x4_t k = EVEN ? nk[kb][t].v : placed(nk[kb][t], (4 * t + quarter) * n, D, odd_k >> kb & 1);
                if constexpr (kF32) {
                    const f32x4_t kf = __builtin_bit_cast(f32x4_t, k), qf = __builtin_bit_cast(f32x4_t, q[t]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[kb] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[e], s[kb], 0, 0, 0);
                } else {
                    s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q[t]), s[kb], 0, 0, 0);
                }
            }
        }
        if (mask || at + KC > end) {
            if (mask)
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) sees |= bytes[kb];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    s[kb][e] = at + kb * 16 + quarter * 4 + e < end && (!mask || (bytes[kb] >> e * 8 & 255)) ? s[kb][e] : -HUGE_VALF;
        }
        if (more) fetch_keys(at + NW * KC);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) settled(s[kb]);
        float top = max3(s[0][0], s[0][1], s[0][2]);
        top = max3(top, s[0][3], s[KB - 1][0]);
        if constexpr (KB > 1) top = max3(max3(top, s[1][1], s[1][2]), s[1][3], top);
        if (__any(top > limit)) {
            const float highest = over_quarters(top);
            const float raised = highest == -HUGE_VALF ? base : fmaxf(base, in_range(highest * p.c)), shrink = base == -HUGE_VALF ? 0.f : __builtin_amdgcn_exp2f(base - raised);
            total *= shrink;
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d] *= shrink;
            base = raised;
            limit = (base + kHeadroom) / p.c;
        }
        const float off = base == -HUGE_VALF ? 0.f : base;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[kb][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][e], p.c, -off));
                total += s[kb][e];
            }
        u32x4_t v[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = EVEN ? nv[i].v : placed(nv[i], value_at(i), D, odd_v >> i & 1);
        if constexpr (kF32) {
            if (more) fetch_values(at + NW * KC);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    o[i / 4 * 4 + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(f32x4_t, v[i])[e], s[0][i % 4], o[i / 4 * 4 + e], 0, 0, 0);
        } else {
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < NV; ++i) area[(lane + 64 * i) / P * SV + (lane + 64 * i) % P] = v[i];
            __builtin_amdgcn_wave_barrier();
            if (more) fetch_values(at + NW * KC);
            typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
            const u32x4_t pt = {bf16_two(s[0][0], s[0][1]), bf16_two(s[0][2], s[0][3]), bf16_two(s[KB - 1][0], s[KB - 1][1]), bf16_two(s[KB - 1][2], s[KB - 1][3])};
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const char *const from = (const char *)(area + (quarter * 4 + l16 / 4) * SV) + d * 32 + (lane & 3) * 8;
                const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)from), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(from + 16 * SV * 16));
                const auto vt = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt), __builtin_bit_cast(bf16x8, pt), o[d], 0, 0, 0);
            }
        }
    }
    // every wavefront's sums against the largest base, added up by all threads, four of a row each, in order of wavefronts
    total += __shfl_xor(total, 16);
    total += __shfl_xor(total, 32);
    sees |= __shfl_xor(sees, 16);
    sees |= __shfl_xor(sees, 32);
    if (sees && base == -HUGE_VALF) base = -__FLT_MAX__;        // all of its scores are -infinity
    if (quarter == 0) bases[wave][l16] = base, totals[wave][l16] = total;
    __syncthreads();
    float most = bases[0][l16];
#pragma unroll
    for (int w = 1; w < NW; ++w) most = fmaxf(most, bases[w][l16]);
    // (without a base the sums are zero, or not finite: of 0 * a masked value)
    const float by = base == -HUGE_VALF ? 1.f : __builtin_amdgcn_exp2f(base - most);
    float *const sums = (float *)lds;
    if (row < p.rows)
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            // the d-th four neighbouring sums of a lane
            f32x4_t v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = by * (kF32 ? o[d / 4 * 4 + e][d % 4] : o[d][e]);
            const int at_d = kF32 ? d / 4 * 64 + quarter * 16 + d % 4 * 4 : d * 16 + quarter * 4;
            if (at_d < DP) *(f32x4_t *)&sums[(wave * 16 + l16) * kRow + at_d] = v;
        }
    if (threadIdx.x < 16) again[threadIdx.x] = 0;
    if (threadIdx.x == 16) some_again = 0;
    __syncthreads();
    constexpr int kQuads = DP / 4, kTurns = (16 * kQuads + 64 * NW - 1) / (64 * NW);
    f32x4_t of[kTurns];
    float top_of[kTurns], sum_of[kTurns];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        const int e = threadIdx.x + t * 64 * NW, r = e / kQuads, d = e % kQuads * 4;
        if (r >= 16 || tile * 16 + r >= p.rows) continue;
        of[t] = *(const f32x4_t *)&sums[r * kRow + d];
#pragma unroll
        for (int w = 1; w < NW; ++w) of[t] += *(const f32x4_t *)&sums[(w * 16 + r) * kRow + d];
        float top = bases[0][r], sum = 0.f;
#pragma unroll
        for (int w = 1; w < NW; ++w) top = fmaxf(top, bases[w][r]);
#pragma unroll
        for (int w = 0; w < NW; ++w) sum += bases[w][r] == -HUGE_VALF ? totals[w][r] : totals[w][r] * __builtin_amdgcn_exp2f(bases[w][r] - top);
        const f32x4_t zeros = 0.f * of[t];      // NaN where a sum is not finite
        if (beyond(top, sum) || !(zeros[0] + zeros[1] + (zeros[2] + zeros[3]) == 0.f)) again[r] = some_again = 1;
        top_of[t] = top, sum_of[t] = sum;
    }
    __syncthreads();
    const bool remake = some_again && (mask || finite_states<T>(p, image, head, first, end));
    if (__builtin_expect(remake, 0)) {
        for (int r = wave; r < 16; r += NW)
            if (again[r]) {
                double m;
                float l;
                row_again<T, DP>(p, image, head, tile * 16 + r, first, end, &sums[r * kRow], m, l);
                if (lane == 0) made[r] = PartSum{m, l};
            }
        __syncthreads();
    }
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        const int e = threadIdx.x + t * 64 * NW, r = e / kQuads, d = e % kQuads * 4;
        if (r >= 16 || tile * 16 + r >= p.rows) continue;
        PartSum own{top_of[t], sum_of[t]};
        if (remake && again[r]) own = made[r], of[t] = *(const f32x4_t *)&sums[r * kRow + d];
        else if (beyond(top_of[t], sum_of[t])) own.total = __builtin_nanf("");
        const long long part = ((long long)share * p.a.N * p.a.kv_heads + ih) * p.rows + tile * 16 + r;
        if (p.shares > 1 && d == 0) p.part_ml[part] = own;
        const T *q_of;
        const uint8_t *mask_of;
        T *to;
        row_of<T>(p, image, head, tile * 16 + r, q_of, mask_of, to);
        const float v[4] = {of[t][0], of[t][1], of[t][2], of[t][3]};
        put4<T>(p, to, part, d, v, own.total, 1.f / own.total);
    }
}

// Four neighbouring results of a row from few shares' sums.
constexpr int kFewShares = 8;
template <typename T> __global__ __launch_bounds__(256) void cross_join_few_kernel(CrossParams p, long long all)
{
    const int quads = p.part_ld / 4;
    const long long e = blockIdx.x * 256ll + threadIdx.x, at = e / quads;
    if (at >= all) return;
    const int d = (int)(e - at * quads) * 4;
    PartSum ml[kFewShares];
    f32x4_t of[kFewShares];
#pragma unroll
    for (int s = 0; s < kFewShares; ++s)
        if (s < p.shares) {
            ml[s] = p.part_ml[s * all + at];
            of[s] = *(const f32x4_t *)(p.part_o + (s * all + at) * p.part_ld + d);      // (not written where a share saw nothing; not used then)
        }
    double most = -HUGE_VAL;
    float total = 0.f;
#pragma unroll
    for (int s = 0; s < kFewShares; ++s)
        if (s < p.shares && ml[s].total != 0.f) most = fmax(most, ml[s].base);
    float w[kFewShares];
#pragma unroll
    for (int s = 0; s < kFewShares; ++s)
        if (s < p.shares && ml[s].total != 0.f) {
            w[s] = __builtin_amdgcn_exp2f((float)(ml[s].base - most));
            total += w[s] * ml[s].total;
        }
    // each share's part of the mean, as the sum of the shares' sums may pass the range
    const float inverse = 1.f / total;
    f32x4_t v = {};
#pragma unroll
    for (int s = 0; s < kFewShares; ++s)
        if (s < p.shares && ml[s].total != 0.f) v += w[s] * inverse * of[s];
    const int ih = (int)(at / p.rows), image = ih / p.a.kv_heads;
    const T *q;
    const uint8_t *mask;
    T *out;
    row_of<T>(p, image, ih - image * p.a.kv_heads, (int)(at - (long long)ih * p.rows), q, mask, out);
    const float f[4] = {v[0], v[1], v[2], v[3]};
    p.shares = 1;
    put4<T>(p, out, 0, d, f, total, 1.f);
}

// The shares' sums of a row, four neighbouring values to a thread, the shares dealt out among as many threads as a workgroup has beside that:
// one after the other they cost a memory latency each (16 shares of 256 rows 21 us, in parallel 4).
constexpr int kMostShares = 64;
template <typename T> __global__ __launch_bounds__(256) void cross_join_kernel(CrossParams p, long long all, int lanes)
{
    __shared__ float weights[kMostShares];
    __shared__ f32x4_t red[256];
    const long long at = blockIdx.x;
    if (threadIdx.x < 64) {
        const PartSum ml = (int)threadIdx.x < p.shares ? p.part_ml[threadIdx.x * all + at] : PartSum{-HUGE_VAL, 0.f};
        const bool none = ml.total == 0.f;
        double most = none ? -HUGE_VAL : ml.base;
        for (int x = 32; x; x >>= 1) most = fmax(most, __shfl_xor(most, x));
        const float w = none ? 0.f : __builtin_amdgcn_exp2f((float)(ml.base - most));
        float sum = none ? 0.f : w * ml.total;
        for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
        weights[threadIdx.x] = w == 0.f ? 0.f : w / sum;        // of the mean, as the sum of the shares' sums may pass the range
    }
    __syncthreads();
    const int group = threadIdx.x / (unsigned)lanes, groups = 256 / lanes, d = ((int)threadIdx.x - group * lanes) * 4;
    f32x4_t v = {};
    if (d < p.part_ld)
#pragma unroll 4
        for (int s = group; s < p.shares; s += groups)
            if (weights[s] != 0.f) v += weights[s] * *(const f32x4_t *)(p.part_o + (s * all + at) * p.part_ld + d);
    red[threadIdx.x] = v;
    __syncthreads();
    if (group || d >= p.a.D) return;
    for (int g = 1; g < groups; ++g) v += red[g * lanes + threadIdx.x];
    const int ih = (int)(at / p.rows), image = ih / p.a.kv_heads;
    const T *q;
    const uint8_t *mask;
    T *out;
    row_of<T>(p, image, ih - image * p.a.kv_heads, (int)(at - (long long)ih * p.rows), q, mask, out);
    Vec<T, 4> o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o.v[i] = from_f32<T>(v[i]);
    store_some<4>(out + d, o, p.a.D - d);
}

// Widths the kernels are made for.
constexpr int wave_count(int DP) { return DP <= 64 ? 16 : DP <= 160 ? 8 : 4; }
int padded(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : D <= 96 ? 96 : D <= 128 ? 128 : D <= 160 ? 160 : 256; }

int part_row(int D) { return (D + 3) / 4 * 4; }
// Workgroups of the launch that joins the shares of `all` rows.
double join_blocks(long long all, int D, int shares) { return shares <= kFewShares ? (double)((all * (part_row(D) / 4) - 1) / 256 + 1) : (double)all; }

// How the rows are shared out, in blocks of `block` (16: the form for few rows), and the states, in shares of `share`.  By estimate: us of a
// workgroup's pass over a tile of states (bf16 64, fp32 32; in the form for few rows what its wavefronts take at a time) when it has a compute
// unit to itself and when units are full, from what heads of 64 measured; a second launch that joins shares costs 4 us, and their sums' bytes.
// (us, blocks of 16 / 128 / 256, bf16, 8 heads of 64: 64 rows x 2000 states 12.2 / 11.0 / 13.3, 512 x 2000 16.0 / 17.6 / 21.5, 2 images of 2000 x
// 2000 108 / 35 / 50; 16 heads: 4 images of 1024 x 4096 366 / 94 / 103, of 3025 x 4096 1049 / 252 / 248, 16 images of these 4190 / 969 / 934.  The
// estimate is short of that where three blocks of 256 come to a unit that holds two, as in the second last, and takes 128.)  Of plans within
// 5 % the one with the most shares: images may have fewer states than the others.
struct Plan { int rows, tiles, share, shares, block; };
bool plan_of(int N, int Lq, int Lk, int heads, int kv_heads, int D, int dtype, Plan &plan)
{
    const long long rows = (long long)Lq * (heads / kv_heads);
    if (rows > 1 << 30 || Lk > 1 << 30) return false;
    const bool f32 = dtype == SQ_F32;
    const int DP = padded(D), waves = wave_count(DP);
    const double g = std::max(DP / 64.0, 0.6);
    struct Form { int block, unit, fit; double alone, full; };
    const Form forms[] = {{16, waves * (f32 ? 16 : 32), 1, f32 ? 3.5 : DP <= 64 ? 2.7 : 2.4, f32 ? 3.5 : DP <= 64 ? 2.7 : 2.4},
                          {128, f32 ? 32 : 64, DP <= 64 ? 3 : DP <= 128 ? 2 : 1, g * (f32 ? 2.5 : 1.05), g * (f32 ? 2.1 : 0.62)},
                          {256, 64, 2, g * 2.2, g * 1.17}};
    double best = HUGE_VAL;
    for (int i = 0; i < (f32 || DP > 64 ? 2 : 3); ++i) {
        const Form &w = forms[i];
        const int tiles = (int)((rows - 1) / w.block + 1), units = std::max((Lk - 1) / w.unit + 1, 1);
        const double blocks = (double)N * kv_heads * tiles;
        for (int want = 1; want <= std::min(units, kMostShares); want += want < 4 ? 1 : want < 16 ? 4 : 16) {
            const int each = (units - 1) / want + 1, shares = (units - 1) / each + 1;
            if ((shares != want && want > 1) || !one_launch(blocks * shares, 1024)) continue;
            if (shares > 1 && !one_launch(join_blocks(N * kv_heads * rows, D, shares), 256)) continue;
            const double on_one = std::ceil(blocks * shares / 256);
            const double us = 3.0 + (w.block == 16 ? 0.8 * on_one : 1.5) + each * std::max(w.alone * std::ceil(on_one / w.fit), w.full * on_one) +
                              (shares > 1 ? 4.0 + 4e-6 * shares * N * kv_heads * rows * D : 0.0);
            if (us < (shares > plan.shares && best < HUGE_VAL && plan.block == w.block && plan.shares > 1 ? 1.05 : 1.0) * best) {
                best = std::min(best, us);
                plan = Plan{(int)rows, tiles, each * w.unit, shares, w.block};
            }
        }
    }
    return best < HUGE_VAL;
}
template <typename T, int DP, bool EVEN> int launch(const CrossParams &p, int block)
{
    const dim3 grid((unsigned)(p.a.N * p.a.kv_heads) * p.tiles * p.shares);
    const LaunchScope prof(block == 16 ? "cross_wave" : "cross_tile", cross_flops(p.a), cross_bytes(p.a));
    constexpr int NW = wave_count(DP);
    if (block == 16) {
        hipLaunchKernelGGL((cross_wave_kernel<T, DP, NW, EVEN>), grid, dim3(64 * NW), 0, current_stream(), p);
        return check_launch();
    }
    if constexpr (sizeof(T) == 2 && DP <= 64)
        if (block == 256) {
            hipLaunchKernelGGL((cross_tile_kernel<T, DP, 2, EVEN>), grid, dim3(256), 0, current_stream(), p);
            return check_launch();
        }
    hipLaunchKernelGGL((cross_tile_kernel<T, DP, 1, EVEN>), grid, dim3(256), 0, current_stream(), p);
    return check_launch();
}
template <typename T, int DP> int launch(const CrossParams &p, int block)
{
    return p.a.D % (16 / (int)sizeof(T)) == 0 ? launch<T, DP, true>(p, block) : launch<T, DP, false>(p, block);
}
template <typename T> int by_width(const CrossParams &p, int block)
{
    switch (padded(p.a.D)) {
        case 32: return launch<T, 32>(p, block);
        case 64: return launch<T, 64>(p, block);
        case 96: return launch<T, 96>(p, block);
        case 128: return launch<T, 128>(p, block);
        case 160: return launch<T, 160>(p, block);
        default: return launch<T, 256>(p, block);
    }
}
template <typename T> int run(const CrossParams &p, int block)
{
    if (const int rc = by_width<T>(p, block)) return rc;
    if (p.shares == 1) return SQ_OK;
    const long long all = (long long)p.a.N * p.a.kv_heads * p.rows;
    const LaunchScope prof("cross_join", 0, 0);
    const dim3 grid((unsigned)join_blocks(all, p.a.D, p.shares));
    if (p.shares <= kFewShares) {
        hipLaunchKernelGGL((cross_join_few_kernel<T>), grid, dim3(256), 0, current_stream(), p, all);
        return check_launch();
    }
    int lanes = 1;
    while (lanes * 4 < p.part_ld) lanes *= 2;
    hipLaunchKernelGGL((cross_join_kernel<T>), grid, dim3(256), 0, current_stream(), p, all, lanes);
    return check_launch();
}

}  // namespace

static size_t need_of(const Plan &plan, int N, int kv_heads, int D)
{
    if (plan.shares == 1) return 0;
    const size_t rows = (size_t)plan.shares * N * kv_heads * plan.rows;
    return align_up(rows * part_row(D) * sizeof(float), 256) + rows * sizeof(PartSum);
}

// The wider blocks have no registers left for a mask by rows: half as wide ones in their place, with the same shares.
static bool for_mask_by_rows(Plan &plan, int N, int kv_heads)
{
    if (plan.block != 256) return true;
    plan.block = 128, plan.tiles = (plan.rows - 1) / 128 + 1;
    return one_launch((double)N * kv_heads * plan.tiles * plan.shares, 256);
}

extern "C" int sq_tune_cross_attention_plan(int N, int Lq, int Lk, int heads, int kv_heads, int D, int dtype, int mask_by_queries, int *plan)
{
    if (!plan || N <= 0 || Lq <= 0 || Lk < 0 || heads <= 0 || kv_heads <= 0 || heads % kv_heads || D <= 0 || D > 256) return SQ_ERR_SHAPE;
    Plan of{};
    if (!plan_of(N, Lq, Lk, heads, kv_heads, D, dtype, of) || (mask_by_queries && !for_mask_by_rows(of, N, kv_heads))) return SQ_ERR_UNSUPPORTED;
    plan[0] = of.block, plan[1] = of.shares, plan[2] = of.share;
    return SQ_OK;
}

size_t cross_attention_workspace_bytes(int N, int Lq, int Lk, int heads, int kv_heads, int D, int dtype)
{
    Plan plan{};
    return plan_of(N, Lq, Lk, heads, kv_heads, D, dtype, plan) ? need_of(plan, N, kv_heads, D) : 0;
}

int cross_attention(const CrossArgs &a, size_t workspace_bytes)
{
    Plan plan{};
    if (!plan_of(a.N, a.Lq, a.Lk, a.heads, a.kv_heads, a.D, a.dtype, plan)) return SQ_ERR_UNSUPPORTED;
    if (!enough_workspace(need_of(plan, a.N, a.kv_heads, a.D), a.workspace, workspace_bytes)) return SQ_ERR_WORKSPACE;
    if (a.mask && a.mask_row && !for_mask_by_rows(plan, a.N, a.kv_heads)) return SQ_ERR_UNSUPPORTED;
    CrossParams p{};
    p.a = a;
    p.group = a.heads / a.kv_heads;
    p.rows = plan.rows, p.tiles = plan.tiles, p.share = plan.share, p.shares = plan.shares;
    p.c = a.scale == 0 ? 1.f : std::fabs(a.scale) * kLog2e;
    p.keep = a.scale == 0 ? 0 : 0xffffffffu;
    p.flip = a.scale < 0 ? (a.dtype == SQ_F32 ? 0x80000000u : 0x80008000u) : 0;
    p.part_ld = part_row(a.D);
    p.part_o = (float *)a.workspace;
    p.part_ml = (PartSum *)((char *)a.workspace + align_up((size_t)p.shares * a.N * a.kv_heads * p.rows * p.part_ld * sizeof(float), 256));
    return a.dtype == SQ_F32 ? run<float>(p, plan.block) : run<bf16_t>(p, plan.block);
}

bool cross_attention_register_kernels()
{
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, (const void *)cross_tile_kernel<bf16_t, 64, 1, true>) == hipSuccess;
}

}  // namespace sq
