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

// The heads of the queries that share a head of the states are further rows to it: row r is query r / group, head r % group of them.
struct CrossParams {
    CrossArgs a;
    int group, rows;        // rows of an image and head of the states
    int tiles;              // of rows
    int share, shares;      // of the states, in tiles of them
    float c;                // |scale| log2 e, or 1 where the scale is 0
    uint32_t keep, flip;    // bits of q that stay (none where the scale is 0), sign bits that turn q into -q where it is below 0
    float *part_o;          // [share][image, head, row][part_ld] and
    float2 *part_ml;        // [share][image, head, row] what the exponents were taken against and their sum, where shares > 1
    int part_ld;
};

template <typename T> __device__ __forceinline__ u32x4_t piece_of(const T *row, int d, int D, bool there)
{
    constexpr int n = 16 / (int)sizeof(T);
    if (!there || d >= D) return u32x4_t{};
    if (d + n <= D) return __builtin_bit_cast(u32x4_t, load_n<n>(row + d));
    Vec<T, n> v;
#pragma unroll
    for (int i = 0; i < n; ++i) v.v[i] = d + i < D ? row[d + i] : T(0);
    return __builtin_bit_cast(u32x4_t, v);
}

__device__ __forceinline__ float other_half(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? r[0] : r[1]);
}
__device__ __forceinline__ uint32_t bf16_two(float a, float b)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
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

// ---- tiles ------------------------------------------------------------------------------------------------------------
// A workgroup of four wavefronts takes 128 rows, each wavefront 32, and goes over the states in tiles of KT, two images of which lie in
// LDS.  Scores are formed transposed, states x rows, so that a lane holds scores of one row alone (lane % 32): its maximum and sum are sums
// within the lane and over the two halves.  The scores' places in the accumulators are, as they are, the second operand of the
// product with the transposed values: lane half h has states 8 i + 4 h to 8 i + 4 h + 3, and the values' lanes take the same ones.
template <typename T> struct Tile;
template <> struct Tile<bf16_t> {
    static constexpr int KT = 64;
    // 16-byte pieces from one state to the next: keys in odd steps (a column of pieces covers all banks), values in steps of 4 modulo 8
    // (the four states of a transposed read lie apart)
    static constexpr int key_step(int DP) { return DP / 8 + 1; }
    static constexpr int value_step(int DP) { return DP / 8 % 8 == 4 ? DP / 8 : DP / 8 + 4; }
};
template <> struct Tile<float> {
    static constexpr int KT = 32;
    static constexpr int key_step(int DP) { return DP / 4 + 1; }
    static constexpr int value_step(int DP) { return DP / 4; }
};

template <typename T, int DP> __global__ __launch_bounds__(256) void cross_tile_kernel(CrossParams p)
{
    constexpr bool kF32 = sizeof(T) == 4;
    constexpr int KT = Tile<T>::KT, n = 16 / (int)sizeof(T), P = DP / n, SK = Tile<T>::key_step(DP), SV = Tile<T>::value_step(DP);
    constexpr int kImage = KT * (SK + SV), NP = KT * P / 256 ? KT * P / 256 : 1, KB = KT / 32, DB = DP / 32;
    static_assert(KT * P % 256 == 0, "whole pieces per thread");
    __shared__ u32x4_t lds[2 * kImage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    // neighbouring workgroups of an XCD take the row tiles of one image and head
    const unsigned all = gridDim.x, xcd = blockIdx.x & 7;
    const unsigned b = (xcd < all % 8 ? xcd * (all / 8 + 1) : all % 8 * (all / 8 + 1) + (xcd - all % 8) * (all / 8)) + (blockIdx.x >> 3);
    const unsigned share = b % (unsigned)p.shares, bt = b / (unsigned)p.shares;
    const int tile = (int)(bt % (unsigned)p.tiles), ih = (int)(bt / (unsigned)p.tiles), image = ih / p.a.kv_heads, head = ih - image * p.a.kv_heads;
    const int D = p.a.D;
    const int len = p.a.lengths ? min(max(p.a.lengths[image], 0), p.a.Lk) : p.a.Lk;
    const int first = min((long long)share * p.share * KT, (long long)len), end = min(((long long)share + 1) * p.share * KT, (long long)len);

    const int row = tile * 128 + wave * 32 + (lane & 31);
    const T *qrow;
    const uint8_t *mask;
    T *out;
    row_of<T>(p, image, head, min(row, p.rows - 1), qrow, mask, out);
    u32x4_t q[P / 2];
#pragma unroll
    for (int t = 0; t < P / 2; ++t) {
        q[t] = piece_of(qrow, (2 * t + half) * n, D, true);
#pragma unroll
        for (int e = 0; e < 4; ++e) q[t][e] = (q[t][e] & p.keep) ^ p.flip;
    }
    const T *const k0 = (const T *)p.a.k + (long long)image * p.a.Lk * p.a.ld_k + head * D, *const v0 = (const T *)p.a.v + (long long)image * p.a.Lk * p.a.ld_v + head * D;
    u32x4_t nk[NP], nv[NP];
    auto fetch = [&](int at) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int e = threadIdx.x + i * 256, j = at + e / P, d = e % P * n;
            nk[i] = piece_of(k0 + j * p.a.ld_k, d, D, j < end);
            nv[i] = piece_of(v0 + j * p.a.ld_v, d, D, j < end);
        }
    };
    auto store = [&](u32x4_t *to) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int e = threadIdx.x + i * 256, j = e / P, d = e % P;
            to[j * SK + d] = nk[i];
            to[KT * SK + j * SV + d] = nv[i];
        }
    };
    f32x16_t o[DB] = {};
    float base = -HUGE_VALF, total = 0.f;      // what the exponents were taken against, in base two
    if (first < end) {
        fetch(first);
        store(lds);
    }
    __syncthreads();
    int img = 0;
    for (int at = first; at < end; at += KT) {
        const bool more = at + KT < end;
        if (more) fetch(at + KT);
        const u32x4_t *const keys = lds + img * kImage, *const values = keys + KT * SK;
        f32x16_t s[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            s[kb] = f32x16_t{};
#pragma unroll
            for (int t = 0; t < P / 2; ++t) {
                const u32x4_t k = keys[(kb * 32 + (lane & 31)) * SK + 2 * t + half];
                if constexpr (kF32) {
                    const f32x4_t kf = __builtin_bit_cast(f32x4_t, k), qf = __builtin_bit_cast(f32x4_t, q[t]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qf[e], s[kb], 0, 0, 0);
                } else {
                    s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q[t]), s[kb], 0, 0, 0);
                }
            }
        }
        if (mask || at + KT > end) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const int j = at + kb * 32 + i * 2 + half * 4;
                    Vec<uint8_t, 4> m = {{1, 1, 1, 1}};
                    if (mask) {
                        if (j + 4 <= end) m = load_n<4>(mask + j);
                        else
#pragma unroll
                            for (int e = 0; e < 4; ++e) m.v[e] = j + e < end ? mask[j + e] : 0;
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[kb][i + e] = j + e < end && m.v[e] ? s[kb][i + e] : -HUGE_VALF;
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
        top = fmaxf(top, other_half(top));
        top *= p.c;
        if (__any(top > base)) {
            const float raised = fmaxf(base, top), shrink = base == -HUGE_VALF ? 0.f : __builtin_amdgcn_exp2f(base - raised);
            total *= shrink;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= shrink;
            base = raised;
        }
        const float mc = base == -HUGE_VALF ? 0.f : base;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[kb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][i], p.c, -mc));
                total += s[kb][i];
            }
        if constexpr (kF32) {
            const float *const vf = (const float *)values;
#pragma unroll
            for (int i = 0; i < 16; ++i)
#pragma unroll
                for (int d = 0; d < DB; ++d)
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[(i / 4 * 8 + half * 4 + i % 4) * SV * 4 + d * 32 + (lane & 31)], s[0][i], o[d], 0, 0, 0);
        } else {
            typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
#pragma unroll
            for (int t = 0; t < KT / 16; ++t) {
                u32x4_t pt;
#pragma unroll
                for (int e = 0; e < 4; ++e) pt[e] = bf16_two(s[t / 2][t % 2 * 8 + 2 * e], s[t / 2][t % 2 * 8 + 2 * e + 1]);
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    // sixteen lanes read four states of sixteen neighbouring values, a lane four of them, and get a column each
                    const char *const from = (const char *)(values + (t * 16 + half * 4 + (lane & 15) / 4) * SV) + d * 64 + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
                    const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)from), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(from + 8 * SV * 16));
                    const auto vt = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vt), __builtin_bit_cast(bf16x8, pt), o[d], 0, 0, 0);
                }
            }
        }
        img ^= 1;
        if (more) store(lds + img * kImage);
        __syncthreads();
    }
    total += other_half(total);
    if (p.a.mask) {
        // A masked value that is not finite has gone into the sums as 0 * it: such rows are made again from the states they see.
        bool odd = false;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) odd |= !__builtin_isfinite(o[d][i]);
        const uint64_t lanes = __ballot(odd);
        uint32_t again = (uint32_t)lanes | (uint32_t)(lanes >> 32);
        float *const area = (float *)lds + wave * DP;       // a row's sums, in the wavefront's own part
        static_assert(4 * DP * 4 <= 2 * kImage * 16, "the areas fit");
        while (again) {
            const int which = __builtin_ctz(again);
            again &= again - 1;
            const T *qr;
            const uint8_t *mr;
            T *unused;
            row_of<T>(p, image, head, min(tile * 128 + wave * 32 + which, p.rows - 1), qr, mr, unused);
            constexpr int E = (DP + 63) / 64;
            float qv[E], sum[E] = {}, m = -HUGE_VALF, l = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) qv[e] = lane + 64 * e < D ? (p.keep ? to_f32(qr[lane + 64 * e]) : 0.f) * (p.flip ? -1.f : 1.f) : 0.f;
            for (int j = first; j < end; ++j) {
                if (!mr[j]) continue;
                float dot = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (lane + 64 * e < D) dot = __builtin_fmaf(qv[e], to_f32(k0[j * p.a.ld_k + lane + 64 * e]), dot);
                for (int x = 32; x; x >>= 1) dot += __shfl_xor(dot, x);
                const float up = fmaxf(m, dot * p.c), upc = up == -HUGE_VALF ? 0.f : up;
                const float shrink = m == -HUGE_VALF ? 0.f : __builtin_amdgcn_exp2f(m - up), w = __builtin_amdgcn_exp2f(__builtin_fmaf(dot, p.c, -upc));
                m = up;
                l = l * shrink + w;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (lane + 64 * e < D) sum[e] = sum[e] * shrink + w * to_f32(v0[j * p.a.ld_v + lane + 64 * e]);
            }
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (lane + 64 * e < DP) area[lane + 64 * e] = sum[e];
            __builtin_amdgcn_wave_barrier();
            if ((lane & 31) == which) {
                base = m, total = l;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] = area[d * 32 + i / 4 * 8 + half * 4 + i % 4];
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
    if (row >= p.rows) return;
    if (p.shares > 1) {
        const long long at = ((long long)share * p.a.N * p.a.kv_heads + ih) * p.rows + row;
        if (half == 0) p.part_ml[at] = float2{base, total};
        if (total == 0.f) return;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int at_d = d * 32 + i * 2 + half * 4;
                if (at_d < p.part_ld) *(f32x4_t *)(p.part_o + at * p.part_ld + at_d) = f32x4_t{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
            }
        return;
    }
    const float inverse = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int at_d = d * 32 + i * 2 + half * 4;
            Vec<T, 4> v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v.v[e] = from_f32<T>(total == 0.f ? 0.f : o[d][i + e] * inverse);
            if (at_d + 4 <= D) {
                __builtin_memcpy(out + at_d, &v, sizeof(v));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (at_d + e < D) out[at_d + e] = v.v[e];
            }
        }
}

// Four neighbouring results of a row from the shares' sums.
template <typename T> __global__ __launch_bounds__(256) void cross_join_kernel(CrossParams p, long long all)
{
    const int quads = p.part_ld / 4;
    const long long e = blockIdx.x * 256ll + threadIdx.x, at = e / quads;
    if (at >= all) return;
    const int d = (int)(e - at * quads) * 4;
    float most = -HUGE_VALF;
    for (int s = 0; s < p.shares; ++s) {
        const float2 ml = p.part_ml[s * all + at];
        if (ml.y != 0.f) most = fmaxf(most, ml.x);
    }
    float total = 0.f;
    f32x4_t sum = {};
    for (int s = 0; s < p.shares; ++s) {
        const float2 ml = p.part_ml[s * all + at];
        if (ml.y == 0.f) continue;
        const float w = ml.x == most ? 1.f : __builtin_amdgcn_exp2f(ml.x - most);
        total += w * ml.y;
        sum += w * *(const f32x4_t *)(p.part_o + (s * all + at) * p.part_ld + d);
    }
    const int ih = (int)(at / p.rows), image = ih / p.a.kv_heads;
    const T *q;
    const uint8_t *mask;
    T *out;
    row_of<T>(p, image, ih - image * p.a.kv_heads, (int)(at - (long long)ih * p.rows), q, mask, out);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (d + i < p.a.D) out[d + i] = from_f32<T>(total == 0.f ? 0.f : sum[i] / total);
}

// Widths the tiles are made for.
int padded(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : D <= 96 ? 96 : D <= 128 ? 128 : D <= 160 ? 160 : 256; }
int tile_keys(int dtype) { return dtype == SQ_F32 ? 32 : 64; }

// How the states are shared out: in as many shares as it takes to fill the chip with workgroups, none shorter than four tiles.
struct Plan { int rows, tiles, share, shares; };
bool plan_of(int N, int Lq, int Lk, int heads, int kv_heads, int dtype, Plan &plan)
{
    const long long rows = (long long)Lq * (heads / kv_heads);
    if (rows > 1 << 30 || Lk > 1 << 30) return false;
    plan.rows = (int)rows;
    plan.tiles = (int)((rows - 1) / 128 + 1);
    const double blocks = (double)N * kv_heads * plan.tiles;
    const int key_tiles = (Lk - 1) / tile_keys(dtype) + 1;
    int shares = blocks >= 256 ? 1 : std::min({(int)(512 / blocks), key_tiles / 4, 64});
    shares = std::max(shares, 1);
    plan.share = (key_tiles - 1) / shares + 1;
    plan.shares = (key_tiles - 1) / plan.share + 1;
    return one_launch(blocks * plan.shares, 256);
}
int part_row(int D) { return (D + 3) / 4 * 4; }

template <typename T, int DP> int launch_tile(const CrossParams &p)
{
    const LaunchScope prof("cross_tile", cross_flops(p.a), cross_bytes(p.a));
    hipLaunchKernelGGL((cross_tile_kernel<T, DP>), dim3((unsigned)(p.a.N * p.a.kv_heads) * p.tiles * p.shares), dim3(256), 0, current_stream(), p);
    return check_launch();
}
template <typename T> int by_width(const CrossParams &p)
{
    switch (padded(p.a.D)) {
        case 32: return launch_tile<T, 32>(p);
        case 64: return launch_tile<T, 64>(p);
        case 96: return launch_tile<T, 96>(p);
        case 128: return launch_tile<T, 128>(p);
        case 160: return launch_tile<T, 160>(p);
        default: return launch_tile<T, 256>(p);
    }
}
template <typename T> int run(const CrossParams &p)
{
    if (const int rc = by_width<T>(p)) return rc;
    if (p.shares == 1) return SQ_OK;
    const long long all = (long long)p.a.N * p.a.kv_heads * p.rows;
    const LaunchScope prof("cross_join", 0, 0);
    hipLaunchKernelGGL((cross_join_kernel<T>), dim3((unsigned)((all * (p.part_ld / 4) - 1) / 256 + 1)), dim3(256), 0, current_stream(), p, all);
    return check_launch();
}

}  // namespace

size_t cross_attention_workspace_bytes(int N, int Lq, int Lk, int heads, int kv_heads, int D, int dtype)
{
    Plan plan;
    if (!plan_of(N, Lq, Lk, heads, kv_heads, dtype, plan) || plan.shares == 1) return 0;
    const size_t rows = (size_t)plan.shares * N * kv_heads * plan.rows;
    return align_up(rows * part_row(D) * sizeof(float), 256) + rows * sizeof(float2);
}

int cross_attention(const CrossArgs &a)
{
    Plan plan;
    if (!plan_of(a.N, a.Lq, a.Lk, a.heads, a.kv_heads, a.dtype, plan)) return SQ_ERR_UNSUPPORTED;
    CrossParams p{};
    p.a = a;
    p.group = a.heads / a.kv_heads;
    p.rows = plan.rows, p.tiles = plan.tiles, p.share = plan.share, p.shares = plan.shares;
    p.c = a.scale == 0 ? 1.f : std::fabs(a.scale) * kLog2e;
    p.keep = a.scale == 0 ? 0 : 0xffffffffu;
    p.flip = a.scale < 0 ? (a.dtype == SQ_F32 ? 0x80000000u : 0x80008000u) : 0;
    p.part_ld = part_row(a.D);
    p.part_o = (float *)a.workspace;
    p.part_ml = (float2 *)((char *)a.workspace + align_up((size_t)p.shares * a.N * a.kv_heads * p.rows * p.part_ld * sizeof(float), 256));
    return a.dtype == SQ_F32 ? run<float>(p) : run<bf16_t>(p);
}

bool cross_attention_register_kernels()
{
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, (const void *)cross_tile_kernel<bf16_t, 64>) == hipSuccess;
}

}  // namespace sq
