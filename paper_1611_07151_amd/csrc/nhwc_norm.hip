// Group norm with an activation on channels-last maps.  Bound by memory: x read once, y written once.
//
// A workgroup owns the pixels of one image (or a chunk of them) in a block of neighbouring layers: some whole groups, or a part
// of one group that is wider than a workgroup.  A thread owns one vector of VB bytes of a row, the same in every row it
// takes, so its layers' groups, gamma and beta are fixed.  Means are summed first and the squares of the deviations from them
// second, from registers, so that nothing cancels and x is read once.
// Where such a block of an image fits one workgroup's registers the same launch also writes the result (group_norm_fused).
// Else a launch for (mean, sum of squared deviations) per chunk, which are combined as
//   mean = sum n_i mean_i / m,  M2 = sum M2_i + n_i (mean_i - mean)^2,
// and one for the result, which reads x again (from the last-level cache where it fits its 256 MB).
// Measured: 13 x 13 x 512 fp32 5.2 us, 16 x 27 x 27 x 384 bf16 10.2 us (launch and two sums across a workgroup), 64 x 55 x 55 x 256
// fp32 105 us (3.8 TB/s) in one launch; 64 x 111 x 111 x 96 bf16 with SiLU 106 us in two (4.3 TB/s for what they move, 2.9 for x and
// the result once; 81 with the same map again, part of which then lies in the memory-side cache, in one launch 126: one workgroup a
// compute unit, whose loads, arithmetic and stores follow each other).
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
    int act;
    // blocks of layers: `width` layers each, holding `groups` whole groups, or (groups == 1) `parts` of them make one group
    int width, groups, parts, blocks;
    int chunks;             // of an image's pixels
    long long chunk;        // pixels in each (the last one may have fewer)
    float *partial;         // [N][G][chunks * parts][mean, M2]
    float *stats;           // [N][G][mean, 1 / sqrt(var + eps)], or nullptr: the last launch combines the chunks itself
};

constexpr int kMaxThreads = 1024;

// n values at any address of a T, held as they lie in memory
template <typename T, int VB> struct Vector {
    static constexpr int n = VB / (int)sizeof(T), words = VB < 4 ? 1 : VB / 4;
    typedef uint32_t W __attribute__((ext_vector_type(words)));
    typedef W WU __attribute__((aligned(sizeof(T))));
    W w;
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (VB == 2) w[0] = *(const uint16_t *)p;
        else w = *(const WU *)p;
    }
    __device__ __forceinline__ void store(T *p) const
    {
        if constexpr (VB == 2) *(uint16_t *)p = (uint16_t)w[0];
        else *(WU *)p = w;
    }
    __device__ __forceinline__ float get(int i) const
    {
        const uint32_t u = w[sizeof(T) == 4 ? i : i / 2];
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, u);
        else return __builtin_bit_cast(float, i & 1 ? u & 0xffff0000u : u << 16);
    }
    __device__ __forceinline__ void set(const float (&v)[n])
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < n; ++i) w[i] = __builtin_bit_cast(uint32_t, v[i]);
        } else if constexpr (n == 1) {
            w[0] = from_f32<bf16_t>(v[0]);
        } else {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int i = 0; i < n; i += 2) {
                const bf16x2 h = {(__bf16)v[i], (__bf16)v[i + 1]};
                w[i / 2] = __builtin_bit_cast(uint32_t, h);
            }
        }
    }
};

// Where a thread stands: its vector of the row, its row of a turn, its group within the block.
struct Place {
    int image, first, width, vectors, rows, vector, row;
    long long begin, end;
    int chunk, part;
    bool live;
    template <int n> __device__ __forceinline__ void set(const NormArgs &p, unsigned b, int threads)
    {
        chunk = (int)(b % (unsigned)p.chunks);
        b /= (unsigned)p.chunks;
        const int block = (int)(b % (unsigned)p.blocks);
        image = (int)(b / (unsigned)p.blocks);
        part = block % p.parts;
        const int cg = p.C / p.G;
        first = p.parts > 1 ? block / p.parts * cg + part * p.width : block * p.width;
        width = p.parts > 1 ? min(p.width, cg - part * p.width) : p.width;
        vectors = width / n;
        rows = threads / vectors;
        vector = threadIdx.x % vectors;
        row = threadIdx.x / vectors;
        live = row < rows;
        if (!live) row = 0;     // threads beyond the last whole row repeat the first one's loads and count nothing
        begin = chunk * p.chunk;
        end = min(begin + p.chunk, p.HW);
    }
};

// The rows of a turn: K times at.rows of the `left` ones.  All but one of the K tests are the same for the whole workgroup.
template <int K> struct Turn {
    int whole;
    bool last;
    __device__ __forceinline__ Turn(const Place &at, long long left)
    {
        whole = (int)min(left / at.rows, (long long)K);
        last = whole < K && at.live && at.row < left - (long long)whole * at.rows;
    }
    __device__ __forceinline__ bool has(int k) const { return k < whole || (k == whole && last); }
};

constexpr int kMostGroups = 256;     // of a block

template <int n> __device__ __forceinline__ void load_floats(const float *p, float (&v)[n]) { __builtin_memcpy(v, p, sizeof(v)); }
template <int n> __device__ __forceinline__ void affine(const NormArgs &p, int c, float (&gamma)[n], float (&beta)[n])
{
#pragma unroll
    for (int i = 0; i < n; ++i) {
        gamma[i] = 1.f;
        beta[i] = 0.f;
    }
    if (p.gamma) load_floats(p.gamma + c, gamma);
    if (p.beta) load_floats(p.beta + c, beta);
}

// f(i, g): g = the group, counted from the block's first, of a thread's i-th layer
template <int n, typename F> __device__ __forceinline__ void each_group(int layer, int cg, F f)
{
    int g = layer / cg, in = layer - g * cg;
#pragma unroll
    for (int i = 0; i < n; ++i) {
        f(i, g);
        if (++in == cg) {
            in = 0;
            ++g;
        }
    }
}

// Teams of 2^shift neighbouring threads (of one wavefront) per group, where the workgroup has as many, with work for each.
__device__ __forceinline__ int team_shift(int groups, int work)
{
    int shift = 0;
    while (shift < 6 && (groups << (shift + 1)) <= (int)blockDim.x && (1 << shift) < work) ++shift;
    return shift;
}
// the sum over a team, whose threads are all here: within 16 lanes by the operand's own lane moves, beyond by exchanging rows of
// lanes (through LDS each of the six steps would wait for it: 16 x 27 x 27 x 384 bfloat16 10.8 us instead of 10.2)
template <int control> __device__ __forceinline__ float plus_moved(float v)
{
    const int u = __builtin_bit_cast(int, v);
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(u, u, control, 0xf, 0xf, false));
}
__device__ __forceinline__ float team_sum(float v, int shift)
{
    if (shift > 0) v = plus_moved<0xb1>(v);        // lane ^ 1
    if (shift > 1) v = plus_moved<0x4e>(v);        // lane ^ 2
    if (shift > 2) v = plus_moved<0x141>(v);       // lane ^ 7: the other four of eight, which hold one sum by now
    if (shift > 3) v = plus_moved<0x140>(v);       // lane ^ 15
    if (shift > 4) {
        const uint32_t u = __builtin_bit_cast(uint32_t, v);
        const auto both = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        const uint32_t a = both[0], b = both[1];
        v = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
    }
    if (shift > 5) {
        const uint32_t u = __builtin_bit_cast(uint32_t, v);
        const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        const uint32_t a = both[0], b = both[1];
        v = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
    }
    return v;
}

// Sums of v[i], which belong to a thread's n layers, over the threads and layers of each group of the block, in v[i].
// A value per vector where its layers are of one group, per layer else.  First over the rows a wavefront holds, lane to
// lane (narrow rows: lanes a row apart hold the same vector), then through LDS over wavefronts (or rows) and layers, each
// group by a team of threads.
template <int n> __device__ __forceinline__ void group_sums(const NormArgs &p, const Place &at, float (&v)[n], float *lds, float *sums)
{
    const int cg = p.parts > 1 ? at.width : p.C / p.G, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, lane = threadIdx.x & 63;
    const bool one = n == 1 || p.groups == 1 || cg % n == 0;
    if (one) {
#pragma unroll
        for (int i = 1; i < n; ++i) v[0] += v[i];
    }
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = at.live ? v[i] : 0.f;
    __syncthreads();        // the areas' last readers are done
    if (p.groups == 1) {
        float all = team_sum(v[0], 6);
        if (lane == 0) lds[wave] = all;
        __syncthreads();
        all = lds[0];
        for (int w = 1; w < waves; ++w) all += lds[w];
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = all;
        return;
    }
    const int items = one ? at.vectors : at.width;      // per row
    const bool narrow = at.vectors <= 32;
    if (narrow)
        for (int d = at.vectors; d < 64; d <<= 1) {
#pragma unroll
            for (int i = 0; i < n; ++i)
                if (i == 0 || !one) {
                    const float other = __shfl_down(v[i], d);
                    v[i] += lane + d < 64 ? other : 0.f;
                }
        }
    const int parts = narrow ? waves : at.rows;
    if (narrow ? lane < at.vectors : at.live) {
        float *const mine = lds + (narrow ? wave : at.row) * items + at.vector * (one ? 1 : n);
        mine[0] = v[0];
        if (!one)
#pragma unroll
            for (int i = 1; i < n; ++i) mine[i] = v[i];
    }
    __syncthreads();
    const int each = items / p.groups, shift = team_shift(p.groups, each), member = threadIdx.x & ((1 << shift) - 1);
    for (int g = threadIdx.x >> shift; g < p.groups; g += blockDim.x >> shift) {
        float s = 0.f;
        for (int m = member; m < each; m += 1 << shift)
            for (int r = 0; r < parts; ++r) s += lds[r * items + g * each + m];
        s = team_sum(s, shift);
        if (member == 0) sums[g] = s;
    }
    __syncthreads();
    each_group<n>(at.vector * n, cg, [&](int i, int g) { v[i] = sums[g]; });
}

// scale[i] = gamma / sqrt(var + eps)
template <int ACT, typename T, int VB, int n>
__device__ __forceinline__ void normalise(Vector<T, VB> &x, const float (&mean)[n], const float (&scale)[n], const float (&beta)[n])
{
    float v[n];
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = activate<ACT>(__builtin_fmaf(x.get(i) - mean[i], scale[i], beta[i]));
    x.set(v);
}

template <typename F> __device__ __forceinline__ void by_act(int act, F f)
{
    switch (act) {      // the same for the whole launch
        case SQ_ACT_RELU: f(std::integral_constant<int, SQ_ACT_RELU>{}); break;
        case SQ_ACT_SILU: f(std::integral_constant<int, SQ_ACT_SILU>{}); break;
        case SQ_ACT_GELU: f(std::integral_constant<int, SQ_ACT_GELU>{}); break;
        default: f(std::integral_constant<int, SQ_ACT_NONE>{});
    }
}

// Neighbouring blocks of an image share cache lines: they go to one XCD.
__device__ __forceinline__ unsigned on_one_xcd(unsigned b, unsigned total)
{
    const unsigned q = total >> 3, rest = total & 7, xcd = b & 7;
    return (xcd < rest ? xcd * (q + 1) : rest * (q + 1) + (xcd - rest) * q) + (b >> 3);
}

template <typename T, int VB, int K> __global__ __launch_bounds__(kMaxThreads) void group_norm_fused(NormArgs p)
{
    constexpr int n = Vector<T, VB>::n;
    __shared__ float lds[kMaxThreads * n], sums[kMostGroups];
    Place at;
    at.set<n>(p, on_one_xcd(blockIdx.x, gridDim.x), blockDim.x);
    const Turn<K> turn(at, p.HW);
    const int c = at.first + at.vector * n;
    const T *in = (const T *)p.in + ((long long)at.image * p.HW + at.row) * p.ld_in + c;
    Vector<T, VB> x[K];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (turn.has(k)) x[k].load(in + (long long)k * at.rows * p.ld_in);
    float gamma[n], beta[n];
    affine(p, c, gamma, beta);
    float mean[n] = {}, scale[n] = {};
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (turn.has(k))
#pragma unroll
            for (int i = 0; i < n; ++i) mean[i] += x[k].get(i);
    const float count = (float)p.HW * (float)(p.C / p.G);
    group_sums(p, at, mean, lds, sums);
#pragma unroll
    for (int i = 0; i < n; ++i) mean[i] /= count;
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (turn.has(k))
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const float d = x[k].get(i) - mean[i];
                scale[i] = __builtin_fmaf(d, d, scale[i]);
            }
    group_sums(p, at, scale, lds, sums);
#pragma unroll
    for (int i = 0; i < n; ++i) scale[i] = gamma[i] * (1.f / sqrtf(scale[i] / count + p.eps));
    if (!at.live) return;
    T *out = (T *)p.out + ((long long)at.image * p.HW + at.row) * p.ld_out + c;
    by_act(p.act, [&](auto act) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (turn.has(k)) {
                normalise<decltype(act)::value>(x[k], mean, scale, beta);
                x[k].store(out + (long long)k * at.rows * p.ld_out);
            }
    });
}

// A thread's own mean and M2 of every layer it holds, K rows at a time and these combined as they come (no thread waits for
// another inside the loop); then those of the threads.
template <typename T, int VB, int K> __global__ __launch_bounds__(256) void group_norm_moments(NormArgs p)
{
    constexpr int n = Vector<T, VB>::n;
    __shared__ float lds[256 * n], sums[kMostGroups];
    Place at;
    at.set<n>(p, blockIdx.x, 256);
    const int c = at.first + at.vector * n;
    const T *in = (const T *)p.in + ((long long)at.image * p.HW + at.begin + at.row) * p.ld_in + c;
    float mean[n] = {}, m2[n] = {}, count = 0.f;
    const long long step = (long long)at.rows * K;
    // full: all K rows, with no test between the loads and their use; first: nothing to combine them with (as an empty count it would be
    // mean^2 * 0, and the square may overflow)
    auto take = [&](auto full, auto first, const Turn<K> &turn) {
        constexpr bool kFull = decltype(full)::value, kFirst = decltype(first)::value;
        Vector<T, VB> x[K];
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (kFull || turn.has(k)) x[k].load(in + (long long)k * at.rows * p.ld_in);
        const int rows = kFull ? K : turn.whole + (turn.last ? 1 : 0);
        if (!rows) return;
        const float here = (float)rows, each = 1.f / here, both = count + here, part = here / both, cross = count * part;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            float s = 0.f, q = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (kFull || turn.has(k)) s += x[k].get(i);
            s *= each;
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (kFull || turn.has(k)) {
                    const float d = x[k].get(i) - s;
                    q = __builtin_fmaf(d, d, q);
                }
            if constexpr (kFirst) {
                mean[i] = s;
                m2[i] = q;
            } else {
                const float d = s - mean[i];
                mean[i] = __builtin_fmaf(d, part, mean[i]);
                m2[i] += q + d * d * cross;
            }
        }
        count = both;
    };
    long long left = at.end - at.begin;
    if (left < step) {
        take(std::false_type{}, std::true_type{}, Turn<K>(at, left));
    } else {
        take(std::true_type{}, std::true_type{}, Turn<K>(at, left));
        for (left -= step, in += step * p.ld_in; left >= step; left -= step, in += step * p.ld_in) take(std::true_type{}, std::false_type{}, Turn<K>(at, left));
        if (left > 0) take(std::false_type{}, std::false_type{}, Turn<K>(at, left));
    }
    const int cg = p.parts > 1 ? at.width : p.C / p.G;
    const float values = (float)(at.end - at.begin) * (float)cg;
    float middle[n];
#pragma unroll
    for (int i = 0; i < n; ++i) middle[i] = mean[i] * (count / values);
    group_sums(p, at, middle, lds, sums);
#pragma unroll
    for (int i = 0; i < n; ++i) {
        const float dd = count > 0.f ? (mean[i] - middle[i]) * (mean[i] - middle[i]) : 0.f;     // a thread without rows has no mean
        m2[i] += dd * count;
    }
    group_sums(p, at, m2, lds, sums);
    // each group's by the thread of the first row that holds its first layer
    if (at.live && at.row == 0) {
#pragma unroll
        for (int i = 0; i < n; ++i)
            if ((at.vector * n + i) % cg == 0) {
                float *to = p.partial + 2 * (((long long)at.image * p.G + (c + i) / (p.C / p.G)) * p.chunks * p.parts + at.chunk * p.parts + at.part);
                to[0] = middle[i];
                to[1] = m2[i];
            }
    }
}

// Mean and 1 / sqrt(var + eps) of `groups` groups from image and group g0 on, from their chunks, into to[2 g], to[2 g + 1].
__device__ __forceinline__ void combine(const NormArgs &p, long long g0, int groups, float *to)
{
    const int cg = p.C / p.G, total = p.chunks * p.parts, shift = team_shift(groups, total), lane = threadIdx.x & ((1 << shift) - 1);
    const float m = (float)p.HW * (float)cg;
    auto count = [&](int i) {
        const int chunk = p.parts > 1 ? i / p.parts : i;
        return (float)min(p.chunk, p.HW - chunk * p.chunk) * (float)(p.parts > 1 ? min(p.width, cg - (i - chunk * p.parts) * p.width) : cg);
    };
    for (int g = threadIdx.x >> shift; g < groups; g += blockDim.x >> shift) {
        const float2 *from = (const float2 *)p.partial + (g0 + g) * total;
        constexpr int B = 8;        // loads that fly together
        float2 v[B];
        auto load = [&](int i0) {
#pragma unroll
            for (int b = 0; b < B; ++b) v[b] = from[min(i0 + (b << shift), total - 1)];
        };
        load(lane);
        const bool again = total > B << shift;      // else what is loaded is all there is
        auto each = [&](auto f) {
            for (int i0 = lane; i0 < total; i0 += B << shift) {
                if (again) load(i0);
#pragma unroll
                for (int b = 0; b < B; ++b)
                    if (i0 + (b << shift) < total) f(v[b], count(i0 + (b << shift)));
            }
        };
        float s = 0.f, q = 0.f;
        each([&](float2 v, float c) { s += v.x * (c / m); });
        s = team_sum(s, shift);
        each([&](float2 v, float c) { q += v.y + (v.x - s) * (v.x - s) * c; });
        q = team_sum(q, shift);
        if (lane == 0) {
            to[2 * g] = s;
            to[2 * g + 1] = 1.f / sqrtf(q / m + p.eps);
        }
    }
}

// One wavefront per image and group.
__global__ __launch_bounds__(64) void group_norm_combine(NormArgs p)
{
    for (long long g = blockIdx.x; g < (long long)p.N * p.G; g += gridDim.x) combine(p, g, 1, p.stats + 2 * g);
}

template <typename T, int VB, int K> __global__ __launch_bounds__(256) void group_norm_apply(NormArgs p)
{
    constexpr int n = Vector<T, VB>::n;
    __shared__ float stats[2 * kMostGroups];
    Place at;
    at.set<n>(p, gridDim.x - 1 - blockIdx.x, 256);      // the map's end was read last and lies nearest
    const int c = at.first + at.vector * n, cg = p.C / p.G, g0 = at.first / cg;
    const long long group = (long long)at.image * p.G + g0, step = (long long)at.rows * K, pixel = (long long)at.image * p.HW + at.begin + at.row;
    const T *in = (const T *)p.in + pixel * p.ld_in + c;
    T *out = (T *)p.out + pixel * p.ld_out + c;
    long long left = at.end - at.begin;
    Vector<T, VB> x[K];
    if (left >= step) {         // on their way while the statistics are made
#pragma unroll
        for (int k = 0; k < K; ++k) x[k].load(in + (long long)k * at.rows * p.ld_in);
    }
    float mean[n], scale[n], beta[n];
    affine(p, c, scale, beta);
    if (!p.stats) {
        combine(p, group, p.groups, stats);
        __syncthreads();
    }
    if (!at.live) return;
    const float *from = p.stats ? p.stats + 2 * group : stats;
    each_group<n>(p.parts > 1 ? 0 : at.vector * n, p.parts > 1 ? p.C + 1 : cg, [&](int i, int g) {
        mean[i] = from[2 * g];
        scale[i] *= from[2 * g + 1];
    });
    by_act(p.act, [&](auto act) {
        // Whole turns with the next one's loads on their way, and no test between loads, arithmetic and stores: a test per row
        // makes every row wait for the store of the row before (64 x 55 x 55 x 256 bfloat16: 43 us instead of 24).
        if (left >= step) {
            Vector<T, VB> next[K];
            for (;;) {
                left -= step;
                in += step * p.ld_in;
                if (left >= step) {
#pragma unroll
                    for (int k = 0; k < K; ++k) next[k].load(in + (long long)k * at.rows * p.ld_in);
                }
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    normalise<decltype(act)::value>(x[k], mean, scale, beta);
                    x[k].store(out + (long long)k * at.rows * p.ld_out);
                }
                out += step * p.ld_out;
                if (left < step) break;
#pragma unroll
                for (int k = 0; k < K; ++k) x[k] = next[k];
            }
        }
        if (left > 0) {
            const Turn<K> turn(at, left);
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (turn.has(k)) x[k].load(in + (long long)k * at.rows * p.ld_in);
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (turn.has(k)) {
                    normalise<decltype(act)::value>(x[k], mean, scale, beta);
                    x[k].store(out + (long long)k * at.rows * p.ld_out);
                }
        }
    });
}

// How a call is cut up; the same for the size of its scratch and for the call.
struct Plan {
    int vec;                // bytes of a thread's vector
    bool fused, combine;    // combine: by a launch of its own
    int threads, keep;      // fused: workgroup, and bytes a thread keeps at most
    int width, groups, parts, blocks, chunks;
    long long chunk;
};

int vector_bytes(int width, int size)
{
    int n = 16 / size;
    while (width % n) n >>= 1;
    return n * size;
}

// bytes a thread keeps in registers at most: 80 registers, 64 where a vector is one register and its addresses cost as much
constexpr int keep_most(int vec) { return vec == 2 ? 128 : vec == 4 ? 256 : 320; }

// Microseconds of the one launch, from what it measured (1 to 64 maps of 7 x 7 to 111 x 111 pixels, 96 to 512 layers): what a
// workgroup takes by itself (more where its vectors are narrow), or all of them from memory.  Pieces of rows below 64 bytes cost memory, vectors that reach over
// the border of groups cost the sums.
double fused_us(const Plan &q, int N, int cg, long long HW, int size)
{
    const double slab = (double)HW * q.width, each = (size == 2 ? 1.15e-6 : 1.45e-6) * slab * N * q.blocks;
    const int piece = q.blocks > 1 ? q.width * size : 64;
    return 4.5 + std::max(0.2e-3 * slab * (q.vec == 2 ? 2.5 : q.vec == 4 ? 1.3 : 1.0), each * (piece < 16 ? 5.0 : piece < 32 ? 1.35 : piece < 64 ? 1.1 : 1.0) * (q.groups > 1 && cg % (q.vec / size) ? 1.4 : 1.0));
}

Plan make_plan(int N, int C, long long HW, int G, int size)
{
    const int cg = C / G;
    Plan q{};
    q.parts = 1;
    const double values = (double)N * HW * C;
    const double us_chunks = 12.0 + values * (size == 2 ? 0.92e-6 : 1.9e-6);       // the launches that read x twice
    double best = 1e30;
    for (int groups = 1; groups <= std::min(G, kMostGroups); ++groups) {
        if (G % groups) continue;
        Plan f{};
        f.fused = true;
        f.groups = groups;
        f.width = groups * cg;
        f.vec = vector_bytes(f.width, size);
        f.parts = 1;
        f.blocks = G / groups;
        f.chunks = 1;
        f.chunk = HW;
        const int n = f.vec / size;
        const long long vectors = f.width / n;
        if (vectors > kMaxThreads) break;
        // the smallest workgroup whose threads keep 32 bytes each (where they do not fill the chip), else 128, else the most
        bool fits = false;
        for (int keep : {32, 128, keep_most(f.vec)}) {
            if (keep == 32 && (long long)N * f.blocks >= 256) continue;
            f.keep = keep;
            const long long rows = (HW * f.vec + keep - 1) / keep;
            f.threads = (int)std::min<long long>(kMaxThreads, std::max<long long>(64, (rows * vectors + 63) / 64 * 64));
            const long long have = f.threads / vectors;
            fits = have && (HW + have - 1) / have * f.vec <= keep;
            if (fits) break;
        }
        if (!fits) continue;
        const double us = fused_us(f, N, cg, HW, size);
        if (us < best && us < us_chunks) {
            best = us;
            q = f;
        }
    }
    if (q.fused) return q;
    // chunks, 256 threads
    if ((long long)cg * size > 256ll * vector_bytes(cg, size)) {     // a group is wider than a workgroup
        q.vec = vector_bytes(cg, size);
        q.width = 256 * (q.vec / size);
        q.groups = 1;
        q.parts = (cg + q.width - 1) / q.width;
        q.blocks = G * q.parts;
    } else {
        // the widest block of whole groups whose vectors are the widest there are
        for (int groups = 1; groups <= std::min(G, kMostGroups); ++groups) {
            if (G % groups) continue;
            const int vec = vector_bytes(groups * cg, size);
            if ((long long)groups * cg * size > 256ll * vec || vec < q.vec) continue;
            q.vec = vec;
            q.groups = groups;
        }
        q.width = q.groups * cg;
        q.blocks = G / q.groups;
    }
    // whole turns of 64 bytes a thread, and not more workgroups than are there at a time
    const long long rows = 256 / (q.width / (q.vec / size)), turn = rows * (q.vec < 4 ? 16 : 64 / q.vec);
    const long long want = std::max<long long>(1, 1024 / std::max<long long>(1, (long long)N * q.blocks));
    q.chunk = ((HW + want - 1) / want + turn - 1) / turn * turn;
    q.chunks = (int)((HW + q.chunk - 1) / q.chunk);
    // the last launch's workgroups combine the chunks of their groups themselves where these are few
    q.combine = (long long)q.groups * q.chunks * q.parts > 2048;
    return q;
}

template <typename T, int VB, int KEEP> int launch_fused(const NormArgs &p, const Plan &q)
{
    const double values = (double)p.N * p.HW * p.C;
    const LaunchScope prof("group_norm", 10.0 * values, 2.0 * sizeof(T) * values, 0.0);
    hipLaunchKernelGGL((group_norm_fused<T, VB, KEEP / VB>), dim3((unsigned)p.N * q.blocks), dim3(q.threads), 0, current_stream(), p);
    return check_launch();
}

template <typename T, int VB> int launch(const NormArgs &p, const Plan &q)
{
    if constexpr (VB < (int)sizeof(T)) {
        return SQ_ERR_UNSUPPORTED;
    } else {
        if (q.fused) {
            if (q.keep == 32) return launch_fused<T, VB, 32>(p, q);
            if (q.keep == 128) return launch_fused<T, VB, 128>(p, q);
            return launch_fused<T, VB, keep_most(VB)>(p, q);
        }
        const double values = (double)p.N * p.HW * p.C;
        const unsigned grid = (unsigned)p.N * q.blocks * q.chunks;
        {
            const LaunchScope prof("group_norm_moments", 4.0 * values, sizeof(T) * values, 0.0);
            // 128 bytes a thread and turn; 64 where a chunk has no whole such turn, whose rows would each be tested for (5 x 73 x 75 x
            // 104 bfloat16 19.6 -> 18.0 us a call, 1 x 49 x 48 x 240 15.0 -> 14.2)
            constexpr int K = VB == 2 ? 16 : VB == 4 ? 16 : 128 / VB;
            if (VB > 4 && q.chunk < (long long)K * (256 / (q.width / (q.vec / (int)sizeof(T)))))
                hipLaunchKernelGGL((group_norm_moments<T, VB, VB == 2 ? 16 : 64 / VB>), dim3(grid), dim3(256), 0, current_stream(), p);
            else
                hipLaunchKernelGGL((group_norm_moments<T, VB, K>), dim3(grid), dim3(256), 0, current_stream(), p);
        }
        int rc = check_launch();
        if (rc) return rc;
        if (q.combine) {
            const LaunchScope prof("group_norm_combine", 0.0, 8.0 * p.N * p.G * q.chunks * q.parts, 0.0);
            hipLaunchKernelGGL(group_norm_combine, dim3((unsigned)std::min<long long>((long long)p.N * p.G, 1 << 16)), dim3(64), 0, current_stream(), p);
            if ((rc = check_launch())) return rc;
        }
        const LaunchScope prof("group_norm_apply", 6.0 * values, 2.0 * sizeof(T) * values, 0.0);
        hipLaunchKernelGGL((group_norm_apply<T, VB, VB == 2 ? 16 : 64 / VB>), dim3(grid), dim3(256), 0, current_stream(), p);
        return check_launch();
    }
}

template <typename T> int by_vector(const NormArgs &p, const Plan &q)
{
    switch (q.vec) {
        case 16: return launch<T, 16>(p, q);
        case 8: return launch<T, 8>(p, q);
        case 4: return launch<T, 4>(p, q);
        default: return launch<T, 2>(p, q);
    }
}

size_t scratch_bytes(const Plan &q, int N, int G)
{
    return q.fused ? 0 : align_up((size_t)N * G * 8, 256) + (size_t)N * G * q.chunks * q.parts * 8;
}

}  // namespace

bool nhwc_norm_register_kernels()
{
    hipFuncAttributes a;
    return hipFuncGetAttributes(&a, (const void *)group_norm_combine) == hipSuccess;
}

size_t nhwc_group_norm_workspace_bytes(int N, int C, long long HW, int G)
{
    // the type is not known here
    return std::max(scratch_bytes(make_plan(N, C, HW, G, 4), N, G), scratch_bytes(make_plan(N, C, HW, G, 2), N, G));
}

int nhwc_group_norm(const void *in, void *out, int dtype, const float *gamma, const float *beta, int N, int C, long long HW, int G,
                    float eps, int act, long long ld_in, long long ld_out, void *workspace, size_t)
{
    const Plan q = make_plan(N, C, HW, G, dtype == SQ_F32 ? 4 : 2);
    NormArgs p{in, out, gamma, beta, N, C, G, HW, ld_in, ld_out, eps, act, q.width, q.groups, q.parts, q.blocks, q.chunks, q.chunk, nullptr, nullptr};
    p.stats = q.combine ? (float *)workspace : nullptr;
    p.partial = (float *)((char *)workspace + align_up((size_t)N * G * 8, 256));
    const int threads = q.fused ? q.threads : 256, size = dtype == SQ_F32 ? 4 : 2;
    const double each = (double)q.blocks * q.chunks;
    if (!one_launch(each, threads)) return SQ_ERR_UNSUPPORTED;
    const int most = images_in_one_launch(N, each, threads);
    for (long long n = 0; n < N; n += most) {       // one after the other, with the same scratch
        p.N = (int)std::min<long long>(most, N - n);
        if (const int rc = size == 4 ? by_vector<float>(p, q) : by_vector<bf16_t>(p, q)) return rc;
        p.in = (const char *)p.in + (long long)p.N * HW * ld_in * size;
        p.out = (char *)p.out + (long long)p.N * HW * ld_out * size;
    }
    return SQ_OK;
}

}  // namespace sq
