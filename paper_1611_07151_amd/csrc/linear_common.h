// Shared by the matrix products of rows: results with bias, activation and residual, the order of tiles.
#pragma once

#include "nhwc_common.h"

namespace sq {
namespace {

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

// The first `have` of n neighbouring values, more than none; the others are the last of them again.  (All loads are on their way
// together: one behind the other, each under its own condition, they cost a memory latency apiece.)
template <int n, typename T> __device__ __forceinline__ Vec<T, n> load_some(const T *p, int have)
{
    if (have >= n) return load_n<n>(p);
    Vec<T, n> r;
#pragma unroll
    for (int i = 0; i < n; ++i) r.v[i] = p[min(i, have - 1)];
    return r;
}
template <int n, typename T> __device__ __forceinline__ void store_some(T *p, const Vec<T, n> &v, int have)
{
    if (have >= n) {
        __builtin_memcpy(p, &v, sizeof(v));
        return;
    }
#pragma unroll
    for (int i = 0; i < n; ++i)
        if (i < have) p[i] = v.v[i];
}
template <int n> __device__ __forceinline__ void activate_all(float (&v)[n], int act)
{
    auto each = [&](auto a) {
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = activate<decltype(a)::value>(v[i]);
    };
    switch (act) {      // the same for the whole launch
        case SQ_ACT_RELU: return each(std::integral_constant<int, SQ_ACT_RELU>{});
        case SQ_ACT_SILU: return each(std::integral_constant<int, SQ_ACT_SILU>{});
        case SQ_ACT_GELU: return each(std::integral_constant<int, SQ_ACT_GELU>{});
        default: return;
    }
}
// Results from sums, bias and residual, out to the first `have` places.
template <typename TO, int n> __device__ __forceinline__ void put(const LinearArgs &p, TO *out, int have, float (&v)[n], const Vec<float, n> &b, const Vec<TO, n> &res)
{
    if (p.b)
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] += b.v[i];
    activate_all(v, p.act);
    Vec<TO, n> o;
#pragma unroll
    for (int i = 0; i < n; ++i) o.v[i] = from_f32<TO>(p.residual ? v[i] + to_f32(res.v[i]) : v[i]);
    store_some<n>(out, o, have);
}

// Bias, activation and residual of n neighbouring results of one row, of which the first `have` exist.
template <typename TO, int n> __device__ __forceinline__ void finish(const LinearArgs &p, long long r, int j, int have, float (&v)[n])
{
    if (have <= 0) return;
    Vec<float, n> b = {};
    Vec<TO, n> res = {};
    if (p.b) b = load_some<n>(p.b + j, have);
    if (p.residual) res = load_some<n>((const TO *)p.residual + r * p.ld_res + j, have);
    put<TO, n>(p, (TO *)p.out + r * p.ld_out + j, have, v, b, res);
}

// Two fp32 values as the sums of three pairs of bfloat16 values: h the upper halves, m = round(x - h), l = x - h - m.
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
    // The edge of the output.  whole: only rows are missing, and no load hangs on a condition of its lane's (with one, bfloat16 residuals are
    // taken apart under it, each load waited for: 729 x 1536 x 384 with residual 8.5 us for 7.5).
    auto edge = [&](auto whole) {
        const int have = decltype(whole)::value ? n : p.Cout - j0 - j;
        Vec<float, n> b = {};
        if (p.b && have > 0) b = load_some<n>(p.b + j0 + j, have);
#pragma unroll
        for (int x = 0; x < XB; ++x) {
            Vec<TO, n> res[kTurns] = {};
            if (p.residual && have > 0)
#pragma unroll
                for (int t = 0; t < kTurns; ++t) res[t] = load_some<n>((const TO *)p.residual + row_at(r0, 32 * x + row + t * kPer, p.rows) * p.ld_res + j0 + j, have);
            stage(x);
#pragma unroll
            for (int t = 0; t < kTurns; ++t) {
                const int i = 32 * x + row + t * kPer;
                float v[n];
                staged(t, v);
                if (have > 0 && row_in(r0, i, p.rows)) put<TO, n>(p, (TO *)p.out + ((long long)r0 + i) * p.ld_out + j0 + j, have, v, b, res[t]);
            }
        }
    };
    if (!row_in(j0, 32 * JB - 1, p.Cout)) return edge(std::false_type{});
    if (!row_in(r0, 32 * XB - 1, p.rows)) return edge(std::true_type{});
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

}  // namespace
}  // namespace sq
