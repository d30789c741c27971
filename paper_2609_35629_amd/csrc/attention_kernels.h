// Kernels and launches of prompt attention and shared-prefix decoding, over
// attention_core.h.  The two .hip files that include this hold one of them each.
#pragma once

#include "attention_core.h"

namespace santapp {

typedef __attribute__((address_space(3))) char lds_char;

// The kernel's one argument, where it was passed.
template <typename A>
__device__ __forceinline__ const A* kernel_args() {
    return (const A*)__builtin_amdgcn_kernarg_segment_ptr();
}

// Joins the split parts of rows.  The parts of a row come in up to two runs
// (prompt, suffix) of at most kMaxParts in all.  Rows of more than kFewParts take a
// workgroup each, several parts in flight (140 rows of 128 parts: 99 us with a
// lane walking all parts of a row, 8 with a workgroup).  Otherwise D / 4 lanes
// take a row (512 tokens of 28 heads in two parts: 35 us with a workgroup a row,
// 15 in one part).
constexpr int kJoinThreads = 256;
constexpr int kMaxParts = 320;
constexpr int kFewParts = 8;

struct JoinRun {
    const float2* ml;  // part i: ml[i stride], values o[i stride d]
    const float* o;
    long long stride;  // rows between parts
    int n;
};

__device__ __forceinline__ void store4(float* p, float4 v, float f) {
    *reinterpret_cast<float4*>(p) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
}
__device__ __forceinline__ void store4(bf16_t* p, float4 v, float f) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    bf16x4 b;
    b[0] = static_cast<__bf16>(v.x * f);
    b[1] = static_cast<__bf16>(v.y * f);
    b[2] = static_cast<__bf16>(v.z * f);
    b[3] = static_cast<__bf16>(v.w * f);
    *reinterpret_cast<bf16x4*>(p) = b;
}

// 1 / l, 0 for a row that attended nothing.
__device__ __forceinline__ float inverse_sum(float l) { return l == 0.f ? 0.f : 1.f / l; }

template <int D>
constexpr int join_rows(int parts) {
    return parts <= kFewParts ? kJoinThreads / (D / 4) : 1;
}

// One row by D / 4 lanes.
template <int D, typename TO>
__device__ __forceinline__ void join_few(const JoinRun (&runs)[2], TO* out) {
    const int c = threadIdx.x % (D / 4), n = runs[0].n + runs[1].n;
    float2 ml[kFewParts];
    float4 y[kFewParts];
#pragma unroll
    for (int i = 0; i < kFewParts; ++i) {
        ml[i] = make_float2(kNegInf, 0.f);
        y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < n) {
            const int x = i < runs[0].n ? 0 : 1;
            const long long at = (i - (x ? runs[0].n : 0)) * runs[x].stride;
            ml[i] = runs[x].ml[at];
            y[i] = reinterpret_cast<const float4*>(runs[x].o + at * D)[c];
        }
    }
    float m = kNegInf, l = 0.f;
#pragma unroll
    for (int i = 0; i < kFewParts; ++i)
        if (ml[i].y != 0.f) m = fmaxf(m, ml[i].x);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kFewParts; ++i) {
        const float f = ml[i].y == 0.f ? 0.f : exp2_fast(ml[i].x - m);
        if (f != 0.f) {  // a part of no weight may hold anything
            l = fmaf(f, ml[i].y, l);
            v.x = fmaf(f, y[i].x, v.x);
            v.y = fmaf(f, y[i].y, v.y);
            v.z = fmaf(f, y[i].z, v.z);
            v.w = fmaf(f, y[i].w, v.w);
        }
    }
    store4(out + 4 * c, v, inverse_sum(l));
}

// One row by the workgroup: every wave finds the maximum and the weights of all
// parts for itself (part i in lane i % 64), while the first values are on their
// way; D / 4 lanes take the values of every kGroups-th part.
template <int D, typename TO>
__device__ __forceinline__ void join_many(const JoinRun (&runs)[2], TO* out) {
    constexpr int L = D / 4, kGroups = kJoinThreads / L;
    constexpr int kEach = kMaxParts / kWave, kChunk = kWave / kGroups;  // parts of a lane; of a group per 64
    static_assert(kEach * kWave == kMaxParts && kChunk * kGroups == kWave, "whole chunks");
    __shared__ float4 s_v[kGroups][L];
    const int n = runs[0].n + runs[1].n, lane = lane_id();
    const int g = threadIdx.x / L, c = threadIdx.x % L;
    auto place = [&](int i, int& x) {
        x = i < runs[0].n ? 0 : 1;
        return (i - (x ? runs[0].n : 0)) * runs[x].stride;
    };
    float2 ml[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = lane + kWave * k;
        ml[k] = make_float2(kNegInf, 0.f);
        if (i < n) {
            int x;
            const long long at = place(i, x);
            ml[k] = runs[x].ml[at];
        }
    }
    float4 y[kChunk];
    auto load = [&](int k) {
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            const int i = kWave * k + kGroups * j + g;
            y[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (i < n) {
                int x;
                const long long at = place(i, x);
                y[j] = reinterpret_cast<const float4*>(runs[x].o + at * D)[c];
            }
        }
    };
    load(0);
    float m = kNegInf, l = 0.f;
#pragma unroll
    for (int k = 0; k < kEach; ++k)
        if (ml[k].y != 0.f) m = fmaxf(m, ml[k].x);
    m = wave_max_f32(m);
    float w[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        w[k] = ml[k].y == 0.f ? 0.f : exp2_fast(ml[k].x - m);  // nothing attended: 0
        if (w[k] != 0.f) l = fmaf(w[k], ml[k].y, l);
    }
    l = row16_sum(l);
    l = add_halves(l);
    l += __shfl_xor(l, 16);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        if (kWave * k >= n) break;  // uniform
        if (k > 0) load(k);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            const float f = __shfl(w[k], kGroups * j + g);
            if (f != 0.f) {  // a part of no weight may hold anything
                v.x = fmaf(f, y[j].x, v.x);
                v.y = fmaf(f, y[j].y, v.y);
                v.z = fmaf(f, y[j].z, v.z);
                v.w = fmaf(f, y[j].w, v.w);
            }
        }
    }
    s_v[g][c] = v;
    __syncthreads();
    if (threadIdx.x < L) {
        v = s_v[0][c];
#pragma unroll
        for (int k = 1; k < kGroups; ++k) {
            const float4 z = s_v[k][c];
            v.x += z.x;
            v.y += z.y;
            v.z += z.z;
            v.w += z.w;
        }
        store4(out + 4 * c, v, inverse_sum(l));
    }
}

// One split's part of row r of a pair: values, and (by the lane of dim 0) its
// maximum and sum.
template <int D>
__device__ __forceinline__ void store_part(const PartArgs& p, long long pair, int split, int rows, int r, int dim,
                                           float4 v, float m, float l) {
    const long long i = (pair * p.splits + split) * rows + r;
    *reinterpret_cast<float4*>(p.o + i * D + dim) = v;
    if (dim == 0) p.ml[i] = make_float2(m, l);
}

inline size_t part_rows(long long pairs, int splits, long long rows) {
    return static_cast<size_t>(pairs) * splits * rows;
}

// Places of a run of parts in the workspace, from byte `at`; the bytes taken.
inline size_t place_parts(PartArgs& p, long long pairs, long long rows, int d, char* ws, size_t at) {
    auto up = [](size_t x) { return (x + 255) & ~static_cast<size_t>(255); };
    const size_t n = part_rows(pairs, p.splits, rows);
    p.ml = reinterpret_cast<float2*>(ws + at);
    p.o = reinterpret_cast<float*>(ws + at + up(n * sizeof(float2)));
    return up(n * sizeof(float2)) + up(n * d * sizeof(float));
}

// Row blocks by the rows of a pair: few rows spread the waves over keys.
// Variant v is WR x WK of row_waves(v) x key_waves(v, dtype), 32 WR rows a block.
constexpr int variant_of(long long rows) { return rows <= 32 ? 0 : rows <= 64 ? 1 : 2; }
constexpr int row_waves(int v) { return v == 0 ? 1 : v == 1 ? 2 : 4; }
// fp32 tiles are twice as large: two waves over keys fill the LDS
constexpr int key_waves(int v, bool f32) { return v == 0 ? (f32 ? 2 : 4) : v == 1 ? 2 : 1; }

template <typename F>
auto with_shape(int v, int d, bool f32, int terms, F&& f) {
    auto shape = [&](auto wr, auto wk32, auto wk16) {
        constexpr int WR = decltype(wr)::value, W32 = decltype(wk32)::value, W16 = decltype(wk16)::value;
        if (f32) return d == 64 ? f(Shape<float, 64, 1, WR, W32>{}) : f(Shape<float, 128, 1, WR, W32>{});
        if (terms == 1) return d == 64 ? f(Shape<bf16_t, 64, 1, WR, W16>{}) : f(Shape<bf16_t, 128, 1, WR, W16>{});
        return d == 64 ? f(Shape<bf16_t, 64, 3, WR, W16>{}) : f(Shape<bf16_t, 128, 3, WR, W16>{});
    };
    using std::integral_constant;
    if (v == 0)
        return shape(integral_constant<int, row_waves(0)>{}, integral_constant<int, key_waves(0, true)>{},
                     integral_constant<int, key_waves(0, false)>{});
    if (v == 1)
        return shape(integral_constant<int, row_waves(1)>{}, integral_constant<int, key_waves(1, true)>{},
                     integral_constant<int, key_waves(1, false)>{});
    return shape(integral_constant<int, row_waves(2)>{}, integral_constant<int, key_waves(2, true)>{},
                 integral_constant<int, key_waves(2, false)>{});
}

// Keys of a tile, and workgroups a compute unit holds, of a variant's kernel.
inline int tile_keys(int v, bool f32) {
    return with_shape(v, 128, f32, 1, [](auto s) { return decltype(s)::BK; });
}
inline int per_cu(int v, int d, bool f32, int terms) {
    return with_shape(v, d, f32, terms, [](auto s) { return decltype(s)::kPerCu; });
}

}  // namespace santapp
