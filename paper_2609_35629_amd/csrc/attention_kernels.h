// Kernels and launches of prompt attention and shared-prefix decoding, over
// attention_core.h.  The two .hip files that include this hold one of them each.
#pragma once

#include "attention_core.h"

namespace santapp {

// Joins the split parts of every row.  D / 4 lanes per row, four dims each; the
// parts of a row come in up to two runs (prompt, suffix).
struct JoinRun {
    const float2* ml;  // part i: ml[i stride], values o[i stride d]
    const float* o;
    long long stride;  // rows between parts
    int n;
};

template <int D>
__device__ __forceinline__ float4 join_parts(const JoinRun (&runs)[2], int dim, float& l) {
    float m = kNegInf;
    for (int x = 0; x < 2; ++x)
        for (int i = 0; i < runs[x].n; ++i) m = fmaxf(m, runs[x].ml[i * runs[x].stride].x);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    l = 0.f;
    for (int x = 0; x < 2; ++x)
        for (int i = 0; i < runs[x].n; ++i) {
            const float2 ml = runs[x].ml[i * runs[x].stride];
            if (ml.y == 0.f) continue;  // nothing attended
            const float f = exp2_fast(ml.x - m);
            const float4 y = *reinterpret_cast<const float4*>(runs[x].o + i * runs[x].stride * D + dim);
            l += f * ml.y;
            v.x += f * y.x;
            v.y += f * y.y;
            v.z += f * y.z;
            v.w += f * y.w;
        }
    return v;
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
// Variant v is WR x WK of row_waves(v) x key_waves(v, dtype).
constexpr int variant_of(long long rows) { return rows <= 32 ? 0 : rows <= 64 ? 1 : 2; }
constexpr int row_waves(int v) { return v == 0 ? 1 : v == 1 ? 2 : 4; }
// fp32 tiles are twice as large: two waves over keys fill the LDS
constexpr int key_waves(int v, bool f32) { return v == 0 ? (f32 ? 2 : 4) : v == 1 ? 2 : 1; }
inline int tile_keys(int v, bool f32) { return f32 ? 32 * key_waves(v, true) : 32 * (key_waves(v, false) == 1 ? 2 : key_waves(v, false)); }

}  // namespace santapp
