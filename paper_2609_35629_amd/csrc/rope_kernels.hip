// Rotary positions of query and key rows, and their way into the cache.
//
// Dims i and i + R (or 2 i and 2 i + 1, interleaved) of a row at position p turn
// by the angle a = p f_i:  y1 = m (x1 cos a - x2 sin a),  y2 = m (x2 cos a + x1 sin a).
// p f_i is formed in fp64 (fp32 would be off by 2^-24 p radians: 0.008 at
// position 131072) and reduced there to an eighth of a turn; sine and cosine
// of the rest are fp32 series.
//
// Bound: the rows are read and written once.  A thread keeps the sines and
// cosines of eight pairs of one token and applies them to several heads, so
// that the angles (about 60 instructions a pair) stay beside the row traffic:
// 470 MB of a 32K prompt's queries in 87 us (5.4 TB/s; a plain copy moves 4.9).
// A kernel of its own for one stream with its types known: with the types
// looked at for every row it took 150 us.
#include <type_traits>

#include "attention.h"
#include "common.h"

namespace santapp {

namespace {

constexpr int kThreads = 256;
constexpr int kPairs = 8;  // pairs per thread

// sin(a), cos(a) of a = p f: a / (2 pi) = n / 4 + r, |r| <= 1/8, both exact in
// fp64 once a is rounded; then the Taylor series at 2 pi r (|x| <= pi / 4: the
// first term left out is below 2^-28 of the result).
__device__ __forceinline__ void turn(double p, double f, float& sn, float& cs) {
    const double t = p * f * 0.15915494309189533577;
    const double n4 = rint(4.0 * t);
    const float x = static_cast<float>((t - 0.25 * n4) * 6.28318530717958647693);
    const int n = static_cast<int>(static_cast<long long>(n4) & 3);
    const float z = x * x;
    const float s = x + x * z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880))));
    const float c = 1.f + z * (-.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320 + z * (-1.f / 3628800)))));
    const float a = (n & 1) ? c : s, b = (n & 1) ? s : c;
    sn = (n & 2) ? -a : a;
    cs = (n == 1 || n == 2) ? -b : b;
}

__device__ __forceinline__ float load1(const void* p, bool f32, long long i) {
    return f32 ? static_cast<const float*>(p)[i] : bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
}

__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v)); }

__device__ __forceinline__ void store1(void* p, bool f32, long long i, float v) {
    if (f32)
        static_cast<float*>(p)[i] = v;
    else
        static_cast<uint16_t*>(p)[i] = to_bf16(v);
}

// Eight consecutive elements, 16-byte aligned.
__device__ __forceinline__ void load8(const void* p, bool f32, long long i, float (&v)[8]) {
    if (f32) {
        const float4* s = reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
        const float4 a = s[0], b = s[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i);
        v[0] = bf16lo(a.x); v[1] = bf16hi(a.x); v[2] = bf16lo(a.y); v[3] = bf16hi(a.y);
        v[4] = bf16lo(a.z); v[5] = bf16hi(a.z); v[6] = bf16lo(a.w); v[7] = bf16hi(a.w);
    }
}

__device__ __forceinline__ void store8(void* p, bool f32, long long i, const float (&v)[8]) {
    if (f32) {
        float4* s = reinterpret_cast<float4*>(static_cast<float*>(p) + i);
        s[0] = make_float4(v[0], v[1], v[2], v[3]);
        s[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = to_bf16(v[2 * e]) | (static_cast<uint32_t>(to_bf16(v[2 * e + 1])) << 16);
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + i) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// A unit's eight elements as loaded, and widened.
template <bool F32>
struct Eight;
template <>
struct Eight<false> {
    uint4 w;
    __device__ __forceinline__ void load(const void* p, long long i) {
        w = load_stream(static_cast<const uint16_t*>(p) + i);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        v[0] = bf16lo(w.x); v[1] = bf16hi(w.x); v[2] = bf16lo(w.y); v[3] = bf16hi(w.y);
        v[4] = bf16lo(w.z); v[5] = bf16hi(w.z); v[6] = bf16lo(w.w); v[7] = bf16hi(w.w);
    }
    static __device__ __forceinline__ void store(void* p, long long i, const float (&v)[8]) {
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = to_bf16(v[2 * e]) | (static_cast<uint32_t>(to_bf16(v[2 * e + 1])) << 16);
        __builtin_nontemporal_store(u32x4_t{o[0], o[1], o[2], o[3]},
                                    reinterpret_cast<u32x4_t*>(static_cast<uint16_t*>(p) + i));
    }
};
template <>
struct Eight<true> {
    float4 a, b;
    __device__ __forceinline__ void load(const void* p, long long i) {
        a = load_stream_f(static_cast<const float*>(p) + i);
        b = load_stream_f(static_cast<const float*>(p) + i + 4);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    static __device__ __forceinline__ void store(void* p, long long i, const float (&v)[8]) {
        float* o = static_cast<float*>(p) + i;
        store_stream(o, make_float4(v[0], v[1], v[2], v[3]));
        store_stream(o + 4, make_float4(v[4], v[5], v[6], v[7]));
    }
};

// x, y: the halves of eight pairs (or, interleaved, the pairs one after the other).
__device__ __forceinline__ void turn8(float (&x)[8], float (&y)[8], const float (&sn)[8], const float (&cs)[8],
                                      bool interleaved) {
    if (interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float u = x[2 * e], w = x[2 * e + 1];
            x[2 * e] = u * cs[e] - w * sn[e];
            x[2 * e + 1] = w * cs[e] + u * sn[e];
            const float u2 = y[2 * e], w2 = y[2 * e + 1];
            y[2 * e] = u2 * cs[e + 4] - w2 * sn[e + 4];
            y[2 * e + 1] = w2 * cs[e + 4] + u2 * sn[e + 4];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float u = x[e], w = y[e];
            x[e] = u * cs[e] - w * sn[e];
            y[e] = w * cs[e] + u * sn[e];
        }
    }
}

// One thread: one token (b, t), one unit of the row and the heads
// h0, h0 + hstep, .. of all streams.  VEC: a unit is eight pairs, or eight
// dims that are not rotated (16-byte accesses); otherwise one pair or one dim.
template <bool VEC>
__global__ __launch_bounds__(kThreads) void k_rope(RopeArgs a) {
    constexpr int E = VEC ? kPairs : 1;
    const int R = a.pairs, rot_units = VEC ? R / kPairs : R;
    const int units = rot_units + (a.d - 2 * R) / E;
    const long long i = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
    const long long per_token = static_cast<long long>(units) * a.hstep;
    const long long token = i / per_token;
    if (token >= static_cast<long long>(a.B) * a.T) return;
    const int rest = static_cast<int>(i - token * per_token);
    const int h0 = rest / units, unit = rest - h0 * units;
    const int b = static_cast<int>(token / a.T), t = static_cast<int>(token - static_cast<long long>(b) * a.T);
    const long long row = (a.at ? a.at[b] : a.at0) + static_cast<long long>(t);
    const bool fits = row >= 0 && row < a.capacity;  // of the streams that are appended
    const bool rotated = unit < rot_units;
    // the unit's first dims: the pair's halves, or the dims copied
    int d1, d2;
    if (rotated) {
        d1 = a.interleaved ? 2 * E * unit : E * unit;
        d2 = a.interleaved ? d1 + E : d1 + R;
    } else {
        d1 = d2 = 2 * R + E * (unit - rot_units);
    }
    float sn[E], cs[E];
    if (rotated) {
        const long long pos = a.positions ? static_cast<long long>(a.positions[token]) : a.first + row;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            turn(static_cast<double>(pos), a.freqs[E * unit + e], sn[e], cs[e]);
            sn[e] *= a.magnitude;
            cs[e] *= a.magnitude;
        }
    }
    for (int h = h0; h < a.heads; h += a.hstep) {
        const int si = h < a.s[0].heads ? 0 : h < a.s[0].heads + a.s[1].heads ? 1 : 2;
        const RopeStream& s = a.s[si];
        const int hs = h - (si > 0 ? a.s[0].heads : 0) - (si > 1 ? a.s[1].heads : 0);
        if (s.append && !fits) continue;
        const long long in = b * s.ib + hs * s.ih + t * s.it;
        const long long out = b * s.ob + hs * s.oh + (s.append ? row : t) * s.ot;
        if constexpr (VEC) {
            float x[8], y[8];
            load8(s.in, s.in32, in + d1, x);
            if (rotated) load8(s.in, s.in32, in + d2, y);
            if (rotated && s.rotate) turn8(x, y, sn, cs, a.interleaved);
            store8(s.out, s.out32, out + d1, x);
            if (rotated) store8(s.out, s.out32, out + d2, y);
        } else {
            float x = load1(s.in, s.in32, in + d1), y = 0.f;
            if (rotated) y = load1(s.in, s.in32, in + d2);
            if (rotated && s.rotate) {
                const float u = x, w = y;
                x = u * cs[0] - w * sn[0];
                y = w * cs[0] + u * sn[0];
            }
            store1(s.out, s.out32, out + d1, x);
            if (rotated) store1(s.out, s.out32, out + d2, y);
        }
    }
}

// One stream of rows whose pairs come in whole units (d / 8 - pairs / 8 units a
// row): one thread, one token and unit, heads h0, h0 + hstep, .., the next
// head's elements in flight while one is turned and stored.
template <bool IN32, bool OUT32, bool INTER>
__global__ __launch_bounds__(kThreads) void k_rope_rows(RopeArgs a) {
    const int R = a.pairs, rot_units = R / kPairs, units = a.d / 8 - rot_units;
    const unsigned per_token = static_cast<unsigned>(units) * a.hstep;
    const long long i = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
    const long long token = i / per_token;
    if (token >= static_cast<long long>(a.B) * a.T) return;
    const unsigned rest = static_cast<unsigned>(i - token * per_token);
    const int h0 = rest / static_cast<unsigned>(units), unit = rest - h0 * units;
    const int b = static_cast<int>(token / a.T), t = static_cast<int>(token - static_cast<long long>(b) * a.T);
    const bool rotated = unit < rot_units;
    const int d1 = !rotated ? 2 * R + 8 * (unit - rot_units) : INTER ? 16 * unit : 8 * unit;
    const int d2 = INTER ? d1 + 8 : d1 + R;
    const RopeStream& s = a.s[0];
    long long in = b * s.ib + h0 * s.ih + t * s.it, out = b * s.ob + h0 * s.oh + t * s.ot;
    Eight<IN32> x, y;
    x.load(s.in, in + d1);
    y = x;
    if (rotated) y.load(s.in, in + d2);
    float sn[8], cs[8];
    if (rotated) {
        const long long pos = a.positions ? static_cast<long long>(a.positions[token]) : a.first + t;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            turn(static_cast<double>(pos), a.freqs[8 * unit + e], sn[e], cs[e]);
            sn[e] *= a.magnitude;
            cs[e] *= a.magnitude;
        }
    }
    for (int h = h0; h < a.heads; h += a.hstep) {
        Eight<IN32> nx = x, ny = y;
        in += a.hstep * s.ih;
        if (h + a.hstep < a.heads) {
            nx.load(s.in, in + d1);
            if (rotated) ny.load(s.in, in + d2);
        }
        float u[8], w[8];
        x.get(u);
        if (rotated) {
            y.get(w);
            turn8(u, w, sn, cs, INTER);
            Eight<OUT32>::store(s.out, out + d2, w);
        }
        Eight<OUT32>::store(s.out, out + d1, u);
        out += a.hstep * s.oh;
        x = nx;
        y = ny;
    }
}

}  // namespace

hipError_t launch_rope(RopeArgs a, int cus, hipStream_t s) {
    a.heads = a.s[0].heads + a.s[1].heads + a.s[2].heads;
    const long long tokens = static_cast<long long>(a.B) * a.T;
    if (tokens == 0 || a.heads == 0) return hipSuccess;
    // 16-byte units need the second half of the pairs, and what is copied
    // behind them, to start on one
    const bool vec = a.pairs % kPairs == 0;
    const int units = vec ? a.d / 8 - a.pairs / kPairs : a.d - a.pairs;
    // as many heads per thread as leave eight waves a SIMD: the queries of a 32K
    // prompt (28 heads of 128, bf16) in 87 us there, 88 at 32 waves, 109 at 128
    const long long most = static_cast<long long>(cus > 0 ? cus : 256) * 2048;
    long long hstep = most / (tokens * units);
    hstep = hstep < 1 ? 1 : hstep > a.heads ? a.heads : hstep;
    a.hstep = static_cast<int>(hstep);
    const long long blocks = (tokens * units * hstep + kThreads - 1) / kThreads;
    const dim3 grid(static_cast<unsigned>(blocks));
    if (vec && a.s[1].heads == 0) {
        const RopeStream& r = a.s[0];
        auto run = [&](auto in32, auto out32) {
            if (a.interleaved)
                k_rope_rows<decltype(in32)::value, decltype(out32)::value, true><<<grid, kThreads, 0, s>>>(a);
            else
                k_rope_rows<decltype(in32)::value, decltype(out32)::value, false><<<grid, kThreads, 0, s>>>(a);
        };
        if (r.in32)
            r.out32 ? run(std::true_type{}, std::true_type{}) : run(std::true_type{}, std::false_type{});
        else
            r.out32 ? run(std::false_type{}, std::true_type{}) : run(std::false_type{}, std::false_type{});
        return hipGetLastError();
    }
    if (vec)
        k_rope<true><<<grid, kThreads, 0, s>>>(a);
    else
        k_rope<false><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace santapp
