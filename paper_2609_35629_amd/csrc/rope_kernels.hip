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
// looked at for every row it took 150 us.  The streams of an append, a few rows
// each, take that one (4 us, a launch's start and end).
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

__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v)); }

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

// The eight elements 8 unit .. of a row, and how each is turned: by cs and sn and
// its partner's place in the row (-1: an element that is copied).
struct Turns {
    float sn[8], cs[8];
    int other[8];
    __device__ __forceinline__ void set(const RopeArgs& a, int unit, long long pos) {
        const int R = a.pairs;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int j = 8 * unit + e;
            const bool second = a.interleaved ? (j & 1) != 0 : j >= R;
            other[e] = j >= 2 * R ? -1 : a.interleaved ? j ^ 1 : second ? j - R : j + R;
            const int f = j >= 2 * R ? 0 : a.interleaved ? j >> 1 : second ? j - R : j;
            turn(static_cast<double>(pos), a.freqs[f], sn[e], cs[e]);
            cs[e] *= a.magnitude;
            sn[e] *= second ? a.magnitude : -a.magnitude;
        }
    }
    // The partners meet in LDS: `mine` is this thread's 32 bytes of its row's.
    __device__ __forceinline__ void apply(float (&u)[8], float4* mine, const float* row, bool rotate) const {
        mine[0] = make_float4(u[0], u[1], u[2], u[3]);
        mine[1] = make_float4(u[4], u[5], u[6], u[7]);
        wave_lds_sync();
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (rotate && other[e] >= 0) u[e] = u[e] * cs[e] + row[other[e]] * sn[e];
        wave_lds_sync();
    }
};

// Several streams, of any types and pairs: one thread, one token (b, t), eight
// elements of a row (the d / 8 lanes of a row are lanes of one wave) and the
// heads h0, h0 + hstep, .. of all streams.
__global__ __launch_bounds__(kThreads) void k_rope(RopeArgs a) {
    __shared__ float4 s_row[2 * kThreads];
    const int units = a.d / 8;
    const unsigned per_token = static_cast<unsigned>(units) * a.hstep;
    const long long i = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
    const long long token = i / per_token;
    if (token >= static_cast<long long>(a.B) * a.T) return;  // whole rows
    const unsigned rest = static_cast<unsigned>(i - token * per_token);
    const int h0 = rest / static_cast<unsigned>(units), unit = rest - h0 * units;
    const int b = static_cast<int>(token / a.T), t = static_cast<int>(token - static_cast<long long>(b) * a.T);
    const long long row = (a.at ? a.at[b] : a.at0) + static_cast<long long>(t);
    const bool fits = row >= 0 && row < a.capacity;  // of the streams that are appended
    Turns turns;
    turns.set(a, unit, a.positions ? static_cast<long long>(a.positions[token]) : a.first + row);
    for (int h = h0; h < a.heads; h += a.hstep) {
        const int si = h < a.s[0].heads ? 0 : h < a.s[0].heads + a.s[1].heads ? 1 : 2;
        const RopeStream& s = a.s[si];
        const int hs = h - (si > 0 ? a.s[0].heads : 0) - (si > 1 ? a.s[1].heads : 0);
        if (s.append && !fits) continue;
        float u[8];
        load8(s.in, s.in32, b * s.ib + hs * s.ih + t * s.it + 8 * unit, u);
        turns.apply(u, s_row + 2 * threadIdx.x, reinterpret_cast<const float*>(s_row + 2 * (threadIdx.x - unit)), s.rotate);
        store8(s.out, s.out32, b * s.ob + hs * s.oh + (s.append ? row : t) * s.ot + 8 * unit, u);
    }
}

// One stream of rows rotated whole, in halves (2 pairs == d, d / 16 units of eight
// pairs a row): one thread, one token and unit, heads h0, h0 + hstep, .., the next
// head's elements in flight while one is turned and stored.
template <bool IN32, bool OUT32>
__global__ __launch_bounds__(kThreads) void k_rope_rows(RopeArgs a) {
    const int R = a.pairs, units = R / kPairs;
    const unsigned per_token = static_cast<unsigned>(units) * a.hstep;
    const long long i = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
    const long long token = i / per_token;
    if (token >= static_cast<long long>(a.B) * a.T) return;
    const unsigned rest = static_cast<unsigned>(i - token * per_token);
    const int h0 = rest / static_cast<unsigned>(units), unit = rest - h0 * units;
    const int b = static_cast<int>(token / a.T), t = static_cast<int>(token - static_cast<long long>(b) * a.T);
    const RopeStream& s = a.s[0];
    long long in = b * s.ib + h0 * s.ih + t * s.it + 8 * unit, out = b * s.ob + h0 * s.oh + t * s.ot + 8 * unit;
    Eight<IN32> x, y;
    x.load(s.in, in);
    y.load(s.in, in + R);
    const long long pos = a.positions ? static_cast<long long>(a.positions[token]) : a.first + t;
    float sn[8], cs[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        turn(static_cast<double>(pos), a.freqs[8 * unit + e], sn[e], cs[e]);
        sn[e] *= a.magnitude;
        cs[e] *= a.magnitude;
    }
    for (int h = h0; h < a.heads; h += a.hstep) {
        Eight<IN32> nx = x, ny = y;
        in += a.hstep * s.ih;
        if (h + a.hstep < a.heads) {
            nx.load(s.in, in);
            ny.load(s.in, in + R);
        }
        float u[8], w[8];
        x.get(u);
        y.get(w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float p = u[e], q = w[e];
            u[e] = p * cs[e] - q * sn[e];
            w[e] = q * cs[e] + p * sn[e];
        }
        Eight<OUT32>::store(s.out, out, u);
        Eight<OUT32>::store(s.out, out + R, w);
        out += a.hstep * s.oh;
        x = nx;
        y = ny;
    }
}

// One stream of rows with other pairs, as k_rope: 8192 tokens of 28 heads of 128,
// bf16, in 23 us whatever the pairs (rows rotated whole in halves, as above: 22;
// with interleaved pairs in one thread, read at 32-byte steps: 39).
template <bool IN32, bool OUT32>
__global__ __launch_bounds__(kThreads) void k_rope_any(RopeArgs a) {
    __shared__ float4 s_row[2 * kThreads];
    const int units = a.d / 8;
    const unsigned per_token = static_cast<unsigned>(units) * a.hstep;
    const long long i = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
    const long long token = i / per_token;
    if (token >= static_cast<long long>(a.B) * a.T) return;  // whole rows
    const unsigned rest = static_cast<unsigned>(i - token * per_token);
    const int h0 = rest / static_cast<unsigned>(units), unit = rest - h0 * units;
    const int b = static_cast<int>(token / a.T), t = static_cast<int>(token - static_cast<long long>(b) * a.T);
    const RopeStream& s = a.s[0];
    long long in = b * s.ib + h0 * s.ih + t * s.it + 8 * unit, out = b * s.ob + h0 * s.oh + t * s.ot + 8 * unit;
    Eight<IN32> x;
    x.load(s.in, in);
    Turns turns;
    turns.set(a, unit, a.positions ? static_cast<long long>(a.positions[token]) : a.first + t);
    for (int h = h0; h < a.heads; h += a.hstep) {
        Eight<IN32> nx = x;
        in += a.hstep * s.ih;
        if (h + a.hstep < a.heads) nx.load(s.in, in);
        float u[8];
        x.get(u);
        turns.apply(u, s_row + 2 * threadIdx.x, reinterpret_cast<const float*>(s_row + 2 * (threadIdx.x - unit)), true);
        Eight<OUT32>::store(s.out, out, u);
        out += a.hstep * s.oh;
        x = nx;
    }
}

}  // namespace

hipError_t launch_rope(RopeArgs a, int cus, hipStream_t s) {
    a.heads = a.s[0].heads + a.s[1].heads + a.s[2].heads;
    const long long tokens = static_cast<long long>(a.B) * a.T;
    if (tokens == 0 || a.heads == 0) return hipSuccess;
    const bool one = a.s[1].heads == 0, halves = one && !a.interleaved && 2 * a.pairs == a.d;
    const int units = halves ? a.d / 16 : a.d / 8;
    // as many heads per thread as leave eight waves a SIMD: the queries of a 32K
    // prompt (28 heads of 128, bf16) in 87 us there, 88 at 32 waves, 109 at 128
    const long long most = static_cast<long long>(cus > 0 ? cus : 256) * 2048;
    long long hstep = most / (tokens * units);
    hstep = hstep < 1 ? 1 : hstep > a.heads ? a.heads : hstep;
    a.hstep = static_cast<int>(hstep);
    const long long blocks = (tokens * units * hstep + kThreads - 1) / kThreads;
    const dim3 grid(static_cast<unsigned>(blocks));
    if (one) {
        const RopeStream& r = a.s[0];
        auto run = [&](auto in32, auto out32) {
            constexpr bool I = decltype(in32)::value, O = decltype(out32)::value;
            if (halves)
                k_rope_rows<I, O><<<grid, kThreads, 0, s>>>(a);
            else
                k_rope_any<I, O><<<grid, kThreads, 0, s>>>(a);
        };
        if (r.in32)
            r.out32 ? run(std::true_type{}, std::true_type{}) : run(std::true_type{}, std::false_type{});
        else
            r.out32 ? run(std::false_type{}, std::true_type{}) : run(std::false_type{}, std::false_type{});
        return hipGetLastError();
    }
    k_rope<<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace santapp
