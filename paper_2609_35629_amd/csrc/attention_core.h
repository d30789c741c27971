// Softmax attention of blocks of query rows over tiles of key rows, on the
// matrix cores; the device code shared by prompt attention and shared-prefix
// decoding.
//
// The query rows of one (sequence, KV head) pair are its tokens' G heads, token
// by token (row r: token r / G, head r % G), so that a block of rows reads each
// key tile once for all of them.  A workgroup of WR x WK waves takes 32 WR rows
// and walks the key tiles in one pass (running maximum m and sum l, in fp32 and
// base 2):  S^T = K Q^T, P = 2^(s - m), O^T += V^T P^T.  The scores are formed
// transposed so that a lane holds scores of one query row (column lane % 32 of the
// 32 x 32 product, keys 8 (i / 4) + 4 (lane / 32) + i % 4 in register i): row
// maxima and sums stay in the lane but for one exchange with the other half of
// the wave, and P^T is the next product's right operand as it stands, once V's
// rows are read in that key order.
//
// K and V tiles are copied to LDS by DMA (no registers), one tile ahead; their
// 16-byte pieces are permuted within the row so that both the row reads of K
// and the transposing reads of V spread over all banks.
//
// bf16 rows: v_mfma_f32_32x32x16_bf16.  fp32 queries over bf16 rows enter as
// three bf16 terms each (q and P: 24 bits), so that the result is as exact as
// fp32 products; bf16 queries as one, with P rounded to bf16 (2^-8 at most, like
// the output's own rounding) or, where rows are few, two terms of it.  fp32 rows:
// v_mfma_f32_32x32x2_f32.
//
// Bound: the matrix cores where rows are many, memory where they are few.  A wave's
// step of 64 keys of 128 dims is 1024 cycles of products and about 950 of softmax,
// which run beside each other only between the two waves of a SIMD: 16384 causal
// tokens of 16 heads take 1055 us (1040 TFLOP/s; a bf16 matrix product of 8192^3
// reaches 1170 on the same card).  Few rows: 67 MB of a 32K prompt's cache for eight
// answers in 28 us, of which the start and end of a block and the join of its
// parts are about 13.
#pragma once

#include "attention.h"
#include "common.h"

#include <type_traits>

namespace santapp {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// One stretch of keys: rows K, V of n keys.
struct KeySeg {
    const char *K, *V;
    long long kt, vt;  // bytes between rows, at most kMaxRowStep
    int n;
};

// What one query row may attend: keys [lo, hi) of the stretch, of its document;
// pos: its position relative to the stretch's first key; slope: log2(e) times
// the bias per key of distance.
struct RowInfo {
    int lo, hi, pos, doc;
    float slope;
};

static_assert(kMaxRowStep < (1ll << 32), "a lane multiplies its row by 32 bits");

constexpr float kNegInf = -__builtin_inff();

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Maximum and sum of a value and that of the other half-wave's lane (lane ^ 32).
__device__ __forceinline__ float max_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Wave-uniform minimum and maximum.
template <typename F>
__device__ __forceinline__ int wave_fold(int v, F&& f) {
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x128, 0xF, 0xF, false));
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x124, 0xF, 0xF, false));
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x122, 0xF, 0xF, false));
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x121, 0xF, 0xF, false));
    return f(f(readlane(v, 0), readlane(v, 16)), f(readlane(v, 32), readlane(v, 48)));
}
__device__ __forceinline__ int wave_min_i32(int v) {
    return wave_fold(v, [](int x, int y) { return min(x, y); });
}
__device__ __forceinline__ int wave_max_i32(int v) {
    return wave_fold(v, [](int x, int y) { return max(x, y); });
}

// tanh: 1 - 2 / (1 + e^2|y|) (absolute error about 2^-23), and where that would
// cancel (|y| < 0.35; EXACT only) its Taylor series to y^13.
template <bool EXACT>
__device__ __forceinline__ float tanh_of(float y) {
    const float a = fabsf(y);
    float r = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + exp2_fast(a * 2.88539008177792681f));
    if constexpr (EXACT) {
        const float z = a * a;
        const float t = a + a * z * (-1.f / 3 + z * (2.f / 15 + z * (-17.f / 315 + z * (62.f / 2835 +
                                     z * (-1382.f / 155925 + z * (21844.f / 6081075))))));
        r = a < 0.35f ? t : r;
    }
    return copysignf(r, y);
}

// Bytes of a row and the permutation of its 16-byte pieces: 16 rows at the
// same piece, and 4 rows at 4 neighbouring pieces, fall into distinct banks.
template <typename T, int D>
struct Tile {
    static constexpr int RB = D * static_cast<int>(sizeof(T));
    static constexpr int SPR = RB / 16;
    static __device__ __forceinline__ int perm(int row) {
        if constexpr (RB >= 256)
            return ((row & 3) << 2) | ((row >> 2) & 3);
        else  // two rows share the 256 bytes of the banks
            return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    }
    static __device__ __forceinline__ int at(int row, int byte) {
        return row * RB + (((byte >> 4) ^ perm(row)) << 4) + (byte & 15);
    }
};

// Query rows as right operands, scores and value sums of 32 keys.  NT, PT: bf16
// terms of a query and of a weight.
template <typename T, int D, int NT, int PT>
struct Ops;

template <int D, int NT, int PT>
struct Ops<bf16_t, D, NT, PT> {
    using TL = Tile<bf16_t, D>;
    bf16x8 q[NT][D / 16];

    // NT == 1: bf16 query rows, else fp32 rows, loaded first and split by
    // ready() once the first tile's copies are under way
    float4 raw[NT > 1 ? D / 8 : 1];
    __device__ __forceinline__ void load_q(const char* row, int hh) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            if constexpr (NT == 1) {
                q[0][k] = *reinterpret_cast<const bf16x8*>(row + 2 * (16 * k + 8 * hh));
            } else {
                const float4* p = reinterpret_cast<const float4*>(row + 4 * (16 * k + 8 * hh));
                raw[2 * k] = p[0];
                raw[2 * k + 1] = p[1];
            }
        }
    }
    __device__ __forceinline__ void ready() {
        if constexpr (NT > 1) {
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const float4 u = raw[2 * k], v = raw[2 * k + 1];
                const float x[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) split(x[e], k, e);
            }
        }
    }
    __device__ __forceinline__ void split(float x, int k, int e) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const __bf16 h = static_cast<__bf16>(x);
            q[t][k][e] = h;
            x -= static_cast<float>(h);
        }
    }
    // Of KS x 32 keys; the keys are read two products ahead.  between(k) is called
    // after the k-th of kSlots products (of each stretch and term).
    static constexpr int kSlots = D / 16;
    template <int KS, typename F>
    __device__ __forceinline__ void scores(const char* ktile, int row0, int lane, f32x16 (&s)[KS], F&& between) const {
        const int row = row0 + (lane & 31), hh = lane >> 5;
        bf16x8 a[3][KS];
        auto load = [&](int k) {
#pragma unroll
            for (int u = 0; u < KS; ++u)
                a[k % 3][u] = *reinterpret_cast<const bf16x8*>(ktile + TL::at(row + 32 * u, 16 * (2 * k + hh)));
        };
        load(0);
        load(1);
#pragma unroll
        for (int u = 0; u < KS; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[u][i] = 0.f;
#pragma unroll
        for (int k = 0; k < kSlots; ++k) {
            if (k + 2 < kSlots) load(k + 2);
#pragma unroll
            for (int t = NT - 1; t >= 0; --t)
#pragma unroll
                for (int u = 0; u < KS; ++u)
                    s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[k % 3][u], q[t][k], s[u], 0, 0, 0);
            between(k);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // V^T of 4 keys x 16 dims per 16 lanes: lane s % 16 addresses key s / 4,
    // dims 4 (s % 4) .. + 4, lane n receives the four keys of dim n.
    static __device__ __forceinline__ bf16x8 values(const char* vtile, int row0, int db, int lane) {
        typedef short v4i16 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) v4i16 lds_v4i16;
        const int s = lane & 15;
        const int row = row0 + 4 * (lane >> 5) + (s >> 2);
        const int byte = 64 * db + 32 * ((lane >> 4) & 1) + 8 * (s & 3);
        const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(vtile + TL::at(row, byte)));
        const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(vtile + TL::at(row + 8, byte)));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // Of KS x 32 keys, 16 at a time; the next 16 keys' values are read while the
    // products of the last run.
    template <int KS>
    static __device__ __forceinline__ void add_values(const char* vtile, int row0, const f32x16 (&p)[KS],
                                                      f32x16 (&o)[D / 32], int lane) {
        bf16x8 a[2][D / 32];
#pragma unroll
        for (int db = 0; db < D / 32; ++db) a[0][db] = values(vtile, row0, db, lane);
#pragma unroll
        for (int k = 0; k < 2 * KS; ++k) {
            if (k + 1 < 2 * KS) {
#pragma unroll
                for (int db = 0; db < D / 32; ++db) a[(k + 1) & 1][db] = values(vtile, row0 + 16 * (k + 1), db, lane);
            }
            __builtin_amdgcn_sched_barrier(0);
            bf16x8 b[PT];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float x = p[k / 2][8 * (k & 1) + e];
#pragma unroll
                for (int t = 0; t < PT; ++t) {
                    const __bf16 h = static_cast<__bf16>(x);
                    b[t][e] = h;
                    x -= static_cast<float>(h);
                }
            }
#pragma unroll
            for (int t = PT - 1; t >= 0; --t)
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[k & 1][db], b[t], o[db], 0, 0, 0);
        }
    }
};

template <int D>
struct Ops<float, D, 1, 1> {
    using TL = Tile<float, D>;
    // dims 8 c + 4 (lane / 32) + e of the row, as q[c].e
    float4 q[D / 8];

    __device__ __forceinline__ void load_q(const char* row, int hh) {
#pragma unroll
        for (int c = 0; c < D / 8; ++c) q[c] = *reinterpret_cast<const float4*>(row + 4 * (8 * c + 4 * hh));
    }
    __device__ __forceinline__ void ready() {}
    static constexpr int kSlots = D / 8;
    template <int KS, typename F>
    __device__ __forceinline__ void scores(const char* ktile, int row0, int lane, f32x16 (&out)[KS], F&& between) const {
        static_assert(KS == 1, "one stretch of fp32 keys at a time");
        const int row = row0 + (lane & 31), hh = lane >> 5;
        float4 a[3];
        auto load = [&](int c) {
            a[c % 3] = *reinterpret_cast<const float4*>(ktile + TL::at(row, 16 * (2 * c + hh)));
        };
        load(0);
        load(1);
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int c = 0; c < kSlots; ++c) {
            if (c + 2 < kSlots) load(c + 2);
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(a[c % 3].x, q[c].x, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(a[c % 3].y, q[c].y, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(a[c % 3].z, q[c].z, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(a[c % 3].w, q[c].w, s, 0, 0, 0);
            between(c);
            __builtin_amdgcn_sched_barrier(0);
        }
        out[0] = s;
    }
    template <int KS>
    static __device__ __forceinline__ void add_values(const char* vtile, int row0, const f32x16 (&p)[KS],
                                                      f32x16 (&o)[D / 32], int lane) {
        float a[2][4][D / 32];  // of four keys
        auto load = [&](int g) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
                    a[g & 1][i][db] = *reinterpret_cast<const float*>(
                        vtile + TL::at(row0 + 8 * g + 4 * (lane >> 5) + i, 4 * (32 * db + (lane & 31))));
        };
        load(0);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (g < 3) load(g + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[g & 1][i][db], p[0][4 * g + i], o[db], 0, 0, 0);
        }
    }
};

// The elements of a word as a pass takes them: pass 1 finite ones (others 0),
// passes 2, 3, 4 ones in place of +infinity, -infinity, NaN (others 0).
template <typename T>
__device__ __forceinline__ uint32_t only_special(uint32_t w, int pass) {
    auto of = [&](uint32_t bits) {  // fp32
        const bool special = (bits & 0x7f800000u) == 0x7f800000u, nan = (bits & 0x7fffffu) != 0;
        if (pass == 1) return special ? 0u : bits;
        const bool on = special && (pass == 4 ? nan : !nan && (bits >> 31) == (pass == 3));
        return on ? 0x3f800000u : 0u;
    };
    if constexpr (sizeof(T) == 4) return of(w);
    return (of(w << 16) >> 16) | of(w & 0xffff0000u);
}

// The run [x, y) of document d's keys among [lo, hi) of a row, x = y if there are
// none, y = -1 if they are no run.  Wave-uniform.  Of the ranges of kDocTile keys
// that may hold d, a run makes neighbours, of which only the first and the last
// may hold other keys: in front of it and behind it.
__device__ __forceinline__ int2 doc_run(const int* docs, const int2* ranges, int d, int lo, int hi, int n) {
    if (d < 0 || lo >= hi) return make_int2(0, 0);
    const int2 none = make_int2(0, -1);
    const int lane = lane_id(), end = (hi + kDocTile - 1) / kDocTile;
    constexpr int kAhead = 4;  // loads of 64 ranges under way
    int first = -1, last = -1, some = 0, mixed = 0;
    for (int r = lo / kDocTile; r < end; r += kAhead * kWave) {
        int2 x[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) x[k] = ranges[min(r + k * kWave + lane, end - 1)];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int rk = r + k * kWave;
            const bool on = rk + lane < end && x[k].x <= d && x[k].y >= d;
            const uint64_t s = __ballot(on);
            if (s == 0) continue;
            if (first < 0) first = rk + static_cast<int>(__builtin_ctzll(s));
            last = rk + 63 - static_cast<int>(__builtin_clzll(s));
            some += static_cast<int>(__builtin_popcountll(s));
            mixed += static_cast<int>(__builtin_popcountll(__ballot(on && x[k].x != x[k].y)));
        }
    }
    if (first < 0) return make_int2(0, 0);
    if (some != last - first + 1) return none;
    // bit i: key i of the first range, and of the last, is d's (half a wave each)
    const int half = lane < kDocTile ? first : last, j = half * kDocTile + (lane & (kDocTile - 1));
    const uint64_t both = __ballot(j < n && docs[min(j, n - 1)] == d);
    const int2 rf = ranges[first], rl = ranges[last];
    const bool mf = rf.x != rf.y, ml = last != first && rl.x != rl.y;
    if (mixed != (mf ? 1 : 0) + (ml ? 1 : 0)) return none;
    int x = first * kDocTile, y = min((last + 1) * kDocTile, n);
    if (mf) {
        const uint32_t e = static_cast<uint32_t>(both);
        if (e == 0) return none;
        const int z = __builtin_ctz(e);
        const uint32_t up = e >> z;
        if ((up & (up + 1)) != 0) return none;
        if (last != first && (e >> 31) == 0) return none;
        x += z;
        if (last == first) y = x + __builtin_popcount(e);
    }
    if (ml) {
        const uint32_t e = static_cast<uint32_t>(both >> 32);
        if (e == 0 || (e & (e + 1)) != 0) return none;
        y = last * kDocTile + __builtin_popcount(e);
    }
    return make_int2(x, y);
}

// Shape of a workgroup: WR x 32 rows, tiles of BK keys taken in SUB steps of which
// each of the WK groups of waves has KS x 32 keys.
template <typename T, int D, int NT, int WR, int WK>
struct Shape {
    static constexpr int NW = WR * WK;
    static constexpr int KS = (sizeof(T) == 2 && WK == 1) ? 2 : 1;
    static constexpr int kStep = 32 * WK * KS;             // keys of a step
    static constexpr int kStepBytes = kStep * Tile<T, D>::RB;
    // workgroups per compute unit, two at most: a wave of each per SIMD, one's
    // softmax beside the other's products; one where the registers of a wave
    // (query terms, sums, scores) would not fit half a SIMD's
    static constexpr int kPerCu = (D == 64 || (sizeof(T) == 2 && NT == 1)) && 4 * kStepBytes <= 64 * 1024 ? 2 : 1;
    // two buffers of K and V in about 128 KB of the compute unit's 160: the more
    // steps to a tile, the fewer waits for its copies
    static constexpr int SUB = kPerCu * 8 * kStepBytes <= 128 * 1024 ? 2 : 1;
    static constexpr int BK = kStep * SUB;
    static constexpr int BM = 32 * WR;
    static constexpr int kTile = BK * Tile<T, D>::RB;      // bytes of one K or V tile
    static constexpr int kState = 32 * (D + 4) * 4;        // bytes of one wave's state (WK > 1)
    static constexpr int kBuf = 2 * kTile > (WK > 1 ? NW * kState / 2 : 0) ? 2 * kTile : NW * kState / 2;
    static_assert(kPerCu * (2 * kBuf + 1024) <= 160 * 1024, "LDS of a compute unit");
    static_assert(kTile % (1024 * NW) == 0, "a tile is a whole number of 1 KB copies per wave");
};

// What the scores and masks of a kernel may have besides the plain ones.
constexpr int kExtra = 1;  // a cap, or a bias by distance
constexpr int kDocs = 2;   // documents

// Attention of one block of rows over tiles of a stretch of keys.
//   rows         rows of the block, 1 .. BM
//   rowinfo(r)   RowInfo of the block's row r < rows
//   qrow(r)      its query row
//   docs         (with kDocs) document of each key; ranges: lowest and highest
//                of every kDocTile keys
//   split/splits the part of the block's key tiles to walk
//   emit(r, dim, o, m, l)  receives four unnormalised values of row r
// False if it has to be done again with SPECIAL (see below).
// buf0, buf1: Shape::kBuf bytes of LDS each.
template <typename T, int D, int NT, int WR, int WK, int MODE, bool EXACT, bool SPECIAL, typename Info, typename QRow,
          typename Emit>
__device__ __forceinline__ bool attend(const KeySeg& seg, const ScoreArgs& sc, const int* docs, const int2* ranges,
                                       int split, int splits, char* buf0, char* buf1, int rows, Info&& rowinfo, QRow&& qrow,
                                       Emit&& emit) {
    using SH = Shape<T, D, NT, WR, WK>;
    using TL = Tile<T, D>;
    // bf16 queries: one term of a weight, where rows are few (blocks of 32 by four
    // waves over keys, which wait for memory) two
    constexpr int PT = sizeof(T) == 2 && NT == 1 && WK == 4 ? 2 : NT;
    using OP = Ops<T, D, NT, PT>;
    constexpr int BK = SH::BK, KS = SH::KS, NW = SH::NW, SUB = SH::SUB;
    constexpr bool EXTRA = (MODE & kExtra) != 0, DOCS = (MODE & kDocs) != 0;
    const int lane = lane_id(), hh = lane >> 5;
    const int wv = __builtin_amdgcn_readfirstlane(wave_id());
    const int wr = wv % WR, wk = wv / WR;

    // keys that any row of the block may attend, and its rows' documents
    int blo = seg.n, bhi = 0, dlo = 0x7fffffff, dhi = -0x7fffffff - 1;
#pragma unroll
    for (int r = lane; r < SH::BM; r += kWave) {
        if (r >= rows) break;
        const RowInfo x = rowinfo(r);
        if (x.lo < x.hi) {
            blo = min(blo, x.lo);
            bhi = max(bhi, x.hi);
        }
        dlo = min(dlo, x.doc);
        dhi = max(dhi, x.doc);
    }
    blo = wave_min_i32(blo);
    bhi = wave_max_i32(bhi);
    if constexpr (DOCS) {
        dlo = wave_min_i32(dlo);
        dhi = wave_max_i32(dhi);
    }
    const bool mine = 32 * wr + (lane & 31) < rows;  // whether the lane's row is one
    RowInfo me = rowinfo(mine ? 32 * wr + (lane & 31) : 0);
    // Rows of one document whose keys are one run [lo, hi) (packed documents)
    // attend within the run; documents are compared key by key otherwise.
    bool by_key = false;
    if constexpr (DOCS) {
        by_key = true;
        const int2 run = dlo == dhi ? doc_run(docs, ranges, dlo, blo, bhi, seg.n) : make_int2(0, -1);
        if (run.y >= 0) {
            by_key = false;
            blo = max(blo, run.x);
            bhi = min(bhi, run.y);
            me.lo = max(me.lo, run.x);
            me.hi = max(me.lo, min(me.hi, run.y));
        }
    }
    // keys that every row of the wave may attend, and that any may
    const int wlo = wave_max_i32(mine ? me.lo : 0), whi = wave_min_i32(mine ? me.hi : seg.n);
    const int vlo = wave_min_i32(mine ? me.lo : seg.n), vhi = wave_max_i32(mine ? me.hi : 0);

    const int wpos = wave_min_i32(mine ? me.pos : 0x7fffffff);  // the foremost query

    // this split's tiles
    int t0 = blo / BK, t1 = bhi > blo ? (bhi + BK - 1) / BK : t0;
    {
        const int n = t1 - t0, per = (n + splits - 1) / splits;
        t0 += min(n, split * per);
        t1 = min(t1, t0 + per);
    }

    // The next tile from t on whose keys share a document with the block.  The
    // lanes look at 64 tiles at once: bit i of `some` and `same` for tile
    // seen + i, which holds some key of the rows' documents, and nothing but keys
    // of the one document that all rows have.
    uint64_t some = 0, same = 0;
    int seen = t0;
    auto look = [&]() {
        constexpr int RT = BK / kDocTile;
        const int nr = (seg.n + kDocTile - 1) / kDocTile;
        bool on = false, one = dlo == dhi;
        if (seen + lane < t1) {
#pragma unroll
            for (int k = 0; k < RT; ++k) {
                const int i = (seen + lane) * RT + k;
                if (i < nr) {
                    const int2 x = ranges[i];
                    on = on || (x.y >= 0 && x.x <= dhi && x.y >= dlo);
                    one = one && x.x == dlo && x.y == dlo;
                }
            }
        }
        some = __ballot(on);
        same = __ballot(one && dlo >= 0);
    };
    if (by_key) look();
    auto next = [&](int t) {
        if (by_key) {
            while (t < t1) {
                if (t >= seen + kWave) {
                    seen += kWave;
                    look();
                }
                const uint64_t left = some >> (t - seen);
                if (left) return t + static_cast<int>(__builtin_ctzll(left));
                t = seen + kWave;
            }
            return t1;
        }
        return t;
    };
    // A wave's 1 KB copies take every NW-th group of rows: row0 + step i, whose
    // permutation differs from row0's by that of step i.
    constexpr int RPC = 64 / TL::SPR, STEP = NW * RPC;
    const int row0 = wv * RPC + lane / TL::SPR;
    const uint32_t piece0 = 16 * ((lane % TL::SPR) ^ TL::perm(row0));
    // The copies of a tile, in kCopies parts (of one K and one V piece): a wave
    // that issues them in a row waits for the other waves' in the queue, so that
    // they go between the products of the tile before (16384 tokens: 1130 us in a
    // row, 1088 between).
    constexpr int kCopies = SH::kTile / (1024 * NW);
    static_assert((STEP & (STEP - 1)) == 0 && kCopies * STEP == BK, "whole groups");
    const char *kb = nullptr, *vb = nullptr;
    char* to = nullptr;
    int last = 0;
    auto target = [&](int t, char* buf) {
        to = buf + 1024 * wv;
        kb = seg.K + static_cast<long long>(t) * BK * seg.kt;
        vb = seg.V + static_cast<long long>(t) * BK * seg.vt;
        last = seg.n - 1 - t * BK;
    };
    const uint32_t kt = static_cast<uint32_t>(seg.kt), vt = static_cast<uint32_t>(seg.vt);
    auto copy_part = [&](int i) {
        const uint32_t piece = piece0 ^ (16 * TL::perm(STEP * i));
        const uint64_t row = static_cast<uint32_t>(min(row0 + STEP * i, last));  // rows behind the last key repeat it
        __builtin_amdgcn_global_load_lds(kb + (row * kt + piece),
                                         (__attribute__((address_space(3))) void*)(to + 1024 * NW * i), 16, 0, 0);
        __builtin_amdgcn_global_load_lds(vb + (row * vt + piece),
                                         (__attribute__((address_space(3))) void*)(to + SH::kTile + 1024 * NW * i), 16, 0, 0);
    };
    auto copy = [&](int t, char* buf) {
        target(t, buf);
#pragma unroll
        for (int i = 0; i < kCopies; ++i) copy_part(i);
    };

    OP op;
    op.load_q(qrow(mine ? 32 * wr + (lane & 31) : 0), hh);
    float m, l;
    f32x16 o[D / 32];

    // Where V holds a NaN or an infinity, the product carries it into every row of
    // the block, also those that mask its key (0 times infinity).  A block that
    // finds a value that is not finite in its sums (false is returned, nothing
    // emitted) is done again with SPECIAL, which walks the tiles four times: in
    // passes 4, 3, 2 over V's NaNs, -infinities and +infinities as ones, with ones
    // for the weights of unmasked keys, which says where they belong (has[]), and in
    // pass 1 over V with zeros in their place.  Sums that still are not finite
    // (values near the largest number, times weights above 1) are walked once more
    // with the reference at the maximum throughout.
    int pass = 0;
    float slack = 8.f;
    auto compute = [&](int t, int sub, const char* buf, bool alone, auto&& between) {
        const int in_tile = sub * SH::kStep + wk * 32 * KS;  // the wave's first key of the step
        const int k0 = t * BK + in_tile;
        if (k0 >= vhi || k0 + 32 * KS <= vlo) {
#pragma unroll
            for (int k = 0; k < OP::kSlots; ++k) between(k);
            return;
        }
        f32x16 s[KS];
        op.scores(buf, in_tile, lane, s, between);
        __builtin_amdgcn_s_setprio(0);
        if constexpr (EXTRA) {
            // s = scale q.k, capped, less the slope times the distance; with no
            // key behind a query of the wave that distance is linear
            if (sc.capped) {
#pragma unroll
                for (int u = 0; u < KS; ++u)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[u][i] = sc.cap_log2 * tanh_of<EXACT>(s[u][i] * sc.inv_cap);
            }
            const float c = sc.capped ? 1.f : sc.scale_log2;
            const float far = static_cast<float>(me.pos - k0 - 4 * hh);
            if (!sc.slopes) {
#pragma unroll
                for (int u = 0; u < KS; ++u)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[u][i] *= c;
            } else if (k0 + 32 * KS - 1 <= wpos) {
                const float base = -me.slope * far;
#pragma unroll
                for (int u = 0; u < KS; ++u)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        s[u][i] = fmaf(s[u][i], c, fmaf(me.slope, static_cast<float>(32 * u + 8 * (i / 4) + i % 4), base));
            } else {
#pragma unroll
                for (int u = 0; u < KS; ++u)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        s[u][i] = fmaf(-me.slope, fabsf(far - static_cast<float>(32 * u + 8 * (i / 4) + i % 4)), s[u][i] * c);
            }
        }
        const bool masked = k0 < wlo || k0 + 32 * KS > whi;
        if (masked) {
#pragma unroll
            for (int u = 0; u < KS; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = k0 + 32 * u + 8 * (i / 4) + 4 * hh + i % 4;
                    if (j < me.lo || j >= me.hi) s[u][i] = kNegInf;
                }
        }
        if (DOCS && by_key && !alone) {
#pragma unroll
            for (int u = 0; u < KS; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = min(k0 + 32 * u + 8 * (i / 4) + 4 * hh + i % 4, seg.n - 1);
                    if (docs[j] != me.doc || me.doc < 0) s[u][i] = kNegInf;
                }
        }
        uint32_t open[KS];  // keys not masked (pass > 1)
        if (SPECIAL && pass > 1) {
#pragma unroll
            for (int u = 0; u < KS; ++u) {
                open[u] = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) open[u] |= s[u][i] == kNegInf ? 0u : 1u << i;
            }
        }
        float top = kNegInf;
#pragma unroll
        for (int u = 0; u < KS; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
        top = max_halves(top);
        if constexpr (!EXTRA) top *= sc.scale_log2;
        // the reference m moves only where a score exceeds it by more than 8
        // (weights up to 2^8 are as exact as those below 1)
        if (__any(top > m + (SPECIAL ? slack : 8.f))) {
            const float mn = fmaxf(m, top);
            const float f = mn == kNegInf || (SPECIAL && pass > 1) ? 1.f : exp2_fast(m - mn);
            l *= f;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[db][i] *= f;
            m = mn;
        }
        const float ref = m == kNegInf ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < KS; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[u][i] = exp2_fast(EXTRA ? s[u][i] - ref : fmaf(s[u][i], sc.scale_log2, -ref));
                sum += s[u][i];
            }
        l += sum;
        if (SPECIAL && pass > 1) {
#pragma unroll
            for (int u = 0; u < KS; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[u][i] = (open[u] >> i) & 1 ? 1.f : 0.f;
        }
        // products first: of two waves on a SIMD, the one in its products keeps
        // the matrix cores busy and the other's softmax fills in (16384 tokens:
        // 1160 us without, 1135 with)
        __builtin_amdgcn_s_setprio(1);
        OP::add_values(buf + SH::kTile, in_tile, s, o, lane);
    };

    // every wave's copies of a tile are in LDS before any wave reads it
    auto arrived = [&]() {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    // V as the pass takes it
    auto prepare = [&](char* buf) {
        for (int x = threadIdx.x; x < SH::kTile / 16; x += NW * kWave) {
            uint32_t* p = reinterpret_cast<uint32_t*>(buf + SH::kTile + 16 * x);
            for (int e = 0; e < 4; ++e) p[e] = only_special<T>(p[e], pass);
        }
        __syncthreads();
    };
    // The steps of tile t in `buf`, with the copies of tile n (n < t1) into `other`.
    auto step = [&](int t, char* buf, bool alone, int n, char* other) {
        if constexpr (SPECIAL) prepare(buf);
        const bool more = n < t1;
        if (more) target(n, other);
        constexpr int kAll = SUB * OP::kSlots;
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub)
            compute(t, sub, buf, alone, [&](int k) {
                if (!more) return;  // uniform
                const int slot = sub * OP::kSlots + k;
#pragma unroll
                for (int i = 0; i < kCopies; ++i)
                    if (i * kAll / kCopies == slot) copy_part(i);
            });
    };
    // one tile ahead; the two buffers are distinct objects, so that the copies
    // into one are known not to touch the reads of the other
    auto walk = [&]() {
        if (by_key && seen != t0) {
            seen = t0;
            look();
        }
        int t = next(t0);
        m = kNegInf;
        l = 0.f;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
        if (t >= t1) return;
        bool alone = (same >> (t - seen)) & 1;
        copy(t, buf0);
        if (!SPECIAL || pass == 4) op.ready();
        for (;;) {
            int n = next(t + 1);
            arrived();
            step(t, buf0, alone, n, buf1);
            if (n >= t1) break;
            t = n;
            alone = (same >> (t - seen)) & 1;
            n = next(t + 1);
            arrived();
            step(t, buf1, alone, n, buf0);
            if (n >= t1) break;
            t = n;
            alone = (same >> (t - seen)) & 1;
        }
    };
    // whether some sum of the wave's rows is not finite
    auto overflows = [&]() {
        float z = 0.f;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) z = fmaf(o[db][i], 0.f, z);
        return __any(mine && z != 0.f) != 0;
    };
    if constexpr (!SPECIAL) {
        __shared__ int s_special;
        if (threadIdx.x == 0) s_special = 0;  // before the first tile's barrier; without tiles no value is special
        walk();
        if (overflows() && lane == 0) s_special = 1;
        __syncthreads();
        if (s_special) return false;  // uniform
    } else {
        uint32_t has[3][D / 64];  // +infinity, -infinity, NaN of value 16 db + i
#pragma unroll 1
        for (pass = 4; pass > 0; --pass) {
            walk();
            __syncthreads();  // the tiles are read before they are copied again
#pragma unroll
            for (int k = 2; k < 5; ++k) {
                if (k != pass) continue;
#pragma unroll
                for (int w = 0; w < D / 64; ++w) {
                    uint32_t bits = 0;
#pragma unroll
                    for (int i = 0; i < 32; ++i) bits |= o[2 * w + i / 16][i % 16] != 0.f ? 1u << i : 0u;
                    has[k - 2][w] = bits;
                }
            }
        }
        if (__syncthreads_or(overflows())) {
            pass = 1;
            slack = 0.f;
            walk();
            __syncthreads();
        }
#pragma unroll
        for (int w = 0; w < D / 64; ++w)
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const uint32_t bit = 1u << i;
                float x = o[2 * w + i / 16][i % 16];
                if (has[0][w] & bit) x = __builtin_inff();
                if (has[1][w] & bit) x = kNegInf;
                if ((has[2][w] | (has[0][w] & has[1][w])) & bit) x = __builtin_nanf("");
                o[2 * w + i / 16][i % 16] = x;
            }
    }
    l = add_halves(l);

    if constexpr (WK == 1) {
        if (mine) {
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    emit(32 * wr + (lane & 31), 32 * db + 2 * i + 4 * hh,
                         make_float4(o[db][i], o[db][i + 1], o[db][i + 2], o[db][i + 3]), m, l);
        }
    } else {
        // the WK states of a row meet in LDS
        constexpr int ST = D + 4;
        __syncthreads();
        auto state = [&](int w) {
            constexpr int HALF = (NW + 1) / 2;
            return reinterpret_cast<float*>((w < HALF ? buf0 : buf1) + (w < HALF ? w : w - HALF) * SH::kState);
        };
        float* own = state(wv) + (lane & 31) * ST;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<float4*>(own + 32 * db + 2 * i + 4 * hh) =
                    make_float4(o[db][i], o[db][i + 1], o[db][i + 2], o[db][i + 3]);
        if (hh == 0) {
            own[D] = m;
            own[D + 1] = l;
        }
        __syncthreads();
        for (int x = threadIdx.x; x < SH::BM * (D / 4); x += NW * kWave) {
            const int r = x / (D / 4), dim = 4 * (x % (D / 4));
            if (r >= rows) continue;
            float mm = kNegInf;
#pragma unroll
            for (int k = 0; k < WK; ++k) mm = fmaxf(mm, state(k * WR + r / 32)[(r % 32) * ST + D]);
            float ll = 0.f;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < WK; ++k) {
                const float* p = state(k * WR + r / 32) + (r % 32) * ST;
                const float f = p[D] == kNegInf ? 0.f : exp2_fast(p[D] - mm);
                const float4 y = *reinterpret_cast<const float4*>(p + dim);
                ll += f * p[D + 1];
                v.x += f * y.x;
                v.y += f * y.y;
                v.z += f * y.z;
                v.w += f * y.w;
            }
            emit(r, dim, v, mm, ll);
        }
    }
    return true;
}

__device__ __forceinline__ int clamp_pos(long long x) {
    constexpr long long most = 1 << 30;
    return static_cast<int>(x < -most ? -most : x > most ? most : x);
}

}  // namespace santapp
