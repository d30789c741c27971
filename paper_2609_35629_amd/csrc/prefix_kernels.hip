// Decoding of several sequences over a prompt they share: each prompt's keys and
// values are read once for all its sequences, each sequence's suffix rows once
// for its heads, and the parts are joined.
#include <algorithm>

#include "attention_kernels.h"

namespace santapp {

namespace {

__device__ __forceinline__ int clamped(const int* p, int i, int most) {
    return p ? min(max(p[i], 0), most) : most;
}

// A workgroup takes a block of a prompt's rows, or (split over keys by SK of its
// waves) one of a sequence's heads over its suffix.
constexpr int suffix_key_waves(int v, bool f32) { return v == 0 ? key_waves(0, f32) : 2; }

template <typename T, int D, int WR, int WK>
struct PrefixShape {
    static constexpr int SK = suffix_key_waves(variant_of(32 * WR), sizeof(T) == 4);
    static constexpr int NT = sizeof(T) == 4 ? 1 : 3;  // bf16 terms of a query
    using Prompt = Shape<T, D, NT, WR, WK>;
    using Suffix = Shape<T, D, NT, WR * WK / SK, SK>;
    static constexpr int kBuf = Prompt::kBuf > Suffix::kBuf ? Prompt::kBuf : Suffix::kBuf;
    static constexpr int kPerCu = Prompt::kPerCu < Suffix::kPerCu ? Prompt::kPerCu : Suffix::kPerCu;
};

// The block of rows of this workgroup; attend()'s answer.
template <typename T, int D, int WR, int WK, int MODE, bool SPECIAL>
__device__ __forceinline__ bool prefix_block(const PrefixArgs& a, char* buf0, char* buf1) {
    using PS = PrefixShape<T, D, WR, WK>;
    using SH = typename PS::Prompt;
    using SS = typename PS::Suffix;
    constexpr int SK = PS::SK, NT = PS::NT;
    const int Hq = a.Hkv * a.G;
    const int prompts = a.P * a.Hkv * a.row_blocks * a.part.splits;
    int x = blockIdx.x;
    if (x < prompts) {
        const int pairs = a.P * a.Hkv, R = a.S * a.G;
        const int pair = x % pairs;
        x /= pairs;
        const int split = x % a.part.splits, r0 = x / a.part.splits * SH::BM;
        const int p = pair / a.Hkv, kv = pair - p * a.Hkv;
        KeySeg seg;
        seg.K = a.K.p + p * a.K.b + kv * a.K.h;
        seg.V = a.V.p + p * a.V.b + kv * a.V.h;
        seg.kt = a.K.t;
        seg.vt = a.V.t;
        seg.n = clamped(a.prefix_lengths, p, a.N);
        auto rowinfo = [&](int r) {
            RowInfo x;
            const int row = r0 + r, i = row / a.G, b = p * a.S + i, h = kv * a.G + row - i * a.G;
            const long long pos = a.positions ? static_cast<long long>(a.positions[b])
                                              : static_cast<long long>(seg.n) + clamped(a.lengths, b, a.T) - 1;
            x.pos = clamp_pos(pos);
            x.lo = 0;
            x.hi = seg.n;
            if (a.score.window > 0) {
                x.lo = static_cast<int>(min(max(pos - a.score.window + 1, 0ll), static_cast<long long>(seg.n)));
                x.hi = static_cast<int>(min(max(pos + a.score.window, 0ll), static_cast<long long>(seg.n)));
            }
            x.doc = 0;
            x.slope = (MODE & kExtra) != 0 && a.score.slopes ? a.score.slopes[h] * 1.44269504088896341f : 0.f;
            return x;
        };
        auto head = [&](int r) {
            const int row = r0 + r, i = row / a.G;
            return (static_cast<long long>(p) * a.S + i) * Hq + kv * a.G + row - i * a.G;
        };
        auto qrow = [&](int r) { return reinterpret_cast<const char*>(a.q + head(r) * D); };
        auto emit = [&](int r, int dim, float4 v, float m, float l) {
            if (a.part.splits + a.spart.splits > 1)
                store_part<D>(a.part, pair, split, R, r0 + r, dim, v, m, l);
            else
                store4(a.out + head(r) * D + dim, v, inverse_sum(l));
        };
        return attend<T, D, NT, WR, WK, MODE, true, SPECIAL>(seg, a.score, nullptr, nullptr, split, a.part.splits, buf0, buf1,
                                              min(SH::BM, R - r0), rowinfo, qrow,
                                            emit);
    }
    x -= prompts;
    const int pairs = a.P * a.S * a.Hkv;
    const int pair = x % pairs;
    x /= pairs;
    const int split = x % a.spart.splits, r0 = x / a.spart.splits * SS::BM;
    const int b = pair / a.Hkv, kv = pair - b * a.Hkv, p = b / a.S;
    KeySeg seg;
    seg.K = a.sK.p + b * a.sK.b + kv * a.sK.h;
    seg.V = a.sV.p + b * a.sV.b + kv * a.sV.h;
    seg.kt = a.sK.t;
    seg.vt = a.sV.t;
    seg.n = clamped(a.lengths, b, a.T);
    const long long pos = (a.positions ? static_cast<long long>(a.positions[b]) - clamped(a.prefix_lengths, p, a.N)
                                       : static_cast<long long>(seg.n) - 1);
    auto rowinfo = [&](int r) {
        RowInfo x;
        x.pos = clamp_pos(pos);
        x.lo = 0;
        x.hi = seg.n;
        if (a.score.window > 0) {
            x.lo = static_cast<int>(min(max(pos - a.score.window + 1, 0ll), static_cast<long long>(seg.n)));
            x.hi = static_cast<int>(min(max(pos + a.score.window, 0ll), static_cast<long long>(seg.n)));
        }
        x.doc = 0;
        x.slope = (MODE & kExtra) != 0 && a.score.slopes ? a.score.slopes[kv * a.G + r0 + r] * 1.44269504088896341f : 0.f;
        return x;
    };
    auto head = [&](int r) { return static_cast<long long>(b) * Hq + kv * a.G + r0 + r; };
    auto qrow = [&](int r) { return reinterpret_cast<const char*>(a.q + head(r) * D); };
    auto emit = [&](int r, int dim, float4 v, float m, float l) {
        if (a.part.splits + a.spart.splits > 1)
            store_part<D>(a.spart, pair, split, a.G, r0 + r, dim, v, m, l);
        else
            store4(a.out + head(r) * D + dim, v, inverse_sum(l));
    };
    return attend<T, D, NT, WR * WK / SK, SK, MODE, true, SPECIAL>(seg, a.score, nullptr, nullptr, split, a.spart.splits, buf0, buf1,
                                                         min(SS::BM, a.G - r0), rowinfo, qrow, emit);
}

// Called, not inlined: what it keeps in registers is no burden to the kernel's loop.
template <typename T, int D, int WR, int WK, int MODE>
__device__ __attribute__((noinline)) void prefix_special(const PrefixArgs* a, lds_char* buf0, lds_char* buf1) {
    prefix_block<T, D, WR, WK, MODE, true>(*a, (char*)buf0, (char*)buf1);
}

template <typename T, int D, int WR, int WK, int MODE>
__global__ __launch_bounds__(64 * WR * WK, (PrefixShape<T, D, WR, WK>::kPerCu)) void k_prefix(PrefixArgs a) {
    using PS = PrefixShape<T, D, WR, WK>;
    __shared__ __align__(16) char buf0[PS::kBuf];
    __shared__ __align__(16) char buf1[PS::kBuf];
    if (!prefix_block<T, D, WR, WK, MODE, false>(a, buf0, buf1))
        prefix_special<T, D, WR, WK, MODE>(kernel_args<PrefixArgs>(), (lds_char*)buf0, (lds_char*)buf1);
}

template <int D>
__global__ __launch_bounds__(kJoinThreads) void k_prefix_join(PrefixArgs a) {
    const int Hq = a.Hkv * a.G, per = join_rows<D>(a.part.splits + a.spart.splits);
    const int row = blockIdx.x * per + (per > 1 ? threadIdx.x / (D / 4) : 0);
    if (row >= a.P * a.S * Hq) return;
    const int b = row / Hq, h = row - b * Hq, kv = h / a.G, g = h - kv * a.G;
    const int p = b / a.S, R = a.S * a.G;
    const long long f0 = (static_cast<long long>(p) * a.Hkv + kv) * a.part.splits * R + (b - p * a.S) * a.G + g;
    const long long f1 = (static_cast<long long>(b) * a.Hkv + kv) * a.spart.splits * a.G + g;
    const JoinRun runs[2] = {{a.part.ml + f0, a.part.o + f0 * D, R, a.part.splits},
                             {a.spart.ml + f1, a.spart.o + f1 * D, a.G, a.spart.splits}};
    if (per > 1)  // uniform
        join_few<D>(runs, a.out + static_cast<long long>(row) * D);
    else
        join_many<D>(runs, a.out + static_cast<long long>(row) * D);
}

template <typename T, int D>
hipError_t launch(const PrefixArgs& a, hipStream_t s) {
    constexpr bool f32 = sizeof(T) == 4;
    const long long n = static_cast<long long>(a.P) * a.Hkv * a.row_blocks * a.part.splits +
                        static_cast<long long>(a.P) * a.S * a.Hkv * a.srow_blocks * a.spart.splits;
    const dim3 grid(static_cast<unsigned>(n));
    auto run = [&](auto variant) {
        constexpr int V = decltype(variant)::value, WK = key_waves(V, f32);
        if (a.score.capped || a.score.slopes)
            k_prefix<T, D, row_waves(V), WK, kExtra><<<grid, 64 * row_waves(V) * WK, 0, s>>>(a);
        else
            k_prefix<T, D, row_waves(V), WK, 0><<<grid, 64 * row_waves(V) * WK, 0, s>>>(a);
    };
    if (a.variant == 0)
        run(std::integral_constant<int, 0>{});
    else if (a.variant == 1)
        run(std::integral_constant<int, 1>{});
    else
        run(std::integral_constant<int, 2>{});
    if (hipError_t e = hipGetLastError()) return e;
    if (a.part.splits + a.spart.splits > 1) {
        const int per = join_rows<D>(a.part.splits + a.spart.splits);
        k_prefix_join<D><<<dim3(static_cast<unsigned>((a.P * a.S * a.Hkv * a.G + per - 1) / per)), kJoinThreads, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

namespace {
// The most splits of the prompts that are considered: two rounds of blocks.
long long most_splits(long long tiles, long long slots, long long blocks) {
    return std::min<long long>(std::min<long long>(tiles, 256), std::max<long long>(1, 2 * slots / blocks));
}
}  // namespace

size_t plan_prefix(PrefixArgs& a, int cus, char* ws) {
    if (cus <= 0) cus = 256;
    const bool f32 = a.dtype == SANTAPP_FP32;
    const long long R = static_cast<long long>(a.S) * a.G, pairs = static_cast<long long>(a.P) * a.Hkv;
    // by rows alone: 448 rows (64 sequences of 7 heads) take 299 us in blocks of 128,
    // an eighth of them empty, and 309 in full blocks of 64, over 131072 keys
    a.variant = variant_of(R);
    const int bm = 32 * row_waves(a.variant), bk = tile_keys(a.variant, f32);
    const long long slots = static_cast<long long>(per_cu(a.variant, a.d, f32, f32 ? 1 : 3)) * cus;
    // the suffixes: a block per 32 heads (times the waves over rows) each, split
    // while they are few
    const int kw = suffix_key_waves(a.variant, f32);
    const int sbm = 32 * (row_waves(a.variant) * key_waves(a.variant, f32) / kw);
    a.srow_blocks = a.T > 0 ? (a.G + sbm - 1) / sbm : 0;
    const long long sblocks = pairs * a.S * a.srow_blocks;
    a.spart.splits = 0;
    if (a.T > 0) {
        const long long tiles = (a.T + 32 * kw - 1) / (32 * kw);
        long long k = slots / 8 / sblocks;
        k = k > tiles ? tiles : k;
        a.spart.splits = static_cast<int>(k < 1 ? 1 : k > 64 ? 64 : k);
    }
    // the prompts: the splits whose blocks, and the suffixes' in the slots left
    // over, are done first; a block costs its tiles and about two tiles' time for
    // its start and end (8 of about 4 us)
    a.row_blocks = a.N > 0 ? static_cast<int>((R + bm - 1) / bm) : 0;
    const long long blocks = pairs * a.row_blocks;
    a.part.splits = 0;
    if (blocks > 0) {
        const long long tiles = (a.N + bk - 1) / bk, ns = sblocks * a.spart.splits;
        const long long scost = 2 + (ns ? ((a.T + 32 * kw - 1) / (32 * kw) + a.spart.splits - 1) / a.spart.splits : 0);
        long long best = -1;
        const long long most = most_splits(tiles, slots, blocks);
        for (long long k = 1; k <= most; ++k) {
            const long long cost = 2 + (tiles + k - 1) / k, rounds = (blocks * k + slots - 1) / slots;
            const long long idle = rounds * slots - blocks * k, more = ns > idle ? (ns - idle + slots - 1) / slots : 0;
            const long long time = std::max(rounds * cost, (rounds - 1) * cost + scost) + more * scost;
            if (best < 0 || time < best) {
                best = time;
                a.part.splits = static_cast<int>(k);
            }
        }
    }
    if (!ws) {  // room for any shorter suffix too, whatever splits it leads to
        PartArgs p = a.part;
        if (blocks > 0) p.splits = static_cast<int>(most_splits((a.N + bk - 1) / bk, slots, blocks));
        size_t at = 0;
        if (p.splits) at += place_parts(p, pairs, R, a.d, ws, at);
        if (a.spart.splits) at += place_parts(a.spart, pairs * a.S, a.G, a.d, ws, at);
        return at;
    }
    if (a.part.splits + a.spart.splits <= 1) return 0;
    size_t at = 0;
    if (a.part.splits) at += place_parts(a.part, pairs, R, a.d, ws, at);
    if (a.spart.splits) at += place_parts(a.spart, pairs * a.S, a.G, a.d, ws, at);
    return at;
}

hipError_t launch_prefix(const PrefixArgs& a, hipStream_t s) {
    if (a.part.splits + a.spart.splits == 0) {  // no rows at all: zeros
        return launch_zero(a.out, static_cast<size_t>(a.P) * a.S * a.Hkv * a.G * a.d * sizeof(float), s);
    }
    if (a.dtype == SANTAPP_BF16) return a.d == 128 ? launch<bf16_t, 128>(a, s) : launch<bf16_t, 64>(a, s);
    return a.d == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
}

}  // namespace santapp
