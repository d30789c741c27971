// Attention of a prompt's query tokens over its keys: causal, prefix, document
// and window masks, capped scores, a bias by distance.
#include "attention_kernels.h"

namespace santapp {

namespace {

// Lowest and highest document of every kDocTile keys of a row [N].
__global__ __launch_bounds__(256) void k_doc_ranges(const int* docs, int B, int N, int2* ranges) {
    const int nr = (N + kDocTile - 1) / kDocTile;
    const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
    const long long row = i / kDocTile / nr;
    if (row >= B) return;  // whole 32-lane halves
    const int r = static_cast<int>(i / kDocTile - row * nr);
    const int doc = docs[row * N + min(r * kDocTile + static_cast<int>(i % kDocTile), N - 1)];
    int lo = doc, hi = doc;
#pragma unroll
    for (int k = 1; k < kDocTile; k *= 2) {
        lo = min(lo, __shfl_xor(lo, k));
        hi = max(hi, __shfl_xor(hi, k));
    }
    if (i % kDocTile == 0) ranges[row * nr + r] = make_int2(lo, hi);
}

// The block of rows of this workgroup; attend()'s answer.
template <typename T, int D, int WR, int WK, int MODE, bool SPECIAL>
__device__ __forceinline__ bool prompt_block(const PromptArgs& a, char* buf0, char* buf1) {
    using SH = Shape<T, D, 1, WR, WK>;
    const int BH = a.B * a.Hkv, R = a.T * a.G;
    // pairs fastest, so that a pair's blocks share an XCD's cache where the
    // pairs divide the XCDs; the last rows (under a causal mask the longest) first
    int x = blockIdx.x;
    const int pair = x % BH;
    x /= BH;
    const int split = x % a.part.splits;
    const int block = a.row_blocks - 1 - x / a.part.splits;
    const int b = pair / a.Hkv, kv = pair - b * a.Hkv, r0 = block * SH::BM;
    KeySeg seg;
    seg.K = a.K.p + b * a.K.b + kv * a.K.h;
    seg.V = a.V.p + b * a.V.b + kv * a.V.h;
    seg.kt = a.K.t;
    seg.vt = a.V.t;
    seg.n = a.N;
    const int* docs = (MODE & kDocs) != 0 ? a.documents + static_cast<long long>(b) * a.N : nullptr;
    const int prefix = a.prefix ? a.prefix[b] : 0;
    auto rowinfo = [&](int r) {
        RowInfo x;
        const int row = r0 + r, t = row / a.G, h = kv * a.G + row - t * a.G;
        x.pos = a.offset + t;
        int lo = 0, hi = a.N;
        if (a.causal) hi = min(hi, max(x.pos + 1, prefix));
        if (a.score.window > 0) {
            lo = static_cast<int>(max(0ll, static_cast<long long>(x.pos) - a.score.window + 1));
            hi = static_cast<int>(min(static_cast<long long>(hi), static_cast<long long>(x.pos) + a.score.window));
        }
        x.lo = lo;
        x.hi = hi;
        x.doc = docs ? docs[x.pos] : 0;
        x.slope = (MODE & kExtra) != 0 && a.score.slopes ? a.score.slopes[h] * 1.44269504088896341f : 0.f;
        return x;
    };
    auto qrow = [&](int r) {
        const int row = r0 + r, t = row / a.G, h = kv * a.G + row - t * a.G;
        return a.q.p + b * a.q.b + h * a.q.h + t * a.q.t;
    };
    auto emit = [&](int r, int dim, float4 v, float m, float l) {
        if (a.part.splits > 1) {
            store_part<D>(a.part, pair, split, R, r0 + r, dim, v, m, l);
            return;
        }
        const int row = r0 + r, t = row / a.G, h = kv * a.G + row - t * a.G;
        char* p = const_cast<char*>(a.out.p) + b * a.out.b + h * a.out.h + t * a.out.t;
        store4(reinterpret_cast<T*>(p) + dim, v, inverse_sum(l));
    };
    const int2* ranges = docs ? a.doc_range + static_cast<long long>(b) * ((a.N + kDocTile - 1) / kDocTile) : nullptr;
    return attend<T, D, 1, WR, WK, MODE, sizeof(T) == 4, SPECIAL>(seg, a.score, docs, ranges, split, a.part.splits, buf0, buf1,
                                                 min(SH::BM, R - r0), rowinfo,
                                                 qrow, emit);
}

// Called, not inlined: what it keeps in registers is no burden to the kernel's loop.
template <typename T, int D, int WR, int WK, int MODE>
__device__ __attribute__((noinline)) void prompt_special(const PromptArgs* a, lds_char* buf0, lds_char* buf1) {
    prompt_block<T, D, WR, WK, MODE, true>(*a, (char*)buf0, (char*)buf1);
}

template <typename T, int D, int WR, int WK, int MODE>
__global__ __launch_bounds__(64 * WR * WK, (Shape<T, D, 1, WR, WK>::kPerCu)) void k_prompt(PromptArgs a) {
    using SH = Shape<T, D, 1, WR, WK>;
    __shared__ __align__(16) char buf0[SH::kBuf];
    __shared__ __align__(16) char buf1[SH::kBuf];
    if (!prompt_block<T, D, WR, WK, MODE, false>(a, buf0, buf1))
        prompt_special<T, D, WR, WK, MODE>(kernel_args<PromptArgs>(), (lds_char*)buf0, (lds_char*)buf1);
}

template <typename T, int D>
__global__ __launch_bounds__(kJoinThreads) void k_prompt_join(PromptArgs a) {
    const int R = a.T * a.G, per = join_rows<D>(a.part.splits);
    const long long row = static_cast<long long>(blockIdx.x) * per + (per > 1 ? threadIdx.x / (D / 4) : 0);
    if (row >= static_cast<long long>(a.B) * a.Hkv * R) return;
    const int pair = static_cast<int>(row / R), r = static_cast<int>(row - static_cast<long long>(pair) * R);
    const long long first = static_cast<long long>(pair) * a.part.splits * R + r;
    const JoinRun runs[2] = {{a.part.ml + first, a.part.o + first * D, R, a.part.splits}, {nullptr, nullptr, 0, 0}};
    const int b = pair / a.Hkv, kv = pair - b * a.Hkv, t = r / a.G, h = kv * a.G + r - t * a.G;
    char* p = const_cast<char*>(a.out.p) + b * a.out.b + h * a.out.h + t * a.out.t;
    if (per > 1)  // uniform
        join_few<D>(runs, reinterpret_cast<T*>(p));
    else
        join_many<D>(runs, reinterpret_cast<T*>(p));
}

template <typename T, int D>
hipError_t launch(const PromptArgs& a, hipStream_t s) {
    constexpr bool f32 = sizeof(T) == 4;
    const long long BH = static_cast<long long>(a.B) * a.Hkv, R = static_cast<long long>(a.T) * a.G;
    if (a.documents && a.N > 0) {
        const long long n = static_cast<long long>(a.B) * ((a.N + kDocTile - 1) / kDocTile) * kDocTile;
        k_doc_ranges<<<dim3(static_cast<unsigned>((n + 255) / 256)), 256, 0, s>>>(a.documents, a.B, a.N, a.doc_range);
        if (hipError_t e = hipGetLastError()) return e;
    }
    const dim3 grid(static_cast<unsigned>(BH * a.part.splits * a.row_blocks));
    auto run = [&](auto variant, auto mode) {
        constexpr int V = decltype(variant)::value, WK = key_waves(V, f32);
        k_prompt<T, D, row_waves(V), WK, decltype(mode)::value><<<grid, 64 * row_waves(V) * WK, 0, s>>>(a);
    };
    auto modes = [&](auto variant) {
        using std::integral_constant;
        if (a.documents)
            a.score.capped || a.score.slopes ? run(variant, integral_constant<int, kExtra | kDocs>{})
                                             : run(variant, integral_constant<int, kDocs>{});
        else
            a.score.capped || a.score.slopes ? run(variant, integral_constant<int, kExtra>{})
                                             : run(variant, integral_constant<int, 0>{});
    };
    if (a.variant == 0)
        modes(std::integral_constant<int, 0>{});
    else if (a.variant == 1)
        modes(std::integral_constant<int, 1>{});
    else
        modes(std::integral_constant<int, 2>{});
    if (hipError_t e = hipGetLastError()) return e;
    if (a.part.splits > 1) {
        const int per = join_rows<D>(a.part.splits);
        k_prompt_join<T, D><<<dim3(static_cast<unsigned>((BH * R + per - 1) / per)), kJoinThreads, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

size_t plan_prompt(PromptArgs& a, int cus, char* ws) {
    if (cus <= 0) cus = 256;
    const bool f32 = a.dtype == SANTAPP_FP32;
    const long long R = static_cast<long long>(a.T) * a.G, BH = static_cast<long long>(a.B) * a.Hkv;
    // Blocks of 128 rows keep the matrix cores busiest, but under a mask they
    // differ in length and the longest of few set the time, and blocks of 64 hide
    // more of their start.  Causal prompts of 28 query and 4 KV heads of 128, bf16:
    // 2048 tokens 62 us with 448 blocks of 128, 55 with 896 of 64; 4096 tokens
    // 139 and 165.  fp32 (2048 tokens): 354 and 321; 16 heads of 64, 1009 tokens of
    // two sequences: 79, 60, and 54 with 1024 blocks of 32.
    auto blocks_of = [&](int v) { return BH * ((R + 32 * row_waves(v) - 1) / (32 * row_waves(v))); };
    a.variant = variant_of(R);
    if (a.variant == 2 && blocks_of(2) < (f32 ? 8ll : 3ll) * cus) a.variant = 1;
    if (a.variant == 1 && f32 && a.d == 64 && blocks_of(1) >= cus && blocks_of(1) <= 2ll * cus) a.variant = 0;
    const int bk = tile_keys(a.variant, f32);
    const long long blocks = blocks_of(a.variant);
    a.row_blocks = static_cast<int>(blocks / BH);
    // Few blocks: their keys are split until every workgroup slot has work, but
    // into parts long enough to pay for their join (rows x parts x d values): 128
    // keys where rows are few, 512 otherwise, and 64 parts at most (5 of 32768
    // tokens: 26 us with 128, 23 with 64; 256 of 8192 tokens: 114 us with one part,
    // 59 with four)
    long long keys = a.N;
    if (a.score.window > 0) keys = keys < 2ll * a.score.window + a.T ? keys : 2ll * a.score.window + a.T;
    long long splits = per_cu(a.variant, a.d, f32, 1) * static_cast<long long>(cus) / blocks;
    const long long most = keys / (R <= 64 ? 128 : 512), tiles = (keys + bk - 1) / bk;
    splits = splits > most ? most : splits;
    splits = splits > tiles ? tiles : splits;
    a.part.splits = static_cast<int>(splits < 1 ? 1 : splits > 64 ? 64 : splits);
    size_t at = 0;
    if (a.documents) {
        a.doc_range = reinterpret_cast<int2*>(ws);
        at = (static_cast<size_t>(a.B) * ((a.N + kDocTile - 1) / kDocTile) * sizeof(int2) + 255) & ~static_cast<size_t>(255);
    }
    if (a.part.splits > 1) at += place_parts(a.part, BH, R, a.d, ws, at);
    return at;
}

hipError_t launch_prompt(const PromptArgs& a, hipStream_t s) {
    if (a.dtype == SANTAPP_BF16) return a.d == 128 ? launch<bf16_t, 128>(a, s) : launch<bf16_t, 64>(a, s);
    return a.d == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
}

}  // namespace santapp
