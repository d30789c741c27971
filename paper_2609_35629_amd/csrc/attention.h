// Internal interface between the C-ABI layer (api.hip) and the kernels of rotary
// positions, prompt attention and shared-prefix decoding.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "internal.h"

namespace santapp {

// Rotary positions: up to three streams of rows [B, heads, T, d] (queries,
// keys, values), each read once and written once; see rope_kernels.hip.
struct RopeStream {
    const void* in;
    void* out;
    long long ib, ih, it, ob, oh, ot;  // strides in elements
    int heads;
    bool in32, out32;  // fp32 rows, else bf16
    bool rotate;
    bool append;  // written at cache row at + t, if that is one
};

struct RopeArgs {
    RopeStream s[3];
    const double* freqs;   // [pairs] radians per position
    const int* positions;  // [B, T], or null: first + at + t
    const int* at;         // [B], or null: at0
    long long first;
    int at0, capacity, pairs, B, T, d;
    int heads, hstep;      // set by launch_rope
    float magnitude;
    bool interleaved;
};

hipError_t launch_rope(RopeArgs a, int cus, hipStream_t s);

// Attention of query rows over key rows on the matrix cores
// (attention_core.h).  Rows of d contiguous elements; strides in bytes.
struct Rows {
    const char* p;
    long long b, h, t;
};

// How scores are formed: s = scale q.k; s = cap tanh(s / cap) with a cap;
// s -= slope_h |position - key position|; in units of log 2 throughout.
struct ScoreArgs {
    float scale_log2;           // scale log2(e)
    float inv_cap, cap_log2;    // scale / cap, cap log2(e) (cap > 0)
    bool capped;
    const float* slopes;        // [Hq] or null
    int window;                 // keys nearer than this only; 0: all
};

// Where the split parts of a row are kept until they are joined: sums and
// maxima [pairs, splits, rows] (float2) and values [pairs, splits, rows, d].
struct PartArgs {
    float2* ml;
    float* o;
    int splits;
};

struct PromptArgs {
    Rows q, K, V, out;
    ScoreArgs score;
    int B, Hkv, G, T, N, d, offset;
    bool causal;
    santapp_dtype dtype;
    const int* documents;  // [B, N] or null
    const int* prefix;     // [B] or null
    int2* doc_range;       // [B, key tiles of kDocTile] lowest and highest document (documents only)
    PartArgs part;         // splits > 1 only
    int variant, row_blocks;
};

struct PrefixArgs {
    const float* q;    // [P S, Hq, d]
    float* out;        // [P S, Hq, d]
    Rows K, V, sK, sV;
    ScoreArgs score;
    int P, S, Hkv, G, N, T, d;
    santapp_dtype dtype;
    const int* prefix_lengths;  // [P] or null
    const int* lengths;         // [P S] or null
    const int* positions;       // [P S] or null
    PartArgs part, spart;       // of the prompt and of the suffixes
    int variant, row_blocks, srow_blocks;
};

constexpr int kDocTile = 32;  // keys per document range
constexpr long long kMaxRowStep = 1ll << 26;  // bytes between the key rows of a pair

// Launch shapes (host arithmetic only): the variant, row blocks and splits of
// `a`, their places in the workspace at `ws` and its bytes; with ws null, the
// bytes to have (plan_prefix: for this and any shorter suffix).
size_t plan_prompt(PromptArgs& a, int cus, char* ws);
size_t plan_prefix(PrefixArgs& a, int cus, char* ws);

hipError_t launch_prompt(const PromptArgs& a, hipStream_t s);
hipError_t launch_prefix(const PrefixArgs& a, hipStream_t s);

}  // namespace santapp
