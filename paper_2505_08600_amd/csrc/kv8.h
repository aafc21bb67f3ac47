// Device-side view of an 8-bit cache and of the rows a call works on; what kv8.hip and attn_kv8.hip share.
#pragma once
#include "sd_internal.h"

#define KV8_SCALE_MIN 8.673617379884035e-19f // 2^-60

struct Kv8View {
    int8_t *k, *v;
    float *ks, *vs;
    int64_t tokens;
    int32_t kv_heads, hd, n_seq;
    const int64_t *off;
    const int32_t *cap;
    int32_t *status; // or nullptr
};

// Rows of a call.  The public calls index len by sequence id and have one entry per sequence.  A forward pass of the
// draft/verify path has `group` plan slots per sequence, `rows` row slots per sequence of which the first sum of nq[] over the
// group are in use, and len per slot; what its unused slots receive is zeros.
struct Kv8Rows {
    const int32_t *seq_ids, *len, *row_start, *nq;
    int32_t n;     // sequences
    int32_t rows;  // per sequence (row_start == nullptr), or row slots in all
    int32_t group;
    int32_t path;
};

// One sequence of a call.
struct Kv8Seq {
    int32_t b;     // sequence id, -1: out of range
    int32_t len;   // tokens before its rows
    int32_t row0, n_rows;
};

// Lengths and capacities are looked at up to 2^30, so that positions, a length and less than 2^30 more, are plain integers.
#define KV8_MAX_TOKENS (1 << 30)
__device__ __forceinline__ int kv8_length(int len) { return min(max(len, -KV8_MAX_TOKENS), KV8_MAX_TOKENS); }
__device__ __forceinline__ int kv8_capacity(const Kv8View &c, int b) { return min(c.cap[b], KV8_MAX_TOKENS); }

// Rows of sequence j, inside the call's rows whatever row_start holds.
__device__ __forceinline__ int kv8_first_row(const Kv8Rows &rw, int j) { return rw.row_start ? min(max(rw.row_start[j], 0), rw.rows) : j * rw.rows; }
__device__ __forceinline__ int kv8_last_row(const Kv8Rows &rw, int j)
{
    return rw.row_start ? max(min(rw.row_start[j + 1], rw.rows), kv8_first_row(rw, j)) : (j + 1) * rw.rows;
}

// uniform over the wave (every lane calls it)
__device__ __forceinline__ Kv8Seq kv8_seq(const Kv8View &c, const Kv8Rows &rw, int j)
{
    Kv8Seq s;
    s.b = rw.seq_ids ? rw.seq_ids[j * rw.group] : j;
    if (s.b < 0 || s.b >= c.n_seq) s.b = -1;
    s.row0 = kv8_first_row(rw, j);
    s.n_rows = kv8_last_row(rw, j) - s.row0;
    s.len = s.b < 0 ? 0 : kv8_length(rw.len[rw.path ? j * rw.group : s.b]);
    if (rw.path) {
        int t = 0;
        for (int g = threadIdx.x & 63; g < rw.group; g += 64) t += rw.nq[j * rw.group + g];
        for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o, 64);
        s.n_rows = t;
    }
    s.b = __builtin_amdgcn_readfirstlane(s.b), s.len = __builtin_amdgcn_readfirstlane(s.len);
    s.row0 = __builtin_amdgcn_readfirstlane(s.row0), s.n_rows = __builtin_amdgcn_readfirstlane(s.n_rows);
    return s;
}

// Sequence that row r belongs to: the last one whose first row is not behind r.  -1: none.  Uniform over the wave.
__device__ __forceinline__ int kv8_owner(const Kv8Rows &rw, int r)
{
    if (!rw.row_start) return r / rw.rows;
    int n = 0;
    for (int j0 = 0; j0 <= rw.n; j0 += 64) {
        const int j = j0 + (threadIdx.x & 63);
        n += __popcll(__ballot(j <= rw.n && rw.row_start[j < rw.n ? j : rw.n] <= r));
    }
    return n > rw.n ? -1 : n - 1;
}

// ---------------------------------------------------------------- launchers
hipError_t launch_kv8_append(hipStream_t s, const Kv8View &c, const Kv8Rows &rw, int n_rows, int dtype, const void *k, int64_t k_row,
                             int64_t k_head, const void *v, int64_t v_row, int64_t v_head);
hipError_t launch_kv8_read(hipStream_t s, const Kv8View &c, const Kv8Rows &rw, int n_rows, int dtype, void *k, int64_t k_row, int64_t k_head,
                           void *v, int64_t v_row, int64_t v_head);
// The path's step between the QKV projection and attention: adds the projection's slabs, turns queries and keys, quantises keys and
// values into the cache and leaves the queries as fp32 rows [M][H * hd].
hipError_t launch_kv8_rope_append(hipStream_t s, const float *qkv, int n_slabs, size_t slab_stride, PlanView pv, CtxView cv, const Kv8View &c,
                                  int M, int H, const float2 *rope, int max_pos, float *q, bool kv_only);

// What attention is asked for, with one entry per thing the kernels read.
struct Kv8Attn {
    const void *q;
    int64_t q_row, q_head;
    void *out;
    int64_t o_row, o_head;
    float *lse;
    int32_t n_heads, dtype;
    int32_t causal, window, sinks;
    float scale;        // of the scores, in base-2 exponent units
    int32_t out_planes; // 1: out is an activation buffer in two bf16 planes (av), not strided rows
    ActView av;
    int32_t total_rows, max_rows, max_len;
};
int64_t kv8_attn_workspace(const Kv8View &c, const Kv8Rows &rw, const Kv8Attn &a); // bytes
hipError_t launch_kv8_attn(hipStream_t s, const Kv8View &c, const Kv8Rows &rw, const Kv8Attn &a, void *ws, int64_t ws_bytes);
