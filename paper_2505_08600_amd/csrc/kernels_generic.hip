// Reference-quality HIP kernels of the draft/verify path: they work for every
// supported shape in fp32 and bf16.  The fp32 (tiny) configuration runs on these
// alone; bf16 models use the MFMA kernels of the other files where their shape
// constraints hold and fall back here otherwise.
//
// Paper (arXiv 2505.08600): Section 1 / Figure 1 (draft rows, verify rows),
// Section 3.1 (LLaMA blocks; speculative-sampling verification, greedy limit).
#include "lora.h"
#include "sd_internal.h"
#include <algorithm>

#define WAVE 64

// ---------------------------------------------------------------- block helpers
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = WAVE / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, WAVE);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int o = WAVE / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, WAVE));
    return v;
}

// The one-block-per-row kernels (norms, samplers, the verify tail) spend their time waiting in block
// reductions, not computing.  These variants use the cross-lane data path of the vector ALU (DPP) instead
// of LDS shuffles, combine the 16 waves' partial results one entry per lane, and use barriers that wait
// for LDS traffic only, so that global stores issued before a reduction (the updated residual row, the q
// row a sampler has just written) drain behind it instead of stalling its first barrier.
// nothing is moved across it by the scheduler
#define SD_SCHED_FENCE() __builtin_amdgcn_sched_barrier(0)
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ int row16_max(int v)
{
    v = max(v, dpp_i<0xB1>(v));
    v = max(v, dpp_i<0x4E>(v));
    v = max(v, dpp_i<0x141>(v));
    v = max(v, dpp_i<0x140>(v));
    return v;
}
__device__ __forceinline__ float row16_maxf(float v)
{
    v = fmaxf(v, dpp_f<0xB1>(v));
    v = fmaxf(v, dpp_f<0x4E>(v));
    v = fmaxf(v, dpp_f<0x141>(v));
    v = fmaxf(v, dpp_f<0x140>(v));
    return v;
}
__device__ __forceinline__ float wave_max_dpp(float v)
{
    v = row16_maxf(v);
    return fmaxf(fmaxf(lane_f(v, 0), lane_f(v, 16)), fmaxf(lane_f(v, 32), lane_f(v, 48)));
}
// smallest value over the wave's 64 lanes (every lane gets it)
__device__ __forceinline__ int wave_min_i(int v)
{
    int m = row16_max(~v); // ~ reverses the order of ints
    m = max(max(__builtin_amdgcn_readlane(m, 0), __builtin_amdgcn_readlane(m, 16)),
            max(__builtin_amdgcn_readlane(m, 32), __builtin_amdgcn_readlane(m, 48)));
    return ~m;
}
__device__ __forceinline__ int wave_max_i(int v)
{
    const int m = row16_max(v);
    return max(max(__builtin_amdgcn_readlane(m, 0), __builtin_amdgcn_readlane(m, 16)),
               max(__builtin_amdgcn_readlane(m, 32), __builtin_amdgcn_readlane(m, 48)));
}
// 1 / T of a sampling call.  T = inf is the uniform distribution over the columns that are not masked: the smallest
// positive factor makes every finite difference vanish and keeps -inf at weight 0 (0 would turn it into a NaN, and reads as
// "greedy" where a zero factor stands for T == 0).
__device__ __forceinline__ float inv_temperature(float T) { return T > 0.f ? fmaxf(1.0f / T, SD_MIN_INV_T) : 0.f; }
// Value that fills a row past its end, where the exponential must be 0: at the largest temperatures a finite one would not do.
__device__ __forceinline__ float row_filler(float T) { return T > 1e30f ? -INFINITY : -3.0e38f; }
// Inverse-CDF placement inside one thread's four weights (indices i0 .. i0 + 3), the running sum continued from
// `cum`: the first index of positive weight whose inclusive sum exceeds the target, 0x7fffffff if there is none.
// Every thread of a scan evaluates it, whatever its starting sum, and the smallest index wins.  A thread's
// starting sum comes out of a parallel scan and is not bit-equal to its predecessor's sequentially added final
// sum, so a target within rounding of a thread boundary can be "not yet reached" at the end of one thread and
// "already passed" at the start of the next: then the next index of positive weight is the answer (and, because
// of the weight test, never an index the distribution gives no mass to).
__device__ __forceinline__ int first_over(float cum, const float4 f, float target, int i0)
{
    int k = 0x7fffffff;
    cum += f.x;
    if (f.x > 0.f && cum > target) k = i0;
    cum += f.y;
    if (k == 0x7fffffff && f.y > 0.f && cum > target) k = i0 + 1;
    cum += f.z;
    if (k == 0x7fffffff && f.z > 0.f && cum > target) k = i0 + 2;
    cum += f.w;
    if (k == 0x7fffffff && f.w > 0.f && cum > target) k = i0 + 3;
    return k;
}
__device__ __forceinline__ int last_positive(const float4 f, int i0)
{
    return f.w > 0.f ? i0 + 3 : f.z > 0.f ? i0 + 2 : f.y > 0.f ? i0 + 1 : f.x > 0.f ? i0 : -1;
}
// largest value, lowest index among equals
__device__ __forceinline__ void take_better(float &v, int &i, float ov, int oi)
{
    if (ov > v || (ov == v && oi < i)) {
        v = ov;
        i = oi;
    }
}
__device__ __forceinline__ void row16_argmax(float &v, int &i)
{
    take_better(v, i, dpp_f<0xB1>(v), dpp_i<0xB1>(i));
    take_better(v, i, dpp_f<0x4E>(v), dpp_i<0x4E>(i));
    take_better(v, i, dpp_f<0x141>(v), dpp_i<0x141>(i));
    take_better(v, i, dpp_f<0x140>(v), dpp_i<0x140>(i));
}
// Inclusive prefix sum over the 64 lanes: four shifted adds inside each row, then the totals of the rows before.
__device__ __forceinline__ float wave_incl_scan_dpp(float v, int lane)
{
    v += dpp_f<0x111>(v);
    v += dpp_f<0x112>(v);
    v += dpp_f<0x114>(v);
    v += dpp_f<0x118>(v);
    const float t0 = lane_f(v, 15), t1 = lane_f(v, 31), t2 = lane_f(v, 47);
    const int row = lane >> 4;
    const float off = row == 0 ? 0.f : row == 1 ? t0 : row == 2 ? t0 + t1 : (t0 + t1) + t2;
    return off + v;
}
// Sum over a block of exactly 16 waves; every thread gets the result.  red: 16 floats of LDS.
__device__ __forceinline__ float block_sum16(float v, float *red)
{
    const int w = threadIdx.x / WAVE, l = threadIdx.x % WAVE;
    v = wave_sum_dpp(v);
    lds_barrier();
    if (l == 0) red[w] = v;
    lds_barrier();
    return row16_sum(red[l & 15]);
}


// Sum over the block; every thread gets the result.  red: >= 32 floats of LDS.
__device__ float block_sum(float v, float *red)
{
    int w = threadIdx.x / WAVE, l = threadIdx.x % WAVE, nw = (blockDim.x + WAVE - 1) / WAVE;
    v = wave_sum(v);
    __syncthreads();
    if (l == 0) red[w] = v;
    __syncthreads();
    float t = 0.f;
    for (int i = 0; i < nw; i++) t += red[i];
    return t;
}
// The same for any block of whole waves, with barriers that wait for LDS traffic only.
__device__ __forceinline__ float block_sum_lds(float v, float *red)
{
    const int w = threadIdx.x / WAVE, l = threadIdx.x % WAVE, nw = blockDim.x / WAVE;
    v = wave_sum_dpp(v);
    lds_barrier();
    if (l == 0) red[w] = v;
    lds_barrier();
    float t = 0.f;
    for (int i = 0; i < nw; i++) t += red[i];
    return t;
}
__device__ float block_max(float v, float *red)
{
    int w = threadIdx.x / WAVE, l = threadIdx.x % WAVE, nw = (blockDim.x + WAVE - 1) / WAVE;
    v = wave_max(v);
    __syncthreads();
    if (l == 0) red[w] = v;
    __syncthreads();
    float t = red[0];
    for (int i = 1; i < nw; i++) t = fmaxf(t, red[i]);
    return t;
}

// Block-wide (value, index) argmax, ties to the lowest index.
__device__ void block_argmax(float &v, int &idx, float *redv, int *redi)
{
    int w = threadIdx.x / WAVE, l = threadIdx.x % WAVE, nw = (blockDim.x + WAVE - 1) / WAVE;
#pragma unroll
    for (int o = WAVE / 2; o > 0; o >>= 1) {
        float ov = __shfl_xor(v, o, WAVE);
        int oi = __shfl_xor(idx, o, WAVE);
        if (ov > v || (ov == v && oi < idx)) {
            v = ov;
            idx = oi;
        }
    }
    __syncthreads();
    if (l == 0) {
        redv[w] = v;
        redi[w] = idx;
    }
    __syncthreads();
    v = redv[0];
    idx = redi[0];
    for (int i = 1; i < nw; i++)
        if (redv[i] > v || (redv[i] == v && redi[i] < idx)) {
            v = redv[i];
            idx = redi[i];
        }
}

// Exclusive prefix sum of one value per thread over the block.  scratch: >= 32 floats.
__device__ float block_excl_scan(float v, float *scratch)
{
    int w = threadIdx.x / WAVE, l = threadIdx.x % WAVE, nw = (blockDim.x + WAVE - 1) / WAVE;
    float inc = v;
#pragma unroll
    for (int o = 1; o < WAVE; o <<= 1) {
        float t = __shfl_up(inc, o, WAVE);
        if (l >= o) inc += t;
    }
    __syncthreads();
    if (l == WAVE - 1) scratch[w] = inc;
    __syncthreads();
    float base = 0.f;
    for (int i = 0; i < w && i < nw; i++) base += scratch[i];
    return base + inc - v;
}

// ---------------------------------------------------------------- row plan
// Builds the row list of one forward from the device-resident sequence state and
// advances the model's cache length.  One thread per selected sequence.
#define PLAN_THREADS 256
__global__ void plan_kernel(int mode, int R, int n_seq, const int32_t *seq_ids, CtxView cv, int slot, int upto_off,
                            const int32_t *cand, int gamma, int cand_idx, int vocab, PlanView pv)
{
    __shared__ int s_len[PLAN_THREADS]; // cache length after this forward, per sequence slot (single-block launches)
    if (threadIdx.x < PLAN_THREADS) s_len[threadIdx.x] = -1;
    __syncthreads();
    for (int j = blockIdx.x * blockDim.x + threadIdx.x; j < n_seq; j += gridDim.x * blockDim.x) {
        int b = seq_ids ? seq_ids[j] : j;
        if (b < 0 || b >= cv.B) { // refuse out-of-range ids: mark every row unused
            atomicOr(cv.status, 4);
            pv.seq_b[j] = 0;
            pv.seq_kv0[j] = 0;
            pv.seq_nq[j] = 0;
            if (gridDim.x > 1 || n_seq == 1) pv.seq_order[j] = j;
            else s_len[j] = 0;
            for (int r = 0; r < R; r++) {
                pv.row_tok[j * R + r] = 0;
                pv.row_pos[j * R + r] = 0;
                pv.row_b[j * R + r] = 0;
                pv.row_valid[j * R + r] = 0;
            }
            pv.lm_row[j] = j * R;
            continue;
        }
        int n = cv.ntok[b];
        int *kvp = cv.kvlen + (size_t)slot * cv.B + b;
        int kv = *kvp;
        int cap = cv.cap[b];
        int64_t off = cv.off[b];
        int nq = 0, kv0 = kv;
        if (mode == PLAN_CATCHUP) {
            int avail = (n - upto_off) - kv;
            nq = avail < 0 ? 0 : (avail > R ? R : avail);
            // a draft call (upto_off == 0) needs the pending token in its last row: a cache further behind
            // than R tokens would draw its candidates from another position - refuse and flag it
            if (upto_off == 0 && avail > R) {
                atomicOr(cv.status, 64);
                nq = 0;
            }
            // (a sequence whose candidate count is 0 still feeds its catch-up rows, so that its draft cache
            // stays within two tokens of the sequence; its sampler draws nothing)
        } else if (mode == PLAN_CAND) {
            nq = 1;
        } else { // PLAN_VERIFY: rows (pending token, candidates) at positions n-1 ..
            nq = seq_gamma(cv, b, gamma) + 1; // (= R unless the context carries per-sequence candidate counts)
            if (kv != n - 1) atomicOr(cv.status, 2);
            kv0 = n - 1;
        }
        if (n < 1) { // an empty sequence has no pending token
            atomicOr(cv.status, 2);
            nq = 0;
        }
        if (kv0 < 0) kv0 = 0;
        if (kv0 + nq > cap) { // never write beyond the sequence's cache rows
            atomicOr(cv.status, 1);
            nq = cap - kv0 > 0 ? cap - kv0 : 0;
            if (mode == PLAN_VERIFY) nq = 0;
        }
        for (int r = 0; r < R; r++) {
            int row = j * R + r;
            int valid = r < nq;
            int tok = 0;
            if (valid) {
                if (mode == PLAN_CATCHUP) tok = cv.tokens[off + kv0 + r];
                else if (mode == PLAN_CAND) tok = cand[j * gamma + cand_idx];
                else tok = r == 0 ? cv.tokens[off + n - 1] : cand[j * gamma + (r - 1)];
                if (tok < 0 || tok >= vocab) { // never index the embedding table out of range
                    atomicOr(cv.status, 16);
                    tok = 0;
                }
            }
            pv.row_tok[row] = tok;
            pv.row_pos[row] = kv0 + r;
            pv.row_b[row] = b;
            pv.row_valid[row] = valid;
        }
        pv.seq_b[j] = b;
        pv.seq_kv0[j] = kv0;
        pv.seq_nq[j] = nq;
        if (gridDim.x > 1 || n_seq == 1) pv.seq_order[j] = j;
        else s_len[j] = nq > 0 ? kv0 + nq : 0;
        if (mode == PLAN_VERIFY) {
            for (int r = 0; r < R; r++) pv.lm_row[j * R + r] = j * R + r;
        } else {
            pv.lm_row[j] = j * R + (nq > 0 ? nq - 1 : 0);
        }
        *kvp = kv0 + nq;
    }
    // Longest sequences first: attention blocks start in seq_order, so the blocks still running when the
    // grid drains are the short ones.  (A launch of several blocks wrote the identity order above.)
    if (gridDim.x == 1 && n_seq > 1) {
        __syncthreads();
        const int j = threadIdx.x;
        if (j < n_seq) {
            const int mine = s_len[j];
            int rank = 0;
            for (int i = 0; i < n_seq; i++) rank += (s_len[i] > mine) || (s_len[i] == mine && i < j);
            pv.seq_order[rank] = j;
        }
    }
}

// Prefill plan: every selected sequence gets G consecutive row groups of R rows (plan slots j*G .. j*G+G-1),
// group g holding the next pending tokens R*g .. R*g+R-1 of the sequence at cache positions kv + R*g ..;
// groups past the pending tokens stay empty.  Each group is a sequence slot of its own to the kernels that
// follow (its rows attend to everything before them, including the rows of the earlier groups, which the
// cache-append kernel has written by then).  One thread per selected sequence.
__global__ void plan_prefill_kernel(int R, int G, int n_seq, const int32_t *seq_ids, CtxView cv, int slot, int upto_off,
                                    int vocab, PlanView pv)
{
    // one block per sequence; its threads share out the (group, row) pairs
    const int j = blockIdx.x;
    int b = seq_ids ? seq_ids[j] : j;
    int total = 0, kv = 0;
    int64_t off = 0;
    int *kvp = nullptr;
    if (b < 0 || b >= cv.B) { // refuse out-of-range ids: every group stays empty
        if (threadIdx.x == 0) atomicOr(cv.status, 4);
        b = 0;
    } else {
        const int n = cv.ntok[b], cap = cv.cap[b];
        kvp = cv.kvlen + (size_t)slot * cv.B + b;
        kv = *kvp;
        off = cv.off[b];
        if (kv < 0) kv = 0;
        total = (n - upto_off) - kv;
        if (n < 1 && threadIdx.x == 0) atomicOr(cv.status, 2); // an empty sequence has nothing to feed
        if (total < 0 || n < 1) total = 0;
        if (kv + total > cap) { // never write beyond the sequence's cache rows
            if (threadIdx.x == 0) atomicOr(cv.status, 1);
            total = cap - kv > 0 ? cap - kv : 0;
        }
        if (total > R * G) total = R * G;
    }
    __syncthreads(); // every thread has read the cache length before thread 0 advances it
    for (int i = threadIdx.x; i < G * R; i += blockDim.x) {
        const int g = i / R, r = i % R;
        const int sl = j * G + g, kv0 = kv + g * R;
        const int nq = total - g * R < 0 ? 0 : (total - g * R > R ? R : total - g * R);
        const int row = sl * R + r, valid = r < nq;
        int tok = 0;
        if (valid) {
            tok = cv.tokens[off + kv0 + r];
            if (tok < 0 || tok >= vocab) { // never index the embedding table out of range
                atomicOr(cv.status, 16);
                tok = 0;
            }
        }
        pv.row_tok[row] = tok;
        pv.row_pos[row] = kv0 + r;
        pv.row_b[row] = b;
        pv.row_valid[row] = valid;
        if (r == 0) {
            pv.seq_b[sl] = b;
            pv.seq_kv0[sl] = kv0;
            pv.seq_nq[sl] = nq;
            pv.seq_order[sl] = sl;
        }
    }
    if (threadIdx.x == 0) {
        pv.lm_row[j] = total > 0 ? (j * G + (total - 1) / R) * R + (total - 1) % R : j * G * R;
        if (kvp) *kvp = kv + total;
    }
}

hipError_t launch_plan_prefill(hipStream_t s, int R, int G, int n_seq, const int32_t *seq_ids, CtxView cv, int slot,
                               int upto_off, int vocab, PlanView pv)
{
    hipLaunchKernelGGL(plan_prefill_kernel, dim3(n_seq), dim3(PLAN_THREADS), 0, s, R, G, n_seq, seq_ids, cv, slot, upto_off,
                       vocab, pv);
    return hipGetLastError();
}

hipError_t launch_plan(hipStream_t s, int mode, int R, int n_seq, const int32_t *seq_ids, CtxView cv, int slot,
                       int upto_off, const int32_t *cand, int gamma, int cand_idx, int vocab, PlanView pv)
{
    int threads = PLAN_THREADS, blocks = (n_seq + threads - 1) / threads;
    hipLaunchKernelGGL(plan_kernel, dim3(blocks), dim3(threads), 0, s, mode, R, n_seq, seq_ids, cv, slot, upto_off,
                       cand, gamma, cand_idx, vocab, pv);
    return hipGetLastError();
}

// ---------------------------------------------------------------- embedding gather
template <typename T>
__global__ void embed_kernel(const T *E, const int32_t *row_tok, int d, float *x)
{
    int r = blockIdx.x;
    const T *src = E + (size_t)row_tok[r] * d;
    for (int i = threadIdx.x; i < d; i += blockDim.x) x[(size_t)r * d + i] = to_float(src[i]);
}

hipError_t launch_embed(hipStream_t s, int dtype, const void *E, const int32_t *row_tok, int M, int d, float *x)
{
    if (dtype == SD_BF16)
        hipLaunchKernelGGL(embed_kernel<bf16_t>, dim3(M), dim3(256), 0, s, (const bf16_t *)E, row_tok, d, x);
    else
        hipLaunchKernelGGL(embed_kernel<float>, dim3(M), dim3(256), 0, s, (const float *)E, row_tok, d, x);
    return hipGetLastError();
}

// ---------------------------------------------------------------- RMSNorm
// out[j] = T( x[src] * rsqrt(mean(x[src]^2) + eps) * g ), src = row_map ? row_map[j] : j.
template <typename T>
__global__ void rmsnorm_kernel(const float *x, const float *g, const int32_t *row_map, int d, float eps, T *out,
                               ActView av)
{
    __shared__ float red[32];
    int j = blockIdx.x;
    int src = row_map ? row_map[j] : j;
    const float *xr = x + (size_t)src * d;
    float ss = 0.f;
    for (int i = threadIdx.x; i < d; i += blockDim.x) ss += xr[i] * xr[i];
    ss = block_sum(ss, red);
    float inv = 1.0f / sqrtf(ss / (float)d + eps);
    for (int i = threadIdx.x; i < d; i += blockDim.x) store_act(out, act_index(av, j, i, d), av.plane, xr[i] * inv * g[i]);
}

hipError_t launch_rmsnorm(hipStream_t s, int dtype, const float *x, const float *g, const int32_t *row_map,
                          int n_rows, int d, float eps, void *out, ActView out_av)
{
    if (dtype == SD_BF16)
        hipLaunchKernelGGL(rmsnorm_kernel<bf16_t>, dim3(n_rows), dim3(256), 0, s, x, g, row_map, d, eps,
                           (bf16_t *)out, out_av);
    else
        hipLaunchKernelGGL(rmsnorm_kernel<float>, dim3(n_rows), dim3(256), 0, s, x, g, row_map, d, eps,
                           (float *)out, out_av);
    return hipGetLastError();
}

// ---------------------------------------------------------------- generic GEMM  C = A . W^T
// One wave per output column n, 16 rows of A per block row; lanes stride over K.
template <typename T, int MODE>
__global__ __launch_bounds__(256) void gemm_generic_kernel(const T *A, ActView a_av, WeightSeg w, int M, int N,
                                                           int K, float *C, T *Cact, ActView c_av)
{
    int n = blockIdx.x * 4 + threadIdx.x / WAVE;
    int lane = threadIdx.x % WAVE;
    int m0 = blockIdx.y * 16;
    if (n >= N) return;
    const T *W0, *W1 = nullptr;
    int nl = n; // row inside its segment
    if (MODE == GEMM_SWIGLU) {
        W0 = (const T *)w.p[0];
        W1 = (const T *)w.p[1];
    } else {
        int seg = n / w.n_per_seg;
        nl = n - seg * w.n_per_seg;
        W0 = (const T *)w.p[seg];
    }
    float acc[16], acc2[16];
#pragma unroll
    for (int m = 0; m < 16; m++) acc[m] = acc2[m] = 0.f;
    int mcount = M - m0 < 16 ? M - m0 : 16;
    for (int k = lane; k < K; k += WAVE) {
        const size_t wi = weight_index(nl, k, K, w.tiled);
        float wv = to_float(W0[wi]);
        float wv2 = MODE == GEMM_SWIGLU ? to_float(W1[wi]) : 0.f;
#pragma unroll
        for (int m = 0; m < 16; m++) {
            if (m < mcount) {
                float a = load_act(A, act_index(a_av, m0 + m, k, K), a_av.plane);
                acc[m] += a * wv;
                if (MODE == GEMM_SWIGLU) acc2[m] += a * wv2;
            }
        }
    }
#pragma unroll
    for (int m = 0; m < 16; m++) {
        acc[m] = wave_sum(acc[m]);
        if (MODE == GEMM_SWIGLU) acc2[m] = wave_sum(acc2[m]);
    }
    if (lane == 0) {
        for (int m = 0; m < mcount; m++) {
            size_t o = (size_t)(m0 + m) * N + n;
            if (MODE == GEMM_STORE) C[o] = acc[m];
            else if (MODE == GEMM_RESID) C[o] += acc[m];
            else {
                float g = acc[m];
                store_act(Cact, act_index(c_av, m0 + m, n, N), c_av.plane, g / (1.0f + expf(-g)) * acc2[m]);
            }
        }
    }
}

// fp32 models: the same product with 16-byte loads.  One wave per output column and MR rows, lane l takes elements
// 4 l .. 4 l + 3 of every 256, four such chunks (two where 16 rows fill the registers) in flight at once.
// Bound: latency of L2 - a wave of the small fp32 shapes reads a few KiB - so what counts is that all its loads are under
// way before the first is used (the kernel above waits for each 64 elements) and that the rows' sums are finished by
// one lane each.  Measured at 5 rows: 688 -> 256 with residual 16.2 -> 3.2 us, 256 -> 688 gate and up 13.6 -> 3.9 us,
// 256 -> 768 10.4 -> 3.2 us; at one row 344 -> 128 6.3 -> 2.6 us.
// Needs K % 4 == 0 and 16-byte aligned operands (launch_gemm_generic); everything else takes the kernel above.
#define GF_WAVES 2
// NORM: A is the residual stream, its RMSNorm is part of the launch: every wave multiplies the rows by the gains as it
// reads them, adds up their squares beside the products and scales its sums by 1 / rms (row_map: source row of output
// row m).  A norm launch costs the small shapes as much as the GEMM behind it; above 16 rows the waves would repeat too
// much of it (launch_gemm_f32_norm).  Whole step of the tiny pair, 12 norm launches of 67 fewer: 277 -> 233 us; the first
// layer's reads the embedding rows themselves and the projection behind its attention adds to them, five launches of 49
// fewer: 205 -> 196 us.
template <int MODE, int MR, bool NORM>
__global__ __launch_bounds__(GF_WAVES * 64) void gemm_f32_rows_kernel(const float *__restrict__ A, WeightSeg w, int M, int N, int K, float *C,
                                                                      float *__restrict__ Cact, const float *__restrict__ gain,
                                                                      const int32_t *row_map, float eps)
{
    constexpr int U = MR > 8 ? 2 : 4, NM = MODE == GEMM_SWIGLU ? 2 : 1;
    const int n = blockIdx.x * GF_WAVES + (threadIdx.x >> 6), lane = threadIdx.x & 63, m0 = blockIdx.y * MR;
    if (n >= N) return;
    const float *W[NM];
    if (MODE == GEMM_SWIGLU) {
#pragma unroll
        for (int c = 0; c < NM; c++) W[c] = (const float *)w.p[c] + (size_t)n * K;
    } else {
        const int seg = n / w.n_per_seg;
        W[0] = (const float *)(seg == 0 ? w.p[0] : seg == 1 ? w.p[1] : w.p[2]) + (size_t)(n - seg * w.n_per_seg) * K;
    }
    const float *Ar[MR]; // rows past M re-read the last one; never stored
#pragma unroll
    for (int m = 0; m < MR; m++) {
        const int r = min(m0 + m, M - 1);
        Ar[m] = A + (size_t)(NORM && row_map ? row_map[r] : r) * K;
    }
    const size_t o = (size_t)(m0 + lane) * N + n; // lane m finishes row m
    const bool live = lane < MR && m0 + lane < M;
    float resid = 0.f; // GEMM_RESID with a row map: the residual rows are rows of `gain`, an embedding table
    if (MODE == GEMM_RESID && live) resid = row_map ? gain[(size_t)row_map[m0 + lane] * N + n] : C[o];
    float acc[NM][MR], ss[MR];
#pragma unroll
    for (int m = 0; m < MR; m++) {
        ss[m] = 0.f;
#pragma unroll
        for (int c = 0; c < NM; c++) acc[c][m] = 0.f;
    }
    for (int k0 = 4 * lane; k0 < K; k0 += 256 * U) {
        float4 wv[U][NM], av[U][MR], gv[U];
#pragma unroll
        for (int u = 0; u < U; u++) { // (chunks past the end re-read the lane's first one; not multiplied)
            const int k = k0 + 256 * u < K ? k0 + 256 * u : k0;
#pragma unroll
            for (int c = 0; c < NM; c++) wv[u][c] = *(const float4 *)(W[c] + k);
#pragma unroll
            for (int m = 0; m < MR; m++) av[u][m] = *(const float4 *)(Ar[m] + k);
            if (NORM) gv[u] = *(const float4 *)(gain + k);
        }
#pragma unroll
        for (int u = 0; u < U; u++)
            if (k0 + 256 * u < K) {
                if (NORM) {
#pragma unroll
                    for (int m = 0; m < MR; m++) {
                        float4 &a = av[u][m];
                        ss[m] = fmaf(a.x, a.x, fmaf(a.y, a.y, fmaf(a.z, a.z, fmaf(a.w, a.w, ss[m]))));
                        a.x *= gv[u].x;
                        a.y *= gv[u].y;
                        a.z *= gv[u].z;
                        a.w *= gv[u].w;
                    }
                }
#pragma unroll
                for (int c = 0; c < NM; c++)
#pragma unroll
                    for (int m = 0; m < MR; m++) {
                        acc[c][m] = fmaf(av[u][m].x, wv[u][c].x, acc[c][m]);
                        acc[c][m] = fmaf(av[u][m].y, wv[u][c].y, acc[c][m]);
                        acc[c][m] = fmaf(av[u][m].z, wv[u][c].z, acc[c][m]);
                        acc[c][m] = fmaf(av[u][m].w, wv[u][c].w, acc[c][m]);
                    }
            }
    }
    float v[NM];
#pragma unroll
    for (int c = 0; c < NM; c++) {
        v[c] = 0.f;
#pragma unroll
        for (int m = 0; m < MR; m++) {
            const float t = wave_sum_dpp(acc[c][m]);
            v[c] = lane == m ? t : v[c];
        }
    }
    if (NORM) {
        float q = 0.f;
#pragma unroll
        for (int m = 0; m < MR; m++) {
            const float t = wave_sum_dpp(ss[m]);
            q = lane == m ? t : q;
        }
        const float inv = 1.0f / sqrtf(q / (float)K + eps);
#pragma unroll
        for (int c = 0; c < NM; c++) v[c] *= inv;
    }
    if (!live) return;
    if (MODE == GEMM_SWIGLU) Cact[o] = v[0] / (1.0f + expf(-v[0])) * v[NM - 1];
    else C[o] = MODE == GEMM_RESID ? resid + v[0] : v[0];
}

template <int MODE, bool NORM>
static void gemm_f32_rows(hipStream_t s, const float *A, WeightSeg w, int M, int N, int K, float *C, float *Cact, const float *gain,
                          const int32_t *row_map, float eps)
{
    const dim3 block(GF_WAVES * 64);
    const int bx = (N + GF_WAVES - 1) / GF_WAVES;
#define SD_GF(MR)                                                                                                            \
    hipLaunchKernelGGL((gemm_f32_rows_kernel<MODE, MR, NORM>), dim3(bx, (M + MR - 1) / MR), block, 0, s, A, w, M, N, K, C, Cact, gain, \
                       row_map, eps)
    if (M == 1) SD_GF(1);
    else if (M == 2) SD_GF(2);
    else if (M <= 5) SD_GF(5);
    else if (M <= 8) SD_GF(8);
    else SD_GF(16);
#undef SD_GF
}

// RMSNorm of x's rows and the product behind it in one launch; hipErrorNotSupported where the two belong apart.
hipError_t launch_gemm_f32_norm(hipStream_t s, int mode, const float *x, const float *gain, const int32_t *row_map, float eps, WeightSeg w,
                                int M, int N, int K, float *C, float *Cact)
{
    const uintptr_t addr = (uintptr_t)x | (uintptr_t)gain | (uintptr_t)w.p[0] | (uintptr_t)w.p[1] | (uintptr_t)w.p[2];
    if (M > 16 || K % 4 != 0 || (addr & 15) || w.tiled || (mode != GEMM_STORE && mode != GEMM_SWIGLU)) return hipErrorNotSupported;
    if (mode == GEMM_STORE) gemm_f32_rows<GEMM_STORE, true>(s, x, w, M, N, K, C, nullptr, gain, row_map, eps);
    else gemm_f32_rows<GEMM_SWIGLU, true>(s, x, w, M, N, K, nullptr, Cact, gain, row_map, eps);
    return hipGetLastError();
}

// C = the embedding rows of the tokens + A . W^T: a projection onto residual rows that no launch has gathered.
hipError_t launch_gemm_f32_embed_resid(hipStream_t s, const float *A, WeightSeg w, int M, int N, int K, float *C, const float *E,
                                       const int32_t *row_tok)
{
    const uintptr_t addr = (uintptr_t)A | (uintptr_t)w.p[0];
    if (M > 16 || K % 4 != 0 || (addr & 15) || w.tiled) return hipErrorNotSupported;
    gemm_f32_rows<GEMM_RESID, false>(s, A, w, M, N, K, C, nullptr, E, row_tok, 0.f);
    return hipGetLastError();
}

// Row-major -> tiled weight order, one 16-byte piece per thread (destination-linear, so stores coalesce).
__global__ __launch_bounds__(256) void retile_bf16_kernel(const uint4 *__restrict__ src, uint4 *__restrict__ dst,
                                                          int N, int K)
{
    const size_t n_vec = (size_t)N * K / 8;
    for (size_t v = (size_t)blockIdx.x * 256 + threadIdx.x; v < n_vec; v += (size_t)gridDim.x * 256) {
        const size_t step = v >> 8;            // 256 pieces per 16 x 128 step
        const int piece = (int)(v & 255);
        const int i = piece >> 6, g = (piece >> 4) & 3, r = piece & 15;
        const size_t steps_per_tile = (size_t)(K >> 7);
        const size_t n = (step / steps_per_tile) * 16 + r;
        const size_t k = (step % steps_per_tile) * 128 + i * 32 + g * 8;
        dst[v] = src[(n * K + k) / 8];
    }
}

hipError_t launch_retile_bf16(hipStream_t s, const void *src, void *dst, int N, int K)
{
    if (N % 16 != 0 || K % 128 != 0) return hipErrorInvalidValue;
    const size_t n_vec = (size_t)N * K / 8;
    const int blocks = (int)std::min<size_t>((n_vec + 255) / 256, 8192);
    hipLaunchKernelGGL(retile_bf16_kernel, dim3(blocks), dim3(256), 0, s, (const uint4 *)src, (uint4 *)dst, N, K);
    return hipGetLastError();
}

template <typename T>
static void gemm_generic_dispatch(hipStream_t s, int mode, const void *A, ActView a_av, WeightSeg w, int M, int N,
                                  int K, float *C, void *Cact, ActView c_av)
{
    dim3 grid((N + 3) / 4, (M + 15) / 16), block(256);
    if (mode == GEMM_STORE)
        hipLaunchKernelGGL((gemm_generic_kernel<T, GEMM_STORE>), grid, block, 0, s, (const T *)A, a_av, w, M, N, K,
                           C, (T *)Cact, c_av);
    else if (mode == GEMM_RESID)
        hipLaunchKernelGGL((gemm_generic_kernel<T, GEMM_RESID>), grid, block, 0, s, (const T *)A, a_av, w, M, N, K,
                           C, (T *)Cact, c_av);
    else
        hipLaunchKernelGGL((gemm_generic_kernel<T, GEMM_SWIGLU>), grid, block, 0, s, (const T *)A, a_av, w, M, N, K,
                           C, (T *)Cact, c_av);
}

hipError_t launch_gemm_generic(hipStream_t s, int dtype, int mode, const void *A, ActView a_av, WeightSeg w, int M,
                               int N, int K, float *C, void *Cact, ActView c_av)
{
    const uintptr_t addr = (uintptr_t)A | (uintptr_t)w.p[0] | (uintptr_t)w.p[1] | (uintptr_t)w.p[2];
    if (dtype == SD_FP32 && K % 4 == 0 && !(addr & 15) && !w.tiled && !a_av.sm && !c_av.sm) {
        if (mode == GEMM_STORE) gemm_f32_rows<GEMM_STORE, false>(s, (const float *)A, w, M, N, K, C, nullptr, nullptr, nullptr, 0.f);
        else if (mode == GEMM_RESID) gemm_f32_rows<GEMM_RESID, false>(s, (const float *)A, w, M, N, K, C, nullptr, nullptr, nullptr, 0.f);
        else gemm_f32_rows<GEMM_SWIGLU, false>(s, (const float *)A, w, M, N, K, nullptr, (float *)Cact, nullptr, nullptr, 0.f);
        return hipGetLastError();
    }
    if (dtype == SD_BF16) gemm_generic_dispatch<bf16_t>(s, mode, A, a_av, w, M, N, K, C, Cact, c_av);
    else gemm_generic_dispatch<float>(s, mode, A, a_av, w, M, N, K, C, Cact, c_av);
    return hipGetLastError();
}

// ---------------------------------------------------------------- RoPE + KV append
// Embedding gather fused with the first layer's RMSNorm: x[r] = E[token_r]; out[r] = rmsnorm(x[r]) * g.
// Row r of one forward, by a whole block (red: 32 floats of LDS).  The element-wise form has the same
// element-to-thread assignment and reduction as rmsnorm_kernel (identical to the two separate launches); the
// vector form sums the squares in another order.
// bf16 rows whose width is a multiple of 8: 16-byte loads and stores, the row kept in registers between the two
// passes (a thread's 8 columns stay inside one 128-column step of the step-major order).
__device__ void embed_rmsnorm_row_vec(const bf16_t *E, int tok, int r, int d, float *x, const float *g, float eps,
                                      bf16_t *out, ActView av, float *red)
{
    constexpr int KEEP = 4; // 8-column pieces a thread holds, with their gains (d <= 8 * KEEP * blockDim.x, else the rest is re-read)
    const uint4 *src = (const uint4 *)(E + (size_t)tok * d);
    float *xr = x + (size_t)r * d;
    const int npiece = d >> 3, bd = blockDim.x;
    uint4 raw[KEEP];
    float4 gain[KEEP][2];
    float ss = 0.f;
    auto unpack = [](const uint4 w, float *f) {
        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; e++) {
            f[2 * e] = __uint_as_float(ws[e] << 16);
            f[2 * e + 1] = __uint_as_float(ws[e] & 0xffff0000u);
        }
    };
    auto take = [&](int p, const uint4 w) {
        float f[8];
        unpack(w, f);
        *(float4 *)(xr + 8 * p) = make_float4(f[0], f[1], f[2], f[3]);
        *(float4 *)(xr + 8 * p + 4) = make_float4(f[4], f[5], f[6], f[7]);
#pragma unroll
        for (int e = 0; e < 8; e++) ss += f[e] * f[e];
    };
    auto give = [&](int p, const uint4 w, const float4 g0, const float4 g1, float inv) {
        float f[8];
        unpack(w, f);
        const size_t o = act_index(av, r, 8 * p, d);
        store_act4(out, o, av.plane, f[0] * inv * g0.x, f[1] * inv * g0.y, f[2] * inv * g0.z, f[3] * inv * g0.w);
        store_act4(out, o + 4, av.plane, f[4] * inv * g1.x, f[5] * inv * g1.y, f[6] * inv * g1.z, f[7] * inv * g1.w);
    };
#pragma unroll
    for (int it = 0; it < KEEP; it++) {
        const int p = threadIdx.x + it * bd;
        if (p < npiece) {
            raw[it] = src[p];
            gain[it][0] = *(const float4 *)(g + 8 * p);
            gain[it][1] = *(const float4 *)(g + 8 * p + 4);
        }
    }
#pragma unroll
    for (int it = 0; it < KEEP; it++) {
        const int p = threadIdx.x + it * bd;
        if (p < npiece) take(p, raw[it]);
    }
    for (int p = threadIdx.x + KEEP * bd; p < npiece; p += bd) take(p, src[p]);
    ss = block_sum_lds(ss, red);
    const float inv = 1.0f / sqrtf(ss / (float)d + eps);
#pragma unroll
    for (int it = 0; it < KEEP; it++) {
        const int p = threadIdx.x + it * bd;
        if (p < npiece) give(p, raw[it], gain[it][0], gain[it][1], inv);
    }
    for (int p = threadIdx.x + KEEP * bd; p < npiece; p += bd)
        give(p, src[p], *(const float4 *)(g + 8 * p), *(const float4 *)(g + 8 * p + 4), inv);
}
template <typename T>
__device__ void embed_rmsnorm_row(const T *E, int tok, int r, int d, float *x, const float *g, float eps, T *out,
                                  ActView av, float *red)
{
    if constexpr (sizeof(T) == 2) {
        if ((d & 7) == 0) { // (uniform)
            embed_rmsnorm_row_vec(E, tok, r, d, x, g, eps, out, av, red);
            return;
        }
    }
    const T *src = E + (size_t)tok * d;
    float *xr = x + (size_t)r * d;
    float ss = 0.f;
    for (int i = threadIdx.x; i < d; i += blockDim.x) {
        const float v = to_float(src[i]);
        xr[i] = v;
        ss += v * v;
    }
    ss = block_sum(ss, red);
    const float inv = 1.0f / sqrtf(ss / (float)d + eps);
    for (int i = threadIdx.x; i < d; i += blockDim.x)
        store_act(out, act_index(av, r, i, d), av.plane, to_float(src[i]) * inv * g[i]);
}

template <typename T>
__global__ __launch_bounds__(256) void embed_rmsnorm_kernel(const T *E, const int32_t *row_tok, int d, float *x,
                                                            const float *g, float eps, T *out, ActView av)
{
    __shared__ float red[32];
    embed_rmsnorm_row(E, row_tok[blockIdx.x], blockIdx.x, d, x, g, eps, out, av, red);
}

hipError_t launch_embed_rmsnorm(hipStream_t s, int dtype, const void *E, const int32_t *row_tok, int M, int d, float *x,
                                const float *g, float eps, void *out, ActView out_av)
{
    if (dtype == SD_BF16)
        hipLaunchKernelGGL(embed_rmsnorm_kernel<bf16_t>, dim3(M), dim3(256), 0, s, (const bf16_t *)E, row_tok, d, x, g,
                           eps, (bf16_t *)out, out_av);
    else
        hipLaunchKernelGGL(embed_rmsnorm_kernel<float>, dim3(M), dim3(256), 0, s, (const float *)E, row_tok, d, x, g,
                           eps, (float *)out, out_av);
    return hipGetLastError();
}

// qkv: fp32 [M][3*HD] (q | k | v).  Rotates q and k of every valid row at its
// position (rotate-half pairing), writes q to qbuf and k, v into the cache in
// place: K in 32-token tiles in MFMA operand order (kt_offset), V in 32-token transposed tiles (vt_offset).
// Residual update fused with the next RMSNorm: x[src] += sum of the split-K slabs of the
// preceding GEMM (added in slab order), then out[j] = rmsnorm(x[src]) * g.  One block of 1024
// threads per row; the loads of all slabs of an element are independent and go out together.
#define ROPE_MAX_SLABS 8
// (MAX_SLABS: 8 covers the K splits of the GEMMs; 16 the per-head slabs an attention kernel that applies the
// output projection itself leaves for a small model)
template <typename T, int ADDNORM_MAX_SLABS>
__global__ __launch_bounds__(1024) void add_rmsnorm_kernel(float *x, const float *part, int n_slabs, size_t slab_stride,
                                                           const float *g, const int32_t *row_map, int d, float eps,
                                                           T *out, ActView av)
{
    __shared__ float red[16];
    int j = blockIdx.x;
    int src = row_map ? row_map[j] : j;
    float *xr = x + (size_t)src * d;
    const float *pr = part + (size_t)src * d;
    float ss = 0.f;
    const int nvec = d / 4; // d is a multiple of 4 (checked at load)
    constexpr int KEEP = 2; // vectors of the row a thread keeps in registers (d <= 8192)
    float4 keep[KEEP], gain[KEEP];
    int it = 0;
    for (int v = threadIdx.x; v < nvec; v += blockDim.x, it++) {
        float4 a = *(const float4 *)(xr + 4 * v);
        float4 p[ADDNORM_MAX_SLABS];
#pragma unroll
        for (int s = 0; s < ADDNORM_MAX_SLABS; s++)
            if (s < n_slabs) p[s] = *(const float4 *)(pr + (size_t)s * slab_stride + 4 * v);
        // the gains are needed only after the reduction; loaded there they would add a memory round trip
        if (it < KEEP) gain[it] = *(const float4 *)(g + 4 * v);
#pragma unroll
        for (int s = 0; s < ADDNORM_MAX_SLABS; s++)
            if (s < n_slabs) {
                a.x += p[s].x;
                a.y += p[s].y;
                a.z += p[s].z;
                a.w += p[s].w;
            }
        *(float4 *)(xr + 4 * v) = a;
        if (it < KEEP) keep[it] = a;
        ss += a.x * a.x + a.y * a.y + a.z * a.z + a.w * a.w;
    }
    ss = block_sum16(ss, red); // 1024 threads; does not wait for the residual stores above
    if (nvec > KEEP * (int)blockDim.x) __syncthreads(); // wider rows are read back below: let the stores land
    float inv = 1.0f / sqrtf(ss / (float)d + eps);
    it = 0;
    for (int v = threadIdx.x; v < nvec; v += blockDim.x, it++) {
        const float4 a = it < KEEP ? keep[it] : *(const float4 *)(xr + 4 * v);
        const float4 gg = it < KEEP ? gain[it] : *(const float4 *)(g + 4 * v);
        const size_t o = act_index(av, j, 4 * v, d); // 4 consecutive columns stay inside one K step
        store_act4(out, o, av.plane, a.x * inv * gg.x, a.y * inv * gg.y, a.z * inv * gg.z, a.w * inv * gg.w);
    }
}

hipError_t launch_add_rmsnorm(hipStream_t s, int dtype, float *x, const float *part, int n_slabs, size_t slab_stride,
                              const float *g, const int32_t *row_map, int n_rows, int d, float eps, void *out,
                              ActView out_av)
{
    if (n_slabs > 16 || (d & 3)) return hipErrorInvalidValue;
    if (dtype == SD_BF16 && n_slabs > 8)
        hipLaunchKernelGGL((add_rmsnorm_kernel<bf16_t, 16>), dim3(n_rows), dim3(1024), 0, s, x, part, n_slabs, slab_stride,
                           g, row_map, d, eps, (bf16_t *)out, out_av);
    else if (dtype == SD_BF16)
        hipLaunchKernelGGL((add_rmsnorm_kernel<bf16_t, 8>), dim3(n_rows), dim3(1024), 0, s, x, part, n_slabs, slab_stride,
                           g, row_map, d, eps, (bf16_t *)out, out_av);
    else if (n_slabs > 8)
        return hipErrorInvalidValue;
    else
        hipLaunchKernelGGL((add_rmsnorm_kernel<float, 8>), dim3(n_rows), dim3(1024), 0, s, x, part, n_slabs, slab_stride,
                           g, row_map, d, eps, (float *)out, out_av);
    return hipGetLastError();
}

// ---------------------------------------------------------------- low-rank adapters
// Measured at width 768, rank 8: 4.6 us for 32 or 64 rows and one or three projections (18.9 us with one block of 256
// threads per row, all projections in it, the factors fetched after the dot products); below that the launch itself remains.
template <typename T, int RQ>
__global__ __launch_bounds__(LORA_WAVES * 64) void lora_delta_kernel(const T *X, ActView x_av, int K, LoraArgs la)
{
    lora_block<T, RQ, LORA_WAVES>(X, x_av, K, la, blockIdx.x, blockIdx.y, blockIdx.z);
}

template <typename T>
static hipError_t lora_launch(hipStream_t s, const T *X, ActView x_av, int M, int K, const LoraArgs &la)
{
    const bool vec = la.rank % 4 == 0 && !(((uintptr_t)la.b0 | (uintptr_t)la.b1 | (uintptr_t)la.b2) & 15);
    const dim3 grid(M, la.n_proj, (la.N + lora_part(LORA_WAVES) - 1) / lora_part(LORA_WAVES)), block(LORA_WAVES * 64);
#define SD_LORA(RQ_) hipLaunchKernelGGL((lora_delta_kernel<T, RQ_>), grid, block, 0, s, X, x_av, K, la)
    if (!vec) SD_LORA(0);
    else if (la.rank == 4) SD_LORA(1);
    else if (la.rank == 8) SD_LORA(2);
    else if (la.rank == 12) SD_LORA(3);
    else SD_LORA(4);
#undef SD_LORA
    return hipGetLastError();
}

bool lora_valid(int M, int K, const LoraArgs &la)
{
    return M >= 1 && K >= 4 && !(K & 3) && K <= LORA_MAX_K && la.n_proj >= 1 && la.n_proj <= 3 && la.rank >= 1 && la.rank <= LORA_MAX_RANK &&
           la.adapter;
}
hipError_t launch_lora_delta(hipStream_t s, int dtype, const void *X, ActView x_av, int M, int K, const LoraArgs &la)
{
    if (!lora_valid(M, K, la)) return hipErrorInvalidValue;
    if (dtype == SD_BF16) return lora_launch(s, (const bf16_t *)X, x_av, M, K, la);
    return lora_launch(s, (const float *)X, x_av, M, K, la);
}

// KV: the rows of `qkv` hold keys and values only, and no queries are wanted (the last layer of a prefill).
template <typename T, bool KV>
__global__ void rope_append_kernel(const float *qkv, int n_slabs, size_t slab_stride, PlanView pv, CtxView cv, int H,
                                   int hd, const float2 *rope,
                                   int max_pos, T *qbuf, ActView q_av, T *Kl, T *Vtl, int64_t total_cap)
{
    int r = blockIdx.x;
    int HD = H * hd, half = hd / 2;
    int valid = pv.row_valid[r];
    int pos = pv.row_pos[r];
    if (pos >= max_pos) {
        if (threadIdx.x == 0 && valid) atomicOr(cv.status, 8);
        valid = 0;
    }
    const float *row = qkv + (size_t)r * (KV ? 2 : 3) * HD - (KV ? HD : 0);
    int64_t off = cv.off[pv.row_b[r]];
    for (int i = threadIdx.x; i < H * half; i += blockDim.x) {
        int h = i / half, e = i % half;
        if (!valid) {
            if (KV) continue;
            store_act(qbuf, act_index(q_av, r, h * hd + e, HD), q_av.plane, 0.f);
            store_act(qbuf, act_index(q_av, r, h * hd + e + half, HD), q_av.plane, 0.f);
            continue;
        }
        float2 cs = rope[(size_t)pos * half + e];
        float q0 = 0.f, q1 = 0.f, k0 = 0.f, k1 = 0.f, v0 = 0.f, v1 = 0.f;
        float ld[ROPE_MAX_SLABS][6];
#pragma unroll
        for (int sl = 0; sl < ROPE_MAX_SLABS; sl++) // split-K slabs of the QKV GEMM: all loads go out first
            if (sl < n_slabs) {
                const float *rs = row + (size_t)sl * slab_stride;
                ld[sl][0] = KV ? 0.f : rs[h * hd + e];
                ld[sl][1] = KV ? 0.f : rs[h * hd + e + half];
                ld[sl][2] = rs[HD + h * hd + e];
                ld[sl][3] = rs[HD + h * hd + e + half];
                ld[sl][4] = rs[2 * HD + h * hd + e];
                ld[sl][5] = rs[2 * HD + h * hd + e + half];
            }
#pragma unroll
        for (int sl = 0; sl < ROPE_MAX_SLABS; sl++) // ... and are added in slab order
            if (sl < n_slabs) {
                q0 += ld[sl][0];
                q1 += ld[sl][1];
                k0 += ld[sl][2];
                k1 += ld[sl][3];
                v0 += ld[sl][4];
                v1 += ld[sl][5];
            }
        if (!KV) {
            store_act(qbuf, act_index(q_av, r, h * hd + e, HD), q_av.plane, q0 * cs.x - q1 * cs.y);
            store_act(qbuf, act_index(q_av, r, h * hd + e + half, HD), q_av.plane, q1 * cs.x + q0 * cs.y);
        }
        T *kh = Kl + (size_t)h * total_cap * hd;
        kh[kt_offset(hd, off + pos, e)] = from_float<T>(k0 * cs.x - k1 * cs.y);
        kh[kt_offset(hd, off + pos, e + half)] = from_float<T>(k1 * cs.x + k0 * cs.y);
        T *vh = Vtl + (size_t)h * hd * total_cap;
        vh[vt_offset(hd, off + pos, e)] = from_float<T>(v0);
        vh[vt_offset(hd, off + pos, e + half)] = from_float<T>(v1);
    }
}

// The same step for bf16 models with head width 64 or 128, one block per (head, group of up to 16 rows whose
// positions follow each other).  The row-per-block kernel above writes every cache element with a 2-byte store
// of its own - V elements of consecutive dimensions lie 64 bytes apart in the transposed tiles - and takes 27 us
// for 576 rows of the 7B shape.  Here a thread owns 8 consecutive dimensions of both rotary halves of one row:
// float4 loads of the slabs (added in slab order, like above: same bits), 16-byte stores of the two q planes and
// of the K pieces (8 consecutive dimensions of a token are one piece of the operand-order tile); the V values go
// through LDS so that a thread can write the 16 tokens of one dimension as 32 contiguous bytes when the group is
// full and starts at a multiple of 16 (every prefill group of a fresh prompt), and token by token otherwise.
template <int HD, bool KV>
__global__ __launch_bounds__(HD) void rope_append_group_kernel(const float *__restrict__ qkv, int n_slabs, size_t slab_stride,
                                                               PlanView pv, CtxView cv, int R, int H,
                                                               const float2 *__restrict__ rope, int max_pos,
                                                               uint16_t *__restrict__ qbuf, ActView q_av,
                                                               uint16_t *__restrict__ Kl, uint16_t *__restrict__ Vtl,
                                                               int64_t total_cap)
{
    constexpr int HALF = HD / 2, GPR = HALF / 8; // 8-dimension groups per rotary half
    __shared__ __attribute__((aligned(16))) uint16_t sV[16][HD + 8];
    __shared__ int s_pos[16];
    const int h = blockIdx.x, j = blockIdx.y;
    const int i = threadIdx.x / GPR, g = threadIdx.x % GPR; // row of the group, dimension group
    const int HDm = H * HD;
    const int r = j * R + min(i, R - 1);
    int valid = i < R && pv.row_valid[r];
    const int pos = pv.row_pos[r];
    if (valid && pos >= max_pos) {
        if (g == 0 && h == 0) atomicOr(cv.status, 8);
        valid = 0;
    }
    const int64_t off = cv.off[pv.row_b[r]];
    const int d0 = 8 * g, d1 = HALF + 8 * g;
    float q[16], k[16], v[16]; // [0..7]: dimensions d0.., [8..15]: d1..
#pragma unroll
    for (int e = 0; e < 16; e++) q[e] = k[e] = v[e] = 0.f;
    if (valid) {
        const float *base = qkv + (size_t)r * (KV ? 2 : 3) * HDm - (KV ? HDm : 0) + h * HD;
        for (int sl = 0; sl < n_slabs; sl++) { // split-K slabs of the QKV GEMM, added in slab order
            const float *rs = base + (size_t)sl * slab_stride;
            float4 ld[12];
#pragma unroll
            for (int m = KV ? 1 : 0; m < 3; m++) {
                ld[4 * m + 0] = *(const float4 *)(rs + m * HDm + d0);
                ld[4 * m + 1] = *(const float4 *)(rs + m * HDm + d0 + 4);
                ld[4 * m + 2] = *(const float4 *)(rs + m * HDm + d1);
                ld[4 * m + 3] = *(const float4 *)(rs + m * HDm + d1 + 4);
            }
#pragma unroll
            for (int c = 0; c < 4; c++) {
                const float4 a = ld[KV ? 4 + c : c], b = ld[4 + c], w = ld[8 + c];
                if (!KV) q[4 * c + 0] += a.x, q[4 * c + 1] += a.y, q[4 * c + 2] += a.z, q[4 * c + 3] += a.w;
                k[4 * c + 0] += b.x, k[4 * c + 1] += b.y, k[4 * c + 2] += b.z, k[4 * c + 3] += b.w;
                v[4 * c + 0] += w.x, v[4 * c + 1] += w.y, v[4 * c + 2] += w.z, v[4 * c + 3] += w.w;
            }
        }
        const float2 *cs = rope + (size_t)pos * HALF + d0;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float2 c = cs[e];
            const float qa = q[e] * c.x - q[8 + e] * c.y, qb = q[8 + e] * c.x + q[e] * c.y;
            const float ka = k[e] * c.x - k[8 + e] * c.y, kb = k[8 + e] * c.x + k[e] * c.y;
            q[e] = qa, q[8 + e] = qb, k[e] = ka, k[8 + e] = kb;
        }
    }
    if (!KV && i < R) { // q planes (zeros for rows without a token), 8 consecutive columns inside one K step
#pragma unroll
        for (int hf = 0; hf < 2; hf++) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; e++) bf16x2_split(q[8 * hf + 2 * e], q[8 * hf + 2 * e + 1], hi[e], lo[e]);
            const size_t o = act_index(q_av, r, h * HD + (hf ? d1 : d0), HDm);
            *(uint4 *)(qbuf + o) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            *(uint4 *)(qbuf + o + q_av.plane) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
    }
    if (valid) {
        uint16_t *kh = Kl + (size_t)h * total_cap * HD;
#pragma unroll
        for (int hf = 0; hf < 2; hf++) {
            uint32_t p[4];
#pragma unroll
            for (int e = 0; e < 4; e++) p[e] = bf16x2_bits_rne(k[8 * hf + 2 * e], k[8 * hf + 2 * e + 1]);
            *(uint4 *)(kh + kt_offset(HD, off + pos, hf ? d1 : d0)) = make_uint4(p[0], p[1], p[2], p[3]);
#pragma unroll
            for (int e = 0; e < 4; e++) p[e] = bf16x2_bits_rne(v[8 * hf + 2 * e], v[8 * hf + 2 * e + 1]);
            *(uint4 *)&sV[i][hf ? d1 : d0] = make_uint4(p[0], p[1], p[2], p[3]);
        }
    }
    if (g == 0) s_pos[i] = valid ? pos : -1;
    __syncthreads();
    // V: thread d writes dimension d of the group's tokens
    const int d = threadIdx.x;
    uint16_t *vh = Vtl + (size_t)h * HD * total_cap;
    const int p0 = s_pos[0];
    bool run16 = p0 >= 0 && (p0 & 15) == 0;
#pragma unroll
    for (int t = 1; t < 16; t++) run16 = run16 && s_pos[t] == p0 + t;
    const int64_t off0 = cv.off[pv.row_b[j * R]]; // (one sequence per group)
    if (run16) {
        uint32_t p[8];
#pragma unroll
        for (int t = 0; t < 8; t++) p[t] = (uint32_t)sV[2 * t][d] | ((uint32_t)sV[2 * t + 1][d] << 16);
        uint16_t *dst = vh + vt_offset(HD, off0 + p0, d); // 16 tokens inside one 32-token tile: 32 contiguous bytes
        *(uint4 *)dst = make_uint4(p[0], p[1], p[2], p[3]);
        *(uint4 *)(dst + 8) = make_uint4(p[4], p[5], p[6], p[7]);
    } else {
        for (int t = 0; t < 16; t++)
            if (s_pos[t] >= 0) vh[vt_offset(HD, off0 + s_pos[t], d)] = sV[t][d];
    }
}

int g_rope_group = 1; // option "rope_group": 0 keeps the row-per-block kernel for bf16 models too
hipError_t launch_rope_append(hipStream_t s, int dtype, const float *qkv, int n_slabs, size_t slab_stride, PlanView pv,
                              CtxView cv, int M, int R, int H, int hd, const float2 *rope, int max_pos, void *qbuf,
                              ActView q_av, void *Kl, void *Vtl, int64_t total_cap, bool kv_only)
{
    if (n_slabs > ROPE_MAX_SLABS) return hipErrorInvalidValue;
    if (dtype == SD_BF16 && g_rope_group && R >= 1 && R <= 16 && M % R == 0 && (hd == 64 || hd == 128) && H <= 65535 &&
        M / R <= 65535 && (q_av.plane & 7) == 0 && ((uintptr_t)qbuf & 15) == 0 && ((uintptr_t)Kl & 15) == 0 &&
        ((uintptr_t)Vtl & 15) == 0 && ((uintptr_t)qkv & 15) == 0 && (slab_stride & 3) == 0 && total_cap % 64 == 0) {
#define SD_ROPE_GROUP(HD_, KV_)                                                                                               \
    hipLaunchKernelGGL((rope_append_group_kernel<HD_, KV_>), dim3(H, M / R), dim3(HD_), 0, s, qkv, n_slabs, slab_stride, pv, cv, R, H, \
                       rope, max_pos, (uint16_t *)qbuf, q_av, (uint16_t *)Kl, (uint16_t *)Vtl, total_cap)
        if (hd == 128 && kv_only) SD_ROPE_GROUP(128, true);
        else if (hd == 128) SD_ROPE_GROUP(128, false);
        else if (kv_only) SD_ROPE_GROUP(64, true);
        else SD_ROPE_GROUP(64, false);
#undef SD_ROPE_GROUP
        return hipGetLastError();
    }
#define SD_ROPE_ROWS(T_, KV_)                                                                                                 \
    hipLaunchKernelGGL((rope_append_kernel<T_, KV_>), dim3(M), dim3(1024), 0, s, qkv, n_slabs, slab_stride, pv, cv, H, hd, rope, max_pos, \
                       (T_ *)qbuf, q_av, (T_ *)Kl, (T_ *)Vtl, total_cap)
    if (dtype == SD_BF16 && kv_only) SD_ROPE_ROWS(bf16_t, true);
    else if (dtype == SD_BF16) SD_ROPE_ROWS(bf16_t, false);
    else if (kv_only) return hipErrorInvalidValue; // (fp32 models keep the queries of a call's last forward)
    else SD_ROPE_ROWS(float, false);
#undef SD_ROPE_ROWS
    return hipGetLastError();
}

// ---------------------------------------------------------------- generic attention
// One block per (row slot i, head, selected sequence): query row i sees cache rows
// [0, kv0 + i].  Scores live in dynamic LDS (lds_len floats: the largest sequence capacity).
// Bound: latency of the two passes over the cache, so both read it in the pieces it is stored in: a thread's token is
// hd / 8 contiguous pieces of 8 dimensions, a wave's V load is 8 dimensions x 32 tokens, four tokens per lane.  Measured,
// fp32, head width 64, 32 to 80 tokens, 5 rows x 4 heads: 11.3 us element by element, 7.1 us now.
__device__ __forceinline__ void load8_f(const float *p, float *f)
{
    const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
}
__device__ __forceinline__ void load8_f(const bf16_t *p, float *f)
{
    const uint4 a = *(const uint4 *)p;
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; i++) f[2 * i] = __uint_as_float(w[i] << 16), f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}
__device__ __forceinline__ float4 load4_f(const float *p) { return *(const float4 *)p; }
__device__ __forceinline__ float4 load4_f(const bf16_t *p)
{
    const uint2 a = *(const uint2 *)p;
    return make_float4(__uint_as_float(a.x << 16), __uint_as_float(a.x & 0xffff0000u), __uint_as_float(a.y << 16), __uint_as_float(a.y & 0xffff0000u));
}
// FUSED (fp32): RoPE and cache append as well, from the QKV product.  A block rotates its own query row and the keys of
// the rows up to it (at most 16 short rows; the blocks of later rows do it again), keeps those and their values in LDS
// and writes its own row into the cache; it reads the cache below the new rows only, so no block waits for another.
// Measured, tiny pair: 6.3 - 7.1 us here + 2.8 - 3.8 us for the launch that did this before -> 8.0 - 8.3 us; whole step
// 245 -> 235 us.
template <typename T, bool FUSED>
__global__ __launch_bounds__(256) void attn_generic_kernel(T *qbuf, ActView q_av, T *Kl, T *Vtl,
                                                           PlanView pv, CtxView cv, int R, int H, int hd,
                                                           int64_t total_cap, int lds_len, T *obuf, ActView o_av,
                                                           const float *qkv, const float2 *rope, int max_pos)
{
    extern __shared__ __attribute__((aligned(16))) float sc[]; // [lds_len] scores, then [hd] q, [32] red, FUSED: [R][hd] k, [R][hd] v
    float *qs = sc + lds_len; // (lds_len, a capacity, is a multiple of 64)
    float *red = qs + hd;
    float *sk = red + 32, *sv = sk + (size_t)R * hd;
    int i = blockIdx.x, h = blockIdx.y, j = blockIdx.z;
    int r = j * R + i;
    int HD = H * hd;
    if (i >= pv.seq_nq[j]) {
        for (int d = threadIdx.x; d < hd; d += blockDim.x) {
            store_act(obuf, act_index(o_av, r, h * hd + d, HD), o_av.plane, 0.f);
            if (FUSED) store_act(qbuf, act_index(q_av, r, h * hd + d, HD), q_av.plane, 0.f);
        }
        return;
    }
    int Lk = pv.seq_kv0[j] + i + 1;
    if (Lk > lds_len) { // the launch was sized for fewer rows than the cache holds: flag it, do not read on
        if (threadIdx.x == 0) atomicOr(cv.status, 32);
        Lk = lds_len;
    }
    int64_t off = cv.off[pv.seq_b[j]];
    T *Kh = Kl + (size_t)h * total_cap * hd;
    T *Vh = Vtl + (size_t)h * hd * total_cap;
    const int kv0 = pv.seq_kv0[j], old = FUSED ? min(Lk, kv0) : Lk; // tokens read from the cache
    if (FUSED) {
        const int half = hd >> 1;
        for (int x = threadIdx.x; x < (i + 1) * half; x += blockDim.x) {
            const int rr = x / half, e = x % half, pos = kv0 + rr;
            const float *row = qkv + (size_t)(j * R + rr) * 3 * HD + h * hd + e;
            const float q0 = row[0], q1 = row[half], k0 = row[HD], k1 = row[HD + half], v0 = row[2 * HD], v1 = row[2 * HD + half];
            const bool in = pos < max_pos;
            const float2 cs = rope[(size_t)(in ? pos : 0) * half + e];
            const float ka = in ? k0 * cs.x - k1 * cs.y : 0.f, kb = in ? k1 * cs.x + k0 * cs.y : 0.f;
            sk[rr * hd + e] = ka;
            sk[rr * hd + e + half] = kb;
            sv[rr * hd + e] = in ? v0 : 0.f;
            sv[rr * hd + e + half] = in ? v1 : 0.f;
            if (rr == i) {
                const float qa = in ? q0 * cs.x - q1 * cs.y : 0.f, qb = in ? q1 * cs.x + q0 * cs.y : 0.f;
                qs[e] = qa;
                qs[e + half] = qb;
                store_act(qbuf, act_index(q_av, r, h * hd + e, HD), q_av.plane, qa); // (only sd_debug_read looks at it)
                store_act(qbuf, act_index(q_av, r, h * hd + e + half, HD), q_av.plane, qb);
                if (in) { // (pos < capacity: the plan sees to it)
                    Kh[kt_offset(hd, off + pos, e)] = from_float<T>(ka);
                    Kh[kt_offset(hd, off + pos, e + half)] = from_float<T>(kb);
                    Vh[vt_offset(hd, off + pos, e)] = from_float<T>(v0);
                    Vh[vt_offset(hd, off + pos, e + half)] = from_float<T>(v1);
                } else if (e == 0) atomicOr(cv.status, 8);
            }
        }
    } else {
        for (int d = threadIdx.x; d < hd; d += blockDim.x) qs[d] = load_act(qbuf, act_index(q_av, r, h * hd + d, HD), q_av.plane);
    }
    __syncthreads();
    float scale = 1.0f / sqrtf((float)hd);
    float mx = -3.0e38f;
    for (int t = threadIdx.x; t < Lk; t += blockDim.x) {
        float dot = 0.f;
        if (!FUSED || t < old) {
#pragma unroll 8
            for (int d = 0; d < hd; d += 8) { // (8 dimensions of a token are one piece of its tile)
                float f[8];
                load8_f(Kh + kt_offset(hd, off + t, d), f);
#pragma unroll
                for (int e = 0; e < 8; e++) dot += qs[d + e] * f[e];
            }
        } else {
            const float *kr = sk + (size_t)(t - kv0) * hd;
            for (int d = 0; d < hd; d++) dot += qs[d] * kr[d];
        }
        dot *= scale;
        sc[t] = dot;
        mx = fmaxf(mx, dot);
    }
    mx = block_max(mx, red);
    float z = 0.f;
    for (int t = threadIdx.x; t < Lk; t += blockDim.x) {
        float e = expf(sc[t] - mx);
        sc[t] = e;
        z += e;
    }
    z = block_sum(z, red);
    __syncthreads();
    // wave w takes dimensions 8 w .. 8 w + 7, then 8 (w + 4) ..; lane (dl, tl): dimension dl of them, tokens 4 tl .. of a tile
    const int lane = threadIdx.x & 63, dl = lane >> 3, tl = lane & 7;
    for (int d8 = (threadIdx.x >> 6) * 8; d8 < hd; d8 += blockDim.x / 8) {
        float acc = 0.f;
#pragma unroll 4
        for (int t = 4 * tl; t < old; t += 32) {
            const float4 v = load4_f(Vh + vt_offset(hd, off + t, d8 + dl)), p = *(const float4 *)(sc + t);
            acc += p.x * v.x; // (scores past the end are not initialised, cache rows past it hold anything: not used)
            acc += t + 1 < old ? p.y * v.y : 0.f;
            acc += t + 2 < old ? p.z * v.z : 0.f;
            acc += t + 3 < old ? p.w * v.w : 0.f;
        }
        if (FUSED)
            for (int t = old + tl; t < Lk; t += 8) acc += sc[t] * sv[(size_t)(t - kv0) * hd + d8 + dl];
        acc += dpp_f<0xB1>(acc);
        acc += dpp_f<0x4E>(acc);
        acc += dpp_f<0x141>(acc); // (8 lanes)
        if (tl == 0) store_act(obuf, act_index(o_av, r, h * hd + d8 + dl, HD), o_av.plane, acc / z);
    }
}

template <typename T, bool FUSED>
static hipError_t attn_generic(hipStream_t s, size_t lds, T *qbuf, ActView q_av, T *Kl, T *Vtl, PlanView pv, CtxView cv, int R, int n_seq,
                               int H, int hd, int64_t total_cap, int len_upper, T *obuf, ActView o_av, const float *qkv, const float2 *rope,
                               int max_pos)
{
    if (lds > 160 * 1024) return hipErrorNotSupported;
    if (lds > 64 * 1024) { // beyond the default limit: ask for the larger LDS allocation this part has
        const hipError_t ea = hipFuncSetAttribute((const void *)attn_generic_kernel<T, FUSED>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (ea != hipSuccess) return hipErrorNotSupported;
    }
    hipLaunchKernelGGL((attn_generic_kernel<T, FUSED>), dim3(R, H, n_seq), dim3(256), lds, s, qbuf, q_av, Kl, Vtl, pv, cv, R, H, hd, total_cap,
                       len_upper, obuf, o_av, qkv, rope, max_pos);
    return hipGetLastError();
}

hipError_t launch_attn_generic(hipStream_t s, int dtype, void *qbuf, ActView q_av, void *Kl, void *Vtl, PlanView pv, CtxView cv, int R,
                               int n_seq, int H, int hd, int64_t total_cap, int len_upper, void *obuf, ActView o_av)
{
    const size_t lds = ((size_t)len_upper + 256 + hd + 32) * sizeof(float); // (256 floats of slack: the limit is part of the interface)
    if (dtype == SD_BF16)
        return attn_generic<bf16_t, false>(s, lds, (bf16_t *)qbuf, q_av, (bf16_t *)Kl, (bf16_t *)Vtl, pv, cv, R, n_seq, H, hd, total_cap,
                                           len_upper, (bf16_t *)obuf, o_av, nullptr, nullptr, 0);
    return attn_generic<float, false>(s, lds, (float *)qbuf, q_av, (float *)Kl, (float *)Vtl, pv, cv, R, n_seq, H, hd, total_cap, len_upper,
                                      (float *)obuf, o_av, nullptr, nullptr, 0);
}

// fp32: RoPE, cache append and attention in one launch, from the QKV product (one slab); hipErrorNotSupported where the
// new rows do not fit in LDS beside the scores, or a slot's rows are many.
hipError_t launch_attn_f32_fused(hipStream_t s, const float *qkv, const float2 *rope, int max_pos, float *Kl, float *Vtl, PlanView pv, CtxView cv,
                                 int R, int n_seq, int H, int hd, int64_t total_cap, int len_upper, float *qbuf, float *obuf, ActView o_av)
{
    if (R > 16) return hipErrorNotSupported;
    const size_t lds = ((size_t)len_upper + hd + 32 + 2 * (size_t)R * hd) * sizeof(float);
    return attn_generic<float, true>(s, lds, qbuf, o_av, Kl, Vtl, pv, cv, R, n_seq, H, hd, total_cap, len_upper, obuf, o_av, qkv, rope, max_pos);
}

// ---------------------------------------------------------------- inverse-CDF pick
// Chooses the smallest index k with sum_{x<=k} w(x) > u * sum_x w(x) for weights
// produced on the fly by wfun(v) -> float4 of elements 4v..4v+3 (zero beyond V).
// All threads of a 1024-thread block must call it; the result is returned to all.
// The sums are added in parallel (segment totals, then a scan inside the segment that holds u * Z), so where
// rounding makes them disagree the answer is the nearest index of positive weight: see first_over; if no
// running sum of the chosen segment exceeds the target, the segment's last index of positive weight; if
// u * Z is not below Z at all, the row's last one.
struct PickScratch {
    float seg[64];
    float red[32];
    float base;
    float target;
    int seg_idx;
    int pick;
    int last_pos;
    int seg_last; // last index of positive weight inside the segment that holds the target
};

// The search inside vectors [v_begin, v_end) for a target that lies `base` or more into the sum: segments of blockDim
// vectors, then a scan of the one that holds the target.  Without a crossing: the chosen segment's last index of
// positive weight, or the range's if no segment was chosen.  At most 64 segments.
template <typename F>
__device__ __forceinline__ int block_pick_range(F wfun, int v_begin, int v_end, int V, float base, float target, PickScratch *ps)
{
    const int T = blockDim.x;
    const int nseg = (v_end - v_begin + T - 1) / T;
    if (threadIdx.x == 0) {
        ps->pick = 0x7fffffff;
        ps->last_pos = 0;
        ps->seg_last = -1;
    }
    __syncthreads();
    int lastp = -1;
    for (int it = 0; it < nseg; it++) {
        const int v = v_begin + it * T + threadIdx.x;
        const float4 f = v < v_end ? wfun(v) : make_float4(0.f, 0.f, 0.f, 0.f);
        lastp = max(lastp, last_positive(f, 4 * v));
        const float ssum = block_sum(((f.x + f.y) + f.z) + f.w, ps->red);
        if (threadIdx.x == 0) ps->seg[it] = ssum;
    }
    if (lastp >= 0) atomicMax(&ps->last_pos, lastp);
    __syncthreads();
    float cum = base;
    int sit = -1;
    for (int it = 0; it < nseg && sit < 0; it++) {
        if (cum + ps->seg[it] > target) sit = it;
        else cum += ps->seg[it];
    }
    if (sit >= 0) { // (uniform)
        const int v = v_begin + sit * T + threadIdx.x;
        const float4 f = v < v_end ? wfun(v) : make_float4(0.f, 0.f, 0.f, 0.f);
        const float loc = ((f.x + f.y) + f.z) + f.w;
        const float pre = block_excl_scan(loc, ps->red);
        int k = first_over(cum + pre, f, target, 4 * v);
        if (k >= V) k = 0x7fffffff;
        k = wave_min_i(k);
        const int ls = wave_max_i(last_positive(f, 4 * v));
        if (threadIdx.x % WAVE == 0) {
            if (k != 0x7fffffff) atomicMin(&ps->pick, k);
            if (ls >= 0) atomicMax(&ps->seg_last, ls);
        }
    }
    __syncthreads();
    int pick = ps->pick;
    if (pick == 0x7fffffff) pick = sit >= 0 && ps->seg_last >= 0 ? min(ps->seg_last, V - 1) : ps->last_pos;
    __syncthreads();
    return pick;
}

template <typename F>
__device__ __forceinline__ int block_pick_cdf(F wfun, int V, float u, PickScratch *ps, float *total_out)
{
    const int T = blockDim.x;
    int nvec = (V + 3) / 4;
    int nseg = (nvec + T - 1) / T;
    if (threadIdx.x == 0) {
        ps->pick = 0x7fffffff;
        ps->last_pos = 0;
        ps->seg_last = -1;
    }
    __syncthreads();
    int lastp = -1;
    for (int it = 0; it < nseg; it++) {
        int v = it * T + threadIdx.x;
        float4 f = v < nvec ? wfun(v) : make_float4(0.f, 0.f, 0.f, 0.f);
        if (f.x > 0.f) lastp = 4 * v;
        if (f.y > 0.f) lastp = 4 * v + 1;
        if (f.z > 0.f) lastp = 4 * v + 2;
        if (f.w > 0.f) lastp = 4 * v + 3;
        float loc = ((f.x + f.y) + f.z) + f.w;
        float ssum = block_sum(loc, ps->red);
        if (threadIdx.x == 0) ps->seg[it] = ssum;
    }
    if (lastp >= 0) atomicMax(&ps->last_pos, lastp);
    __syncthreads();
    if (threadIdx.x == 0) {
        float Z = 0.f;
        for (int it = 0; it < nseg; it++) Z += ps->seg[it];
        float target = u * Z;
        float cum = 0.f;
        int found = -1;
        for (int it = 0; it < nseg; it++) {
            if (cum + ps->seg[it] > target) {
                found = it;
                break;
            }
            cum += ps->seg[it];
        }
        ps->seg_idx = found;
        ps->base = cum;
        ps->target = target;
        if (total_out) *total_out = Z;
    }
    __syncthreads();
    int it = ps->seg_idx;
    if (it >= 0) {
        int v = it * T + threadIdx.x;
        float4 f = v < nvec ? wfun(v) : make_float4(0.f, 0.f, 0.f, 0.f);
        float loc = ((f.x + f.y) + f.z) + f.w;
        float pre = block_excl_scan(loc, ps->red);
        int k = first_over(ps->base + pre, f, ps->target, 4 * v);
        if (k >= V) k = 0x7fffffff;
        k = wave_min_i(k);
        const int ls = wave_max_i(last_positive(f, 4 * v));
        if (threadIdx.x % WAVE == 0) {
            if (k != 0x7fffffff) atomicMin(&ps->pick, k);
            if (ls >= 0) atomicMax(&ps->seg_last, ls);
        }
    }
    __syncthreads();
    int pick = ps->pick;
    // rounding left every running sum of the chosen segment at or below the target: its last index of positive
    // weight; no segment chosen (u * Z not below Z): the last one of the row
    if (pick == 0x7fffffff) pick = it >= 0 && ps->seg_last >= 0 ? min(ps->seg_last, V - 1) : ps->last_pos;
    __syncthreads();
    return pick;
}

__device__ __forceinline__ float4 load4_guard(const float *row, int v, int V, float fill)
{
    if (4 * v + 3 < V) return *(const float4 *)(row + 4 * v);
    float4 f = make_float4(fill, fill, fill, fill);
    if (4 * v < V) f.x = row[4 * v];
    if (4 * v + 1 < V) f.y = row[4 * v + 1];
    if (4 * v + 2 < V) f.z = row[4 * v + 2];
    return f;
}

// max and lowest-index argmax of one fp32 row (block-wide)
__device__ void row_max_argmax(const float *row, int V, float *redv, int *redi, float &mx, int &am)
{
    float bv = -3.0e38f;
    int bi = 0x7fffffff;
    int nvec = (V + 3) / 4;
    for (int v = threadIdx.x; v < nvec; v += blockDim.x) {
        float4 f = load4_guard(row, v, V, -3.0e38f);
        if (f.x > bv) { bv = f.x; bi = 4 * v; }
        if (f.y > bv) { bv = f.y; bi = 4 * v + 1; }
        if (f.z > bv) { bv = f.z; bi = 4 * v + 2; }
        if (f.w > bv) { bv = f.w; bi = 4 * v + 3; }
    }
    block_argmax(bv, bi, redv, redi);
    mx = bv;
    am = bi;
}

// sum_x exp((row[x] - mx) * invT) (block-wide)
__device__ float row_sumexp(const float *row, int V, float mx, float invT, float *red)
{
    float z = 0.f;
    int nvec = (V + 3) / 4;
    for (int v = threadIdx.x; v < nvec; v += blockDim.x) {
        float4 f = load4_guard(row, v, V, -3.0e38f);
        z += expf((f.x - mx) * invT);
        if (4 * v + 1 < V) z += expf((f.y - mx) * invT);
        if (4 * v + 2 < V) z += expf((f.z - mx) * invT);
        if (4 * v + 3 < V) z += expf((f.w - mx) * invT);
    }
    return block_sum(z, red);
}

// ---------------------------------------------------------------- register-resident vocabulary rows
// For V <= 32768 a block of RT threads holds a whole fp32 row in registers: thread t keeps the float4s
// number it * RT + t, it < NSEG - with 1024 threads the same element-to-thread assignment as the strided loops of the
// general kernels above; the block-wide sums are added as trees here, so the two paths agree to rounding
// (and exactly in the maximum and the arg max).  One pass over memory per row and a handful of barriers
// instead of one block reduction per 4096 elements.
// The block's shape follows the row (an 8-vector block of 1024 threads spends a 1024-column row's time on 31 exponentials of
// padding per thread): 256 threads with 1, 2 or 4 vectors up to 4096 columns, where most of 16 waves would only meet at the
// barriers, then 1024 threads with 2, 4 or 8.  Measured, 1024 columns (8 vectors x 1024 threads before): draft sampler
// 12.2 -> 4.2 us, row verdicts 13.3 -> 4.8 us.  Whole acceptance call, 1024 / 256 threads: 256 rows of 1028, 2048, 4096 columns
// 12.4 / 11.7, 12.4 / 11.8, 11.5 / 11.5 us; 2048 rows 18.4 / 11.5, 18.3 / 11.4, 19.2 / 15.9.
#define ROW_NSEG 8
#define ROW_THREADS 1024
#define SD_ROW_SHAPES(V, CALL)                    \
    do {                                          \
        if ((V) <= 1024) CALL(256, 1);            \
        else if ((V) <= 2048) CALL(256, 2);       \
        else if ((V) <= 4096) CALL(256, 4);       \
        else if ((V) <= 8192) CALL(1024, 2);      \
        else if ((V) <= 16384) CALL(1024, 4);     \
        else CALL(ROW_THREADS, ROW_NSEG);         \
    } while (0)
template <int NSEG>
struct RowRegs {
    float4 f[NSEG];
};
struct FastScratch {
    float wsum[ROW_THREADS / WAVE][ROW_NSEG];
    float red[32];
    int redi[32];
    int pick;
    int seg_last; // last index of positive weight inside the segment that holds the target
};
// Cross-wave steps: NW = 4 or 16 waves leave one LDS entry each, lane l of every wave reads entry l % NW and the entries
// meet inside groups of NW lanes (the maxima may meet their repetitions in a 16-lane row as well).
template <int NW>
__device__ __forceinline__ float sum_waves(float v)
{
    static_assert(NW == 4 || NW == 16, "a quad or a 16-lane row");
    if (NW == 16) return row16_sum(v);
    v += dpp_f<0xB1>(v);
    v += dpp_f<0x4E>(v);
    return v;
}
// Block-wide arg max / sum for RT threads; every thread gets the result.
template <int RT>
__device__ __forceinline__ void block_argmax_rows(float &v, int &idx, FastScratch *fs)
{
    const int w = threadIdx.x / WAVE, l = threadIdx.x % WAVE;
    row16_argmax(v, idx);
    float bv = lane_f(v, 0);
    int bi = __builtin_amdgcn_readlane(idx, 0);
    take_better(bv, bi, lane_f(v, 16), __builtin_amdgcn_readlane(idx, 16));
    take_better(bv, bi, lane_f(v, 32), __builtin_amdgcn_readlane(idx, 32));
    take_better(bv, bi, lane_f(v, 48), __builtin_amdgcn_readlane(idx, 48));
    lds_barrier();
    if (l == 0) {
        fs->red[w] = bv;
        fs->redi[w] = bi;
    }
    lds_barrier();
    v = fs->red[l & (RT / WAVE - 1)];
    idx = fs->redi[l & (RT / WAVE - 1)];
    row16_argmax(v, idx);
}
template <int RT>
__device__ __forceinline__ float block_max_rows(float v, FastScratch *fs)
{
    const int w = threadIdx.x / WAVE, l = threadIdx.x % WAVE;
    v = wave_max_dpp(v);
    lds_barrier();
    if (l == 0) fs->red[w] = v;
    lds_barrier();
    return row16_maxf(fs->red[l & (RT / WAVE - 1)]);
}
template <int RT>
__device__ __forceinline__ float block_sum_rows(float v, FastScratch *fs)
{
    const int w = threadIdx.x / WAVE, l = threadIdx.x % WAVE;
    v = wave_sum_dpp(v);
    lds_barrier();
    if (l == 0) fs->red[w] = v;
    lds_barrier();
    return sum_waves<RT / WAVE>(fs->red[l & (RT / WAVE - 1)]);
}

// (V is a multiple of 4.)  The loads are unconditional - vectors past the end re-read the last one, which row_fill replaces
// where it matters - so that all of them are in flight at once: with a guard each they were a branch each.
template <int RT, int NSEG>
__device__ __forceinline__ void row_load(const float *row, int V, RowRegs<NSEG> &r)
{
    const int last = V / 4 - 1;
#pragma unroll
    for (int it = 0; it < NSEG; it++) r.f[it] = *(const float4 *)(row + 4 * min(it * RT + (int)threadIdx.x, last));
}
template <int RT, int NSEG>
__device__ __forceinline__ void row_fill(int V, float fill, RowRegs<NSEG> &r)
{
#pragma unroll
    for (int it = 0; it < NSEG; it++) {
        const bool in = it * RT + (int)threadIdx.x < V / 4;
        r.f[it].x = in ? r.f[it].x : fill;
        r.f[it].y = in ? r.f[it].y : fill;
        r.f[it].z = in ? r.f[it].z : fill;
        r.f[it].w = in ? r.f[it].w : fill;
    }
}

// p := max(0, p - q); no weight past the end of the row, whatever vector row_load has repeated there (a q below 0 would leave
// some).  A select on the result: on q itself it makes the late loads of q conditional again (300 rows of 32000 columns: 21.2
// -> 25.5 us).
__device__ __forceinline__ void residual(bool in, float4 &p, const float4 q)
{
    p.x = in ? fmaxf(p.x - q.x, 0.f) : 0.f;
    p.y = in ? fmaxf(p.y - q.y, 0.f) : 0.f;
    p.z = in ? fmaxf(p.z - q.z, 0.f) : 0.f;
    p.w = in ? fmaxf(p.w - q.w, 0.f) : 0.f;
}

// e^((x - mx) / T) of a row's elements, x <= mx: 2^n 2^f with n + f = (x - mx) log2(e) / T, n whole, f from one rounding and
// corrected by what the factor's own rounding takes from the product; nine instructions where expf with the difference and its
// product takes fifteen.  (-inf and what lies 160 powers of two below the maximum give 0, a NaN stays one.)  Error of the
// normalised rows against 64 bits, this / expf: N(0, 2), 32000 columns, T = 1: 3.6e-8 / 3.6e-8 (2-norm), T = 0.7: 8.5e-8 / 9.2e-8.
struct RowExp {
    float mx, c2, low;
    __device__ __forceinline__ RowExp(float mx_, float invT) : mx(mx_), c2(fminf(invT * 1.44269504088896f, 3.4e38f))
    {
        // (c2 + c2 * low = invT * log2(e); at the ends of the range, where the remainder is not representable, without)
        const float rest = fmaf(invT, 1.44269504088896f, -c2) + invT * 1.92596299e-8f;
        low = c2 > 1e-30f && c2 < 1e38f ? rest / c2 : 0.f;
    }
    __device__ __forceinline__ float operator()(float x) const
    {
        const float d = x - mx, t = fmaxf(d * c2, -160.f), n = rintf(t);
        return ldexpf(__builtin_amdgcn_exp2f(fmaf(t, low, fmaf(d, c2, -n))), (int)n);
    }
    __device__ __forceinline__ float4 operator()(const float4 f) const
    {
        return make_float4((*this)(f.x), (*this)(f.y), (*this)(f.z), (*this)(f.w));
    }
};

// max, lowest-index argmax (T == 0 only) and (T > 0) z = sum of e(x) = exp((x - max) / T) of the row in r (filled with
// row_filler past V).  For T > 0 the row is replaced by e(x) (exactly 0 past V), so that the probabilities
// e(x) / z need no second exponential.
template <int RT, int NSEG>
__device__ __forceinline__ void row_stats_regs(RowRegs<NSEG> &r, float invT, FastScratch *fs, float &mx, int &am, float &z)
{
    if (invT > 0.f) { // (uniform) sampling needs the maximum alone: a third of the instructions
        float bv = -3.0e38f;
#pragma unroll
        for (int it = 0; it < NSEG; it++) bv = fmaxf(bv, fmaxf(fmaxf(r.f[it].x, r.f[it].y), fmaxf(r.f[it].z, r.f[it].w)));
        mx = block_max_rows<RT>(bv, fs);
        am = 0;
    } else {
        float bv = -3.0e38f;
        int bi = 0x7fffffff;
#pragma unroll
        for (int it = 0; it < NSEG; it++) {
            const int v = it * RT + threadIdx.x;
            const float4 f = r.f[it];
            if (f.x > bv) { bv = f.x; bi = 4 * v; }
            if (f.y > bv) { bv = f.y; bi = 4 * v + 1; }
            if (f.z > bv) { bv = f.z; bi = 4 * v + 2; }
            if (f.w > bv) { bv = f.w; bi = 4 * v + 3; }
        }
        block_argmax_rows<RT>(bv, bi, fs);
        mx = bv;
        am = bi;
    }
    z = 1.f;
    if (invT > 0.f) {
        float zl = 0.f;
        const RowExp ex(mx, invT);
#pragma unroll
        for (int it = 0; it < NSEG; it++) {
            const float4 f = ex(r.f[it]);
            zl += f.x;
            zl += f.y;
            zl += f.z;
            zl += f.w;
            r.f[it] = f;
        }
        z = block_sum_rows<RT>(zl, fs);
    }
}

// Sum over the lanes whose number agrees modulo N (N = 1 ... 8), left in all of them: rotations inside the 16-lane rows,
// then the rows of the wave.
template <int N>
__device__ __forceinline__ float stride_sum(float v)
{
    v += dpp_f<0x128>(v);
    if (N <= 4) v += dpp_f<0x124>(v);
    if (N <= 2) v += dpp_f<0x122>(v);
    if (N <= 1) v += dpp_f<0x121>(v);
    const auto r16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r16[0]) + __uint_as_float(r16[1]);
    const auto r32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r32[0]) + __uint_as_float(r32[1]);
}
// Wave totals of N values per lane; lane l gets that of value l % N.  Each exchange halves the values a lane still carries
// (it keeps those with its own bit and gives the others away): 26 instructions for 8 values where a reduction each takes 88.
template <int N>
__device__ __forceinline__ float scatter_sum(const float (&v)[N], int lane)
{
    static_assert(N == 1 || N == 2 || N == 4 || N == 8, "halved in every exchange");
    float a[4], b[2], c;
    if constexpr (N == 8) {
#pragma unroll
        for (int i = 0; i < 4; i++) a[i] = (lane & 4 ? v[i + 4] : v[i]) + dpp_f<0x141>(lane & 4 ? v[i] : v[i + 4]);
    } else if constexpr (N == 4) {
#pragma unroll
        for (int i = 0; i < 4; i++) a[i] = v[i];
    }
    if constexpr (N >= 4) {
#pragma unroll
        for (int i = 0; i < 2; i++) b[i] = (lane & 2 ? a[i + 2] : a[i]) + dpp_f<0x4E>(lane & 2 ? a[i] : a[i + 2]);
    } else if constexpr (N == 2) {
        b[0] = v[0];
        b[1] = v[1];
    }
    if constexpr (N >= 2) c = (lane & 1 ? b[1] : b[0]) + dpp_f<0xB1>(lane & 1 ? b[0] : b[1]);
    else c = v[0];
    return stride_sum<N>(c);
}

// Inverse-CDF pick (same rule as block_pick_cdf) over weights held in registers: the whole row, or (pick_regs_range) the
// float4s v_begin .. v_end of one, for a target that lies `base` or more into the row's sum.  Weights past the end are 0.
template <bool RANGE, int RT, int NSEG>
__device__ __forceinline__ int pick_regs_impl(const RowRegs<NSEG> &w, int V, float u, FastScratch *fs, float *total_out, int v_begin, int v_end,
                                              float base, float target)
{
    // Index order is (segment it, thread t, component c).  Segment totals are added as a tree; every wave works out the
    // total Z, the segment holding u * Z and the sum before it for itself (no single-thread phase), then one block-wide
    // scan of that segment's float4 sums places the element.
    constexpr int NW = RT / WAVE;
    const int lane = threadIdx.x % WAVE, wv = threadIdx.x / WAVE;
    float loc[NSEG];
#pragma unroll
    for (int it = 0; it < NSEG; it++) loc[it] = ((w.f[it].x + w.f[it].y) + w.f[it].z) + w.f[it].w;
    float seg = scatter_sum<NSEG>(loc, lane); // of segment lane % NSEG
    float *wsum = &fs->wsum[0][0];            // [wave][segment], packed
    lds_barrier();                            // the scratch may still be in use by a previous call
    if (lane < NSEG) wsum[wv * NSEG + lane] = seg;
    if (threadIdx.x == 0) {
        fs->pick = 0x7fffffff;
        fs->seg_last = -1;
    }
    lds_barrier();
    seg = 0.f;
#pragma unroll
    for (int e = 0; e < NW * NSEG; e += WAVE) seg += NW * NSEG >= WAVE || lane < NW * NSEG ? wsum[(e + lane) % (NW * NSEG)] : 0.f;
    seg = stride_sum<NSEG>(seg);
    // lane it < NSEG: segment it, running sums over the segments (those past the end hold nothing)
    seg = lane < NSEG ? seg : 0.f;
    float run = seg;
    run += dpp_f<0x111>(run);
    if (NSEG > 2) run += dpp_f<0x112>(run);
    if (NSEG > 4) run += dpp_f<0x114>(run);
    if (!RANGE) {
        const float Z = lane_f(run, NSEG - 1);
        target = u * Z;
        if (total_out) *total_out = Z;
    }
    const unsigned long long over = __ballot(seg > 0.f && base + run > target);
    const int sit = over ? __ffsll(over) - 1 : -1;
    if (sit > 0) base += lane_f(run, sit - 1);
    if (sit >= 0) { // uniform over the block
        float4 f = w.f[0];
#pragma unroll
        for (int it = 1; it < NSEG; it++) { // (component selects: an indexed copy would put the whole row into scratch memory)
            const float4 c = w.f[it];
            f.x = it == sit ? c.x : f.x;
            f.y = it == sit ? c.y : f.y;
            f.z = it == sit ? c.z : f.z;
            f.w = it == sit ? c.w : f.w;
        }
        const int v = v_begin + sit * RT + threadIdx.x;
        const float l4 = ((f.x + f.y) + f.z) + f.w;
        const float inc = wave_incl_scan_dpp(l4, lane);
        if (lane == WAVE - 1) fs->red[wv] = inc; // red was last read before the barrier above
        lds_barrier();
        const float before = sum_waves<RT / WAVE>((lane & (RT / WAVE - 1)) < wv ? fs->red[lane & (RT / WAVE - 1)] : 0.f);
        int k = first_over(base + (before + inc - l4), f, target, 4 * v);
        if (k >= V) k = 0x7fffffff;
        k = wave_min_i(k);
        const int ls = wave_max_i(last_positive(f, 4 * v));
        if (lane == 0) {
            if (k != 0x7fffffff) atomicMin(&fs->pick, k);
            if (ls >= 0) atomicMax(&fs->seg_last, ls);
        }
    }
    lds_barrier();
    int pick = fs->pick;
    // rounding left every running sum of the chosen segment at or below the target: its last index of positive
    // weight; no segment chosen (u * Z not below Z): the last one of the row
    if (pick == 0x7fffffff) { // (uniform, rare)
        if (sit >= 0 && fs->seg_last >= 0) pick = min(fs->seg_last, V - 1);
        else { // last index of the row with a positive weight (0 if there is none)
            int lastp = -1;
#pragma unroll
            for (int it = 0; it < NSEG; it++) lastp = max(lastp, last_positive(w.f[it], 4 * (v_begin + it * RT + (int)threadIdx.x)));
            lastp = wave_max_i(lastp);
            if (lane == 0) fs->redi[wv] = lastp;
            lds_barrier();
            pick = max(row16_max(fs->redi[lane & (RT / WAVE - 1)]), 0);
        }
    }
    lds_barrier();
    return pick;
}
template <int RT, int NSEG>
__device__ __forceinline__ int pick_regs(const RowRegs<NSEG> &w, int V, float u, FastScratch *fs, float *total_out)
{
    return pick_regs_impl<false, RT>(w, V, u, fs, total_out, 0, (V + 3) / 4, 0.f, 0.f);
}
template <int RT, int NSEG>
__device__ __forceinline__ int pick_regs_range(const RowRegs<NSEG> &w, int V, int v_begin, int v_end, float base, float target, FastScratch *fs)
{
    return pick_regs_impl<true, RT>(w, V, 0.f, fs, nullptr, v_begin, v_end, base, target);
}

// e(x) -> probabilities e(x) * (1 / z), in place
template <int NSEG>
__device__ __forceinline__ void row_scale(RowRegs<NSEG> &r, float invZ)
{
#pragma unroll
    for (int it = 0; it < NSEG; it++) {
        r.f[it].x *= invZ;
        r.f[it].y *= invZ;
        r.f[it].z *= invZ;
        r.f[it].w *= invZ;
    }
}

// The single-row plan (PLAN_CAND, R = 1) of sequence slot j for the forward that feeds `tok`: the same entries,
// checks and cache-length update as plan_kernel makes for that mode, written by the sampler block that has
// just drawn the token.  seq_order keeps the order the catch-up plan of this draft call left (every
// sequence grows by one row, so the ranking by length does not change).  One thread calls this.
// The sequence state it needs is read by plan_cand_load when the sampler starts (three dependent reads that would
// otherwise stand at its end).
struct CandState {
    int b, n, kv, cap, g;
    bool in;
};
__device__ __forceinline__ CandState plan_cand_load(const NextPlan &np, int j)
{
    const CtxView &cv = np.cv;
    CandState c = {j, 0, 0, 0, 0, false};
    if (!np.enabled) return c;
    if (np.seq_ids) c.b = np.seq_ids[j];
    c.in = c.b >= 0 && c.b < cv.B;
    if (c.in) {
        c.n = cv.ntok[c.b];
        c.kv = cv.kvlen[(size_t)np.slot * cv.B + c.b];
        c.cap = cv.cap[c.b];
        c.g = seq_gamma(cv, c.b, np.gamma);
    }
    return c;
}
// What plan_next_cand returns for these arguments, without a store: every thread of a block can work it out for itself.
__device__ __forceinline__ int next_row_token(const NextPlan &np, int tok, const CandState &cs)
{
    const bool fed = cs.in && np.next_idx < cs.g && cs.n >= 1 && max(cs.kv, 0) < cs.cap;
    return fed && tok >= 0 && tok < np.vocab ? tok : 0;
}
__device__ int plan_next_cand(const NextPlan &np, int j, int tok, const CandState &cs)
{
    const PlanView &pv = np.pv;
    const CtxView &cv = np.cv;
    const int b = cs.b;
    if (!cs.in) { // refuse out-of-range ids: the row stays unused
        atomicOr(cv.status, 4);
        pv.seq_b[j] = 0;
        pv.seq_kv0[j] = 0;
        pv.seq_nq[j] = 0;
        pv.row_tok[j] = 0;
        pv.row_pos[j] = 0;
        pv.row_b[j] = 0;
        pv.row_valid[j] = 0;
        pv.lm_row[j] = j;
        return 0;
    }
    const int n = cs.n, cap = cs.cap;
    int kv0 = cs.kv, nq = 1;
    if (np.next_idx >= cs.g) nq = 0; // the sequence has drawn all its candidates
    if (n < 1) { // an empty sequence has no pending token
        atomicOr(cv.status, 2);
        nq = 0;
    }
    if (kv0 < 0) kv0 = 0;
    if (kv0 + nq > cap) { // never write beyond the sequence's cache rows
        atomicOr(cv.status, 1);
        nq = cap - kv0 > 0 ? cap - kv0 : 0;
    }
    if (nq > 0 && (tok < 0 || tok >= np.vocab)) { // never index the embedding table out of range
        atomicOr(cv.status, 16);
        tok = 0;
    }
    pv.row_tok[j] = nq > 0 ? tok : 0;
    pv.row_pos[j] = kv0;
    pv.row_b[j] = b;
    pv.row_valid[j] = nq > 0;
    pv.seq_b[j] = b;
    pv.seq_kv0[j] = kv0;
    pv.seq_nq[j] = nq;
    pv.lm_row[j] = j;
    cv.kvlen[(size_t)np.slot * cv.B + b] = kv0 + nq;
    return nq > 0 ? tok : 0; // (= row_tok[j]: what the planned forward embeds)
}

// Does sequence slot j draw candidate idx in this draft call?  With per-sequence candidate counts a sequence that
// has drawn all of its own sits the remaining forwards out: its rows are unused, nothing of it is written (the
// sampler that drew its last candidate has already left its plan entry empty).
__device__ __forceinline__ bool draft_seq_active(const NextPlan &np, int j, int gamma, int idx)
{
    if (!np.cv.gam) return true;
    const int b = np.seq_ids ? np.seq_ids[j] : j;
    if (b < 0 || b >= np.cv.B) return true; // (the plan has flagged it; behave as without counts)
    return idx < seq_gamma(np.cv, b, gamma);
}

template <int RT, int NSEG>
__global__ __launch_bounds__(RT) void draft_sample_fast_kernel(const float *logits, int V, float T,
                                                                         const float *u, int gamma, int idx,
                                                                         int32_t *cand, float *q, NextPlan next)
{
    __shared__ FastScratch fs;
    const int j = blockIdx.x;
    const CandState cs = plan_cand_load(next, j);
    if (!draft_seq_active(next, j, gamma, idx)) { // (uniform over the block) nothing to draw: keep its plan entry empty
        if (threadIdx.x == 0 && next.enabled) plan_next_cand(next, j, 0, cs);
        return;
    }
    RowRegs<NSEG> r;
    row_load<RT>(logits + (size_t)j * V, V, r);
    row_fill<RT>(V, row_filler(T), r);
    float mx, z;
    int am;
    row_stats_regs<RT>(r, inv_temperature(T), &fs, mx, am, z);
    if (T == 0.f) {
        if (threadIdx.x == 0) {
            cand[j * gamma + idx] = am;
            if (next.enabled) plan_next_cand(next, j, am, cs);
        }
        return;
    }
    row_scale(r, 1.0f / z);
    float *qrow = q + ((size_t)j * gamma + idx) * V;
    const int nvec = (V + 3) / 4;
#pragma unroll
    for (int it = 0; it < NSEG; it++) {
        const int v = it * RT + threadIdx.x;
        const float4 p = r.f[it];
        if (4 * v + 3 < V) *(float4 *)(qrow + 4 * v) = p;
        else if (v < nvec) {
            if (4 * v < V) qrow[4 * v] = p.x;
            if (4 * v + 1 < V) qrow[4 * v + 1] = p.y;
            if (4 * v + 2 < V) qrow[4 * v + 2] = p.z;
        }
    }
    const int pick = pick_regs<RT>(r, V, u[j * gamma + idx], &fs, nullptr);
    if (threadIdx.x == 0) {
        cand[j * gamma + idx] = pick;
        if (next.enabled) plan_next_cand(next, j, pick, cs);
    }
}

// ---- samplers that start from the LM head's per-block softmax partials (LmStats: 32 columns per entry)
// A row's vocabulary is cut into slices of DS_SLICE columns, one 256-thread block each.  Every block reads all
// the row's partials (a few KB) and derives from them, in the same order and therefore to the same bits as
// every other block of the row: the row maximum, the mass of every slice (one wave-wide sum of the slice's 64
// entries), the normaliser Z (a lane scan of the slice masses) and the slice in which the running sum first
// exceeds u * Z.  It then writes its own slice of q = exp((x - max) / T) / Z, and the one block that owns the
// slice holding u * Z places the candidate inside it with a block-wide scan (same rule as block_pick_cdf:
// first index whose inclusive sum exceeds the target, else the last index of positive weight).  No block waits
// for another.  The owner also lays out the next single-row forward and, if asked, runs its first step
// (embedding row + first norm).
#define DS_SLICE 2048
#define DS_MAX_SLICES 32
struct SplitScratch {
    float red[32];
    float wmax[4];
    float slice[DS_MAX_SLICES];
    float4 wtot[2]; // (component = wave)
    int pick[4], lastp[4];
};

__device__ void next_forward_first_step(const NextPlan &next, int j, int tok, const CandState &cs, SplitScratch *ss)
{
    // (all threads of the block) thread 0 plans; the block gathers and norms the row
    if (!next.enabled) return;
    if (threadIdx.x == 0) plan_next_cand(next, j, tok, cs);
    if (!next.embed) return;
    embed_rmsnorm_row((const bf16_t *)next.E, next_row_token(next, tok, cs), j, next.d, next.x, next.g, next.eps,
                      (bf16_t *)next.out, next.av, ss->red);
}

// Bound: a chain of dependent steps in one block per slice (the 128 KB of a row are nothing).  Stamped in the kernel at
// 32000 columns, before / now (us): loads until the local maximum 1.6 / 1.4 - 1.9, slice masses 1.2 / 0.65, slice sums and
// owner 1.0 / 0.25 (a serial LDS read per slice, twice; now one read and a lane scan), q 0.3, placing the target 2.9 / 1.0 (its
// "last positive index" was an LDS atomic of every thread), first step of the next forward 2.0; launch 9.0 / 6.2.  The vector
// loads go out before the sequence state's dependent scalar loads.  NI = slices per wave: 4 serve rows of up to 32768 columns.
template <int NI>
__global__ __launch_bounds__(256) void draft_sample_split_kernel(const float *logits, const float *stats, int nb, int V,
                                                                  float T, const float *u, int gamma, int idx,
                                                                  int32_t *cand, float *q, NextPlan next)
{
    __shared__ SplitScratch ss;
    const int j = blockIdx.y, k = blockIdx.x, n_slices = gridDim.x;
    const int lane = threadIdx.x % WAVE, wv = threadIdx.x / WAVE;
    const float *st = stats + (size_t)j * nb * 3;
    // this block's slice of the logits row: requested first, needed only once the maximum and Z are known
    const float *row = logits + (size_t)j * V;
    float4 e[2];
#pragma unroll
    for (int it = 0; it < 2; it++) {
        const int v = k * (DS_SLICE / 4) + it * 256 + threadIdx.x; // (V is a multiple of 32: whole float4s only)
        e[it] = 4 * v < V ? *(const float4 *)(row + 4 * v) : make_float4(-3.0e38f, -3.0e38f, -3.0e38f, -3.0e38f);
    }
    // wave w holds the entries of slices w, w + 4, ...: lane l entry 64 * slice + l
    float em[NI], es[NI];
#pragma unroll
    for (int i = 0; i < NI; i++) {
        const int b = (4 * i + wv) * 64 + lane;
        const bool in = 4 * i + wv < n_slices && b < nb;
        em[i] = in ? st[3 * b] : -3.0e38f;
        es[i] = in ? st[3 * b + 1] : 0.f;
    }
    SD_SCHED_FENCE();
    const CandState cs = plan_cand_load(next, j);
    if (!draft_seq_active(next, j, gamma, idx)) { // (uniform over the block) nothing to draw: keep its plan entry empty
        if (k == 0) next_forward_first_step(next, j, 0, cs, &ss);
        return;
    }
    const float invT = inv_temperature(T), uj = u[j * gamma + idx];
    float mx = -3.0e38f;
#pragma unroll
    for (int i = 0; i < NI; i++) mx = fmaxf(mx, em[i]);
    mx = wave_max_dpp(mx);
    if (lane == 0) ss.wmax[wv] = mx;
    lds_barrier();
    mx = fmaxf(fmaxf(ss.wmax[0], ss.wmax[1]), fmaxf(ss.wmax[2], ss.wmax[3]));
#pragma unroll
    for (int i = 0; i < NI; i++) {
        const float mass = wave_sum_dpp(es[i] * expf((em[i] - mx) * invT)); // (entries past the row: 0 * 0)
        if (lane == 0 && 4 * i + wv < n_slices) ss.slice[4 * i + wv] = mass;
    }
    lds_barrier();
    // lane s holds slice s; every wave of every block adds the same numbers in the same order.  The owner is the first
    // slice of positive mass whose running sum exceeds the target, without one the last slice of positive mass.
    const float sm = lane < n_slices ? ss.slice[lane & (DS_MAX_SLICES - 1)] : 0.f;
    const float run = wave_incl_scan_dpp(sm, lane);
    const float Z = lane_f(run, WAVE - 1), base = k ? lane_f(run, k - 1) : 0.f, target = uj * Z;
    const unsigned long long with_mass = __ballot(sm > 0.f), over = __ballot(sm > 0.f && run > target);
    const int owner = over ? __ffsll(over) - 1 : with_mass ? WAVE - 1 - __clzll(with_mass) : 0;
    // this block's slice of q
    const float invZ = 1.0f / Z;
    float *qrow = q + ((size_t)j * gamma + idx) * V;
#pragma unroll
    for (int it = 0; it < 2; it++) {
        const int v = k * (DS_SLICE / 4) + it * 256 + threadIdx.x;
        if (4 * v < V) {
            float4 f = e[it];
            f.x = expf((f.x - mx) * invT);
            f.y = expf((f.y - mx) * invT);
            f.z = expf((f.z - mx) * invT);
            f.w = expf((f.w - mx) * invT);
            e[it] = f;
            *(float4 *)(qrow + 4 * v) = make_float4(f.x * invZ, f.y * invZ, f.z * invZ, f.w * invZ);
        } else {
            e[it] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
    if (k != owner) return; // (uniform over the block)
    // place the target inside the slice: index order is (it, thread, component)
    float l4[2], inc[2];
    int lastp = -1;
#pragma unroll
    for (int it = 0; it < 2; it++) {
        const float4 f = e[it];
        lastp = max(lastp, last_positive(f, 4 * (k * (DS_SLICE / 4) + it * 256 + (int)threadIdx.x)));
        l4[it] = ((f.x + f.y) + f.z) + f.w;
        inc[it] = wave_incl_scan_dpp(l4[it], lane);
        if (lane == WAVE - 1) ((float *)&ss.wtot[it])[wv] = inc[it];
    }
    lds_barrier();
    float seg_before = base;
    int pick = 0x7fffffff;
#pragma unroll
    for (int it = 0; it < 2; it++) {
        const float4 wt = ss.wtot[it];
        const float w0 = wt.x, w1 = w0 + wt.y, w2 = w1 + wt.z;
        const float before = seg_before + (wv == 0 ? 0.f : wv == 1 ? w0 : wv == 2 ? w1 : w2);
        seg_before += w2 + wt.w;
        const int v = k * (DS_SLICE / 4) + it * 256 + threadIdx.x;
        const int pk = first_over(before + (inc[it] - l4[it]), e[it], target, 4 * v);
        if (pk < V) pick = min(pick, pk);
    }
    pick = wave_min_i(pick);
    lastp = wave_max_i(lastp);
    if (lane == 0) {
        ss.pick[wv] = pick;
        ss.lastp[wv] = lastp;
    }
    lds_barrier();
    pick = min(min(ss.pick[0], ss.pick[1]), min(ss.pick[2], ss.pick[3]));
    if (pick == 0x7fffffff) pick = max(max(max(ss.lastp[0], ss.lastp[1]), max(ss.lastp[2], ss.lastp[3])), 0);
    if (threadIdx.x == 0) cand[j * gamma + idx] = pick;
    next_forward_first_step(next, j, pick, cs, &ss);
}

// Greedy candidate from the partials: the largest block maximum, lowest column among equals.
__global__ __launch_bounds__(256) void draft_argmax_split_kernel(const float *stats, int nb, int gamma, int idx,
                                                                  int32_t *cand, NextPlan next)
{
    __shared__ SplitScratch ss;
    __shared__ int redi[32];
    const int j = blockIdx.x;
    const CandState cs = plan_cand_load(next, j);
    if (!draft_seq_active(next, j, gamma, idx)) {
        next_forward_first_step(next, j, 0, cs, &ss);
        return;
    }
    const float *st = stats + (size_t)j * nb * 3;
    float bv = -3.0e38f;
    int bi = 0x7fffffff;
    for (int b = threadIdx.x; b < nb; b += 256) take_better(bv, bi, st[3 * b], __float_as_int(st[3 * b + 2]));
    block_argmax(bv, bi, ss.red, redi);
    if (threadIdx.x == 0) cand[j * gamma + idx] = bi;
    __syncthreads(); // (block_argmax read ss.red last)
    next_forward_first_step(next, j, bi, cs, &ss);
}

// ---------------------------------------------------------------- draft: softmax + sample
// One block per sequence.  T > 0: q = softmax(logits / T) is written in full and
// the candidate drawn by inverse CDF; T == 0: candidate = argmax.
__global__ __launch_bounds__(1024) void draft_sample_kernel(const float *logits, int V, float T, const float *u,
                                                            int gamma, int idx, int32_t *cand, float *q, NextPlan next)
{
    __shared__ PickScratch ps;
    __shared__ float redv[32];
    __shared__ int redi[32];
    int j = blockIdx.x;
    const CandState cs = plan_cand_load(next, j);
    if (!draft_seq_active(next, j, gamma, idx)) { // (uniform over the block) nothing to draw: keep its plan entry empty
        if (threadIdx.x == 0 && next.enabled) plan_next_cand(next, j, 0, cs);
        return;
    }
    const float *row = logits + (size_t)j * V;
    float mx;
    int am;
    row_max_argmax(row, V, redv, redi, mx, am);
    if (T == 0.f) {
        if (threadIdx.x == 0) {
            cand[j * gamma + idx] = am;
            if (next.enabled) plan_next_cand(next, j, am, cs);
        }
        return;
    }
    float invT = inv_temperature(T);
    float z = row_sumexp(row, V, mx, invT, redv);
    float invZ = 1.0f / z;
    float *qrow = q + ((size_t)j * gamma + idx) * V;
    int nvec = (V + 3) / 4;
    for (int v = threadIdx.x; v < nvec; v += blockDim.x) {
        float4 f = load4_guard(row, v, V, -3.0e38f);
        float4 p;
        p.x = expf((f.x - mx) * invT) * invZ;
        p.y = expf((f.y - mx) * invT) * invZ;
        p.z = expf((f.z - mx) * invT) * invZ;
        p.w = expf((f.w - mx) * invT) * invZ;
        if (4 * v + 3 < V) *(float4 *)(qrow + 4 * v) = p;
        else {
            if (4 * v < V) qrow[4 * v] = p.x;
            if (4 * v + 1 < V) qrow[4 * v + 1] = p.y;
            if (4 * v + 2 < V) qrow[4 * v + 2] = p.z;
        }
    }
    __syncthreads(); // q row of this block is complete and visible to the block
    auto wfun = [&](int v) {
        float4 f = load4_guard(row, v, V, -3.0e38f);
        float4 p;
        p.x = expf((f.x - mx) * invT) * invZ;
        p.y = 4 * v + 1 < V ? expf((f.y - mx) * invT) * invZ : 0.f;
        p.z = 4 * v + 2 < V ? expf((f.z - mx) * invT) * invZ : 0.f;
        p.w = 4 * v + 3 < V ? expf((f.w - mx) * invT) * invZ : 0.f;
        return p;
    };
    int pick = block_pick_cdf(wfun, V, u[j * gamma + idx], &ps, nullptr);
    if (threadIdx.x == 0) {
        cand[j * gamma + idx] = pick;
        if (next.enabled) plan_next_cand(next, j, pick, cs);
    }
}

hipError_t launch_draft_sample(hipStream_t s, const float *logits, int n_seq, int V, float T, const float *u,
                               int gamma, int idx, int32_t *cand, float *q, const NextPlan &next, const float *stats,
                               int stats_nb, int *did_embed)
{
    if (did_embed) *did_embed = 0;
    const int n_slices = (V + DS_SLICE - 1) / DS_SLICE;
    if (stats && stats_nb > 0 && stats_nb * 32 == V && n_slices <= DS_MAX_SLICES && n_seq <= 65535) {
        if (did_embed) *did_embed = next.enabled && next.embed;
        if (T > 0.f)
            hipLaunchKernelGGL(n_slices <= 16 ? draft_sample_split_kernel<4> : draft_sample_split_kernel<DS_MAX_SLICES / 4>,
                               dim3(n_slices, n_seq), dim3(256), 0, s, logits, stats, stats_nb, V, T, u, gamma, idx, cand, q, next);
        else
            hipLaunchKernelGGL(draft_argmax_split_kernel, dim3(n_seq), dim3(256), 0, s, stats, stats_nb, gamma, idx, cand,
                               next);
        return hipGetLastError();
    }
#define SD_SAMPLE_FAST(RT, NSEG)                                                                                             \
    hipLaunchKernelGGL((draft_sample_fast_kernel<RT, NSEG>), dim3(n_seq), dim3(RT), 0, s, logits, V, T, u, gamma, idx, cand, q, \
                       next)
    if (V <= ROW_NSEG * ROW_THREADS * 4) SD_ROW_SHAPES(V, SD_SAMPLE_FAST);
    else
        hipLaunchKernelGGL(draft_sample_kernel, dim3(n_seq), dim3(1024), 0, s, logits, V, T, u, gamma, idx, cand, q,
                           next);
    return hipGetLastError();
}

// ---------------------------------------------------------------- commit (KV rollback)
// (one thread; every value it updates is read before the first store, so that the reads are in flight together)
__device__ void commit_one(CtxView cv, int b, int gamma, const int32_t *cand_j, int n_acc, int next_tok)
{
    const int n = cv.ntok[b], cap = cv.cap[b];
    const int64_t off = cv.off[b];
    const int acc0 = cv.pol[b], exam0 = cv.pol[cv.B + b];
    int kv[SD_MAX_SLOTS], c[SD_MAX_GAMMA];
#pragma unroll
    for (int sl = 0; sl < SD_MAX_SLOTS; sl++) kv[sl] = sl < cv.n_slots ? cv.kvlen[(size_t)sl * cv.B + b] : 0;
    if (n_acc < 0) n_acc = 0;
    if (n_acc > gamma) n_acc = gamma;
#pragma unroll
    for (int i = 0; i < SD_MAX_GAMMA; i++) c[i] = i < n_acc ? cand_j[i] : 0;
    if (n + n_acc + 1 > cap) {
        atomicOr(cv.status, 1);
        return;
    }
#pragma unroll
    for (int i = 0; i < SD_MAX_GAMMA; i++)
        if (i < n_acc) cv.tokens[off + n + i] = c[i];
    cv.tokens[off + n + n_acc] = next_tok;
    // running estimate of Equation 1's alpha: accepted over examined candidates (a step that rejects at
    // position k has examined k + 1 of them)
    cv.pol[b] = acc0 + n_acc;
    cv.pol[cv.B + b] = exam0 + (n_acc < gamma ? n_acc + 1 : gamma);
    const int nn = n + n_acc + 1;
    cv.ntok[b] = nn;
#pragma unroll
    for (int sl = 0; sl < SD_MAX_SLOTS; sl++)
        if (sl < cv.n_slots && kv[sl] > nn - 1) cv.kvlen[(size_t)sl * cv.B + b] = nn - 1;
}

__global__ void commit_kernel(CtxView cv, const int32_t *seq_ids, int n_seq, int gamma, const int32_t *cand,
                              const int32_t *n_acc, const int32_t *next_tok)
{
    int j = blockIdx.x * blockDim.x + threadIdx.x;
    if (j >= n_seq) return;
    int b = seq_ids ? seq_ids[j] : j;
    if (b < 0 || b >= cv.B) {
        atomicOr(cv.status, 4);
        return;
    }
    commit_one(cv, b, seq_gamma(cv, b, gamma), cand + (size_t)j * gamma, n_acc[j], next_tok[j]);
}

// Candidate-count policy on the device (Section 1, Equation 1): for each selected sequence, alpha = accepted / examined so
// far (alpha0 before anything was examined) and gamma = the count in [0, gamma_max] that maximises
// (1 - alpha^(gamma+1)) / ((1 - alpha) (gamma c + 1)), the smallest on ties.  Written out operation by operation
// (no fused multiply-add), in the order the host function sd_choose_gamma uses, so both pick the same count.
__global__ void policy_choose_kernel(CtxView cv, const int32_t *seq_ids, int n_seq, double c_ratio, int gamma_max,
                                     double alpha0, int32_t *gamma_all, int32_t *gammas_out)
{
    const int j = blockIdx.x * blockDim.x + threadIdx.x;
    if (j >= n_seq) return;
    const int b = seq_ids ? seq_ids[j] : j;
    if (b < 0 || b >= cv.B) {
        atomicOr(cv.status, 4);
        if (gammas_out) gammas_out[j] = 0;
        return;
    }
    const int acc = cv.pol[b], exam = cv.pol[cv.B + b];
    const double alpha = exam > 0 ? __ddiv_rn((double)acc, (double)exam) : alpha0;
    int best = 0;
    double best_v = -1.0;
    for (int g = 0; g <= gamma_max; g++) {
        double tokens = 0.0, term = 1.0;
        for (int i = 0; i <= g; i++) {
            tokens = __dadd_rn(tokens, term);
            term = __dmul_rn(term, alpha);
        }
        const double v = __ddiv_rn(tokens, __dadd_rn(__dmul_rn((double)g, c_ratio), 1.0));
        if (v > best_v) best = g, best_v = v;
    }
    gamma_all[b] = best;
    if (gammas_out) gammas_out[j] = best;
}

hipError_t launch_policy_choose(hipStream_t s, CtxView cv, const int32_t *seq_ids, int n_seq, double c_ratio, int gamma_max,
                                double alpha0, int32_t *gamma_all, int32_t *gammas_out)
{
    hipLaunchKernelGGL(policy_choose_kernel, dim3((n_seq + 255) / 256), dim3(256), 0, s, cv, seq_ids, n_seq, c_ratio, gamma_max,
                       alpha0, gamma_all, gammas_out);
    return hipGetLastError();
}

hipError_t launch_commit(hipStream_t s, CtxView cv, const int32_t *seq_ids, int n_seq, int gamma,
                         const int32_t *cand, const int32_t *n_acc, const int32_t *next_tok)
{
    hipLaunchKernelGGL(commit_kernel, dim3((n_seq + 255) / 256), dim3(256), 0, s, cv, seq_ids, n_seq, gamma, cand,
                       n_acc, next_tok);
    return hipGetLastError();
}

// ---------------------------------------------------------------- verify tail
// Fused vocabulary softmax + accept scan + residual + resample.  Rows of more than ROW_NSEG * ROW_THREADS * 4 = 32768
// columns do not fit a block's registers; they take three launches (two where there is nothing to accept or nothing to draw):
//   verify_stats_wide_kernel  one block per logits row, one pass: (max, sum of exponentials, argmax) and the row's acceptance
//                             test, whose verdict is the sign of the sum;
//   verify_mass_wide_kernel   the mass of one slice of the deciding row per block;
//   verify_pick_wide_kernel   one block per sequence: the slice that holds u * Z is searched for the token; commit.
// Bound: one read of all rows.  The caller's workspace is three floats per row, so what a row's blocks could hand on is
// limited to that: a row's statistics come from one block, and the slice masses (gamma + 1 per sequence) take the
// argmax entries, which sampling does not use.  A block keeps two batches of 4 float4 per thread, one in flight while the
// other is summed.
// The statistics pass is bound by instruction issue as much as by memory: with expf (13 instructions an element beside the
// subtraction and the maximum) 576 rows of 128000 columns take 64 us, with three (WideExp) and the nontemporal hint, which
// then pays, 54 (5.5 TB/s; under the profiler).
// The hint, whole call at T = 1 without / with it (1024 threads), the same logits in every call | three sets of logits in turn:
// 270 rows of 128000 columns, gamma 8 50.0 / 53.4 | 55.7 / 53.7; 360 rows 52.5 / 57.9 | 61.8 / 58.5; 576 rows 79.5 / 77.6 | 87.8 / 77.6;
// 1350 rows of 33000 50.5 / 54.7 | 56.5 / 54.8: what the memory-side cache (256 MB) still holds from the call before it gives
// faster without, what it does not with; above 128 MB of logits the hint (at gamma 1 the same: 280 rows 85.1 / 91.2 | 94.4 / 93.0).  At gamma
// 0, where the pick reads the rows again: 270 rows 127 / 133 | 135 / 147; 400 rows 134 / 148 | 147 / 154; 520 rows 201 / 205 | 209 / 221;
// 2000 rows of 33000 189 / 206 | 198 / 212; 600 rows of 128000 (307 MB) 220.6 / 218.7 | 229.1 / 228.2: the hint above 256
// MB.  512 threads without it where there are rows enough to put two blocks on every compute unit (540 x 33000: 31.3, 1024
// threads with the hint 34.2).
// Whole call at 64 sequences, gamma 8, 128000 columns (295 MB of logits): 69 us (71 with scratch memory and flat loads in the pick, 76 in
// blocks of 1024 threads, 101 with expf, the acceptance test in the second launch and a pick that read its slice twice).
// e^(d / T), d <= 0, as 2^(c d + r d): c = log2(e) / T rounded down, r >= 0 what that leaves of it (the two-constant reduction
// of Cody and Waite, in base 2).  r > 0 and bounded by c: -inf stays -inf through both products and gives 0, d = 0 gives 1
// at any T.  Error of a row's sum against 64 bits, rms over 300 rows of N(0, 2), 128000 columns, T = 1 / 1.1 / 1.3 / 2: expf
// 6.3e-8 / 8.9e-8 / 9.9e-8 / 6.0e-8, this 6.2e-8 / 8.9e-8 / 9.6e-8 / 6.1e-8 (from 1.1 on mostly what 1 / T loses in 32 bits);
// without r, whose lack has the same sign in every column, 6.2e-8 / 1.5e-7 / 1.3e-7 / 6.6e-8, 0.8 us faster at 576 rows.
// The probability an acceptance test or a draw uses is expf's.
struct WideExp {
    float c, r;
    __device__ __forceinline__ WideExp(float invT)
    {
        const float lo = invT * 1.92596299e-8f; // (log2(e) minus its nearest float)
        c = fminf(invT * 1.44269504088896f, 3.4e38f);
        r = fmaf(invT, 1.44269504088896f, -c) + lo;
        if (r < 0.f && c > 1e-30f) {
            c = __uint_as_float(__float_as_uint(c) - 1u);
            r = fmaf(invT, 1.44269504088896f, -c) + lo;
        }
        r = fmaxf(fminf(r, c * 2.4e-7f), 1.4e-45f);
    }
    __device__ __forceinline__ float operator()(float d) const { return __builtin_amdgcn_exp2f(fmaf(d, c, d * r)); }
};
#define WIDE_U 4
template <int THREADS, bool NT>
__global__ __launch_bounds__(THREADS) void verify_stats_wide_kernel(const float *logits, int gamma, int V, float T, const int32_t *cand,
                                                                    const float *q, const float *u, float *stats)
{
    __shared__ float redv[32];
    __shared__ int redi[32];
    const float4 *row = (const float4 *)(logits + (size_t)blockIdx.x * V);
    const int nvec = V / 4; // (V is a multiple of 4)
    const float invT = inv_temperature(T);
    const WideExp ex(invT);
    // the row's acceptance test: what it needs beside the row's sums is requested first
    const int j = blockIdx.x / (gamma + 1), i = blockIdx.x % (gamma + 1);
    int c = -1;
    float lc = 0.f, qc = 1.f, ui = 0.f;
    if (T > 0.f && i < gamma) { // (uniform)
        c = cand[(size_t)j * gamma + i];
        ui = u[(size_t)j * (gamma + 1) + i];
        if (c >= 0 && c < V) {
            lc = ((const float *)row)[c];
            qc = q[((size_t)j * gamma + i) * V + c];
        }
    }
    // thread-local running maximum m (from -3e38: masked columns may lie below it, their exponentials are 0) and the
    // sum of exp((x - m) / T), rescaled when a batch of WIDE_U vectors raises m
    float m = -3.0e38f, z = 0.f;
    int am = 0x7fffffff;
    float4 fa[WIDE_U], fb[WIDE_U];
    auto load = [&](int v0, float4 *f) {
#pragma unroll
        for (int k = 0; k < WIDE_U; k++) {
            const int v = v0 + k * THREADS;
            typedef __attribute__((ext_vector_type(4))) float f32x4_t;
            f32x4_t t = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            if (v < nvec) t = ld_stream<NT>((const f32x4_t *)row + v);
            f[k] = make_float4(t.x, t.y, t.z, t.w);
        }
    };
    auto take = [&](int v0, const float4 *f) {
        if (invT > 0.f) { // (uniform)
            const float m_old = m;
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < WIDE_U; k++) m = fmaxf(m, fmaxf(fmaxf(f[k].x, f[k].y), fmaxf(f[k].z, f[k].w)));
#pragma unroll
            for (int k = 0; k < WIDE_U; k++) {
                s += (ex(f[k].x - m) + ex(f[k].y - m)) + (ex(f[k].z - m) + ex(f[k].w - m));
            }
            z = m > m_old ? z * ex(m_old - m) + s : z + s;
        } else {
#pragma unroll
            for (int k = 0; k < WIDE_U; k++) {
                const int i = 4 * (v0 + k * THREADS);
                if (f[k].x > m) { m = f[k].x; am = i; }
                if (f[k].y > m) { m = f[k].y; am = i + 1; }
                if (f[k].z > m) { m = f[k].z; am = i + 2; }
                if (f[k].w > m) { m = f[k].w; am = i + 3; }
            }
        }
    };
    constexpr int STEP = WIDE_U * THREADS;
    load(threadIdx.x, fa);
    for (int v0 = threadIdx.x; v0 < nvec; v0 += 2 * STEP) {
        load(v0 + STEP, fb); // (past the row: -inf, exponentials 0)
        take(v0, fa);
        if (v0 + 2 * STEP < nvec) load(v0 + 2 * STEP, fa);
        if (v0 + STEP < nvec) take(v0 + STEP, fb);
    }
    float mx = m;
    block_argmax(mx, am, redv, redi);
    if (invT > 0.f) {
        __syncthreads(); // redv is read above
        z = block_sum(m < mx ? z * expf((m - mx) * invT) : z, redv);
    } else {
        z = 1.f;
    }
    if (threadIdx.x == 0) {
        // candidate i is accepted iff u_i < p_i / q_i: the verdict is the sign bit of z (a NaN accepts nothing)
        const bool ok = c >= 0 && c < V && ui < expf((lc - mx) * invT) / z / fmaxf(qc, 1.17549435e-38f);
        z = ok ? -fabsf(z) : fabsf(z);
        stats[3 * blockIdx.x] = mx;
        stats[3 * blockIdx.x + 1] = z;
        stats[3 * blockIdx.x + 2] = __int_as_float(am);
    }
}

// Length of the accepted prefix of a sequence with `gamma` candidates, from the signs verify_stats_wide_kernel gave its sums
// (every wave for itself: one load and a vote).
__device__ __forceinline__ int accepted_prefix(const float *st, int gamma)
{
    const int lane = threadIdx.x % WAVE;
    const int ok = lane < gamma ? __float_as_int(st[3 * lane + 1]) < 0 : 0;
    return __ffsll((unsigned long long)~__ballot(ok)) - 1; // (lane gamma <= SD_MAX_GAMMA always votes 0)
}

// Weights the next token is drawn from: p of the deciding row, or max(0, p - q) where it was rejected (q != nullptr).
struct DrawWeights {
    const float4 *row, *q;
    float mx, invT, invZ;
    __device__ __forceinline__ float4 operator()(int v) const { return of(row[v], q ? q[v] : make_float4(0.f, 0.f, 0.f, 0.f)); }
    __device__ __forceinline__ float4 of(float4 f, float4 w) const
    {
        float4 p;
        p.x = expf((f.x - mx) * invT) * invZ;
        p.y = expf((f.y - mx) * invT) * invZ;
        p.z = expf((f.z - mx) * invT) * invZ;
        p.w = expf((f.w - mx) * invT) * invZ;
        if (q) { // (uniform)
            p = make_float4(fmaxf(p.x - w.x, 0.f), fmaxf(p.y - w.y, 0.f), fmaxf(p.z - w.z, 0.f), fmaxf(p.w - w.w, 0.f));
        }
        return p;
    }
};

// T > 0.  Block j * (gamma + 1) + s: mass of slice s of sequence j's deciding row, left in the argmax entry of its row s.
__global__ __launch_bounds__(512) void verify_mass_wide_kernel(const float *logits, float *stats, int gamma, int V, float T,
                                                               const float *q, const int32_t *seq_ids, CtxView cv)
{
    __shared__ float red[32];
    const int n_slices = gamma + 1, j = blockIdx.x / n_slices, s = blockIdx.x % n_slices, stride_g = gamma;
    {   // with per-sequence candidate counts this sequence has gj <= gamma candidates (and gj + 1 live rows)
        const int bb = seq_ids ? seq_ids[j] : j;
        if (cv.gam && bb >= 0 && bb < cv.B) gamma = seq_gamma(cv, bb, gamma);
    }
    const float *rows = logits + (size_t)j * (stride_g + 1) * V, *qj = q + (size_t)j * stride_g * V;
    float *st = stats + (size_t)j * (stride_g + 1) * 3;
    const float invT = inv_temperature(T);
    const int n_acc = accepted_prefix(st, gamma);
    const DrawWeights w = {(const float4 *)(rows + (size_t)n_acc * V),
                           n_acc < gamma ? (const float4 *)(qj + (size_t)n_acc * V) : nullptr, st[3 * n_acc], invT,
                           1.0f / fabsf(st[3 * n_acc + 1])};
    const int nvec = V / 4, per = (nvec + n_slices - 1) / n_slices, v_end = min(nvec, (s + 1) * per);
    float mass = 0.f;
#pragma unroll 4
    for (int v = s * per + threadIdx.x; v < v_end; v += 512) {
        const float4 f = w(v);
        mass += ((f.x + f.y) + f.z) + f.w;
    }
    mass = block_sum(mass, red);
    if (threadIdx.x == 0) st[3 * s + 2] = mass;
}

// T > 0.  One block per sequence: the slice whose masses pass u * Z, searched with the rule of block_pick_cdf (segments
// of 1024 vectors, then a scan of the segment that holds the target).  Without candidates (gamma == 0) there is one slice,
// the whole row: its masses are left to block_pick_cdf and no launch before this one adds them up (one row of 32772
// / 128000 / 262144 columns, whole call: 34 / 86 / 158 us with that launch, 27 / 65 / 118 without).  That is an instance of its own
// (NSEG -1): sharing the one whose slices do not fit registers costs 8 rows of 33000 columns 25.8 us instead of 24.8, of 50000 31.5
// instead of 30.4.
template <int NSEG>
__global__ __launch_bounds__(1024) void verify_pick_wide_kernel(const float *logits, const float *stats, int gamma, int V, float T,
                                                                const int32_t *cand, const float *q, const float *u,
                                                                const int32_t *seq_ids, int32_t *n_acc_out,
                                                                int32_t *next_out, int commit, CtxView cv)
{
    __shared__ PickScratch ps;
    __shared__ FastScratch fs;
    const int j = blockIdx.x, stride_g = gamma, n_slices = gamma + 1;
    const int bb = seq_ids ? seq_ids[j] : j;
    if (cv.gam && bb >= 0 && bb < cv.B) gamma = seq_gamma(cv, bb, gamma);
    const float *rows = logits + (size_t)j * (stride_g + 1) * V;
    const float *st = stats + (size_t)j * (stride_g + 1) * 3;
    const int n_acc = accepted_prefix(st, gamma);
    const float uu = u[(size_t)j * (stride_g + 1) + gamma];
    const DrawWeights w = {(const float4 *)(rows + (size_t)n_acc * V),
                     n_acc < gamma ? (const float4 *)(q + ((size_t)j * stride_g + n_acc) * V) : nullptr, st[3 * n_acc],
                     inv_temperature(T), 1.0f / fabsf(st[3 * n_acc + 1])};
    const int nvec = V / 4, per = (nvec + n_slices - 1) / n_slices;
    float Z = 0.f;
    if (NSEG >= 0 && stride_g)
        for (int s = 0; s < n_slices; s++) Z += st[3 * s + 2];
    int next;
    const bool whole = NSEG < 0 || (NSEG == 0 && !stride_g), empty = w.q && !(Z > 0.f);
    if (whole || empty) { // (whole: w.q is null anyway) numerically empty residual: draw from p
        const DrawWeights p = {w.row, nullptr, w.mx, w.invT, w.invZ};
        next = block_pick_cdf(p, V, uu, &ps, nullptr);
    } else {
        // every thread walks the slice masses in the same order: first slice whose running sum exceeds the target, else
        // (rounding) the last slice of positive mass
        const float target = uu * Z;
        float cum = 0.f, base = 0.f, base_last = 0.f;
        int s_pick = -1, s_last = 0;
        for (int s = 0; s < n_slices; s++) {
            const float mass = st[3 * s + 2];
            if (mass > 0.f) {
                s_last = s;
                base_last = cum;
            }
            if (s_pick < 0 && cum + mass > target) {
                s_pick = s;
                base = cum;
            }
            cum += mass;
        }
        if (s_pick < 0) {
            s_pick = s_last;
            base = base_last;
        }
        const int v_begin = s_pick * per, v_end = min(nvec, v_begin + per);
        if constexpr (NSEG > 0) { // the slice fits the block's registers
            RowRegs<NSEG> f, r;
            const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int it = 0; it < NSEG; it++) {
                // (unconditional loads: a choice between a vector of the row and a zero one would be made of their addresses, with
                // the zero in scratch memory and flat loads)
                const int v = min(v_begin + it * 1024 + (int)threadIdx.x, v_end - 1);
                f.f[it] = w.row[v];
                r.f[it] = zero;
                if (w.q) r.f[it] = w.q[v]; // (uniform)
            }
#pragma unroll
            for (int it = 0; it < NSEG; it++) f.f[it] = v_begin + it * 1024 + (int)threadIdx.x < v_end ? w.of(f.f[it], r.f[it]) : zero;
            next = pick_regs_range<1024>(f, V, v_begin, v_end, base, target, &fs);
        } else
            next = block_pick_range(w, v_begin, v_end, V, base, target, &ps);
    }
    if (threadIdx.x == 0) {
        n_acc_out[j] = n_acc;
        next_out[j] = next;
        if (commit) {
            if (bb >= 0 && bb < cv.B) commit_one(cv, bb, gamma, cand + (size_t)j * stride_g, n_acc, next);
            else atomicOr(cv.status, 4);
        }
    }
}

// Rows that fit a block's registers, in two launches.  verify_rows_kernel: one block per logits row (n_seq * (gamma + 1)
// blocks), which reads the row once into registers and settles everything that row could decide: its acceptance test
// and - if its candidate is rejected, or it is the row behind the last candidate - the token that would be drawn there,
// from registers it holds anyway.  Later rows of a sequence do that in vain; they run beside the others.  The verdicts
// take the three words per row of the caller's workspace: (accepted, token drawn, argmax).  verify_finish_kernel: one
// wave per sequence reads its verdicts: accepted prefix, token of the row behind it, commit.
// Bound: latency of one row's chain (load, max, exponentials, sum, q, scan).  Measured, 32000 columns, kernel durations
// under the profiler (before: row statistics in one launch, the decision from a second reading of the deciding row in
// another): 6 rows 8.1 + 17.9 -> 12.7 + 2.7 us, 192 rows 10.2 + 25.1 -> 18.3 + 4.1; whole call of 6 rows among others 21.4 ->
// 13.5 us.
// Stamped in the kernel at 6 rows of 32000 columns, before / now (us): loads until the row is there 1.4 / 0.7 (a branch per
// vector), maximum, exponentials and sum 4.6 / 3.9 (expf), residual 0.25, pick 3.8 / 2.5 (a reduction over the wave per
// segment): 11.0 -> 8.1.  What is left of it is instruction issue, four waves on each SIMD of one compute unit.
// EARLY_Q (up to 256 rows, a block per compute unit): q is requested together with the row, whatever the verdict will be
// (6 rows: 1.1 us); with more rows than units two blocks share one, q is read only where it is needed.
// DRAW false (more rows, see launch_verify_tail): the row settles its test only and leaves (max, sum, accepted) for verify_draw_kernel.
template <bool DRAW, bool EARLY_Q, int RT, int NSEG>
__global__ __launch_bounds__(RT, EARLY_Q ? 4 : 8) void verify_rows_kernel(const float *logits, int gamma, int V, float T, const int32_t *cand,
                                                                  const float *q, const float *u, const int32_t *seq_ids,
                                                                  CtxView cv, float *stats)
{
    constexpr int QH = NSEG < 4 ? NSEG : 4;
    __shared__ FastScratch fs;
    __shared__ PickScratch ps;
    const int stride_g = gamma; // row slots of the call: strides of cand, q and u
    const int j = blockIdx.x / (gamma + 1), i = blockIdx.x % (gamma + 1);
    const int bb = seq_ids ? seq_ids[j] : j;
    // with per-sequence candidate counts this sequence has gj <= gamma candidates (and gj + 1 live rows)
    if (cv.gam && bb >= 0 && bb < cv.B) gamma = seq_gamma(cv, bb, gamma);
    const float *row = logits + ((size_t)j * (stride_g + 1) + i) * V;
    float *st = stats + ((size_t)j * (stride_g + 1) + i) * 3;
    if (i > gamma) return; // (uniform) not a live row
    RowRegs<NSEG> r;
    row_load<RT>(row, V, r);
    const int c = i < gamma ? cand[(size_t)j * stride_g + i] : -1;
    const bool c_in = c >= 0 && c < V;
    float lc = 0.f, qc = 1.f, ui = 0.f, uu = 0.f;
    const float *qrow = q + ((size_t)j * stride_g + i) * V;
    if (T > 0.f) {
        ui = u[(size_t)j * (stride_g + 1) + i];
        uu = u[(size_t)j * (stride_g + 1) + gamma];
        if (c_in) {
            lc = row[c];
            qc = qrow[c];
        }
    }
    RowRegs<NSEG> qr;
    if (EARLY_Q && T > 0.f && i < gamma) row_load<RT>(qrow, V, qr);
    row_fill<RT>(V, row_filler(T), r);
    const float invT = inv_temperature(T);
    float mx, z;
    int am;
    row_stats_regs<RT>(r, invT, &fs, mx, am, z);
    // candidate i is accepted iff u_i < p_i / q_i (T > 0) or it is the row's argmax (T == 0)
    bool ok = false;
    int pick = am;
    if (T == 0.f) {
        ok = i < gamma && c == am;
    } else {
        if (c_in) ok = ui < expf((lc - mx) * invT) / z / fmaxf(qc, 1.17549435e-38f);
        if (DRAW && !ok) { // (uniform) the draw this row would make: from max(0, p - q), behind the last candidate from p
            const float invZ = 1.0f / z;
            row_scale(r, invZ);
            if (i < gamma) {
#pragma unroll
                for (int h = 0; h < NSEG; h += QH) { // (four segments of q at a time: registers for two blocks per unit)
                    float4 w[QH];
#pragma unroll
                    for (int k = 0; k < QH; k++) {
                        if (EARLY_Q) w[k] = qr.f[h + k];
                        else w[k] = *(const float4 *)(qrow + 4 * min((h + k) * RT + (int)threadIdx.x, V / 4 - 1));
                    }
#pragma unroll
                    for (int k = 0; k < QH; k++) residual((h + k) * RT + (int)threadIdx.x < V / 4, r.f[h + k], w[k]);
                    if (!EARLY_Q) SD_SCHED_FENCE();
                }
            }
            float mass;
            pick = pick_regs<RT>(r, V, uu, &fs, &mass);
            if (i < gamma && !(mass > 0.f)) { // (uniform) numerically empty residual: draw from p
                auto p_of = [&](int v) {
                    float4 f = load4_guard(row, v, V, -3.0e38f);
                    f.x = expf((f.x - mx) * invT) * invZ;
                    f.y = expf((f.y - mx) * invT) * invZ;
                    f.z = expf((f.z - mx) * invT) * invZ;
                    f.w = expf((f.w - mx) * invT) * invZ;
                    return f;
                };
                pick = block_pick_cdf(p_of, V, uu, &ps, nullptr);
            }
        }
    }
    if (threadIdx.x == 0) {
        st[0] = DRAW ? __int_as_float(ok ? 1 : 0) : mx;
        st[1] = DRAW ? __int_as_float(pick) : z;
        st[2] = __int_as_float(DRAW ? am : ok ? 1 : 0);
    }
}

// Behind verify_rows_kernel<false>: one block per sequence finds the accepted prefix and draws from the row behind it, which
// it reads again with the maximum and sum that are known.
template <int RT, int NSEG>
__global__ __launch_bounds__(RT, 4) void verify_draw_kernel(const float *logits, const float *stats, int gamma, int V, float T,
                                                            const int32_t *cand, const float *q, const float *u,
                                                            const int32_t *seq_ids, int32_t *n_acc_out, int32_t *next_out,
                                                            int commit, CtxView cv)
{
    __shared__ FastScratch fs;
    const int j = blockIdx.x, lane = threadIdx.x % WAVE, stride_g = gamma;
    const int bb = seq_ids ? seq_ids[j] : j;
    if (cv.gam && bb >= 0 && bb < cv.B) gamma = seq_gamma(cv, bb, gamma);
    const float *st = stats + (size_t)j * (stride_g + 1) * 3;
    const int ok = lane < gamma ? __float_as_int(st[3 * lane + 2]) : 0;
    const int n_acc = __ffsll((unsigned long long)~__ballot(ok)) - 1; // (lane gamma <= SD_MAX_GAMMA always votes 0)
    const float uu = u[(size_t)j * (stride_g + 1) + gamma], invT = inv_temperature(T);
    const float mx = st[3 * n_acc], invZ = 1.0f / st[3 * n_acc + 1];
    RowRegs<NSEG> r, w;
    row_load<RT>(logits + ((size_t)j * (stride_g + 1) + n_acc) * V, V, r);
    if (n_acc < gamma) row_load<RT>(q + ((size_t)j * stride_g + n_acc) * V, V, w);
    row_fill<RT>(V, row_filler(T), r);
    const RowExp ex(mx, invT);
#pragma unroll
    for (int it = 0; it < NSEG; it++) r.f[it] = ex(r.f[it]);
    row_scale(r, invZ);
    float mass = 0.f;
    int next = 0;
    if (n_acc < gamma) { // (uniform)
#pragma unroll
        for (int it = 0; it < NSEG; it++) {
            float4 f = r.f[it];
            residual(it * RT + (int)threadIdx.x < V / 4, f, w.f[it]);
            w.f[it] = f;
        }
        next = pick_regs<RT>(w, V, uu, &fs, &mass);
    }
    if (!(mass > 0.f)) next = pick_regs<RT>(r, V, uu, &fs, nullptr); // everything accepted, or a numerically empty residual: draw from p
    if (threadIdx.x == 0) {
        n_acc_out[j] = n_acc;
        next_out[j] = next;
        if (commit) {
            if (bb >= 0 && bb < cv.B) commit_one(cv, bb, gamma, cand + (size_t)j * stride_g, n_acc, next);
            else atomicOr(cv.status, 4);
        }
    }
}

// One wave per sequence.  T > 0: the verdicts of verify_rows_kernel; T == 0: the rows' argmax entries, whichever kernel
// left them.
__global__ __launch_bounds__(WAVE) void verify_finish_kernel(const float *stats, int gamma, float T, const int32_t *cand,
                                                             const int32_t *seq_ids, int32_t *n_acc_out, int32_t *next_out,
                                                             int commit, CtxView cv)
{
    const int j = blockIdx.x, i = threadIdx.x, stride_g = gamma;
    const int bb = seq_ids ? seq_ids[j] : j;
    const bool in = bb >= 0 && bb < cv.B;
    const float *st = stats + (size_t)j * (stride_g + 1) * 3;
    const int32_t *cj = cand + (size_t)j * stride_g;
    if (cv.gam && in) gamma = seq_gamma(cv, bb, gamma);
    int ok = 0, tok = 0;
    if (i <= gamma) {
        const int am = __float_as_int(st[3 * i + 2]);
        tok = T == 0.f ? am : __float_as_int(st[3 * i + 1]);
        if (i < gamma) ok = T == 0.f ? cj[i] == am : __float_as_int(st[3 * i]) != 0;
    }
    const int n_acc = __ffsll((unsigned long long)~__ballot(ok)) - 1; // (lane gamma <= SD_MAX_GAMMA always votes 0)
    const int next = __builtin_amdgcn_readlane(tok, n_acc);
    if (i == 0) {
        n_acc_out[j] = n_acc;
        next_out[j] = next;
        if (commit) {
            if (in) commit_one(cv, bb, gamma, cj, n_acc, next);
            else atomicOr(cv.status, 4);
        }
    }
}

hipError_t launch_verify_tail(hipStream_t s, const float *logits, int n_seq, int gamma, int V, float T,
                              const int32_t *cand, const float *q, const float *u, const int32_t *seq_ids,
                              int32_t *n_acc, int32_t *next_tok, int commit, CtxView cv, float *stats)
{
    const int n_rows = n_seq * (gamma + 1);
    if (V <= ROW_NSEG * ROW_THREADS * 4) {
#define SD_VERIFY_ROWS(DRAW, EARLY, RT, NSEG)                                                                                \
    hipLaunchKernelGGL((verify_rows_kernel<DRAW, EARLY, RT, NSEG>), dim3(n_rows), dim3(RT), 0, s, logits, gamma, V, T, cand, \
                       q, u, seq_ids, cv, stats)
#define SD_VERIFY_ROWS_EARLY(RT, NSEG) SD_VERIFY_ROWS(true, true, RT, NSEG)
#define SD_VERIFY_ROWS_LATE(RT, NSEG) SD_VERIFY_ROWS(true, false, RT, NSEG)
#define SD_VERIFY_ROWS_TEST(RT, NSEG) SD_VERIFY_ROWS(false, false, RT, NSEG)
#define SD_VERIFY_DRAW(RT, NSEG)                                                                                             \
    hipLaunchKernelGGL((verify_draw_kernel<RT, NSEG>), dim3(n_seq), dim3(RT), 0, s, logits, stats, gamma, V, T, cand, q, u,  \
                       seq_ids, n_acc, next_tok, commit, cv)
        // More rows than compute units: a draw made in vain takes the unit from a row that still waits for one, so the rows
        // settle their tests only and one block per sequence draws.  Measured, 32000 columns, draws in every row / in the
        // deciding row (us; all candidates rejected, three in four accepted, all accepted): 288 rows 28.0 / 24.5, 26.8 / 24.9,
        // 21.2 / 22.8; 576 rows 41.6 / 31.4, 34.8 / 31.7, 29.0 / 29.6; 4096 rows 225 / 107, 152 / 106, 127 / 102.  With one
        // candidate every other row draws anyway (512 sequences: 53.9 / 58.1, 44.4 / 51.9, 40.3 / 50.3).
        if (T > 0.f && gamma > 1 && n_rows > 256) {
            SD_ROW_SHAPES(V, SD_VERIFY_ROWS_TEST);
            SD_ROW_SHAPES(V, SD_VERIFY_DRAW);
            return hipGetLastError();
        }
        if (n_rows <= 256) SD_ROW_SHAPES(V, SD_VERIFY_ROWS_EARLY);
        else SD_ROW_SHAPES(V, SD_VERIFY_ROWS_LATE);
        hipLaunchKernelGGL(verify_finish_kernel, dim3(n_seq), dim3(WAVE), 0, s, stats, gamma, T, cand, seq_ids, n_acc, next_tok, commit,
                           cv);
        return hipGetLastError();
    }
#define SD_STATS_WIDE(RT, NT)                                                                                             \
    hipLaunchKernelGGL((verify_stats_wide_kernel<RT, NT>), dim3(n_rows), dim3(RT), 0, s, logits, gamma, V, T, cand, q, u, stats)
    // (128 MB of logits; 256 MB where they are read again)
    // Blocks of 1024 threads put two rows on a compute unit, so a little more than one row or two rows a unit leaves most of
    // the chip waiting for the few units with another: 257 to 511 rows go in blocks of 512 threads, 513 to 767 in blocks of
    // 256, all resident at once.  Whole call, T = 0.7, 1024 / 512 / 256 threads (us): 270 rows of 128000 columns 53.2 / 48.8 /
    // 57.7, of 262144 91.5 / 81.1 / 95.7; 360 rows of 262144 94.9 / 90.0 / 99.5; 576 rows of 128000 74.4 / 77.2 / 70.7, of 262144 133 /
    // 136 / 122; 800 rows of 128000 104.3 / 103.9 / 104.2; 1350 rows of 128000 139 / 138 / 144.
    // The upper edge, in turn in one process: 603, 675, 765 and 810 rows of 64000 columns 45.3 / 46.0 / 42.4, 46.7 / 47.3 / 45.1, 49.1 / 49.6 / 48.1, 53.9 / 53.9 /
    // 53.9, of 128000 72.4 / 73.9 / 68.5, 75.3 / 76.2 / 73.5, 80.9 / 81.5 / 80.4, 90.1 / 91.4 / 90.3, of 262144 131.9 / 133.2 / 124.2, 137.2 / 138.4 / 134.8,
    // 151.4 / 149.9 / 148.9, 171.2 / 170.7 / 169.9; greedy 3 to 10 % at 603 rows and 1 to 5 at 765.  (180000 columns, 765 rows: 2 % behind, greedy 7.)
    if ((size_t)n_rows * V > ((size_t)1 << (T > 0.f && gamma == 0 ? 26 : 25))) {
        if (n_rows > 256 && n_rows < 512) SD_STATS_WIDE(512, true);
        else if (n_rows > 512 && n_rows < 768) SD_STATS_WIDE(256, true);
        else SD_STATS_WIDE(1024, true);
    } else if (n_rows >= 512) SD_STATS_WIDE(512, false);
    else SD_STATS_WIDE(1024, false);
    if (T > 0.f) {
        if (gamma > 0)
            hipLaunchKernelGGL(verify_mass_wide_kernel, dim3(n_rows), dim3(512), 0, s, logits, stats, gamma, V, T, q, seq_ids, cv);
#define SD_PICK_WIDE(NSEG)                                                                                                    \
    hipLaunchKernelGGL((verify_pick_wide_kernel<NSEG>), dim3(n_seq), dim3(1024), 0, s, logits, stats, gamma, V, T, cand, q, u, \
                       seq_ids, n_acc, next_tok, commit, cv)
        const int per = (V / 4 + gamma) / (gamma + 1); // vectors of a slice
        if (gamma == 0) SD_PICK_WIDE(-1);
        else if (per > 8192) SD_PICK_WIDE(0);
        else if (per > 4096) SD_PICK_WIDE(8);
        else if (per > 2048) SD_PICK_WIDE(4);
        else SD_PICK_WIDE(2);
    } else // (greedy: the decision needs the argmax entries only)
        hipLaunchKernelGGL(verify_finish_kernel, dim3(n_seq), dim3(WAVE), 0, s, stats, gamma, T, cand, seq_ids, n_acc, next_tok, commit,
                           cv);
    return hipGetLastError();
}

// ---------------------------------------------------------------- routing
__global__ void route_kernel(const float *W, const float *b, int n_drafts, int emb, const float *e, int n,
                             int32_t *id)
{
    int i = blockIdx.x;
    int lane = threadIdx.x;
    float best = -3.0e38f;
    int bi = 0;
    for (int k = 0; k < n_drafts; k++) {
        float acc = 0.f;
        for (int t = lane; t < emb; t += WAVE) acc += W[(size_t)k * emb + t] * e[(size_t)i * emb + t];
        acc = wave_sum(acc) + (b ? b[k] : 0.f);
        if (acc > best) {
            best = acc;
            bi = k;
        }
    }
    if (lane == 0) id[i] = bi;
}

hipError_t launch_route(hipStream_t s, const float *W, const float *b, int n_drafts, int emb, const float *e, int n,
                        int32_t *id)
{
    hipLaunchKernelGGL(route_kernel, dim3(n), dim3(WAVE), 0, s, W, b, n_drafts, emb, e, n, id);
    return hipGetLastError();
}

// ---------------------------------------------------------------- new sequences
__global__ __launch_bounds__(256) void set_tokens_kernel(CtxView cv, const int32_t *staged, int n)
{
    const int32_t *entry = staged + 3 * (size_t)blockIdx.x;
    const int b = entry[0], len = entry[1];
    const int32_t *src = staged + 3 * (size_t)n + entry[2];
    int32_t *dst = cv.tokens + cv.off[b];
    for (int i = threadIdx.x; i < len; i += 256) dst[i] = src[i];
    if (threadIdx.x < SD_MAX_SLOTS) cv.kvlen[(size_t)threadIdx.x * cv.B + b] = 0;
    if (threadIdx.x < 2) cv.pol[(size_t)threadIdx.x * cv.B + b] = 0; // a new sequence starts without acceptance history
    if (threadIdx.x == 0) cv.ntok[b] = len;
}

hipError_t launch_set_tokens(hipStream_t s, CtxView cv, const int32_t *staged, int n)
{
    hipLaunchKernelGGL(set_tokens_kernel, dim3(n), dim3(256), 0, s, cv, staged, n);
    return hipGetLastError();
}

// ---------------------------------------------------------------- synthetic cache load
template <typename T>
__global__ void set_kv_kernel(const T *k_rows, const T *v_rows, int len, int H, int hd, int64_t seq_off,
                              int64_t total_cap, T *Kl, T *Vtl)
{
    size_t n = (size_t)len * H * hd;
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (size_t)gridDim.x * blockDim.x) {
        int d = i % hd;
        int h = (i / hd) % H;
        int t = i / ((size_t)hd * H);
        Kl[(size_t)h * total_cap * hd + kt_offset(hd, seq_off + t, d)] = k_rows[i];
        Vtl[(size_t)h * hd * total_cap + vt_offset(hd, seq_off + t, d)] = v_rows[i];
    }
}

hipError_t launch_set_kv(hipStream_t s, int dtype, const void *k_rows, const void *v_rows, int len, int H, int hd,
                         int64_t seq_off, int64_t total_cap, void *Kl, void *Vtl)
{
    size_t n = (size_t)len * H * hd;
    int blocks = (int)((n + 255) / 256);
    if (blocks > 65535) blocks = 65535;
    if (blocks < 1) blocks = 1;
    if (dtype == SD_BF16)
        hipLaunchKernelGGL(set_kv_kernel<bf16_t>, dim3(blocks), dim3(256), 0, s, (const bf16_t *)k_rows,
                           (const bf16_t *)v_rows, len, H, hd, seq_off, total_cap, (bf16_t *)Kl, (bf16_t *)Vtl);
    else
        hipLaunchKernelGGL(set_kv_kernel<float>, dim3(blocks), dim3(256), 0, s, (const float *)k_rows,
                           (const float *)v_rows, len, H, hd, seq_off, total_cap, (float *)Kl, (float *)Vtl);
    return hipGetLastError();
}

template <typename T>
__global__ void get_kv_kernel(T *k_rows, T *v_rows, int len, int H, int hd, int64_t seq_off, int64_t total_cap, const T *Kl, const T *Vtl)
{
    size_t n = (size_t)len * H * hd;
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (size_t)gridDim.x * blockDim.x) {
        int d = i % hd;
        int h = (i / hd) % H;
        int t = i / ((size_t)hd * H);
        k_rows[i] = Kl[(size_t)h * total_cap * hd + kt_offset(hd, seq_off + t, d)];
        v_rows[i] = Vtl[(size_t)h * hd * total_cap + vt_offset(hd, seq_off + t, d)];
    }
}

hipError_t launch_get_kv(hipStream_t s, int dtype, void *k_rows, void *v_rows, int len, int H, int hd, int64_t seq_off, int64_t total_cap,
                         const void *Kl, const void *Vtl)
{
    const int blocks = (int)std::min<size_t>(65535, ((size_t)len * H * hd + 255) / 256);
    if (dtype == SD_BF16)
        hipLaunchKernelGGL(get_kv_kernel<bf16_t>, dim3(blocks), dim3(256), 0, s, (bf16_t *)k_rows, (bf16_t *)v_rows, len, H, hd, seq_off, total_cap,
                           (const bf16_t *)Kl, (const bf16_t *)Vtl);
    else
        hipLaunchKernelGGL(get_kv_kernel<float>, dim3(blocks), dim3(256), 0, s, (float *)k_rows, (float *)v_rows, len, H, hd, seq_off, total_cap,
                           (const float *)Kl, (const float *)Vtl);
    return hipGetLastError();
}

// ---------------------------------------------------------------- measurement helper: a plain streaming read
// Reads `n_vec` 16-byte vectors once and folds them into one word (written only if it hits a magic value, so that
// the loads cannot be dropped): what the memory system gives a kernel that does nothing but read, the practical
// ceiling the weight-streaming GEMMs are held against.  NT = false: grid-strided, ordinary loads; NT = true: every
// block reads one contiguous range with the nontemporal hint, eight loads in flight per thread - the fastest
// pattern found on this part (1 GiB: 7.0 against 5.4-6.3 TB/s).
typedef __attribute__((ext_vector_type(4))) unsigned int sr_u32x4;
template <bool NT, bool FOLD>
__global__ __launch_bounds__(256) void stream_read_kernel(const sr_u32x4 *__restrict__ p, size_t n_vec, uint32_t *out)
{
    constexpr int U = NT ? 8 : 4;
    size_t i, stride, end;
    if (NT) {
        const size_t per = (n_vec + gridDim.x - 1) / gridDim.x;
        i = (size_t)blockIdx.x * per + threadIdx.x;
        stride = 256;
        end = min(n_vec, (size_t)(blockIdx.x + 1) * per);
    } else {
        i = (size_t)blockIdx.x * 256 + threadIdx.x;
        stride = (size_t)gridDim.x * 256;
        end = n_vec;
    }
    uint32_t acc = 0;
    for (; i + (U - 1) * stride < end; i += U * stride) {
        sr_u32x4 v[U];
#pragma unroll
        for (int u = 0; u < U; u++) v[u] = ld_stream<NT>(p + i + u * stride);
#pragma unroll
        for (int u = 0; u < U; u++) acc ^= v[u].x ^ v[u].y ^ v[u].z ^ v[u].w;
    }
    for (; i < end; i += stride) {
        const sr_u32x4 a = ld_stream<NT>(p + i);
        acc ^= a.x ^ a.y ^ a.z ^ a.w;
    }
    if (FOLD) { // checking mode: XOR of every word read, accumulated into out[0] (one atomic per wave)
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) acc ^= __shfl_xor(acc, o, 64);
        if ((threadIdx.x & 63) == 0) atomicXor(out, acc);
    } else if (acc == 0x9e3779b9u) {
        out[0] = acc;
    }
}

int g_stream_read_nt = 1; // option "stream_read_nt"
hipError_t launch_stream_read(hipStream_t s, const void *buf, size_t bytes, uint32_t *out)
{
    const sr_u32x4 *p = (const sr_u32x4 *)buf;
    const size_t n_vec = bytes / 16;
    switch ((g_stream_read_nt & 1) | (g_stream_read_nt & 2)) { // bit 1: checking mode (XOR of all words into *out)
    case 0: hipLaunchKernelGGL((stream_read_kernel<false, false>), dim3(2048), dim3(256), 0, s, p, n_vec, out); break;
    case 1: hipLaunchKernelGGL((stream_read_kernel<true, false>), dim3(2048), dim3(256), 0, s, p, n_vec, out); break;
    case 2: hipLaunchKernelGGL((stream_read_kernel<false, true>), dim3(2048), dim3(256), 0, s, p, n_vec, out); break;
    default: hipLaunchKernelGGL((stream_read_kernel<true, true>), dim3(2048), dim3(256), 0, s, p, n_vec, out); break;
    }
    return hipGetLastError();
}
