// Attention over an 8-bit cache (kv8.hip): softmax(scale q K^T) V with K and V held as codes and a scale per (token, head).
//
//   s_j = scale * ks_j * (q . kc_j),   out = sum_j exp2(s_j) vs_j vc_j / sum_j exp2(s_j)      (scale in base-2 exponent units)
#include <algorithm>

#include "kv8.h"

// Tokens [0, n_first) and [lo, hi) are what row i of a sequence sees.
struct Kv8Seen {
    int n_first, lo, hi;
};
__device__ __forceinline__ Kv8Seen kv8_seen(const Kv8Attn &a, int len, int i, int cap)
{
    const int64_t end = a.causal ? (int64_t)len + i + 1 : len;
    Kv8Seen s;
    s.hi = (int)max((int64_t)0, min(end, (int64_t)cap));
    s.lo = a.window ? (int)min((int64_t)s.hi, max((int64_t)0, end - a.window)) : 0;
    s.n_first = min(a.sinks, s.lo);
    return s;
}

__device__ __forceinline__ void kv8_store_out(const Kv8Attn &a, int r, int h, int hd, int d, float v)
{
    if (a.out_planes) store_act((bf16_t *)a.out, act_index(a.av, r, h * hd + d, a.n_heads * hd), a.av.plane, v);
    else if (a.dtype == SD_BF16) ((bf16_t *)a.out)[r * a.o_row + h * a.o_head + d] = from_float<bf16_t>(v);
    else ((float *)a.out)[r * a.o_row + h * a.o_head + d] = v;
}

// ---------------------------------------------------------------- the plain kernel
// One block per (row, head), every head width; 32-bit arithmetic throughout.  A chunk of 256 tokens at a time: a thread per token
// for the scores, then threads over dimensions and token groups for the output.
#define KG_CHUNK 256
__global__ __launch_bounds__(256) void kv8_attn_generic_kernel(Kv8View c, Kv8Rows rw, Kv8Attn a)
{
    __shared__ float sq[256], sp[KG_CHUNK], red[8], sacc[256 * 4];
    const int r = blockIdx.x, h = blockIdx.y, hd = c.hd, tid = threadIdx.x;
    const int j = kv8_owner(rw, r);
    if (j < 0 || j >= rw.n) return;
    const Kv8Seq s = kv8_seq(c, rw, j);
    const int i = r - s.row0;
    if (s.b < 0 || i >= s.n_rows) { // an unused slot of the path, or a sequence id out of range
        if (s.b < 0 && c.status && tid == 0) atomicOr(c.status, 4);
        if (rw.path)
            for (int d = tid; d < hd; d += 256) kv8_store_out(a, r, h, hd, d, 0.f);
        return;
    }
    const Kv8Seen seen = kv8_seen(a, s.len, i, c.cap[s.b]);
    const int n = seen.n_first + (seen.hi - seen.lo);
    const int64_t base = (int64_t)(h / (a.n_heads / c.kv_heads)) * c.tokens + c.off[s.b];
    for (int d = tid; d < hd; d += 256)
        sq[d] = a.dtype == SD_BF16 ? to_float(((const bf16_t *)a.q)[r * a.q_row + h * a.q_head + d]) : ((const float *)a.q)[r * a.q_row + h * a.q_head + d];
    // (a thread of the second step owns four dimensions, dg, of the tokens tg, tg + n_tg, ...)
    const int n_dg = hd / 4, dg = tid % n_dg, tg = tid / n_dg, n_tg = 256 / n_dg;
    float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int u0 = 0; u0 < n; u0 += KG_CHUNK) {
        __syncthreads(); // sq is there; nobody reads sp and red any more
        const int u = u0 + tid;
        const int t = u < seen.n_first ? u : seen.lo + (u - seen.n_first);
        float x = -INFINITY, vs = 0.f;
        if (u < n) {
            const uint4 *kp = (const uint4 *)(c.k + (base + t) * hd);
            float dot = 0.f;
            for (int d = 0; d < hd; d += 16) {
                const uint4 w = kp[d / 16];
                const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int e = 0; e < 16; e++) dot = fmaf(sq[d + e], (float)((int32_t)(ww[e / 4] << (24 - 8 * (e % 4))) >> 24), dot);
            }
            x = dot * c.ks[base + t] * a.scale;
            vs = c.vs[base + t];
        }
        float mx = x;
        for (int o = 32; o; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
        if ((tid & 63) == 0) red[tid >> 6] = mx;
        __syncthreads();
        const float m_new = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
        const float m_ref = m_new == -INFINITY ? 0.f : m_new; // (a NaN among the scores reaches the sum below)
        const float p = u < n ? __builtin_amdgcn_exp2f(x - m_ref) : 0.f, corr = __builtin_amdgcn_exp2f(m - m_ref);
        l = l * corr + p;
        sp[tid] = p * vs;
        m = m_new;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; e++) acc[e] *= corr;
        if (tg < n_tg)
            for (int k = tg; k < min(KG_CHUNK, n - u0); k += n_tg) {
                const int uu = u0 + k, tt = uu < seen.n_first ? uu : seen.lo + (uu - seen.n_first);
                const uint32_t w = *(const uint32_t *)(c.v + (base + tt) * hd + 4 * dg);
#pragma unroll
                for (int e = 0; e < 4; e++) acc[e] = fmaf(sp[k], (float)((int32_t)(w << (24 - 8 * e)) >> 24), acc[e]);
            }
    }
    for (int o = 32; o; o >>= 1) l += __shfl_xor(l, o, 64);
    __syncthreads();
    if ((tid & 63) == 0) red[4 + (tid >> 6)] = l;
#pragma unroll
    for (int e = 0; e < 4; e++) sacc[tid * 4 + e] = acc[e];
    __syncthreads();
    l = (red[4] + red[5]) + (red[6] + red[7]);
    for (int d = tid; d < hd; d += 256) {
        float o = 0.f;
        for (int g = 0; g < n_tg; g++) o += sacc[(g * n_dg + d / 4) * 4 + d % 4];
        kv8_store_out(a, r, h, hd, d, n ? o / l : 0.f);
    }
    if (a.lse && tid == 0) a.lse[(int64_t)r * a.n_heads + h] = n ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
}

int64_t kv8_attn_workspace(const Kv8View &c, const Kv8Rows &rw, const Kv8Attn &a)
{
    return 0;
}

hipError_t launch_kv8_attn(hipStream_t s, const Kv8View &c, const Kv8Rows &rw, const Kv8Attn &a, void *ws, int64_t ws_bytes)
{
    hipLaunchKernelGGL(kv8_attn_generic_kernel, dim3(a.total_rows, a.n_heads), dim3(256), 0, s, c, rw, a);
    return hipGetLastError();
}
