// Attention over an 8-bit cache (kv8.hip): softmax(scale q K^T) V with K and V held as codes and a scale per (token, head).
//
//   s_j = scale * ks_j * (q . kc_j),   out = sum_j exp2(s_j) vs_j vc_j / sum_j exp2(s_j)      (scale in base-2 exponent units)
#include <algorithm>
#include <type_traits>

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

// N (4 or 8) adjacent dimensions of one (row, head), d a multiple of N.  wide: rows of out allow 16-byte accesses.
template <int N>
__device__ __forceinline__ void kv8_store_run(const Kv8Attn &a, bool wide, int r, int h, int hd, int d, const float (&v)[N])
{
    if (a.out_planes) {
#pragma unroll
        for (int e = 0; e < N; e += 4)
            store_act4((bf16_t *)a.out, act_index(a.av, r, h * hd + d + e, a.n_heads * hd), a.av.plane, v[e], v[e + 1], v[e + 2], v[e + 3]);
    } else if (!wide) {
#pragma unroll
        for (int e = 0; e < N; e++) kv8_store_out(a, r, h, hd, d + e, v[e]);
    } else if (a.dtype == SD_BF16) {
        bf16_t *p = (bf16_t *)a.out + (r * a.o_row + h * a.o_head + d);
#pragma unroll
        for (int e = 0; e < N; e += 4) *(uint2 *)(p + e) = make_uint2(bf16x2_bits_rne(v[e], v[e + 1]), bf16x2_bits_rne(v[e + 2], v[e + 3]));
    } else {
        float *p = (float *)a.out + (r * a.o_row + h * a.o_head + d);
#pragma unroll
        for (int e = 0; e < N; e += 4) *(float4 *)(p + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
    }
}
__device__ __forceinline__ bool kv8_wide(const void *p, int64_t row, int64_t head, int dtype)
{
    const int64_t n = dtype == SD_BF16 ? 8 : 4;
    return (uintptr_t)p % 16 == 0 && row % n == 0 && head % n == 0;
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

// ---------------------------------------------------------------- few rows: one pass over the cache on the matrix cores
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
struct __attribute__((packed, aligned(4))) F4 { // four floats at any element
    float v[4];
};

#define K8_TILE 32
#define K8_P_SHIFT 14 // probabilities enter as p * (vs / E) * 2^14 < 2^15

union Half8 {
    f16x8 v;
    f16x2 h[4];
    uint32_t w[4];
};

// Eight codes of one token -> eight halves, exactly: with the sign bit flipped a code c is the byte c + 128, and 0x6400 | byte is the
// half 1024 + byte.
__device__ __forceinline__ f16x8 codes_to_half(uint32_t a, uint32_t b)
{
    Half8 r;
    const f16x2 bias = {(_Float16)1152.f, (_Float16)1152.f};
    a ^= 0x80808080u, b ^= 0x80808080u;
    r.w[0] = __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u);
    r.w[1] = __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u);
    r.w[2] = __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u);
    r.w[3] = __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u);
#pragma unroll
    for (int e = 0; e < 4; e++) r.h[e] -= bias;
    return r.v;
}
// Byte j of two words (sign bits flipped) -> two halves (c, c') * 2^-9: as 16-bit integers the bytes are the subnormal halves
// byte * 2^-24, and byte * 2^-24 * 2^15 - 2^-2 = (byte - 128) * 2^-9 without rounding.
template <int J>
__device__ __forceinline__ f16x2 pair_to_half(uint32_t lo, uint32_t hi)
{
    const uint32_t u = __builtin_amdgcn_perm(hi, lo, 0x0c000c00u | ((4 + J) << 16) | J);
    const f16x2 x = __builtin_bit_cast(f16x2, u), m = {(_Float16)32768.f, (_Float16)32768.f}, c = {(_Float16)-0.25f, (_Float16)-0.25f};
    return __builtin_elementwise_fma(x, m, c);
}
// two floats -> two halves, to nearest
__device__ __forceinline__ f16x2 half2_of(float a, float b)
{
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    const f32x2 v = {a, b};
    return __builtin_convertvector(v, f16x2);
}

// Maximum over the four 16-lane rows of a wave, left in every lane (see attn_mfma.hip).
__device__ __forceinline__ float rows4_max(float v)
{
    unsigned u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    u = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float rows4_sum(float v)
{
    unsigned u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    u = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// What the rows i0 .. i1 (inclusive) of a sequence see together, in tiles of 32 tokens: first the n_sink tiles from 0 on, then those from
// w0 on; T in all.  hi_max / lo_min: of any row, hi_min / lo_max: of every row.
struct Kv8Tiles {
    int hi_max, hi_min, lo_min, lo_max, n_sink, w0, T;
    __device__ __forceinline__ int token0(int t) const { return (t < n_sink ? t : w0 + (t - n_sink)) * K8_TILE; }
};
__device__ __forceinline__ Kv8Tiles kv8_tiles(const Kv8Attn &a, int len, int i0, int i1, int cap)
{
    const Kv8Seen first = kv8_seen(a, len, i0, cap), last = kv8_seen(a, len, i1, cap);
    Kv8Tiles t;
    t.hi_max = last.hi, t.hi_min = first.hi, t.lo_min = first.lo, t.lo_max = last.lo;
    t.w0 = t.lo_min / K8_TILE;
    t.n_sink = min((a.sinks + K8_TILE - 1) / K8_TILE, t.w0);
    t.T = t.n_sink + (t.hi_max + K8_TILE - 1) / K8_TILE - t.w0;
    return t;
}
// The tiles [t_begin, t_end) in the order a block takes them: those that every row sees whole lie together, [f0, f1), and come last (the order
// does not matter to the sums), so that the loops over either kind have one body each.
struct Kv8Order {
    int t_begin, f0, f1, n_left, n_edge, n;
    __device__ __forceinline__ int tile(int u) const { return u < n_left ? t_begin + u : u < n_edge ? f1 + (u - n_left) : f0 + (u - n_edge); }
};
__device__ __forceinline__ Kv8Order kv8_order(const Kv8Tiles &tl, int t_begin, int t_end)
{
    Kv8Order o;
    o.t_begin = t_begin;
    o.f0 = min(max(tl.n_sink + (tl.lo_max + K8_TILE - 1) / K8_TILE - tl.w0, t_begin), t_end);
    o.f1 = max(o.f0, min(tl.n_sink + tl.hi_min / K8_TILE - tl.w0, t_end));
    o.n_left = o.f0 - t_begin, o.n_edge = o.n_left + (t_end - o.f1), o.n = max(0, t_end - t_begin);
    return o;
}

// Tiles per split: what the launch was sized for, so that the blocks of short and long sequences do the same work - or, of a sequence
// longer than the launch was told of, an even share.
__device__ __forceinline__ int kv8_per_split(int T, int S, int per) { return max(per, (T + S - 1) / S); }

// 16 adjacent elements of a query row
template <int TERMS>
__device__ __forceinline__ void load_q16(const Kv8Attn &a, bool wide, int64_t at, float *x)
{
    if constexpr (TERMS == 1) {
        const bf16_t *p = (const bf16_t *)a.q + at;
        if (wide) {
#pragma unroll
            for (int v = 0; v < 2; v++) {
                const uint4 w = ((const uint4 *)p)[v];
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int e = 0; e < 4; e++) x[8 * v + 2 * e] = __uint_as_float(u[e] << 16), x[8 * v + 2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; e++) x[e] = to_float(p[e]);
        }
    } else {
        const float *p = (const float *)a.q + at;
        if (wide) {
#pragma unroll
            for (int v = 0; v < 4; v++) {
                const float4 w = ((const float4 *)p)[v];
                x[4 * v] = w.x, x[4 * v + 1] = w.y, x[4 * v + 2] = w.z, x[4 * v + 3] = w.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; e++) x[e] = p[e];
        }
    }
}
// Queries enter the products as halves.  They are scaled by one power of two for all rows that share it, so that the largest element
// (mx) lies in [2^14, 2^15): a half then holds every bf16 element down to 2^-31 of the largest exactly, two halves hold 22 bits of an
// fp32 one, and what smaller elements lose is 2^-39 of the largest - nothing in a score.
struct QScale {
    float up, down; // to the halves, and back
};
__device__ __forceinline__ QScale q_scale(float mx)
{
    const int e = min(127, max(-100, (int)(__float_as_uint(mx) >> 23) - 127)); // (kept where both factors are normal numbers)
    return QScale{__uint_as_float((uint32_t)(127 + 14 - e) << 23), __uint_as_float((uint32_t)(127 - 14 + e) << 23)};
}
// The Q^T operands of a 16-row set: lane (qi, grp) takes dimensions 64 j + 16 grp + 8 s .. + 8 into step 2 j + s, the order a 16-byte
// piece of the codes has them in.
template <int HD, int TERMS>
__device__ __forceinline__ void query_operands(const float (&x)[HD / 4], float up, f16x8 (&q)[TERMS][HD / 32])
{
#pragma unroll
    for (int s = 0; s < HD / 32; s++) {
        Half8 hi, lo;
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const float u = x[8 * s + 2 * k] * up, v = x[8 * s + 2 * k + 1] * up;
            hi.h[k] = half2_of(u, v);
            if (TERMS == 2) lo.h[k] = half2_of(u - (float)hi.h[k][0], v - (float)hi.h[k][1]);
        }
        q[0][s] = hi.v;
        if constexpr (TERMS == 2) q[1][s] = lo.v;
    }
}
// MT sets of 16 rows from product row m0 on (row i, head g of the group: m = i * grps + g); returns what a product has to be multiplied
// by to be a score.
template <int HD, int MT, int TERMS, typename MX>
__device__ __forceinline__ float load_queries(const Kv8Attn &a, const Kv8Seq &sq, int n_rows, int kvh, int grps, int64_t m0, f16x8 (&q)[MT][TERMS][HD / 32],
                                              MX all_max)
{
    const int qi = threadIdx.x & 15, grp = (threadIdx.x & 63) >> 4;
    const bool wide = kv8_wide(a.q, a.q_row, a.q_head, a.dtype);
    float x[MT][HD / 4], mx = 0.f;
#pragma unroll
    for (int mt = 0; mt < MT; mt++) {
        const int64_t m = m0 + 16 * mt + qi;
        const int i = (int)(m / grps), g = (int)(m % grps);
#pragma unroll
        for (int e = 0; e < HD / 4; e++) x[mt][e] = 0.f;
        if (i < n_rows) {
            const int64_t at = (int64_t)(sq.row0 + i) * a.q_row + (int64_t)(kvh * grps + g) * a.q_head;
#pragma unroll
            for (int j = 0; j < HD / 64; j++) load_q16<TERMS>(a, wide, at + 64 * j + 16 * grp, &x[mt][16 * j]);
        }
#pragma unroll
        for (int e = 0; e < HD / 4; e++) mx = fmaxf(mx, fabsf(x[mt][e]));
    }
    const QScale qs = q_scale(all_max(mx));
#pragma unroll
    for (int mt = 0; mt < MT; mt++) query_operands<HD, TERMS>(x[mt], qs.up, q[mt]);
    return qs.down * a.scale;
}
// over the wave
__device__ __forceinline__ float wave_max(float v)
{
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

// One wave's share of a tile's bytes, in flight while the tile before it is consumed.
template <int HD>
struct K8Regs {
    struct __attribute__((aligned(HD / 16))) VRow { // a lane's words of a V row
        uint32_t w[HD / 64];
    };
    uint4 k[2][HD / 64];
    VRow v[8];
    F4 ks[2], vs[2]; // tokens 4 grp .. + 4 and 16 + 4 grp .. + 4
};

// Block: 4 waves over the tiles of one (sequence, cache head, set of MT * 16 rows, split), each with a running softmax of its own.
//   S^T = K Q^T: two operands of 16 tokens each, read from the codes' rows in 16-byte pieces.  The result leaves lane (qi, grp)
//   tokens 4 grp + r of both halves for row qi, which are the eight k-slots of the P^T operand of
//   O^T = V^T P^T: V's rows are read as they lie (lane (m, grp): VB dimensions from VB m on of eight tokens) and transposed by
//   the byte permutes that widen them.
// E, a power of two above half the largest V scale so far, takes the scales' range out of the 16-bit probabilities.
// Bound: memory; per code about 1.2 vector operations to widen it, beside one matrix instruction per 512 codes and 16 rows.
template <int HD, int MT, int TERMS>
__global__ __launch_bounds__(256, MT == 1 ? 3 : 2) void kv8_attn_stream_kernel(Kv8View c, Kv8Rows rw, Kv8Attn a, int n_chunks, int S, int per_want, float *part)
{
    constexpr int NS = HD / 32, VB = HD / 16, VW = HD / 64, ND = VB;
    constexpr int DP = HD < 128 ? HD : 128; // dimensions merged at a time
    __shared__ float sO[4][DP * 17];
    __shared__ float sM[4][16], sL[4][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int qi = lane & 15, grp = lane >> 4;
    const int kvh = blockIdx.x % c.kv_heads, j = blockIdx.x / c.kv_heads % rw.n, chunk0 = blockIdx.x / c.kv_heads / rw.n, split = blockIdx.y;
    const Kv8Seq sq = kv8_seq(c, rw, j);
    const int grps = a.n_heads / c.kv_heads;
    if (sq.b < 0 && c.status && threadIdx.x == 0) atomicOr(c.status, 4);
    const int n_rows = sq.b < 0 ? 0 : sq.n_rows;
    const int64_t all = (int64_t)(rw.path ? rw.rows : n_rows) * grps; // (unused slots of the path receive zeros)
    const int cap = sq.b < 0 ? 0 : c.cap[sq.b];
    const int64_t base = (int64_t)kvh * c.tokens + (sq.b < 0 ? 0 : c.off[sq.b]);
    const int8_t *K = c.k + base * HD, *V = c.v + base * HD;
    const float *KS = c.ks + base, *VS = c.vs + base;
    for (int64_t m0 = (int64_t)chunk0 * MT * 16; m0 < all; m0 += (int64_t)n_chunks * MT * 16) {
        const int i_first = (int)(m0 / grps), i_last = (int)min((int64_t)n_rows - 1, (m0 + MT * 16 - 1) / grps);
        Kv8Tiles tl = {};
        if (i_first < n_rows) tl = kv8_tiles(a, sq.len, i_first, i_last, cap);
        const int per = kv8_per_split(tl.T, S, per_want), t_begin = split * per, t_end = min(tl.T, t_begin + per);
        if (split > 0 && t_begin >= tl.T) continue;
        f16x8 q[MT][TERMS][NS];
        const float qf = load_queries<HD, MT, TERMS>(a, sq, n_rows, kvh, grps, m0, q, wave_max); // (the same for every wave: they hold the same rows)
        float m_run[MT], l_run[MT];
        Kv8Seen seen[MT]; // of the lane's row in each set
        f32x4 o[MT][ND];
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            const int i = (int)((m0 + 16 * mt + qi) / grps);
            seen[mt] = kv8_seen(a, sq.len, i, cap);
            if (i >= n_rows) seen[mt] = Kv8Seen{0, 0, 0};
            m_run[mt] = -INFINITY, l_run[mt] = 0.f;
#pragma unroll
            for (int d = 0; d < ND; d++) o[mt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        float E = KV8_SCALE_MIN;
        const int last_tok = max(0, tl.hi_max - 1);
        const uint32_t k_lane = qi * HD + 16 * grp, v_lane = 4 * grp * HD + VB * qi; // byte offsets of the lane inside a tile
        // One tile's bytes: they are asked for where the tile before it has used the registers up, K and the scales behind the score
        // products, V behind the output products.
        K8Regs<HD> r;
        auto load_k = [&](int t) {
            const int t0 = tl.token0(t);
            if (t0 + K8_TILE <= tl.hi_max) { // (uniform) a whole tile: one address and constant offsets
                const int8_t *kt = K + (int64_t)t0 * HD;
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int p = 0; p < HD / 64; p++) r.k[h][p] = *(const uint4 *)(kt + k_lane + (16 * h * HD + 64 * p));
#pragma unroll
                for (int h = 0; h < 2; h++) r.ks[h] = *(const F4 *)(KS + t0 + 16 * h + 4 * grp), r.vs[h] = *(const F4 *)(VS + t0 + 16 * h + 4 * grp);
            } else { // tokens behind the last one any row sees repeat that one
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int p = 0; p < HD / 64; p++) r.k[h][p] = *(const uint4 *)(K + (int64_t)min(t0 + 16 * h + qi, last_tok) * HD + 64 * p + 16 * grp);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const int tok = min(t0 + 16 * (e / 4) + 4 * grp + e % 4, last_tok);
                    r.ks[e / 4].v[e % 4] = KS[tok], r.vs[e / 4].v[e % 4] = VS[tok];
                }
            }
        };
        auto load_v = [&](int t) {
            const int t0 = tl.token0(t);
            if (t0 + K8_TILE <= tl.hi_max) {
                const int8_t *vt = V + (int64_t)t0 * HD;
#pragma unroll
                for (int e = 0; e < 8; e++) r.v[e] = *(const typename K8Regs<HD>::VRow *)(vt + v_lane + (e < 4 ? e : 12 + e) * HD);
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    r.v[e] = *(const typename K8Regs<HD>::VRow *)(V + (int64_t)min(t0 + 16 * (e / 4) + 4 * grp + e % 4, last_tok) * HD + VB * qi);
            }
        };
        auto consume = [&](int t, int t_next, auto masked) { // t_next < 0: none
            constexpr bool MASKED = decltype(masked)::value;
            const int rel = tl.token0(t) + 4 * grp; // tokens are counted from the lane's first one
            f32x4 s[MT][2];
#pragma unroll
            for (int mt = 0; mt < MT; mt++) s[mt][0] = s[mt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int p = 0; p < HD / 64; p++) {
                    const f16x8 k0 = codes_to_half(r.k[h][p].x, r.k[h][p].y), k1 = codes_to_half(r.k[h][p].z, r.k[h][p].w);
#pragma unroll
                    for (int mt = 0; mt < MT; mt++)
#pragma unroll
                        for (int w = 0; w < TERMS; w++) {
                            s[mt][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[mt][w][2 * p], s[mt][h], 0, 0, 0);
                            s[mt][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[mt][w][2 * p + 1], s[mt][h], 0, 0, 0);
                        }
                }
            float ks[8], vs[8], big = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                ks[e] = r.ks[e / 4].v[e % 4] * qf;
                vs[e] = r.vs[e / 4].v[e % 4];
                if (MASKED) { // scales of tokens that no row sees are not looked at
                    const int tok = 16 * (e / 4) + e % 4;
                    if (!(tok < tl.hi_max - rel && (tok >= tl.lo_min - rel || tok < a.sinks - rel))) vs[e] = 0.f;
                }
                big = fmaxf(big, vs[e]);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (t_next >= 0) load_k(t_next);
            __builtin_amdgcn_sched_barrier(0);
            // the tile's V scales over E
            big = __uint_as_float(min(__float_as_uint(rows4_max(big)), 0x7e000000u) & 0x7f800000u);
            const float E_new = fmaxf(E, big);
            const float inv = __uint_as_float(0x7f000000u + (K8_P_SHIFT << 23) - __float_as_uint(E_new));
            const float shrink = E * __uint_as_float(0x7f000000u - __float_as_uint(E_new));
            E = E_new;
#pragma unroll
            for (int e = 0; e < 8; e++) vs[e] *= inv;
            Half8 ph[MT][TERMS];
#pragma unroll
            for (int mt = 0; mt < MT; mt++) {
                float x[8], mx = -INFINITY;
                bool vis[8];
                const int hi = seen[mt].hi - rel, lo = seen[mt].lo - rel, sk = a.sinks - rel;
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    x[e] = s[mt][e / 4][e % 4] * ks[e];
                    if (MASKED) {
                        const int tok = 16 * (e / 4) + e % 4;
                        vis[e] = tok < hi && (tok >= lo || tok < sk);
                        x[e] = vis[e] ? x[e] : -INFINITY;
                    }
                    mx = fmaxf(mx, x[e]);
                }
                const float m_new = fmaxf(m_run[mt], rows4_max(mx));
                const float ref = m_new == -INFINITY ? 0.f : m_new;
                const float corr = __builtin_amdgcn_exp2f(m_run[mt] - ref), corr_o = corr * shrink;
                m_run[mt] = m_new;
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    float p[2];
#pragma unroll
                    for (int f = 0; f < 2; f++) {
                        p[f] = __builtin_amdgcn_exp2f(x[e + f] - ref);
                        sum += p[f];
                        p[f] *= vs[e + f];
                        if (MASKED) p[f] = vis[e + f] ? p[f] : 0.f;
                    }
                    ph[mt][0].h[e / 2] = half2_of(p[0], p[1]);
                    if constexpr (TERMS == 2)
                        ph[mt][1].h[e / 2] = half2_of(p[0] - (float)ph[mt][0].h[e / 2][0], p[1] - (float)ph[mt][0].h[e / 2][1]);
                }
                l_run[mt] = l_run[mt] * corr + sum;
                if (__any(corr_o != 1.0f)) {
                    asm volatile("" ::: "memory");
#pragma unroll
                    for (int d = 0; d < ND; d++) o[mt][d] *= corr_o;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // V^T fragments, byte by byte of the words
#pragma unroll
            for (int w = 0; w < VW; w++) {
                Half8 f[4];
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const uint32_t a0 = r.v[2 * e].w[w] ^ 0x80808080u, a1 = r.v[2 * e + 1].w[w] ^ 0x80808080u;
                    f[0].h[e] = pair_to_half<0>(a0, a1);
                    f[1].h[e] = pair_to_half<1>(a0, a1);
                    f[2].h[e] = pair_to_half<2>(a0, a1);
                    f[3].h[e] = pair_to_half<3>(a0, a1);
                }
#pragma unroll
                for (int b = 0; b < 4; b++)
#pragma unroll
                    for (int mt = 0; mt < MT; mt++)
#pragma unroll
                        for (int u = 0; u < TERMS; u++)
                            o[mt][4 * w + b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[b].v, ph[mt][u].v, o[mt][4 * w + b], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (t_next >= 0) load_v(t_next);
            __builtin_amdgcn_sched_barrier(0);
        };
        const Kv8Order od = kv8_order(tl, t_begin, t_end);
        if (wave < od.n) {
            int u = wave;
            load_k(od.tile(u));
            load_v(od.tile(u));
            for (; u < od.n_edge; u += 4) consume(od.tile(u), u + 4 < od.n ? od.tile(u + 4) : -1, std::true_type{});
            for (; u < od.n; u += 4) consume(od.tile(u), u + 4 < od.n ? od.tile(u + 4) : -1, std::false_type{});
        }
        // the waves' parts meet: O in true units (E and the shifts undone), weighted by their maxima
        const float unit = E * 0.03125f; // 2^(9 - 14)
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            const float l = rows4_sum(l_run[mt]);
#pragma unroll
            for (int d0 = 0; d0 < HD; d0 += DP) { // (a pass holds the accumulators of VB / (HD / DP) bytes of each lane's dimensions)
                __syncthreads();
                if (grp == 0 && d0 == 0) sM[wave][qi] = m_run[mt], sL[wave][qi] = l;
                constexpr int NB = VB / (HD / DP);
#pragma unroll
                for (int b = 0; b < NB; b++)
#pragma unroll
                    for (int r = 0; r < 4; r++) sO[wave][(NB * (4 * grp + r) + b) * 17 + qi] = o[mt][d0 / DP * NB + b][r] * unit;
                __syncthreads();
                for (int u = threadIdx.x; u < DP * 16; u += 256) {
                    const int dd = u % DP, row = u / DP;
                    const int d = VB * (dd / NB) + d0 / DP * NB + dd % NB;
                    const int64_t m = m0 + 16 * mt + row;
                    if (m >= all) continue;
                    const float M = fmaxf(fmaxf(sM[0][row], sM[1][row]), fmaxf(sM[2][row], sM[3][row])), ref = M == -INFINITY ? 0.f : M;
                    float O = 0.f, L = 0.f;
#pragma unroll
                    for (int w = 0; w < 4; w++) {
                        const float f = __builtin_amdgcn_exp2f(sM[w][row] - ref);
                        O += sO[w][dd * 17 + row] * f;
                        L += sL[w][row] * f;
                    }
                    const int i = (int)(m / grps), h = kvh * grps + (int)(m % grps), r = sq.row0 + i;
                    if (i >= n_rows) kv8_store_out(a, r, h, HD, d, 0.f); // an unused slot of the path
                    else if (tl.T <= per) { // one split: this is the result
                        // (nothing seen: L is 0.  A sum that is not a number stays one.)
                        kv8_store_out(a, r, h, HD, d, L == 0.f ? 0.f : O / L);
                        if (a.lse && d == 0) a.lse[(int64_t)r * a.n_heads + h] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
                    } else {
                        float *p = part + (((int64_t)r * a.n_heads + h) * S + split) * (HD + 4);
                        p[4 + d] = O;
                        if (d == 0) p[0] = M, p[1] = L;
                    }
                }
            }
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- many rows: tiles shared through LDS
// Block: 4 waves of MT * 16 product rows each, one (sequence, cache head), one share of the tiles.  Each 32-token tile of codes is
// widened once per block, into LDS and in the order the operands are read in (fragments of 64 x 16 bytes, so writes and reads are
// linear), two waves doing K and two V; the next tile's codes are in flight meanwhile.  One barrier per tile.
// The softmax's maximum follows lazily: it moves only where a score exceeds it by more than 2^K8_LAZY, so that a score costs one
// fused multiply-add (its scale and the maximum) and one exponential.  E (see above) is known before the first tile: the block
// looks at the V scales of its tiles once, which is 1/64 of their bytes.
// Bound: the vector unit (per score a multiply-add, half a maximum, an exponential, a sum, a product and half a conversion, besides
// the widening) and the matrix unit next to it.
#define K8_LAZY 4.0f
#define K8_P_SHIFT_LAZY 10 // p * (vs / E) * 2^10 < 2^15
template <int HD, int MT, int TERMS>
__global__ __launch_bounds__(256, 3) void kv8_attn_tile_kernel(Kv8View c, Kv8Rows rw, Kv8Attn a, int S, int per_want, float *part)
{
    constexpr int NS = HD / 32, VB = HD / 16, ND = VB, NF = 2 * NS + ND; // fragments of a tile: K's, then V's
    constexpr int ROWS = 4 * MT * 16;
    struct Buf {
        uint4 frag[NF][64];
        float ks[K8_TILE], vs[K8_TILE];
    };
    __shared__ Buf buf[2];
    __shared__ float red[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int qi = lane & 15, grp = lane >> 4;
    const int kvh = blockIdx.x % c.kv_heads, split = blockIdx.y, grps = a.n_heads / c.kv_heads;
    // which sequence and which of its sets of rows: the last sets (they see most) come first
    int j, chunk;
    {
        int b = blockIdx.x / c.kv_heads;
        if (!rw.row_start) {
            const int sets = (int)(((int64_t)rw.rows * grps + ROWS - 1) / ROWS);
            j = b % rw.n, chunk = sets - 1 - b / rw.n;
        } else { // sets of every sequence, counted by the lanes
            int found = -1, left = b;
            for (int j0 = 0; j0 < rw.n && found < 0; j0 += 64) {
                const int jj = j0 + lane;
                const int n = jj < rw.n ? rw.row_start[jj + 1] - rw.row_start[jj] : 0;
                const int sets = n > 0 ? (int)(((int64_t)n * grps + ROWS - 1) / ROWS) : 0;
                int upto = sets; // of the lanes up to this one
                for (int o = 1; o < 64; o <<= 1) {
                    const int v = __shfl_up(upto, o, 64);
                    if (lane >= o) upto += v;
                }
                const uint64_t behind = __ballot(upto > left);
                if (behind) {
                    const int l = __ffsll((unsigned long long)behind) - 1;
                    found = j0 + l;
                    left = __shfl(upto, l, 64) - 1 - left; // (counted from the sequence's end)
                } else left -= __shfl(upto, 63, 64);
            }
            if (found < 0) return;
            j = __builtin_amdgcn_readfirstlane(found), chunk = __builtin_amdgcn_readfirstlane(left);
        }
    }
    const Kv8Seq sq = kv8_seq(c, rw, j);
    if (sq.b < 0 && c.status && threadIdx.x == 0) atomicOr(c.status, 4);
    const int n_rows = sq.b < 0 ? 0 : sq.n_rows;
    const int64_t all = (int64_t)(rw.path ? rw.rows : n_rows) * grps, m_blk = (int64_t)chunk * ROWS, m0 = m_blk + wave * (MT * 16);
    if (m_blk >= all) return;
    const int cap = sq.b < 0 ? 0 : c.cap[sq.b];
    const int64_t base = (int64_t)kvh * c.tokens + (sq.b < 0 ? 0 : c.off[sq.b]);
    const int8_t *K = c.k + base * HD, *V = c.v + base * HD;
    const float *KS = c.ks + base, *VS = c.vs + base;
    const int i_first = (int)(m_blk / grps), i_last = (int)min((int64_t)n_rows - 1, (m_blk + ROWS - 1) / grps);
    Kv8Tiles tl = {};
    if (i_first < n_rows) tl = kv8_tiles(a, sq.len, i_first, i_last, cap);
    const int per = kv8_per_split(tl.T, S, per_want), t_begin = split * per, t_end = min(tl.T, t_begin + per);
    if (split > 0 && t_begin >= tl.T) return;
    // what the wave's rows see
    const int w_first = (int)(m0 / grps), w_last = (int)min((int64_t)n_rows - 1, (m0 + MT * 16 - 1) / grps);
    Kv8Tiles wt = {};
    if (w_first < n_rows) wt = kv8_tiles(a, sq.len, w_first, w_last, cap);
    auto block_max = [&](float v) {
        v = wave_max(v);
        __syncthreads();
        if (lane == 0) red[wave] = v;
        __syncthreads();
        return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    };
    f16x8 q[MT][TERMS][NS];
    const float qf = load_queries<HD, MT, TERMS>(a, sq, n_rows, kvh, grps, m0, q, block_max);
    float m_run[MT], l_run[MT];
    Kv8Seen seen[MT];
    f32x4 o[MT][ND];
#pragma unroll
    for (int mt = 0; mt < MT; mt++) {
        const int i = (int)((m0 + 16 * mt + qi) / grps);
        seen[mt] = kv8_seen(a, sq.len, i, cap);
        if (i >= n_rows) seen[mt] = Kv8Seen{0, 0, 0};
        m_run[mt] = -INFINITY, l_run[mt] = 0.f;
#pragma unroll
        for (int d = 0; d < ND; d++) o[mt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    auto any_sees = [&](int tok) { return tok < tl.hi_max && (tok >= tl.lo_min || tok < a.sinks); };
    float big = 0.f;
    for (int u = t_begin * K8_TILE + threadIdx.x; u < t_end * K8_TILE; u += 256) {
        const int tok = tl.token0(u / K8_TILE) + u % K8_TILE;
        if (any_sees(tok)) big = fmaxf(big, VS[tok]);
    }
    const float E = fmaxf(KV8_SCALE_MIN, __uint_as_float(min(__float_as_uint(block_max(big)), 0x7e000000u) & 0x7f800000u));
    const float inv_E = __uint_as_float(0x7f000000u + (K8_P_SHIFT_LAZY << 23) - __float_as_uint(E));
    const int last_tok = max(0, tl.hi_max - 1);
    // staging: waves 0 and 1 take 16 tokens of K each, waves 2 and 3 half of V's bytes each
    uint32_t st[8]; // K: words of HD / 64 pieces; V: a word of each of eight tokens
    float ss = 0.f;
    // (byte offsets inside a tile)
    const uint32_t stage_at = wave < 2 ? (16 * wave + qi) * HD + 16 * grp : 4 * grp * HD + VB * qi + (HD == 128 ? 4 * (wave - 2) : 0);
    auto fetch = [&](int t) {
        const int t0 = tl.token0(t);
        if (t0 + K8_TILE <= tl.hi_max) {
            const int8_t *tile = (wave < 2 ? K : V) + (int64_t)t0 * HD;
            if (wave < 2) {
#pragma unroll
                for (int p = 0; p < HD / 64; p++) *(uint4 *)&st[4 * p] = *(const uint4 *)(tile + stage_at + 64 * p);
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++) st[e] = *(const uint32_t *)(tile + stage_at + (e < 4 ? e : 12 + e) * HD);
            }
        } else if (wave < 2) { // tokens behind the last one any row sees repeat that one
#pragma unroll
            for (int p = 0; p < HD / 64; p++)
                *(uint4 *)&st[4 * p] = *(const uint4 *)(K + (int64_t)min(t0 + 16 * wave + qi, last_tok) * HD + 64 * p + 16 * grp);
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++)
                st[e] = *(const uint32_t *)(V + (int64_t)min(t0 + 16 * (e / 4) + 4 * grp + e % 4, last_tok) * HD + VB * qi + (HD == 128 ? 4 * (wave - 2) : 0));
        }
        if ((wave & 1) == 0 && lane < K8_TILE) {
            const int tok = t0 + lane;
            ss = (wave ? VS : KS)[min(tok, last_tok)];
            if (wave && !any_sees(tok)) ss = 0.f;
        }
    };
    auto stage = [&](Buf &b) {
        if (wave < 2) {
#pragma unroll
            for (int p = 0; p < HD / 64; p++) {
                *(f16x8 *)&b.frag[wave * NS + 2 * p][lane] = codes_to_half(st[4 * p], st[4 * p + 1]);
                *(f16x8 *)&b.frag[wave * NS + 2 * p + 1][lane] = codes_to_half(st[4 * p + 2], st[4 * p + 3]);
            }
        } else {
            Half8 f[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const uint32_t a0 = st[2 * e] ^ 0x80808080u, a1 = st[2 * e + 1] ^ 0x80808080u;
                if (HD == 128 || wave == 2) f[0].h[e] = pair_to_half<0>(a0, a1), f[1].h[e] = pair_to_half<1>(a0, a1);
                if (HD == 128 || wave == 3) f[2].h[e] = pair_to_half<2>(a0, a1), f[3].h[e] = pair_to_half<3>(a0, a1);
            }
            uint4(*v)[64] = b.frag + 2 * NS + (HD == 128 ? 4 * (wave - 2) : 0);
            if (HD == 128 || wave == 2) *(f16x8 *)&v[0][lane] = f[0].v, *(f16x8 *)&v[1][lane] = f[1].v;
            if (HD == 128 || wave == 3) *(f16x8 *)&v[2][lane] = f[2].v, *(f16x8 *)&v[3][lane] = f[3].v;
        }
        if ((wave & 1) == 0 && lane < K8_TILE) (wave ? b.vs : b.ks)[lane] = ss * (wave ? inv_E : qf);
    };
    auto consume = [&](int t, const Buf &b, auto masked) {
        constexpr bool MASKED = decltype(masked)::value;
        const int t0 = tl.token0(t);
        f32x4 s[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; mt++) s[mt][0] = s[mt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < NS; p++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const f16x8 k = *(const f16x8 *)&b.frag[h * NS + p][lane];
#pragma unroll
                for (int mt = 0; mt < MT; mt++)
#pragma unroll
                    for (int w = 0; w < TERMS; w++) s[mt][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[mt][w][p], s[mt][h], 0, 0, 0);
            }
        __builtin_amdgcn_sched_barrier(0);
        f32x4 ks[2], vs[2];
#pragma unroll
        for (int h = 0; h < 2; h++) ks[h] = *(const f32x4 *)&b.ks[16 * h + 4 * grp], vs[h] = *(const f32x4 *)&b.vs[16 * h + 4 * grp];
        Half8 ph[MT][TERMS];
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            float y[8], mx = -INFINITY;
            bool vis[8];
            const int rel = t0 + 4 * grp, hi = seen[mt].hi - rel, lo = seen[mt].lo - rel, sk = a.sinks - rel;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                y[e] = fmaf(s[mt][e / 4][e % 4], ks[e / 4][e % 4], -m_run[mt]);
                if (MASKED) {
                    const int tok = 16 * (e / 4) + e % 4;
                    vis[e] = tok < hi && (tok >= lo || tok < sk);
                    y[e] = vis[e] ? y[e] : -INFINITY;
                }
                mx = fmaxf(mx, y[e]);
            }
            if (__any(mx > K8_LAZY)) { // (from the start, where m_run is -infinity, too)
                asm volatile("" ::: "memory");
                mx = -INFINITY;
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    y[e] = s[mt][e / 4][e % 4] * ks[e / 4][e % 4];
                    if (MASKED) y[e] = vis[e] ? y[e] : -INFINITY;
                    mx = fmaxf(mx, y[e]);
                }
                const float m_new = fmaxf(m_run[mt], rows4_max(mx)), ref = m_new == -INFINITY ? 0.f : m_new;
                const float corr = __builtin_amdgcn_exp2f(m_run[mt] - ref);
                m_run[mt] = m_new;
                l_run[mt] *= corr;
#pragma unroll
                for (int d = 0; d < ND; d++) o[mt][d] *= corr;
#pragma unroll
                for (int e = 0; e < 8; e++) y[e] -= ref;
            }
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                float p[2];
#pragma unroll
                for (int f = 0; f < 2; f++) {
                    p[f] = __builtin_amdgcn_exp2f(y[e + f]);
                    sum += p[f];
                    p[f] *= vs[e / 4][e % 4 + f];
                    if (MASKED) p[f] = vis[e + f] ? p[f] : 0.f;
                }
                ph[mt][0].h[e / 2] = half2_of(p[0], p[1]);
                if constexpr (TERMS == 2)
                    ph[mt][1].h[e / 2] = half2_of(p[0] - (float)ph[mt][0].h[e / 2][0], p[1] - (float)ph[mt][0].h[e / 2][1]);
            }
            l_run[mt] += sum;
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int d = 0; d < ND; d++) {
            const f16x8 v = *(const f16x8 *)&b.frag[2 * NS + d][lane];
#pragma unroll
            for (int mt = 0; mt < MT; mt++)
#pragma unroll
                for (int w = 0; w < TERMS; w++) o[mt][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, ph[mt][w].v, o[mt][d], 0, 0, 0);
        }
    };
    const Kv8Order od = kv8_order(tl, t_begin, t_end);
    const int n = od.n;
    auto tile_at = [&](int u) { return od.tile(u); };
    if (n > 0) {
        fetch(tile_at(0));
        stage(buf[0]);
        if (n > 1) fetch(tile_at(1));
        auto turn = [&](int u) { // -> this turn's tile, staged
            Buf &now = buf[u & 1], &next = buf[(u + 1) & 1];
            __syncthreads(); // `now` is complete, and nobody reads `next` any more
            if (u + 1 < n) stage(next);
            __builtin_amdgcn_sched_barrier(0);
            if (u + 2 < n) fetch(tile_at(u + 2));
            __builtin_amdgcn_sched_barrier(0);
            return &now;
        };
        int u = 0;
        for (; u < od.n_edge; u++) {
            const Buf *b = turn(u);
            const int t = tile_at(u), t0 = tl.token0(t);
            if (t0 < wt.hi_max && (t0 + K8_TILE > wt.lo_min || t0 < a.sinks)) consume(t, *b, std::true_type{}); // (else the wave's rows see nothing of it)
        }
        for (; u < n; u++) consume(tile_at(u), *turn(u), std::false_type{});
    }
    // lane (qi, grp) holds dimensions VB (4 grp + r) .. + VB of its row in o[..][r]
    const bool wide = kv8_wide(a.out, a.o_row, a.o_head, a.dtype);
    const float unit = E * (K8_P_SHIFT_LAZY == 10 ? 0.5f : 0.f); // 2^(9 - 10)
#pragma unroll
    for (int mt = 0; mt < MT; mt++) {
        const float l = rows4_sum(l_run[mt]);
        const int64_t m = m0 + 16 * mt + qi;
        if (m >= all) continue;
        const int i = (int)(m / grps), h = kvh * grps + (int)(m % grps), r = sq.row0 + i;
        if (i >= n_rows) { // an unused slot of the path
#pragma unroll
            for (int k = 0; k < 4; k++) kv8_store_run<VB>(a, wide, r, h, HD, VB * (4 * grp + k), {});
            continue;
        }
        const bool done = tl.T <= per;
        const float f = done ? (l == 0.f ? 0.f : unit / l) : unit;
        float *p = part + (((int64_t)r * a.n_heads + h) * S + split) * (HD + 4);
#pragma unroll
        for (int k = 0; k < 4; k++) {
            float v[VB];
#pragma unroll
            for (int d = 0; d < VB; d++) v[d] = o[mt][d][k] * f;
            const int d0 = VB * (4 * grp + k);
            if (done) kv8_store_run<VB>(a, wide, r, h, HD, d0, v);
            else {
#pragma unroll
                for (int d = 0; d < VB; d += 4) *(float4 *)(p + 4 + d0 + d) = make_float4(v[d], v[d + 1], v[d + 2], v[d + 3]);
            }
        }
        if (grp == 0) {
            if (!done) p[0] = m_run[mt], p[1] = l;
            else if (a.lse) a.lse[(int64_t)r * a.n_heads + h] = l == 0.f ? -INFINITY : (m_run[mt] + log2f(l)) * 0.69314718055994531f;
        }
    }
}

// Joins the splits of one (row, head).
template <int HD>
__global__ __launch_bounds__(HD) void kv8_attn_join_kernel(Kv8View c, Kv8Rows rw, Kv8Attn a, int set_rows, int S, int per_want, const float *__restrict__ part)
{
    const int r = blockIdx.x, h = blockIdx.y, d = threadIdx.x;
    const int j = kv8_owner(rw, r);
    if (j < 0 || j >= rw.n) return;
    const Kv8Seq sq = kv8_seq(c, rw, j);
    const int i = r - sq.row0, grps = a.n_heads / c.kv_heads;
    if (sq.b < 0 || i >= sq.n_rows) return;
    const int64_t m0 = ((int64_t)i * grps + h % grps) / set_rows * set_rows; // the set of rows that the row went with
    const int i_last = (int)min((int64_t)sq.n_rows - 1, (m0 + set_rows - 1) / grps);
    const int T = kv8_tiles(a, sq.len, (int)(m0 / grps), i_last, c.cap[sq.b]).T, per = kv8_per_split(T, S, per_want), used = (T + per - 1) / per;
    if (used <= 1) return; // the block has written the result
    const float *p = part + ((int64_t)r * a.n_heads + h) * S * (HD + 4);
    float M = -INFINITY;
    for (int s = 0; s < used; s++) M = fmaxf(M, p[s * (HD + 4)]);
    const float ref = M == -INFINITY ? 0.f : M;
    float O = 0.f, L = 0.f;
    for (int s = 0; s < used; s++) {
        const float f = __builtin_amdgcn_exp2f(p[s * (HD + 4)] - ref);
        O += p[s * (HD + 4) + 4 + d] * f;
        L += p[s * (HD + 4) + 1] * f;
    }
    kv8_store_out(a, r, h, HD, d, L == 0.f ? 0.f : O / L);
    if (a.lse && d == 0) a.lse[(int64_t)r * a.n_heads + h] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
}

// ---------------------------------------------------------------- which kernel, how many blocks
#define K8_MIN_TILES 16
#define K8_MAX_SPLITS 64
enum Kv8Kernel { KV8_PLAIN, KV8_STREAM, KV8_TILES };
struct Kv8Plan {
    int kernel, mt, set_rows, splits, per; // 16-row sets of a wave; product rows of a block; splits of a context and tiles of one
    int64_t blocks;                   // per cache head and split
};
static Kv8Plan kv8_plan(const Kv8View &c, const Kv8Rows &rw, const Kv8Attn &a, int64_t ws_bytes)
{
    Kv8Plan p = {KV8_PLAIN, 0, 0, 1, 0, 0};
    if ((g_force_generic & 2) || (c.hd != 64 && c.hd != 128)) return p;
    const int64_t max_rows = a.max_rows > 0 ? std::min(a.max_rows, a.total_rows) : a.total_rows, grps = a.n_heads / c.kv_heads;
    const int64_t R = max_rows * grps; // product rows of a sequence
    int64_t goal; // blocks wanted on the chip
    if (R <= 32) {
        p.kernel = KV8_STREAM, p.mt = R <= 16 ? 1 : 2, p.set_rows = 16 * p.mt;
        p.blocks = rw.n * ((R + p.set_rows - 1) / p.set_rows);
        goal = 2048;
    } else {
        p.kernel = KV8_TILES, p.mt = 2, p.set_rows = 64 * p.mt;
        p.blocks = rw.row_start ? a.total_rows * grps / p.set_rows + rw.n : rw.n * ((R + p.set_rows - 1) / p.set_rows);
        goal = 512;
    }
    const int64_t tokens = a.window ? std::min<int64_t>((int64_t)a.window + a.sinks + max_rows, (int64_t)a.max_len + max_rows) : (int64_t)a.max_len + max_rows;
    const int64_t tiles = (tokens + K8_TILE - 1) / K8_TILE, blocks = p.blocks * c.kv_heads;
    // a split takes K8_MIN_TILES tiles at least and the context K8_MAX_SPLITS splits at most
    p.per = (int)std::max(std::max<int64_t>((tiles * blocks + goal - 1) / goal, (tiles + K8_MAX_SPLITS - 1) / K8_MAX_SPLITS), (int64_t)K8_MIN_TILES);
    p.splits = (int)std::max<int64_t>(1, (tiles + p.per - 1) / p.per);
    const int64_t one = (int64_t)a.total_rows * a.n_heads * (c.hd + 4) * sizeof(float);
    if (ws_bytes >= 0 && p.splits > 1) p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(p.splits, ws_bytes / one));
    return p;
}

int64_t kv8_attn_workspace(const Kv8View &c, const Kv8Rows &rw, const Kv8Attn &a)
{
    const Kv8Plan p = kv8_plan(c, rw, a, -1);
    return p.splits > 1 ? (int64_t)a.total_rows * a.n_heads * (c.hd + 4) * sizeof(float) * p.splits : 0;
}

template <int HD>
static hipError_t mfma_launch(hipStream_t s, const Kv8Plan &p, const Kv8View &c, const Kv8Rows &rw, const Kv8Attn &a, float *part)
{
    if (p.blocks * c.kv_heads > 0x7fffffff / 256) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(p.blocks * c.kv_heads), p.splits);
#define STREAM(MT, T) hipLaunchKernelGGL((kv8_attn_stream_kernel<HD, MT, T>), grid, dim3(256), 0, s, c, rw, a, (int)(p.blocks / rw.n), p.splits, p.per, part)
#define TILES(T) hipLaunchKernelGGL((kv8_attn_tile_kernel<HD, 2, T>), grid, dim3(256), 0, s, c, rw, a, p.splits, p.per, part)
    const bool bf16 = a.dtype == SD_BF16;
    if (p.kernel == KV8_TILES) {
        if (bf16) TILES(1);
        else TILES(2);
    } else if (p.mt == 1) {
        if (bf16) STREAM(1, 1);
        else STREAM(1, 2);
    } else {
        if (bf16) STREAM(2, 1);
        else STREAM(2, 2);
    }
#undef STREAM
#undef TILES
    if (p.splits > 1)
        hipLaunchKernelGGL(kv8_attn_join_kernel<HD>, dim3(a.total_rows, a.n_heads), dim3(HD), 0, s, c, rw, a, p.set_rows, p.splits, p.per, part);
    return hipGetLastError();
}

hipError_t launch_kv8_attn(hipStream_t s, const Kv8View &c, const Kv8Rows &rw, const Kv8Attn &a, void *ws, int64_t ws_bytes)
{
    const Kv8Plan p = kv8_plan(c, rw, a, ws_bytes);
    if (p.kernel != KV8_PLAIN) return c.hd == 64 ? mfma_launch<64>(s, p, c, rw, a, (float *)ws) : mfma_launch<128>(s, p, c, rw, a, (float *)ws);
    hipLaunchKernelGGL(kv8_attn_generic_kernel, dim3(a.total_rows, a.n_heads), dim3(256), 0, s, c, rw, a);
    return hipGetLastError();
}
