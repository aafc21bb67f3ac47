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
    const int end = a.causal ? len + i + 1 : len;
    Kv8Seen s;
    s.hi = max(0, min(end, cap));
    s.lo = a.window ? min(s.hi, max(0, end - a.window)) : 0;
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
    const Kv8Seen seen = kv8_seen(a, s.len, i, kv8_capacity(c, s.b));
    const int n = seen.n_first + (seen.hi - seen.lo);
    const int64_t base = (int64_t)(h / (a.n_heads / c.kv_heads)) * c.tokens + c.off[s.b];
    bool bad = false;
    for (int d = tid; d < hd; d += 256) {
        sq[d] = a.dtype == SD_BF16 ? to_float(((const bf16_t *)a.q)[r * a.q_row + h * a.q_head + d]) : ((const float *)a.q)[r * a.q_row + h * a.q_head + d];
        bad |= !(fabsf(sq[d]) < INFINITY);
    }
    const float scale = __syncthreads_or(bad) ? NAN : a.scale; // (everything of such a row is NaN)
    // (a thread of the second step owns four dimensions, dg, of the tokens tg, tg + n_tg, ...)
    const int n_dg = hd / 4, dg = tid % n_dg, tg = tid / n_dg, n_tg = 256 / n_dg;
    float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int u0 = 0; u0 < n; u0 += KG_CHUNK) {
#pragma clang fp contract(off) // x - m_ref is a difference of rounded scores: 0 for the largest, however large they are
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
            x = dot * c.ks[base + t] * scale;
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

#define K8_TILE 32
#define K8_UNIT_COST 8   // tiles whose time a unit's start and end take
// Few rows: contexts of up to K8_WHOLE tiles are not split (a token in 1024 of 8 heads of 128: 14.5 us in parts and joined, 13.4 whole; 32 times
// that with 32 heads 64.7 and 59.3; but one in 1536 tokens 16.0 and 17.7), parts of longer ones have K8_MIN_TILES at least (one in 2048
// tokens: 16.6 us in parts of 16 tiles, 13.2 in parts of 8).
#define K8_WHOLE 40
#define K8_MIN_TILES 8
#define K8_MIN_SPLIT 16  // many rows: tiles of a split at least
#define K8_MAX_SPLITS 64 // splits of a context at most (of 4096 tiles or more, few rows: twice that)
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
__device__ __forceinline__ uint32_t rows4_most(uint32_t u)
{
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    u = max(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return max(b[0], b[1]);
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
    __device__ __forceinline__ int token0(int t) const { return (t + (t < n_sink ? 0 : w0 - n_sink)) * K8_TILE; }
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
    __device__ __forceinline__ int tile(int u) const
    {
        const int far = u < n_edge ? f1 - n_left : f0 - n_edge;
        return u + (u < n_left ? t_begin : far);
    }
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

// 16 adjacent elements of a query row, as they lie
template <int TERMS>
struct Q16 {
    static constexpr int N = 8 * TERMS;
    uint32_t w[N];
    __device__ __forceinline__ float operator[](int e) const
    {
        if constexpr (TERMS == 1) return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
        else return __uint_as_float(w[e]);
    }
};
template <int TERMS>
__device__ __forceinline__ Q16<TERMS> load_q16(const Kv8Attn &a, bool wide, int64_t at)
{
    Q16<TERMS> r;
    if (wide) {
        const uint4 *p = (const uint4 *)((const char *)a.q + at * (TERMS == 1 ? 2 : 4));
#pragma unroll
        for (int v = 0; v < r.N / 4; v++) {
            const uint4 w = p[v];
            r.w[4 * v] = w.x, r.w[4 * v + 1] = w.y, r.w[4 * v + 2] = w.z, r.w[4 * v + 3] = w.w;
        }
    } else if constexpr (TERMS == 1) {
        const uint16_t *p = (const uint16_t *)a.q + at;
#pragma unroll
        for (int e = 0; e < 8; e++) r.w[e] = p[2 * e] | (uint32_t)p[2 * e + 1] << 16;
    } else {
        const uint32_t *p = (const uint32_t *)a.q + at;
#pragma unroll
        for (int e = 0; e < 16; e++) r.w[e] = p[e];
    }
    return r;
}
// Queries are scaled by a power of two, so that a largest element (of magnitude bits mx) lies in [2^bits, 2^(bits + 1)): 2^(bits - q_exp(mx)).
#define K8_INF 0x7f800000u // bits of a magnitude from here on: infinite, or not a number
__device__ __forceinline__ int q_exp(uint32_t mx) { return min(127, max(-100, (int)(mx >> 23) - 127)); } // (kept where 2^+-(e - bits) are normal numbers)
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
// As halves (bits = 14): one holds every bf16 element down to 2^-31 of the largest exactly, two hold 22 bits of an fp32 one, and what
// smaller elements lose is 2^-39 of the largest.
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
// MT sets of 16 rows from product row m0 on (row i, head g of the group: m = i * grps + g), HD / 4 elements a lane: of dimensions
// 64 j + 16 grp .. + 16 for each j.
template <int HD, int MT, int TERMS>
__device__ __forceinline__ void load_rows(const Kv8Attn &a, const Kv8Seq &sq, int n_rows, int kvh, int grps, int m0, Q16<TERMS> (&raw)[MT][HD / 64])
{
    const int qi = threadIdx.x & 15, grp = (threadIdx.x & 63) >> 4;
    const bool wide = kv8_wide(a.q, a.q_row, a.q_head, a.dtype);
#pragma unroll
    for (int mt = 0; mt < MT; mt++) {
        const int m = m0 + 16 * mt + qi, i = (unsigned)m / (unsigned)grps, g = m - i * grps;
#pragma unroll
        for (int j = 0; j < HD / 64; j++) raw[mt][j] = {};
        if ((unsigned)i < (unsigned)n_rows) {
            const int64_t at = (int64_t)(sq.row0 + i) * a.q_row + (int64_t)(kvh * grps + g) * a.q_head;
#pragma unroll
            for (int j = 0; j < HD / 64; j++) raw[mt][j] = load_q16<TERMS>(a, wide, at + 64 * j + 16 * grp);
        }
    }
}
// ... as numbers, and the bits of the largest magnitude of the lane's row (a NaN's are above infinity's, which are above every number's)
template <int HD, int TERMS>
__device__ __forceinline__ uint32_t row_values(const Q16<TERMS> (&raw)[HD / 64], float (&x)[HD / 4])
{
    uint32_t mx = 0;
#pragma unroll
    for (int e = 0; e < HD / 4; e++) {
        x[e] = raw[e / 16][e % 16];
        mx = max(mx, __float_as_uint(x[e]) & 0x7fffffffu);
    }
    return rows4_most(mx);
}
// maximum over a wave on the vector unit's own paths
__device__ __forceinline__ float wave_max(float v)
{
    v = fmaxf(v, dpp_f<0xB1>(v));
    v = fmaxf(v, dpp_f<0x4E>(v));
    v = fmaxf(v, dpp_f<0x141>(v));
    v = fmaxf(v, dpp_f<0x140>(v));
    return rows4_max(v);
}

// How the tiles of all (sequence, cache head, set of rows) units are dealt out.  Units stand in a row, a sequence's next to each other and as
// long as what any row of the sequence sees and K8_UNIT_COST more (32 x 6 rows over up to 4096 tokens 132.8 us without, 130.6 with); block b
// takes the stretch [b * chunk, (b + 1) * chunk), which may reach over several units and cover parts of the first and the last: every
// block has the same work, whatever the lengths.  With too little work for that (`cross` = false) units are rounded up to whole
// stretches instead, and no block has parts of two.
// Positions in the row are 32-bit: they count 2^grain tiles each, grain > 0 only where units or tiles are very many.
// Tiles of a unit of sequence j and number of its units (each lane for a j of its own); {0, 0}: nothing to do.
struct Kv8Units {
    int T, n;
};
template <int SET>
__device__ __forceinline__ Kv8Units kv8_units(const Kv8View &c, const Kv8Rows &rw, const Kv8Attn &a, int j)
{
    if (j >= rw.n) return Kv8Units{0, 0};
    const int b = rw.seq_ids ? rw.seq_ids[j * rw.group] : j;
    const int n_rows = kv8_last_row(rw, j) - kv8_first_row(rw, j); // (unused slots of the path count: they are written too)
    if (b < 0 || b >= c.n_seq || n_rows < 1) return Kv8Units{0, 0};
    const int T = kv8_tiles(a, kv8_length(rw.len[rw.path ? j * rw.group : b]), 0, n_rows - 1, kv8_capacity(c, b)).T;
    return Kv8Units{max(T, 1), (n_rows * (a.n_heads / c.kv_heads) + SET - 1) / SET * c.kv_heads}; // (rows that see nothing are written: a tile at least)
}
__device__ __forceinline__ int64_t uniform64(int64_t v)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}
__device__ __forceinline__ int wave_total(int v)
{
    v += dpp_i<0xB1>(v), v += dpp_i<0x4E>(v), v += dpp_i<0x141>(v), v += dpp_i<0x140>(v);
    return __builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16) + __builtin_amdgcn_readlane(v, 32) + __builtin_amdgcn_readlane(v, 48);
}
__device__ __forceinline__ int wave_most(int v)
{
    v = max(v, dpp_i<0xB1>(v)), v = max(v, dpp_i<0x4E>(v)), v = max(v, dpp_i<0x141>(v)), v = max(v, dpp_i<0x140>(v));
    return max(max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)), max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}
__device__ __forceinline__ int wave_upto(int v) // sum of the lanes up to this one
{
    v += dpp_i<0x111>(v), v += dpp_i<0x112>(v), v += dpp_i<0x114>(v), v += dpp_i<0x118>(v);
    const int a = __builtin_amdgcn_readlane(v, 15), b = __builtin_amdgcn_readlane(v, 31), c = __builtin_amdgcn_readlane(v, 47), row = (threadIdx.x & 63) >> 4;
    return v + (row > 0 ? a : 0) + (row > 1 ? b : 0) + (row > 2 ? c : 0);
}
// The deal, and the first 64 sequences' share of it in the lanes.
struct Kv8Deal {
    int total, chunk; // positions in the row, and of a stretch
    int grain;
    bool cross;
    Kv8Units mine;    // of sequence `lane`
    int upto;         // where its units end
    __device__ __forceinline__ int length(int T) const
    {
        const int t = grain ? (T + (1 << grain) - 1) >> grain : T;
        return cross ? t + K8_UNIT_COST : (int)(((unsigned)t + chunk - 1) / (unsigned)chunk) * chunk;
    }
};
// S: parts a unit may end up in; goal: blocks that are wanted.  Uniform over the grid.
template <int SET>
__device__ __forceinline__ Kv8Deal kv8_deal(const Kv8View &c, const Kv8Rows &rw, const Kv8Attn &a, int S, int goal)
{
    const int lane = threadIdx.x & 63;
    Kv8Deal d;
    d.mine = kv8_units<SET>(c, rw, a, lane);
    auto over_all = [&](auto f) { // sum of f(units of a sequence) over all
        int v = f(d.mine);
        for (int j = lane + 64; j - lane < rw.n; j += 64) v += f(kv8_units<SET>(c, rw, a, j));
        return wave_total(v);
    };
    int T_max = max(1, d.mine.T);
    for (int j = lane + 64; j - lane < rw.n; j += 64) T_max = max(T_max, kv8_units<SET>(c, rw, a, j).T);
    T_max = wave_most(T_max);
    // at most `units` of them (two for a row and cache head; 2^25: kv8_plan), so that 2^28 positions hold all (a block's next stretch may lie
    // four times as far) and the longest is no longer than 2^18
    const uint64_t units = (uint64_t)(unsigned)a.total_rows * (unsigned)c.kv_heads * 2, most = units * (unsigned)(T_max + K8_UNIT_COST) >> 28 | (unsigned)T_max >> 18;
    d.grain = most ? 64 - __builtin_clzll(most) : 0;
    T_max = (T_max + (1 << d.grain) - 1) >> d.grain;
    d.cross = true;
    const int W = over_all([&](Kv8Units u) { return d.length(u.T) * u.n; });
    d.cross = S > 1 && W > goal * K8_MIN_TILES;
    // (a stretch that starts inside a unit makes one more part of it)
    d.chunk = d.cross ? (int)max((unsigned)(W + goal - 1) / (unsigned)goal, (unsigned)(T_max + K8_UNIT_COST + S - 2) / (unsigned)(S - 1))
              : S > 1 ? max(K8_MIN_TILES, (int)((unsigned)(T_max + S - 1) / (unsigned)S)) : T_max;
    d.upto = wave_upto(d.length(d.mine.T) * d.mine.n);
    d.total = d.cross ? W : over_all([&](Kv8Units u) { return d.length(u.T) * u.n; });
    return d;
}
// The sequence that position `at` < total lies in, its unit's length, where its units start and end.
struct Kv8Found {
    int j, len, start, end;
};
template <int SET>
__device__ __forceinline__ Kv8Found kv8_find(const Kv8View &c, const Kv8Rows &rw, const Kv8Attn &a, const Kv8Deal &d, int at)
{
    Kv8Units u = d.mine;
    int upto = d.upto;
    for (int j0 = 0, before = 0;; j0 += 64) {
        const uint64_t behind = __ballot(upto > at);
        if (behind || j0 + 64 >= rw.n) {
            const int l = __builtin_amdgcn_readfirstlane(behind ? __ffsll((unsigned long long)behind) - 1 : 63);
            const int len = d.length(__builtin_amdgcn_readlane(u.T, l)), end = __builtin_amdgcn_readlane(upto, l);
            return Kv8Found{min(j0 + l, rw.n - 1), len, end - len * __builtin_amdgcn_readlane(u.n, l), end};
        }
        before = __builtin_amdgcn_readlane(upto, 63);
        u = kv8_units<SET>(c, rw, a, j0 + 64 + (threadIdx.x & 63));
        upto = before + wave_upto(d.length(u.T) * u.n);
    }
}

// As integers of 22 bits (bits = 21) in three signed bytes, n = (d[2] * 256 + d[1]) * 256 + d[0]: the products with the codes are exact
// integers, and the codes need no widening.  Lane (qi, grp) takes dimensions 64 j + 16 grp .. + 16 into step j, the order a 16-byte
// piece of the codes has them in.
typedef __attribute__((ext_vector_type(4))) int i32x4;
template <int HD>
__device__ __forceinline__ void query_digits(const float (&x)[HD / 4], float up, i32x4 (&q)[3][HD / 64])
{
#pragma unroll
    for (int j = 0; j < HD / 64; j++)
#pragma unroll
        for (int w = 0; w < 4; w++) {
            uint32_t n[4];
#pragma unroll
            for (int e = 0; e < 4; e++) // 1.5 * 2^23 + x rounds x to an integer and has it in its low bits; the bytes of n + 0x808080 are the digits + 128
                n[e] = __float_as_uint(fmaf(x[16 * j + 4 * w + e], up, 12582912.f)) - (0x4b400000u - 0x00808080u);
            const uint32_t a = __builtin_amdgcn_perm(n[1], n[0], 0x05010400u), b = __builtin_amdgcn_perm(n[3], n[2], 0x05010400u); // bytes 0, 0, 1, 1
            const uint32_t c = __builtin_amdgcn_perm(n[1], n[0], 0x0c0c0602u), d = __builtin_amdgcn_perm(n[3], n[2], 0x0c0c0602u); // bytes 2, 2
            q[0][j][w] = (int)(__builtin_amdgcn_perm(b, a, 0x05040100u) ^ 0x80808080u);
            q[1][j][w] = (int)(__builtin_amdgcn_perm(b, a, 0x07060302u) ^ 0x80808080u);
            q[2][j][w] = (int)(__builtin_amdgcn_perm(d, c, 0x05040100u) ^ 0x80808080u);
        }
}
// Codes are read once per call: with the nontemporal hint (verify, 32 x 6 rows over up to 4096 tokens: 131 us without, 122 with).
template <typename T>
__device__ __forceinline__ T read_once(const int8_t *p)
{
    typedef __attribute__((ext_vector_type(sizeof(T) / 4))) uint32_t words;
    return __builtin_bit_cast(T, __builtin_nontemporal_load((const words *)p));
}

// One wave's share of a tile's bytes, in flight while the tile before it is consumed.
template <int HD>
struct K8Regs {
    struct __attribute__((aligned(HD / 16))) VRow { // a lane's words of a V row
        uint32_t w[HD / 64];
    };
    uint4 k[2][HD / 64];
    VRow v[8];
    float sc; // lanes 0..31: the K scale of the tile's token of that number, lanes 32..63: V scales
};

// Block: 4 waves over its stretch of the tiles of (sequence, cache head, set of MT * 16 rows) units, each with a running softmax of its own.
//   S^T = K Q^T in integers: two operands of 16 tokens each are the codes' rows as they lie, in 16-byte pieces; the queries are three
//   signed bytes.  The result leaves lane (qi, grp)
//   tokens 4 grp + r of both halves for row qi, which are the eight k-slots of the P^T operand of
//   O^T = V^T P^T: V's rows are read as they lie (lane (m, grp): VB dimensions from VB m on of eight tokens) and transposed by
//   the byte permutes that widen them.
// E, a power of two above half the largest V scale so far, takes the scales' range out of the 16-bit probabilities.
// Bound: memory.  A tile of 8192 codes (head width 128) takes a wave some 335 instructions between the edges, 20 of them matrix products of
// 16 rows.  32 x 6 rows over up to 4096 tokens of 32 heads of 128, bf16: 642 MB in 121 us with the join, 5.3 TB/s.
template <int HD, int MT, int TERMS>
__global__ __launch_bounds__(256, 2) void kv8_attn_stream_kernel(Kv8View c, Kv8Rows rw, Kv8Attn a, int S, int goal, float *part)
{
    constexpr int VB = HD / 16, VW = HD / 64, ND = VB, SET = 16 * MT;
    __shared__ __attribute__((aligned(16))) float sO[4][16][HD + 4];
    __shared__ float sM[4][16], sL[4][16];
    __shared__ __attribute__((aligned(16))) float sS[4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int qi = lane & 15, grp = lane >> 4;
    const int grps = a.n_heads / c.kv_heads;
    if (blockIdx.x == 0 && c.status) // sequence ids out of range have no units
        for (int j = threadIdx.x; j < rw.n; j += 256)
            if (rw.seq_ids && (rw.seq_ids[j * rw.group] < 0 || rw.seq_ids[j * rw.group] >= c.n_seq)) atomicOr(c.status, 4);
    const Kv8Deal deal = kv8_deal<SET>(c, rw, a, S, goal);
    Kv8Found f = {0, 1, 0, 0};
    for (int blk = blockIdx.x; blk * deal.chunk < deal.total; blk += gridDim.x)
    for (int at = blk * deal.chunk, end = min(at + deal.chunk, deal.total); at < end;) {
        // the unit that position `at` lies in, and this block's part of it
        if (at >= f.end || at < f.start) f = kv8_find<SET>(c, rw, a, deal, at);
        const int j = f.j, unit = (unsigned)(at - f.start) / (unsigned)f.len;
        const int u0 = f.start + unit * f.len; // the unit's first position
        const int t_begin = (at - u0) << deal.grain, first_blk = (unsigned)u0 / (unsigned)deal.chunk, split = blk - first_blk;
        const bool only = u0 + f.len <= (first_blk + 1) * deal.chunk; // the whole unit is this block's
        const int parts = split ? 0 : (unsigned)(u0 + f.len - 1) / (unsigned)deal.chunk - first_blk + 1; // what the unit ends up in
        const int set = (unsigned)unit / (unsigned)c.kv_heads, kvh = unit - set * c.kv_heads, m0 = set * SET;
        const int n_here = max(1, min(end, u0 + f.len) - at); // (always one: should rows overlap, which row_start must not say, the loop still ends)
        at += n_here;
        const int t_stop = (int)min((int64_t)1 << 30, (int64_t)t_begin + ((int64_t)n_here << deal.grain));
        const Kv8Seq sq = kv8_seq(c, rw, j);
        const int n_rows = sq.n_rows, all = (rw.path ? rw.rows : n_rows) * grps; // (unused slots of the path receive zeros)
        const int cap = kv8_capacity(c, sq.b);
        const int64_t base = uniform64((int64_t)kvh * c.tokens + c.off[sq.b]);
        const int8_t *K = c.k + base * HD, *V = c.v + base * HD;
        const float *KS = c.ks + base, *VS = c.vs + base;
        // (tiles are those of the whole sequence, so that a unit's parts are known without its rows; what the set's rows see bounds them)
        const int i_first = (unsigned)m0 / (unsigned)grps, i_last = min(n_rows - 1, (int)((unsigned)(m0 + SET - 1) / (unsigned)grps));
        Kv8Tiles tl = {};
        if (i_first < n_rows) {
            tl = kv8_tiles(a, sq.len, 0, (rw.path ? rw.rows : n_rows) - 1, cap);
            const Kv8Seen first = kv8_seen(a, sq.len, i_first, cap), last = kv8_seen(a, sq.len, i_last, cap);
            tl.hi_min = first.hi, tl.lo_max = last.lo;
            tl.hi_max = last.hi;
        }
        const int t_end = min(min(tl.T, tl.n_sink + (tl.hi_max + K8_TILE - 1) / K8_TILE - tl.w0), t_stop);
        float m_run[MT], l_run[MT];
        Kv8Seen seen[MT]; // of the lane's row in each set
        f32x4 o[MT][ND];
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            const int i = (unsigned)(m0 + 16 * mt + qi) / (unsigned)grps;
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
        // One row set of 64 dimensions leaves registers for a second tile in flight (16 x 2 rows in a window of 1024 tokens, 16 heads of 64: 14.5
        // us with one, 13.1 with two; with 128 dimensions the 122 us of a verify call become 131).
        constexpr int DEPTH = MT == 1 && HD == 64 ? 2 : 1;
        K8Regs<HD> r0, r1;
        // (edge: a tile that may reach behind the last token.  Those between the edges are loaded without the question, from a uniform base:
        // 4 x 65536 tokens of 8 heads of 128 for 6 x 32 query rows 85 us with the question everywhere, 79 so.)
        auto load_k = [&](K8Regs<HD> &r, int t, auto edge) {
            const int t0 = tl.token0(t);
            if (!decltype(edge)::value || t0 + K8_TILE <= tl.hi_max) { // (uniform) a whole tile: one address and constant offsets
                const int8_t *kt = K + (int64_t)t0 * HD;
                uint32_t lane_at = k_lane;
                asm volatile("" : "+v"(lane_at)); // (kept 32 bits wide next to the loads, whose base is uniform)
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int p = 0; p < HD / 64; p++) r.k[h][p] = read_once<uint4>(kt + lane_at + (16 * h * HD + 64 * p));
            } else { // tokens behind the last one any row sees repeat that one
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int p = 0; p < HD / 64; p++) r.k[h][p] = *(const uint4 *)(K + (int64_t)min(t0 + 16 * h + qi, last_tok) * HD + 64 * p + 16 * grp);
            }
            const int tok = t0 + (lane & 31);
            r.sc = (lane < 32 ? KS : VS)[min(tok, last_tok)];
        };
        auto load_v = [&](K8Regs<HD> &r, int t, auto edge) {
            const int t0 = tl.token0(t);
            if (!decltype(edge)::value || t0 + K8_TILE <= tl.hi_max) {
                const int8_t *vt = V + (int64_t)t0 * HD;
                uint32_t lane_at = v_lane;
                asm volatile("" : "+v"(lane_at));
#pragma unroll
                for (int e = 0; e < 8; e++) r.v[e] = read_once<typename K8Regs<HD>::VRow>(vt + lane_at + (e < 4 ? e : 12 + e) * HD);
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    r.v[e] = *(const typename K8Regs<HD>::VRow *)(V + (int64_t)min(t0 + 16 * (e / 4) + 4 * grp + e % 4, last_tok) * HD + VB * qi);
            }
        };
        const Kv8Order od = kv8_order(tl, t_begin, t_end);
        Q16<TERMS> raw[MT][HD / 64];
        load_rows<HD, MT, TERMS>(a, sq, n_rows, kvh, grps, m0, raw);
        if (wave < od.n) { // the first tile is on its way while the queries are looked at
            load_k(r0, od.tile(wave), std::true_type{});
            load_v(r0, od.tile(wave), std::true_type{});
            if constexpr (DEPTH == 2) {
                load_k(r1, od.tile(min(wave + 4, od.n - 1)), std::true_type{});
                load_v(r1, od.tile(min(wave + 4, od.n - 1)), std::true_type{});
            }
        }
        // Each row has a scale of its own, whatever the rows beside it hold: a score is its product times the token's scale, a.scale / 2^21
        // (both in sS) and 2^e (q2e, folded into the exponential's argument).  Of a row with a NaN or an infinity everything is NaN.
        i32x4 q[MT][3][HD / 64];
        float q2e[MT];
        const float qf = a.scale * pow2(-21);
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            float x[HD / 4];
            const uint32_t mx = row_values<HD, TERMS>(raw[mt], x);
            const int e = q_exp(mx);
            query_digits<HD>(x, pow2(21 - e), q[mt]);
            q2e[mt] = mx >= K8_INF && (seen[mt].hi > seen[mt].lo || seen[mt].n_first) ? NAN : pow2(e);
        }
        // (t_next is asked for whether it is wanted or not: with loads that may be left out, the wait for K would have to be one for V too)
        auto consume = [&](K8Regs<HD> &r, int u, auto masked) {
            constexpr bool MASKED = decltype(masked)::value;
            const int t = od.tile(u), t_next = od.tile(min(u + 4 * DEPTH, od.n - 1));
            const int rel = tl.token0(t) + 4 * grp; // tokens are counted from the lane's first one
            float sc = r.sc;
            if (MASKED) { // V scales of tokens that no row sees are not looked at
                const int tok = tl.token0(t) + (lane & 31);
                if (lane >= 32 && !(tok < tl.hi_max && (tok >= tl.lo_min || tok < a.sinks))) sc = 0.f;
            }
            // the tile's V scales over E, and the scales to the lanes that need them (the LDS takes a wave's accesses in order)
            const float big = __uint_as_float(min(__float_as_uint(wave_max(lane < 32 ? 0.f : sc)), 0x7e000000u) & 0x7f800000u);
            const float E_new = fmaxf(E, big);
            const float inv = __uint_as_float(0x7f000000u + (K8_P_SHIFT << 23) - __float_as_uint(E_new));
            const float shrink = E * __uint_as_float(0x7f000000u - __float_as_uint(E_new));
            E = E_new;
            sS[wave][lane] = sc * (lane < 32 ? qf : inv);
            asm volatile("" ::: "memory");
            f32x4 s[MT][2];
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int mt = 0; mt < MT; mt++) {
                    i32x4 d[3];
#pragma unroll
                    for (int k = 0; k < 3; k++) {
                        d[k] = i32x4{0, 0, 0, 0};
#pragma unroll
                        for (int p = 0; p < HD / 64; p++)
                            d[k] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, r.k[h][p]), q[mt][k][p], d[k], 0, 0, 0);
                    }
#pragma unroll
                    for (int e = 0; e < 4; e++) s[mt][h][e] = fmaf((float)((d[2][e] << 8) + d[1][e]), 256.f, (float)d[0][e]);
                }
            const f32x4 ka = *(const f32x4 *)&sS[wave][4 * grp], kb = *(const f32x4 *)&sS[wave][16 + 4 * grp];
            const f32x4 va = *(const f32x4 *)&sS[wave][32 + 4 * grp], vb = *(const f32x4 *)&sS[wave][48 + 4 * grp];
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            load_k(r, t_next, masked);
            __builtin_amdgcn_sched_barrier(0);
            Half8 ph[MT][TERMS];
#pragma unroll
            for (int mt = 0; mt < MT; mt++) {
                float x[8], mx = -INFINITY;
                bool vis[8];
                const int hi = seen[mt].hi - rel, lo = seen[mt].lo - rel, sk = a.sinks - rel;
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    x[e] = s[mt][e / 4][e % 4] * (e < 4 ? ka[e] : kb[e - 4]);
                    if (MASKED) {
                        const int tok = 16 * (e / 4) + e % 4;
                        vis[e] = tok < hi && (tok >= lo || tok < sk);
                        x[e] = vis[e] ? x[e] : -INFINITY;
                    }
                    mx = fmaxf(mx, x[e]);
                }
                const float m_new = fmaxf(m_run[mt], rows4_max(mx) * q2e[mt]);
                const float ref = m_new == -INFINITY ? 0.f : m_new;
                const float corr = __builtin_amdgcn_exp2f(m_run[mt] - ref), corr_o = corr * shrink;
                m_run[mt] = m_new;
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    float p[2];
#pragma unroll
                    for (int f = 0; f < 2; f++) {
                        p[f] = __builtin_amdgcn_exp2f(fmaf(x[e + f], q2e[mt], -ref));
                        sum += p[f];
                        p[f] *= e < 4 ? va[e + f] : vb[e - 4 + f];
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
            load_v(r, t_next, masked);
            __builtin_amdgcn_sched_barrier(0);
        };
        if (wave < od.n) {
            int u = wave;
            if constexpr (DEPTH == 1) {
                for (; u < od.n_edge; u += 4) consume(r0, u, std::true_type{});
                for (; u < od.n; u += 4) consume(r0, u, std::false_type{});
            } else { // the registers take turns
                auto whole = [&](K8Regs<HD> &x, K8Regs<HD> &y) {
                    for (; u + 4 < od.n; u += 8) {
                        consume(x, u, std::false_type{});
                        consume(y, u + 4, std::false_type{});
                    }
                    if (u < od.n) consume(x, u, std::false_type{});
                };
                for (; u + 4 < od.n_edge; u += 8) {
                    consume(r0, u, std::true_type{});
                    consume(r1, u + 4, std::true_type{});
                }
                if (u < od.n_edge) {
                    consume(r0, u, std::true_type{});
                    u += 4;
                    whole(r1, r0);
                } else whole(r0, r1);
            }
        }
        // the waves' parts meet: O in true units (E and the shifts undone), weighted by their maxima.  Thread (row, c) of the sum holds
        // VB adjacent dimensions of a row.
        const float back = E * pow2(9 - K8_P_SHIFT); // (V's halves are codes * 2^-9)
        const int row = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * VB;
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            const float l = rows4_sum(l_run[mt]);
            __syncthreads(); // what was there has been read
            if (grp == 0) sM[wave][qi] = m_run[mt], sL[wave][qi] = l;
#pragma unroll
            for (int r = 0; r < 4; r++)
#pragma unroll
                for (int b = 0; b < VB; b += 4)
                    *(f32x4 *)&sO[wave][qi][VB * (4 * grp + r) + b] =
                        f32x4{o[mt][b][r], o[mt][b + 1][r], o[mt][b + 2][r], o[mt][b + 3][r]} * back;
            __syncthreads();
            const int m = m0 + 16 * mt + row;
            if ((unsigned)m >= (unsigned)all) continue;
            const float M = fmaxf(fmaxf(sM[0][row], sM[1][row]), fmaxf(sM[2][row], sM[3][row])), ref = M == -INFINITY ? 0.f : M;
            float v[VB], L = 0.f;
#pragma unroll
            for (int d = 0; d < VB; d++) v[d] = 0.f;
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const float g = __builtin_amdgcn_exp2f(sM[w][row] - ref);
                L = fmaf(sL[w][row], g, L);
#pragma unroll
                for (int d = 0; d < VB; d += 4) {
                    const f32x4 x = *(const f32x4 *)&sO[w][row][d0 + d];
#pragma unroll
                    for (int e = 0; e < 4; e++) v[d + e] = fmaf(x[e], g, v[d + e]);
                }
            }
            const int i = (unsigned)m / (unsigned)grps, h = kvh * grps + (m - i * grps), r = sq.row0 + i;
            if (only || i >= n_rows) { // this is the result (of an unused slot of the path: zeros)
                // (nothing seen: L is 0.  A sum that is not a number stays one.)
                const float g = L == 0.f || i >= n_rows ? 0.f : 1.0f / L;
#pragma unroll
                for (int d = 0; d < VB; d++) v[d] = i >= n_rows ? 0.f : v[d] * g;
                kv8_store_run<VB>(a, kv8_wide(a.out, a.o_row, a.o_head, a.dtype), r, h, HD, d0, v);
                if (a.lse && d0 == 0) a.lse[(int64_t)r * a.n_heads + h] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
                if (S > 1 && d0 == 0) part[((int64_t)r * a.n_heads + h) * S * (HD + 4) + 2] = __uint_as_float(1); // (nothing to join)
            } else if ((unsigned)split < (unsigned)S) { // (always, but for such rows)
                float *p = part + (((int64_t)r * a.n_heads + h) * S + split) * (HD + 4);
#pragma unroll
                for (int d = 0; d < VB; d += 4) *(float4 *)(p + 4 + d0 + d) = make_float4(v[d], v[d + 1], v[d + 2], v[d + 3]);
                if (d0 == 0) *(float4 *)p = make_float4(M, L, __uint_as_float(parts), 0.f);
            }
        }
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
// the widening) and the matrix unit next to it.  Pieces of three prompts of up to 4095 rows, 32 heads over 8 of 128, bf16: 257 GFLOP in
// 341 us, 752 TFLOP/s, with three waves a SIMD; 425 us with two.
#define K8_LAZY 4.0f
#define K8_P_SHIFT_LAZY 10 // p * (vs / E) * 2^10 < 2^15
template <int HD, int MT, int TERMS>
__global__ __launch_bounds__(256, MT == 1 ? 4 : 3) void kv8_attn_tile_kernel(Kv8View c, Kv8Rows rw, Kv8Attn a, int S, int per_want, float *part)
{
    constexpr int NS = HD / 32, VB = HD / 16, ND = VB, NF = 2 * NS + ND; // fragments of a tile: K's, then V's
    constexpr int ROWS = 4 * MT * 16;
    struct Buf {
        uint4 frag[NF][64];
        float ks[K8_TILE], vs[K8_TILE];
    };
    __shared__ Buf buf[2];
    __shared__ float red[4], row_factor[4][MT * 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int qi = lane & 15, grp = lane >> 4;
    const int kvh = blockIdx.x % c.kv_heads, split = blockIdx.y, grps = a.n_heads / c.kv_heads;
    // which sequence and which of its sets of rows: the last sets (they see most) come first
    int j, chunk;
    {
        int b = blockIdx.x / c.kv_heads;
        if (!rw.row_start) {
            const int sets = (rw.rows * grps + ROWS - 1) / ROWS;
            j = b % rw.n, chunk = sets - 1 - b / rw.n;
        } else { // sets of every sequence, counted by the lanes
            int found = -1, left = b;
            for (int j0 = 0; j0 < rw.n && found < 0; j0 += 64) {
                const int jj = j0 + lane;
                const int n = jj < rw.n ? kv8_last_row(rw, jj) - kv8_first_row(rw, jj) : 0;
                const int upto = wave_upto(n > 0 ? (n * grps + ROWS - 1) / ROWS : 0);
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
    const int all = (rw.path ? rw.rows : n_rows) * grps, m_blk = chunk * ROWS, m0 = m_blk + wave * (MT * 16);
    if (m_blk >= all) return;
    const int cap = sq.b < 0 ? 0 : kv8_capacity(c, sq.b);
    const int64_t base = uniform64((int64_t)kvh * c.tokens + (sq.b < 0 ? 0 : c.off[sq.b]));
    const int8_t *K = c.k + base * HD, *V = c.v + base * HD;
    const float *KS = c.ks + base, *VS = c.vs + base;
    const int i_first = (unsigned)m_blk / (unsigned)grps, i_last = min(n_rows - 1, (int)((unsigned)(m_blk + ROWS - 1) / (unsigned)grps));
    Kv8Tiles tl = {};
    if (i_first < n_rows) tl = kv8_tiles(a, sq.len, i_first, i_last, cap);
    const int per = kv8_per_split(tl.T, S, per_want), t_begin = split * per, t_end = min(tl.T, t_begin + per);
    if (split > 0 && t_begin >= tl.T) return;
    // what the wave's rows see
    const int w_first = (unsigned)m0 / (unsigned)grps, w_last = min(n_rows - 1, (int)((unsigned)(m0 + MT * 16 - 1) / (unsigned)grps));
    Kv8Tiles wt = {};
    if (w_first < n_rows) wt = kv8_tiles(a, sq.len, w_first, w_last, cap);
    auto block_max = [&](float v) {
        v = wave_max(v);
        __syncthreads();
        if (lane == 0) red[wave] = v;
        __syncthreads();
        return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    };
    float m_run[MT], l_run[MT];
    Kv8Seen seen[MT];
    f32x4 o[MT][ND];
#pragma unroll
    for (int mt = 0; mt < MT; mt++) {
        const int i = (unsigned)(m0 + 16 * mt + qi) / (unsigned)grps;
        seen[mt] = kv8_seen(a, sq.len, i, cap);
        if (i >= n_rows) seen[mt] = Kv8Seen{0, 0, 0};
        m_run[mt] = -INFINITY, l_run[mt] = 0.f;
#pragma unroll
        for (int d = 0; d < ND; d++) o[mt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // One scale for the rows of the block, from the largest number among them: what a row's elements lose is 2^-39 of that, less than 2^-22 of
    // the row's own largest, unless that is 2^17 times smaller.  Such a row has a scale of its own, and so has one with a NaN or an
    // infinity, whose scores are all NaN; only then are products looked up a factor (`uneven`): a multiplication of every score makes 351 us
    // of a prompt 370.
    f16x8 q[MT][TERMS][NS];
    float qf; // what a product has to be multiplied by to be a score
    bool uneven;
    {
        Q16<TERMS> raw[MT][HD / 64];
        float x[MT][HD / 4], most = 0.f;
        uint32_t mx[MT];
        load_rows<HD, MT, TERMS>(a, sq, n_rows, kvh, grps, m0, raw);
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            mx[mt] = row_values<HD, TERMS>(raw[mt], x[mt]);
            most = fmaxf(most, mx[mt] < K8_INF ? __uint_as_float(mx[mt]) : 0.f);
        }
        const int e = q_exp(__float_as_uint(block_max(most)));
        qf = a.scale * pow2(e - 14);
        bool odd = false;
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            const int own = q_exp(mx[mt]);
            const bool small = mx[mt] && own < e - 16, bad = mx[mt] >= K8_INF && (seen[mt].hi > seen[mt].lo || seen[mt].n_first);
            query_operands<HD, TERMS>(x[mt], pow2(14 - (small ? own : e)), q[mt]);
            if (grp == 0) row_factor[wave][16 * mt + qi] = bad ? NAN : small ? ldexpf(1.f, own - e) : 1.f;
            odd |= small || bad;
        }
        uneven = __syncthreads_or(odd);
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
    auto fetch = [&](int t, auto edge) { // (the empty statements keep the compiler from merging the kinds of loads into single words with an address each)
        const int t0 = tl.token0(t);
        const bool whole = !decltype(edge)::value || t0 + K8_TILE <= tl.hi_max; // else: tokens behind the last one any row sees repeat that one
        if (wave < 2) {
            const int8_t *p = K + (int64_t)t0 * HD;
            uint32_t at = whole ? stage_at : min(16 * wave + qi, last_tok - t0) * HD + 16 * grp;
            asm volatile("" : "+v"(at)); // (kept 32 bits wide next to the loads, whose base is uniform)
#pragma unroll
            for (int k = 0; k < HD / 64; k++) {
                const uint4 w = *(const uint4 *)(p + at + 64 * k);
                st[4 * k] = w.x, st[4 * k + 1] = w.y, st[4 * k + 2] = w.z, st[4 * k + 3] = w.w;
            }
            asm volatile("; keys" ::: "memory");
        } else if (whole) {
            const int8_t *p = V + (int64_t)t0 * HD;
            uint32_t at = stage_at;
            asm volatile("" : "+v"(at));
#pragma unroll
            for (int e = 0; e < 8; e++) st[e] = *(const uint32_t *)(p + at + (e < 4 ? e : 12 + e) * HD);
            asm volatile("; values" ::: "memory");
        } else {
            const int8_t *p = V + (int64_t)t0 * HD + VB * qi + (HD == 128 ? 4 * (wave - 2) : 0);
#pragma unroll
            for (int e = 0; e < 8; e++) st[e] = *(const uint32_t *)(p + min(16 * (e / 4) + 4 * grp + e % 4, last_tok - t0) * HD);
            asm volatile("; last values" ::: "memory");
        }
        if ((wave & 1) == 0) {
            const int tok = t0 + (lane & 31);
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
            asm volatile("; keys" ::: "memory");
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
            asm volatile("; values" ::: "memory");
        }
        if ((wave & 1) == 0) (wave ? b.vs : b.ks)[lane & 31] = ss * (wave ? inv_E : qf); // (two lanes write the same)
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
        if (uneven) {
            asm volatile("" ::: "memory");
#pragma unroll
            for (int mt = 0; mt < MT; mt++) {
                const float f = row_factor[wave][16 * mt + qi];
                s[mt][0] *= f, s[mt][1] *= f;
            }
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
#pragma clang fp contract(off) // the maximum is one of the rounded scores: what they are off by must not be left over from their difference
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
        fetch(tile_at(0), std::true_type{});
        stage(buf[0]);
        if (n > 1) fetch(tile_at(1), std::true_type{});
        auto turn = [&](int u, auto edge) { // -> this turn's tile, staged
            Buf &now = buf[u & 1], &next = buf[(u + 1) & 1];
            __syncthreads(); // `now` is complete, and nobody reads `next` any more
            if (u + 1 < n) stage(next);
            __builtin_amdgcn_sched_barrier(0);
            if (u + 2 < n) fetch(tile_at(u + 2), edge);
            __builtin_amdgcn_sched_barrier(0);
            return &now;
        };
        int u = 0;
        for (; u < od.n_edge; u++) {
            const Buf *b = turn(u, std::true_type{});
            const int t = tile_at(u), t0 = tl.token0(t);
            if (t0 < wt.hi_max && (t0 + K8_TILE > wt.lo_min || t0 < a.sinks)) consume(t, *b, std::true_type{}); // (else the wave's rows see nothing of it)
        }
        for (; u < n; u++) consume(tile_at(u), *turn(u, std::false_type{}), std::false_type{});
    }
    // lane (qi, grp) holds dimensions VB (4 grp + r) .. + VB of its row in o[..][r]
    const bool wide = kv8_wide(a.out, a.o_row, a.o_head, a.dtype);
    const float unit = E * pow2(9 - K8_P_SHIFT_LAZY); // (V's halves are codes * 2^-9)
#pragma unroll
    for (int mt = 0; mt < MT; mt++) {
        const float l = rows4_sum(l_run[mt]);
        const int m = m0 + 16 * mt + qi;
        if (m >= all) continue;
        const int i = (unsigned)m / (unsigned)grps, h = kvh * grps + (m - i * grps), r = sq.row0 + i;
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

// ---------------------------------------------------------------- parts of a context meet
// HD / 4 threads per product row; parts lie one after the other, { maximum, sum, number of parts (in the first one), -, HD outputs } each.
template <int HD>
__device__ __forceinline__ void kv8_join_row(const Kv8Attn &a, int r, int h, int used, int S, const float *part)
{
    const int dg = threadIdx.x % (HD / 4);
    const float *p = part + ((int64_t)r * a.n_heads + h) * S * (HD + 4);
    float M = -INFINITY, L = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int s = 0; s < used; s++) M = fmaxf(M, p[s * (HD + 4)]);
    const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll 8
    for (int s = 0; s < used; s++) {
        const float2 ml = *(const float2 *)(p + s * (HD + 4));
        const float4 w = *(const float4 *)(p + s * (HD + 4) + 4 + 4 * dg);
        const float f = __builtin_amdgcn_exp2f(ml.x - ref);
        L = fmaf(ml.y, f, L);
        o.x = fmaf(w.x, f, o.x), o.y = fmaf(w.y, f, o.y), o.z = fmaf(w.z, f, o.z), o.w = fmaf(w.w, f, o.w);
    }
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    const float v[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
    kv8_store_run<4>(a, kv8_wide(a.out, a.o_row, a.o_head, a.dtype), r, h, HD, 4 * dg, v);
    if (a.lse && dg == 0) a.lse[(int64_t)r * a.n_heads + h] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
}

// Of kv8_attn_stream_kernel<HD, ..>: a block takes 1024 / HD product rows of one (sequence, cache head) at a time.
template <int HD>
__global__ __launch_bounds__(256) void kv8_attn_join_kernel(Kv8View c, Kv8Rows rw, Kv8Attn a, int n_groups, int S, const float *__restrict__ part)
{
    constexpr int NG = 1024 / HD;
    const int kvh = blockIdx.x % c.kv_heads, j = blockIdx.x / c.kv_heads % rw.n, g0 = blockIdx.x / c.kv_heads / rw.n;
    const Kv8Seq sq = kv8_seq(c, rw, j);
    if (sq.b < 0) return;
    const int grps = a.n_heads / c.kv_heads;
    for (int m = g0 * NG + threadIdx.x / (HD / 4); m < sq.n_rows * grps; m += n_groups * NG) {
        const int i = (unsigned)m / (unsigned)grps, r = sq.row0 + i, h = kvh * grps + (m - i * grps);
        const int used = min((int)__float_as_uint(part[((int64_t)r * a.n_heads + h) * S * (HD + 4) + 2]), S);
        if (used > 1) kv8_join_row<HD>(a, r, h, used, S, part); // (else the result is there)
    }
}

// Of kv8_attn_tile_kernel<HD, SET / 64, ..>: 1024 / HD (row, head) pairs per block.
template <int HD, int SET>
__global__ __launch_bounds__(256) void kv8_attn_join_tiles_kernel(Kv8View c, Kv8Rows rw, Kv8Attn a, int S, int per_want, const float *__restrict__ part)
{
    constexpr int NG = 1024 / HD;
    const int r = blockIdx.x, h = blockIdx.y * NG + threadIdx.x / (HD / 4);
    const int j = kv8_owner(rw, r);
    if (j < 0 || j >= rw.n) return;
    const Kv8Seq sq = kv8_seq(c, rw, j);
    const int i = r - sq.row0, grps = a.n_heads / c.kv_heads;
    if (sq.b < 0 || i >= sq.n_rows || h >= a.n_heads) return;
    const int set0 = (i * grps + h % grps) / SET * SET; // the set of rows that the row went with
    const int T = kv8_tiles(a, sq.len, set0 / grps, min(sq.n_rows - 1, (set0 + SET - 1) / grps), kv8_capacity(c, sq.b)).T;
    const int per = kv8_per_split(T, S, per_want), used = (T + per - 1) / per;
    if (used > 1) kv8_join_row<HD>(a, r, h, used, S, part);
}

// ---------------------------------------------------------------- which kernel, how many blocks
enum Kv8Kernel { KV8_PLAIN, KV8_STREAM, KV8_TILES };
struct Kv8Plan {
    int kernel, mt, splits; // 16-row sets of a wave; parts that a context may be in
    int goal, per;          // KV8_STREAM: blocks wanted; KV8_TILES: tiles of a split
    int64_t blocks, max_m;  // launched (KV8_TILES: per split); product rows of a sequence, as far as is known
};
static Kv8Plan kv8_plan(const Kv8View &c, const Kv8Rows &rw, const Kv8Attn &a, int64_t ws_bytes)
{
    Kv8Plan p = {KV8_PLAIN, 0, 1, 0, 0, 0, 0};
    if ((g_force_generic & 2) || (c.hd != 64 && c.hd != 128)) return p;
    const int64_t max_rows = a.max_rows > 0 ? std::min(a.max_rows, a.total_rows) : a.total_rows, grps = a.n_heads / c.kv_heads;
    const int64_t R = max_rows * grps; // product rows of a sequence
    const int64_t tokens = a.window ? std::min<int64_t>((int64_t)a.window + a.sinks + max_rows, (int64_t)a.max_len + max_rows) : (int64_t)a.max_len + max_rows;
    const int64_t tiles = (tokens + K8_TILE - 1) / K8_TILE;
    const int64_t one = (int64_t)a.total_rows * a.n_heads * (c.hd + 4) * sizeof(float); // workspace of a split
    // Up to 64 product rows blocks stream the cache past 16 or 32 of them, more are worth widening tiles once for all rows of a block.  Streaming
    // and tiles, 16 sequences of 4096 tokens, 8 heads of 128, bf16 (fp32): 32 rows 44 and 60 us (47, 55), 64 rows 54 and 64 (57, 59), 96 rows
    // 102 and 70 (107, 95); one such sequence: 32 rows 17 and 29 (18, 26), 64 rows 21 and 30 (23, 28), 128 rows 28 and 32 (30, 29).
    // (2^24: the units fit the deal.)
    if (R <= 64 && (int64_t)a.total_rows * c.kv_heads <= 1 << 24) {
        p.kernel = KV8_STREAM, p.mt = R <= 16 ? 1 : 2, p.max_m = R;
        const int64_t units = (int64_t)rw.n * c.kv_heads * ((R + 16 * p.mt - 1) / (16 * p.mt));
        // Two blocks for each of the 256 compute units (32 x 6 rows over up to 4096 tokens of 32 heads of 128: 135 us with one a unit, 122 with
        // two, 130 with three, 142 with six; 64 x 50 rows over up to 4000 of 16 of 64: 233 with one, 174 with two); a context in about as
        // many parts as there are blocks for it (twice that, and one more at either end, where lengths differ)
        p.goal = 512;
        // (but for few units of long contexts: one in a million tokens and 2 heads of 128 141 us with 64 parts, 96 with 128; in 32768 tokens and 4
        // heads 25 and 29, the join being longer)
        const int64_t most = tiles >= 4096 ? 2 * K8_MAX_SPLITS : K8_MAX_SPLITS;
        p.splits = tiles <= K8_WHOLE ? 1 : (int)std::min<int64_t>(most, 2 + 2 * ((p.goal + units - 1) / units));
        if (ws_bytes >= 0) p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(p.splits, ws_bytes / one));
        p.blocks = p.splits > 1 ? p.goal + std::min<int64_t>(units, 2 * p.goal) : units; // (with more units than that kv8_deal makes at most `goal` stretches)
    } else {
        // (two 16-row sets a wave share an operand read from LDS; two terms of everything leave registers for one: 4096 fp32 rows of 32 heads over
        // 8 of 128 450 us with two, 278 with one)
        p.kernel = KV8_TILES, p.mt = a.dtype == SD_BF16 ? 2 : 1;
        const int64_t set = 64 * p.mt, goal = 512;
        p.blocks = (rw.row_start ? a.total_rows * grps / set + rw.n : rw.n * ((R + set - 1) / set)) * c.kv_heads;
        // a split takes K8_MIN_SPLIT tiles at least and the context K8_MAX_SPLITS splits at most
        p.per = (int)std::max(std::min(tiles, std::max((tiles * p.blocks + goal - 1) / goal, (tiles + K8_MAX_SPLITS - 1) / K8_MAX_SPLITS)), (int64_t)K8_MIN_SPLIT);
        p.splits = (int)std::max<int64_t>(1, (tiles + p.per - 1) / p.per);
        if (ws_bytes >= 0) p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(p.splits, ws_bytes / one));
    }
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
    if (p.blocks > 0x7fffffff / 256) return hipErrorInvalidValue;
    const bool bf16 = a.dtype == SD_BF16;
    constexpr int NG = 1024 / HD; // rows that a block of a join has in hand
#define STREAM(MT, T)                                                                                                                            \
    do {                                                                                                                                         \
        hipLaunchKernelGGL((kv8_attn_stream_kernel<HD, MT, T>), dim3((unsigned)p.blocks), dim3(256), 0, s, c, rw, a, p.splits, p.goal, part);      \
        if (p.splits > 1) {                                                                                                                      \
            const int groups = (int)((p.max_m + NG - 1) / NG);                                                                                   \
            hipLaunchKernelGGL(kv8_attn_join_kernel<HD>, dim3((unsigned)((int64_t)rw.n * c.kv_heads * groups)), dim3(256), 0, s, c, rw, a, groups,  \
                               p.splits, part);                                                                                  \
        }                                                                                                                                        \
    } while (0)
#define TILES(MT, T)                                                                                                                             \
    do {                                                                                                                                         \
        hipLaunchKernelGGL((kv8_attn_tile_kernel<HD, MT, T>), dim3((unsigned)p.blocks, p.splits), dim3(256), 0, s, c, rw, a, p.splits, p.per, part); \
        if (p.splits > 1)                                                                                                                        \
            hipLaunchKernelGGL((kv8_attn_join_tiles_kernel<HD, 64 * MT>), dim3(a.total_rows, (a.n_heads + NG - 1) / NG), dim3(256), 0, s, c, rw, a, \
                               p.splits, p.per, part);                                                                                           \
    } while (0)
    if (p.kernel == KV8_TILES) {
        if (bf16) TILES(2, 1);
        else TILES(1, 2);
    } else if (p.mt == 1) {
        if (bf16) STREAM(1, 1);
        else STREAM(1, 2);
    } else {
        if (bf16) STREAM(2, 1);
        else STREAM(2, 2);
    }
#undef STREAM
#undef TILES
    return hipGetLastError();
}

hipError_t launch_kv8_attn(hipStream_t s, const Kv8View &c, const Kv8Rows &rw, const Kv8Attn &a, void *ws, int64_t ws_bytes)
{
    const Kv8Plan p = kv8_plan(c, rw, a, ws_bytes);
    if (p.kernel != KV8_PLAIN) return c.hd == 64 ? mfma_launch<64>(s, p, c, rw, a, (float *)ws) : mfma_launch<128>(s, p, c, rw, a, (float *)ws);
    hipLaunchKernelGGL(kv8_attn_generic_kernel, dim3(a.total_rows, a.n_heads), dim3(256), 0, s, c, rw, a);
    return hipGetLastError();
}
