// An 8-bit cache of keys and values: quantising rows as they are written, reading them back, and the calls of the C ABI.
//
// A vector is one row of one head, K or V: scale = max|x| * (1 / 127), at least 2^-60, code = nearest integer to x / scale.
// Bound of both kernels: memory.  D / 8 lanes hold a vector, 8 elements each: a 16-byte load (two for fp32), a maximum over the
// lanes, an 8-byte store.  8191 fp32 rows of 32 heads of 128 in and back: 65 and 59 us, 5.6 TB/s over both.
#include <cmath>

#include <algorithm>

#include "kv8.h"

// The 8 elements that lane l of a vector holds: bf16 the adjacent ones from 8 l on; fp32 four from 4 l on and four from hd / 2 + 4 l on, so
// that each access of the lanes together is one piece (8191 rows of 32 heads read back as fp32: 88 us with 8 adjacent, 68 so).
// NT: with the nontemporal hint, for what is read or written once and is much (8191 fp32 rows of 32 heads into the cache: 99 us without,
// 80 with the loads, 64 with loads and stores; back out of it 70, 70, 65).
template <bool NT, typename V>
__device__ __forceinline__ V load_v(const void *p)
{
    typedef __attribute__((ext_vector_type(sizeof(V) / 4))) uint32_t words;
    return __builtin_bit_cast(V, ld_stream<NT>((const words *)p));
}
template <typename T, bool WIDE, bool NT>
__device__ __forceinline__ void load8(const T *p, int l, int hd, float x[8])
{
    const int d0 = sizeof(T) == 2 ? 8 * l : 4 * l, d1 = sizeof(T) == 2 ? d0 + 4 : hd / 2 + d0;
    if constexpr (WIDE && sizeof(T) == 2) {
        const uint4 w = load_v<NT, uint4>(p + d0);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; e++) x[2 * e] = __uint_as_float(u[e] << 16), x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    } else if constexpr (WIDE) {
        const float4 a = load_v<NT, float4>(p + d0), b = load_v<NT, float4>(p + d1);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++) x[e] = to_float(p[d0 + e]), x[4 + e] = to_float(p[d1 + e]);
    }
}

template <bool NT, typename V>
__device__ __forceinline__ void store_v(void *p, V v)
{
    typedef __attribute__((ext_vector_type(sizeof(V) / 4))) uint32_t words;
    if constexpr (NT) __builtin_nontemporal_store(__builtin_bit_cast(words, v), (words *)p);
    else *(V *)p = v;
}
template <typename T, bool WIDE, bool NT>
__device__ __forceinline__ void store8(T *p, int l, int hd, const float x[8])
{
    const int d0 = sizeof(T) == 2 ? 8 * l : 4 * l, d1 = sizeof(T) == 2 ? d0 + 4 : hd / 2 + d0;
    if constexpr (WIDE && sizeof(T) == 2) {
        store_v<NT>(p + d0, make_uint4(bf16x2_bits_rne(x[0], x[1]), bf16x2_bits_rne(x[2], x[3]), bf16x2_bits_rne(x[4], x[5]), bf16x2_bits_rne(x[6], x[7])));
    } else if constexpr (WIDE) {
        store_v<NT>(p + d0, make_float4(x[0], x[1], x[2], x[3]));
        store_v<NT>(p + d1, make_float4(x[4], x[5], x[6], x[7]));
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++) p[d0 + e] = from_float<T>(x[e]), p[d1 + e] = from_float<T>(x[4 + e]);
    }
}
// ... and their codes
template <typename T, bool NT>
__device__ __forceinline__ uint2 load_codes(const int8_t *p, int l, int hd)
{
    if constexpr (sizeof(T) == 2) return load_v<NT, uint2>(p + 8 * l);
    else return make_uint2(ld_stream<NT>((const uint32_t *)(p + 4 * l)), ld_stream<NT>((const uint32_t *)(p + hd / 2 + 4 * l)));
}
template <typename T>
__device__ __forceinline__ void store_codes(int8_t *p, int l, int hd, uint2 u)
{
    if constexpr (sizeof(T) == 2) *(uint2 *)(p + 8 * l) = u;
    else *(uint32_t *)(p + 4 * l) = u.x, *(uint32_t *)(p + hd / 2 + 4 * l) = u.y;
}

// Largest magnitude of 8 elements as bits (a NaN's are above infinity's, which are above every finite value's) ...
__device__ __forceinline__ uint32_t amax_bits8(const float x[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) m = max(m, __float_as_uint(x[e]) & 0x7fffffffu);
    return m;
}
// ... over the 2^bits adjacent lanes of a vector, left in each of them (the exchanges stay inside a row of 16 lanes but the last) ...
__device__ __forceinline__ uint32_t amax_lanes(uint32_t m, int bits)
{
    m = max(m, (uint32_t)dpp_i<0xB1>((int)m));
    if (bits > 1) m = max(m, (uint32_t)dpp_i<0x4E>((int)m));
    if (bits > 2) m = max(m, (uint32_t)dpp_i<0x141>((int)m));
    if (bits > 3) m = max(m, (uint32_t)dpp_i<0x140>((int)m));
    if (bits > 4) {
        const auto s = __builtin_amdgcn_permlane16_swap(m, m, false, false);
        m = max(s[0], s[1]);
    }
    return m;
}
// ... and the scale it gives: NaN where the vector holds a NaN or an infinity.
__device__ __forceinline__ float kv8_scale(uint32_t amax)
{
    return amax >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : fmaxf(__uint_as_float(amax) * (1.0f / 127.0f), KV8_SCALE_MIN);
}

// The integer nearest to x / s, ties to even.  x * (1 / s) is off by a few parts in 2^24, so its rounding can end on the wrong
// side of a half; e = x - q s is exact (a multiple of the coarser of the two last places, and no larger than s), so comparing it
// with s / 2 settles the case.
__device__ __forceinline__ uint32_t quantise(float x, float s, float inv)
{
    const float q = rintf(x * inv), e = fmaf(-q, s, x), half = 0.5f * s;
    const int c = (int)q;
    const bool over = fabsf(e) > half || (fabsf(e) == half && (c & 1));
    return (uint32_t)(over ? c + (e > 0.f ? 1 : -1) : c) & 255u;
}
// Eight of them.  1.5 * 2^23 + x / s, rounded once, has the integer in its low byte; only where some |e| reaches s / 2 is there
// anything to settle (30 vector operations an element done singly, 7 so).
__device__ __forceinline__ uint2 quantise8(const float x[8], float s, float inv)
{
    uint32_t t[8];
    float e[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float f = fmaf(x[i], inv, 12582912.f);
        t[i] = __float_as_uint(f);
        e[i] = fmaf(12582912.f - f, s, x[i]);
    }
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) m = fmaxf(m, fabsf(e[i]));
    if (__any(m >= 0.5f * s)) {
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < 8; i++) t[i] = quantise(x[i], s, inv);
    }
    const uint32_t a = __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0400u), b = __builtin_amdgcn_perm(t[3], t[2], 0x04000c0cu);
    const uint32_t c = __builtin_amdgcn_perm(t[5], t[4], 0x0c0c0400u), d = __builtin_amdgcn_perm(t[7], t[6], 0x04000c0cu);
    return make_uint2(a | b, c | d);
}
// codes of four bytes, as values
__device__ __forceinline__ void dequantise4(uint32_t u, float s, float x[4])
{
#pragma unroll
    for (int e = 0; e < 4; e++) x[e] = (float)((int32_t)(u << (24 - 8 * e)) >> 24) * s;
}

// Place of row r: its cache row in every head, or -1 (none: not a row of the call, or outside its sequence).  Each thread for a row of its
// own.
__device__ __forceinline__ int64_t row_place(const Kv8View &c, const Kv8Rows &rw, int r, bool flag)
{
    int j, first;
    if (rw.row_start) { // the last sequence whose first row is not behind r
        int lo = 0, hi = rw.n;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (rw.row_start[mid] <= r) lo = mid;
            else hi = mid - 1;
        }
        j = lo, first = rw.row_start[j];
        if (j == rw.n || first > r) return -1;
    } else j = (unsigned)r / (unsigned)rw.rows, first = j * rw.rows;
    const int b = rw.seq_ids ? rw.seq_ids[j] : j;
    if (b < 0 || b >= c.n_seq) {
        if (flag && c.status) atomicOr(c.status, 4);
        return -1;
    }
    const int t = kv8_length(rw.len[b]) + (r - first);
    if (t < 0 || t >= kv8_capacity(c, b)) {
        if (flag && c.status) atomicOr(c.status, 1);
        return -1;
    }
    return c.off[b] + t;
}

// Both kernels: a block serves 2^row_bits adjacent rows.  Its first threads find the rows' places;
// pieces of 8 elements are then dealt out with a vector's lanes innermost, then the rows, then the vectors (K and V of each head), so
// that the codes of adjacent tokens are touched together, and four at a time per thread, so that their loads are in flight together.
#define KV8_MAX_ROWS 32 // of a block
struct Kv8Piece {
    int l, row, w; // lane of the vector, row of the block, vector (2 * head + (0: K, 1: V))
};
__device__ __forceinline__ Kv8Piece kv8_piece(int u, int lane_bits, int row_bits)
{
    return Kv8Piece{u & ((1 << lane_bits) - 1), (u >> lane_bits) & ((1 << row_bits) - 1), u >> (lane_bits + row_bits)};
}

template <typename T, bool WIDE, bool NT>
__global__ __launch_bounds__(256) void kv8_append_kernel(Kv8View c, Kv8Rows rw, int n_rows, int lane_bits, int row_bits, const T *__restrict__ k, int64_t k_row,
                                                         int64_t k_head, const T *__restrict__ v, int64_t v_row, int64_t v_head)
{
    __shared__ int64_t s_at[KV8_MAX_ROWS];
    const int r0 = blockIdx.x << row_bits;
    if (threadIdx.x < 1u << row_bits) s_at[threadIdx.x] = r0 + (int)threadIdx.x < n_rows ? row_place(c, rw, r0 + threadIdx.x, blockIdx.y == 0) : -1;
    __syncthreads();
    const int n = 2 * c.kv_heads << (lane_bits + row_bits);
    for (int u0 = blockIdx.y * 1024; u0 < n; u0 += gridDim.y * 1024) { // (the same count for every lane: shuffles)
        float x[4][8];
#pragma unroll
        for (int q = 0; q < 4; q++) {
#pragma unroll
            for (int e = 0; e < 8; e++) x[q][e] = 0.f;
            const int u = u0 + 256 * q + threadIdx.x;
            const Kv8Piece p = kv8_piece(u, lane_bits, row_bits);
            if (u >= n || p.l * 8 >= c.hd || s_at[p.row] < 0) continue;
            const int64_t r = r0 + p.row;
            const int h = p.w >> 1;
            load8<T, WIDE, NT>(p.w & 1 ? v + r * v_row + h * v_head : k + r * k_row + h * k_head, p.l, c.hd, x[q]);
        }
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const int u = u0 + 256 * q + threadIdx.x;
            const Kv8Piece p = kv8_piece(u, lane_bits, row_bits);
            const float s = kv8_scale(amax_lanes(amax_bits8(x[q]), lane_bits)), inv = 1.0f / s;
            if (u >= n || p.l * 8 >= c.hd || s_at[p.row] < 0) continue;
            const int64_t row = (int64_t)(p.w >> 1) * c.tokens + s_at[p.row];
            const uint2 codes = s == s ? quantise8(x[q], s, inv) : make_uint2(0, 0);
            store_codes<T>((p.w & 1 ? c.v : c.k) + row * c.hd, p.l, c.hd, codes);
            if (p.l == 0) (p.w & 1 ? c.vs : c.ks)[row] = s;
        }
    }
}

template <typename T, bool WIDE, bool NT>
__global__ __launch_bounds__(256) void kv8_read_kernel(Kv8View c, Kv8Rows rw, int n_rows, int lane_bits, int row_bits, T *__restrict__ k, int64_t k_row,
                                                       int64_t k_head, T *__restrict__ v, int64_t v_row, int64_t v_head)
{
    __shared__ int64_t s_at[KV8_MAX_ROWS];
    const int r0 = blockIdx.x << row_bits;
    if (threadIdx.x < 1u << row_bits) s_at[threadIdx.x] = r0 + (int)threadIdx.x < n_rows ? row_place(c, rw, r0 + threadIdx.x, blockIdx.y == 0) : -1;
    __syncthreads();
    const int n = 2 * c.kv_heads << (lane_bits + row_bits);
    for (int u0 = blockIdx.y * 1024; u0 < n; u0 += gridDim.y * 1024) {
        uint2 w[4];
        float s[4];
        bool live[4];
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const int u = u0 + 256 * q + threadIdx.x;
            const Kv8Piece p = kv8_piece(u, lane_bits, row_bits);
            live[q] = u < n && p.l * 8 < c.hd && s_at[p.row] >= 0 && (p.w & 1 ? v : k);
            if (!live[q]) continue;
            const int64_t row = (int64_t)(p.w >> 1) * c.tokens + s_at[p.row];
            w[q] = load_codes<T, NT>((p.w & 1 ? c.v : c.k) + row * c.hd, p.l, c.hd);
            s[q] = (p.w & 1 ? c.vs : c.ks)[row];
        }
#pragma unroll
        for (int q = 0; q < 4; q++) {
            if (!live[q]) continue;
            const Kv8Piece p = kv8_piece(u0 + 256 * q + threadIdx.x, lane_bits, row_bits);
            const int64_t r = r0 + p.row;
            const int h = p.w >> 1;
            float x[8];
            dequantise4(w[q].x, s[q], x);
            dequantise4(w[q].y, s[q], x + 4);
            store8<T, WIDE, NT>(p.w & 1 ? v + r * v_row + h * v_head : k + r * k_row + h * k_head, p.l, c.hd, x);
        }
    }
}

// lanes of a vector: the power of two that holds head_dim / 8
static int vector_lane_bits(int hd)
{
    int b = 1;
    while ((8 << b) < hd) b++;
    return b;
}
static bool wide_rows(int esz, const void *p, int64_t row, int64_t head)
{
    return ((uintptr_t)p % 16) == 0 && row * esz % 16 == 0 && head * esz % 16 == 0;
}
// Rows of a block, as a power of two: enough for two pieces a thread as long as 512 blocks are left (35000 rows of 2 heads of 64, bf16, in and
// out: 43 and 38 us with a row per block, 12 and 10 so; 2048 rows of 8 of 128 7.1 and 5.5 either way).  `many` (2^23 elements of K: more
// than stays in a cache beside what else a step touches): eight at least, whose codes lie together, and the nontemporal hint: 51200
// rows of 8 heads of 128, bf16, one row per block and eight: 100 and 71 us in, 90 and 68 out; 32 rows 78 and 71.
static int kv8_row_bits(int n_rows, int pieces, bool many)
{
    int b = many ? 3 : 0;
    while (1 << b < KV8_MAX_ROWS && (int64_t)pieces << b < 512 && n_rows >> (b + 1) >= 512) b++;
    return b;
}
static dim3 vector_grid(int n_rows, int row_bits, int pieces)
{
    const int gx = (n_rows + (1 << row_bits) - 1) >> row_bits, turns = (int)((((int64_t)pieces << row_bits) + 1023) / 1024);
    return dim3(gx, std::max(1, std::min(turns, 2048 / gx)));
}

#define KV8_MOVE(KERNEL, CV)                                                                                                                   \
    const int esz = dtype == SD_BF16 ? 2 : 4, bits = vector_lane_bits(c.hd), pieces = 2 * c.kv_heads << bits;                                  \
    const bool wide = wide_rows(esz, k, k_row, k_head) && wide_rows(esz, v, v_row, v_head); /* (a null pointer counts as aligned) */            \
    const bool many = (int64_t)n_rows * c.kv_heads * c.hd >= 1 << 23;                                                                          \
    const int row_bits = kv8_row_bits(n_rows, pieces, many);                                                                                   \
    const dim3 grid = vector_grid(n_rows, row_bits, pieces);                                                                                   \
    if (dtype == SD_BF16) {                                                                                                                    \
        if (wide && many) KV8_GO(KERNEL, CV bf16_t, bf16_t, true, true);                                                                       \
        else if (wide) KV8_GO(KERNEL, CV bf16_t, bf16_t, true, false);                                                                         \
        else if (many) KV8_GO(KERNEL, CV bf16_t, bf16_t, false, true);                                                                         \
        else KV8_GO(KERNEL, CV bf16_t, bf16_t, false, false);                                                                                  \
    } else {                                                                                                                                   \
        if (wide && many) KV8_GO(KERNEL, CV float, float, true, true);                                                                         \
        else if (wide) KV8_GO(KERNEL, CV float, float, true, false);                                                                           \
        else if (many) KV8_GO(KERNEL, CV float, float, false, true);                                                                           \
        else KV8_GO(KERNEL, CV float, float, false, false);                                                                                    \
    }                                                                                                                                          \
    return hipGetLastError();
#define KV8_GO(KERNEL, P, T, W, NT) \
    hipLaunchKernelGGL((KERNEL<T, W, NT>), grid, dim3(256), 0, s, c, rw, n_rows, bits, row_bits, (P *)k, k_row, k_head, (P *)v, v_row, v_head)

hipError_t launch_kv8_append(hipStream_t s, const Kv8View &c, const Kv8Rows &rw, int n_rows, int dtype, const void *k, int64_t k_row,
                             int64_t k_head, const void *v, int64_t v_row, int64_t v_head)
{
    KV8_MOVE(kv8_append_kernel, const)
}

hipError_t launch_kv8_read(hipStream_t s, const Kv8View &c, const Kv8Rows &rw, int n_rows, int dtype, void *k, int64_t k_row, int64_t k_head,
                           void *v, int64_t v_row, int64_t v_head)
{
    KV8_MOVE(kv8_read_kernel, )
}

// ---------------------------------------------------------------- the path's step between projection and attention
// hd / 8 lanes per vector as above, but a lane holds four dimensions of each rotary half, so that a pair never crosses lanes.
#define KV8_MAX_SLABS 8
__global__ __launch_bounds__(256) void kv8_rope_append_kernel(const float *__restrict__ qkv, int n_slabs, size_t slab_stride, PlanView pv,
                                                              CtxView cv, Kv8View c, int lane_bits, int H, const float2 *__restrict__ rope, int max_pos,
                                                              float *__restrict__ q, int first)
{
    const int r = blockIdx.x, hd = c.hd, half = hd / 2, HD = H * hd;
    const int pos = pv.row_pos[r];
    bool valid = pv.row_valid[r];
    if (pos >= max_pos) {
        if (threadIdx.x == 0 && blockIdx.y == 0 && valid) atomicOr(cv.status, 8);
        valid = false;
    }
    const int64_t at = cv.off[pv.row_b[r]] + pos;
    const int lanes = 1 << lane_bits, per_block = 256 / lanes, l = threadIdx.x & (lanes - 1), d0 = 4 * l, d1 = half + 4 * l;
    // vectors: the H heads of q (unless first = 1: the rows hold keys and values only), of k, of v
    const int n = (3 - first) * H;
    const float *row = qkv + (size_t)r * n * hd;
    for (int u = blockIdx.y * per_block; u < n; u += gridDim.y * per_block) {
        const int w = min(u + (int)threadIdx.x / lanes, n - 1), part = w / H + first, h = w % H;
        const bool live = u + (int)threadIdx.x / lanes < n;
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (valid)
            for (int sl = 0; sl < n_slabs; sl++) { // split-K slabs, added in slab order
                const float *p = row + (size_t)sl * slab_stride + (size_t)w * hd;
                const float4 a = *(const float4 *)(p + d0), b = *(const float4 *)(p + d1);
                x[0] += a.x, x[1] += a.y, x[2] += a.z, x[3] += a.w, x[4] += b.x, x[5] += b.y, x[6] += b.z, x[7] += b.w;
            }
        if (valid && part < 2) {
            const float2 *cs = rope + (size_t)pos * half + d0;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float2 t = cs[e];
                const float a = x[e] * t.x - x[4 + e] * t.y, b = x[4 + e] * t.x + x[e] * t.y;
                x[e] = a, x[4 + e] = b;
            }
        }
        if (part == 0) {
            if (live) {
                float *dst = q + (size_t)r * HD + h * hd;
                *(float4 *)(dst + d0) = make_float4(x[0], x[1], x[2], x[3]);
                *(float4 *)(dst + d1) = make_float4(x[4], x[5], x[6], x[7]);
            }
        }
        const float s = kv8_scale(amax_lanes(amax_bits8(x), lane_bits)), inv = 1.0f / s; // (every lane takes part)
        if (!valid || !live || part == 0) continue;
        const bool fine = s == s;
        const int64_t i = (int64_t)h * c.tokens + at;
        int8_t *dst = (part == 2 ? c.v : c.k) + i * hd;
        const uint2 codes = fine ? quantise8(x, s, inv) : make_uint2(0, 0);
        *(uint32_t *)(dst + d0) = codes.x;
        *(uint32_t *)(dst + d1) = codes.y;
        if (l == 0) (part == 2 ? c.vs : c.ks)[i] = s;
    }
}

hipError_t launch_kv8_rope_append(hipStream_t s, const float *qkv, int n_slabs, size_t slab_stride, PlanView pv, CtxView cv, const Kv8View &c,
                                  int M, int H, const float2 *rope, int max_pos, float *q, bool kv_only)
{
    if (n_slabs > KV8_MAX_SLABS || c.hd < 16 || c.hd > 128 || (c.hd & (c.hd - 1))) return hipErrorInvalidValue; // (the path's head widths: powers of two)
    const int lanes = c.hd / 8, first = kv_only ? 1 : 0, passes = ((3 - first) * H * lanes + 255) / 256;
    const dim3 grid(M, std::max(1, std::min(passes, 2048 / M)));
    hipLaunchKernelGGL(kv8_rope_append_kernel, grid, dim3(256), 0, s, qkv, n_slabs, slab_stride, pv, cv, c, vector_lane_bits(c.hd), H, rope, max_pos, q, first);
    return hipGetLastError();
}

// ---------------------------------------------------------------- calls
static int check_cache(const char *who, const sd_kv8 *c)
{
    if (!c) return sd_fail(SD_EINVAL, std::string(who) + ": null cache");
    if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->off || !c->cap) return sd_fail(SD_EINVAL, std::string(who) + ": null pointer in the cache");
    if (c->n_kv_heads < 1 || c->n_kv_heads > 65535 || c->n_seq < 1 || c->tokens < 1)
        return sd_fail(SD_EINVAL, std::string(who) + ": n_kv_heads, n_seq and tokens must be positive");
    if (c->head_dim < 16 || c->head_dim > 256 || c->head_dim % 16) return sd_fail(SD_EINVAL, std::string(who) + ": head_dim must be a multiple of 16 in 16..256");
    if (((uintptr_t)c->k | (uintptr_t)c->v) % 16) return sd_fail(SD_EINVAL, std::string(who) + ": codes must be 16-byte aligned");
    if (((uintptr_t)c->k_scale | (uintptr_t)c->v_scale | (uintptr_t)c->cap | (uintptr_t)c->status) % 4 || (uintptr_t)c->off % 8)
        return sd_fail(SD_EINVAL, std::string(who) + ": a pointer in the cache is not aligned to its elements");
    return SD_OK;
}
static int check_rows(const char *who, const sd_kv8 *c, const int32_t *len, int n_seq, const int32_t *row_start, int rows)
{
    if (!len) return sd_fail(SD_EINVAL, std::string(who) + ": null lengths");
    if (n_seq < 1 || n_seq > c->n_seq) return sd_fail(SD_EINVAL, std::string(who) + ": n_seq out of range");
    if (rows < 1 || rows > (1 << 23)) return sd_fail(SD_EINVAL, std::string(who) + ": rows must be 1..2^23"); // (a block per row)
    if (!row_start && rows % n_seq) return sd_fail(SD_EINVAL, std::string(who) + ": without row_start, rows must be a multiple of n_seq");
    return SD_OK;
}
static int check_strided(const char *who, const char *what, const void *p, int esz, int64_t row, int64_t head, int rows, int heads, int hd)
{
    if ((uintptr_t)p % esz) return sd_fail(SD_EINVAL, std::string(who) + ": " + what + " is not aligned to its elements");
    if ((rows > 1 ? row < hd : row < 0) || (heads > 1 ? head < hd : head < 0))
        return sd_fail(SD_EINVAL, std::string(who) + ": strides of " + what + " must be at least head_dim");
    return SD_OK;
}
static Kv8View view_of(const sd_kv8 *c)
{
    return Kv8View{c->k, c->v, c->k_scale, c->v_scale, c->tokens, c->n_kv_heads, c->head_dim, c->n_seq, c->off, c->cap, c->status};
}
static Kv8Rows rows_of(const int32_t *seq_ids, int n_seq, const int32_t *len, const int32_t *row_start, int rows)
{
    return Kv8Rows{seq_ids, len, row_start, nullptr, n_seq, row_start ? rows : rows / n_seq, 1, 0};
}

extern "C" int sd_kv8_append(const sd_kv8 *c, const int32_t *seq_ids, int32_t n_seq, const int32_t *len, const int32_t *row_start,
                             int32_t rows, int32_t dtype, const void *k, int64_t k_row, int64_t k_head, const void *v, int64_t v_row,
                             int64_t v_head, void *stream)
{
    const char *who = "sd_kv8_append";
    int rc = check_cache(who, c);
    if (!rc) rc = check_rows(who, c, len, n_seq, row_start, rows);
    if (rc) return rc;
    if (!k || !v) return sd_fail(SD_EINVAL, "sd_kv8_append: null rows");
    if (dtype != SD_FP32 && dtype != SD_BF16) return sd_fail(SD_EINVAL, "sd_kv8_append: bad dtype");
    const int esz = dtype == SD_BF16 ? 2 : 4;
    rc = check_strided(who, "k", k, esz, k_row, k_head, rows, c->n_kv_heads, c->head_dim);
    if (!rc) rc = check_strided(who, "v", v, esz, v_row, v_head, rows, c->n_kv_heads, c->head_dim);
    if (rc) return rc;
    SD_HIP(launch_kv8_append((hipStream_t)stream, view_of(c), rows_of(seq_ids, n_seq, len, row_start, rows), rows, dtype, k, k_row, k_head, v,
                             v_row, v_head));
    return SD_OK;
}

extern "C" int sd_kv8_read(const sd_kv8 *c, const int32_t *seq_ids, int32_t n_seq, const int32_t *start, const int32_t *row_start, int32_t rows,
                           int32_t dtype, void *k, int64_t k_row, int64_t k_head, void *v, int64_t v_row, int64_t v_head, void *stream)
{
    const char *who = "sd_kv8_read";
    int rc = check_cache(who, c);
    if (!rc) rc = check_rows(who, c, start, n_seq, row_start, rows);
    if (rc) return rc;
    if (!k && !v) return sd_fail(SD_EINVAL, "sd_kv8_read: neither k nor v is wanted");
    if (dtype != SD_FP32 && dtype != SD_BF16) return sd_fail(SD_EINVAL, "sd_kv8_read: bad dtype");
    const int esz = dtype == SD_BF16 ? 2 : 4;
    if (k) rc = check_strided(who, "k", k, esz, k_row, k_head, rows, c->n_kv_heads, c->head_dim);
    if (!rc && v) rc = check_strided(who, "v", v, esz, v_row, v_head, rows, c->n_kv_heads, c->head_dim);
    if (rc) return rc;
    SD_HIP(launch_kv8_read((hipStream_t)stream, view_of(c), rows_of(seq_ids, n_seq, start, row_start, rows), rows, dtype, k, k ? k_row : 0,
                           k ? k_head : 0, v, v ? v_row : 0, v ? v_head : 0));
    return SD_OK;
}

static int check_attn(const char *who, const sd_kv8 *c, const sd_kv8_attn *a)
{
    int rc = check_cache(who, c);
    if (rc) return rc;
    if (!a) return sd_fail(SD_EINVAL, std::string(who) + ": null arguments");
    rc = check_rows(who, c, a->len, a->n_seq, a->row_start, a->rows);
    if (rc) return rc;
    if (!a->q || !a->out) return sd_fail(SD_EINVAL, std::string(who) + ": null q or out");
    if (a->dtype != SD_FP32 && a->dtype != SD_BF16) return sd_fail(SD_EINVAL, std::string(who) + ": bad dtype");
    if (a->n_heads < 1 || a->n_heads > 65535 || a->n_heads % c->n_kv_heads)
        return sd_fail(SD_EINVAL, std::string(who) + ": n_heads must be a multiple of n_kv_heads");
    if ((int64_t)a->rows * (a->n_heads / c->n_kv_heads) > 0x7fffffff)
        return sd_fail(SD_EINVAL, std::string(who) + ": rows times query heads per cache head must fit 31 bits");
    if (a->max_rows < 0 || a->max_len < 0) return sd_fail(SD_EINVAL, std::string(who) + ": max_rows and max_len must not be negative");
    if (!std::isfinite(a->scale * 1.44269504088896341f)) return sd_fail(SD_EINVAL, std::string(who) + ": scale must be finite");
    if (a->window < 0 || a->sinks < 0) return sd_fail(SD_EINVAL, std::string(who) + ": window and sinks must not be negative");
    if (a->sinks && !a->window) return sd_fail(SD_EINVAL, std::string(who) + ": sinks need a window");
    if (a->window && !a->causal) return sd_fail(SD_EINVAL, std::string(who) + ": a window needs causal rows");
    const int esz = a->dtype == SD_BF16 ? 2 : 4;
    rc = check_strided(who, "q", a->q, esz, a->q_row, a->q_head, a->rows, a->n_heads, c->head_dim);
    if (!rc) rc = check_strided(who, "out", a->out, esz, a->o_row, a->o_head, a->rows, a->n_heads, c->head_dim);
    if (rc) return rc;
    if ((uintptr_t)a->lse % 4) return sd_fail(SD_EINVAL, std::string(who) + ": lse is not aligned to its elements");
    return SD_OK;
}
static Kv8Attn attn_of(const sd_kv8_attn *a)
{
    Kv8Attn k = {};
    k.q = a->q, k.q_row = a->q_row, k.q_head = a->q_head;
    k.out = a->out, k.o_row = a->o_row, k.o_head = a->o_head;
    k.lse = a->lse, k.n_heads = a->n_heads, k.dtype = a->dtype;
    k.causal = a->causal != 0, k.window = std::min(a->window, KV8_MAX_TOKENS), k.sinks = std::min(a->sinks, KV8_MAX_TOKENS);
    k.scale = a->scale * 1.44269504088896341f;
    k.total_rows = a->rows, k.max_len = a->max_len;
    k.max_rows = a->row_start ? a->max_rows : a->rows / a->n_seq;
    return k;
}

extern "C" int64_t sd_kv8_attend_workspace(const sd_kv8 *c, const sd_kv8_attn *a)
{
    int rc = check_attn("sd_kv8_attend_workspace", c, a);
    if (rc) return rc;
    return kv8_attn_workspace(view_of(c), rows_of(a->seq_ids, a->n_seq, a->len, a->row_start, a->rows), attn_of(a));
}

extern "C" int sd_kv8_attend(const sd_kv8 *c, const sd_kv8_attn *a, void *stream)
{
    int rc = check_attn("sd_kv8_attend", c, a);
    if (rc) return rc;
    if (a->workspace_bytes < 0 || (uintptr_t)a->workspace % 16) return sd_fail(SD_EINVAL, "sd_kv8_attend: workspace must be 16-byte aligned, its size not negative");
    const Kv8View v = view_of(c);
    const Kv8Rows rw = rows_of(a->seq_ids, a->n_seq, a->len, a->row_start, a->rows);
    const Kv8Attn k = attn_of(a);
    if (a->workspace && a->workspace_bytes < kv8_attn_workspace(v, rw, k))
        return sd_fail(SD_ECAP, "sd_kv8_attend: workspace smaller than sd_kv8_attend_workspace says");
    SD_HIP(launch_kv8_attn((hipStream_t)stream, v, rw, k, a->workspace, a->workspace ? a->workspace_bytes : 0));
    return SD_OK;
}
