// Rotary positions as calls of their own: the frequencies (host) and the rotation of rows the caller holds.
#include <math.h>

#include <algorithm>
#include <cmath>

#include "sd_internal.h"

// ---------------------------------------------------------------- frequencies
static int check_rope_config(const char *who, const sd_rope_config *c)
{
    if (!c) return sd_fail(SD_EINVAL, std::string(who) + ": null configuration");
    if (c->rot_dim < 2 || c->rot_dim > 512 || c->rot_dim % 2) return sd_fail(SD_EINVAL, std::string(who) + ": rot_dim must be even, 2..512");
    if (c->scaling < SD_ROPE_PLAIN || c->scaling > SD_ROPE_RAMP) return sd_fail(SD_EINVAL, std::string(who) + ": unknown scaling");
    if (!(c->base > 1.0) || !std::isfinite(c->base)) return sd_fail(SD_EINVAL, std::string(who) + ": base must be above 1");
    if (c->scaling != SD_ROPE_PLAIN && (!(c->factor >= 1.0) || !std::isfinite(c->factor)))
        return sd_fail(SD_EINVAL, std::string(who) + ": factor must be at least 1");
    if (c->scaling >= SD_ROPE_BANDS && (!(c->low > 0.0) || !(c->low < c->high) || !std::isfinite(c->high) || !(c->trained_len >= 1.0) ||
                                        !std::isfinite(c->trained_len)))
        return sd_fail(SD_EINVAL, std::string(who) + ": scaling by bands or by a ramp needs 0 < low < high and trained_len >= 1");
    return SD_OK;
}

extern "C" int sd_rope_freqs(const sd_rope_config *cfg, double *out)
{
    int rc = check_rope_config("sd_rope_freqs", cfg);
    if (rc) return rc;
    if (!out) return sd_fail(SD_EINVAL, "sd_rope_freqs: null output");
    const double R = cfg->rot_dim, two_pi = 2.0 * M_PI;
    // the (fractional) pair that makes r turns over the trained length: trained_len * base^(-2i / R) = 2 pi r
    auto pair_of = [&](double r) { return R * log(cfg->trained_len / (two_pi * r)) / (2.0 * log(cfg->base)); };
    double lo = 0.0, hi = 1.0;
    if (cfg->scaling == SD_ROPE_RAMP) {
        lo = fmax(0.0, floor(pair_of(cfg->high)));
        hi = fmin(R - 1.0, ceil(pair_of(cfg->low)));
    }
    for (int i = 0; i < cfg->rot_dim / 2; i++) {
        const double f = pow(cfg->base, -2.0 * i / R);
        double keep = 1.0; // share of the unscaled frequency
        if (cfg->scaling == SD_ROPE_LINEAR) keep = 0.0;
        if (cfg->scaling == SD_ROPE_BANDS) keep = (cfg->trained_len * f / two_pi - cfg->low) / (cfg->high - cfg->low);
        if (cfg->scaling == SD_ROPE_RAMP) keep = 1.0 - (i - lo) / fmax(hi - lo, 1e-3);
        keep = fmin(1.0, fmax(0.0, keep));
        out[i] = cfg->scaling == SD_ROPE_PLAIN ? f : keep * f + (1.0 - keep) * f / cfg->factor;
    }
    return SD_OK;
}

// ---------------------------------------------------------------- rotation of rows
// One block turns up to RR rows: first every (row, pair) angle once - a 64-bit product, reduced to a fraction of a turn, then
// 32-bit sine and cosine into LDS - and then the heads, which share them (without that the sines cost more than the bytes).
// What is left is bound by memory: 8192 rows of 40 heads of 128, bf16, in 30 us, 5.6 TB/s.
template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
    T v[N];
};

#define ROPE_LDS_PAIRS 512 // angles a block holds: 4 KiB

// VE: elements of one access (16 bytes, or 1 where alignment or widths rule that out).  NT: x is read with the nontemporal hint (8192
// rows of 40 heads of 128, bf16: 37 us without, 30 with; with y written so too 34).
template <bool NT, typename V>
__device__ __forceinline__ V rope_load(const void *p)
{
    if constexpr (NT && sizeof(V) == 16) {
        typedef __attribute__((ext_vector_type(4))) uint32_t words;
        return __builtin_bit_cast(V, __builtin_nontemporal_load((const words *)p));
    } else return *(const V *)p;
}
template <typename T, int VE, bool INTERLEAVED, bool NT>
__global__ __launch_bounds__(256) void rope_kernel(const T *x, int64_t x_row, int64_t x_head, T *y, int64_t y_row, int64_t y_head,
                                                   int n_rows, int RR, int n_heads, int hd, int rot, const int32_t *__restrict__ pos,
                                                   const double *__restrict__ inv_freq, float gain, float sign, bool copy_rest)
{
    __shared__ float2 cs[ROPE_LDS_PAIRS];
    typedef Vec<T, VE> V;
    const int half = rot / 2;
    for (int64_t row0 = (int64_t)blockIdx.x * RR; row0 < n_rows; row0 += (int64_t)gridDim.x * RR) {
    const int nr = (int)min((int64_t)RR, n_rows - row0);
    for (int a = threadIdx.x; a < nr * half; a += 256) {
        const double t = (double)pos[row0 + a / half] * inv_freq[a % half] * (1.0 / (2.0 * M_PI)); // turns
        const float frac = (float)(t - rint(t));
        float s, c;
        sincospif(2.0f * frac, &s, &c);
        cs[a] = make_float2(gain * c, sign * gain * s);
    }
    __syncthreads();
    // items of a head: rot / (2 VE) accesses that hold both members of VE pairs, then the dimensions that stay
    const int turning = half / VE, items = turning + (copy_rest ? (hd - rot) / VE : 0);
    const int per_row = n_heads * items;
    for (int u = blockIdx.y * 256 + threadIdx.x; u < nr * per_row; u += gridDim.y * 256) {
        const int r = u / per_row, rem = u - r * per_row, h = rem / items, it = rem - h * items;
        const T *px = x + (row0 + r) * x_row + h * x_head;
        T *py = y + (row0 + r) * y_row + h * y_head;
        if (it >= turning) {
            const int d = rot + (it - turning) * VE;
            *(V *)(py + d) = *(const V *)(px + d);
            continue;
        }
        const int d0 = INTERLEAVED ? 2 * it * VE : it * VE, d1 = INTERLEAVED ? d0 + VE : d0 + half;
        V a = rope_load<NT, V>(px + d0), b = rope_load<NT, V>(px + d1);
        const float2 *c = cs + r * half + it * VE;
        if constexpr (INTERLEAVED && VE == 1) { // d1 = d0 + 1: the pair itself
            const float2 w = c[0];
            const float p = to_float(a.v[0]), q = to_float(b.v[0]);
            a.v[0] = from_float<T>(p * w.x - q * w.y), b.v[0] = from_float<T>(q * w.x + p * w.y);
        } else if constexpr (INTERLEAVED) {
#pragma unroll
            for (int e = 0; e < VE / 2; e++) {
                float2 w = c[e];
                float p = to_float(a.v[2 * e]), q = to_float(a.v[2 * e + 1]);
                a.v[2 * e] = from_float<T>(p * w.x - q * w.y), a.v[2 * e + 1] = from_float<T>(q * w.x + p * w.y);
                w = c[VE / 2 + e];
                p = to_float(b.v[2 * e]), q = to_float(b.v[2 * e + 1]);
                b.v[2 * e] = from_float<T>(p * w.x - q * w.y), b.v[2 * e + 1] = from_float<T>(q * w.x + p * w.y);
            }
        } else {
#pragma unroll
            for (int e = 0; e < VE; e++) {
                const float2 w = c[e];
                const float p = to_float(a.v[e]), q = to_float(b.v[e]);
                a.v[e] = from_float<T>(p * w.x - q * w.y), b.v[e] = from_float<T>(q * w.x + p * w.y);
            }
        }
        *(V *)(py + d0) = a;
        *(V *)(py + d1) = b;
    }
    __syncthreads(); // the next rows' angles take this place
    }
}

template <typename T, int VE>
static void rope_launch(hipStream_t s, const void *x, int64_t x_row, int64_t x_head, void *y, int64_t y_row, int64_t y_head, int n_rows,
                        int n_heads, int hd, int rot, const int32_t *pos, const double *inv_freq, float gain, bool interleaved, float sign)
{
    const bool copy_rest = (const void *)x != y && hd > rot;
    const int64_t per_row = (int64_t)n_heads * (rot / 2 / VE + (copy_rest ? (hd - rot) / VE : 0));
    // Rows per block: as many as LDS has angles for and still eight blocks for each of the 256 compute units (3873 rows of 11 heads of 128,
    // half of each, fp32: 17.1 us with two, 10.8 with eight; 2000 of 10, bf16, 4.8 and 5.1); few rows are split over their heads instead.
    int RR = std::max(1, std::min(ROPE_LDS_PAIRS / (rot / 2), n_rows / 2048));
    RR = std::min(RR, 8);
    const unsigned gx = (unsigned)std::min(((int64_t)n_rows + RR - 1) / RR, (int64_t)1 << 22);
    const unsigned gy = (unsigned)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(512 / gx, 64), (RR * per_row + 255) / 256));
#define ROPE_GO(I, NT) hipLaunchKernelGGL((rope_kernel<T, VE, I, NT>), dim3(gx, gy), dim3(256), 0, s, (const T *)x, x_row, x_head, (T *)y, y_row, \
                                      y_head, n_rows, RR, n_heads, hd, rot, pos, inv_freq, gain, sign, copy_rest)
    if (interleaved && RR > 1) ROPE_GO(true, true); // (many rows: more than stays in a cache)
    else if (interleaved) ROPE_GO(true, false);
    else if (RR > 1) ROPE_GO(false, true);
    else ROPE_GO(false, false);
#undef ROPE_GO
}

extern "C" int sd_rope(const void *x, int64_t x_row, int64_t x_head, void *y, int64_t y_row, int64_t y_head, int32_t dtype, int32_t n_rows,
                       int32_t n_heads, int32_t head_dim, int32_t rot_dim, const int32_t *pos, const double *inv_freq, float gain,
                       int32_t interleaved, int32_t inverse, void *stream)
{
    if (!x || !y || !pos || !inv_freq) return sd_fail(SD_EINVAL, "sd_rope: null argument");
    if (dtype != SD_FP32 && dtype != SD_BF16) return sd_fail(SD_EINVAL, "sd_rope: bad dtype");
    if (n_rows < 1 || n_heads < 1) return sd_fail(SD_EINVAL, "sd_rope: n_rows and n_heads must be at least 1");
    if (head_dim < 2 || head_dim > 512 || rot_dim < 2 || rot_dim > head_dim || rot_dim % 2)
        return sd_fail(SD_EINVAL, "sd_rope: head_dim must be 2..512 and rot_dim even, 2..head_dim");
    auto bad = [&](int64_t row, int64_t head) {
        return (n_rows > 1 ? row < head_dim : row < 0) || (n_heads > 1 ? head < head_dim : head < 0);
    };
    if (bad(x_row, x_head) || bad(y_row, y_head)) return sd_fail(SD_EINVAL, "sd_rope: strides must be at least head_dim");
    if ((int64_t)n_heads * head_dim > (1 << 24)) return sd_fail(SD_EINVAL, "sd_rope: more than 2^24 elements in a row");
    if (x == y && ((n_rows > 1 && x_row != y_row) || (n_heads > 1 && x_head != y_head)))
        return sd_fail(SD_EINVAL, "sd_rope: in place the strides must agree");
    if (!std::isfinite(gain)) return sd_fail(SD_EINVAL, "sd_rope: gain must be finite");
    if (interleaved != 0 && interleaved != 1) return sd_fail(SD_EINVAL, "sd_rope: interleaved is 0 or 1");
    const int esz = dtype == SD_BF16 ? 2 : 4, ve = 16 / esz;
    if (((uintptr_t)x | (uintptr_t)y) % esz || (uintptr_t)inv_freq % 8 || (uintptr_t)pos % 4)
        return sd_fail(SD_EINVAL, "sd_rope: a pointer is not aligned to its elements");
    const bool wide = ((uintptr_t)x | (uintptr_t)y) % 16 == 0 && (x_row | x_head | y_row | y_head) % ve == 0 && rot_dim % (2 * ve) == 0 &&
                      (head_dim - rot_dim) % ve == 0;
    const float sign = inverse ? -1.f : 1.f;
    hipStream_t s = (hipStream_t)stream;
#define ROPE_T(T, VE) rope_launch<T, VE>(s, x, x_row, x_head, y, y_row, y_head, n_rows, n_heads, head_dim, rot_dim, pos, inv_freq, gain, interleaved != 0, sign)
    if (dtype == SD_BF16) {
        if (wide) ROPE_T(bf16_t, 8);
        else ROPE_T(bf16_t, 1);
    } else {
        if (wide) ROPE_T(float, 4);
        else ROPE_T(float, 1);
    }
#undef ROPE_T
    SD_HIP(hipGetLastError());
    return SD_OK;
}

extern "C" int sd_model_set_rope(sd_model *m, const sd_rope_config *cfg, double gain)
{
    if (!m) return sd_fail(SD_EINVAL, "sd_model_set_rope: null model");
    int rc = check_rope_config("sd_model_set_rope", cfg);
    if (rc) return rc;
    if (cfg->rot_dim != m->cfg.head_dim) return sd_fail(SD_EINVAL, "sd_model_set_rope: the path turns whole heads: rot_dim must be head_dim");
    if (!std::isfinite(gain)) return sd_fail(SD_EINVAL, "sd_model_set_rope: gain must be finite");
    double f[256];
    rc = sd_rope_freqs(cfg, f);
    if (rc) return rc;
    SD_HIP(hipDeviceSynchronize()); // forwards in flight keep their angles
    SD_HIP(set_rope_table(m, f, gain));
    return SD_OK;
}
