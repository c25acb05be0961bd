// The 4-bit cache of Keys and Values: rows are quantized as they are written, and read back as values.
//
//     lo = min(0, min x), hi = max(0, max x);   step = (hi - lo) / 13, to 20 significant bits (half up);   z = rne(-lo / step)
//     u = x / step:   1/4 < u <= 3/4 -> +step/2;   -3/4 <= u < -1/4 -> -step/2;   else step * (clamp(rne(u) + z, 0, 13) - z)
//
// i.e. the rule of the weights (Eq. 5) with a row of D channels for the group, and a step that leaves the last four bits of its
// 32 to the zero-point.  16-bit values lie on the borders of this rule often (x = step / 4, u = 2.5, -lo = hi), so the borders
// are decided as in exact arithmetic, which the 20-bit step makes possible in binary32:
//   - |x| is compared with step / 4 and 3 step / 4 themselves (at most 22 bits: exact);
//   - u = x / step is rounded once, fma(x, inv, x * inv_lo) with inv + inv_lo the reciprocal to 48 bits.  x has at most 11
//     bits and step 20, so u is either a half-integer or at least 2^-21 from one, and u < 16 is rounded by at most that: rne(u)
//     is that of the exact quotient.  (binary32 inputs: by this u.)
//   - the step's half-up at bit 20 looks at the sign of the division's remainder, what hi - lo lost included.
#include "kv_dint4.hpp"
#include "row_quant.hpp"

namespace w4a8 {

constexpr float KV_F32_MIN = 1.1754943508222875e-38f;   // a row whose step would be subnormal counts as all-zero
constexpr float KV_MAGIC = 12582912.0f;                 // 1.5 * 2^23: adding it rounds to integers, ties to even

struct KvRows {            // [B][S][heads][D], D contiguous
    void *x[2];            // Keys, Values
    int64_t ld_b[2], ld_s[2], ld_h[2];
};

// How a wave's 64 / L groups of L lanes are spent: on `tokens` consecutive tokens of 64 / L / tokens consecutive heads
struct KvTiles {
    int tokens_log, s_tiles, h_tiles;
};

struct RowScale {
    float step, inv, inv_lo, zero;
};
// lo_neg = -lo >= 0, hi >= 0
__device__ __forceinline__ RowScale row_scale(float lo_neg, float hi)
{
    RowScale r;
    const float d = hi + lo_neg, back = d - hi;
    const float lost = (hi - (d - back)) + (lo_neg - back);          // hi + lo_neg = d + lost exactly
    const float q = d / 13.0f;
    // half up at the last four bits of (d + lost) / 13, whose nearest binary32 number is within two units of q: the sign of
    // 13 (q - border) + (d - 13 q) + lost; the first two terms are exact, and so is their sum
    const uint32_t base = __float_as_uint(q) & ~15u;
    const float rem = __builtin_fmaf(q - __uint_as_float(base + 8u), 13.0f, __builtin_fmaf(-q, 13.0f, d)) + lost;
    const float step = __uint_as_float(base + (rem >= 0.0f ? 16u : 0u));
    const bool live = step >= KV_F32_MIN;
    r.step = live ? step : 0.0f;
    r.inv = live ? 1.0f / step : 0.0f;
    r.inv_lo = live ? __builtin_fmaf(-r.inv, step, 1.0f) * r.inv : 0.0f;
    const float z = __builtin_fmaf(lo_neg, r.inv, lo_neg * r.inv_lo);
    r.zero = fminf(__builtin_rintf(z), 13.0f);
    return r;
}

// Eight values -> their packed word
__device__ __forceinline__ uint32_t encode8(const float (&x)[8], const RowScale &r)
{
    const float q1 = 0.25f * r.step, q3 = 0.75f * r.step;
    uint32_t c[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float u = __builtin_fmaf(x[j], r.inv, x[j] * r.inv_lo);
        const float k = fminf(fmaxf(u, -r.zero), 13.0f - r.zero);    // (the ends are integers: clamping first changes nothing)
        const uint32_t code = __float_as_uint((k + KV_MAGIC) + r.zero);
        const uint32_t half = 14u + (__float_as_uint(x[j]) >> 31);
        const float ax = fabsf(x[j]);
        c[j] = ((ax > q1) & (ax <= q3)) ? half : code;
    }
    return recode8(pack4_low_bytes(c[0], c[1], c[2], c[3]), pack4_low_bytes(c[4], c[5], c[6], c[7]), 0x01010101u);
}

// A row's place: which (b, s, head) a group of lanes has, and whether there is such a row
struct KvPlace {
    int b, s, head;
    bool in;
};
template <int L>
__device__ __forceinline__ KvPlace kv_place(const KvTokens &t, const KvView &c, const KvTiles &n)
{
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int g = (threadIdx.x & 63) / L, tokens = 1 << n.tokens_log, heads = 64 / L >> n.tokens_log;
    const int64_t rest = wave / n.h_tiles;
    KvPlace p;
    p.head = (int)(wave - rest * n.h_tiles) * heads + (g >> n.tokens_log);
    p.b = (int)(rest / n.s_tiles);
    p.s = (int)(rest - (int64_t)p.b * n.s_tiles) * tokens + (g & (tokens - 1));
    p.in = p.b < t.B && p.s < t.S && p.head < c.heads;
    return p;
}

// L lanes (8 channels each) per row, Keys and Values of it
template <typename T, int L, bool VEC>
__global__ __launch_bounds__(256) void kv_write_kernel(KvRows in, KvView c, KvTokens t, KvTiles n)
{
    const KvPlace at = kv_place<L>(t, c, n);
    const int lane = threadIdx.x & (L - 1), words = c.D / 8;
    bool there = at.in;
    int64_t row = -1;
    if (there) {
        const KvLength len = kv_length(t, c, at.b);
        there = at.s < len.count;
        if (there) row = kv_row(t, c, at.b, at.head, len.start + at.s);
        there = row >= 0;
    }
    const bool mine = there && lane < words;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (mine) {
            const T *p = (const T *)in.x[kv] + at.b * in.ld_b[kv] + at.s * in.ld_s[kv] + at.head * in.ld_h[kv] + lane * 8;
            if (VEC) {
                load8<T>(p, x);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = to_f32(p[j]);
            }
        }
        float lo = 0.0f, hi = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            lo = fmaxf(lo, -x[j]);
            hi = fmaxf(hi, x[j]);
        }
        const RowScale r = row_scale(group_max<L>(lo), group_max<L>(hi));
        if (mine) {
            reinterpret_cast<uint32_t *>(c.packed[kv])[row * words + lane] = encode8(x, r);
            if (lane == 0) c.words[kv][row] = __float_as_int(r.step) | (int)r.zero;
        }
    }
}

template <typename T> __device__ __forceinline__ void store8(T *p, const float (&v)[8]);
template <>
__device__ __forceinline__ void store8<float>(float *p, const float (&v)[8])
{
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
template <>
__device__ __forceinline__ void store8<__half>(__half *p, const float (&v)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_to_f16_bits(v[2 * i]) | (uint32_t)f32_to_f16_bits(v[2 * i + 1]) << 16;
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
template <>
__device__ __forceinline__ void store8<bf16_t>(bf16_t *p, const float (&v)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_to_bf16_bits(v[2 * i]) | (uint32_t)f32_to_bf16_bits(v[2 * i + 1]) << 16;
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// The same map the other way; rows that are not there are zeros
template <typename T, int L>
__global__ __launch_bounds__(256) void kv_read_kernel(KvRows out, KvView c, KvTokens t, KvTiles n)
{
    const KvPlace at = kv_place<L>(t, c, n);
    const int lane = threadIdx.x & (L - 1), words = c.D / 8;
    if (!at.in || lane >= words) return;
    const KvLength len = kv_length(t, c, at.b);
    const int64_t row = at.s < len.count ? kv_row(t, c, at.b, at.head, len.start + at.s) : -1;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (row >= 0) {
            const int32_t word = c.words[kv][row];
            kv_decode8(reinterpret_cast<const uint32_t *>(c.packed[kv])[row * words + lane], make_decode_lut(word & 15), v);
            const float unit = 0.125f * kv_step(word);   // (20 bits and above the subnormals by 2^3 at least where it matters)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= unit;
        }
        store8<T>((T *)out.x[kv] + at.b * out.ld_b[kv] + at.s * out.ld_s[kv] + at.head * out.ld_h[kv] + lane * 8, v);
    }
}

static KvTiles kv_tiles(const KvTokens &t, const KvView &c, int L, int64_t &blocks)
{
    KvTiles n;
    const int groups = 64 / L;
    n.tokens_log = 0;
    while (1 << n.tokens_log < groups && 1 << n.tokens_log < t.S) ++n.tokens_log;
    const int tokens = 1 << n.tokens_log, heads = groups / tokens;
    n.s_tiles = (t.S + tokens - 1) / tokens;
    n.h_tiles = (c.heads + heads - 1) / heads;
    blocks = ((int64_t)t.B * n.s_tiles * n.h_tiles + 3) / 4;
    return n;
}

template <typename T, int L>
static int launch_kv(bool write, const KvRows &rows, const KvView &c, const KvTokens &t, bool vec, hipStream_t st)
{
    int64_t blocks;
    const KvTiles n = kv_tiles(t, c, L, blocks);
    if (blocks > 0x7fffffffLL) return W4A8_ERR_SHAPE;
    const dim3 grid((unsigned)blocks), block(256);
    if (!write) {
        hipLaunchKernelGGL((kv_read_kernel<T, L>), grid, block, 0, st, rows, c, t, n);
    } else if (vec) {
        hipLaunchKernelGGL((kv_write_kernel<T, L, true>), grid, block, 0, st, rows, c, t, n);
    } else {
        hipLaunchKernelGGL((kv_write_kernel<T, L, false>), grid, block, 0, st, rows, c, t, n);
    }
    return hip_status(hipGetLastError());
}

template <typename T>
static int launch_kv_t(bool write, const KvRows &rows, const KvView &c, const KvTokens &t, hipStream_t st)
{
    bool vec = true;
    for (int kv = 0; kv < 2; ++kv)
        vec = vec && (uintptr_t)rows.x[kv] % 16 == 0 && (rows.ld_b[kv] | rows.ld_s[kv] | rows.ld_h[kv]) * (int64_t)sizeof(T) % 16 == 0;
    const int words = c.D / 8;
    if (words <= 8) return launch_kv<T, 8>(write, rows, c, t, vec, st);
    if (words <= 16) return launch_kv<T, 16>(write, rows, c, t, vec, st);
    if (words <= 32) return launch_kv<T, 32>(write, rows, c, t, vec, st);
    return launch_kv<T, 64>(write, rows, c, t, vec, st);
}

int launch_kv_cache(bool write, const void *K, const int64_t *k_ld, const void *V, const int64_t *v_ld, int dtype, const KvView &c,
                    const KvTokens &t, hipStream_t st)
{
    const KvRows rows = {{(void *)K, (void *)V}, {k_ld[0], v_ld[0]}, {k_ld[1], v_ld[1]}, {k_ld[2], v_ld[2]}};
    switch (dtype) {
        case W4A8_F32: return launch_kv_t<float>(write, rows, c, t, st);
        case W4A8_F16: return launch_kv_t<__half>(write, rows, c, t, st);
        case W4A8_BF16: return launch_kv_t<bf16_t>(write, rows, c, t, st);
        default: return W4A8_ERR_DTYPE;
    }
}

}  // namespace w4a8
