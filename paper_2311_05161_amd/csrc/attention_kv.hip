// Attention over the 4-bit cache of Keys and Values:
//
//     o[b, i, h] = sum_t p_t v_t,   p = softmax_t(scale q[b, i, h] . k_t),   t = 0 .. start[b] + i
//
// with the h / (Hq / Hkv)-th head of the cache.  A query that is not there (i >= count[b]) gives zeros.
#include "kv_dint4.hpp"

namespace w4a8 {

struct AttnArgs {
    const void *q;
    void *out;                    // [B][S][Hq][D]
    int64_t q_ld_b, q_ld_s, q_ld_h;
    int Hq, group;                // query heads to a head of the cache
    int max_len;                  // no token at or past it is looked at
    float scale_log2;             // scale / ln 2
};

template <typename T> __device__ __forceinline__ T attn_from_f32(float v);
template <> __device__ __forceinline__ float attn_from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half attn_from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ bf16_t attn_from_f32<bf16_t>(float v) { return bf16_t{f32_to_bf16_bits(v)}; }

// Any head size (a multiple of 8, at most 512), page size and alignment: a workgroup per query row, L lanes (8 channels each) per
// token, 256 / L tokens at a time, each group of lanes with a running maximum, sum and output of its own, joined at the end.
template <typename T, int L>
__global__ __launch_bounds__(256) void attn_rows_kernel(AttnArgs p, KvView c, KvTokens t)
{
    constexpr int GROUPS = 256 / L;
    __shared__ float part_m[GROUPS], part_l[GROUPS];
    __shared__ float part_o[GROUPS][L * 8 + 1];
    const int h = blockIdx.x % p.Hq;
    const int64_t row = blockIdx.x / p.Hq;
    const int b = (int)(row / t.S), i = (int)(row - (int64_t)b * t.S);
    const int tid = threadIdx.x, lane = tid & (L - 1), g = tid / L, words = c.D / 8;
    const KvLength len = kv_length(t, c, b);
    const int seen = i < len.count ? min(len.start + i + 1, p.max_len) : 0;
    float q[8], o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        q[j] = lane < words ? to_f32(((const T *)p.q)[b * p.q_ld_b + i * p.q_ld_s + h * p.q_ld_h + lane * 8 + j]) : 0.0f;
        o[j] = 0.0f;
    }
    float m = -INFINITY, l = 0.0f;
    for (int t0 = 0; t0 < seen; t0 += GROUPS) {      // (uniform: the groups' sums need all lanes)
        const int64_t at = t0 + g < seen ? kv_row(t, c, b, h / p.group, t0 + g) : -1;
        const bool mine = at >= 0 && lane < words;
        float k[8];
        const int32_t kw = at >= 0 ? c.words[0][at] : 0, vw = at >= 0 ? c.words[1][at] : 0;
        kv_decode8(mine ? reinterpret_cast<const uint32_t *>(c.packed[0])[at * words + lane] : 0, make_decode_lut(kw & 15), k);
        float dot = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) dot = __builtin_fmaf(q[j], k[j], dot);
        dot = group_sum<L>(dot);
        if (at >= 0) {                               // (uniform over the group)
            const float s = dot * (0.125f * kv_step(kw) * p.scale_log2);
            const float top = fmaxf(m, s), keep = exp2f(m - top), w = exp2f(s - top);
            m = top;
            l = l * keep + w;
            float v[8];
            kv_decode8(mine ? reinterpret_cast<const uint32_t *>(c.packed[1])[at * words + lane] : 0, make_decode_lut(vw & 15), v);
            const float wv = w * (0.125f * kv_step(vw));
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = __builtin_fmaf(wv, v[j], o[j] * keep);
        }
    }
    if (lane == 0) {
        part_m[g] = m;
        part_l[g] = l;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) part_o[g][lane * 8 + j] = o[j];
    __syncthreads();
    float top = -INFINITY, sum = 0.0f;
    for (int x = 0; x < GROUPS; ++x) top = fmaxf(top, part_m[x]);
    const bool any = top > -INFINITY;
    for (int x = 0; x < GROUPS; ++x) sum += any ? part_l[x] * exp2f(part_m[x] - top) : 0.0f;
    T *out = (T *)p.out + (row * p.Hq + h) * (int64_t)c.D;
    for (int d = tid; d < c.D; d += 256) {
        float v = 0.0f;
        for (int x = 0; x < GROUPS; ++x) v += any ? part_o[x][d] * exp2f(part_m[x] - top) : 0.0f;
        out[d] = attn_from_f32<T>(any ? v / sum : 0.0f);
    }
}

template <typename T>
static int launch_attn_t(const AttnArgs &p, const KvView &c, const KvTokens &t, hipStream_t st)
{
    const int64_t blocks = (int64_t)t.B * t.S * p.Hq;
    if (blocks > 0x7fffffffLL) return W4A8_ERR_SHAPE;
    const dim3 grid((unsigned)blocks), block(256);
    const int words = c.D / 8;
    if (words <= 8) {
        hipLaunchKernelGGL((attn_rows_kernel<T, 8>), grid, block, 0, st, p, c, t);
    } else if (words <= 16) {
        hipLaunchKernelGGL((attn_rows_kernel<T, 16>), grid, block, 0, st, p, c, t);
    } else if (words <= 32) {
        hipLaunchKernelGGL((attn_rows_kernel<T, 32>), grid, block, 0, st, p, c, t);
    } else {
        hipLaunchKernelGGL((attn_rows_kernel<T, 64>), grid, block, 0, st, p, c, t);
    }
    return hip_status(hipGetLastError());
}

size_t attention_kv_workspace(int, const KvView &, const KvTokens &, int, int64_t) { return 0; }

int launch_attention_kv(const void *Q, const int64_t *q_ld, int dtype, int Hq, const KvView &c, const KvTokens &t, float scale,
                        int64_t max_len, void *out, void *, hipStream_t st)
{
    const int64_t room = (int64_t)t.table_cols * c.page_size;
    const AttnArgs p = {Q, out, q_ld[0], q_ld[1], q_ld[2], Hq, Hq / c.heads, (int)(max_len < room ? max_len : room),
                        scale * 1.44269504088896341f};
    switch (dtype) {
        case W4A8_F32: return launch_attn_t<float>(p, c, t, st);
        case W4A8_F16: return launch_attn_t<__half>(p, c, t, st);
        case W4A8_BF16: return launch_attn_t<bf16_t>(p, c, t, st);
        default: return W4A8_ERR_DTYPE;
    }
}

}  // namespace w4a8
