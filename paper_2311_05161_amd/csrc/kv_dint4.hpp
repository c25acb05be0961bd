// The 4-bit cache of Keys and Values as the kernels see it.
//
// A row is one (token, head): D channels as dINT4 nibbles (the re-encoded nibbles of the tiled weight layout: word q of the row
// holds channels 8 q .. 8 q + 7, the first four in the low nibbles of its bytes, the others in the high ones) and one 32-bit
// word, the bits of the row's step with the zero-point in the last four.  Rows lie in pages [pages][heads][page_size]; the
// table gives each sequence's pages in the order of its tokens.
#pragma once
#include "w4a8_common.hpp"

namespace w4a8 {

struct KvView {
    uint8_t *packed[2];     // Keys, Values: [pages][heads][page_size][D / 2], the last two contiguous
    int32_t *words[2];      // [pages][heads][page_size]
    int64_t pages, page_ld, head_ld;    // (ld: in rows)
    int heads, page_size, D;
};
struct KvTokens {
    const int32_t *start, *count, *table;   // [B], [B] (null: all S), [B][table_ld]
    int64_t table_ld;
    int B, S, table_cols;
};

// Tokens of a sequence: how many are cached before this step, and how many of the S new ones are there.  What the device memory
// holds is clamped to what the table can name, so that no value of it leads out of bounds.
struct KvLength {
    int start, count;
};
__device__ __forceinline__ KvLength kv_length(const KvTokens &t, const KvView &c, int b)
{
    const int64_t room = (int64_t)t.table_cols * c.page_size;
    KvLength n;
    n.start = (int)min(max((int64_t)t.start[b], (int64_t)0), min(room, (int64_t)0x7fffffff));
    n.count = t.count ? min(max(t.count[b], 0), t.S) : t.S;
    n.count = (int)min((int64_t)n.count, room - n.start);
    return n;
}

// The index of a token's row; -1 where the table names no page of the cache.
__device__ __forceinline__ int64_t kv_row(const KvTokens &t, const KvView &c, int b, int head, int token)
{
    const int j = token / c.page_size;
    const int64_t page = t.table[b * t.table_ld + j];
    return page < 0 || page >= c.pages ? -1 : page * c.page_ld + head * c.head_ld + (token - j * c.page_size);
}

// One word's eight values in units of step / 8: the decode of the packed weights (D = 4 (d + beta), unsigned bytes), widened.
__device__ __forceinline__ void kv_decode8(uint32_t p, const DecodeLut &t, float (&v)[8])
{
    int a, b;
    decode_word(p, t, a, b);
    const float beta = (float)t.beta_q;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = (float)((uint32_t)a >> (8 * i) & 255u) - beta;
        v[i + 4] = (float)((uint32_t)b >> (8 * i) & 255u) - beta;
    }
}
__device__ __forceinline__ float kv_step(int32_t word) { return __int_as_float(word & -16); }

// reductions over groups of L lanes (a power of two); all 64 lanes active
// (numbers that are not negative are ordered as their bits are, and the integer maximum takes the other lane's value as it comes)
template <int L>
__device__ __forceinline__ float group_max_positive(float f)
{
    uint32_t v = __float_as_uint(f) & 0x7fffffffu;          // (-0 is 0)
    if (L > 1) v = max(v, (uint32_t)dpp_i32<DPP_QUAD_XOR1>((int)v));
    if (L > 2) v = max(v, (uint32_t)dpp_i32<DPP_QUAD_XOR2>((int)v));
    if (L > 4) v = max(v, (uint32_t)dpp_i32<DPP_ROW_HALF_MIRROR>((int)v));
    if (L > 8) v = max(v, (uint32_t)dpp_i32<DPP_ROW_MIRROR>((int)v));
    if (L > 16) v = max(v, (uint32_t)__shfl_xor((int)v, 16));
    if (L > 32) v = max(v, (uint32_t)__shfl_xor((int)v, 32));
    return __uint_as_float(v);
}
template <int L>
__device__ __forceinline__ float group_sum(float v)
{
    if (L > 1) v += dpp_f32<DPP_QUAD_XOR1>(v);
    if (L > 2) v += dpp_f32<DPP_QUAD_XOR2>(v);
    if (L > 4) v += dpp_f32<DPP_ROW_HALF_MIRROR>(v);
    if (L > 8) v += dpp_f32<DPP_ROW_MIRROR>(v);
    if (L > 16) v += __shfl_xor(v, 16);
    if (L > 32) v += __shfl_xor(v, 32);
    return v;
}

// Host-side launchers; ld: distances between sequences, tokens and heads in elements.
int launch_kv_cache(bool write, const void *K, const int64_t *k_ld, const void *V, const int64_t *v_ld, int dtype, const KvView &c,
                    const KvTokens &t, hipStream_t st);
size_t attention_kv_workspace(int dtype, const KvView &c, const KvTokens &t, int Hq, int64_t max_len);
int launch_attention_kv(const void *Q, const int64_t *q_ld, int dtype, int Hq, const KvView &c, const KvTokens &t, float scale,
                        int64_t max_len, void *out, void *workspace, hipStream_t st);

}  // namespace w4a8
