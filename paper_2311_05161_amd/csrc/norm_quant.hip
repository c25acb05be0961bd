// Root-mean-square norm in front of a W4A8 linear: the residual's addition, the norm, the fold of the AQAS scale and the
// per-token INT8 quantization in one pass over the row.
//
//     h = cast(x + r);   t[k] = h[k] * (w[k] * (1 / s[k]));   a = max |t|;   n = 1 / sqrt(mean h^2 + eps)
//     Xq[k] = rne(t[k] * (127 / a));   sx = a * n / 127
//
// The norm's factor n is one number for the row and cancels in t / a, so the codes do not wait for it: only sx does.  The
// steps up to the codes are binary32 operations in the order written (as in quantize_act_int8); the sum of squares and sx are
// evaluated in binary64, which squares of any binary32 value neither overflow nor lose.
#include "row_quant.hpp"

namespace w4a8 {

// The binary64 sum over the wave (all 64 lanes active).
__device__ __forceinline__ double wave_sum_f64(double v)
{
    auto dpp = [](double x, auto ctrl) {
        const int lo = dpp_i32<decltype(ctrl)::value>(__double2loint(x)), hi = dpp_i32<decltype(ctrl)::value>(__double2hiint(x));
        return __hiloint2double(hi, lo);
    };
    auto lane = [](double x, int l) {
        return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), l), __builtin_amdgcn_readlane(__double2loint(x), l));
    };
    v += dpp(v, std::integral_constant<int, DPP_QUAD_XOR1>());
    v += dpp(v, std::integral_constant<int, DPP_QUAD_XOR2>());
    v += dpp(v, std::integral_constant<int, DPP_ROW_HALF_MIRROR>());
    v += dpp(v, std::integral_constant<int, DPP_ROW_MIRROR>());
    return (lane(v, 0) + lane(v, 16)) + (lane(v, 32) + lane(v, 48));
}

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ bf16_t from_f32<bf16_t>(float v) { return bf16_t{f32_to_bf16_bits(v)}; }

struct NormArgs {
    const void *x, *r, *w;   // r null: nothing is added
    const float *s;          // null: 1
    void *h;                 // null: the sum is not kept (given where r is)
    int8_t *q;
    float *sx;
    int64_t M, ldx, ldr, ldh;
    int K, w_f32;            // w_f32: w is binary32 rather than of the row's type
    double eps;
};

// 127 / a, 0 for a row that counts as all-zero, and the row's scale
__device__ __forceinline__ float row_inverse(float a)
{
    const float inv = 127.0f / a;
    return inv <= AQ_FLT_MAX ? inv : 0.0f;
}
__device__ __forceinline__ float row_scale(float a, float inv, double squares, const NormArgs &p)
{
    if (inv == 0.0f) return 1.0f;
    return (float)((double)a / sqrt(squares / p.K + p.eps) / 127.0);
}

template <typename T>
__device__ __forceinline__ float norm_gain(const NormArgs &p, int k)
{
    const float w = p.w_f32 ? ((const float *)p.w)[k] : to_f32(((const T *)p.w)[k]);
    return p.s ? w * (1.0f / p.s[k]) : w;
}

// Any width, alignment and row distance: a workgroup per row, one element at a time, the row read twice (the second time the
// sum as it was kept, so that h may lie on x or r).
template <typename T>
__global__ __launch_bounds__(256) void norm_quant_generic_kernel(NormArgs p)
{
    __shared__ float red[4];
    __shared__ double red2[4];
    const int64_t m = blockIdx.x;
    const T *x = (const T *)p.x + m * p.ldx, *r = (const T *)p.r + m * p.ldr;
    T *h = (T *)p.h + m * p.ldh;
    float a = 0.0f;
    double ss = 0.0;
    for (int k = threadIdx.x; k < p.K; k += 256) {
        T v = x[k];
        if (p.r) {
            v = from_f32<T>(to_f32(v) + to_f32(r[k]));
            h[k] = v;
        }
        const float f = to_f32(v);
        ss += (double)f * (double)f;
        a = fmaxf(a, fabsf(f * norm_gain<T>(p, k)));
    }
    a = block_max<4>(a, red);
    ss = wave_sum_f64(ss);
    if ((threadIdx.x & 63) == 0) red2[threadIdx.x >> 6] = ss;
    __syncthreads();
    const float inv = row_inverse(a);
    if (threadIdx.x == 0) p.sx[m] = row_scale(a, inv, (red2[0] + red2[1]) + (red2[2] + red2[3]), p);
    const T *again = p.r ? h : x;
    for (int k = threadIdx.x; k < p.K; k += 256)
        p.q[m * (int64_t)p.K + k] = (int8_t)quant1_bits(to_f32(again[k]) * norm_gain<T>(p, k), inv);
}

template <typename T>
static int launch_norm_quant_t(const NormArgs &p, hipStream_t st)
{
    hipLaunchKernelGGL((norm_quant_generic_kernel<T>), dim3((unsigned)p.M), dim3(256), 0, st, p);
    return hip_status(hipGetLastError());
}

int launch_norm_quant(const void *X, int x_dtype, int64_t M, int64_t K, int64_t ldx, const void *R, int64_t ldr, const void *w,
                      int w_dtype, const float *s, double eps, void *H, int64_t ldh, int8_t *Xq, float *sx, hipStream_t st)
{
    const NormArgs p = {X, R, w, s, H, Xq, sx, M, ldx, ldr, ldh, (int)K, w_dtype == W4A8_F32, eps};
    switch (x_dtype) {
        case W4A8_F32: return launch_norm_quant_t<float>(p, st);
        case W4A8_F16: return launch_norm_quant_t<__half>(p, st);
        case W4A8_BF16: return launch_norm_quant_t<bf16_t>(p, st);
        default: return W4A8_ERR_DTYPE;
    }
}

}  // namespace w4a8
