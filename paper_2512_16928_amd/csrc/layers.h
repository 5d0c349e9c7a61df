// Launch interfaces and device helpers of the layer operators: a linear
// layer's three products, an activation's gradient, and layer norm.
//
// Layouts: W and G are the step's, row-major contiguous [rows][cols] =
// [fan-out][fan-in]. Activations are row-major [tokens][width] with a pitch
// (elements from one token's row to the next) of their own.
#pragma once

#include "dion2_device.h"

namespace dion2 {

enum Act { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_GELU_TANH = 3, ACT_SILU = 4 };

// -------------------------------------------------------------- activations
// Phi(x) = erfc(-x / sqrt 2) / 2 from erfc(u) = t e^{-u^2} P(t), t = 1 / (1 + 0.3 u),
// u >= 0, so neither tail cancels. P is a polynomial of degree 8 fitted here by
// weighted least squares (Lawson's iteration) to erfc(u) e^{u^2} / t for the
// smallest largest relative error on u <= 10, 2e-8. Evaluated in fp32 the result
// is within 1.5e-6 relative for |x| <= 4, 5e-6 for |x| <= 9 and 1e-5 for |x| <= 12
// (the rounding of x^2 grows through the exponential; beyond it is below 2e-33).
// The value is for -|x|, and with SLOPE that of Phi(x) + x phi(x) for it,
// which takes no second exponential: either is for x > 0 one less what it is there.
// FINE (fp32 calls), here and in logistic(): a division, where the reciprocal
// instruction is off by up to a unit of fp32's last place.
template <bool FINE, bool SLOPE>
__device__ __forceinline__ float normal_cdf(float x) {
    const float u = __builtin_fabsf(x);
    const float e = __builtin_amdgcn_exp2f(-0.72134752f * x * x);
    const float d = __builtin_fmaf(0.21213203f, u, 1.0f);   // 0.3 / sqrt 2
    const float t = FINE ? 1.0f / d : __builtin_amdgcn_rcpf(d);
    float p = -0.0647770372f;             // P's coefficients, halved
    p = __builtin_fmaf(p, t, 0.2428634512f);
    p = __builtin_fmaf(p, t, -0.2563233373f);
    p = __builtin_fmaf(p, t, 0.2740919430f);
    p = __builtin_fmaf(p, t, -0.0475035953f);
    p = __builtin_fmaf(p, t, 0.1075485246f);
    p = __builtin_fmaf(p, t, 0.0741446257f);
    p = __builtin_fmaf(p, t, 0.0853616619f);
    p = __builtin_fmaf(p, t, 0.0845937237f);
    const float h = (SLOPE ? __builtin_fmaf(p, t, -0.39894228f * u) : p * t) * e;
    return x > 0.0f ? 1.0f - h : h;
}

// 1 / (1 + e^-x)
template <bool FINE>
__device__ __forceinline__ float logistic(float x) {
    const float d = 1.0f + __builtin_amdgcn_exp2f(-1.44269504f * x);
    return FINE ? 1.0f / d : __builtin_amdgcn_rcpf(d);
}

// act(z). A NaN stays a NaN.
template <int ACT, bool FINE>
__device__ __forceinline__ float act_value(float z) {
    if constexpr (ACT == ACT_RELU) return z < 0.0f ? 0.0f : z;
    if constexpr (ACT == ACT_GELU) return z * normal_cdf<FINE, false>(z);
    // z (1 + tanh v) / 2 = z logistic(2 v), v = sqrt(2 / pi) (z + 0.044715 z^3)
    if constexpr (ACT == ACT_GELU_TANH) return z * logistic<FINE>(z * __builtin_fmaf(0.07135482f, z * z, 1.59576912f));
    if constexpr (ACT == ACT_SILU) return z * logistic<FINE>(z);
    return z;
}

// act'(z); for ReLU 0 at 0.
template <int ACT, bool FINE>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (ACT == ACT_RELU) return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
    if constexpr (ACT == ACT_GELU) return normal_cdf<FINE, true>(z);
    if constexpr (ACT == ACT_GELU_TANH) {
        const float s = logistic<FINE>(z * __builtin_fmaf(0.07135482f, z * z, 1.59576912f));
        // from |z| = 100 on s (1 - s) is 0, and z^2 must not become infinite beside it
        return __builtin_fmaf(z * s * (1.0f - s), __builtin_fmaf(0.21406445f, __builtin_fminf(z * z, 1e4f), 1.59576912f), s);
    }
    if constexpr (ACT == ACT_SILU) {
        const float s = logistic<FINE>(z);
        return s * __builtin_fmaf(z, 1.0f - s, 1.0f);
    }
    return 1.0f;
}

// f with the activation as a compile-time constant: one uniform branch for
// all the entries that f handles.
template <int A> struct ActIs { static constexpr int value = A; };
template <typename F>
__host__ __device__ __forceinline__ void with_act(int act, F&& f) {
    switch (act) {
        case ACT_RELU: f(ActIs<ACT_RELU>{}); break;
        case ACT_GELU: f(ActIs<ACT_GELU>{}); break;
        case ACT_GELU_TANH: f(ActIs<ACT_GELU_TANH>{}); break;
        case ACT_SILU: f(ActIs<ACT_SILU>{}); break;
        default: f(ActIs<ACT_NONE>{}); break;
    }
}

// ------------------------------------------------- eight consecutive entries
// of a row, of which the first n exist (the others read as zero and are not
// written); any alignment of whole elements.
__device__ __forceinline__ void unpack8(const uint4& x, float (&v)[8]) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const uint16_t* p, int n, float (&v)[8]) {
    if (n >= 8) {
        unpack8(ldg<uint4>(p), v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? bf16_bits_to_f32(ldg<uint16_t>(p + i)) : 0.0f;
    }
}
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8]) {
    if (n >= 8) {
        const float4 a = ldg<float4>(p), b = ldg<float4>(p + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? ldg<float>(p + i) : 0.0f;
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float x, float y) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    const bf16x2 v = {(__bf16)x, (__bf16)y};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ void store8(uint16_t* p, int n, const float (&v)[8]) {
    if (n >= 8) {
        stg(p, make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) stg(p + i, f32_to_bf16(v[i]));
    }
}
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
    if (n >= 8) {
        stg(p, make_float4(v[0], v[1], v[2], v[3]));
        stg(p + 4, make_float4(v[4], v[5], v[6], v[7]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) stg(p + i, v[i]);
    }
}
// the same from (to) a pointer whose type a flag gives
__device__ __forceinline__ void load8_as(const void* p, int64_t at, bool bf16, int n, float (&v)[8]) {
    if (bf16) load8(static_cast<const uint16_t*>(p) + at, n, v);
    else load8(static_cast<const float*>(p) + at, n, v);
}
__device__ __forceinline__ void store8_as(void* p, int64_t at, bool bf16, int n, const float (&v)[8]) {
    if (bf16) store8(static_cast<uint16_t*>(p) + at, n, v);
    else store8(static_cast<float*>(p) + at, n, v);
}

// ---------------------------------------------------------------- products
// C[m][n] = sum_k A(m, k) B(n, k), m < M, n < N, k < K.
//   PROD_FORWARD  A = X [M][K], B = W [N][K]; z = C + bias[n]; Z = z where set;
//                 out = act(z) + R
//   PROD_INPUT    A = dY [M][K], B(n, k) = W[k][n]; out = C act'(Z)
//   PROD_WEIGHT   A(m, k) = dY[k][m], B(n, k) = X[k][n]; out = C, or out + C
//                 (accumulate), in the gradients' type
enum Product { PROD_FORWARD = 0, PROD_INPUT = 1, PROD_WEIGHT = 2 };
struct ProductArgs {
    const void* A;
    const void* B;
    int64_t lda, ldb;   // elements between consecutive rows as stored
    int64_t M, N, K;
    void* out;
    int64_t ldo;
    const void* bias;   // nullable
    const void* R;      // nullable; [M][N], pitch ldr
    int64_t ldr;
    void* Z;            // nullable; written by PROD_FORWARD, read by PROD_INPUT
    int64_t ldz;
    int act;
    int bf16;           // type of A, B, R, Z and (PROD_FORWARD, PROD_INPUT) out
    int bias_bf16;
    int out_bf16;       // type of PROD_WEIGHT's out
    int accumulate;
    float* part;        // product_workspace bytes, 256-byte aligned: copies, partial sums
    int splits;         // set by launch_product
    float* row_sums;    // nullable, PROD_WEIGHT: [product_row_sums(a)][M], partial sums
                        // over k of A's rows (the bias gradient's)
};
// How many rows of row_sums PROD_WEIGHT gives; 0 where its form gives none.
int64_t product_row_sums(const ProductArgs& a);
// Bytes of workspace of this call without row_sums, and the most of any call of
// these sizes and pitches, with them.
size_t product_workspace(Product kind, const ProductArgs& a);
size_t product_workspace_most(Product kind, ProductArgs a);
hipError_t launch_product(Product kind, ProductArgs a, hipStream_t s);

// -------------------------------------------------------- streaming passes
struct ActGradArgs {
    const void* dY;
    const void* Z;
    void* dZ;
    int64_t ldy, ldz, ldo;
    int64_t tokens, width;
    int act, bf16;
};
hipError_t launch_act_grad(const ActGradArgs& a, hipStream_t s);

// out[j] (+)= sum_t X[t][j]: partial sums of row blocks, then those in order.
struct ColSumArgs {
    const void* X;
    int64_t ldx, tokens, width;
    int bf16;
    float* part;        // [blocks][width]
    int64_t blocks;     // col_sum_blocks(tokens, width)
    void* out;
    int out_bf16, accumulate;
};
int64_t col_sum_blocks(int64_t tokens, int64_t width);
hipError_t launch_col_sum(const ColSumArgs& a, hipStream_t s);
// The second half alone: out from part [blocks][width].
hipError_t launch_col_join(const ColSumArgs& a, hipStream_t s);

struct NormArgs {
    const void* X;
    const void* gamma;  // nullable (1)
    const void* beta;   // nullable (0)
    void* Y;
    float* mean;        // nullable
    float* rstd;        // nullable
    int64_t ldx, ldy, tokens, cols;
    float eps;
    int bf16, p_bf16;
};
hipError_t launch_norm(const NormArgs& a, hipStream_t s);

struct NormGradArgs {
    const void* dY;
    const void* X;
    const float* mean;
    const float* rstd;
    const void* gamma;  // nullable (1)
    const void* dR;     // nullable: added to dX
    void* dX;           // nullable
    void* dgamma;       // nullable
    void* dbeta;        // nullable
    int64_t lddy, ldx, lddr, lddx, tokens, cols;
    int bf16, p_bf16, g_bf16, accumulate;
    float* part;        // [blocks][2][cols], where dgamma or dbeta is set
    int64_t blocks;     // norm_grad_blocks(...)
    int64_t run;        // rows a block; set by launch_norm_grad
};
int64_t norm_grad_blocks(int64_t tokens, int64_t cols, int bf16);
hipError_t launch_norm_grad(NormGradArgs a, hipStream_t s);

}  // namespace dion2
