// Streaming passes of the layers: layer norm forward and backward, column
// sums (bias gradients) and an activation's gradient.
//
//   y  = (x - mean) rstd gamma + beta,  rstd = 1 / sqrt(var + eps)
//   dx = rstd (h - mean(h) - xh mean(h xh)) + dR,  h = dy gamma,  xh = (x - mean) rstd
//   dgamma = sum_t dy xh,  dbeta = sum_t dy
#include <algorithm>
#include <type_traits>

#include "layers.h"

namespace dion2 {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
// Sum over the block in every thread; `red` holds one float a wave.
__device__ __forceinline__ float block_sum(float v, float* red) {
    v = wave_sum(v);
    __syncthreads();   // red's last use is over
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) s += red[w];
    return s;
}

__device__ __forceinline__ int part8(int64_t n, int64_t at) { return n - at < 8 ? (int)(n - at) : 8; }

// One block a row, the row read once per pass.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_rows(NormArgs a) {
    __shared__ float red[kThreads / 64];
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const T* x = static_cast<const T*>(a.X) + t * a.ldx;
        T* y = static_cast<T*>(a.Y) + t * a.ldy;
        float v[8], s = 0.0f;
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            load8(x + c, part8(a.cols, c), v);
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
        const float n = (float)a.cols;
        float mean = block_sum(s, red) / n;
        // the deviations' own mean takes up what rounding left of the mean
        float d1 = 0.0f, d2 = 0.0f;
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            const int k = part8(a.cols, c);
            load8(x + c, k, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = i < k ? v[i] - mean : 0.0f;
                d1 += d;
                d2 += d * d;
            }
        }
        const float off = block_sum(d1, red) / n;
        const float rstd = 1.0f / sqrtf(block_sum(d2, red) / n - off * off + a.eps);
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            const int k = part8(a.cols, c);
            float g[8], b[8];
            load8(x + c, k, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (v[i] - mean - off) * rstd;
            if (a.gamma) {
                load8_as(a.gamma, c, a.p_bf16, k, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= g[i];
            }
            if (a.beta) {
                load8_as(a.beta, c, a.p_bf16, k, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += b[i];
            }
            store8(y + c, k, v);
        }
        if (threadIdx.x == 0) {
            if (a.mean) stg(a.mean + t, mean + off);
            if (a.rstd) stg(a.rstd + t, rstd);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void norm_grad_rows(NormGradArgs a) {
    __shared__ float red[kThreads / 64];
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const T* x = static_cast<const T*>(a.X) + t * a.ldx;
        const T* dy = static_cast<const T*>(a.dY) + t * a.lddy;
        const T* dr = a.dR ? static_cast<const T*>(a.dR) + t * a.lddr : nullptr;
        T* dx = static_cast<T*>(a.dX) + t * a.lddx;
        const float mean = ldg<float>(a.mean + t), rstd = ldg<float>(a.rstd + t);
        float h[8], xh[8], g[8], s1 = 0.0f, s2 = 0.0f;
        auto load = [&](int64_t c, int k) {
            load8(dy + c, k, h);
            load8(x + c, k, xh);
            if (a.gamma) {
                load8_as(a.gamma, c, a.p_bf16, k, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[i] *= g[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) xh[i] = (xh[i] - mean) * rstd;
        };
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            const int k = part8(a.cols, c);
            load(c, k);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < k) {
                    s1 += h[i];
                    s2 += h[i] * xh[i];
                }
        }
        s1 = block_sum(s1, red) / (float)a.cols;
        s2 = block_sum(s2, red) / (float)a.cols;
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            const int k = part8(a.cols, c);
            load(c, k);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = rstd * (h[i] - s1 - xh[i] * s2);
            if (dr) {
                load8(dr + c, k, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[i] += g[i];
            }
            store8(dx + c, k, h);
        }
    }
}

// Column sums over row blocks: a block takes kColW columns and one row block;
// its eight groups of 32 threads take every eighth row.
constexpr int kColW = 256;
constexpr int kGroups = kThreads / 32;

// partial sums of X (MODE 0), or of dY xh and dY (MODE 1)
template <typename T, int MODE, typename Args>
__global__ __launch_bounds__(kThreads) void col_parts(Args a, int64_t width) {
    __shared__ float lds[kGroups][kColW];
    const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * kColW + lane * 8;
    const int k = c < width ? part8(width, c) : 0;
    const int64_t t0 = a.tokens * blockIdx.y / a.blocks, t1 = a.tokens * (blockIdx.y + 1) / a.blocks;
    float s0[8] = {}, s1[8] = {};
    if (k > 0) {
        for (int64_t t = t0 + grp; t < t1; t += kGroups) {
            float v[8];
            if constexpr (MODE == 0) {
                load8(static_cast<const T*>(a.X) + t * a.ldx + c, k, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) s0[i] += v[i];
            } else {
                float x[8];
                load8(static_cast<const T*>(a.dY) + t * a.lddy + c, k, v);
                load8(static_cast<const T*>(a.X) + t * a.ldx + c, k, x);
                const float mean = ldg<float>(a.mean + t), rstd = ldg<float>(a.rstd + t);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s0[i] += v[i] * ((x[i] - mean) * rstd);
                    s1[i] += v[i];
                }
            }
        }
    }
#pragma unroll
    for (int m = 0; m <= MODE; ++m) {
#pragma unroll
        for (int i = 0; i < 8; ++i) lds[grp][lane * 8 + i] = m ? s1[i] : s0[i];
        __syncthreads();
        const int64_t j = (int64_t)blockIdx.x * kColW + threadIdx.x;
        if (j < width) {
            float s = 0.0f;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) s += lds[g][threadIdx.x];
            stg(a.part + ((int64_t)blockIdx.y * (MODE + 1) + m) * width + j, s);
        }
        __syncthreads();
    }
}

// out[j] (+)= sum over blocks of part[b * step + j], in order of b
__global__ __launch_bounds__(kThreads) void col_join(const float* part, int64_t blocks, int64_t step, int64_t width,
                                                     void* out, int out_bf16, int accumulate) {
    const int64_t j = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (j >= width) return;
    float s = 0.0f;
    for (int64_t b = 0; b < blocks; ++b) s += ldg<float>(part + b * step + j);
    if (out_bf16) {
        uint16_t* o = static_cast<uint16_t*>(out) + j;
        if (accumulate) s += bf16_bits_to_f32(ldg<uint16_t>(o));
        stg(o, f32_to_bf16(s));
    } else {
        float* o = static_cast<float*>(out) + j;
        if (accumulate) s += ldg<float>(o);
        stg(o, s);
    }
}

hipError_t join(const float* part, int64_t blocks, int64_t step, int64_t width, void* out, int out_bf16, int accumulate,
                hipStream_t s) {
    col_join<<<(unsigned)((width + kThreads - 1) / kThreads), kThreads, 0, s>>>(part, blocks, step, width, out, out_bf16,
                                                                               accumulate);
    return hipGetLastError();
}

template <int ACT, typename T>
__global__ __launch_bounds__(kThreads) void act_grad(ActGradArgs a) {
    constexpr bool FINE = std::is_same<T, float>::value;
    const int64_t chunks = (a.width + 7) / 8, total = a.tokens * chunks;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t t = i / chunks, c = i % chunks * 8;
        const int k = part8(a.width, c);
        float dy[8], z[8];
        load8(static_cast<const T*>(a.dY) + t * a.ldy + c, k, dy);
        load8(static_cast<const T*>(a.Z) + t * a.ldz + c, k, z);
#pragma unroll
        for (int j = 0; j < 8; ++j) dy[j] *= act_slope<ACT, FINE>(z[j]);
        store8(static_cast<T*>(a.dZ) + t * a.ldo + c, k, dy);
    }
}

unsigned row_grid(int64_t tokens) { return (unsigned)std::min<int64_t>(tokens, 1 << 16); }

}  // namespace

int64_t col_sum_blocks(int64_t tokens, int64_t width) {
    const int64_t strips = (width + kColW - 1) / kColW;
    return std::max<int64_t>(1, std::min<int64_t>((tokens + 63) / 64, std::max<int64_t>(1, 1024 / strips)));
}
int64_t norm_grad_blocks(int64_t tokens, int64_t cols) { return col_sum_blocks(tokens, cols); }

hipError_t launch_col_sum(const ColSumArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.width + kColW - 1) / kColW), (unsigned)a.blocks);
    if (a.bf16) col_parts<uint16_t, 0><<<grid, kThreads, 0, s>>>(a, a.width);
    else col_parts<float, 0><<<grid, kThreads, 0, s>>>(a, a.width);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return join(a.part, a.blocks, a.width, a.width, a.out, a.out_bf16, a.accumulate, s);
}

hipError_t launch_act_grad(const ActGradArgs& a, hipStream_t s) {
    if (a.tokens == 0) return hipSuccess;
    const int64_t chunks = a.tokens * ((a.width + 7) / 8);
    const unsigned grid = (unsigned)std::min<int64_t>((chunks + kThreads - 1) / kThreads, 8192);
    auto launch = [&](auto act) {
        if (a.bf16) act_grad<decltype(act)::value, uint16_t><<<grid, kThreads, 0, s>>>(a);
        else act_grad<decltype(act)::value, float><<<grid, kThreads, 0, s>>>(a);
    };
    with_act(a.act, launch);
    return hipGetLastError();
}

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
    if (a.tokens == 0) return hipSuccess;
    if (a.bf16) norm_rows<uint16_t><<<row_grid(a.tokens), kThreads, 0, s>>>(a);
    else norm_rows<float><<<row_grid(a.tokens), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_norm_grad(const NormGradArgs& a, hipStream_t s) {
    hipError_t e = hipSuccess;
    // the parameters' sums first: dX may be dY's own storage
    if (a.dgamma || a.dbeta) {
        const dim3 grid((unsigned)((a.cols + kColW - 1) / kColW), (unsigned)a.blocks);
        if (a.bf16) col_parts<uint16_t, 1><<<grid, kThreads, 0, s>>>(a, a.cols);
        else col_parts<float, 1><<<grid, kThreads, 0, s>>>(a, a.cols);
        e = hipGetLastError();
        if (e == hipSuccess && a.dgamma)
            e = join(a.part, a.blocks, 2 * a.cols, a.cols, a.dgamma, a.g_bf16, a.accumulate, s);
        if (e == hipSuccess && a.dbeta)
            e = join(a.part + a.cols, a.blocks, 2 * a.cols, a.cols, a.dbeta, a.g_bf16, a.accumulate, s);
    }
    if (e == hipSuccess && a.dX && a.tokens) {
        if (a.bf16) norm_grad_rows<uint16_t><<<row_grid(a.tokens), kThreads, 0, s>>>(a);
        else norm_grad_rows<float><<<row_grid(a.tokens), kThreads, 0, s>>>(a);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace dion2
