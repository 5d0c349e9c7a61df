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

template <typename V>
__device__ __forceinline__ V wave_sum(V v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
// Sum over the waves of a block in every thread; `red` holds one value a wave.
// Calls in turn use two of them in turn, so one barrier a call is enough.
template <int WAVES, typename V>
__device__ __forceinline__ V block_sum(V v, V* red) {
    v = wave_sum(v);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += red[w];
    }
    return v;
}

// A row's mean, summed in 64 bits, as the nearest float and what that leaves: a
// mean many times the row's spread then costs its deviations nothing, and what is
// stored is the mean rounded once. (Deviations from a rounded mean, summed in 32
// bits to correct it, round alike wherever the entries have few bits: on rows of
// bf16 that mean was off by up to 1.8e-6 relative where a plain sum has 5e-8.)
struct Mean {
    float mean, off;
    __device__ __forceinline__ Mean(double sum, int64_t cols) {
        const double m = sum / (double)cols;
        mean = (float)m;
        off = __builtin_isfinite(mean) ? (float)(m - (double)mean) : 0.0f;
    }
};

__device__ __forceinline__ int part8(int64_t n, int64_t at) { return n - at < 8 ? (int)(n - at) : 8; }

// ---- rows held in registers
// WPR waves take a row, CH chunks of eight entries a lane: rows of at most 512
// WPR CH entries, read once. The entries stay as they are stored (4 or 8
// registers a chunk) and are widened where they are used. RAGGED: the length
// is no multiple of 8.
template <typename T> struct Raw;
template <> struct Raw<uint16_t> {
    uint4 v;
    template <bool NT = false>
    __device__ __forceinline__ void load(const uint16_t* p) { v = NT ? ldg_nt<uint4>(p) : ldg<uint4>(p); }
    __device__ __forceinline__ void get(float (&x)[8]) const { unpack8(v, x); }
    // the first k entries dropped, zeros behind the others
    __device__ __forceinline__ void drop(int k) {
        const uint64_t lo = (uint64_t)v.y << 32 | v.x, hi = (uint64_t)v.w << 32 | v.z;
        const int b = 16 * (k & 3);
        const uint64_t carry = b ? hi << (64 - b) : 0;
        const uint64_t l = k < 4 ? lo >> b | carry : k < 8 ? hi >> b : 0, h = k < 4 ? hi >> b : 0;
        v = make_uint4((uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32));
    }
    __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
    // what was widened before is not kept
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w)); }
};
template <> struct Raw<float> {
    float4 a, b;
    template <bool NT = false>
    __device__ __forceinline__ void load(const float* p) {
        a = NT ? ldg_nt<float4>(p) : ldg<float4>(p);
        b = NT ? ldg_nt<float4>(p + 4) : ldg<float4>(p + 4);
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
    __device__ __forceinline__ void drop(int k) {
        float x[8];
        get(x);
#pragma unroll
        for (int s = 4; s; s >>= 1)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = i + s < 8 ? x[(i + s) & 7] : 0.0f;
                x[i] = k & s ? y : x[i];
            }
        a = make_float4(x[0], x[1], x[2], x[3]);
        b = make_float4(x[4], x[5], x[6], x[7]);
    }
    __device__ __forceinline__ void zero() { a = b = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
    __device__ __forceinline__ void forget() {}
};

template <typename T, int WPR, int CH, bool RAGGED>
struct Row {
    Raw<T> raw[CH];
    // first column of chunk i, and how many of its entries exist
    __device__ __forceinline__ static int col(int i) { return ((i * WPR + threadIdx.x / 64 % WPR) * 64 + (threadIdx.x & 63)) * 8; }
    __device__ __forceinline__ static int have(int i, int cols) {
        const int n = cols - col(i);
        return RAGGED ? (n < 0 ? 0 : n < 8 ? n : 8) : (n > 0 ? 8 : 0);
    }
    template <bool NT = false>
    __device__ __forceinline__ void load(const T* p, int cols) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if constexpr (RAGGED) {
                // a row's last chunk is read as its last eight entries (rows of
                // eight at least), of which the first ones belong to the chunk before
                const int past = col(i) + 8 - cols;
                if (past < 8) {
                    raw[i].template load<NT>(p + (past > 0 ? cols - 8 : col(i)));
                    if (past > 0) raw[i].drop(past);
                } else {
                    raw[i].zero();
                }
            } else {
                if (col(i) < cols) raw[i].template load<NT>(p + col(i));
                else raw[i].zero();
            }
        }
    }
};

// Sums over a row's waves, in every lane. red holds 2 floats for each of the
// block's waves, twice: alternate calls use alternate halves, so one barrier
// a call is enough.
template <int WPR>
__device__ __forceinline__ void row_sums(float& a, float& b, float* red, int& turn) {
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        a += __shfl_xor(a, d);
        b += __shfl_xor(b, d);
    }
    if constexpr (WPR > 1) {
        float* r = red + turn * 2 * WPR;
        turn ^= 1;
        const int w = threadIdx.x / 64;
        if ((threadIdx.x & 63) == 0) {
            r[2 * w] = a;
            r[2 * w + 1] = b;
        }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int i = 0; i < WPR; ++i) {
            a += r[2 * i];
            b += r[2 * i + 1];
        }
    }
}

// a block's waves: one row's, or those of four rows of a wave each
constexpr int row_waves(int wpr) { return wpr > 1 ? wpr : 4; }

template <typename T, int WPR, int CH, bool RAGGED>
__global__ __launch_bounds__(64 * row_waves(WPR)) void norm_regs(NormArgs a) {
    using R = Row<T, WPR, CH, RAGGED>;
    constexpr int RPB = row_waves(WPR) / WPR;   // rows a block
    __shared__ double red[WPR];
    __shared__ float red2[WPR];
    const int cols = (int)a.cols;
    const float inv = 1.0f / (float)cols;
    // a row a wave, or a block; the grid has a second dimension because a
    // launch's threads fit 32 bits in each
    const int64_t t = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * RPB + threadIdx.x / 64 / WPR;
    if (t >= a.tokens) return;   // whole waves, or the whole block
    R x;
    x.load(static_cast<const T*>(a.X) + t * a.ldx, cols);
    double sum = 0.0;
    float v[8];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        x.raw[i].get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += (double)v[j];
    }
    const Mean m(block_sum<WPR>(sum, red), cols);
    float d2 = 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int n = R::have(i, cols);
        x.raw[i].get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) {
                const float d = v[j] - m.mean - m.off;
                d2 += d * d;
            }
    }
    const float rstd = 1.0f / sqrtf(block_sum<WPR>(d2, red2) * inv + a.eps);
    T* y = static_cast<T*>(a.Y) + t * a.ldy;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int n = R::have(i, cols), c = R::col(i);
        if (n == 0) continue;
        float g[8];
        x.raw[i].get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (v[j] - m.mean - m.off) * rstd;
        if (a.gamma) {
            load8_as(a.gamma, c, a.p_bf16, RAGGED ? n : 8, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= g[j];
        }
        if (a.beta) {
            load8_as(a.beta, c, a.p_bf16, RAGGED ? n : 8, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += g[j];
        }
        store8(y + c, RAGGED ? n : 8, v);
    }
    if ((threadIdx.x & 63) == 0 && threadIdx.x / 64 % WPR == 0) {
        if (a.mean) stg(a.mean + t, m.mean);
        if (a.rstd) stg(a.rstd + t, rstd);
    }
}

// The gradient: a block's waves (four, or the WPR of one row) walk down a run
// of rows with the sums of dgamma and dbeta of their own columns in registers;
// they leave the block as one row of partial sums. gamma is kept in LDS in
// fp32 (ones where there is none).
template <typename T, int WPR, int CH, bool RAGGED>
__global__ __launch_bounds__(64 * row_waves(WPR), 4) void norm_grad_regs(NormGradArgs a) {
    using R = Row<T, WPR, CH, RAGGED>;
    constexpr int WAVES = row_waves(WPR), RPB = WAVES / WPR;   // rows at a time
    __shared__ float red[4 * WAVES];
    extern __shared__ __align__(16) float lds[];                // gamma, and where RPB > 1 the sums
    const int cols = (int)a.cols, wave = threadIdx.x / 64;
    const float inv = 1.0f / (float)cols;
    const int padded = (cols + 7) & ~7;
    for (int c = threadIdx.x; c < padded; c += 64 * WAVES) {
        float g = 1.0f;
        if (a.gamma && c < cols)
            g = a.p_bf16 ? bf16_bits_to_f32(ldg<uint16_t>(static_cast<const uint16_t*>(a.gamma) + c))
                         : ldg<float>(static_cast<const float*>(a.gamma) + c);
        lds[c] = g;
    }
    __syncthreads();
    int turn = 0;
    float sg[CH][8], sb[CH][8];
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) sg[i][j] = sb[i][j] = 0.0f;
    const int64_t t0 = (int64_t)blockIdx.x * a.run;
    const int64_t t1 = t0 + a.run < a.tokens ? t0 + a.run : a.tokens;
    // a row's entries are requested while the row before it is worked on; X and
    // dR, written long before and not read again, past the caches (all three
    // inputs out of HBM, 16384 x 2048: 67 -> 64 us)
    R dy_next, x_next;
    auto request = [&](int64_t t) {
        dy_next.load(static_cast<const T*>(a.dY) + t * a.lddy, cols);
        x_next.template load<true>(static_cast<const T*>(a.X) + t * a.ldx, cols);
    };
    const int64_t first = t0 + wave / WPR;
    if (first < t1) request(first);
    for (int64_t t = first; t < t1; t += RPB) {   // WPR > 1 fills the block: all its waves see the same t
        R dy = dy_next, x = x_next, dr;
        if (a.dR) dr.template load<true>(static_cast<const T*>(a.dR) + t * a.lddr, cols);
        if (t + RPB < t1) request(t + RPB);
        const float mean = ldg<float>(a.mean + t), rstd = ldg<float>(a.rstd + t);
        float s1 = 0.0f, s2 = 0.0f, h[8], xh[8], g[8];
        auto get = [&](int i) {   // dy and xh; gamma
            dy.raw[i].get(h);
            x.raw[i].get(xh);
#pragma unroll
            for (int j = 0; j < 8; ++j) xh[j] = (xh[j] - mean) * rstd;
            const float4* p = reinterpret_cast<const float4*>(lds + R::col(i));
            const float4 lo = p[0], hi = p[1];
            g[0] = lo.x; g[1] = lo.y; g[2] = lo.z; g[3] = lo.w;
            g[4] = hi.x; g[5] = hi.y; g[6] = hi.z; g[7] = hi.w;
        };
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int n = R::have(i, cols);
            if (n == 0) continue;
            get(i);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // entries past the row's end: dy is 0 and xh of no meaning
                const float p = RAGGED && j >= n ? 0.0f : h[j] * xh[j];
                sg[i][j] += p;
                sb[i][j] += h[j];
                s1 = __builtin_fmaf(h[j], g[j], s1);
                s2 = __builtin_fmaf(p, g[j], s2);
            }
        }
        if (!a.dX) continue;
        row_sums<WPR>(s1, s2, red, turn);
        s1 *= inv;
        s2 *= inv;
        T* dx = static_cast<T*>(a.dX) + t * a.lddx;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int n = R::have(i, cols), c = R::col(i);
            if (n == 0) continue;
            dy.raw[i].forget();
            x.raw[i].forget();
            get(i);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = rstd * (h[j] * g[j] - s1 - xh[j] * s2);
            if (a.dR) {
                dr.raw[i].get(g);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[j] += g[j];
            }
            store8(dx + c, RAGGED ? n : 8, h);
        }
    }
    if (!a.part) return;
    float* part = a.part + (int64_t)blockIdx.x * 2 * cols;
    if constexpr (RPB == 1) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int n = R::have(i, cols), c = R::col(i);
            if (n == 0) continue;
            store8(part + c, RAGGED ? n : 8, sg[i]);
            store8(part + cols + c, RAGGED ? n : 8, sb[i]);
        }
    } else {
        // the waves' sums, one wave after the other
        float* sums = lds + padded;
#pragma unroll 1
        for (int w = 0; w < RPB; ++w) {
            if (wave == w) {
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const int n = R::have(i, cols), c = R::col(i);
                    if (n == 0) continue;
                    float4* p = reinterpret_cast<float4*>(sums + c);
                    float4* q = reinterpret_cast<float4*>(sums + padded + c);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float4 u = make_float4(sg[i][4 * k], sg[i][4 * k + 1], sg[i][4 * k + 2], sg[i][4 * k + 3]);
                        float4 v = make_float4(sb[i][4 * k], sb[i][4 * k + 1], sb[i][4 * k + 2], sb[i][4 * k + 3]);
                        if (w) {
                            const float4 x = p[k], y = q[k];
                            u.x += x.x; u.y += x.y; u.z += x.z; u.w += x.w;
                            v.x += y.x; v.y += y.y; v.z += y.z; v.w += y.w;
                        }
                        p[k] = u;
                        q[k] = v;
                    }
                }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < cols; c += 64 * WAVES) {
            stg(part + c, sums[c]);
            stg(part + cols + c, sums[padded + c]);
        }
    }
}

// ---- rows of any length
// One block a row, the row read once per pass.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_rows(NormArgs a) {
    __shared__ double red[kThreads / 64];
    __shared__ float red2[kThreads / 64];
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const T* x = static_cast<const T*>(a.X) + t * a.ldx;
        T* y = static_cast<T*>(a.Y) + t * a.ldy;
        float v[8];
        double sum = 0.0;
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            load8(x + c, part8(a.cols, c), v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += (double)v[i];
        }
        const Mean m(block_sum<kThreads / 64>(sum, red), a.cols);
        float d2 = 0.0f;
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            const int k = part8(a.cols, c);
            load8(x + c, k, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = i < k ? v[i] - m.mean - m.off : 0.0f;
                d2 += d * d;
            }
        }
        const float rstd = 1.0f / sqrtf(block_sum<kThreads / 64>(d2, red2) / (float)a.cols + a.eps);
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
            const int k = part8(a.cols, c);
            float g[8];
            load8(x + c, k, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (v[i] - m.mean - m.off) * rstd;
            if (a.gamma) {
                load8_as(a.gamma, c, a.p_bf16, k, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= g[i];
            }
            if (a.beta) {
                load8_as(a.beta, c, a.p_bf16, k, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += g[i];
            }
            store8(y + c, k, v);
        }
        if (threadIdx.x == 0) {
            if (a.mean) stg(a.mean + t, m.mean);
            if (a.rstd) stg(a.rstd + t, rstd);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void norm_grad_rows(NormGradArgs a) {
    __shared__ float red[2][kThreads / 64];
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
        s1 = block_sum<kThreads / 64>(s1, red[0]) / (float)a.cols;
        s2 = block_sum<kThreads / 64>(s2, red[1]) / (float)a.cols;
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

// out[j] (+)= sum over blocks of part[b * step + j]: a block takes 64 columns,
// each of its sixteen waves a run of the partial sums, then those in order.
// Columns from `split` on belong to out2.
constexpr int kJoinWaves = 16;
struct JoinArgs {
    const float* part;
    int64_t blocks, step, width, split;
    void* out;
    void* out2;
    int out_bf16, accumulate;
};
__global__ __launch_bounds__(64 * kJoinWaves) void col_join(JoinArgs a) {
    __shared__ float lds[kJoinWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t j = (int64_t)blockIdx.x * 64 + lane;
    const int64_t b0 = a.blocks * wave / kJoinWaves, b1 = a.blocks * (wave + 1) / kJoinWaves;
    float s = 0.0f;
    if (j < a.width) {
#pragma unroll 8
        for (int64_t b = b0; b < b1; ++b) s += ldg<float>(a.part + b * a.step + j);
    }
    lds[wave][lane] = s;
    __syncthreads();
    if (wave || j >= a.width) return;
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinWaves; ++w) s += lds[w][lane];
    void* out = j < a.split ? a.out : a.out2;
    const int64_t at = j < a.split ? j : j - a.split;
    if (!out) return;
    if (a.out_bf16) {
        uint16_t* o = static_cast<uint16_t*>(out) + at;
        if (a.accumulate) s += bf16_bits_to_f32(ldg<uint16_t>(o));
        stg(o, f32_to_bf16(s));
    } else {
        float* o = static_cast<float*>(out) + at;
        if (a.accumulate) s += ldg<float>(o);
        stg(o, s);
    }
}

hipError_t join(const JoinArgs& a, hipStream_t s) {
    col_join<<<(unsigned)((a.width + 63) / 64), 64 * kJoinWaves, 0, s>>>(a);
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

// The register forms by row length. WPR 0: none, the row is too long.
template <typename T_, int WPR_, int CH_, bool RAGGED_>
struct RowForm {
    using T = T_;
    static constexpr int WPR = WPR_, CH = CH_;
    static constexpr bool RAGGED = RAGGED_;
};
template <typename T, int WPR, int CH, typename F>
hipError_t with_ragged(int64_t cols, F&& f) {
    return cols % 8 ? f(RowForm<T, WPR, CH, true>{}) : f(RowForm<T, WPR, CH, false>{});
}
// Few rows leave most of the chip idle, so four waves share each (one row of
// 2048: a lane then has one chunk to wait for instead of four).
constexpr int64_t kFewRows = 1024;
template <typename T, typename F>
hipError_t with_row_of(int64_t cols, bool few, F&& f) {
    if (cols < 8) return f(RowForm<T, 0, 0, true>{});
    if (!few) {
        if (cols <= 512) return with_ragged<T, 1, 1>(cols, f);
        if (cols <= 1024) return with_ragged<T, 1, 2>(cols, f);
        if (cols <= 2048) return with_ragged<T, 1, 4>(cols, f);
    }
    if (cols <= 2048) return with_ragged<T, 4, 1>(cols, f);
    if (cols <= 4096) return with_ragged<T, 4, 2>(cols, f);
    if (cols <= 8192) return with_ragged<T, 8, 2>(cols, f);
    if (cols <= 16384) return with_ragged<T, 16, 2>(cols, f);
    return f(RowForm<T, 0, 0, true>{});
}
template <typename F>
hipError_t with_row(int bf16, int64_t cols, bool few, F&& f) {
    return bf16 ? with_row_of<uint16_t>(cols, few, f) : with_row_of<float>(cols, few, f);
}
// The gradient's: as many waves a row as leave a lane one chunk, sixteen at
// most, but one wave up to 1024 entries (512 in fp32): four rows' sums then
// leave the block as one.
bool grad_in_regs(int bf16, int64_t cols) { return cols >= 8 && cols <= (bf16 ? 16384 : 8192); }
int grad_wpr(int bf16, int64_t cols) {
    return cols <= 512 ? 1 : cols <= 1024 ? (bf16 ? 1 : 2) : cols <= 2048 ? 4 : cols <= 4096 ? 8 : 16;
}
template <typename T, typename F>
hipError_t with_grad_row_of(int64_t cols, F&& f) {
    if (cols <= 512) return with_ragged<T, 1, 1>(cols, f);
    if constexpr (sizeof(T) == 2) {
        if (cols <= 1024) return with_ragged<T, 1, 2>(cols, f);
    } else {
        if (cols <= 1024) return with_ragged<T, 2, 1>(cols, f);
    }
    if (cols <= 2048) return with_ragged<T, 4, 1>(cols, f);
    if (cols <= 4096) return with_ragged<T, 8, 1>(cols, f);
    if constexpr (sizeof(T) == 2) {
        if (cols > 8192) return with_ragged<T, 16, 2>(cols, f);
    }
    return with_ragged<T, 16, 1>(cols, f);
}
template <typename F>
hipError_t with_grad_row(int bf16, int64_t cols, F&& f) {
    return bf16 ? with_grad_row_of<uint16_t>(cols, f) : with_grad_row_of<float>(cols, f);
}

unsigned row_grid(int64_t tokens) { return (unsigned)std::min<int64_t>(tokens, 1 << 16); }

}  // namespace

int64_t col_sum_blocks(int64_t tokens, int64_t width) {
    const int64_t strips = (width + kColW - 1) / kColW;
    return std::max<int64_t>(1, std::min<int64_t>((tokens + 63) / 64, std::max<int64_t>(1, 1024 / strips)));
}
int64_t norm_grad_blocks(int64_t tokens, int64_t cols, int bf16) {
    if (!grad_in_regs(bf16, cols)) return col_sum_blocks(tokens, cols);
    // sixteen waves a CU
    const int wpr = grad_wpr(bf16, cols), waves = row_waves(wpr);
    return std::max<int64_t>(1, std::min<int64_t>((tokens * wpr + waves - 1) / waves, 256 * 16 / waves));
}

hipError_t launch_col_sum(const ColSumArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.width + kColW - 1) / kColW), (unsigned)a.blocks);
    if (a.bf16) col_parts<uint16_t, 0><<<grid, kThreads, 0, s>>>(a, a.width);
    else col_parts<float, 0><<<grid, kThreads, 0, s>>>(a, a.width);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return launch_col_join(a, s);
}

hipError_t launch_col_join(const ColSumArgs& a, hipStream_t s) {
    return join({a.part, a.blocks, a.width, a.width, a.width, a.out, nullptr, a.out_bf16, a.accumulate}, s);
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
    return with_row(a.bf16, a.cols, a.tokens < kFewRows, [&](auto row) {
        using R = decltype(row);
        if constexpr (R::WPR == 0) {
            norm_rows<typename R::T><<<row_grid(a.tokens), kThreads, 0, s>>>(a);
        } else {
            constexpr int WAVES = row_waves(R::WPR), RPB = WAVES / R::WPR;
            const int64_t blocks = (a.tokens + RPB - 1) / RPB, x = std::min<int64_t>(blocks, 1 << 20);
            const dim3 grid((unsigned)x, (unsigned)((blocks + x - 1) / x));
            norm_regs<typename R::T, R::WPR, R::CH, R::RAGGED><<<grid, 64 * WAVES, 0, s>>>(a);
        }
        return hipGetLastError();
    });
}

hipError_t launch_norm_grad(NormGradArgs a, hipStream_t s) {
    const bool params = a.dgamma || a.dbeta;
    if (!params) a.part = nullptr;
    a.run = (a.tokens + a.blocks - 1) / a.blocks;
    hipError_t e = hipSuccess;
    if (grad_in_regs(a.bf16, a.cols)) {
        e = with_grad_row(a.bf16, a.cols, [&](auto row) {
            using R = decltype(row);
            const size_t padded = 4 * ((a.cols + 7) / 8 * 8), lds = R::WPR == 1 ? 3 * padded : padded;
            auto* kernel = &norm_grad_regs<typename R::T, R::WPR, R::CH, R::RAGGED>;
            if (lds > 48 * 1024) {   // more than a launch is given unasked
                hipError_t set = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
                if (set != hipSuccess) return set;
            }
            kernel<<<(unsigned)a.blocks, 64 * row_waves(R::WPR), lds, s>>>(a);
            return hipGetLastError();
        });
    } else {
        if (params) {   // these first: dX may be dY's own storage
            const dim3 grid((unsigned)((a.cols + kColW - 1) / kColW), (unsigned)a.blocks);
            if (a.bf16) col_parts<uint16_t, 1><<<grid, kThreads, 0, s>>>(a, a.cols);
            else col_parts<float, 1><<<grid, kThreads, 0, s>>>(a, a.cols);
            e = hipGetLastError();
        }
        if (e == hipSuccess && a.dX && a.tokens) {
            if (a.bf16) norm_grad_rows<uint16_t><<<row_grid(a.tokens), kThreads, 0, s>>>(a);
            else norm_grad_rows<float><<<row_grid(a.tokens), kThreads, 0, s>>>(a);
            e = hipGetLastError();
        }
    }
    if (e != hipSuccess || !params) return e;
    return join({a.part, a.blocks, 2 * a.cols, 2 * a.cols, a.cols, a.dgamma, a.dbeta, a.g_bf16, a.accumulate}, s);
}

}  // namespace dion2
