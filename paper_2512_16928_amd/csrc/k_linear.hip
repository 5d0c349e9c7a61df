// The three products of a linear layer on MFMA, with what follows them fused:
//   forward   Y = act(X W^T + b) + R      both operands have k contiguous
//   input     dX = (dY W) act'(Z)         W has n contiguous
//   weight    G = dY^T X                  both have m or n contiguous
// Sums are fp32 (the MFMA accumulators); a result is rounded once, at its
// store. Where a launch has too few tiles for the chip, K is cut into parts:
// their fp32 sums go to the workspace and a second launch adds them in order
// and finishes the entries, so results depend on the sizes alone.
#include <algorithm>
#include <type_traits>

#include "layers.h"

namespace dion2 {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((ext_vector_type(8))) short i16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;

// ------------------------------------------------------------- the epilogue
// Finishes entries n .. n + 7 of row m (those that exist) from their sums.
template <Product KIND, typename T>
__device__ __forceinline__ void finish8(const ProductArgs& a, int64_t m, int64_t n, float (&v)[8]) {
    constexpr bool FINE = std::is_same<T, float>::value;
    if (m >= a.M || n >= a.N) return;
    const int nv = a.N - n < 8 ? (int)(a.N - n) : 8;
    float x[8];
    if constexpr (KIND == PROD_FORWARD) {
        if (a.bias) {
            load8_as(a.bias, n, a.bias_bf16, nv, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += x[i];
        }
        if (a.Z) store8(static_cast<T*>(a.Z) + m * a.ldz + n, nv, v);
        if (a.act != ACT_NONE) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = act_value<FINE>(v[i], a.act);
        }
        if (a.R) {
            load8(static_cast<const T*>(a.R) + m * a.ldr + n, nv, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += x[i];
        }
        store8(static_cast<T*>(a.out) + m * a.ldo + n, nv, v);
    } else if constexpr (KIND == PROD_INPUT) {
        if (a.act != ACT_NONE) {
            load8(static_cast<const T*>(a.Z) + m * a.ldz + n, nv, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= act_slope<FINE>(x[i], a.act);
        }
        store8(static_cast<T*>(a.out) + m * a.ldo + n, nv, v);
    } else {
        if (a.accumulate) {
            load8_as(a.out, m * a.ldo + n, a.out_bf16, nv, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += x[i];
        }
        store8_as(a.out, m * a.ldo + n, a.out_bf16, nv, v);
    }
}

// A 32 x 32 block's accumulators hold C transposed (the B fragment is the
// MFMA's first operand): lane l has row m = l mod 32 and, in registers 4 q ..
// 4 q + 3, columns 8 q + 4 (l / 32) + 0 .. 3. Swapping the lane halves of
// registers q and q + 1 leaves every lane eight consecutive columns.
template <typename F>
__device__ __forceinline__ void each_row_of_8(const f32x16& acc, int lane, F&& f) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[8 * c + j]),
                                                            __float_as_uint(acc[8 * c + 4 + j]), false, false);
            v[j] = __uint_as_float(s[0]);
            v[4 + j] = __uint_as_float(s[1]);
        }
        f(lane & 31, 16 * c + 8 * (lane >> 5), v);
    }
}

// ---------------------------------------------------- tiles of any alignment
// 128 x 128 tiles, four waves of 64 x 64. Operands come through registers,
// 16 bytes a load from any element boundary, with zeros past the matrix's
// edges, one slice ahead of the MFMAs, into one of two LDS buffers.
//
// bf16: slices of 32. k-contiguous operands are kept [row][k], m/n-contiguous
// ones [k][row] and read with the transposing LDS read; both with their
// 16-byte chunks swizzled against bank conflicts. fp32: slices of 16, always
// kept [k][row] (a fragment of v_mfma_f32_32x32x2_f32 is one float of 32
// consecutive rows), rows padded by 16 bytes.
constexpr int kGT = 128;
constexpr int kGThreads = 256;

template <typename T> struct GSlice;
template <> struct GSlice<uint16_t> { static constexpr int K = 32, BYTES = kGT * 64; };
template <> struct GSlice<float> { static constexpr int K = 16, LD = kGT + 4, BYTES = 16 * LD * 4; };

__device__ __forceinline__ uint4 load_chunk(const uint16_t* p, int n) {
    if (n >= 8) return ldg<uint4>(p);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) w[i / 2] |= (uint32_t)ldg<uint16_t>(p + i) << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 load_chunk(const float* p, int n) {
    if (n >= 4) return ldg<uint4>(p);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) w[i] = ldg<uint32_t>(p + i);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// One operand's part of a slice: two 16-byte chunks a thread.
template <typename T, bool KMAJOR>
struct GOperand {
    static constexpr int E = 16 / sizeof(T);        // entries a chunk
    static constexpr int SK = GSlice<T>::K;
    static constexpr int CPR = (KMAJOR ? SK : kGT) / E;   // chunks a stored row
    uint4 reg[2];

    // row0: the tile's first row (m or n); rows, K: the operand's extents
    __device__ __forceinline__ void load(const T* p, int64_t ld, int64_t row0, int64_t rows, int64_t k0, int64_t K, int tid) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int i = tid + q * kGThreads;
            const int64_t outer = (KMAJOR ? row0 : k0) + i / CPR, inner = (KMAJOR ? k0 : row0) + i % CPR * E;
            const int64_t n_outer = KMAJOR ? rows : K, n_inner = KMAJOR ? K : rows;
            const int64_t left = n_inner - inner;
            const int n = outer < n_outer ? (int)(left < E ? left : E) : 0;
            reg[q] = n > 0 ? load_chunk(p + outer * ld + inner, n) : make_uint4(0, 0, 0, 0);
        }
    }
    __device__ __forceinline__ void stage(unsigned char* lds, int tid) const {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int i = tid + q * kGThreads;
            const int r = i / CPR, c = i % CPR;
            if constexpr (sizeof(T) == 2) {
                const int off = KMAJOR ? r * 64 + 16 * (c ^ ((r / 4) % 4)) : r * 256 + 16 * (c ^ ((r & 3) << 2));
                *reinterpret_cast<uint4*>(lds + off) = reg[q];
            } else {
                float* f = reinterpret_cast<float*>(lds);
                if constexpr (KMAJOR) {
                    const uint32_t w[4] = {reg[q].x, reg[q].y, reg[q].z, reg[q].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[(4 * c + j) * GSlice<float>::LD + r] = __uint_as_float(w[j]);
                } else {
                    *reinterpret_cast<uint4*>(f + r * GSlice<float>::LD + 4 * c) = reg[q];
                }
            }
        }
    }
};

// Fragment of 32 rows from `row` on, k-step kk, of a bf16 operand.
template <bool KMAJOR>
__device__ __forceinline__ bf16x8 g_frag(const unsigned char* lds, int row, int kk, int lane) {
    if constexpr (KMAJOR) {
        const int r = row + (lane & 31), c = 2 * kk + (lane >> 5);
        return *reinterpret_cast<const bf16x8*>(lds + r * 64 + 16 * (c ^ ((r / 4) % 4)));
    } else {
        // a lane of a 16-lane group receives element (i mod 4) of the 8 bytes
        // addressed by source lane 4 e + i / 4, e = 0 .. 3
        typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
        const int g = lane >> 4, s = lane & 15;
        const int k = 16 * kk + 8 * (g >> 1) + (s >> 2);
        const int r = row + 16 * (g & 1) + 4 * (s & 3);
        auto at = [&](int kr) { return kr * 256 + 16 * ((r >> 3) ^ ((kr & 3) << 2)) + 2 * (r & 7); };
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lds + at(k)));
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lds + at(k + 4)));
        const i16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        return __builtin_bit_cast(bf16x8, v);
    }
}

template <Product KIND, typename T>
__global__ __launch_bounds__(kGThreads) void product_any(ProductArgs a) {
    constexpr bool AK = KIND != PROD_WEIGHT, BKM = KIND == PROD_FORWARD;
    constexpr int SK = GSlice<T>::K, SB = GSlice<T>::BYTES;
    __shared__ __align__(16) unsigned char lds[2][2][SB];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
    const int64_t tiles_n = (a.N + kGT - 1) / kGT;
    const int64_t m0 = blockIdx.x / tiles_n * kGT, n0 = blockIdx.x % tiles_n * kGT;
    const int64_t slices = (a.K + SK - 1) / SK;
    const int64_t s0 = slices * blockIdx.y / a.splits, s1 = slices * (blockIdx.y + 1) / a.splits;
    const T* A = static_cast<const T*>(a.A);
    const T* B = static_cast<const T*>(a.B);
    GOperand<T, AK> ga;
    GOperand<T, BKM> gb;
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    if (s0 < s1) {
        ga.load(A, a.lda, m0, a.M, s0 * SK, a.K, tid);
        gb.load(B, a.ldb, n0, a.N, s0 * SK, a.K, tid);
    }
    for (int64_t s = s0; s < s1; ++s) {
        unsigned char* la = lds[(s - s0) & 1][0];
        unsigned char* lb = lds[(s - s0) & 1][1];
        ga.stage(la, tid);
        gb.stage(lb, tid);
        __syncthreads();   // and every wave is done with this buffer's slice before last
        if (s + 1 < s1) {
            ga.load(A, a.lda, m0, a.M, (s + 1) * SK, a.K, tid);
            gb.load(B, a.ldb, n0, a.N, (s + 1) * SK, a.K, tid);
        }
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int kk = 0; kk < SK / 16; ++kk) {
                bf16x8 fa[2], fb[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    fa[i] = g_frag<AK>(la, wm + 32 * i, kk, lane);
                    fb[i] = g_frag<BKM>(lb, wn + 32 * i, kk, lane);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
            }
        } else {
            const float* pa = reinterpret_cast<const float*>(la) + wm + (lane & 31);
            const float* pb = reinterpret_cast<const float*>(lb) + wn + (lane & 31);
#pragma unroll
            for (int kk = 0; kk < SK / 2; ++kk) {
                const int k = (2 * kk + (lane >> 5)) * GSlice<float>::LD;
                const float fa[2] = {pa[k], pa[k + 32]}, fb[2] = {pb[k], pb[k + 32]};
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fb[j], fa[i], acc[i][j], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
            each_row_of_8(acc[i][j], lane, [&](int r, int c, float (&v)[8]) {
                const int64_t m = m0 + wm + 32 * i + r, n = n0 + wn + 32 * j + c;
                if (a.splits > 1) {
                    if (m < a.M && n < a.N)
                        store8(a.part + ((int64_t)blockIdx.y * a.M + m) * a.N + n, a.N - n < 8 ? (int)(a.N - n) : 8, v);
                } else {
                    finish8<KIND, T>(a, m, n, v);
                }
            });
}

// Adds the parts of a split product in order and finishes its entries.
template <Product KIND, typename T>
__global__ __launch_bounds__(256) void product_join(ProductArgs a) {
    const int64_t chunks = (a.N + 7) / 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.M * chunks) return;
    const int64_t m = i / chunks, n = i % chunks * 8;
    const int nv = a.N - n < 8 ? (int)(a.N - n) : 8;
    float v[8] = {};
    for (int s = 0; s < a.splits; ++s) {
        float x[8];
        load8(a.part + ((int64_t)s * a.M + m) * a.N + n, nv, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += x[j];
    }
    finish8<KIND, T>(a, m, n, v);
}

template <Product KIND, typename T>
hipError_t launch_kind(const ProductArgs& a, hipStream_t s) {
    const int64_t tiles = ((a.M + kGT - 1) / kGT) * ((a.N + kGT - 1) / kGT);
    product_any<KIND, T><<<dim3((unsigned)tiles, (unsigned)a.splits), kGThreads, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t chunks = a.M * ((a.N + 7) / 8);
    product_join<KIND, T><<<(unsigned)((chunks + 255) / 256), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

int product_splits(Product kind, int64_t M, int64_t N, int64_t K, int bf16) {
    const int64_t tiles = ((M + kGT - 1) / kGT) * ((N + kGT - 1) / kGT);
    const int64_t slices = (K + 63) / 64;
    // two tiles a CU, but at least 256 of k a part
    const int64_t want = tiles >= 512 ? 1 : 512 / std::max<int64_t>(tiles, 1);
    return (int)std::max<int64_t>(1, std::min<int64_t>({want, slices / 4, 32}));
}

hipError_t launch_product(Product kind, const ProductArgs& a, hipStream_t s) {
    if (a.M == 0 || a.N == 0) return hipSuccess;
    if (a.bf16) {
        if (kind == PROD_FORWARD) return launch_kind<PROD_FORWARD, uint16_t>(a, s);
        if (kind == PROD_INPUT) return launch_kind<PROD_INPUT, uint16_t>(a, s);
        return launch_kind<PROD_WEIGHT, uint16_t>(a, s);
    }
    if (kind == PROD_FORWARD) return launch_kind<PROD_FORWARD, float>(a, s);
    if (kind == PROD_INPUT) return launch_kind<PROD_INPUT, float>(a, s);
    return launch_kind<PROD_WEIGHT, float>(a, s);
}

}  // namespace dion2
