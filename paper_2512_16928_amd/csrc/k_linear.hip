// The three products of a linear layer on MFMA, with what follows them fused:
//   forward   Y = act(X W^T + b) + R      both operands have k contiguous
//   input     dX = (dY W) act'(Z)         W has n contiguous
//   weight    G = dY^T X                  both have m or n contiguous
// Sums are fp32 (the MFMA accumulators); a result is rounded once, at its
// store. Where a launch has too few tiles for the chip, K is cut into parts:
// their fp32 sums go to the workspace and a second launch adds them in order
// and finishes the entries, so results depend on the sizes, pitches and
// alignment alone.
#include <algorithm>
#include <type_traits>

#include "layers.h"

namespace dion2 {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((ext_vector_type(8))) short i16x8;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;

// ------------------------------------------------------------- the epilogue
// with_act where the product has an activation.
template <Product KIND, typename F>
__device__ __forceinline__ void with_act_of(int act, F&& f) {
    if constexpr (KIND == PROD_WEIGHT) f(ActIs<ACT_NONE>{});
    else with_act(act, f);
}

// The epilogue's own operand, [M][N]: the residual, the pre-activation, or
// the gradient that is added to. Null where there is none.
template <Product KIND>
__device__ __forceinline__ const void* epilogue_operand(const ProductArgs& a, int64_t* ld) {
    *ld = KIND == PROD_FORWARD ? a.ldr : KIND == PROD_INPUT ? a.ldz : a.ldo;
    return KIND == PROD_FORWARD ? a.R : KIND == PROD_INPUT ? (a.act != ACT_NONE ? a.Z : nullptr) : (a.accumulate ? a.out : nullptr);
}

// Finishes entries n .. n + nv - 1 of row m from their sums v and the
// operand's entries x (unused where there is none). BIAS: not in the sums yet.
template <Product KIND, int ACT, bool BIAS, typename T>
__device__ __forceinline__ void finish8(const ProductArgs& a, int64_t m, int64_t n, int nv, float (&v)[8], const float (&x)[8]) {
    constexpr bool FINE = std::is_same<T, float>::value;
    if constexpr (KIND == PROD_FORWARD) {
        if (BIAS && a.bias) {
            float b[8];
            load8_as(a.bias, n, a.bias_bf16, nv, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += b[i];
        }
        if (a.Z) store8(static_cast<T*>(a.Z) + m * a.ldz + n, nv, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = act_value<ACT, FINE>(v[i]);
        if (a.R) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += x[i];
        }
        store8(static_cast<T*>(a.out) + m * a.ldo + n, nv, v);
    } else if constexpr (KIND == PROD_INPUT) {
        if constexpr (ACT != ACT_NONE) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= act_slope<ACT, FINE>(x[i]);
        }
        store8(static_cast<T*>(a.out) + m * a.ldo + n, nv, v);
    } else {
        if (a.accumulate) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += x[i];
        }
        store8_as(a.out, m * a.ldo + n, a.out_bf16, nv, v);
    }
}

// The same where the entries may lie past the edges.
template <Product KIND, int ACT, bool BIAS, typename T>
__device__ __forceinline__ void finish8_edge(const ProductArgs& a, int64_t m, int64_t n, float (&v)[8]) {
    if (m >= a.M || n >= a.N) return;
    const int nv = a.N - n < 8 ? (int)(a.N - n) : 8;
    float x[8];
    int64_t ld;
    const void* p = epilogue_operand<KIND>(a, &ld);
    if (p) load8_as(p, m * ld + n, KIND == PROD_WEIGHT ? a.out_bf16 : std::is_same<T, uint16_t>::value, nv, x);
    finish8<KIND, ACT, BIAS, T>(a, m, n, nv, v, x);
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

// A 32 x 32 block of a product cut into parts, at rows m0.., columns n0..: its
// sums as they are, in register order (16 bytes a lane), for product_join.
__device__ __forceinline__ void store_part(const ProductArgs& a, int64_t m0, int64_t n0, const f32x16& acc, int lane) {
    if (m0 >= a.M || n0 >= a.N) return;
    const int64_t mb = (a.M + 31) / 32, nb = (a.N + 31) / 32;
    float* p = a.part + ((blockIdx.y * mb + m0 / 32) * nb + n0 / 32) * 1024 + lane * 4;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        stg(p + 256 * q, make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]));
}

// ---------------------------------------------------- tiles of any alignment
// 128 x 128 tiles, four waves of 64 x 64, or 64 x 64 tiles, four waves of 32 x
// 32, with slices twice as deep, in launches of few tiles. Operands come
// through registers, 16 bytes a load from any element boundary, with zeros past
// the matrix's edges, one slice ahead of the MFMAs, into one of two LDS buffers.
//
// bf16: slices of 32 (64). k-contiguous operands are kept [row][k],
// m/n-contiguous ones [k][row] and read with the transposing LDS read; both
// with their 16-byte chunks swizzled against bank conflicts. fp32: slices of 16
// (32), always kept [k][row] (a fragment of v_mfma_f32_32x32x2_f32 is one float
// of 32 consecutive rows), rows padded by 16 bytes.
constexpr int kGThreads = 256;

template <typename T, int GT> struct GSlice;
template <int GT> struct GSlice<uint16_t, GT> { static constexpr int K = 4096 / GT, BYTES = GT * K * 2; };
template <int GT> struct GSlice<float, GT> { static constexpr int K = 2048 / GT, LD = GT + 4, BYTES = K * LD * 4; };

// The n entries (1 to all of a chunk's) from p on, zeros behind them. `before`
// entries of the row lie before p: with enough of them a chunk that the row's
// end cuts is read as the row's last 16 bytes, and the entries before it dropped.
__device__ __forceinline__ uint4 load_chunk(const uint16_t* p, int n, int64_t before = 0) {
    if (n >= 8) return ldg<uint4>(p);
    if (before >= 8 - n) {
        const uint4 v = ldg<uint4>(p - (8 - n));
        const uint64_t lo = (uint64_t)v.y << 32 | v.x, hi = (uint64_t)v.w << 32 | v.z;
        const int b = 16 * (-n & 3);   // 8 - n entries: whole quads of them and b bits
        const uint64_t carry = b ? hi << (64 - b) : 0;
        const uint64_t l = n > 4 ? lo >> b | carry : hi >> b, h = n > 4 ? hi >> b : 0;
        return make_uint4((uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32));
    }
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) w[i / 2] |= (uint32_t)ldg<uint16_t>(p + i) << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 load_chunk(const float* p, int n, int64_t before = 0) {
    if (n >= 4) return ldg<uint4>(p);
    if (before >= 4 - n) {
        const uint4 v = ldg<uint4>(p - (4 - n));
        return n == 3 ? make_uint4(v.y, v.z, v.w, 0) : n == 2 ? make_uint4(v.z, v.w, 0, 0) : make_uint4(v.w, 0, 0, 0);
    }
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) w[i] = ldg<uint32_t>(p + i);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// One operand's part of a slice: two 16-byte chunks a thread.
template <typename T, int GT, bool KMAJOR>
struct GOperand {
    static constexpr int E = 16 / sizeof(T);        // entries a chunk
    static constexpr int SK = GSlice<T, GT>::K;
    static constexpr int CPR = (KMAJOR ? SK : GT) / E;   // chunks a stored row
    static constexpr int PITCH = CPR * 16;               // bytes of a bf16 one
    uint4 reg[2];

    __device__ __forceinline__ static int swizzle(int row) { return KMAJOR ? (row / (PITCH < 256 ? 256 / PITCH : 1)) % CPR : (row & 3) << (GT == 128 ? 2 : 1); }

    // row0: the tile's first row (m or n); rows, K: the operand's extents
    __device__ __forceinline__ void load(const T* p, int64_t ld, int64_t row0, int64_t rows, int64_t k0, int64_t K, int tid) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int i = tid + q * kGThreads;
            const int64_t outer = (KMAJOR ? row0 : k0) + i / CPR, inner = (KMAJOR ? k0 : row0) + i % CPR * E;
            const int64_t n_outer = KMAJOR ? rows : K, n_inner = KMAJOR ? K : rows;
            const int64_t left = n_inner - inner;
            const int n = outer < n_outer ? (int)(left < E ? left : E) : 0;
            reg[q] = n > 0 ? load_chunk(p + outer * ld + inner, n, inner) : make_uint4(0, 0, 0, 0);
        }
    }
    __device__ __forceinline__ void stage(unsigned char* lds, int tid) const {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int i = tid + q * kGThreads;
            const int r = i / CPR, c = i % CPR;
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<uint4*>(lds + r * PITCH + 16 * (c ^ swizzle(r))) = reg[q];
            } else {
                float* f = reinterpret_cast<float*>(lds);
                if constexpr (KMAJOR) {
                    const uint32_t w[4] = {reg[q].x, reg[q].y, reg[q].z, reg[q].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[(4 * c + j) * GSlice<float, GT>::LD + r] = __uint_as_float(w[j]);
                } else {
                    *reinterpret_cast<uint4*>(f + r * GSlice<float, GT>::LD + 4 * c) = reg[q];
                }
            }
        }
    }
};

// Fragment of 32 rows from `row` on, k-step kk, of a bf16 operand.
template <typename O, bool KMAJOR>
__device__ __forceinline__ bf16x8 g_frag(const unsigned char* lds, int row, int kk, int lane) {
    if constexpr (KMAJOR) {
        const int r = row + (lane & 31), c = 2 * kk + (lane >> 5);
        return *reinterpret_cast<const bf16x8*>(lds + r * O::PITCH + 16 * (c ^ O::swizzle(r)));
    } else {
        // a lane of a 16-lane group receives element (i mod 4) of the 8 bytes
        // addressed by source lane 4 e + i / 4, e = 0 .. 3
        typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
        const int g = lane >> 4, s = lane & 15;
        const int k = 16 * kk + 8 * (g >> 1) + (s >> 2);
        const int r = row + 16 * (g & 1) + 4 * (s & 3);
        auto at = [&](int kr) { return kr * O::PITCH + 16 * ((r >> 3) ^ O::swizzle(kr)) + 2 * (r & 7); };
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lds + at(k)));
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lds + at(k + 4)));
        const i16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        return __builtin_bit_cast(bf16x8, v);
    }
}

template <Product KIND, typename T, int GT>
__global__ __launch_bounds__(kGThreads) void product_any(ProductArgs a) {
    constexpr bool AK = KIND != PROD_WEIGHT, BKM = KIND == PROD_FORWARD;
    constexpr int SK = GSlice<T, GT>::K, SB = GSlice<T, GT>::BYTES, F = GT / 64;   // F x F blocks a wave
    __shared__ __align__(16) unsigned char lds[2][2][SB];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = (wave >> 1) * 32 * F, wn = (wave & 1) * 32 * F;
    const int64_t tiles_n = (a.N + GT - 1) / GT;
    const int64_t m0 = blockIdx.x / tiles_n * GT, n0 = blockIdx.x % tiles_n * GT;
    const int64_t slices = (a.K + SK - 1) / SK;
    const int64_t s0 = slices * blockIdx.y / a.splits, s1 = slices * (blockIdx.y + 1) / a.splits;
    const T* A = static_cast<const T*>(a.A);
    const T* B = static_cast<const T*>(a.B);
    using GA = GOperand<T, GT, AK>;
    using GB = GOperand<T, GT, BKM>;
    GA ga;
    GB gb;
    f32x16 acc[F][F];
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j)
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
                bf16x8 fa[F], fb[F];
#pragma unroll
                for (int i = 0; i < F; ++i) {
                    fa[i] = g_frag<GA, AK>(la, wm + 32 * i, kk, lane);
                    fb[i] = g_frag<GB, BKM>(lb, wn + 32 * i, kk, lane);
                }
#pragma unroll
                for (int i = 0; i < F; ++i)
#pragma unroll
                    for (int j = 0; j < F; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
            }
        } else {
            const float* pa = reinterpret_cast<const float*>(la) + wm + (lane & 31);
            const float* pb = reinterpret_cast<const float*>(lb) + wn + (lane & 31);
#pragma unroll
            for (int kk = 0; kk < SK / 2; ++kk) {
                const int k = (2 * kk + (lane >> 5)) * GSlice<float, GT>::LD;
                float fa[F], fb[F];
#pragma unroll
                for (int i = 0; i < F; ++i) {
                    fa[i] = pa[k + 32 * i];
                    fb[i] = pb[k + 32 * i];
                }
#pragma unroll
                for (int i = 0; i < F; ++i)
#pragma unroll
                    for (int j = 0; j < F; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fb[j], fa[i], acc[i][j], 0, 0, 0);
            }
        }
    }
    if (a.splits > 1) {
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
            for (int j = 0; j < F; ++j) store_part(a, m0 + wm + 32 * i, n0 + wn + 32 * j, acc[i][j], lane);
        return;
    }
    with_act_of<KIND>(a.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
            for (int j = 0; j < F; ++j)
                each_row_of_8(acc[i][j], lane, [&](int r, int c, float (&v)[8]) {
                    finish8_edge<KIND, decltype(act)::value, true, T>(a, m0 + wm + 32 * i + r, n0 + wn + 32 * j + c, v);
                });
    });
}

// ------------------------------------------------------- tiles, LDS fed directly
// For operands whose rows start on 16-byte boundaries and are whole chunks of 16
// bytes long (others are copied so first, with zeros behind). K-slices go from
// global memory straight into LDS (16 bytes a lane, a wave's 1 KB a time), S
// slices in flight, through buffer descriptors: a lane whose chunk lies past
// an edge asks for an offset past the descriptor's range and gets zeros.
//
// k-contiguous tiles are kept [row][k] in rows of 128 bytes, m/n-contiguous
// ones [k][row]; 16-byte chunks are swizzled so that the fragment reads of a
// sixteenth of a wave (and the transposing reads' 64-byte pieces of four k)
// fall into distinct LDS banks. fp32's [k][row] is read an entry a lane.
template <typename T_, int BM_, int BN_, int BK_, int S_, int WM_, int WN_>
struct Tile {
    using T = T_;
    static constexpr int BM = BM_, BN = BN_, BK = BK_, S = S_, WM = WM_, WN = WN_, E = sizeof(T);
    static_assert(BK * E == 128, "a slice is 128 bytes of a k-contiguous row");
    static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int TM = BM / WM, TN = BN / WN, FM = TM / 32, FN = TN / 32;
    static constexpr int A_BYTES = BM * BK * E, STAGE = (BM + BN) * BK * E;
    static constexpr int LOADS = STAGE / 1024 / WAVES;   // of a wave a slice
    // the epilogue's staging of a wave: 32 rows of its part of the tile, padded
    static constexpr int EPI_ROWS = 32, EPI_LD = TN + 4;
    static constexpr int SMEM = S * STAGE;
    static_assert(WAVES * EPI_ROWS * EPI_LD * 4 <= SMEM, "the staging fits the ring");
    static_assert(STAGE % (1024 * WAVES) == 0 && A_BYTES % (1024 * WAVES) == 0, "whole loads");
};

template <int N>
__device__ __forceinline__ void wait_loads() {   // at most N of this wave's loads still on their way, no LDS read
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
}

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4)); }

// Rows of an operand: an m/n-contiguous one has them in whole chunks of C.
template <bool KMAJOR, int C>
__device__ __forceinline__ int64_t extent(int64_t rows) { return KMAJOR ? rows : (rows + C - 1) & ~(int64_t)(C - 1); }

// One operand of a tile: R rows (m or n), slices of BK. HALF 0, 1: every first,
// second run of 64 rows of a tile of 2 R (what a wave of a 256-row tile reads
// in its first, second half); -1: the rows as they are.
template <typename T, int R, int BK, int WAVES, bool KMAJOR, int HALF = -1>
struct Operand {
    static constexpr int E = sizeof(T), C = 16 / E;            // bytes an entry, entries a chunk
    static constexpr int PITCH = KMAJOR ? BK * E : R * E;      // LDS row
    static constexpr int CPR = PITCH / 16;
    static constexpr int RPB = 1024 / PITCH;                   // LDS rows a 1 KB block holds
    static constexpr int Q = R * BK * E / 1024 / WAVES;        // blocks a wave
    static constexpr uint32_t OUT = 0x80000000u;               // past every descriptor's range
    __amdgpu_buffer_rsrc_t rsrc;
    const unsigned char* base;
    int64_t step;          // bytes a slice
    uint32_t off[Q];       // of the lane's chunks in the wave's blocks
    int k_lane;            // k of the lane's chunk in the wave's first block
    int k_left;            // from the slice loaded next on

    __device__ __forceinline__ static int swizzle(int row) {
        return KMAJOR ? (row / (PITCH < 256 ? 256 / PITCH : 1)) % CPR : E == 2 ? (row & 3) << (PITCH < 256 ? 1 : 2) : 0;
    }
    __device__ __forceinline__ static int tile_row(int r) {
        return HALF < 0 ? r : r / 64 * 128 + HALF * 64 + r % 64;
    }
    // p: the operand's first row of the tile and first k; rows: of them that exist
    __device__ __forceinline__ void init(const T* p, int64_t ld, int64_t rows, int64_t k, int wave, int lane) {
        const int lr = lane / CPR, slot = lane % CPR;
        const int c = slot ^ swizzle(wave * RPB + lr);   // alike in all of a wave's blocks (an even number of rows apart)
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int r = (wave + q * WAVES) * RPB + lr;
            const int row = tile_row(KMAJOR ? r : C * c);
            off[q] = row < rows ? (uint32_t)(KMAJOR ? row * ld * E + 16 * c : r * ld * E + E * row) : OUT;
        }
        k_lane = KMAJOR ? C * c : wave * RPB + lr;
        base = reinterpret_cast<const unsigned char*>(p);
        step = KMAJOR ? E * BK : E * BK * ld;
        k_left = (int)k;
        rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base), 0, (int)0x7ffffff0, 0x00020000);
    }
    __device__ __forceinline__ void load(int q, unsigned char* lds, int wave) const {
        const uint32_t v = k_lane + (KMAJOR ? 0 : q * WAVES * RPB) < k_left ? off[q] : OUT;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(lds + (wave + q * WAVES) * 1024),
                                                 16, v, 0, 0, 0);
    }
    __device__ __forceinline__ void advance() {
        base += step;
        k_left -= BK;
        rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base), 0, (int)0x7ffffff0, 0x00020000);
    }
};

// Finishes a wave's part of a tile. 32 rows at a time go through LDS, so that
// a row of the output leaves in whole lines (a lane takes eight columns, TN / 8
// lanes a row) and one copy of the code serves all of them: unrolled over the
// accumulators it would be eight times as long. Steps of 64 / (TN / 8) rows run
// in groups (of four) whose operand entries are requested one group ahead.
template <Product KIND, int ACT, typename T, bool EDGE>
__device__ __forceinline__ void finish_tile(const ProductArgs& a, const f32x16 (&acc)[T::FM][T::FN], float* stage, int64_t m0,
                                            int64_t n0, int lane) {
    constexpr int LPR = T::TN / 8, RPS = 64 / LPR, STEPS = 32 / RPS;   // lanes a row, rows a step, steps of 32 rows
    constexpr int G = STEPS < 4 ? STEPS : 4, GROUPS = T::FM * STEPS / G;   // steps a group
    const int lr = lane / LPR, lc = lane % LPR * 8;
    const int64_t n = n0 + lc;
    const int nv = EDGE ? (int)(a.N - n < 8 ? a.N - n : 8) : 8;
    int64_t ldx;
    const void* xp = epilogue_operand<KIND>(a, &ldx);
    // a gradient that is added to may be fp32: read where it is used
    const bool ahead = xp && (KIND != PROD_WEIGHT || a.out_bf16);
    uint4 x[G], x_next[G];
    auto fetch = [&](int g) {
#pragma unroll
        for (int u = 0; u < G; ++u) {
            const int64_t m = m0 + (G * g + u) * RPS + lr;
            const uint16_t* p = static_cast<const uint16_t*>(xp) + m * ldx + n;
            if constexpr (EDGE) x_next[u] = m < a.M && nv > 0 ? load_chunk(p, nv) : make_uint4(0, 0, 0, 0);
            else x_next[u] = ldg<uint4>(p);
        }
    };
    if (ahead) fetch(0);
#pragma unroll 1
    for (int g = 0; g < GROUPS; ++g) {
#pragma unroll
        for (int u = 0; u < G; ++u) x[u] = x_next[u];
        if (ahead && g + 1 < GROUPS) fetch(g + 1);
        if (g % (STEPS / G) == 0) {
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < T::FM; ++i)
                if (i == g / (STEPS / G)) {
#pragma unroll
                    for (int j = 0; j < T::FN; ++j)
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            *reinterpret_cast<float4*>(stage + (lane & 31) * T::EPI_LD + 32 * j + 8 * q + 4 * (lane >> 5)) =
                                make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
                }
            __builtin_amdgcn_wave_barrier();
        }
#pragma unroll
        for (int u = 0; u < G; ++u) {
            const int row = (G * g + u) * RPS + lr;
            const float4* p = reinterpret_cast<const float4*>(stage + row % 32 * T::EPI_LD + lc);
            const float4 lo = p[0], hi = p[1];
            float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}, xv[8];
            if constexpr (EDGE) {
                if (m0 + row >= a.M || nv <= 0) continue;
            }
            if (ahead || KIND != PROD_WEIGHT || !xp) unpack8(x[u], xv);
            else load8(static_cast<const float*>(xp) + (m0 + row) * ldx + n, nv, xv);
            finish8<KIND, ACT, false, uint16_t>(a, m0 + row, n, nv, v, xv);
        }
    }
}

// The sums' start: the bias, where they are not parts (a lane's columns are
// 8 q + 4 (lane / 32) + 0 .. 3 of a block).
template <Product KIND, typename T>
__device__ __forceinline__ void start_sums(const ProductArgs& a, f32x16 (&acc)[T::FM][T::FN], int64_t n0, int lane) {
    const bool bias = KIND == PROD_FORWARD && a.bias && a.splits == 1;
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
        f32x16 start;
#pragma unroll
        for (int r = 0; r < 16; ++r) start[r] = 0.0f;
        if (bias) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                int64_t n = n0 + 32 * j + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
                n = n < a.N ? n : a.N - 1;
                start[r] = a.bias_bf16 ? bf16_bits_to_f32(ldg<uint16_t>(static_cast<const uint16_t*>(a.bias) + n))
                                       : ldg<float>(static_cast<const float*>(a.bias) + n);
            }
        }
#pragma unroll
        for (int i = 0; i < T::FM; ++i) acc[i][j] = start;
    }
}

// The bias gradient beside PROD_WEIGHT: sums over k of A's rows, from the
// fragments that are in registers anyway. The waves that share rows (the tiles
// of a row of tiles, WN waves each) take a slice each in turn; what they have is
// a row of partial sums each, added up in order by a launch of its own.
template <typename T>
struct RowSums {
    float sum[T::FM];
    int turn, turns;   // slices until this wave's next, and from one to the next
    __device__ __forceinline__ void init(const ProductArgs& a, uint32_t in, uint32_t tn, int wn, int s0) {
#pragma unroll
        for (int i = 0; i < T::FM; ++i) sum[i] = 0.0f;
        turns = (int)tn * T::WN;
        turn = (int)(((int64_t)(wn * tn + in) - s0 % turns + turns) % turns);
        if (!a.row_sums) turn = turns = 0x7fffffff;
    }
    template <int N>
    __device__ __forceinline__ void add(const bf16x8 (&f)[4][N], int first) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                const u32x4 w = __builtin_bit_cast(u32x4, f[kk][i]);
#pragma unroll
                for (int q = 0; q < 4; ++q) sum[first + i] += __uint_as_float(w[q] << 16) + __uint_as_float(w[q] & 0xffff0000u);
            }
    }
    __device__ __forceinline__ bool mine() const { return turn == 0; }
    __device__ __forceinline__ void next() { turn = turn == 0 ? turns - 1 : turn - 1; }
    __device__ __forceinline__ void store(const ProductArgs& a, uint32_t in, uint32_t tn, int wn, int64_t m0, int lane) {
        if (!a.row_sums) return;
        float* p = a.row_sums + (((int64_t)blockIdx.y * T::WN + wn) * tn + in) * a.M;
#pragma unroll
        for (int i = 0; i < T::FM; ++i) {
            const float v = sum[i] + __shfl_xor(sum[i], 32);   // the halves of a wave have different k
            const int64_t m = m0 + 32 * i + (lane & 31);
            if (lane < 32 && m < a.M) stg(p + m, v);
        }
    }
};

// The end of a wave's sums: parts as they are, else finished through LDS.
template <Product KIND, typename T, typename E>
__device__ __forceinline__ void finish_sums(const ProductArgs& a, const f32x16 (&acc)[T::FM][T::FN], unsigned char* lds, int64_t m0,
                                            int64_t n0, bool whole, int wave, int lane) {
    wait_loads<0>();   // none may land in what LDS is used for next
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (a.splits > 1) {
#pragma unroll
        for (int i = 0; i < T::FM; ++i)
#pragma unroll
            for (int j = 0; j < T::FN; ++j) store_part(a, m0 + 32 * i, n0 + 32 * j, acc[i][j], lane);
        return;
    }
    if constexpr (std::is_same<E, float>::value) {   // 32 bytes a lane as they are
        with_act_of<KIND>(a.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < T::FM; ++i)
#pragma unroll
                for (int j = 0; j < T::FN; ++j)
                    each_row_of_8(acc[i][j], lane, [&](int r, int c, float (&v)[8]) {
                        finish8_edge<KIND, decltype(act)::value, false, float>(a, m0 + 32 * i + r, n0 + 32 * j + c, v);
                    });
        });
        return;
    }
    float* stage = reinterpret_cast<float*>(lds) + wave * T::EPI_ROWS * T::EPI_LD;
    with_act_of<KIND>(a.act, [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        if (whole) finish_tile<KIND, ACT, T, false>(a, acc, stage, m0, n0, lane);
        else finish_tile<KIND, ACT, T, true>(a, acc, stage, m0, n0, lane);
    });
}

// A lane's 16 bytes of a row of 32, and the MFMAs of two of them: eight
// consecutive k of bf16 make one; four of fp32 four, lanes 0 .. 31 and 32 .. 63
// taking k and k + 4 (an order of k that both operands have).
template <typename T> struct FragmentOf { using Type = bf16x8; };
template <> struct FragmentOf<float> { using Type = __attribute__((ext_vector_type(4))) float; };
template <typename T> using Fragment = typename FragmentOf<T>::Type;
__device__ __forceinline__ void multiply(const Fragment<uint16_t>& b, const Fragment<uint16_t>& a, f32x16& acc) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, a, acc, 0, 0, 0);
}
__device__ __forceinline__ void multiply(const Fragment<float>& b, const Fragment<float>& a, f32x16& acc) {
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(b[j], a[j], acc, 0, 0, 0);
}

// The fragments of one or two neighbouring blocks of 32 rows (from `row` on)
// over a whole slice of 128 bytes. The transposing reads are one piece of assembly
// that ends with their wait: as the compiler's own loads, each would first wait
// for every load to LDS still on its way.
template <typename O, int PITCH, typename F, int N>
__device__ __forceinline__ void read_slice(const unsigned char* lds, int row, int lane, F (&f)[4][N], std::true_type) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = row + 32 * i + (lane & 31), c = 2 * kk + (lane >> 5);
            f[kk][i] = *reinterpret_cast<const F*>(lds + r * PITCH + 16 * (c ^ O::swizzle(r)));
        }
}
template <typename O, int PITCH, int N>
__device__ __forceinline__ void read_slice(const unsigned char* lds, int row, int lane, Fragment<float> (&f)[4][N], std::false_type) {
    const unsigned char* p = lds + 4 * (lane >> 5) * PITCH + 4 * (row + (lane & 31));
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) f[kk][i][j] = *reinterpret_cast<const float*>(p + (8 * kk + j) * PITCH + 128 * i);
}
// A lane of a 16-lane group receives element (i mod 4) of the 8 bytes addressed
// by source lane 4 e + i / 4, e = 0 .. 3: four consecutive k of its row.
template <typename O, int PITCH>
__device__ __forceinline__ uint32_t tr_address(const unsigned char* lds, int row, int lane) {
    const int g = lane >> 4, s = lane & 15;
    const int k = 8 * (g >> 1) + (s >> 2), r = row + 16 * (g & 1) + 4 * (s & 3);
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const unsigned char*)(lds + k * PITCH +
                                                                                        16 * ((r >> 3) ^ O::swizzle(k)) + 2 * (r & 7));
}
__device__ __forceinline__ bf16x8 tr_frag(u32x2 lo, u32x2 hi) {
    const u32x4 v = {lo[0], lo[1], hi[0], hi[1]};
    return __builtin_bit_cast(bf16x8, v);
}
template <typename O, int PITCH>
__device__ __forceinline__ void read_slice(const unsigned char* lds, int row, int lane, bf16x8 (&f)[4][1], std::false_type) {
    const uint32_t p = tr_address<O, PITCH>(lds, row, lane);
    u32x2 x[4][2];   // [k-step][first, second four of eight k]
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%c9\n\t"
        "ds_read_b64_tr_b16 %2, %8 offset:%c10\n\tds_read_b64_tr_b16 %3, %8 offset:%c11\n\t"
        "ds_read_b64_tr_b16 %4, %8 offset:%c12\n\tds_read_b64_tr_b16 %5, %8 offset:%c13\n\t"
        "ds_read_b64_tr_b16 %6, %8 offset:%c14\n\tds_read_b64_tr_b16 %7, %8 offset:%c15\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1]), "=&v"(x[3][0]),
          "=&v"(x[3][1])
        : "v"(p), "i"(4 * PITCH), "i"(16 * PITCH), "i"(20 * PITCH), "i"(32 * PITCH), "i"(36 * PITCH), "i"(48 * PITCH), "i"(52 * PITCH)
        : "memory");
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) f[kk][0] = tr_frag(x[kk][0], x[kk][1]);
}
template <typename O, int PITCH>
__device__ __forceinline__ void read_slice(const unsigned char* lds, int row, int lane, bf16x8 (&f)[4][2], std::false_type) {
    const uint32_t p0 = tr_address<O, PITCH>(lds, row, lane), p1 = tr_address<O, PITCH>(lds, row + 32, lane);
    u32x2 x[4][2][2];   // [k-step][block][first, second four of eight k]
    asm volatile(
        "ds_read_b64_tr_b16 %0, %16\n\tds_read_b64_tr_b16 %1, %16 offset:%c18\n\t"
        "ds_read_b64_tr_b16 %2, %17\n\tds_read_b64_tr_b16 %3, %17 offset:%c18\n\t"
        "ds_read_b64_tr_b16 %4, %16 offset:%c19\n\tds_read_b64_tr_b16 %5, %16 offset:%c20\n\t"
        "ds_read_b64_tr_b16 %6, %17 offset:%c19\n\tds_read_b64_tr_b16 %7, %17 offset:%c20\n\t"
        "ds_read_b64_tr_b16 %8, %16 offset:%c21\n\tds_read_b64_tr_b16 %9, %16 offset:%c22\n\t"
        "ds_read_b64_tr_b16 %10, %17 offset:%c21\n\tds_read_b64_tr_b16 %11, %17 offset:%c22\n\t"
        "ds_read_b64_tr_b16 %12, %16 offset:%c23\n\tds_read_b64_tr_b16 %13, %16 offset:%c24\n\t"
        "ds_read_b64_tr_b16 %14, %17 offset:%c23\n\tds_read_b64_tr_b16 %15, %17 offset:%c24\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0][0]), "=&v"(x[0][0][1]), "=&v"(x[0][1][0]), "=&v"(x[0][1][1]), "=&v"(x[1][0][0]), "=&v"(x[1][0][1]),
          "=&v"(x[1][1][0]), "=&v"(x[1][1][1]), "=&v"(x[2][0][0]), "=&v"(x[2][0][1]), "=&v"(x[2][1][0]), "=&v"(x[2][1][1]),
          "=&v"(x[3][0][0]), "=&v"(x[3][0][1]), "=&v"(x[3][1][0]), "=&v"(x[3][1][1])
        : "v"(p0), "v"(p1), "i"(4 * PITCH), "i"(16 * PITCH), "i"(20 * PITCH), "i"(32 * PITCH), "i"(36 * PITCH), "i"(48 * PITCH),
          "i"(52 * PITCH)
        : "memory");
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int i = 0; i < 2; ++i) f[kk][i] = tr_frag(x[kk][i][0], x[kk][i][1]);
}

// Which tile a block takes: each of the eight dies (blocks go to them in
// turn) gets neighbouring ones, in columns of kGroup tiles of m, so that its
// L2 holds the operand rows its blocks share.
constexpr int kDies = 8, kGroup = 4;
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t total, uint32_t tm, uint32_t tn, uint32_t* m, uint32_t* n) {
    const uint32_t q = total / kDies, r = total % kDies, die = id % kDies;
    const uint32_t at = die * q + (die < r ? die : r) + id / kDies;
    const uint32_t strip = at / (kGroup * tn), in = at % (kGroup * tn);
    const uint32_t h = tm - strip * kGroup < kGroup ? tm - strip * kGroup : kGroup;
    *m = strip * kGroup + in % h;
    *n = in / h;
}

// Tiles of 64 or 128 a side for launches that 256 x 256 tiles would not fill
// the chip with: four waves, several blocks a CU, so that one's MFMAs run while
// another reads fragments. S - 1 slices are on their way; one barrier a slice
// says that it has landed for every wave and that the one before it is read.
// fp32, 8192 x 2048, K 2048: 505 us on tiles of 128, 136 of the matrix cores'
// 157 TFLOP/s; through registers 640.
template <Product KIND, typename T>
__global__ __launch_bounds__(T::THREADS) void product_tiles(ProductArgs a) {
    constexpr bool AK = KIND != PROD_WEIGHT, BKM = KIND == PROD_FORWARD;
    constexpr bool FINE = T::E == 4;
    using OA = Operand<typename T::T, T::BM, T::BK, T::WAVES, AK>;
    using OB = Operand<typename T::T, T::BN, T::BK, T::WAVES, BKM>;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / T::WN * T::TM, wn = wave % T::WN * T::TN;
    const uint32_t tm = (uint32_t)((a.M + T::BM - 1) / T::BM), tn = (uint32_t)((a.N + T::BN - 1) / T::BN);
    uint32_t im, in;
    tile_of(blockIdx.x, tm * tn, tm, tn, &im, &in);
    const int64_t m0 = (int64_t)im * T::BM, n0 = (int64_t)in * T::BN;
    const int slices = (int)((a.K + T::BK - 1) / T::BK);
    const int s0 = (int)((int64_t)slices * blockIdx.y / a.splits), s1 = (int)((int64_t)slices * (blockIdx.y + 1) / a.splits);
    const int64_t k0 = (int64_t)s0 * T::BK;
    const int64_t k_end = s1 == slices ? a.K : (int64_t)s1 * T::BK;
    OA oa;
    OB ob;
    oa.init(static_cast<const typename T::T*>(a.A) + (AK ? m0 * a.lda + k0 : k0 * a.lda + m0), a.lda, extent<AK, OA::C>(a.M) - m0, k_end - k0,
            wave, lane);
    ob.init(static_cast<const typename T::T*>(a.B) + (BKM ? n0 * a.ldb + k0 : k0 * a.ldb + n0), a.ldb, extent<BKM, OB::C>(a.N) - n0, k_end - k0,
            wave, lane);
    auto request = [&](unsigned char* st) {
#pragma unroll
        for (int q = 0; q < OA::Q; ++q) oa.load(q, st, wave);
#pragma unroll
        for (int q = 0; q < OB::Q; ++q) ob.load(q, st + T::A_BYTES, wave);
        oa.advance();
        ob.advance();
    };
    static_assert(OA::Q + OB::Q == T::LOADS, "every load is a whole block of one operand");

    f32x16 acc[T::FM][T::FN];
    start_sums<KIND, T>(a, acc, n0 + wn, lane);
    RowSums<T> rows;
    if constexpr (!AK && !FINE) rows.init(a, in, tn, wave % T::WN, s0);
    const int n = s1 - s0;
#pragma unroll
    for (int p = 0; p < T::S - 1; ++p) request(lds + p * T::STAGE);
    for (int s = 0; s < n; ++s) {
        // slices past the end are requested too (zeros): the count stays exact
        wait_vmcnt<(T::S - 2) * T::LOADS>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const unsigned char* st = lds + s % T::S * T::STAGE;
        Fragment<typename T::T> fa[4][T::FM], fb[4][T::FN];
        read_slice<OA, OA::PITCH>(st, wm, lane, fa, std::bool_constant<AK>{});
        read_slice<OB, OB::PITCH>(st + T::A_BYTES, wn, lane, fb, std::bool_constant<BKM>{});
        __builtin_amdgcn_sched_barrier(0);
        request(lds + (s + T::S - 1) % T::S * T::STAGE);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int i = 0; i < T::FM; ++i)
#pragma unroll
                for (int j = 0; j < T::FN; ++j) multiply(fb[kk][j], fa[kk][i], acc[i][j]);
        if constexpr (!AK && !FINE) {
            if (rows.mine()) rows.add(fa, 0);
            rows.next();
        }
    }
    if constexpr (!AK && !FINE) rows.store(a, in, tn, wave % T::WN, m0 + wm, lane);
    finish_sums<KIND, T, typename T::T>(a, acc, lds, m0 + wm, n0 + wn, m0 + T::BM <= a.M && n0 + T::BN <= a.N, wave, lane);
}

// 256 x 256 tiles, eight waves in two groups of four, one of each group on
// every SIMD, that take turns: while one group's MFMAs run, the other reads its
// next fragments and requests slices, and a barrier swaps them. A wave (128 x
// 64 of the tile) goes through a slice of 64 in four phases:
//   P0  reads B and the first half (64 rows) of A;  requests the next slice's
//       second half of A
//   C0  16 MFMAs
//   P1  reads the second half of A;  requests B and the first half of A of the
//       slice after the next
//   C1  16 MFMAs
// with the second group one phase behind. All of a slice is in registers
// shortly after its first use, so a stage is requested again early and loads
// have five to six of a slice's eight half-phases to arrive, with two stages.
//
// Requests of a slice are, in a wave's order, 6 (B and A's first half), then 2.
// Before the phase in which the first group reads either part of slice s + 1,
// every wave has at most 8 younger loads on their way: the barriers ahead of
// the first group's P phases follow a wait for that, in the first group's C
// and the second group's P phases.
struct PairTile {
    static constexpr int BM = 256, BN = 256, BK = 64, WM = 2, WN = 4, WAVES = 8, THREADS = 512;
    static constexpr int TM = BM / WM, TN = BN / WN, FM = TM / 32, FN = TN / 32;
    static constexpr int HALF_A = BM / 2 * BK * 2, B_BYTES = BN * BK * 2, STAGE = 2 * HALF_A + B_BYTES;
    static constexpr int EPI_ROWS = 32, EPI_LD = TN + 4;
    static constexpr int SMEM = 2 * STAGE;
    static_assert(WAVES * EPI_ROWS * EPI_LD * 4 <= SMEM, "the staging fits the ring");
};

template <Product KIND>
__global__ __launch_bounds__(PairTile::THREADS) void product_pairs(ProductArgs a) {
    using T = PairTile;
    constexpr bool AK = KIND != PROD_WEIGHT, BKM = KIND == PROD_FORWARD;
    using O0 = Operand<uint16_t, T::BM / 2, T::BK, T::WAVES, AK, 0>;
    using O1 = Operand<uint16_t, T::BM / 2, T::BK, T::WAVES, AK, 1>;
    using OB = Operand<uint16_t, T::BN, T::BK, T::WAVES, BKM>;
    static_assert(O0::Q == 2 && O1::Q == 2 && OB::Q == 4, "loads of a wave a slice: 6 and 2");
    extern __shared__ __align__(1024) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / T::WN, wn = wave % T::WN;
    const bool second = wave >= 4;
    const uint32_t tm = (uint32_t)((a.M + T::BM - 1) / T::BM), tn = (uint32_t)((a.N + T::BN - 1) / T::BN);
    uint32_t im, in;
    tile_of(blockIdx.x, tm * tn, tm, tn, &im, &in);
    const int64_t m0 = (int64_t)im * T::BM, n0 = (int64_t)in * T::BN;
    const int slices = (int)((a.K + T::BK - 1) / T::BK);
    const int s0 = (int)((int64_t)slices * blockIdx.y / a.splits), s1 = (int)((int64_t)slices * (blockIdx.y + 1) / a.splits);
    const int64_t k0 = (int64_t)s0 * T::BK;
    const int64_t k = (s1 == slices ? a.K : (int64_t)s1 * T::BK) - k0;
    const uint16_t* A = static_cast<const uint16_t*>(a.A) + (AK ? m0 * a.lda + k0 : k0 * a.lda + m0);
    const uint16_t* B = static_cast<const uint16_t*>(a.B) + (BKM ? n0 * a.ldb + k0 : k0 * a.ldb + n0);
    O0 o0;
    O1 o1;
    OB ob;
    o0.init(A, a.lda, extent<AK, 8>(a.M) - m0, k, wave, lane);
    o1.init(A, a.lda, extent<AK, 8>(a.M) - m0, k, wave, lane);
    ob.init(B, a.ldb, extent<BKM, 8>(a.N) - n0, k, wave, lane);
    // a stage: A's first half, its second, B
    auto request_first = [&](unsigned char* st) {
#pragma unroll
        for (int q = 0; q < OB::Q; ++q) ob.load(q, st + 2 * T::HALF_A, wave);
#pragma unroll
        for (int q = 0; q < O0::Q; ++q) o0.load(q, st, wave);
        ob.advance();
        o0.advance();
    };
    auto request_second = [&](unsigned char* st) {
#pragma unroll
        for (int q = 0; q < O1::Q; ++q) o1.load(q, st + T::HALF_A, wave);
        o1.advance();
    };

    f32x16 acc[T::FM][T::FN];
    start_sums<KIND, T>(a, acc, n0 + wn * T::TN, lane);

    RowSums<T> rows;
    if constexpr (!AK) rows.init(a, in, tn, wn, s0);

    request_first(lds);
    request_second(lds);
    request_first(lds + T::STAGE);
    auto swap = [&] {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    bf16x8 fa[4][2], fb[4][2];
    auto compute = [&](auto half) {
        constexpr int h = decltype(half)::value;
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[2 * h + i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[kk][j], fa[kk][i], acc[2 * h + i][j], 0, 0, 0);
        if constexpr (!AK) {
            if (rows.mine()) rows.add(fa, 2 * h);
        }
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        if (!second) wait_vmcnt<8>();
        swap();
    };
    auto read_a = [&](const unsigned char* half) {
        read_slice<O0, O0::PITCH>(half, wm * 64, lane, fa, std::bool_constant<AK>{});
    };
    auto end_reads = [&] {
        __builtin_amdgcn_sched_barrier(0);
        if (second) wait_loads<8>();
        else wait_lds();
        swap();
    };
    wait_loads<8>();
    swap();
    if (second) swap();
    const int n = s1 - s0;
    for (int s = 0; s < n; ++s) {
        unsigned char* st = lds + (s & 1) * T::STAGE;
        unsigned char* other = lds + T::STAGE - (s & 1) * T::STAGE;
        // requests go out while reads are waited for: behind reads that the
        // compiler waits for, ahead of those that end with their wait
        if constexpr (!BKM) request_second(other);
        if constexpr (AK) read_a(st);
        read_slice<OB, OB::PITCH>(st + 2 * T::HALF_A, wn * T::TN, lane, fb, std::bool_constant<BKM>{});
        if constexpr (!AK) read_a(st);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (BKM) request_second(other);
        end_reads();
        compute(std::integral_constant<int, 0>{});
        if constexpr (!AK) request_first(st);
        read_a(st + T::HALF_A);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (AK) request_first(st);
        end_reads();
        compute(std::integral_constant<int, 1>{});
        if constexpr (!AK) rows.next();
    }
    if (!second) swap();
    if constexpr (!AK) rows.store(a, in, tn, wn, m0 + wm * T::TM, lane);
    finish_sums<KIND, T, uint16_t>(a, acc, lds, m0 + wm * T::TM, n0 + wn * T::TN, m0 + T::BM <= a.M && n0 + T::BN <= a.N, wave, lane);
}

// ----------------------------------------------------------- few tokens
// Y for at most 32 tokens (an answering model's steps): W's rows are the work,
// read once, straight into MFMA fragments (16 x 16 x 32: a lane has 8
// consecutive k of one of 16 rows, so an instruction reads 64-byte pieces, from
// any element boundary); a block's waves share 16 rows, each a run of k, and add
// up in LDS.
template <int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void product_few(ProductArgs a) {
    constexpr int U = NT == 1 ? (WAVES == 4 ? 16 : 8) : 4;   // k-steps whose loads are on their way together
    typedef __attribute__((ext_vector_type(4))) float f32x4;
    __shared__ __align__(16) float part[WAVES][NT][16][20];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int kl = 8 * (lane >> 4);
    // rows past the edges read the last one; what they give is not stored
    const int64_t n = n0 + (lane & 15);
    const uint16_t* w = static_cast<const uint16_t*>(a.B) + (n < a.N ? n : a.N - 1) * a.ldb + kl;
    const uint16_t* x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t m = 16 * t + (lane & 15);
        x[t] = static_cast<const uint16_t*>(a.A) + (m < a.M ? m : a.M - 1) * a.lda + kl;
    }
    f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int K = (int)a.K, whole = K & ~7, steps = (K + 31) / 32;
    const int s1 = steps * (wave + 1) / WAVES;
    for (int s = steps * wave / WAVES; s < s1; s += U) {
        uint4 fw[U], fx[U][NT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool in = s + u < s1 && 32 * (s + u) + kl < whole;
            fw[u] = in ? ldg<uint4>(w + 32 * (s + u)) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int t = 0; t < NT; ++t) fx[u][t] = in ? ldg<uint4>(x[t] + 32 * (s + u)) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int t = 0; t < NT; ++t)
                acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fw[u]),
                                                                 __builtin_bit_cast(bf16x8, fx[u][t]), acc[t], 0, 0, 0);
    }
    if (whole < K && wave == WAVES - 1) {   // the last 1 to 7 of k, as the first lanes' chunk
        const bool in = lane < 16;
        const uint4 z = make_uint4(0, 0, 0, 0), f = in ? load_chunk(w + whole, K - whole, whole) : z;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint4 g = in ? load_chunk(x[t] + whole, K - whole, whole) : z;
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), __builtin_bit_cast(bf16x8, g),
                                                             acc[t], 0, 0, 0);
        }
    }
    // lane l has rows 4 (l / 16) + 0 .. 3 of token l mod 16
#pragma unroll
    for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4*>(&part[wave][t][lane & 15][4 * (lane >> 4)]) = acc[t];
    __syncthreads();
    const int id = threadIdx.x;
    if (id >= 32 * NT) return;
    const int t = id / 32, tok = id / 2 % 16, c = 8 * (id & 1);
    float v[8] = {};
#pragma unroll
    for (int g = 0; g < WAVES; ++g)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += part[g][t][tok][c + j];
    with_act(a.act, [&](auto act) {
        finish8_edge<PROD_FORWARD, decltype(act)::value, true, uint16_t>(a, 16 * t + tok, n0 + c, v);
    });
}

// ------------------------------------------------------- small fp32 products
// One 32 x 32 tile a block, its waves taking a run of k each and adding up in
// LDS: products of few tiles in one launch, spread over the chip. Operands come
// straight into the fragments of v_mfma_f32_32x32x2_f32: a lane holds four
// consecutive k of its row (16 bytes, or four rows of k), the other half of the
// wave the next four, and the order of k is the same for both operands. Bound by
// the loads' latency, a wave's 32 k at a time: 301 x 256, K 256 5.4 us.
template <bool KMAJOR>
__device__ __forceinline__ uint4 near_chunk(const float* p, int64_t ld, int64_t row, int64_t k, int n) {
    if constexpr (KMAJOR) {
        return load_chunk(p + row * ld + k, n, k);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = j < n ? ldg<uint32_t>(p + (k + j) * ld + row) : 0;
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}
constexpr int kNearWaves = 4;   // eight: equal; sixteen: 1 us more
template <Product KIND>
__global__ __launch_bounds__(64 * kNearWaves) void product_near(ProductArgs a) {
    constexpr bool AK = KIND != PROD_WEIGHT, BKM = KIND == PROD_FORWARD;
    constexpr int WAVES = kNearWaves, U = 4;   // steps of eight k whose loads are on their way together (eight: 1 us more)
    __shared__ float part[WAVES][16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t tiles_n = (a.N + 31) / 32;
    const int64_t m0 = blockIdx.x / tiles_n * 32, n0 = blockIdx.x % tiles_n * 32;
    // rows past the edges read the last one; what they give is not stored
    const int64_t m = m0 + (lane & 31) < a.M ? m0 + (lane & 31) : a.M - 1;
    const int64_t n = n0 + (lane & 31) < a.N ? n0 + (lane & 31) : a.N - 1;
    const int kl = 4 * (lane >> 5);
    const float* A = static_cast<const float*>(a.A);
    const float* B = static_cast<const float*>(a.B);
    const int64_t steps = (a.K + 7) / 8, whole = a.K & ~(int64_t)3;
    const int64_t s1 = steps * (wave + 1) / WAVES;
    f32x16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
    auto multiply = [&](const uint4& fa, const uint4& fb) {
        const uint32_t x[4] = {fa.x, fa.y, fa.z, fa.w}, y[4] = {fb.x, fb.y, fb.z, fb.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(y[j]), __uint_as_float(x[j]), acc, 0, 0, 0);
    };
    const uint4 zero = make_uint4(0, 0, 0, 0);
    for (int64_t s = steps * wave / WAVES; s < s1; s += U) {
        uint4 fa[U], fb[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t k = 8 * (s + u) + kl;
            const bool in = s + u < s1 && k < whole;
            fa[u] = in ? near_chunk<AK>(A, a.lda, m, k, 4) : zero;
            fb[u] = in ? near_chunk<BKM>(B, a.ldb, n, k, 4) : zero;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) multiply(fa[u], fb[u]);
    }
    if (whole < a.K && wave == WAVES - 1) {   // the last 1 to 3 of k, of the first half
        const int left = kl ? 0 : (int)(a.K - whole);
        multiply(left ? near_chunk<AK>(A, a.lda, m, whole, left) : zero, left ? near_chunk<BKM>(B, a.ldb, n, whole, left) : zero);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) part[wave][r][lane] = acc[r];
    __syncthreads();
    // lane l of the sums has row l mod 32 and, in registers 4 q .. 4 q + 3,
    // columns 8 q + 4 (l / 32) + 0 .. 3; a thread finishes eight of a row
    const int id = threadIdx.x;
    if (id >= 128) return;
    const int r = id & 31, q = id >> 5;
    float v[8] = {};
#pragma unroll
    for (int g = 0; g < WAVES; ++g)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += part[g][4 * q + (j & 3)][r + 32 * (j >> 2)];
    with_act_of<KIND>(a.act, [&](auto act) {
        finish8_edge<KIND, decltype(act)::value, true, float>(a, m0 + r, n0 + 8 * q, v);
    });
}

// Copies of operands in whole chunks of 16 bytes, zeros behind each row: a chunk
// a thread; blockIdx.y is the operand. ld and width count two bytes.
struct CopyArgs {
    const uint16_t* from[2];
    uint16_t* to[2];
    int64_t ld[2], rows[2], width[2];
};
__global__ __launch_bounds__(256) void copy_chunks(CopyArgs a) {
    const int o = blockIdx.y;
    const int64_t chunks = (a.width[o] + 7) / 8, total = a.rows[o] * chunks;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / chunks, c = i % chunks * 8;
        const int n = a.width[o] - c < 8 ? (int)(a.width[o] - c) : 8;
        stg(a.to[o] + 8 * i, load_chunk(a.from[o] + r * a.ld[o] + c, n, c));
    }
}

// Adds the parts of a split product in order and finishes its entries: one
// wave a 32 x 32 block.
template <Product KIND, typename T>
__global__ __launch_bounds__(64) void product_join(ProductArgs a) {
    const int64_t mb = (a.M + 31) / 32, nb = (a.N + 31) / 32;
    const float* p = a.part + (int64_t)blockIdx.x * 1024 + threadIdx.x * 4;
    f32x16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
    constexpr int U = 8;   // parts on their way together (one by one: 0.3 us a part, 6 of 20 where there are 32)
    for (int s = 0; s < a.splits; s += U) {
        float4 x[U][4];
#pragma unroll
        for (int u = 0; u < U; ++u, p += mb * nb * 1024)
#pragma unroll
            for (int q = 0; q < 4; ++q) x[u][q] = s + u < a.splits ? ldg<float4>(p + 256 * q) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                acc[4 * q] += x[u][q].x;
                acc[4 * q + 1] += x[u][q].y;
                acc[4 * q + 2] += x[u][q].z;
                acc[4 * q + 3] += x[u][q].w;
            }
    }
    const int64_t m0 = blockIdx.x / nb * 32, n0 = blockIdx.x % nb * 32;
    with_act_of<KIND>(a.act, [&](auto act) {
        each_row_of_8(acc, threadIdx.x, [&](int r, int c, float (&v)[8]) {
            finish8_edge<KIND, decltype(act)::value, true, T>(a, m0 + r, n0 + c, v);
        });
    });
}

template <typename T> using MiddleTile = Tile<T, 128, 128, 128 / sizeof(T), 2, 2, 2>;
template <typename T> using SmallTile = Tile<T, 64, 64, 128 / sizeof(T), 4, 2, 2>;

enum Form { FORM_ANY, FORM_ANY_64, FORM_NEAR, FORM_FEW, FORM_SMALL, FORM_MIDDLE, FORM_BIG };
struct Plan {
    Form form;
    int splits;
    bool copy_a, copy_b;   // the operand is copied in whole chunks first
};

// An operand as it is stored: outer rows of inner entries.
struct Stored {
    const void* p;
    int64_t ld, outer, inner;
    int e;   // bytes an entry
    // Rows are whole chunks of 16 bytes from one 16-byte boundary to the next.
    // Sizes and pitches alone say whether a copy is needed, so that the
    // workspace can be told in advance; of the others the pointer must be aligned.
    bool whole() const { return ld * e % 16 == 0 && inner * e % 16 == 0 && ld < (int64_t(1) << 21); }
    bool aligned() const { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
    int64_t chunks() const { return (inner * e + 15) / 16; }   // a row
    size_t copy_bytes() const { return ((size_t)outer * chunks() * 16 + 255) & ~size_t(255); }
};
Stored stored_a(Product kind, const ProductArgs& a) {
    if (kind == PROD_WEIGHT) return {a.A, a.lda, a.K, a.M, a.bf16 ? 2 : 4};
    return {a.A, a.lda, a.M, a.K, a.bf16 ? 2 : 4};
}
Stored stored_b(Product kind, const ProductArgs& a) {
    if (kind == PROD_FORWARD) return {a.B, a.ldb, a.N, a.K, a.bf16 ? 2 : 4};
    return {a.B, a.ldb, a.K, a.N, a.bf16 ? 2 : 4};
}

int64_t tiles_of(int64_t M, int64_t N, int bm, int bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); }

size_t part_bytes(const ProductArgs& a, int splits) { return splits > 1 ? (size_t)splits * tiles_of(a.M, a.N, 32, 32) * 4096 : 0; }

// A launch's time by its tiles: 256 CUs take up to `most` tiles each at a time,
// and such a round lasts `fixed` us (the start and the epilogue) plus, for every
// 64 of K, unit[n - 1] us where a CU holds n tiles. Measured in graphs of 30
// calls at 64 to 4096 tokens, rows and columns; the model is within a fifth of
// the measurements, the forms it decides between are often twice apart:
//   1024 x 1024, K 1024:  64 6.2, 128 12.0 us;  1024 x 2048:  8.6, 12.4
//   2048 x 4096, K 1024:  64 30, 128 21.8, 256 28.6
//   2048 x 8192, K 2048:  64 107, 128 69, 256 58.7
// A product cut into parts adds their round trip through the caches at 8 TB/s
// and a launch: 2048 x 2048, K 8192 on 128 x 128 tiles 86.6 whole, 73.3 in two;
// 64 x 2048, K 8192 on 64 x 64 tiles 28 whole, 13.2 in eight.
// fp32 on tiles of 32, 64, 128 and, through registers, 64 and 128: 301 x 256, K 256
// 5.7, 7.9, -, 8.9, -; 512 x 512, K 512 7.8, 10.7, -, 12.7, -; 2048 x 512, K 512 22.6,
// 13.3, -, 22.2, -; 2048 x 2048, K 2048 -, 143, 137, -, 177.
struct Cost {
    int tile, most;
    double fixed, unit[4];
};
constexpr Cost kNearCost = {32, 4, 3.6, {0.42, 1.1, 1.6, 2.2}};
constexpr Cost kSmallCost[2] = {{64, 2, 2.7, {1.0, 2.0}}, {64, 2, 2.7, {0.21, 0.38}}};   // fp32, bf16
constexpr Cost kMiddleCost[2] = {{128, 2, 4.0, {4.0, 7.5}}, {128, 2, 5.5, {0.65, 0.93}}};
constexpr Cost kBigCost = {256, 1, 10.0, {1.5}};
constexpr Cost kAny64Cost[2] = {{64, 4, 2.7, {2.3, 3.2, 4.3, 5.5}}, {64, 4, 2.7, {0.6, 0.9, 1.05, 1.2}}};
constexpr Cost kAnyCost[2] = {{128, 2, 4.0, {6.1, 10.4}}, {128, 2, 4.0, {1.5, 2.0}}};

double time_of(const Cost& c, const ProductArgs& a, int splits, double slow) {
    const int64_t tiles = tiles_of(a.M, a.N, c.tile, c.tile) * splits;
    const double units = slow * (double)((a.K + 63) / 64) / splits;
    const int64_t rounds = tiles / (256 * c.most), left = (tiles % (256 * c.most) + 255) / 256;
    double t = rounds * (c.fixed + units * c.unit[c.most - 1]);
    if (left) t += c.fixed + units * c.unit[left - 1];
    if (splits > 1) t += 2.5 + 0.1 * splits + (double)splits * a.M * a.N * 8 / 8e6;
    return t;
}

// Copies cost a launch and their bytes at 4 TB/s. Forward, input and weight
// gradient of 8191 tokens through 2047 x 2041: 77, 76 and 107 us with copies, on
// tiles of any alignment 144, 202 and 284; 1531 tokens through 1000 x 517: 12.5,
// 10.6, 13.3 and 10.3, 18.7, 16.4, in fp32 30, 28, 36 and 32, 35, 39.
// Beyond kCopiesMost they would hold more memory than that time is worth.
constexpr size_t kCopiesMost = size_t(2) << 30;
// Parts are for few output tiles: on 512 of 256 x 256 (two rounds) four of them
// are 512 MiB. More is refused, and so is a cut that by the model gains less than
// a twentieth over the same tiles' whole sums, well inside what it is off by:
// 262144 tokens through 32000 x 8192 would take 4 GB of parts for 0.02% of 98 ms.
constexpr size_t kPartsMost = size_t(512) << 20;
constexpr double kPartsWorth = 1.05;
constexpr int64_t kNearTiles = 1 << 16;   // none of its wins has more, and a launch takes them
Plan plan_of(Product kind, const ProductArgs& a) {
    Plan best{FORM_FEW, 1, false, false};
    const Stored sa = stored_a(kind, a), sb = stored_b(kind, a);
    const bool copy_a = !sa.whole(), copy_b = !sb.whole();
    const size_t copied = (copy_a ? sa.copy_bytes() : 0) + (copy_b ? sb.copy_bytes() : 0);
    const bool direct = (copy_a || sa.aligned()) && (copy_b || sb.aligned()) && copied <= kCopiesMost;
    if (a.bf16 && kind == PROD_FORWARD && a.M <= 32) return best;
    double least = 0.0;
    // slow: of the units; more: us once
    auto offer = [&](Form form, const Cost& c, double slow, double more, bool ca, bool cb) {
        const double whole = time_of(c, a, 1, slow) + more;
        for (int splits = 1; splits <= 32 && (splits == 1 || (a.K + 63) / 64 >= splits); splits *= 2) {
            if (part_bytes(a, splits) > kPartsMost) break;
            const double t = splits == 1 ? whole : time_of(c, a, splits, slow) + more;
            if (splits > 1 && t * kPartsWorth > whole) continue;
            if (best.form == FORM_FEW || t < least) {
                best = {form, splits, ca, cb};
                least = t;
            }
        }
    };
    if (direct) {
        const double more = copy_a || copy_b ? 5.0 + 2.0 * copied / 4e6 : 0.0;
        if (a.bf16) offer(FORM_BIG, kBigCost, 1.0, more, copy_a, copy_b);
        offer(FORM_MIDDLE, kMiddleCost[a.bf16], 1.0, more, copy_a, copy_b);
        offer(FORM_SMALL, kSmallCost[a.bf16], 1.0, more, copy_a, copy_b);
    }
    if (!direct || copy_a || copy_b) {
        // rows of odd width read across: in bf16 1.1 to 2.2 times a unit's time, by
        // 1.4 for each m/n-contiguous operand; in fp32 up to 1.3
        const double across = a.bf16 ? 1.4 : 1.15;
        double slow = 1.0;
        if (copy_a && kind == PROD_WEIGHT) slow *= across;
        if (copy_b && kind != PROD_FORWARD) slow *= across;
        offer(FORM_ANY, kAnyCost[a.bf16], slow, 0.0, false, false);
        offer(FORM_ANY_64, kAny64Cost[a.bf16], slow, 0.0, false, false);
    }
    if (!a.bf16 && tiles_of(a.M, a.N, 32, 32) < kNearTiles && time_of(kNearCost, a, 1, 1.0) < least)
        best = {FORM_NEAR, 1, false, false};
    return best;
}

template <typename T, typename F>
hipError_t launch_tiles(F kernel, const ProductArgs& a, hipStream_t s) {
    static_assert(T::SMEM <= 160 * 1024, "LDS of a CU");
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, T::SMEM);
    if (e != hipSuccess) return e;
    kernel<<<dim3((unsigned)tiles_of(a.M, a.N, T::BM, T::BN), (unsigned)a.splits), T::THREADS, T::SMEM, s>>>(a);
    return hipGetLastError();
}

template <Product KIND, typename T, int GT>
hipError_t launch_any(const ProductArgs& a, hipStream_t s) {
    product_any<KIND, T, GT><<<dim3((unsigned)tiles_of(a.M, a.N, GT, GT), (unsigned)a.splits), kGThreads, 0, s>>>(a);
    return hipGetLastError();
}

// One token through 8192 x 2048: four waves a block 7.9 us, eight 8.3, sixteen
// 10.3; through 2048 x 8192, where sixteen are needed to have as many loads on
// their way, 12.0.
hipError_t launch_few(const ProductArgs& a, hipStream_t s) {
    const unsigned blocks = (unsigned)((a.N + 15) / 16);
    if (a.M > 16) product_few<2, 8><<<blocks, 512, 0, s>>>(a);
    else if (blocks < 256 && a.K >= 4096) product_few<1, 16><<<blocks, 1024, 0, s>>>(a);
    else product_few<1, 4><<<blocks, 256, 0, s>>>(a);
    return hipGetLastError();
}

template <Product KIND, typename T>
hipError_t launch_kind(const ProductArgs& a, Form form, hipStream_t s) {
    hipError_t e = hipSuccess;
    if constexpr (std::is_same<T, uint16_t>::value) {
        if (form == FORM_BIG) e = launch_tiles<PairTile>(&product_pairs<KIND>, a, s);
        else if (form == FORM_FEW) return launch_few(a, s);
    }
    if constexpr (std::is_same<T, float>::value) {
        if (form == FORM_NEAR) {
            product_near<KIND><<<(unsigned)tiles_of(a.M, a.N, 32, 32), 64 * kNearWaves, 0, s>>>(a);
            return hipGetLastError();
        }
    }
    if (form == FORM_MIDDLE) e = launch_tiles<MiddleTile<T>>(&product_tiles<KIND, MiddleTile<T>>, a, s);
    else if (form == FORM_SMALL) e = launch_tiles<SmallTile<T>>(&product_tiles<KIND, SmallTile<T>>, a, s);
    else if (form == FORM_ANY) e = launch_any<KIND, T, 128>(a, s);
    else if (form == FORM_ANY_64) e = launch_any<KIND, T, 64>(a, s);
    if (e != hipSuccess || a.splits == 1) return e;
    product_join<KIND, T><<<(unsigned)tiles_of(a.M, a.N, 32, 32), 64, 0, s>>>(a);
    return hipGetLastError();
}

template <Product KIND>
hipError_t launch_type(const ProductArgs& a, Form form, hipStream_t s) {
    return a.bf16 ? launch_kind<KIND, uint16_t>(a, form, s) : launch_kind<KIND, float>(a, form, s);
}

size_t copy_bytes(Product kind, const ProductArgs& a, const Plan& p) {
    return (p.copy_a ? stored_a(kind, a).copy_bytes() : 0) + (p.copy_b ? stored_b(kind, a).copy_bytes() : 0);
}

// The copies that the plan asks for, at the workspace's start; the product then
// reads them, and its parts follow.
hipError_t make_copies(Product kind, ProductArgs& a, const Plan& p, hipStream_t s) {
    CopyArgs c{};
    int n = 0;
    char* to = reinterpret_cast<char*>(a.part);
    int64_t chunks = 0;
    auto add = [&](const Stored& o, const void** pointer, int64_t* ld) {
        c.from[n] = static_cast<const uint16_t*>(o.p);
        c.to[n] = reinterpret_cast<uint16_t*>(to);
        c.ld[n] = o.ld * o.e / 2; c.rows[n] = o.outer; c.width[n] = o.inner * o.e / 2;
        chunks = std::max(chunks, o.outer * o.chunks());
        *pointer = to;
        *ld = o.chunks() * 16 / o.e;
        to += o.copy_bytes();
        ++n;
    };
    if (p.copy_a) add(stored_a(kind, a), &a.A, &a.lda);
    if (p.copy_b) add(stored_b(kind, a), &a.B, &a.ldb);
    a.part = reinterpret_cast<float*>(to);
    if (!n || !chunks) return hipSuccess;
    copy_chunks<<<dim3((unsigned)std::min<int64_t>((chunks + 255) / 256, 8192), (unsigned)n), 256, 0, s>>>(c);
    return hipGetLastError();
}

size_t plan_bytes(Product kind, const ProductArgs& a, const Plan& p) {
    return copy_bytes(kind, a, p) + part_bytes(a, p.splits);
}

}  // namespace

size_t product_workspace(Product kind, const ProductArgs& a) { return plan_bytes(kind, a, plan_of(kind, a)); }

int64_t product_row_sums(const ProductArgs& a) {
    const Plan p = plan_of(PROD_WEIGHT, a);
    const int tile = !a.bf16 ? 0 : p.form == FORM_BIG ? 256 : p.form == FORM_MIDDLE ? 128 : p.form == FORM_SMALL ? 64 : 0;
    const int waves = p.form == FORM_BIG ? PairTile::WN : 2;
    return tile ? (int64_t)p.splits * waves * ((a.N + tile - 1) / tile) : 0;
}

size_t product_workspace_most(Product kind, ProductArgs a) {
    // the most over what the pointers can be: aligned or not
    size_t most = 0;
    for (uintptr_t at : {(uintptr_t)0, (uintptr_t)2}) {
        a.A = a.B = reinterpret_cast<const void*>(at);
        const size_t sums = kind == PROD_WEIGHT ? (size_t)product_row_sums(a) * a.M * 4 : 0;
        most = std::max(most, product_workspace(kind, a) + sums);
    }
    return most;
}

hipError_t launch_product(Product kind, ProductArgs a, hipStream_t s) {
    if (a.M == 0 || a.N == 0) return hipSuccess;
    const Plan p = plan_of(kind, a);
    a.splits = p.splits;
    hipError_t e = make_copies(kind, a, p, s);
    if (e != hipSuccess) return e;
    if (kind == PROD_FORWARD) return launch_type<PROD_FORWARD>(a, p.form, s);
    if (kind == PROD_INPUT) return launch_type<PROD_INPUT>(a, p.form, s);
    return launch_type<PROD_WEIGHT>(a, p.form, s);
}

}  // namespace dion2
