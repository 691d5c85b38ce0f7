// Activations kept in 8 bits: packing, unpacking, and the (gated) activation's two passes.
#include <type_traits>

#include "act8.cuh"

namespace ss {
namespace {

// f and f' in fp32, with the hardware's exponential and reciprocal (each within two units in the
// last place; the results are held to 1e-6 of |x|, and stored in 8 or 24 bits).
//   silu: s = 1 / (1 + exp(-x)), f = x s, f' = s (1 + x (1 - s))
//   gelu: f = x Phi(x), f' = Phi(x) + x phi(x), phi(x) = exp(-x^2 / 2) / sqrt(2 pi)
// Phi(-|x|) = exp(-x^2 / 2) P(u), u = 1 / (1 + p |x|), the form of Hastings' approximations of erfc
// (Approximations for Digital Computers, 1955). p and the coefficients of P, of degree 6 without a
// constant, were fitted for this kernel to erfcx on [0, 10], to 1e-8 of Phi; evaluated in fp32 Phi is within 2.4e-7, and
// x Phi(x) within 3.8e-7 over [-9, 9] (PyTorch's fp32 GELU: 4.9e-7). It shares the
// exponential with f' and costs half of erff: with erff the bf16 kernels were bound by
// instructions (285 us instead of 197 us at 16384 x 8192, gated).
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ float reciprocal_fast(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ float sigmoid_fast(float x) { return reciprocal_fast(1.0f + exp2_fast(x * -1.4426950408889634f)); }

__device__ __forceinline__ float normal_cdf(float x, float* exp_half_square) {
    const float e = exp2_fast(x * x * -0.72134752044448170f), u = reciprocal_fast(fmaf(0.275771645f, fabsf(x), 1.0f));
    float q = fmaf(-0.113644886f, u, 0.442823028f);
    q = fmaf(q, u, -0.316866405f);
    q = fmaf(q, u, 0.324101073f);
    q = fmaf(q, u, 0.0459687229f);
    q = fmaf(q, u, 0.11761847f);
    q *= u * e;
    *exp_half_square = e;
    return x < 0.0f ? q : 1.0f - q;
}

template <int ACT>
__device__ __forceinline__ float act_value(float x) {
    if constexpr (ACT == SS_ACT_SILU) {
        return x * sigmoid_fast(x);
    } else {
        float e;
        return x * normal_cdf(x, &e);
    }
}

template <int ACT>
__device__ __forceinline__ void act_value_slope(float x, float* f, float* slope) {
    if constexpr (ACT == SS_ACT_SILU) {
        const float s = sigmoid_fast(x);
        *f = x * s;
        *slope = s * fmaf(x, 1.0f - s, 1.0f);
    } else {
        float e;
        const float cdf = normal_cdf(x, &e);
        *f = x * cdf;
        *slope = fmaf(x * 0.39894228040143268f, e, cdf);
    }
}

// ---- pieces of 8 columns ---------------------------------------------------------------------------
// A thread takes 8 columns of a row, four neighbouring lanes a group of 32. Pieces are numbered in
// the checkpoint's order, so its values and exponents are read and written in one run; row and
// column follow by a division.
//
// Bound by memory where rows start on 16 bytes: 16384 x 8192 bf16, gated silu, forward 176 and backward 176
// us (6.1 TB/s; DRAM at 67-69 % of its nominal rate, instructions issued in 72 % of the cycles); gated gelu 203 and 199, the
// instructions' share; pack 74 us (5.5 TB/s; fp32 96, 7.0 TB/s; 16384 x 4096 bf16 37), unpack 68; the gated silu forward that keeps
// nothing 115 (7.0 TB/s). Rows at odd places cost
// the shifting of vectors: 4099 x 2731 gated silu 29.1 and 26.7 us in a row of calls (3.2 TB/s), the integer pipe 70 % busy; a column
// to a thread, element by element, took 149 us for both passes.
constexpr int kPiece = 8;
constexpr int kBlock = 256;

// Where rows do not start on 16 bytes: threads over which stored vectors are put together. A block's
// for bf16 (gated silu 16384 x 8191, forward and backward: 280 and 246 us; a warp's 284 and 281), a warp's for
// fp32 (8192 x 8191: 188 and 166 us; a block's 195 and 174).
template <typename T>
constexpr int kRun = sizeof(T) == 2 ? kBlock : 32;
// Blocks that an SM holds at least. (Without the bound on registers the same took 309 and 268 us in bf16, 211 and 182 in
// fp32; with one more block 268 and 266, and 190 and 168.)
template <typename T>
constexpr int kBlocks = sizeof(T) == 2 ? 5 : 4;

struct Pieces {
    int64_t groups;      // of one row
    int64_t total;       // pieces: rows * groups * 4
    int64_t cols;
    uint32_t mul;        // n / groups = (n * mul) >> (32 + shift) for n < 2^31
    int shift;           // -1: groups == 1, -2: too many for 32 bits

    __device__ __forceinline__ int64_t row_of(int64_t g) const {
        if (shift >= 0) return __umulhi(static_cast<uint32_t>(g), mul) >> shift;
        return shift == -1 ? g : g / groups;
    }
};

// With l = ceil(log2 d) and m = ceil(2^(31+l) / d) < 2^32: n m = n 2^(31+l) / d + n r with r < 1, and
// n r < 2^31 does not reach the next multiple of 2^(31+l) / d for n < 2^31.
Pieces pieces_of(int64_t rows, int64_t cols) {
    Pieces p{act8_groups(cols), 0, cols, 0, -2};
    p.total = rows * p.groups * 4;
    if (p.groups == 1) {
        p.shift = -1;
    } else if (rows * p.groups < (int64_t(1) << 31)) {
        int l = 1;
        while ((int64_t(1) << l) < p.groups) ++l;
        p.mul = static_cast<uint32_t>(((uint64_t(1) << (31 + l)) + p.groups - 1) / p.groups);
        p.shift = l - 1;
    }
    return p;
}

// One matrix of a call. In a kernel for aligned rows every row starts on 16 bytes.
struct Side {
    void* p;
    int64_t stride;  // elements
    int64_t bytes;   // extent
};

// Words s .. of a run of words, and half a word further if `half`.
template <int N, int KEEP>
__device__ __forceinline__ void shift_words(uint32_t (&w)[N], uint32_t s, bool half) {
#pragma unroll
    for (int i = 0; i + 2 < N; ++i) w[i] = (s & 2) ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i + 1 < N; ++i) w[i] = (s & 1) ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < KEEP; ++i) w[i] = half ? __funnelshift_r(w[i], w[i + 1], 16) : w[i];
}

template <typename T>
struct Eight {
    static constexpr int kWords = kPiece * sizeof(T) / 4;
    uint32_t w[kWords];

    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float((i & 1) ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
    }
    __device__ __forceinline__ void set(const float (&v)[kPiece]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < kPiece; ++i) w[i] = __float_as_uint(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kPiece; i += 2) w[i >> 1] = bf16_pair(v[i], v[i + 1]);
        }
    }

    // `n` columns that exist (0 .. 8) from p on; the others are 0. Rows that do not start on 16
    // bytes are read as the aligned vectors around the piece, shifted into place, where all of
    // those lie within the matrix.
    template <bool ALIGNED>
    __device__ __forceinline__ void load(const Side& m, const T* p, int n) {
        if (ALIGNED && n == kPiece) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const uint4 v = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint32_t*>(p) + i);
                w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
            }
            return;
        }
        const uintptr_t at = reinterpret_cast<uintptr_t>(p), begin = reinterpret_cast<uintptr_t>(m.p);
        const uintptr_t base = at & ~static_cast<uintptr_t>(15);
        if (!ALIGNED && n == kPiece && base >= begin && base + 4 * kWords + 16 <= begin + m.bytes) {
            uint32_t x[kWords + 4];
#pragma unroll
            for (int i = 0; i < kWords + 4; i += 4) {
                const uint4 v = *reinterpret_cast<const uint4*>(base + 4 * i);
                x[i] = v.x, x[i + 1] = v.y, x[i + 2] = v.z, x[i + 3] = v.w;
            }
            shift_words<kWords + 4, kWords>(x, (at & 15) >> 2, sizeof(T) == 2 && (at & 2) != 0);
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = x[i];
            return;
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            if (i >= n) break;
            if constexpr (sizeof(T) == 4) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
            else w[i >> 1] |= static_cast<uint32_t>(p[i]) << (16 * (i & 1));
        }
    }

    __device__ __forceinline__ void store_some(T* p, int from, int to) const {
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            if (i < from || i >= to) continue;
            if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t*>(p)[i] = w[i];
            else p[i] = static_cast<T>(w[i >> 1] >> (16 * (i & 1)));
        }
    }

    // Where rows do not start on 16 bytes, the aligned vectors that begin in the previous piece
    // are put together from the thread before, so that all but the ends of a row, or of a run of
    // kRun threads, are whole vectors. `joined`: the thread before holds the piece before, whole; `follows`:
    // so does this one for the next. hand_on() comes before, and between the two every thread of the block
    // waits for the others; a place in `ends` is used once.
    template <bool ALIGNED>
    __device__ __forceinline__ void hand_on(uint4* ends) const {
        if (!ALIGNED && kRun<T> > 32 && (threadIdx.x & 31) == 31) ends[threadIdx.x >> 5] = make_uint4(w[kWords - 4], w[kWords - 3], w[kWords - 2], w[kWords - 1]);
    }
    template <bool ALIGNED>
    __device__ __forceinline__ void store(T* p, int n, bool joined, bool follows, const uint4* ends) const {
        if (ALIGNED) {
            if (n == kPiece) {
#pragma unroll
                for (int i = 0; i < kWords; i += 4)
                    *reinterpret_cast<uint4*>(reinterpret_cast<uint32_t*>(p) + i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
            } else {
                store_some(p, 0, n);
            }
            return;
        }
        uint32_t x[kWords + 4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __shfl_up_sync(0xFFFFFFFFu, w[kWords - 4 + i], 1);
#pragma unroll
        for (int i = 0; i < kWords; ++i) x[4 + i] = w[i];
        if (kRun<T> > 32 && (threadIdx.x & 31) == 0 && joined) {
            const uint4 v = ends[(threadIdx.x >> 5) - 1];
            x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
        }
        const uint32_t m = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 15u;
        const bool vector = joined && n == kPiece;  // writes from its aligned address on
        const int end = follows ? kPiece - static_cast<int>(m / sizeof(T)) : n;
        if (vector) {
            const uint32_t o = 16u - m;  // of the run, from where the vectors are taken
            if (o < 16u) {
                shift_words<kWords + 4, kWords>(x, o >> 2, sizeof(T) == 2 && (o & 2) != 0);
            } else {
#pragma unroll
                for (int i = 0; i < kWords; ++i) x[i] = w[i];
            }
            uint4* q = reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(p) & ~static_cast<uintptr_t>(15));
#pragma unroll
            for (int i = 0; i < kWords; i += 4) q[i / 4] = make_uint4(x[i], x[i + 1], x[i + 2], x[i + 3]);
            if (!follows) store_some(p, kPiece - static_cast<int>(m / sizeof(T)), kPiece);
        } else {
            store_some(p, 0, end);
        }
    }
};

// Largest magnitude of a piece, as the bits of an fp32.
__device__ __forceinline__ uint32_t largest(const Eight<float>& v) {
    uint32_t a = 0;
#pragma unroll
    for (int j = 0; j < kPiece; ++j) a = max(a, v.w[j] & 0x7FFFFFFFu);
    return a;
}

__device__ __forceinline__ uint32_t largest(const Eight<uint16_t>& v) {
    uint32_t a = v.w[0] & 0x7FFF7FFFu;
#pragma unroll
    for (int j = 1; j < 4; ++j) a = __vmaxu2(a, v.w[j] & 0x7FFF7FFFu);
    return max(a & 0xFFFF0000u, a << 16);
}

// Codes of columns 4 h .. 4 h + 3: magnitudes from the low bytes, signs from the top bits.
__device__ __forceinline__ uint32_t codes(const Eight<float>& v, int h, uint32_t exp_byte) {
    const float inverse = act8_inverse(exp_byte);
    const uint32_t* w = v.w + 4 * h;
    uint32_t m[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) m[j] = act8_magnitude(__uint_as_float(w[j]), inverse);
    const uint32_t q = __byte_perm(__byte_perm(m[0], m[1], 0x0040), __byte_perm(m[2], m[3], 0x0040), 0x5410);
    const uint32_t s = __byte_perm(__byte_perm(w[0], w[1], 0x0073), __byte_perm(w[2], w[3], 0x0073), 0x5410);
    return (q & 0x7F7F7F7Fu) | (s & 0x80808080u);
}

__device__ __forceinline__ uint32_t codes(const Eight<uint16_t>& v, int h, uint32_t exp_byte) {
    const uint32_t inverse = __float_as_uint(act8_inverse(exp_byte)), pair = inverse | (inverse >> 16);
    const uint32_t* w = v.w + 2 * h;
    const uint32_t lo = act8_magnitude_pair(w[0] & 0x7FFF7FFFu, pair), hi = act8_magnitude_pair(w[1] & 0x7FFF7FFFu, pair);
    return (__byte_perm(lo, hi, 0x6420) & 0x7F7F7F7Fu) | (__byte_perm(w[0], w[1], 0x7531) & 0x80808080u);
}

// A piece to the checkpoint; every lane of the warp calls it.
template <typename T>
__device__ __forceinline__ void keep(const Ckpt& c, int64_t i, bool in, const Eight<T>& v) {
    uint32_t a = largest(v);
    a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
    a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
    const uint32_t e = act8_exp_byte(a);
    if (!in) return;
    *reinterpret_cast<uint2*>(c.values + i * kPiece) = make_uint2(codes(v, 0, e), codes(v, 1, e));
    if ((i & 3) == 0) c.exps[i >> 2] = static_cast<uint8_t>(e);
}

struct Kept {
    uint2 w;
    uint32_t e;
    __device__ __forceinline__ void load(const Ckpt& c, int64_t i) {
        w = *reinterpret_cast<const uint2*>(c.values + i * kPiece);
        e = c.exps[i >> 2];
    }
    // The eight values, exact in bf16.
    __device__ __forceinline__ Eight<uint16_t> values() const {
        const uint32_t e2 = act8_exponent_pair(e);
        Eight<uint16_t> v;
        v.w[0] = act8_value_pair<0>(w.x, e2), v.w[1] = act8_value_pair<1>(w.x, e2);
        v.w[2] = act8_value_pair<0>(w.y, e2), v.w[3] = act8_value_pair<1>(w.y, e2);
        return v;
    }
};

// Where a thread's piece lies.
template <typename T>
struct At {
    int64_t i, row, col;
    int n;  // columns that exist; 0 beyond the last piece
    bool in, joined, follows;

    __device__ __forceinline__ At(const Pieces& p, int u) {
        i = (static_cast<int64_t>(blockIdx.x) * 2 + u) * kBlock + threadIdx.x;
        in = i < p.total;
        const int64_t g = (in ? i : 0) >> 2;
        row = p.row_of(g);
        const int64_t piece = (i & 3) + (g - row * p.groups) * 4;
        col = piece * kPiece;
        const int64_t left = p.cols - col;
        n = !in || left <= 0 ? 0 : (left >= kPiece ? kPiece : static_cast<int>(left));
        joined = in && piece > 0 && threadIdx.x % kRun<T> != 0;
        follows = in && left >= 2 * kPiece && threadIdx.x % kRun<T> != kRun<T> - 1;
    }
    __device__ __forceinline__ T* of(const Side& m) const {
        return static_cast<T*>(m.p) + row * m.stride + col;
    }
};

// A block takes 2 * 256 pieces, both loads of a thread under way before the first is used.
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kBlock) act8_pack_kernel(const __grid_constant__ Pieces p, const __grid_constant__ Side x, const __grid_constant__ Ckpt c) {
    const At<T> at[2] = {At<T>(p, 0), At<T>(p, 1)};
    Eight<T> v[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) v[u].template load<ALIGNED>(x, at[u].of(x), at[u].n);
#pragma unroll
    for (int u = 0; u < 2; ++u) keep(c, at[u].i, at[u].in, v[u]);
}

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kBlock) act8_unpack_kernel(const __grid_constant__ Pieces p, const __grid_constant__ Ckpt c, const __grid_constant__ Side out) {
    const At<T> at[2] = {At<T>(p, 0), At<T>(p, 1)};
    __shared__ uint4 ends[ALIGNED ? 1 : 2][kBlock / 32];
    Kept k[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
        if (at[u].in) k[u].load(c, at[u].i);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const Eight<uint16_t> kept = k[u].values();
        Eight<T> v;
        if constexpr (sizeof(T) == 2) {
            v = kept;
        } else {
#pragma unroll
            for (int j = 0; j < kPiece; ++j) v.w[j] = __float_as_uint(kept.get(j));
        }
        uint4* const end = ends[ALIGNED ? 0 : u];
        v.template hand_on<ALIGNED>(end);
        if constexpr (!ALIGNED && kRun<T> > 32) __syncthreads();
        v.template store<ALIGNED>(at[u].of(out), at[u].n, at[u].joined, at[u].follows, end);
    }
}

struct Forward {
    Pieces p;
    Side x, up, y;
    Ckpt cx, cu, cy;
};

// KEEP: the inputs' checkpoints are written. (A test of the pointer in the kernel instead: gated silu 4099 x 2736 bf16 20.5 us
// instead of 19.7, 16384 x 8192 172.6 instead of 170.3.)
template <typename T, int ACT, bool GATED, bool ALIGNED, bool KEEP>
__global__ void __launch_bounds__(kBlock, kBlocks<T>) act8_forward_kernel(const __grid_constant__ Forward a) {
    const At<T> at[2] = {At<T>(a.p, 0), At<T>(a.p, 1)};
    __shared__ uint4 ends[ALIGNED ? 1 : 2][kBlock / 32];
    Eight<T> x[2], up[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        x[u].template load<ALIGNED>(a.x, at[u].of(a.x), at[u].n);
        if constexpr (GATED) up[u].template load<ALIGNED>(a.up, at[u].of(a.up), at[u].n);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        float f[kPiece];
#pragma unroll
        for (int j = 0; j < kPiece; ++j) {
            f[j] = act_value<ACT>(x[u].get(j));
            if constexpr (GATED) f[j] *= up[u].get(j);
        }
        Eight<T> y;  // columns that do not exist: f(0) = 0
        y.set(f);
        uint4* const end = ends[ALIGNED ? 0 : u];
        y.template hand_on<ALIGNED>(end);
        if constexpr (KEEP) {
            keep(a.cx, at[u].i, at[u].in, x[u]);
            if constexpr (GATED) keep(a.cu, at[u].i, at[u].in, up[u]);
        }
        if (a.cy.values != nullptr) keep(a.cy, at[u].i, at[u].in, y);  // of what the next layer reads
        if constexpr (!ALIGNED && kRun<T> > 32) __syncthreads();  // (in place too: every thread has its inputs)
        y.template store<ALIGNED>(at[u].of(a.y), at[u].n, at[u].joined, at[u].follows, end);
    }
}

struct Backward {
    Pieces p;
    Side dy, dx, dup;
    Ckpt cx, cu;
};

template <typename T, int ACT, bool GATED, bool ALIGNED>
__global__ void __launch_bounds__(kBlock, kBlocks<T>) act8_backward_kernel(const __grid_constant__ Backward a) {
    const At<T> at[2] = {At<T>(a.p, 0), At<T>(a.p, 1)};
    __shared__ uint4 ends[ALIGNED ? 1 : 4][kBlock / 32];
    Eight<T> dy[2];
    Kept kx[2], ku[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        dy[u].template load<ALIGNED>(a.dy, at[u].of(a.dy), at[u].n);
        if (at[u].in) {
            kx[u].load(a.cx, at[u].i);
            if constexpr (GATED) ku[u].load(a.cu, at[u].i);
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const Eight<uint16_t> x = kx[u].values(), up = GATED ? ku[u].values() : Eight<uint16_t>{};
        float dx[kPiece], dup[kPiece];
#pragma unroll
        for (int j = 0; j < kPiece; ++j) {
            float f, slope;
            act_value_slope<ACT>(x.get(j), &f, &slope);
            const float d = dy[u].get(j);
            if constexpr (GATED) {
                dx[j] = d * up.get(j) * slope;
                dup[j] = d * f;
            } else {
                dx[j] = d * slope;
            }
        }
        Eight<T> vx, vu;
        vx.set(dx);
        uint4 *const end_x = ends[ALIGNED ? 0 : 2 * u], *const end_u = ends[ALIGNED ? 0 : 2 * u + 1];
        vx.template hand_on<ALIGNED>(end_x);
        if constexpr (GATED) {
            vu.set(dup);
            vu.template hand_on<ALIGNED>(end_u);
        }
        if constexpr (!ALIGNED && kRun<T> > 32) __syncthreads();  // (in place too: every thread has its inputs)
        vx.template store<ALIGNED>(at[u].of(a.dx), at[u].n, at[u].joined, at[u].follows, end_x);
        if constexpr (GATED) vu.template store<ALIGNED>(at[u].of(a.dup), at[u].n, at[u].joined, at[u].follows, end_u);
    }
}

inline unsigned piece_grid(const Pieces& p) { return static_cast<unsigned>((p.total + 2 * kBlock - 1) / (2 * kBlock)); }

inline Side side_of(const Mat& m) { return Side{const_cast<void*>(m.p), m.stride, static_cast<int64_t>(m.extent())}; }

// The kernel variant of a call: element type, aligned rows, activation, gate.
template <typename F>
void pick(ss_dtype dt, bool aligned, F&& launch) {
    if (dt == SS_F32) {
        if (aligned) launch(float{}, std::true_type{}); else launch(float{}, std::false_type{});
    } else {
        if (aligned) launch(uint16_t{}, std::true_type{}); else launch(uint16_t{}, std::false_type{});
    }
}

template <typename F>
void pick(ss_dtype dt, bool aligned, ss_act act, bool gated, F&& launch) {
    pick(dt, aligned, [&](auto t, auto al) {
        if (act == SS_ACT_GELU) {
            const std::integral_constant<int, SS_ACT_GELU> f;
            if (gated) launch(t, al, f, std::true_type{}); else launch(t, al, f, std::false_type{});
        } else {
            const std::integral_constant<int, SS_ACT_SILU> f;
            if (gated) launch(t, al, f, std::true_type{}); else launch(t, al, f, std::false_type{});
        }
    });
}

// A checkpoint argument: present, aligned.
int ckpt_check(const uint8_t* p) {
    if (p == nullptr) return SS_ERR_INVALID_ARG;
    return addr_aligned(p, 16) ? SS_OK : SS_ERR_MISALIGNED;
}

int mat_check(const Mat& m, int64_t stride) {
    if (m.p == nullptr || !stride_ok(m.rows, m.cols, stride)) return SS_ERR_INVALID_ARG;
    return addr_aligned(m.p, m.eb) ? SS_OK : SS_ERR_MISALIGNED;
}

}  // namespace
}  // namespace ss

using namespace ss;

#define SS_TRY(expr)                         \
    do {                                     \
        const int status_ = (expr);          \
        if (status_ != SS_OK) return status_; \
    } while (0)

extern "C" {
#pragma GCC visibility push(default)

int64_t ss_act8_bytes(int64_t rows, int64_t cols) {
    if (!sides_ok(rows, cols)) return -1;
    return rows * act8_groups(cols) * (SS_ACT8_GROUP + 1);
}

int ss_act8_pack(const void* x, int64_t x_stride, ss_dtype dt, int64_t rows, int64_t cols, uint8_t* ckpt,
                 void* cuda_stream) {
    if (!dtype_known(dt) || !sides_ok(rows, cols) || !stride_ok(rows, cols, x_stride)) return SS_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return SS_OK;
    const Mat mx = mat(x, rows, cols, x_stride, dtype_bytes(dt));
    SS_TRY(mat_check(mx, x_stride));
    SS_TRY(ckpt_check(ckpt));
    if (mat_overlaps(mx, ckpt, ss_act8_bytes(rows, cols))) return SS_ERR_INVALID_ARG;
    const Ckpt c = ckpt_of(ckpt, rows, cols);
    const Pieces p = pieces_of(rows, cols);
    pick(dt, mx.row_aligned(16), [&](auto t, auto al) {
        act8_pack_kernel<decltype(t), al.value><<<piece_grid(p), kBlock, 0, static_cast<cudaStream_t>(cuda_stream)>>>(p, side_of(mx), c);
    });
    return cuda_status_public(cudaGetLastError());
}

int ss_act8_unpack(const uint8_t* ckpt, int64_t rows, int64_t cols, void* out, int64_t out_stride, ss_dtype dt,
                   void* cuda_stream) {
    if (!dtype_known(dt) || !sides_ok(rows, cols) || !stride_ok(rows, cols, out_stride)) return SS_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return SS_OK;
    const Mat mo = mat(out, rows, cols, out_stride, dtype_bytes(dt));
    SS_TRY(mat_check(mo, out_stride));
    SS_TRY(ckpt_check(ckpt));
    if (mat_overlaps(mo, ckpt, ss_act8_bytes(rows, cols))) return SS_ERR_INVALID_ARG;
    const Ckpt c = ckpt_of(const_cast<uint8_t*>(ckpt), rows, cols);
    const Pieces p = pieces_of(rows, cols);
    pick(dt, mo.row_aligned(16), [&](auto t, auto al) {
        act8_unpack_kernel<decltype(t), al.value><<<piece_grid(p), kBlock, 0, static_cast<cudaStream_t>(cuda_stream)>>>(p, c, side_of(mo));
    });
    return cuda_status_public(cudaGetLastError());
}

int ss_act8_forward(const void* x, int64_t x_stride, const void* up, int64_t up_stride, ss_dtype dt, ss_act act,
                    int64_t rows, int64_t cols, void* y, int64_t y_stride, uint8_t* ckpt_x, uint8_t* ckpt_up,
                    uint8_t* ckpt_y, void* cuda_stream) {
    if (!dtype_known(dt) || (act != SS_ACT_GELU && act != SS_ACT_SILU) || !sides_ok(rows, cols)) return SS_ERR_INVALID_ARG;
    if (!stride_ok(rows, cols, x_stride) || !stride_ok(rows, cols, y_stride)) return SS_ERR_INVALID_ARG;
    if ((up == nullptr && ckpt_up != nullptr) || (up != nullptr && !stride_ok(rows, cols, up_stride))) return SS_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return SS_OK;
    if (up != nullptr && (ckpt_x != nullptr) != (ckpt_up != nullptr)) return SS_ERR_INVALID_ARG;
    const size_t eb = dtype_bytes(dt), kept = ss_act8_bytes(rows, cols);
    const Mat mx = mat(x, rows, cols, x_stride, eb), my = mat(y, rows, cols, y_stride, eb);
    const Mat mu = mat(up, rows, cols, up_stride, eb);
    SS_TRY(mat_check(mx, x_stride));
    SS_TRY(mat_check(my, y_stride));
    if (up != nullptr) SS_TRY(mat_check(mu, up_stride));
    if (ckpt_x != nullptr) SS_TRY(ckpt_check(ckpt_x));
    if (ckpt_up != nullptr) SS_TRY(ckpt_check(ckpt_up));
    if (ckpt_y != nullptr) SS_TRY(ckpt_check(ckpt_y));
    if (mats_overlap(my, mx) && !same_mat(my, mx)) return SS_ERR_INVALID_ARG;
    if (up != nullptr && mats_overlap(my, mu) && !same_mat(my, mu)) return SS_ERR_INVALID_ARG;
    uint8_t* const cks[3] = {ckpt_x, ckpt_up, ckpt_y};
    for (int i = 0; i < 3; ++i) {
        if (cks[i] == nullptr) continue;
        if (mat_overlaps(mx, cks[i], kept) || mat_overlaps(my, cks[i], kept)) return SS_ERR_INVALID_ARG;
        if (up != nullptr && mat_overlaps(mu, cks[i], kept)) return SS_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (cks[j] != nullptr && bytes_overlap(cks[i], kept, cks[j], kept)) return SS_ERR_INVALID_ARG;
    }
    const Forward a{pieces_of(rows, cols), side_of(mx), side_of(mu), side_of(my), ckpt_of(ckpt_x, rows, cols),
                    ckpt_of(ckpt_up, rows, cols), ckpt_of(ckpt_y, rows, cols)};
    const bool aligned = mx.row_aligned(16) && my.row_aligned(16) && (up == nullptr || mu.row_aligned(16));
    pick(dt, aligned, act, up != nullptr, [&](auto t, auto al, auto f, auto gated) {
        const auto kernel = ckpt_x != nullptr ? act8_forward_kernel<decltype(t), f.value, gated.value, al.value, true>
                                              : act8_forward_kernel<decltype(t), f.value, gated.value, al.value, false>;
        kernel<<<piece_grid(a.p), kBlock, 0, static_cast<cudaStream_t>(cuda_stream)>>>(a);
    });
    return cuda_status_public(cudaGetLastError());
}

int ss_act8_backward(const void* dy, int64_t dy_stride, const uint8_t* ckpt_x, const uint8_t* ckpt_up, ss_dtype dt,
                     ss_act act, int64_t rows, int64_t cols, void* dx, int64_t dx_stride, void* dup,
                     int64_t dup_stride, void* cuda_stream) {
    if (!dtype_known(dt) || (act != SS_ACT_GELU && act != SS_ACT_SILU) || !sides_ok(rows, cols)) return SS_ERR_INVALID_ARG;
    if (!stride_ok(rows, cols, dy_stride) || !stride_ok(rows, cols, dx_stride)) return SS_ERR_INVALID_ARG;
    if ((dup != nullptr) != (ckpt_up != nullptr) || (dup != nullptr && !stride_ok(rows, cols, dup_stride))) return SS_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return SS_OK;
    const size_t eb = dtype_bytes(dt), kept = ss_act8_bytes(rows, cols);
    const Mat my = mat(dy, rows, cols, dy_stride, eb), mx = mat(dx, rows, cols, dx_stride, eb);
    const Mat mu = mat(dup, rows, cols, dup_stride, eb);
    SS_TRY(mat_check(my, dy_stride));
    SS_TRY(mat_check(mx, dx_stride));
    if (dup != nullptr) SS_TRY(mat_check(mu, dup_stride));
    SS_TRY(ckpt_check(ckpt_x));
    if (ckpt_up != nullptr) SS_TRY(ckpt_check(ckpt_up));
    if (mats_overlap(mx, my) && !same_mat(mx, my)) return SS_ERR_INVALID_ARG;
    if (dup != nullptr && ((mats_overlap(mu, my) && !same_mat(mu, my)) || mats_overlap(mu, mx))) return SS_ERR_INVALID_ARG;
    const uint8_t* const cks[2] = {ckpt_x, ckpt_up};
    for (const uint8_t* c : cks) {
        if (c == nullptr) continue;
        if (mat_overlaps(mx, c, kept) || (dup != nullptr && mat_overlaps(mu, c, kept))) return SS_ERR_INVALID_ARG;
    }
    const Backward a{pieces_of(rows, cols), side_of(my), side_of(mx), side_of(mu),
                     ckpt_of(const_cast<uint8_t*>(ckpt_x), rows, cols), ckpt_of(const_cast<uint8_t*>(ckpt_up), rows, cols)};
    const bool aligned = my.row_aligned(16) && mx.row_aligned(16) && (dup == nullptr || mu.row_aligned(16));
    pick(dt, aligned, act, dup != nullptr, [&](auto t, auto al, auto f, auto gated) {
        act8_backward_kernel<decltype(t), f.value, gated.value, al.value>
            <<<piece_grid(a.p), kBlock, 0, static_cast<cudaStream_t>(cuda_stream)>>>(a);
    });
    return cuda_status_public(cudaGetLastError());
}

#pragma GCC visibility pop
}  // extern "C"
