// Softmax cross entropy of x W^T from the hidden states x and the head W, with the gradients of both.
//
// Rows that count are gathered first; the others cost nothing. Then, for some rows at a time (kChunkBytes):
//   logits     a product whose tiles end in registers: each thread has 128 logits of a row, whose
//              maximum m and sum of e = exp(c (z - m)) it keeps, with e itself where a gradient is wanted
//   rows       the parts' maxima and sums joined, log p, the factors of the row's gradient
//   gradient   e -> P, the gradient with respect to the logits, in place
//   dx = P W,  dW (+)= P^T x: products whose operands lie with the contraction index slow or fast, as they are
// So neither the logits nor P exist as a whole, and three products do, where forming the logits again for the backward pass
// would take four; the pass over e costs a few percent of a product.
//
// Rounding. The sums of a logit leave the matrix unit, which truncates as it adds, every 256 contraction indices and
// are added in registers, to nearest: log p would otherwise lose 1e-4 at width 4096. e is fp16 (relative to its part's
// maximum, 11 bits), P is bf16 as the gradient of bf16 logits is; the entry of the target, which is a
// difference, is formed in fp32 from log p. With fp32 inputs e is fp32 and P the sum of three bf16.
#include "product.cuh"

#include <cuda_fp16.h>

#include <cmath>

namespace ss {
namespace {

constexpr int kPartCols = kProdHalf;              // logits of a thread
constexpr int kLogitChunk = 4;                    // stages that the matrix unit sums of a logit
// Stages that it sums of a gradient: 16384 contraction indices lose 2e-5, nothing next to an operand of bf16; 2048 lose 5e-7.
constexpr int kGradChunk = 256, kGradChunkF32 = 32;
constexpr int64_t kChunkBytes = int64_t(1) << 30; // of e and P
constexpr int64_t kMostChunkRows = 16384;

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// What the kernels of one chunk share.
struct Head {
    const int64_t* targets;
    const float *weights, *grad_scale;
    float *totals, *logp;
    int64_t rows, x_stride, w_stride, dx_stride;
    const void *x, *w;
    void* dx;
    int width, vocab, vectors, dx_vectors, w_vectors;
    float c, k, z_coef;  // k = c log2 e
    // workspace
    int *index, *target, *live;     // of the rows that count, one after another
    float *target_logit, *top, *factor, *target_grad, *loss, *square;
    uint16_t *gathered, *staged_w;
    float2* parts;                  // [chunk rows][n_parts]: maximum, sum
    uint16_t *e16, *p16;            // e, P of bf16 inputs (the same place); planes of P of fp32 ones
    float *e32, *acc;
    int64_t width_ld, e_ld, row_cap, chunk_rows;
    int n_parts, first;             // first row of the chunk
};

__device__ __forceinline__ bool counts(const Head& a, int64_t t) {
    const int64_t y = a.targets[t];
    return a.weights[t] != 0.0f && y >= 0 && y < a.vocab;
}

// Which rows count, in their order.
__global__ void __launch_bounds__(1024) head_rows_kernel(const __grid_constant__ Head a) {
    next_may_begin();
    __shared__ int sums[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int base = 0;
    for (int64_t t0 = 0; t0 < a.rows; t0 += 1024) {
        const int64_t t = t0 + threadIdx.x;
        const bool in = t < a.rows && counts(a, t);
        const uint32_t votes = __ballot_sync(0xFFFFFFFFu, in);
        if (lane == 0) sums[warp] = __popc(votes);
        __syncthreads();
        int before = 0, all = 0;
        for (int i = 0; i < 32; ++i) {
            const int n = sums[i];
            if (i < warp) before += n;
            all += n;
        }
        if (in) {
            const int s = base + before + __popc(votes & ((1u << lane) - 1u));
            a.index[s] = static_cast<int>(t);
            a.target[s] = static_cast<int>(a.targets[t]);
        }
        base += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) *a.live = base;
}

// An fp32 value as three bf16 whose sum it is: its leading 8 bits, the next 8 and the last 8, cut off. An infinity or NaN is
// carried by the first alone.
__device__ __forceinline__ void terms_of(float f, uint32_t (&t)[3]) {
    uint32_t hi = __float_as_uint(f) & 0xFFFF0000u, mid = 0, lo = 0;
    if ((hi & 0x7F800000u) == 0x7F800000u) {
        if (f != f) hi = kNanBits;
    } else {
        const float rest = f - __uint_as_float(hi);
        mid = __float_as_uint(rest) & 0xFFFF0000u;
        lo = __float_as_uint(rest - __uint_as_float(mid));
    }
    t[0] = hi, t[1] = mid, t[2] = lo;
}

__device__ __forceinline__ void store_terms(uint16_t* dst, int64_t plane, const float (&v)[4]) {
    uint32_t t[4][3];
#pragma unroll
    for (int j = 0; j < 4; ++j) terms_of(v[j], t[j]);
#pragma unroll
    for (int q = 0; q < 3; ++q)
        *reinterpret_cast<uint2*>(dst + q * plane) = make_uint2(__byte_perm(t[0][q], t[1][q], 0x7632), __byte_perm(t[2][q], t[3][q], 0x7632));
}

// A row to the layout of an operand: bf16 as it is, fp32 as three terms.
template <typename T>
__device__ __forceinline__ void stage_row(const T* src, uint16_t* dst, int64_t plane, int width, bool vectors, int lane) {
    for (int c = 4 * lane; c < width; c += 128) {
        const int n = width - c;
        if constexpr (sizeof(T) == 2) {
            uint2 r;
            if (vectors && n >= 4) {
                r = *reinterpret_cast<const uint2*>(src + c);
            } else {
                uint32_t v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = j < n ? src[c + j] : 0;
                r = make_uint2(v[0] | (v[1] << 16), v[2] | (v[3] << 16));
            }
            *reinterpret_cast<uint2*>(dst + c) = r;
        } else {
            float v[4];
            if (vectors && n >= 4) {
                const float4 r = *reinterpret_cast<const float4*>(src + c);
                v[0] = r.x, v[1] = r.y, v[2] = r.z, v[3] = r.w;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = j < n ? src[c + j] : 0.0f;
            }
            store_terms(dst + c, plane, v);
        }
    }
}

// Rows that count gathered; behind them zeros up to a whole stage, since dW sums over whole stages; the results of the others.
template <typename T>
__global__ void __launch_bounds__(256) head_gather_kernel(const __grid_constant__ Head a) {
    next_may_begin();
    after_previous();
    const int lane = threadIdx.x & 31;
    const int64_t live = *a.live, padded = (live + kProdK - 1) / kProdK * kProdK, plane = a.row_cap * a.width_ld;
    const int64_t upto = padded > kProdK ? padded : kProdK;
    for (int64_t i = blockIdx.x * 8 + (threadIdx.x >> 5); i < a.rows + kProdK; i += gridDim.x * 8) {
        if (i < upto) {
            uint16_t* const dst = a.gathered + i * a.width_ld;
            if (i < live) {
                stage_row(static_cast<const T*>(a.x) + a.index[i] * a.x_stride, dst, plane, a.width, a.vectors, lane);
            } else {
                for (int q = 0; q < (sizeof(T) == 4 ? kTerms : 1); ++q)
                    for (int c = lane; c < a.width; c += 32) dst[q * plane + c] = 0;
            }
        }
        if (i < a.rows && !counts(a, i)) {
            if (lane == 0) a.logp[i] = 0.0f;
            if (a.dx != nullptr) {
                T* const dst = static_cast<T*>(a.dx) + i * a.dx_stride;
                for (int c = lane; c < a.width; c += 32) dst[c] = T(0);
            }
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) head_stage_w_kernel(const __grid_constant__ Head a) {
    next_may_begin();
    after_previous();
    const int64_t plane = static_cast<int64_t>(a.vocab) * a.width_ld;
    for (int64_t i = blockIdx.x * 8 + (threadIdx.x >> 5); i < a.vocab; i += gridDim.x * 8)
        stage_row(static_cast<const T*>(a.w) + i * a.w_stride, a.staged_w + i * a.width_ld, plane, a.width, a.w_vectors, threadIdx.x & 31);
}

__device__ __forceinline__ uint4 half8(const float* v) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 p = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// ---- the end of the logits' product
struct Logits {
    static constexpr bool kWhole = true;
    const int* target;  // of the chunk's rows
    float* target_logit;
    float2* parts;
    uint16_t* e16;      // at most one of these
    float* e32;
    int64_t e_ld;
    int n_parts, vocab;
    float k;

    __device__ __forceinline__ void whole(const ProdUnit&, int m, int row, int col, int lane, uint32_t buf, float (&z)[kPartCols]) const {
        if (row >= m) return;
        const int r = row + lane, there = vocab - col;
        if (there < kPartCols) {
#pragma unroll
            for (int i = 0; i < kPartCols; ++i) z[i] = i < there ? z[i] : -INFINITY;
        }
        const int y = r < m ? target[r] - col : -1;
        if (y >= 0 && y < kPartCols) {
            float v = 0.0f;
#pragma unroll
            for (int i = 0; i < kPartCols; ++i) v = i == y ? z[i] : v;
            target_logit[r] = v;
        }
        float top = z[0], sum = 0.0f;
#pragma unroll
        for (int i = 1; i < kPartCols; ++i) top = fmaxf(top, z[i]);
        const float from = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int i = 0; i < kPartCols; ++i) {
            z[i] = ex2((z[i] - from) * k);
            sum += z[i];
        }
        if (r < m) parts[static_cast<int64_t>(r) * n_parts + col / kPartCols] = make_float2(top, sum);
        if (e16 != nullptr) {
#pragma unroll
            for (int h = 0; h < kPartCols; h += 64) {
#pragma unroll
                for (int i = 0; i < 8; ++i) square_set(buf, lane, i, half8(z + h + 8 * i));
                out_square(reinterpret_cast<char*>(e16), 2, m, row, col + h, lane, buf);
            }
        } else if (e32 != nullptr) {
#pragma unroll
            for (int h = 0; h < kPartCols; h += 32) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    square_set(buf, lane, i, make_uint4(__float_as_uint(z[h + 4 * i]), __float_as_uint(z[h + 4 * i + 1]),
                                                        __float_as_uint(z[h + 4 * i + 2]), __float_as_uint(z[h + 4 * i + 3])));
                out_square(reinterpret_cast<char*>(e32), 4, m, row, col + h, lane, buf);
            }
        }
    }
    // 32 rows of 128 bytes: columns that the padded rows have.
    __device__ __forceinline__ void out_square(char* e, int size, int m, int row, int col, int lane, uint32_t buf) const {
        __syncwarp();
        const int c = col + 16 / size * (lane & 7);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int q = (lane >> 3) + 4 * i;
            const uint4 v = square_get(buf, q, lane & 7);
            if (row + q < m && c < e_ld) *reinterpret_cast<uint4*>(e + ((row + q) * e_ld + c) * size) = v;
        }
        __syncwarp();
    }
};

// log p, and what the row's gradient is made of: P_v = factor e_v 2^(k (m_part - top)), the target's in fp32 from log p:
// p - 1 = exp(log p) - 1 keeps its digits near certainty. A warp to a row.
__global__ void __launch_bounds__(256) head_statistics_kernel(const __grid_constant__ Head a) {
    next_may_begin();
    after_previous();
    const int lane = threadIdx.x & 31;
    const int64_t here = min(static_cast<int64_t>(*a.live) - a.first, a.chunk_rows);
    for (int64_t r = blockIdx.x * 8 + (threadIdx.x >> 5); r < here; r += gridDim.x * 8) {
        const float2* const p = a.parts + r * a.n_parts;
        float top = -INFINITY, sum = 0.0f;
        for (int i = lane; i < a.n_parts; i += 32) top = fmaxf(top, p[i].x);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        const float from = top == -INFINITY ? 0.0f : top;
        for (int i = lane; i < a.n_parts; i += 32) {
            const float2 v = p[i];
            sum += v.y * ex2((v.x - from) * a.k);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        if (lane != 0) continue;
        const int64_t s = a.first + r;
        const int t = a.index[s];
        const float w = a.weights[t], rest = logf(sum);
        const float lse = a.c * top + rest, logp = a.c * (a.target_logit[r] - top) - rest;
        const float scale = w * a.c * (a.grad_scale == nullptr ? 1.0f : *a.grad_scale);
        float loss = -w * logp, all = 1.0f, extra = 0.0f;
        if (a.z_coef != 0.0f) {
            loss += a.z_coef * w * lse * lse;
            extra = 2.0f * a.z_coef * lse;
            all += extra;
        }
        a.logp[t] = logp;
        a.loss[s] = loss, a.square[s] = w * lse * lse;
        a.top[r] = top;
        a.factor[r] = scale * all / sum;
        a.target_grad[r] = scale * (expm1f(logp) + extra * expf(logp));
    }
}

// e -> P: eight columns to a thread. Rows behind the last up to a whole stage become zeros.
template <bool F32>
__global__ void __launch_bounds__(256) head_gradient_kernel(const __grid_constant__ Head a) {
    next_may_begin();
    after_previous();
    const int64_t r = blockIdx.y + static_cast<int64_t>(blockIdx.z) * 65535, here = min(static_cast<int64_t>(*a.live) - a.first, a.chunk_rows);
    const int64_t upto = max((here + kProdK - 1) / kProdK * kProdK, static_cast<int64_t>(a.first == 0 ? kProdK : 0));
    const int c = (blockIdx.x * 256 + threadIdx.x) * 8;
    if (r >= min(upto, a.chunk_rows) || c >= a.e_ld) return;
    float v[8];
    if (r >= here) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.0f;
    } else {
        const float2 part = a.parts[r * a.n_parts + c / kPartCols];
        // an empty part, or one of -inf alone, has m = -inf and zeros for e
        const float f = a.factor[r] * (part.x == -INFINITY ? 0.0f : ex2((part.x - a.top[r]) * a.k));
        if constexpr (F32) {
            const float4* const src = reinterpret_cast<const float4*>(a.e32 + r * a.e_ld + c);
            const float4 x = src[0], y = src[1];
            v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w, v[4] = y.x, v[5] = y.y, v[6] = y.z, v[7] = y.w;
        } else {
            const uint4 x = *reinterpret_cast<const uint4*>(a.e16 + r * a.e_ld + c);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
                v[2 * j] = p.x, v[2 * j + 1] = p.y;
            }
        }
        const int y = a.target[a.first + r] - c;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j == y ? a.target_grad[r] : v[j] * f;
    }
    if constexpr (F32) {
        const int64_t plane = a.chunk_rows * a.e_ld;
        const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
        store_terms(a.p16 + r * a.e_ld + c, plane, lo);
        store_terms(a.p16 + r * a.e_ld + c + 4, plane, hi);
    } else {
        *reinterpret_cast<uint4*>(a.p16 + r * a.e_ld + c) = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
    }
}

// ---- the end of the gradients' products: written, or added by the memory itself (the same lane adds to an element each
// time, so its sums come in their order).
struct Gradient {
    static constexpr bool kWhole = false;
    struct Fetched {};
    float* dst;
    uint16_t* dst16;  // bf16 instead; every chunk but the first would be lost, so there is one
    int64_t stride;
    int cols, vectors, add;

    __device__ __forceinline__ void fetch(const ProdUnit&, int, int, int, int, Fetched&) const {}
    __device__ __forceinline__ void square(const ProdUnit&, int m, int row, int col, int lane, uint32_t buf, const Fetched&, bool first) const {
        const int c = col + 4 * (lane & 7);
        if (c >= cols) return;
        const bool adds = add || !first;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int q = (lane >> 3) + 4 * i;
            const uint4 w = square_get(buf, q, lane & 7);
            if (row + q >= m) continue;
            const int64_t at = (row + q) * stride + c;
            const float v[4] = {__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w)};
            if (vectors && c + 4 <= cols) {
                if (dst16 != nullptr) *reinterpret_cast<uint2*>(dst16 + at) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
                else if (adds) asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(__cvta_generic_to_global(dst + at)), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]) : "memory");
                else *reinterpret_cast<float4*>(dst + at) = make_float4(v[0], v[1], v[2], v[3]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (c + j >= cols) break;
                    if (dst16 != nullptr) Elem<uint16_t>::store(dst16 + at + j, v[j]);
                    else if (adds) asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" ::"l"(__cvta_generic_to_global(dst + at + j)), "f"(v[j]) : "memory");
                    else dst[at + j] = v[j];
                }
            }
        }
    }
};

// dx of the chunk's rows, from their sums to their places.
template <typename T>
__global__ void __launch_bounds__(256) head_dx_kernel(const __grid_constant__ Head a) {
    next_may_begin();
    after_previous();
    const int lane = threadIdx.x & 31;
    const int64_t here = min(static_cast<int64_t>(*a.live) - a.first, a.chunk_rows);
    for (int64_t r = blockIdx.x * 8 + (threadIdx.x >> 5); r < here; r += gridDim.x * 8) {
        const float* const src = a.acc + r * a.width_ld;
        T* const dst = static_cast<T*>(a.dx) + a.index[a.first + r] * a.dx_stride;
        for (int c = 4 * lane; c < a.width; c += 128) {
            const float4 v = *reinterpret_cast<const float4*>(src + c);
            if (a.dx_vectors && c + 4 <= a.width) {
                if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(dst + c) = v;
                else *reinterpret_cast<uint2*>(dst + c) = make_uint2(bf16_pair(v.x, v.y), bf16_pair(v.z, v.w));
            } else {
                const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (c + j < a.width) Elem<T>::store(dst + c + j, e[j]);
            }
        }
    }
}

// Sums in fp32 to a dW of bf16, where they came in several chunks.
__global__ void __launch_bounds__(256) head_round_kernel(const float* src, int64_t src_stride, uint16_t* dst, int64_t stride, int64_t rows, int width) {
    next_may_begin();
    after_previous();
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int c = threadIdx.x; c < width; c += 256) Elem<uint16_t>::store(dst + r * stride + c, src[r * src_stride + c]);
}

__global__ void __launch_bounds__(256) head_zero_kernel(void* dst, int64_t row_bytes, int64_t stride_bytes, int64_t rows) {
    next_may_begin();
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = threadIdx.x * 2; c < row_bytes; c += 512) *reinterpret_cast<uint16_t*>(static_cast<char*>(dst) + r * stride_bytes + c) = 0;
}

// Loss and sum of weighted squares: fp64, in a fixed order.
__global__ void __launch_bounds__(1024) head_totals_kernel(const __grid_constant__ Head a, int none) {
    next_may_begin();
    if (!none) after_previous();
    __shared__ double part[2][32];
    const int64_t live = none ? 0 : *a.live;
    double loss = 0.0, square = 0.0;
    for (int64_t s = threadIdx.x; s < live; s += 1024) loss += a.loss[s], square += a.square[s];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        loss += __shfl_xor_sync(0xFFFFFFFFu, loss, d);
        square += __shfl_xor_sync(0xFFFFFFFFu, square, d);
    }
    if ((threadIdx.x & 31) == 0) part[0][threadIdx.x >> 5] = loss, part[1][threadIdx.x >> 5] = square;
    __syncthreads();
    if (threadIdx.x < 2) {
        double v = 0.0;
        for (int i = 0; i < 32; ++i) v += part[threadIdx.x][i];
        a.totals[threadIdx.x] = static_cast<float>(v);
    }
}

// ---- host side -------------------------------------------------------------------------------------

constexpr int64_t kMostRows = int64_t(1) << 24, kMostTilesHead = int64_t(1) << 24;

inline int64_t up_to(int64_t n, int64_t m) { return (n + m - 1) / m * m; }

struct Layout {
    bool f32, dx, dw, stage_w, sums_w;  // sums_w: dW of bf16 from several chunks
    int64_t planes, width_ld, e_ld, n_parts, chunks, chunk_rows, row_cap;
    int64_t index, target, live, rows_f32, gathered, staged_w, parts, e, p, acc, w32, bytes;
};

int layout_of(const void* w, int64_t w_stride, ss_dtype dt, int64_t rows, int64_t width, int64_t vocab, bool dx, bool dw, ss_dtype dw_dt, Layout* l) {
    const int64_t tiles_v = (vocab + kProdTile - 1) / kProdTile, tiles_d = (width + kProdTile - 1) / kProdTile;
    if (rows > kMostRows || tiles_v * ((rows + kProdTile - 1) / kProdTile) > kMostTilesHead || tiles_v * tiles_d > kMostTilesHead) return SS_ERR_UNSUPPORTED;
    l->f32 = dt == SS_F32, l->dx = dx, l->dw = dw, l->planes = l->f32 ? kTerms : 1;
    const Mat m = mat(w, vocab, width, w_stride, dtype_bytes(dt));
    l->stage_w = l->f32 || !m.row_aligned(16) || m.stride * 2 % 16 != 0 || m.stride * 2 >= (int64_t(1) << 38);
    l->width_ld = up_to(width, 64), l->e_ld = up_to(vocab, 64);
    l->n_parts = 2 * tiles_v;
    const int64_t per_row = dx || dw ? l->e_ld * (l->f32 ? 4 + 2 * kTerms : 2) : l->n_parts * 8;
    int64_t most = kChunkBytes / per_row / kProdTile * kProdTile;
    most = most < kProdTile ? kProdTile : (most > kMostChunkRows ? kMostChunkRows : most);
    l->chunks = rows > 0 ? (rows + most - 1) / most : 1;
    l->chunk_rows = up_to((rows + l->chunks - 1) / l->chunks, kProdTile);
    l->row_cap = l->chunks * l->chunk_rows;
    l->sums_w = dw && dw_dt == SS_BF16 && l->chunks > 1;
    int64_t at = 0;
    auto place = [&](int64_t bytes) {
        const int64_t p = at;
        at += up_to(bytes, 256);
        return p;
    };
    l->index = place(rows * 4), l->target = place(l->row_cap * 4), l->live = place(4);
    l->rows_f32 = place((2 * l->row_cap + 4 * l->chunk_rows) * 4);
    l->gathered = place(l->planes * l->row_cap * l->width_ld * 2);
    l->staged_w = place(l->stage_w ? l->planes * vocab * l->width_ld * 2 : 0);
    l->parts = place(l->chunk_rows * l->n_parts * 8);
    l->e = place(dx || dw ? l->chunk_rows * l->e_ld * (l->f32 ? 4 : 2) : 0);
    l->p = l->f32 && (dx || dw) ? place(kTerms * l->chunk_rows * l->e_ld * 2) : l->e;
    l->acc = place(dx ? l->chunk_rows * l->width_ld * 4 : 0);
    l->w32 = place(l->sums_w ? vocab * l->width_ld * 4 : 0);
    l->bytes = at;
    return SS_OK;
}

bool sizes_ok(int64_t rows, int64_t width, int64_t vocab) {
    return sides_ok(rows, width) && sides_ok(rows, vocab) && (rows == 0 || (width > 0 && vocab > 0));
}

unsigned blocks_for(int64_t warps, int sms) {
    const int64_t want = (warps + 7) / 8, most = static_cast<int64_t>(sms) * 8;
    return static_cast<unsigned>(want < 1 ? 1 : (want < most ? want : most));
}

int run(Head& a, const Layout& l, uint8_t* ws, void* dw, int64_t dw_stride, ss_dtype dw_dt, bool dw_vectors, int accumulate, cudaStream_t st) {
    cudaError_t e = cudaSuccess;
    const int sms = device_sm_count(&e);
    if (e != cudaSuccess) return cuda_status_public(e);
    a.index = reinterpret_cast<int*>(ws + l.index), a.target = reinterpret_cast<int*>(ws + l.target), a.live = reinterpret_cast<int*>(ws + l.live);
    float* f = reinterpret_cast<float*>(ws + l.rows_f32);
    a.loss = f, a.square = f + l.row_cap, f += 2 * l.row_cap;
    a.target_logit = f, a.top = f + l.chunk_rows, a.factor = f + 2 * l.chunk_rows, a.target_grad = f + 3 * l.chunk_rows;
    a.gathered = reinterpret_cast<uint16_t*>(ws + l.gathered), a.staged_w = reinterpret_cast<uint16_t*>(ws + l.staged_w);
    a.parts = reinterpret_cast<float2*>(ws + l.parts);
    a.e16 = reinterpret_cast<uint16_t*>(ws + l.e), a.e32 = reinterpret_cast<float*>(ws + l.e), a.p16 = reinterpret_cast<uint16_t*>(ws + l.p);
    a.acc = reinterpret_cast<float*>(ws + l.acc);
    a.width_ld = l.width_ld, a.e_ld = l.e_ld, a.row_cap = l.row_cap, a.chunk_rows = l.chunk_rows, a.n_parts = static_cast<int>(l.n_parts);
    const bool grads = l.dx || l.dw;
    const int64_t rows = a.rows, width = a.width, vocab = a.vocab;

    CUtensorMap w_cols, w_rows;  // W as an operand of the logits and of dx
    const void* const w = l.stage_w ? a.staged_w : a.w;
    const int64_t w_row = l.stage_w ? l.width_ld * 2 : a.w_stride * 2, w_plane = vocab * l.width_ld * 2;
    int status = map_operand(&w_cols, w, true, width, vocab, w_row, l.planes, w_plane, false);
    if (status == SS_OK && l.dx) status = map_operand(&w_rows, w, true, width, vocab, w_row, l.planes, w_plane, true);
    if (status != SS_OK) return status;

    e = launch_next(false, head_rows_kernel, 1, 1024, st, a);
    if (e == cudaSuccess) e = l.f32 ? launch_next(true, head_gather_kernel<float>, blocks_for(rows + kProdK, sms), 256, st, a)
                                    : launch_next(true, head_gather_kernel<uint16_t>, blocks_for(rows + kProdK, sms), 256, st, a);
    if (e == cudaSuccess && l.stage_w) e = l.f32 ? launch_next(true, head_stage_w_kernel<float>, blocks_for(vocab, sms), 256, st, a)
                                                 : launch_next(true, head_stage_w_kernel<uint16_t>, blocks_for(vocab, sms), 256, st, a);
    if (e != cudaSuccess) return cuda_status_public(e);

    for (int64_t i = 0; i < l.chunks; ++i) {
        const int64_t first = i * l.chunk_rows;
        a.first = static_cast<int>(first);
        const uint16_t* const x = a.gathered + first * l.width_ld;
        const int64_t x_row = l.width_ld * 2, x_plane = l.row_cap * l.width_ld * 2, p_row = l.e_ld * 2, p_plane = l.chunk_rows * l.e_ld * 2;
        CUtensorMap x_cols, x_rows, p_cols, p_rows;
        status = map_operand(&x_cols, x, true, width, l.chunk_rows, x_row, l.planes, x_plane, false);
        if (status == SS_OK && l.dw) status = map_operand(&x_rows, x, true, width, l.chunk_rows, x_row, l.planes, x_plane, true);
        if (status == SS_OK && l.dx) status = map_operand(&p_cols, a.p16, true, vocab, l.chunk_rows, p_row, l.planes, p_plane, false);
        if (status == SS_OK && l.dw) status = map_operand(&p_rows, a.p16, true, vocab, l.chunk_rows, p_row, l.planes, p_plane, true);
        if (status != SS_OK) return status;

        Product pz = product_of(l.chunk_rows, vocab, width, l.f32);
        pz.chunk = kLogitChunk, pz.m_fast = 1, pz.follows = 1, pz.live = a.live, pz.live_from = a.first, pz.live_side = 1;
        const Logits ez{a.target + first, a.target_logit, a.parts, grads && !l.f32 ? a.e16 : nullptr, grads && l.f32 ? a.e32 : nullptr,
                        l.e_ld, a.n_parts, a.vocab, a.k};
        status = launch_product<Logits, false, false>(x_cols, w_cols, pz, ez, st);
        if (status != SS_OK) return status;
        e = launch_next(true, head_statistics_kernel, blocks_for(l.chunk_rows, sms), 256, st, a);
        if (e != cudaSuccess) return cuda_status_public(e);
        if (!grads) continue;
        const dim3 grid(static_cast<unsigned>((l.e_ld / 8 + 255) / 256), static_cast<unsigned>(l.chunk_rows));
        e = l.f32 ? launch_next(true, head_gradient_kernel<true>, grid, 256, st, a) : launch_next(true, head_gradient_kernel<false>, grid, 256, st, a);
        if (e != cudaSuccess) return cuda_status_public(e);
        if (l.dx) {
            Product px = product_of(l.chunk_rows, width, vocab, l.f32);
            px.chunk = l.f32 ? kGradChunkF32 : kGradChunk, px.m_fast = 1, px.follows = 1, px.live = a.live, px.live_from = a.first, px.live_side = 1;
            const Gradient ex{a.acc, nullptr, l.width_ld, a.width, 1, 0};
            status = launch_product<Gradient, false, true>(p_cols, w_rows, px, ex, st);
            if (status != SS_OK) return status;
            e = l.f32 ? launch_next(true, head_dx_kernel<float>, blocks_for(l.chunk_rows, sms), 256, st, a)
                      : launch_next(true, head_dx_kernel<uint16_t>, blocks_for(l.chunk_rows, sms), 256, st, a);
            if (e != cudaSuccess) return cuda_status_public(e);
        }
        if (l.dw) {
            Product pw = product_of(vocab, width, l.chunk_rows, l.f32);
            pw.follows = 1, pw.live = a.live, pw.live_from = a.first, pw.live_side = 2;
            Gradient ew{};
            ew.cols = a.width, ew.add = accumulate || i > 0;
            if (l.sums_w) {
                ew.dst = reinterpret_cast<float*>(ws + l.w32), ew.stride = l.width_ld, ew.vectors = 1, ew.add = i > 0;
            } else if (dw_dt == SS_BF16) {
                ew.dst16 = static_cast<uint16_t*>(dw), ew.stride = dw_stride, ew.vectors = dw_vectors;
            } else {
                ew.dst = static_cast<float*>(dw), ew.stride = dw_stride, ew.vectors = dw_vectors;
            }
            if (ew.dst16 == nullptr) pw.chunk = l.f32 ? kGradChunkF32 : kGradChunk;
            status = launch_product<Gradient, true, true>(p_rows, x_rows, pw, ew, st);
            if (status != SS_OK) return status;
        }
    }
    if (l.sums_w) {
        const int64_t most = static_cast<int64_t>(sms) * 16;
        e = launch_next(true, head_round_kernel, static_cast<unsigned>(vocab < most ? vocab : most), 256, st, reinterpret_cast<const float*>(ws + l.w32), l.width_ld,
                        static_cast<uint16_t*>(dw), dw_stride, vocab, a.width);
        if (e != cudaSuccess) return cuda_status_public(e);
    }
    return cuda_status_public(launch_next(true, head_totals_kernel, 1, 1024, st, a, 0));
}

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" {
#pragma GCC visibility push(default)

int64_t ss_linear_cross_entropy_workspace(const void* w, int64_t w_stride, ss_dtype dt, int64_t rows, int64_t width, int64_t vocab,
                                          int want_dx, int want_dw, ss_dtype dw_dt) {
    if (!dtype_known(dt) || !sizes_ok(rows, width, vocab) || !stride_ok(vocab, width, w_stride) || (want_dw && !dtype_known(dw_dt))) return -1;
    if (rows == 0) return 0;
    Layout l;
    return layout_of(w, w_stride, dt, rows, width, vocab, want_dx != 0, want_dw != 0, dw_dt, &l) == SS_OK ? l.bytes : -1;
}

int ss_linear_cross_entropy(const void* x, int64_t x_stride, const void* w, int64_t w_stride, ss_dtype dt, int64_t rows,
                            int64_t width, int64_t vocab, const int64_t* targets, const float* weights,
                            float inv_temperature, float z_coef, const float* grad_scale, float* totals, float* logp,
                            void* dx, int64_t dx_stride, void* dw, int64_t dw_stride, ss_dtype dw_dt, int accumulate,
                            void* workspace, int64_t workspace_bytes, void* cuda_stream) {
    if (!dtype_known(dt) || !sizes_ok(rows, width, vocab)) return SS_ERR_INVALID_ARG;
    if (dw != nullptr && (!dtype_known(dw_dt) || (dt == SS_F32 && dw_dt != SS_F32) || (accumulate && dw_dt != SS_F32))) return SS_ERR_INVALID_ARG;
    if (!stride_ok(rows, width, x_stride) || !stride_ok(vocab, width, w_stride)) return SS_ERR_INVALID_ARG;
    if ((dx != nullptr && !stride_ok(rows, width, dx_stride)) || (dw != nullptr && !stride_ok(vocab, width, dw_stride))) return SS_ERR_INVALID_ARG;
    if (!(inv_temperature > 0.0f) || !std::isfinite(inv_temperature) || !std::isfinite(z_coef) || totals == nullptr) return SS_ERR_INVALID_ARG;
    const size_t eb = dtype_bytes(dt), web = dtype_bytes(dw_dt);
    const bool any_w = vocab > 0 && width > 0;
    if (rows > 0 && (x == nullptr || w == nullptr || targets == nullptr || weights == nullptr || logp == nullptr)) return SS_ERR_INVALID_ARG;
    const size_t n = static_cast<size_t>(rows);
    const void* const vecs[] = {targets, weights, grad_scale, totals, logp};
    const size_t align[] = {8, 4, 4, 4, 4}, size[] = {8 * n, 4 * n, grad_scale == nullptr ? 0u : 4u, 8, 4 * n};
    for (int i = 0; i < 5; ++i)
        if (!addr_aligned(vecs[i], align[i])) return SS_ERR_MISALIGNED;
    if (!addr_aligned(x, eb) || !addr_aligned(w, eb) || !addr_aligned(dx, eb) || !addr_aligned(dw, web)) return SS_ERR_MISALIGNED;
    const Mat mx = mat(x, rows, width, x_stride, eb), mw = mat(w, vocab, width, w_stride, eb);
    const Mat mdx = mat(dx, dx == nullptr ? 0 : rows, width, dx_stride, eb), mdw = mat(dw, dw == nullptr ? 0 : vocab, width, dw_stride, web);
    // dx may be x in place: x is gathered before dx is written
    if (mats_overlap(mdx, mw) || (mats_overlap(mdx, mx) && !same_mat(mdx, mx)) || mats_overlap(mdw, mw) || mats_overlap(mdw, mx) || mats_overlap(mdw, mdx)) return SS_ERR_INVALID_ARG;
    for (int i = 0; i < 5; ++i) {
        if (mat_overlaps(mdx, vecs[i], size[i]) || mat_overlaps(mdw, vecs[i], size[i])) return SS_ERR_INVALID_ARG;
        for (int o = 3; o < 5; ++o)
            if (i < o && bytes_overlap(vecs[o], size[o], vecs[i], size[i])) return SS_ERR_INVALID_ARG;
        if (i >= 3 && (mat_overlaps(mx, vecs[i], size[i]) || mat_overlaps(mw, vecs[i], size[i]))) return SS_ERR_INVALID_ARG;
    }
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    Head a{};
    a.targets = targets, a.weights = weights, a.grad_scale = grad_scale, a.totals = totals, a.logp = logp;
    if (rows == 0) {
        cudaError_t e = launch_next(false, head_totals_kernel, 1, 1024, st, a, 1);
        if (e == cudaSuccess && dw != nullptr && any_w && !accumulate)
            e = launch_next(false, head_zero_kernel, static_cast<unsigned>(vocab < 4096 ? vocab : 4096), 256, st, dw, static_cast<int64_t>(width * web),
                            static_cast<int64_t>(mdw.stride * web), vocab);
        return cuda_status_public(e);
    }
    Layout l;
    const int status = layout_of(w, w_stride, dt, rows, width, vocab, dx != nullptr, dw != nullptr, dw_dt, &l);
    if (status != SS_OK) return status;
    if (workspace == nullptr || workspace_bytes < l.bytes) return SS_ERR_INVALID_ARG;
    if (!addr_aligned(workspace, 256)) return SS_ERR_MISALIGNED;
    for (const Mat* m : {&mx, &mw, &mdx, &mdw})
        if (mat_overlaps(*m, workspace, l.bytes)) return SS_ERR_INVALID_ARG;
    for (int i = 0; i < 5; ++i)
        if (bytes_overlap(vecs[i], size[i], workspace, l.bytes)) return SS_ERR_INVALID_ARG;
    a.rows = rows, a.x_stride = mx.stride, a.w_stride = mw.stride, a.dx_stride = mdx.stride, a.x = x, a.w = w, a.dx = dx;
    a.width = static_cast<int>(width), a.vocab = static_cast<int>(vocab);
    a.vectors = mx.row_aligned(4 * eb), a.w_vectors = mw.row_aligned(4 * eb), a.dx_vectors = mdx.row_aligned(4 * eb);
    a.c = inv_temperature, a.k = inv_temperature * 1.44269504f, a.z_coef = z_coef;
    return run(a, l, static_cast<uint8_t*>(workspace), dw, mdw.stride, dw_dt, mdw.row_aligned(4 * web), accumulate, st);
}

#pragma GCC visibility pop
}  // extern "C"
