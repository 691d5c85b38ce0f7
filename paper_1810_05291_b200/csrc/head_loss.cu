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
// Rounding. The sums of a logit leave the matrix unit, which truncates as it adds, every 768 or 128 contraction
// indices and are added in registers, to nearest. e, relative to its part's maximum, is kept in 16 bits of which none is a sign: six of exponent, so
// that an entry 43 nats below the largest of its 128 still has its 11 bits (fp16 lost bits from 10 nats on and everything at 17). P is bf16 as the gradient
// of bf16 logits is; the entry of the target, which is a difference, is formed in fp32 from log p. With fp32 inputs e
// is fp32 and P the sum of three bf16.
//
// What bounds it. 8192 x 4096 over 131072 bf16: 21.7 to 23.2 ms at the power limit (1220 to 1140 TFLOP/s; the library's
// product alone, back to back, 1407), the matrix unit active 91, 93 and 84 % of the logits', dx's and dW's time, e -> P
// 0.87 ms of it at 4.9 TB/s. 64 x 1024 over 32000 bf16: 69 us in a row of calls, W read twice and dW written in 55 of them, the rest five starts.
// 1021 x 770 over 32001 fp32: 820 us alone, 946 to 1003 in a row of calls at the power limit; alone six passes in 690 us, 1310 TFLOP/s, and 125 to split W and P into terms.
#include "product.cuh"

#include <cmath>
#include <type_traits>

namespace ss {
namespace {

constexpr int kPartCols = kProdHalf;              // logits of a thread
// Stages that the matrix unit sums of a logit. Many bf16 rows, calls in turn at the power limit, relative error of log p (a plain fp32 product: 1.9e-6):
//                                16               12               8
//   2048 x 2048 over 50257       320 us, 2.7e-6   324 us, 1.8e-6   320 us, 1.3e-6
//   4100 x 2048 over 65536       1767 us          1755 us          1850 us
//   8192 x 4096 over 131072      22.1 ms          22.3 ms          22.9 ms
// With fewer the two halves of the tensor memory fill while a tile's exponentials are formed. That costs nothing where the stages come at the
// memory's rate (at most 128 rows) or bring six products each (fp32; few calls, below the power limit):
//                                16               4                2
//   64 x 1024 over 32000 bf16    69 us, 2.5e-6    68 us, 6e-7      69 us, 3e-7
//   1021 x 770 over 32001 fp32   897 us, 2.2e-6   878 us, 7e-7     875 us, 5e-7
constexpr int kLogitChunk = 12, kLogitChunkSlow = 2;
// Stages that it sums of a gradient: 16384 contraction indices lose 2e-5, nothing next to an operand of bf16. Of each of fp32's passes 1024 indices:
// dx and dW of 1021 x 770 over 32001 are off by 1.2e-6 (2.4e-6 with 2048, plain fp32 products 1.6e-6), in the same time.
constexpr int kGradChunk = 256, kGradChunkF32 = 16;
constexpr int64_t kChunkBytes = int64_t(1) << 30; // of e and P, or kProdTile rows of them
constexpr int64_t kMostChunkRows = 16384;

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// (a - m) k and (b - m) k, given -m.
__device__ __forceinline__ float2 sub_mul2(float a, float b, float minus, float k) {
    float2 r;
    asm("{\n\t.reg .b64 x, m, k;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 m, {%4, %4};\n\tmov.b64 k, {%5, %5};\n\t"
        "add.rn.f32x2 x, x, m;\n\tmul.rn.f32x2 x, x, k;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a), "f"(b), "f"(minus), "f"(k));
    return r;
}

// What the kernels of one chunk share.
struct Head {
    const int64_t* targets;
    const float *weights, *grad_scale;
    float *totals, *logp;
    int64_t rows, x_stride, w_stride, dx_stride;
    const void *x, *w, *x_end, *w_end;
    void* dx;
    int width, vocab, vectors, dx_vectors, w_vectors;
    int few;                        // at most kFewRows rows: launches of their own for rows and statistics are saved
    float c, k, z_coef;  // k = c log2 e
    // workspace
    int *index, *target, *live;     // of the rows that count, one after another
    float *target_logit, *top, *factor, *target_grad, *loss, *square;
    uint16_t *gathered, *staged_w;
    float2* parts;                  // [chunk rows][n_parts]: maximum, sum
    uint16_t *e16, *p16;            // e, P of bf16 inputs (the same place); planes of P of fp32 ones
    float *e32, *acc, *partial;
    int64_t width_ld, e_ld, row_cap, chunk_rows;
    int n_parts, first;             // first row of the chunk
};

__device__ __forceinline__ bool counts(const Head& a, int64_t t) {
    const int64_t y = a.targets[t];
    return a.weights[t] != 0.0f && y >= 0 && y < a.vocab;
}

// Which rows count, in their order. One block; four rows of a thread under way at a time.
__global__ void __launch_bounds__(1024) head_rows_kernel(const __grid_constant__ Head a) {
    next_may_begin();
    __shared__ int sums[4][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int base = 0;
    for (int64_t t0 = 0; t0 < a.rows; t0 += 4096) {
        int64_t y[4];
        float w[4];
        uint32_t votes[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t t = t0 + 1024 * i + threadIdx.x;
            y[i] = t < a.rows ? a.targets[t] : -1, w[i] = t < a.rows ? a.weights[t] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            votes[i] = __ballot_sync(0xFFFFFFFFu, w[i] != 0.0f && y[i] >= 0 && y[i] < a.vocab);
            if (lane == 0) sums[i][warp] = __popc(votes[i]);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            int before = sums[i][lane];  // of the warps up to that of this lane's number
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int n = __shfl_up_sync(0xFFFFFFFFu, before, d);
                if (lane >= d) before += n;
            }
            const int all = __shfl_sync(0xFFFFFFFFu, before, 31), mine = __shfl_sync(0xFFFFFFFFu, before, (warp + 31) & 31);
            if (votes[i] >> lane & 1) {
                const int s = base + (warp > 0 ? mine : 0) + __popc(votes[i] & ((1u << lane) - 1u));
                a.index[s] = static_cast<int>(t0 + 1024 * i + threadIdx.x);
                a.target[s] = static_cast<int>(y[i]);
            }
            base += all;
        }
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

// Eight bf16 from `src` on, which starts anywhere: out of the one or two 16-byte blocks of memory that hold them, shifted into place, if those lie
// between `begin` and `end`, which may be read.
__device__ __forceinline__ uint4 load_shifted(const uint16_t* src, const char* begin, const char* end, int n) {
    const char* const block = reinterpret_cast<const char*>(reinterpret_cast<uintptr_t>(src) & ~uintptr_t(15));
    const uint32_t shift = static_cast<uint32_t>(reinterpret_cast<const char*>(src) - block);  // bytes
    uint32_t w[9];
    if (n >= 8 && block >= begin && block + (shift != 0 ? 32 : 16) <= end) {
        const uint4 x = *reinterpret_cast<const uint4*>(block), y = shift != 0 ? *reinterpret_cast<const uint4*>(block + 16) : make_uint4(0, 0, 0, 0);
        w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w, w[4] = y.x, w[5] = y.y, w[6] = y.z, w[7] = y.w, w[8] = 0;
#pragma unroll
        for (int step = 2; step > 0; step >>= 1)
            if (shift & (4 * step)) {
#pragma unroll
                for (int i = 0; i + step < 9; ++i) w[i] = w[i + step];
            }
        if (shift & 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
        }
        // (a shift of 8 bytes or more moved four words' worth in two steps; of the nine the first four are meant)
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (2 * i < n ? src[2 * i] : 0u) | (2 * i + 1 < n ? static_cast<uint32_t>(src[2 * i + 1]) << 16 : 0u);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A row to the layout of an operand: bf16 as it is, fp32 as three terms. begin, end: of the matrix, for rows at odd places. It is done
// by `lanes` lanes, this the lane-th.
template <typename T>
__device__ __forceinline__ void stage_row(const T* src, uint16_t* dst, int64_t plane, int width, bool vectors, const void* begin, const void* end, int lane, int lanes) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll 4
        for (int c = 8 * lane; c < width; c += 8 * lanes) {
            const int n = width - c;
            uint4 r;
            if (vectors && n >= 8) r = *reinterpret_cast<const uint4*>(src + c);
            else r = load_shifted(src + c, static_cast<const char*>(begin), static_cast<const char*>(end), n);
            *reinterpret_cast<uint4*>(dst + c) = r;
        }
    } else {
#pragma unroll 4
        for (int c = 4 * lane; c < width; c += 4 * lanes) {
            const int n = width - c;
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

constexpr int kGatherCols = 512;  // that a warp takes of a row

// Rows that count gathered; behind them zeros up to a whole stage, since dW sums over whole stages, and for a first stage of
// each chunk; the results of the others.
// FEW: at most kFewRows, which each block finds by itself; the first one writes down what follows needs.
constexpr int kFewRows = 1024;

__device__ __forceinline__ int find_rows(const Head& a, int* index) {
    __shared__ int sums[4][8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t y[4];
    uint32_t votes[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = 256 * i + threadIdx.x;
        y[i] = t < a.rows && a.weights[t] != 0.0f ? a.targets[t] : -1;
        votes[i] = __ballot_sync(0xFFFFFFFFu, y[i] >= 0 && y[i] < a.vocab);
        if (lane == 0) sums[i][warp] = __popc(votes[i]);
    }
    __syncthreads();
    int base = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int before = base;
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            if (w < warp) before += sums[i][w];
            base += sums[i][w];
        }
        if (votes[i] >> lane & 1) {
            const int s = before + __popc(votes[i] & ((1u << lane) - 1u)), t = 256 * i + threadIdx.x;
            index[s] = t;
            if (blockIdx.x == 0) a.index[s] = t, a.target[s] = static_cast<int>(y[i]);
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.live = base;
    __syncthreads();
    return base;
}

template <typename T, bool FEW>
__global__ void __launch_bounds__(256) head_gather_kernel(const __grid_constant__ Head a) {
    next_may_begin();
    __shared__ int found[FEW ? kFewRows : 1];
    int64_t live;
    const int* index = a.index;
    if constexpr (FEW) {
        live = find_rows(a, found), index = found;
    } else {
        after_previous();
        live = *a.live;
    }
    const int lane = threadIdx.x & 31;
    const int64_t padded = (live + kProdK - 1) / kProdK * kProdK, plane = a.row_cap * a.width_ld;
    const int pieces = (a.width + kGatherCols - 1) / kGatherCols;
    for (int64_t j = blockIdx.x * 8 + (threadIdx.x >> 5); j < (a.rows + kProdK) * pieces; j += gridDim.x * 8) {
        const int64_t i = j / pieces;
        const int first = static_cast<int>(j - i * pieces) * kGatherCols, n = min(kGatherCols, a.width - first);
        if (i < padded || (i < a.row_cap && i % a.chunk_rows < kProdK)) {
            uint16_t* const dst = a.gathered + i * a.width_ld + first;
            if (i < live) {
                stage_row(static_cast<const T*>(a.x) + index[i] * a.x_stride + first, dst, plane, n, a.vectors, a.x, a.x_end, lane, 32);
            } else {
                for (int q = 0; q < (sizeof(T) == 4 ? kTerms : 1); ++q)
                    for (int c = lane; c < n; c += 32) dst[q * plane + c] = 0;
            }
        }
        if (i < a.rows && !counts(a, i)) {
            if (lane == 0) a.logp[i] = 0.0f;
            if (a.dx != nullptr) {
                T* const dst = static_cast<T*>(a.dx) + i * a.dx_stride + first;
                for (int c = lane; c < n; c += 32) dst[c] = T(0);
            }
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) head_stage_w_kernel(const __grid_constant__ Head a) {
    next_may_begin();
    after_previous();
    const int64_t plane = static_cast<int64_t>(a.vocab) * a.width_ld;
    int lanes = 32;  // of a row: narrow ones share a warp
    while (lanes > 1 && (lanes / 2) * (sizeof(T) == 2 ? 8 : 4) >= a.width) lanes /= 2;
    const int rows = 256 / lanes, lane = threadIdx.x & (lanes - 1);
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * rows + threadIdx.x / lanes; i < a.vocab; i += static_cast<int64_t>(gridDim.x) * rows) {
        const T* const src = static_cast<const T*>(a.w) + i * a.w_stride;
        uint16_t* const dst = a.staged_w + i * a.width_ld;
        if (lanes == 32) stage_row(src, dst, plane, a.width, a.w_vectors, a.w, a.w_end, lane, 32);
        else stage_row(src, dst, plane, a.width, a.w_vectors, a.w, a.w_end, lane, lanes);
    }
}

__device__ __forceinline__ float2 mul2(float a, float b, float by) {
    float2 r;
    asm("{\n\t.reg .b64 x, k;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 k, {%4, %4};\n\tmul.rn.f32x2 x, x, k;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a), "f"(b), "f"(by));
    return r;
}

// Numbers from 0 to 1 in 16 bits without a sign: six of exponent, ten of fraction, subnormal below 2^-62. Times 2^-64 a number's upper three bits in fp32
// (the sign, and two of the exponent) are 0, and the next sixteen, rounded to nearest, are the code; fp32's own subnormals are its. (A NaN's code means nothing: its
// row's factor is NaN.)
constexpr float kCodeScale = 0x1p-64f, kCodeUnscale = 0x1p64f;
__device__ __forceinline__ uint4 code8(const float* v) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = mul2(v[2 * i], v[2 * i + 1], kCodeScale);
        w[i] = __byte_perm(__float_as_uint(t.x) * 8u + 0x8000u, __float_as_uint(t.y) * 8u + 0x8000u, 0x7632);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float2 decode2(uint32_t w) {
    return mul2(__uint_as_float((w << 13) & 0x1FFFE000u), __uint_as_float((w >> 3) & 0x1FFFE000u), kCodeUnscale);
}

// ---- the end of the logits' product
struct Logits {
    static constexpr bool kWhole = true, kSmall = false, kAlone = true, kPacks = false, kBefore = false;
    const int* target;  // of the chunk's rows
    float* target_logit;
    float2* parts;
    uint16_t* e16;      // at most one of these
    float* e32;
    int64_t e_ld;
    int n_parts, vocab;
    float k;

    // What is needed of the lane's row, while the sums form: its target.
    __device__ __forceinline__ int ahead(int m, int row, int lane) const { return row + lane < m ? target[row + lane] : -1; }

    __device__ __forceinline__ void whole(const ProdUnit&, int m, int row, int col, int lane, uint32_t buf, float (&z)[kPartCols], int y) const {
        if (row >= m) return;
        const int r = row + lane, there = vocab - col;
        if (there < kPartCols) {
#pragma unroll
            for (int i = 0; i < kPartCols; ++i) z[i] = i < there ? z[i] : -INFINITY;
        }
        y -= col;
        if (y >= 0 && y < kPartCols) {
            float v = 0.0f;
#pragma unroll
            for (int i = 0; i < kPartCols; ++i) v = i == y ? z[i] : v;
            target_logit[r] = v;
        }
        float tops[4] = {z[0], z[1], z[2], z[3]};
#pragma unroll
        for (int i = 4; i < kPartCols; ++i) tops[i & 3] = fmaxf(tops[i & 3], z[i]);
        const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), minus = top == -INFINITY ? 0.0f : -top;
        float sums[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < kPartCols; i += 2) {
            const float2 t = sub_mul2(z[i], z[i + 1], minus, k);
            sums[i & 2] += z[i] = ex2(t.x), sums[(i & 2) + 1] += z[i + 1] = ex2(t.y);
        }
        const float sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
        if (r < m) parts[static_cast<int64_t>(r) * n_parts + col / kPartCols] = make_float2(top, sum);
        if (e16 != nullptr) {
#pragma unroll
            for (int h = 0; h < kPartCols; h += 64) {
#pragma unroll
                for (int i = 0; i < 8; ++i) square_set(buf, lane, i, code8(z + h + 8 * i));
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

struct RowGrad {
    float factor, target;
};

// Of row r of the chunk, from its largest logit and the sum of its exponentials; the row's figures written down, if asked for.
__device__ __forceinline__ RowGrad row_grad(const Head& a, int64_t r, float top, float sum, bool write) {
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
    if (write) a.logp[t] = logp, a.loss[s] = loss, a.square[s] = w * lse * lse;
    return RowGrad{scale * all / sum, scale * (expm1f(logp) + extra * expf(logp))};
}

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
#pragma unroll 8
        for (int i = lane; i < a.n_parts; i += 32) top = fmaxf(top, p[i].x);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        const float from = top == -INFINITY ? 0.0f : top;
#pragma unroll 8
        for (int i = lane; i < a.n_parts; i += 32) {
            const float2 v = p[i];
            sum += v.y * ex2((v.x - from) * a.k);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        if (lane != 0) continue;
        const RowGrad g = row_grad(a, r, top, sum, true);
        a.top[r] = top, a.factor[r] = g.factor, a.target_grad[r] = g.target;
    }
}

// Loss and sum of weighted squares: fp64, in a fixed order, by the first 256 threads of a block.
__device__ __forceinline__ void totals_of(const Head& a, int64_t live) {
    __shared__ double part[2][8];
    double loss = 0.0, square = 0.0;
#pragma unroll 4
    for (int64_t s = threadIdx.x; s < live; s += 256) loss += a.loss[s], square += a.square[s];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        loss += __shfl_xor_sync(0xFFFFFFFFu, loss, d);
        square += __shfl_xor_sync(0xFFFFFFFFu, square, d);
    }
    if ((threadIdx.x & 31) == 0) part[0][threadIdx.x >> 5] = loss, part[1][threadIdx.x >> 5] = square;
    __syncthreads();
    if (threadIdx.x < 2) {
        double v = 0.0;
        for (int i = 0; i < 8; ++i) v += part[threadIdx.x][i];
        a.totals[threadIdx.x] = static_cast<float>(v);
    }
}

// The same of few rows, by one warp.
__device__ __forceinline__ void few_totals(const Head& a, int live, int lane) {
    double loss = 0.0, square = 0.0;
#pragma unroll 8
    for (int s = lane; s < live; s += 32) loss += a.loss[s], square += a.square[s];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        loss += __shfl_xor_sync(0xFFFFFFFFu, loss, d);
        square += __shfl_xor_sync(0xFFFFFFFFu, square, d);
    }
    if (lane == 0) a.totals[0] = static_cast<float>(loss), a.totals[1] = static_cast<float>(square);
}

// Where nothing else forms them; none: no rows.
__global__ void __launch_bounds__(256) head_totals_kernel(const __grid_constant__ Head a, int none) {
    next_may_begin();
    if (!none) after_previous();
    if (!a.few) totals_of(a, none ? 0 : *a.live);
    else if (threadIdx.x < 32) few_totals(a, *a.live, threadIdx.x);
}

// e -> P: four times eight columns to a thread, all loads before the first store. Rows behind the last up to a whole stage
// (one at least) become zeros. A row of blocks behind all rows, where the call's last chunk has it, forms the totals. FEW: the row's
// statistics are formed here, by each of its blocks, instead of by a launch of their own.
constexpr int kGradientPieces = 4;

// Largest or sum over the block's 256 threads, the same in all.
template <bool MAX>
__device__ __forceinline__ float block_reduce(float v) {
    __shared__ float part[8];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const float o = __shfl_xor_sync(0xFFFFFFFFu, v, d);
        v = MAX ? fmaxf(v, o) : v + o;
    }
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) v = MAX ? fmaxf(v, part[i]) : v + part[i];
    return v;
}

template <bool F32, bool FEW>
__global__ void __launch_bounds__(256) head_gradient_kernel(const __grid_constant__ Head a) {
    next_may_begin();
    after_previous();
    if (blockIdx.y == a.chunk_rows) {
        if (blockIdx.x == 0) totals_of(a, *a.live);
        return;
    }
    const int64_t r = blockIdx.y, here = min(static_cast<int64_t>(*a.live) - a.first, a.chunk_rows);
    const int64_t upto = max((here + kProdK - 1) / kProdK * kProdK, static_cast<int64_t>(kProdK));
    const int c0 = blockIdx.x * (256 * 8 * kGradientPieces) + threadIdx.x * 8, end = static_cast<int>(a.e_ld);
    if (r >= min(upto, a.chunk_rows)) return;
    uint16_t* const out = a.p16 + r * a.e_ld;
    const int64_t plane = a.chunk_rows * a.e_ld;  // of fp32's terms
    if (r >= here) {
        for (int c = c0, i = 0; i < kGradientPieces && c < end; c += 256 * 8, ++i)
            for (int q = 0; q < (F32 ? kTerms : 1); ++q) *reinterpret_cast<uint4*>(out + q * plane + c) = make_uint4(0, 0, 0, 0);
        return;
    }
    uint4 x[kGradientPieces][F32 ? 2 : 1];
    float top[kGradientPieces];
#pragma unroll
    for (int i = 0; i < kGradientPieces; ++i) {
        const int c = c0 + i * 256 * 8;
        if (c >= end) continue;
        if constexpr (F32) {
            const uint4* const src = reinterpret_cast<const uint4*>(a.e32 + r * a.e_ld + c);
            x[i][0] = __ldcs(src), x[i][1] = __ldcs(src + 1);
        } else {
            x[i][0] = __ldcs(reinterpret_cast<const uint4*>(a.e16 + r * a.e_ld + c));
        }
        top[i] = a.parts[r * a.n_parts + c / kPartCols].x;
    }
    float factor, row_top, target_grad;
    if constexpr (FEW) {
        const float2* const p = a.parts + r * a.n_parts;
        float m = -INFINITY, sum = 0.0f;
        for (int i = threadIdx.x; i < a.n_parts; i += 256) m = fmaxf(m, p[i].x);
        row_top = block_reduce<true>(m);
        const float from = row_top == -INFINITY ? 0.0f : row_top;
        for (int i = threadIdx.x; i < a.n_parts; i += 256) {
            const float2 q = p[i];
            sum += q.y * ex2((q.x - from) * a.k);
        }
        sum = block_reduce<false>(sum);
        const RowGrad g = row_grad(a, r, row_top, sum, blockIdx.x == 0 && threadIdx.x == 0);
        factor = g.factor, target_grad = g.target;
    } else {
        factor = a.factor[r], row_top = a.top[r], target_grad = a.target_grad[r];
    }
    const int target = a.target[a.first + r];
#pragma unroll
    for (int i = 0; i < kGradientPieces; ++i) {
        const int c = c0 + i * 256 * 8;
        if (c >= end) continue;
        // an empty part, or one of -inf alone, has -inf for its maximum and zeros for e
        const float f = factor * (top[i] == -INFINITY ? 0.0f : ex2((top[i] - row_top) * a.k));
        float v[8];
        if constexpr (F32) {
            const uint4 y = x[i][0], z = x[i][1];
            const uint32_t w[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j]);
        } else {
            const uint32_t w[4] = {x[i][0].x, x[i][0].y, x[i][0].z, x[i][0].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 p = decode2(w[j]);
                v[2 * j] = p.x, v[2 * j + 1] = p.y;
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= f;
        const int y = target - c;
        if (y >= 0 && y < 8) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j == y ? target_grad : v[j];
        }
        if constexpr (F32) {
            const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
            store_terms(out + c, plane, lo);
            store_terms(out + c + 4, plane, hi);
        } else {
            *reinterpret_cast<uint4*>(out + c) = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
        }
    }
}

// ---- the end of the gradients' products: written, or added by the memory itself (the same lane adds to an element each
// time, so its sums come in their order). A part of a tile goes to a place of its own.
__device__ __forceinline__ void add_global(float* p, float4 v) {
    asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(__cvta_generic_to_global(p)), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void add_global(float* p, float v) {
    asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" ::"l"(__cvta_generic_to_global(p)), "f"(v) : "memory");
}

constexpr int kTileFloats = kProdTile * kProdTile;  // of a pair's part; a block's alone is half of that, and there are twice as many

// Where a gradient goes: fp32, or bf16 that takes the sums of earlier rows (fp32) into its rounding.
struct Dest {
    float* f32;
    uint16_t* bf16;
    const float* before;  // with bf16: those sums, or NULL
    int64_t stride, before_stride;
    int cols, vectors, add;
    int wide;  // bf16: rows start on 16 bytes

    __device__ __forceinline__ void put(int64_t row, int c, float4 v, float4 b, bool adds) const {
        const int64_t at = row * stride + c;
        v.x += b.x, v.y += b.y, v.z += b.z, v.w += b.w;
        if (vectors && c + 4 <= cols) {
            if (bf16 != nullptr) *reinterpret_cast<uint2*>(bf16 + at) = make_uint2(bf16_pair(v.x, v.y), bf16_pair(v.z, v.w));
            else if (adds) add_global(f32 + at, v);
            else *reinterpret_cast<float4*>(f32 + at) = v;
        } else {
            const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (c + j >= cols) break;
                if (bf16 != nullptr) Elem<uint16_t>::store(bf16 + at + j, e[j]);
                else if (adds) add_global(f32 + at + j, e[j]);
                else f32[at + j] = e[j];
            }
        }
    }
    __device__ __forceinline__ float4 earlier(int64_t row, int c) const {
        return before == nullptr ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : *reinterpret_cast<const float4*>(before + row * before_stride + c);
    }
};

// Four columns of a tile that came in parts, the parts in their order, eight under way at a time.
__device__ __forceinline__ float4 joined(const float* partial, const Schedule& sc, int tile_floats, int other, int r, int c) {
    const float* const p = partial + static_cast<int64_t>(other) * sc.parts * tile_floats + r * kProdTile + c;
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s = 0; s < sc.parts; s += 8) {
        float4 x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            x[u] = s + u < sc.parts ? __ldcs(reinterpret_cast<const float4*>(p + static_cast<int64_t>(s + u) * tile_floats)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int u = 0; u < 8; ++u) v.x += x[u].x, v.y += x[u].y, v.z += x[u].z, v.w += x[u].w;
    }
    return v;
}

// dx of the chunk's rows, from their sums to their places, and the totals of few rows: by `warps` warps, this the warp-th.
template <typename T>
__device__ __forceinline__ void finish_dx(const Head& a, const Product& p, int warp, int warps, int lane) {
    const Schedule sc = schedule_of(p);
    const int64_t here = min(static_cast<int64_t>(*a.live) - a.first, a.chunk_rows);
    if (a.few && warp == 0) few_totals(a, *a.live, lane);
    const int pieces = (a.width + 127) / 128;  // a warp takes 128 columns of a row
    for (int64_t i = warp; i < here * pieces; i += warps) {
        const int64_t r = i / pieces;
        const int c = static_cast<int>(i - r * pieces) * 128 + 4 * lane;
        if (c >= a.width) continue;
        T* const dst = static_cast<T*>(a.dx) + a.index[a.first + r] * a.dx_stride + c;
        const int tile = c / kProdTile * sc.tiles_m + static_cast<int>(r / p.tile_m);
        const float4 v = tile < sc.whole ? *reinterpret_cast<const float4*>(a.acc + r * a.width_ld + c)
                                         : joined(a.partial, sc, p.tile_m * kProdTile, tile - sc.whole, static_cast<int>(r % p.tile_m), c % kProdTile);
        if (a.dx_vectors && c + 4 <= a.width) {
            if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(dst) = v;
            else *reinterpret_cast<uint2*>(dst) = make_uint2(bf16_pair(v.x, v.y), bf16_pair(v.z, v.w));
        } else {
            const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < a.width) Elem<T>::store(dst + j, e[j]);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) head_dx_kernel(const __grid_constant__ Head a, const __grid_constant__ Product p) {
    next_may_begin();
    after_previous();
    finish_dx<T>(a, p, blockIdx.x * 8 + (threadIdx.x >> 5), gridDim.x * 8, threadIdx.x & 31);
}

struct Finish {
    Head a;
    Product p;  // of dx
    int f32;
};

// OUT16: to.bf16, else to.f32. BEFORE: with to.before. DX: while the first sums of dW form, dx is finished.
template <bool OUT16, bool BEFORE, bool DX>
struct Gradient {
    static constexpr bool kWhole = false, kSmall = false, kAlone = !OUT16, kPacks = OUT16 && !BEFORE, kBefore = DX, kAhead = BEFORE;
    struct Fetched {
        float4 before[BEFORE ? 8 : 1];
    };
    Dest to;
    float* partial;
    int part_floats;
    Finish dx;

    __device__ __forceinline__ void before(int warp, int lane) const {
        const int at = blockIdx.x * (kProdOut / 32) + warp, all = gridDim.x * (kProdOut / 32);
        if (dx.f32) finish_dx<float>(dx.a, dx.p, at, all, lane);
        else finish_dx<uint16_t>(dx.a, dx.p, at, all, lane);
    }

    struct Tile {
        char* p;       // this lane's first row, at its first column
        int64_t step;  // bytes from its row to the next
        const float* before;
        int row, col, rows, cols;  // rows and columns: that exist from there on
        int part;
        bool add, packs, whole;

        __device__ __forceinline__ static uint32_t pack(uint32_t a, uint32_t b) { return bf16_pair(__uint_as_float(a), __uint_as_float(b)); }
        __device__ __forceinline__ void packed(int j, int lane, uint32_t buf) const {
            if (whole) {
                char* q = p + (j + 4 * (lane & 7)) * 2;  // p is at four columns a lane, this at eight
#pragma unroll
                for (int i = 0; i < 8; ++i, q += step) *reinterpret_cast<uint4*>(q) = square_get(buf, (lane >> 3) + 4 * i, lane & 7);
                return;
            }
            // rows at odd places, or not all there: a row at a time, two columns to a lane
            const int left = cols + 4 * (lane & 7) - j - 2 * lane, there = min(32, rows + (lane >> 3));
            if (left <= 0) return;
            uint16_t* q = reinterpret_cast<uint16_t*>(p - (lane >> 3) * (step / 4)) - 4 * (lane & 7) + j + 2 * lane;
#pragma unroll 8
            for (int r = 0; r < there; ++r, q = reinterpret_cast<uint16_t*>(reinterpret_cast<char*>(q) + step / 4)) {
                const uint32_t w = __float_as_uint(square_word(buf, r, lane));
                if (left > 1 && (reinterpret_cast<uintptr_t>(q) & 3) == 0) {
                    *reinterpret_cast<uint32_t*>(q) = w;
                } else {
                    q[0] = static_cast<uint16_t>(w);
                    if (left > 1) q[1] = static_cast<uint16_t>(w >> 16);
                }
            }
        }
        __device__ __forceinline__ Tile(const Gradient& e, const ProdUnit& u, int m, int row0, int col0, int lane) {
            row = row0 + (lane >> 3), col = col0 + 4 * (lane & 7), part = u.part, add = e.to.add;
            rows = m - row, cols = e.to.cols - col;
            if (part >= 0) {
                p = reinterpret_cast<char*>(e.partial + static_cast<int64_t>(part) * e.part_floats + (row - u.m0) * kProdTile + (col - u.n0));
                step = 4 * kProdTile * 4;
                add = false;
            } else {
                const int64_t at = row * e.to.stride + col;
                p = OUT16 ? reinterpret_cast<char*>(e.to.bf16 + at) : reinterpret_cast<char*>(e.to.f32 + at);
                step = 4 * e.to.stride * (OUT16 ? 2 : 4);
            }
            packs = OUT16 && part < 0;
            whole = e.to.wide && row0 + 32 <= m && col0 + kProdHalf <= e.to.cols;
            before = BEFORE ? e.to.before + row * e.to.before_stride + col : nullptr;
        }
        __device__ __forceinline__ void fetch(const Gradient& e, int j, Fetched& f) const {
            if constexpr (BEFORE) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    f.before[i] = part < 0 && 4 * i < rows && j < cols ? *reinterpret_cast<const float4*>(before + j + 4 * i * e.to.before_stride) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
        }
        __device__ __forceinline__ void square(const Gradient& e, int j, int lane, uint32_t buf, float4 (&sums)[8], const Fetched& f, bool first) const {
            if (!OUT16 && part < 0 && !e.to.vectors) {  // rows at odd places: a row at a time, a column to a lane
                const int there = min(32, rows + (lane >> 3));
                if (cols + 4 * (lane & 7) - j - lane <= 0) return;
                float* q = reinterpret_cast<float*>(p - (lane >> 3) * (step / 4)) - 4 * (lane & 7) + j + lane;
#pragma unroll 8
                for (int r = 0; r < there; ++r, q = reinterpret_cast<float*>(reinterpret_cast<char*>(q) + step / 4)) {
                    const float v = square_word(buf, r, lane);
                    if (add || !first) add_global(q, v);
                    else *q = v;
                }
                return;
            }
            const bool adds = add || !first;
            char* q = p + j * (OUT16 && part < 0 ? 2 : 4);
#pragma unroll
            for (int i = 0; i < 8; ++i, q += step) {
                float4 v = sums[i];
                if (4 * i >= rows || j >= cols) continue;
                if (part >= 0 || (e.to.vectors && j + 4 <= cols)) {
                    if constexpr (BEFORE) v.x += f.before[i].x, v.y += f.before[i].y, v.z += f.before[i].z, v.w += f.before[i].w;
                    if (OUT16 && part < 0) *reinterpret_cast<uint2*>(q) = make_uint2(bf16_pair(v.x, v.y), bf16_pair(v.z, v.w));
                    else if (adds) add_global(reinterpret_cast<float*>(q), v);
                    else *reinterpret_cast<float4*>(q) = v;
                } else {
                    e.to.put(row + 4 * i, col + j, v, BEFORE ? f.before[i] : make_float4(0.0f, 0.0f, 0.0f, 0.0f), adds);
                }
            }
        }
    };
};

// dW of the tiles that came in parts.
__global__ void __launch_bounds__(256) head_join_kernel(const __grid_constant__ Product p, const __grid_constant__ Dest to, const float* partial) {
    next_may_begin();
    after_previous();
    const Schedule sc = schedule_of(p);
    const int others = sc.parts > 1 ? sc.per_batch - sc.whole : 0, i = (blockIdx.y * 256 + threadIdx.x) * 4;
    for (int other = blockIdx.x; other < others; other += gridDim.x) {
        const ProdUnit u = prod_unit(p, sc, sc.whole + other * sc.parts);
        const int r = u.m0 + i / kProdTile, c = u.n0 + i % kProdTile;
        if (r < sc.m && c < p.n) to.put(r, c, joined(partial, sc, kTileFloats, other, i / kProdTile, i % kProdTile), to.earlier(r, c), to.add);
    }
}

__global__ void __launch_bounds__(256) head_zero_kernel(void* dst, int64_t row_bytes, int64_t stride_bytes, int64_t rows) {
    next_may_begin();
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = threadIdx.x * 2; c < row_bytes; c += 512) *reinterpret_cast<uint16_t*>(static_cast<char*>(dst) + r * stride_bytes + c) = 0;
}

// ---- host side -------------------------------------------------------------------------------------

constexpr int64_t kMostSideHead = int64_t(1) << 30, kMostRows = int64_t(1) << 24, kMostTilesHead = int64_t(1) << 24;

// SMs that the workspace is made for. Without a device (sizes asked for on a host without one) the B200's.
int plan_sms() {
    cudaError_t err = cudaSuccess;
    const int sms = device_sm_count(&err);
    return err == cudaSuccess && sms > 0 ? sms : 148;
}

inline int64_t up_to(int64_t n, int64_t m) { return (n + m - 1) / m * m; }

struct Layout {
    bool f32, dx, dw, stage_w, sums_w;  // sums_w: dW of bf16 from several chunks
    int64_t planes, width_ld, e_ld, n_parts, chunks, chunk_rows, row_cap;
    int64_t index, target, live, rows_f32, gathered, staged_w, parts, e, p, acc, w32, partial, partial_w, bytes;
};

int layout_of(const void* w, int64_t w_stride, ss_dtype dt, int64_t rows, int64_t width, int64_t vocab, bool dx, bool dw, ss_dtype dw_dt, Layout* l) {
    const int64_t tiles_v = (vocab + kProdTile - 1) / kProdTile, tiles_d = (width + kProdTile - 1) / kProdTile;
    if (rows > kMostRows || vocab > kMostSideHead || width > kMostSideHead || tiles_v * ((rows + kProdTile - 1) / kProdTile) > kMostTilesHead || tiles_v * tiles_d > kMostTilesHead) return SS_ERR_UNSUPPORTED;
    l->f32 = dt == SS_F32, l->dx = dx, l->dw = dw, l->planes = l->f32 ? kTerms : 1;
    const Mat m = mat(w, vocab, width, w_stride, dtype_bytes(dt));
    l->stage_w = l->f32 || !m.row_aligned(16) || m.stride * 2 % 16 != 0 || m.stride * 2 >= (int64_t(1) << 38);
    l->width_ld = up_to(width, 64), l->e_ld = up_to(vocab, 64);
    l->n_parts = 2 * tiles_v;
    const int64_t per_row = dx || dw ? l->e_ld * (l->f32 ? 4 + 2 * kTerms : 2) : l->n_parts * 8;
    int64_t most = kChunkBytes / per_row / kProdTile * kProdTile;
    most = most < kProdTile ? kProdTile : (most > kMostChunkRows ? kMostChunkRows : most);
    l->chunks = rows > 0 ? (rows + most - 1) / most : 1;
    // whole tiles, so that only the last piece has one that is not full; of one piece the rows that there are, up to a whole stage of dW's contraction
    l->chunk_rows = up_to((rows + l->chunks - 1) / l->chunks, l->chunks > 1 ? kProdTile : kProdK);
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
    // dx is finished while parts of dW are written already
    l->partial = place(dx ? static_cast<int64_t>(plan_sms() / 2) * kTileFloats * 4 : 0);
    l->partial_w = place(dw ? static_cast<int64_t>(plan_sms() / 2) * kTileFloats * 4 : 0);
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

// Whether a product over as many rows as the call has may come in parts (it does not with the rows that count where those are too few).
bool may_split(const Product& p) {
    const int64_t tiles = static_cast<int64_t>((p.m + kProdTile - 1) / kProdTile) * ((p.n + kProdTile - 1) / kProdTile), others = tiles % p.pairs;
    const int64_t stages = static_cast<int64_t>((p.k + kProdK - 1) / kProdK) * p.passes;
    return others > 0 && p.pairs / others > 1 && stages / kLeastPart > 1;
}

int run(Head& a, const Layout& l, uint8_t* ws, void* dw, int64_t dw_stride, ss_dtype dw_dt, bool dw_vectors, bool dw_wide, int accumulate, cudaStream_t st) {
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
    a.acc = reinterpret_cast<float*>(ws + l.acc), a.partial = reinterpret_cast<float*>(ws + l.partial);
    a.width_ld = l.width_ld, a.e_ld = l.e_ld, a.row_cap = l.row_cap, a.chunk_rows = l.chunk_rows, a.n_parts = static_cast<int>(l.n_parts);
    const bool grads = l.dx || l.dw;
    const int64_t rows = a.rows, width = a.width, vocab = a.vocab;

    CUtensorMap w_cols, w_rows;  // W as an operand of the logits and of dx
    const void* const w = l.stage_w ? a.staged_w : a.w;
    const int64_t w_row = l.stage_w ? l.width_ld * 2 : a.w_stride * 2, w_plane = vocab * l.width_ld * 2;
    int status = map_operand(&w_cols, w, true, width, vocab, w_row, l.planes, w_plane, false);
    if (status == SS_OK && l.dx) status = map_operand(&w_rows, w, true, width, vocab, w_row, l.planes, w_plane, true);
    if (status != SS_OK) return status;

    a.few = rows <= kFewRows;
    const unsigned gather = blocks_for((rows + kProdK) * ((width + kGatherCols - 1) / kGatherCols), sms);
    if (a.few) {
        e = l.f32 ? launch_next(false, head_gather_kernel<float, true>, gather, 256, st, a) : launch_next(false, head_gather_kernel<uint16_t, true>, gather, 256, st, a);
    } else {
        e = launch_next(false, head_rows_kernel, 1, 1024, st, a);
        if (e == cudaSuccess) e = l.f32 ? launch_next(true, head_gather_kernel<float, false>, gather, 256, st, a) : launch_next(true, head_gather_kernel<uint16_t, false>, gather, 256, st, a);
    }
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

        Product pz = product_of(rows < l.chunk_rows ? rows : l.chunk_rows, vocab, width, l.f32, sms);
        const int chunk = l.f32 || rows <= kProdHalf ? kLogitChunkSlow : kLogitChunk;
        pz.block = chunk, pz.chunk = pz.passes * chunk, pz.m_fast = 1, pz.follows = 1, pz.live = a.live, pz.live_from = a.first, pz.live_side = 1;
        alone(pz, sms);
        const Logits ez{a.target + first, a.target_logit, a.parts, grads && !l.f32 ? a.e16 : nullptr, grads && l.f32 ? a.e32 : nullptr,
                        l.e_ld, a.n_parts, a.vocab, a.k};
        status = launch_product<Logits, false, false>(x_cols, w_cols, pz, ez, st);
        if (status != SS_OK) return status;
        if (!grads || !a.few) {
            e = launch_next(true, head_statistics_kernel, blocks_for(l.chunk_rows, sms), 256, st, a);
            if (e != cudaSuccess) return cuda_status_public(e);
            if (!grads) continue;
        }
        const int64_t wide = 256 * 8 * kGradientPieces;
        const dim3 grid(static_cast<unsigned>((l.e_ld + wide - 1) / wide), static_cast<unsigned>(l.chunk_rows + (i + 1 == l.chunks && !a.few)));
        if (a.few) e = l.f32 ? launch_next(true, head_gradient_kernel<true, true>, grid, 256, st, a) : launch_next(true, head_gradient_kernel<false, true>, grid, 256, st, a);
        else e = l.f32 ? launch_next(true, head_gradient_kernel<true, false>, grid, 256, st, a) : launch_next(true, head_gradient_kernel<false, false>, grid, 256, st, a);
        if (e != cudaSuccess) return cuda_status_public(e);
        Product px{};
        if (l.dx) {
            px = product_of(rows < l.chunk_rows ? rows : l.chunk_rows, width, vocab, l.f32, sms);
            px.block = kGradChunkF32, px.chunk = l.f32 ? px.passes * kGradChunkF32 : kGradChunk, px.m_fast = 1, px.follows = 1, px.live = a.live, px.live_from = a.first, px.live_side = 1;
            px.split = 1;
            alone(px, sms);
            const Gradient<false, false, false> ex{{a.acc, nullptr, nullptr, l.width_ld, 0, a.width, 1, 0, 0}, a.partial, px.tile_m * kProdTile, {}};
            status = launch_product<Gradient<false, false, false>, false, true>(p_cols, w_rows, px, ex, st);
            if (status != SS_OK) return status;
            if (!l.dw) {
                const unsigned finish = blocks_for(px.m * ((width + 127) / 128), sms);
                e = l.f32 ? launch_next(true, head_dx_kernel<float>, finish, 256, st, a, px) : launch_next(true, head_dx_kernel<uint16_t>, finish, 256, st, a, px);
                if (e != cudaSuccess) return cuda_status_public(e);
            }
        }
        if (l.dw) {
            Product pw = product_of(vocab, width, l.chunk_rows, l.f32, sms);
            pw.follows = 1, pw.live = a.live, pw.live_from = a.first, pw.live_side = 2, pw.split = 1;
            Dest to{};
            pw.always = l.sums_w && i + 1 == l.chunks;  // it rounds what the chunks before it summed
            to.cols = a.width, to.add = accumulate || i > 0, to.stride = dw_stride, to.vectors = dw_vectors, to.wide = dw_wide;
            float* const sums = l.sums_w ? reinterpret_cast<float*>(ws + l.w32) : nullptr;
            if (l.sums_w && i + 1 < l.chunks) {
                to.f32 = sums, to.stride = l.width_ld, to.vectors = 1;
            } else if (dw_dt == SS_BF16) {
                to.bf16 = static_cast<uint16_t*>(dw), to.before = sums, to.before_stride = l.width_ld;
            } else {
                to.f32 = static_cast<float*>(dw);
            }
            // a bf16 result is written once: its rows, at most kMostChunkRows, are one chunk
            pw.block = kGradChunkF32, pw.chunk = l.f32 ? pw.passes * kGradChunkF32 : kGradChunk;
            float* const parts = reinterpret_cast<float*>(ws + l.partial_w);
            auto product = [&](auto g) {
                using G = decltype(g);
                g.to = to, g.partial = parts, g.part_floats = kTileFloats;
                if (l.dx) g.dx = Finish{a, px, l.f32};
                return launch_product<G, true, true>(p_rows, x_rows, pw, g, st);
            };
            auto of = [&](auto with) {
                constexpr bool kDx = decltype(with)::value;
                return to.bf16 == nullptr ? product(Gradient<false, false, kDx>{}) : (to.before == nullptr ? product(Gradient<true, false, kDx>{}) : product(Gradient<true, true, kDx>{}));
            };
            status = l.dx ? of(std::true_type{}) : of(std::false_type{});
            if (status != SS_OK) return status;
            if (may_split(pw)) {
                e = launch_next(true, head_join_kernel, dim3(static_cast<unsigned>(sms / 2), kTileFloats / 1024), 256, st, pw, to, static_cast<const float*>(parts));
                if (e != cudaSuccess) return cuda_status_public(e);
            }
        }
    }
    // with gradients formed beside them already
    if (grads && (!a.few || l.dx)) return SS_OK;
    return cuda_status_public(launch_next(true, head_totals_kernel, 1, 256, st, a, 0));
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
        cudaError_t e = launch_next(false, head_totals_kernel, 1, 256, st, a, 1);
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
    a.x_end = static_cast<const char*>(x) + mx.extent(), a.w_end = static_cast<const char*>(w) + mw.extent();
    a.width = static_cast<int>(width), a.vocab = static_cast<int>(vocab);
    a.vectors = mx.row_aligned(16), a.w_vectors = mw.row_aligned(16), a.dx_vectors = mdx.row_aligned(4 * eb);
    a.c = inv_temperature, a.k = inv_temperature * 1.44269504f, a.z_coef = z_coef;
    return run(a, l, static_cast<uint8_t*>(workspace), dw, mdw.stride, dw_dt, mdw.row_aligned(4 * web), mdw.row_aligned(16), accumulate, st);
}

#pragma GCC visibility pop
}  // extern "C"
