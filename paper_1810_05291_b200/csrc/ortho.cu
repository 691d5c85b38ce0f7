// The orthogonal update: X <- a X + (b S + c S S) X with S = X X^T over the smaller side, some steps.
//
// A step is three products: S (symmetric: tiles on and above the diagonal, each stored twice), Q = b S + c S S
// (symmetric as well) and Y = a X + Q X, the sums of each brought from the tensor memory straight into what the
// next one reads. A tall matrix has S = X^T X and X Q instead; the operands' maps differ, nothing is transposed.
//
// Rounding. The operands X, S and Q are fp16: with bf16 (8 bits) the result is 1 to 3 % off, with fp16 0.2 %. The
// term a X takes X from fp32: it alone carries the directions whose singular values are small, which each step
// enlarges 3.4 times; with 11 bits there a momentum of few strong directions comes out 0.35 % off instead of
// 0.03 %. (As the sum of two fp16, the first of them the operand, X has two bytes less to move for each element and
// step and 22 bits, but takes seven instructions more: the same time within 2 %.)
//
// What bounds it. 4096 x 4096 bf16: 1140 us alone, 1330 to 1400 in a row of calls at the power limit; alone S and Q take 54 to 58 us each (136
// tiles in two rounds of 74 pairs, the matrix unit active 75 %), X + Q X 101 to 109 (79 %), the two passes of the start 40. Twelve of 4096 x 1024
// with momenta and parameters: 1260 us alone, 1420 to 1500 in a row; alone X + Q X takes 125 of them each, where its products alone take 62 and its 600 MB 92.
// 1000 x 2048: 151 us, 15 products of 8 to 10 us one after another. 128 x 128: 25 us in one launch.
#include "../../include/signsgd_ortho.h"
#include "product.cuh"

#include <cuda_fp16.h>

#include <atomic>
#include <cmath>

namespace ss {
namespace {

constexpr int kMostMatrices = SS_ORTHO_MAX_MATRICES;

struct Table {
    const void* p[kMostMatrices];
};

__device__ __forceinline__ uint2 half4(float4 v) {
    const __half2 a = __floats2half2_rn(v.x, v.y), b = __floats2half2_rn(v.z, v.w);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ float4 float4_of(uint2 h) {
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&h.x)), b = __half22float2(*reinterpret_cast<const __half2*>(&h.y));
    return make_float4(a.x, a.y, b.x, b.y);
}
// ---- ends of the products --------------------------------------------------------------------------

// out = c sums (+ b lin), symmetric: a square of a tile above the diagonal is stored a second time, mirrored.
template <bool LIN>
struct Symmetric {
    static constexpr bool kWhole = false, kSmall = true, kAlone = false, kPacks = false, kBefore = false, kAhead = true;
    static constexpr int kSmallBlocks = 2;
    struct Fetched {
        uint2 lin[LIN ? 8 : 1];
    };
    uint16_t* out;
    const uint16_t* lin;
    int64_t plane;
    int ld;
    float b, c;

    struct Tile {
        uint16_t *to, *mirrored;
        const uint16_t* from;
        int rows, cols;  // that exist from this lane's first row on, and from its first column's mirrored row on
        bool mirror;

        __device__ __forceinline__ Tile(const Symmetric& e, const ProdUnit& u, int m, int row, int col, int lane) {
            const int64_t r = row + (lane >> 3), c = col + (lane >> 3);
            const int64_t at = u.batch * e.plane + r * e.ld + col + 4 * (lane & 7);
            to = e.out + at, from = LIN ? e.lin + at : nullptr;
            mirrored = e.out + u.batch * e.plane + c * e.ld + row + 4 * (lane & 7);
            rows = m - static_cast<int>(r), cols = m - static_cast<int>(c);
            mirror = u.m0 != u.n0;
        }
        __device__ __forceinline__ void fetch(const Symmetric& e, int j, Fetched& f) const {
            if constexpr (LIN) {
                const uint16_t* p = from + j;
#pragma unroll
                for (int i = 0; i < 8; ++i, p += 4 * e.ld) f.lin[i] = 4 * i < rows ? *reinterpret_cast<const uint2*>(p) : make_uint2(0, 0);
            }
        }
        __device__ __forceinline__ void square(const Symmetric& e, int j, int lane, uint32_t buf, float4 (&sums)[8], const Fetched& f, bool) const {
            uint16_t* p = to + j;
#pragma unroll
            for (int i = 0; i < 8; ++i, p += 4 * e.ld) {
                float4 v = make_float4(e.c * sums[i].x, e.c * sums[i].y, e.c * sums[i].z, e.c * sums[i].w);
                if constexpr (LIN) {
                    const float4 l = float4_of(f.lin[i]);
                    v.x += e.b * l.x, v.y += e.b * l.y, v.z += e.b * l.z, v.w += e.b * l.w;
                }
                if (4 * i < rows) *reinterpret_cast<uint2*>(p) = half4(v);
                if (mirror) square_set(buf, (lane >> 3) + 4 * i, lane & 7, make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)));
            }
            if (!mirror) return;
            __syncwarp();
            p = mirrored + static_cast<int64_t>(j) * e.ld;
#pragma unroll
            for (int i = 0; i < 8; ++i, p += 4 * e.ld) {
                const int c = (lane >> 3) + 4 * i, r = 4 * (lane & 7);
                const float4 v = make_float4(square_word(buf, r, c), square_word(buf, r + 1, c), square_word(buf, r + 2, c), square_word(buf, r + 3, c));
                if (j + 4 * i < cols) *reinterpret_cast<uint2*>(p) = half4(v);
            }
        }
    };
};

// X carried in fp32, scaled by a power of two: the next one is a X + sums.
struct Carried {
    float* x;
    int64_t plane;
    int ld;
    float a;
};

__device__ __forceinline__ float4 next_of(float a, float4 sums, float4 x) { return make_float4(a * x.x + sums.x, a * x.y + sums.y, a * x.z + sums.z, a * x.w + sums.w); }

struct Next {
    static constexpr bool kWhole = false, kSmall = true, kAlone = false, kPacks = false, kBefore = false, kAhead = true;
    static constexpr int kSmallBlocks = 2;
    struct Fetched {
        float4 x[8];
    };
    Carried x;
    uint16_t* out;  // the next operand

    struct Tile {
        float* x;
        uint16_t* out;
        int rows;

        __device__ __forceinline__ Tile(const Next& e, const ProdUnit& u, int m, int row, int col, int lane) {
            const int64_t r = row + (lane >> 3), at = u.batch * e.x.plane + r * e.x.ld + col + 4 * (lane & 7);
            x = e.x.x + at, out = e.out + at;
            rows = m - static_cast<int>(r);
        }
        __device__ __forceinline__ void fetch(const Next& e, int j, Fetched& f) const {
            const float* p = x + j;
#pragma unroll
            for (int i = 0; i < 8; ++i, p += 4 * e.x.ld) f.x[i] = 4 * i < rows ? *reinterpret_cast<const float4*>(p) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
        __device__ __forceinline__ void square(const Next& e, int j, int lane, uint32_t buf, float4 (&sums)[8], const Fetched& f, bool) const {
            float* p = x + j;
            uint16_t* q = out + j;
#pragma unroll
            for (int i = 0; i < 8; ++i, p += 4 * e.x.ld, q += 4 * e.x.ld) {
                const float4 v = next_of(e.x.a, sums[i], f.x[i]);
                if (4 * i >= rows) continue;
                *reinterpret_cast<float4*>(p) = v;  // nothing but this place of this tile reads it
                *reinterpret_cast<uint2*>(q) = half4(v);
            }
        }
    };
};

enum { kToF32, kToBf16, kToParam };

// The last step's result, to the caller: O, or the parameter moved by it.
template <int TO>
struct Result {
    static constexpr bool kWhole = false, kSmall = true, kAlone = false, kPacks = false, kBefore = false, kAhead = TO != kToParam;
    static constexpr int kSmallBlocks = TO == kToParam ? 1 : 2;
    struct Fetched {
        float4 x[8], p[TO == kToParam ? 8 : 1];
    };
    Carried x;
    float unscale;  // of the power of two
    int64_t stride;
    int cols;       // of out
    int vectors;    // every row of every matrix starts on 16 bytes
    float lr, scale, decay;
    Table out, param;

    __device__ __forceinline__ float moved(float p, float o) const { return p - lr * (scale * o + decay * p); }

    struct Tile {
        const float* x;
        char* to;
        const float* from;
        int rows, cols;  // that exist from this lane's first ones on

        __device__ __forceinline__ Tile(const Result& e, const ProdUnit& u, int m, int row, int col, int lane) {
            const int64_t r = row + (lane >> 3), c = col + 4 * (lane & 7), at = u.batch * e.x.plane + r * e.x.ld + c;
            x = e.x.x + at;
            to = static_cast<char*>(const_cast<void*>(e.out.p[u.batch])) + (r * e.stride + c) * (TO == kToBf16 ? 2 : 4);
            from = TO == kToParam ? static_cast<const float*>(e.param.p[u.batch]) + r * e.stride + c : nullptr;
            rows = m - static_cast<int>(r), cols = e.cols - static_cast<int>(c);
        }
        __device__ __forceinline__ void fetch(const Result& e, int j, Fetched& f) const {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f.x[i] = 4 * i < rows ? *reinterpret_cast<const float4*>(x + j + 4 * i * static_cast<int64_t>(e.x.ld)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if constexpr (TO == kToParam) {
                    if (e.vectors && 4 * i < rows && j + 4 <= cols) f.p[i] = *reinterpret_cast<const float4*>(from + j + 4 * i * e.stride);
                }
            }
        }
        __device__ __forceinline__ void square(const Result& e, int j, int lane, uint32_t buf, float4 (&sums)[8], const Fetched& f, bool) const {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float4 n = next_of(e.x.a, sums[i], f.x[i]);
                if (4 * i >= rows || j >= cols) continue;
                float4 o = make_float4(n.x * e.unscale, n.y * e.unscale, n.z * e.unscale, n.w * e.unscale);
                char* const p = to + (j + 4 * i * e.stride) * (TO == kToBf16 ? 2 : 4);
                if (e.vectors && j + 4 <= cols) {
                    if constexpr (TO == kToParam) o = make_float4(e.moved(f.p[i].x, o.x), e.moved(f.p[i].y, o.y), e.moved(f.p[i].z, o.z), e.moved(f.p[i].w, o.w));
                    if constexpr (TO == kToBf16) *reinterpret_cast<uint2*>(p) = make_uint2(bf16_pair(o.x, o.y), bf16_pair(o.z, o.w));
                    else *reinterpret_cast<float4*>(p) = o;
                } else {
                    const float v[4] = {o.x, o.y, o.z, o.w};
                    const float* const q = from + j + 4 * i * e.stride;
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        if (j + d >= cols) break;
                        if constexpr (TO == kToBf16) Elem<uint16_t>::store(reinterpret_cast<uint16_t*>(p) + d, v[d]);
                        else if constexpr (TO == kToParam) reinterpret_cast<float*>(p)[d] = e.moved(q[d], v[d]);
                        else reinterpret_cast<float*>(p)[d] = v[d];
                    }
                }
            }
        }
    };
};

// ---- the start: momentum, norm, first operand ------------------------------------------------------

struct Start {
    Table in, momentum, momentum_out;  // momentum: unused without update
    int64_t in_stride, momentum_stride, plane, rows;
    int cols, ld, update, nesterov, vectors, blocks, row_threads;
    float beta, rest;  // rest = 1 - beta
    double scale;      // the power of two
    double* partial;   // [count][blocks]
    float* x;
    uint16_t* operand;
};

// Eight neighbouring columns; those that do not exist are 0.
struct Eight {
    float v[8];
};

template <typename T>
__device__ __forceinline__ Eight load_eight(const T* p, int n, bool vectors) {
    Eight e;
    if (vectors && n >= 8) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
            e = Eight{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
        } else {
            const uint4 r = *reinterpret_cast<const uint4*>(p);
            const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) e.v[2 * j] = __uint_as_float(w[j] << 16), e.v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) e.v[j] = j < n ? Elem<T>::load(p + j) : 0.0f;
    }
    return e;
}

__device__ __forceinline__ Eight mix(const Eight& g, const Eight& v, float rest, float beta) {
    Eight u;
#pragma unroll
    for (int j = 0; j < 8; ++j) u.v[j] = rest * g.v[j] + beta * v.v[j];
    return u;
}

// Sum over the block, the same in every thread; the order is fixed.
__device__ __forceinline__ double block_sum(double s) {
    __shared__ double part[8];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    s = part[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) s += part[i];
    return s;
}

// Eight columns of a row at a time, over all of the matrix. A row is taken by row_threads (a power of two) neighbouring threads: no
// divisions. (Four columns at a running index, divided for its row, and everything in fp64: 150 instructions for four elements, and 24
// + 25 us for 4096 x 4096 bf16.)
template <typename F>
__device__ __forceinline__ void over_eights(const Start& a, F f) {
    const int tc = threadIdx.x & (a.row_threads - 1), tr = threadIdx.x / a.row_threads, rows = 256 / a.row_threads;
    for (int64_t r = static_cast<int64_t>(blockIdx.x) * rows + tr; r < a.rows; r += static_cast<int64_t>(gridDim.x) * rows)
        for (int c = tc * 8; c < a.cols; c += a.row_threads * 8) f(r, c, a.cols - c);
}

// The momentum's update, and partial sums of u's squares. A thread's squares are summed in fp32, threads in fp64. A block whose
// squares leave fp32's range, or come near its lower end, forms them in fp64 again.
template <typename T>
__global__ void __launch_bounds__(256) ortho_norm_kernel(const __grid_constant__ Start a) {
    next_may_begin();
    const T* const in = static_cast<const T*>(a.in.p[blockIdx.y]);
    const float* const mom = static_cast<const float*>(a.momentum.p[blockIdx.y]);
    float* const mom_out = static_cast<float*>(const_cast<void*>(a.momentum_out.p[blockIdx.y]));
    float squares = 0.0f;
    over_eights(a, [&](int64_t r, int c, int n) {
        Eight u = load_eight(in + r * a.in_stride + c, n, a.vectors);
        if (a.update) {
            const int64_t k = r * a.momentum_stride + c;
            const Eight g = u, v = mix(g, load_eight(mom + k, n, a.vectors), a.rest, a.beta);
            if (a.vectors && n >= 8) {
                reinterpret_cast<float4*>(mom_out + k)[0] = make_float4(v.v[0], v.v[1], v.v[2], v.v[3]);
                reinterpret_cast<float4*>(mom_out + k)[1] = make_float4(v.v[4], v.v[5], v.v[6], v.v[7]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < n) mom_out[k + j] = v.v[j];
            }
            u = a.nesterov ? mix(g, v, a.rest, a.beta) : v;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) squares += u.v[j] * u.v[j];
    });
    double sum = block_sum(squares);
    if (!(sum > 1e-20 && sum < INFINITY)) {
        double again = 0.0;
        over_eights(a, [&](int64_t r, int c, int n) {
            Eight u;
            if (a.update) {
                u = load_eight(mom_out + r * a.momentum_stride + c, n, a.vectors);
                if (a.nesterov) u = mix(load_eight(in + r * a.in_stride + c, n, a.vectors), u, a.rest, a.beta);
            } else {
                u = load_eight(in + r * a.in_stride + c, n, a.vectors);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) again += static_cast<double>(u.v[j]) * u.v[j];
        });
        sum = block_sum(again);
    }
    if (threadIdx.x == 0) a.partial[static_cast<int64_t>(blockIdx.y) * a.blocks + blockIdx.x] = sum;
}

// X_0 = u / |u|, scaled, and the operand made of it.
template <typename T>
__global__ void __launch_bounds__(256) ortho_start_kernel(const __grid_constant__ Start a) {
    next_may_begin();
    after_previous();
    double sum = 0.0;
    for (int i = threadIdx.x; i < a.blocks; i += 256) sum += a.partial[static_cast<int64_t>(blockIdx.y) * a.blocks + i];
    sum = block_sum(sum);
    // nothing but zeros stays that; an infinity or a NaN anywhere is NaN everywhere
    const double factor = sum == 0.0 ? 0.0 : (sum < INFINITY ? a.scale / sqrt(sum) : NAN);
    const float factor32 = static_cast<float>(factor);
    const bool wide = !(factor32 > 1e-30f && factor32 < 1e30f);  // a factor, or what it is applied to, outside fp32's safe range
    const T* const in = static_cast<const T*>(a.in.p[blockIdx.y]);
    const float* const mom = static_cast<const float*>(a.momentum_out.p[blockIdx.y]);
    over_eights(a, [&](int64_t r, int c, int n) {
        Eight u;
        if (a.update) {
            u = load_eight(mom + r * a.momentum_stride + c, n, a.vectors);
            if (a.nesterov) u = mix(load_eight(in + r * a.in_stride + c, n, a.vectors), u, a.rest, a.beta);
        } else {
            u = load_eight(in + r * a.in_stride + c, n, a.vectors);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) u.v[j] = wide ? static_cast<float>(u.v[j] * factor) : u.v[j] * factor32;
        const float4 p = make_float4(u.v[0], u.v[1], u.v[2], u.v[3]), q = make_float4(u.v[4], u.v[5], u.v[6], u.v[7]);
        const int64_t k = blockIdx.y * a.plane + r * a.ld + c;
        reinterpret_cast<float4*>(a.x + k)[0] = p, reinterpret_cast<float4*>(a.x + k)[1] = q;
        const uint2 lo = half4(p), hi = half4(q);
        *reinterpret_cast<uint4*>(a.operand + k) = make_uint4(lo.x, lo.y, hi.x, hi.y);
    });
}

// ---- matrices with a side of at most 128: all steps in one launch -----------------------------------
// A cluster of up to sixteen blocks (eight, where the device has no place for more) holds a matrix on chip: each has 256 of the longer side's indices l, as fp32 in registers (a
// thread has 128 neighbouring elements of a row, in memory's order: rows are the shorter side's indices i, or l where the matrix is tall)
// and as fp16 operand in shared memory. A step is three products within the block; between them S is summed over the cluster, each
// block a share of its rows, which it hands to all. A step takes one block 3 us (0.45 to write the operand, 0.5, 0.45 and 0.45 for the
// products from start to end, 0.3, 0.45 and 0.7 to bring their sums out), eight 7; in a row of calls 128 x 128 takes 25 us, 128 x 2048 49, 128 x 4096 54, as 15
// products of their own 98, 140 and 145. Loading, the norm and storing take 6.
constexpr int kHeldSide = 128, kHeldLong = 256, kHeldThreads = 256, kMostHeldBlocks = 16, kPortableBlocks = 8;
constexpr uint32_t kHeldX = kHeldSide * kHeldLong * 2, kHeldS = kHeldSide * kHeldSide * 2, kHeldPart = kHeldSide * kHeldSide * 4;
// X; S; Q, whose place the others' shares of S take before it is formed, and 32 KB more of those; this block's part of S
constexpr size_t kHeldSmem = 1024 + kHeldX + 3 * kHeldS + kHeldPart;
static_assert(kHeldPart == 2 * kHeldS, "the others' shares are as many bytes as a part");

struct Held {
    Start start;        // in, momentum, momentum_out, strides, rows, cols, update, nesterov, beta, rest, scale
    Table out, param;
    int64_t out_stride;
    int in_vectors, out_vectors, to, steps;
    float unscale, lr, scale, decay;
    float coefficients[3 * SS_ORTHO_MAX_STEPS];
};

// Four neighbouring columns of a row.
__device__ __forceinline__ float4 load_whole(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load_whole(const uint16_t* p) {
    const uint2 r = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xFFFF0000u), __uint_as_float(r.y << 16), __uint_as_float(r.y & 0xFFFF0000u));
}
template <typename T>
__device__ __forceinline__ float4 load_four(const T* p, int n, bool vectors) {
    if (vectors && n >= 4) return load_whole(p);
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = j < n ? Elem<T>::load(p + j) : 0.0f;
    return make_float4(v[0], v[1], v[2], v[3]);
}
template <typename T>
__device__ __forceinline__ void store_four(T* p, float4 v, int n, bool vectors) {
    if (vectors && n >= 4) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p) = v;
        else *reinterpret_cast<uint2*>(p) = make_uint2(bf16_pair(v.x, v.y), bf16_pair(v.z, v.w));
    } else {
        const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) Elem<T>::store(p + j, e[j]);
    }
}
__device__ __forceinline__ float4 mix(float4 g, float4 v, float rest, float beta) {
    return make_float4(rest * g.x + beta * v.x, rest * g.y + beta * v.y, rest * g.z + beta * v.z, rest * g.w + beta * v.w);
}

__device__ __forceinline__ float4 shared_load4(uint32_t at) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}
// Chunk c (16 bytes) of row r of a square of 32 rows of 512 bytes.
__device__ __forceinline__ void turn_put(uint32_t at, int r, int c, float4 v) {
    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at + r * 512 + ((c ^ (r & 7)) << 4)), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ float4 turn_get(uint32_t at, int r, int c) { return shared_load4(at + r * 512 + ((c ^ (r & 7)) << 4)); }

// Row r of an operand of 64 elements (128 bytes, swizzled) a row: its 16-byte chunk c.
__device__ __forceinline__ uint32_t held_chunk(uint32_t panel, int r, int c) { return panel + r * 128 + ((c ^ (r & 7)) << 4); }

template <typename T, bool TALL>
__global__ void __launch_bounds__(kHeldThreads, 1) ortho_held_kernel(const __grid_constant__ Held a) {
    extern __shared__ uint8_t dynamic[];
    __shared__ uint64_t bar, came, handed;
    __shared__ uint32_t tmem_address;
    __shared__ int gave_up[2];
    __shared__ double norm_part;
    const uint32_t xs = (smem_addr(dynamic) + 1023u) & ~1023u, ss_ = xs + kHeldX, qs = ss_ + kHeldS, ps = qs + 2 * kHeldS;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, quarter = warp & 3, half = warp >> 2;
    uint32_t rank, blocks;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks));
    const int matrix = blockIdx.x / blocks;

    if (tid == 0) {
        mbar_init(smem_addr(&bar), 1);
        mbar_init(smem_addr(&came), 1);
        mbar_init(smem_addr(&handed), 1);
        gave_up[0] = gave_up[1] = 0;
        mbar_init_visible();
    }
    if (warp == 0) tmem_alloc(smem_addr(&tmem_address), 512);

    // This thread's elements: one row of the matrix, 128 columns from `col` on. A warp has 32 rows from `row0` on; they come and
    // go a row at a time, four columns to a lane, and are turned in shared memory. (A row a lane in global memory takes a cycle for each of a load's 32
    // lines: 6 us for 128 x 128 instead of 2.)
    const int i_or_l = quarter * 32 + lane;
    const int64_t row0 = TALL ? static_cast<int64_t>(rank) * kHeldLong + half * 128 + quarter * 32 : quarter * 32;
    const int64_t col = TALL ? 0 : static_cast<int64_t>(rank) * kHeldLong + half * 128;
    const int rows = static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(32), a.start.rows - row0)));
    const int cols = static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(128), a.start.cols - col)));
    const uint32_t turn = (warp < 4 ? xs + warp * 16384 : ps + (warp - 4) * 16384);  // 32 rows of 512 bytes
    float x[128];
    double sum = 0.0;
    {
        const Start& st = a.start;
        const T* const in = static_cast<const T*>(st.in.p[matrix]) + row0 * st.in_stride + col;
        const float* const mom = static_cast<const float*>(st.momentum.p[matrix]) + row0 * st.momentum_stride + col;
        float* const mom_out = static_cast<float*>(const_cast<void*>(st.momentum_out.p[matrix])) + row0 * st.momentum_stride + col;
        const int n = cols - 4 * lane;
        const bool whole = a.in_vectors && n >= 4;  // of this lane
        auto take = [&](int r, float4 g, float4 v) {
            float4 u = g;
            if (st.update) {
                u = mix(g, v, st.rest, st.beta);
                if (r < rows) store_four(mom_out + r * st.momentum_stride + 4 * lane, u, n, a.in_vectors);
                if (st.nesterov) u = mix(g, u, st.rest, st.beta);
            }
            turn_put(turn, r, lane, u);
        };
        if (__all_sync(0xFFFFFFFFu, whole || n <= 0)) {
#pragma unroll 1
            for (int r0 = 0; r0 < 32; r0 += 8) {
                float4 g[8], v[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    g[r] = v[r] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    if (r0 + r >= rows || n <= 0) continue;
                    g[r] = load_whole(in + (r0 + r) * st.in_stride + 4 * lane);
                    if (st.update) v[r] = load_whole(mom + (r0 + r) * st.momentum_stride + 4 * lane);
                }
#pragma unroll
                for (int r = 0; r < 8; ++r) take(r0 + r, g[r], v[r]);
            }
        } else {
#pragma unroll 2
            for (int r = 0; r < 32; ++r) {
                const int m = r < rows ? n : 0;
                take(r, load_four(in + r * st.in_stride + 4 * lane, m, a.in_vectors),
                     st.update ? load_four(mom + r * st.momentum_stride + 4 * lane, m, a.in_vectors) : make_float4(0.0f, 0.0f, 0.0f, 0.0f));
            }
        }
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 32; ++c) {
            const float4 u = turn_get(turn, lane, c);
            x[4 * c] = u.x, x[4 * c + 1] = u.y, x[4 * c + 2] = u.z, x[4 * c + 3] = u.w;
        }
    }
    {   // fp32 holds the squares' sum unless it leaves the range: then again in fp64
        float squares = 0.0f;
#pragma unroll
        for (int j = 0; j < 128; ++j) squares += x[j] * x[j];
        sum = block_sum(squares);
        if (!(sum > 1e-20 && sum < INFINITY)) {
            double again = 0.0;
#pragma unroll
            for (int j = 0; j < 128; ++j) again += static_cast<double>(x[j]) * x[j];
            sum = block_sum(again);
        }
    }
    if (tid == 0) norm_part = sum;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (blocks > 1) {
        cluster_sync();
        sum = 0.0;
        for (uint32_t q = 0; q < blocks; ++q) sum += cluster_load_double(cluster_addr(smem_addr(&norm_part), q));
    }
    const double factor = sum == 0.0 ? 0.0 : (sum < INFINITY ? a.start.scale / sqrt(sum) : NAN);
    const float factor32 = static_cast<float>(factor);
    if (factor32 > 1e-30f && factor32 < 1e30f) {
#pragma unroll
        for (int j = 0; j < 128; ++j) x[j] *= factor32;
    } else {
#pragma unroll
        for (int j = 0; j < 128; ++j) x[j] = static_cast<float>(x[j] * factor);
    }

    const uint32_t tmem = tmem_address, lanes = static_cast<uint32_t>(quarter * 32) << 16;
    const float inverse = a.unscale * a.unscale;
    uint32_t parity = 0;
    // Each wait is bounded. A warp whose wait ran out writes NaN from there on, into the operands too, which take it to all others. The first
    // warp, which issues products and copies, gives up only after a whole wait of its own, never because others did, and issues nothing more: so
    // nothing of this block's is under way, nor anything that others sent it, when it has gone through the rest.
    bool ok = true;
    auto wait = [&](uint64_t* barrier, uint32_t phase) {
        ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_addr(barrier), phase, &gave_up[warp == 0])) && ok;
        if (!ok) gave_up[0] = 1;
    };
    auto unless_late = [&](float v) { return ok ? v : __uint_as_float(kNanBits); };
    // one warp issues, all wait for the products to have ended
    auto products = [&](auto issue) {
        smem_to_async();
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        if (warp == 0 && ok) {
            if (elect_one()) {
                issue();
                tc_commit(smem_addr(&bar));
            }
            __syncwarp();
        }
        wait(&bar, parity);
        parity ^= 1;
        tc_fence_after();
    };
    constexpr uint32_t kIdescCols = tc_idesc(128, 128, false, false, false);
    // of this block's 256 long indices, those that the matrix has, in sixteens (one at least: S is written by it)
    const int64_t longest = (TALL ? a.start.rows : static_cast<int64_t>(a.start.cols)) - static_cast<int64_t>(rank) * kHeldLong;
    const int long_steps = static_cast<int>(max(static_cast<int64_t>(1), min(static_cast<int64_t>(kHeldLong / 16), (longest + 15) / 16)));

    if (blocks > 1) cluster_arrive();
    for (int step = 0; step < a.steps; ++step) {
        // ---- the operand: rows of 64 elements in panels, wide: [l / 64][i][l % 64], tall: [i / 64][l][i % 64]
        {
            const int r = TALL ? half * 128 + i_or_l : i_or_l;
            const uint32_t panel = TALL ? kHeldLong * 128 : kHeldSide * 128, first = xs + (TALL ? 0 : half * 2 * panel);
#pragma unroll
            for (int c = 0; c < 16; ++c) {
                const uint2 lo = half4(make_float4(x[8 * c], x[8 * c + 1], x[8 * c + 2], x[8 * c + 3])), hi = half4(make_float4(x[8 * c + 4], x[8 * c + 5], x[8 * c + 6], x[8 * c + 7]));
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(held_chunk(first + (c >> 3) * panel, r, c & 7)), "r"(lo.x), "r"(lo.y), "r"(hi.x), "r"(hi.y) : "memory");
            }
        }
        // ---- S of this block's part
        products([&] {
            constexpr uint32_t idesc = tc_idesc(128, 128, false, TALL, TALL);
#pragma unroll 1
            for (int k = 0; k < long_steps; ++k) {
                const uint64_t d = TALL ? tc_desc_rows(xs + k * 2048, kHeldLong * 128) : tc_desc_cols(xs + (k >> 2) * kHeldSide * 128 + (k & 3) * 32);
                tc_mma_f16(tmem, d, d, idesc, k != 0);
            }
        });
        // ---- S as an operand: rows of 128, in two panels of 64. This thread: row i_or_l, columns 64 half on
        if (blocks == 1) {
            const float by = unless_late(inverse);
#pragma unroll
            for (int c = 0; c < 8; c += 2) {
                uint32_t r[16];
                tmem_load16(tmem + lanes + half * 64 + c * 8, r);
                tmem_load_wait();
                uint2 w[4];
#pragma unroll
                for (int d = 0; d < 4; ++d)
                    w[d] = half4(make_float4(by * __uint_as_float(r[4 * d]), by * __uint_as_float(r[4 * d + 1]), by * __uint_as_float(r[4 * d + 2]), by * __uint_as_float(r[4 * d + 3])));
#pragma unroll
                for (int d = 0; d < 2; ++d)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(held_chunk(ss_ + half * kHeldSide * 128, i_or_l, c + d)), "r"(w[2 * d].x), "r"(w[2 * d].y), "r"(w[2 * d + 1].x), "r"(w[2 * d + 1].y) : "memory");
            }
        } else {
            // Each block gets its share of S's rows from all, adds them up and hands the sum to all, by copies between the blocks' memories.
            // (Rows of 512 bytes, chunks swizzled by the row. Loads from the others instead of copies took 7 us a step with eight blocks, stores to
            // them 5.6.) The others have used what the copies overwrite: they arrived after their last product with it.
            cluster_wait();
#pragma unroll
            for (int c = 0; c < 16; c += 4) {
                uint32_t w[16];
                tmem_load16(tmem + lanes + half * 64 + c * 4, w);
                tmem_load_wait();
                if (!ok) {
#pragma unroll
                    for (int d = 0; d < 16; ++d) w[d] = kNanBits;
                }
#pragma unroll
                for (int d = 0; d < 4; ++d)
                    turn_put(ps, i_or_l, half * 16 + c + d, make_float4(__uint_as_float(w[4 * d]), __uint_as_float(w[4 * d + 1]), __uint_as_float(w[4 * d + 2]), __uint_as_float(w[4 * d + 3])));
            }
            const uint32_t share = kHeldSide / blocks;  // rows; a multiple of 8
            smem_to_async();
            __syncthreads();
            if (tid == 0 && ok) {
                mbar_expect(smem_addr(&came), (blocks - 1) * share * 512);
                for (uint32_t d = 1; d < blocks; ++d) {
                    const uint32_t q = (rank + d) % blocks;
                    bulk_to_cluster(cluster_addr(qs + rank * share * 512, q), ps + q * share * 512, share * 512, cluster_addr(smem_addr(&came), q));
                }
            }
            wait(&came, step & 1);
            const float by = unless_late(inverse);
            for (uint32_t e = tid; e < share * 16; e += kHeldThreads) {  // eight columns to a thread
                const uint32_t r = e >> 4, c = e & 15;
                float v[8];
#pragma unroll
                for (int d = 0; d < 8; ++d) v[d] = 0.0f;
#pragma unroll 2
                for (uint32_t q = 0; q < blocks; ++q) {  // in the order of the ranks
                    const uint32_t at = (q == rank ? ps : qs) + q * share * 512;
                    const float4 y = turn_get(at, r, 2 * c), z = turn_get(at, r, 2 * c + 1);
                    v[0] += y.x, v[1] += y.y, v[2] += y.z, v[3] += y.w, v[4] += z.x, v[5] += z.y, v[6] += z.z, v[7] += z.w;
                }
                const uint2 lo = half4(make_float4(by * v[0], by * v[1], by * v[2], by * v[3])), hi = half4(make_float4(by * v[4], by * v[5], by * v[6], by * v[7]));
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(held_chunk(ss_ + (c >> 3) * kHeldSide * 128, rank * share + r, c & 7)), "r"(lo.x), "r"(lo.y), "r"(hi.x), "r"(hi.y) : "memory");
            }
            smem_to_async();
            __syncthreads();
            if (tid == 0 && ok) {
                mbar_expect(smem_addr(&handed), (blocks - 1) * share * 256);
                for (uint32_t d = 1; d < blocks; ++d) {
                    const uint32_t q = (rank + d) % blocks;
                    for (uint32_t panel = 0; panel < 2; ++panel) {
                        const uint32_t at = ss_ + panel * kHeldSide * 128 + rank * share * 128;
                        bulk_to_cluster(cluster_addr(at, q), at, share * 128, cluster_addr(smem_addr(&handed), q));
                    }
                }
            }
            wait(&handed, step & 1);
        }
        // ---- Q = b S + c S S
        products([&] {
#pragma unroll
            for (int k = 0; k < kHeldSide / 16; ++k) {
                const uint64_t d = tc_desc_cols(ss_ + (k >> 2) * kHeldSide * 128 + (k & 3) * 32);
                tc_mma_f16(tmem, d, d, kIdescCols, k != 0);
            }
        });
        const float cb = unless_late(a.coefficients[3 * step + 1]), cc = a.coefficients[3 * step + 2];
#pragma unroll
        for (int c = 0; c < 8; c += 2) {
            uint32_t r[16];
            tmem_load16(tmem + lanes + half * 64 + c * 8, r);
            tmem_load_wait();
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                uint4 s;
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(s.x), "=r"(s.y), "=r"(s.z), "=r"(s.w) : "r"(held_chunk(ss_ + half * kHeldSide * 128, i_or_l, c + d)) : "memory");
                const float4 y = float4_of(make_uint2(s.x, s.y)), z = float4_of(make_uint2(s.z, s.w));
                const uint32_t* const p = r + 8 * d;
                const uint2 lo = half4(make_float4(cb * y.x + cc * __uint_as_float(p[0]), cb * y.y + cc * __uint_as_float(p[1]), cb * y.z + cc * __uint_as_float(p[2]), cb * y.w + cc * __uint_as_float(p[3])));
                const uint2 hi = half4(make_float4(cb * z.x + cc * __uint_as_float(p[4]), cb * z.y + cc * __uint_as_float(p[5]), cb * z.z + cc * __uint_as_float(p[6]), cb * z.w + cc * __uint_as_float(p[7])));
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(held_chunk(qs + half * kHeldSide * 128, i_or_l, c + d)), "r"(lo.x), "r"(lo.y), "r"(hi.x), "r"(hi.y) : "memory");
            }
        }
        // ---- X = a X + Q X
        products([&] {
            if constexpr (TALL) {  // X Q, 128 rows of X at a time
#pragma unroll 1
                for (int h = 0; h < kHeldLong / 128; ++h)
#pragma unroll 1
                    for (int k = 0; k < kHeldSide / 16; ++k)
                        tc_mma_f16(tmem + 128 + h * 128, tc_desc_cols(xs + (k >> 2) * kHeldLong * 128 + h * 128 * 128 + (k & 3) * 32),
                                   tc_desc_cols(qs + (k >> 2) * kHeldSide * 128 + (k & 3) * 32), kIdescCols, k != 0);
            } else {
                constexpr uint32_t idesc = tc_idesc(128, kHeldLong, false, false, true);
#pragma unroll 1
                for (int k = 0; k < kHeldSide / 16; ++k)
                    tc_mma_f16(tmem + 128, tc_desc_cols(qs + (k >> 2) * kHeldSide * 128 + (k & 3) * 32), tc_desc_rows(xs + k * 2048, kHeldSide * 128), idesc, k != 0);
            }
        });
        if (blocks > 1 && step + 1 < a.steps) cluster_arrive();
        const float ca = unless_late(a.coefficients[3 * step]);
#pragma unroll
        for (int j = 0; j < 128; j += 16) {
            uint32_t r[16];
            tmem_load16(tmem + lanes + 128 + half * 128 + j, r);
            tmem_load_wait();
#pragma unroll
            for (int d = 0; d < 16; ++d) x[j + d] = ca * x[j + d] + __uint_as_float(r[d]);
        }
    }
    // ---- out
    {
#pragma unroll
        for (int c = 0; c < 32; ++c) turn_put(turn, lane, c, make_float4(x[4 * c] * a.unscale, x[4 * c + 1] * a.unscale, x[4 * c + 2] * a.unscale, x[4 * c + 3] * a.unscale));
        __syncwarp();
        const int64_t at = row0 * a.out_stride + col + 4 * lane;
        float* const to32 = static_cast<float*>(const_cast<void*>(a.out.p[matrix])) + at;
        uint16_t* const to16 = static_cast<uint16_t*>(const_cast<void*>(a.out.p[matrix])) + at;
        const float* const from = static_cast<const float*>(a.param.p[matrix]) + at;
        const int n = cols - 4 * lane;
        if (a.to == kToBf16) {
#pragma unroll 4
            for (int r = 0; r < rows; ++r) store_four(to16 + r * a.out_stride, turn_get(turn, r, lane), n, a.out_vectors);
        } else if (a.to == kToF32) {
#pragma unroll 4
            for (int r = 0; r < rows; ++r) store_four(to32 + r * a.out_stride, turn_get(turn, r, lane), n, a.out_vectors);
        } else {
#pragma unroll 1
            for (int r0 = 0; r0 < rows; r0 += 8) {
                float4 p[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) p[r] = load_four(from + (r0 + r) * a.out_stride, r0 + r < rows ? n : 0, a.out_vectors);
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    if (r0 + r >= rows) continue;
                    const float4 o = turn_get(turn, r0 + r, lane);
                    store_four(to32 + (r0 + r) * a.out_stride,
                               make_float4(p[r].x - a.lr * (a.scale * o.x + a.decay * p[r].x), p[r].y - a.lr * (a.scale * o.y + a.decay * p[r].y),
                                           p[r].z - a.lr * (a.scale * o.z + a.decay * p[r].z), p[r].w - a.lr * (a.scale * o.w + a.decay * p[r].w)), n, a.out_vectors);
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (blocks > 1) cluster_sync();  // the others may still be reading this block's memory
    tc_fence_after();
    if (warp == 0) tmem_free(tmem, 512);
}

// ---- host side -------------------------------------------------------------------------------------

constexpr int64_t kMostSide = int64_t(1) << 20, kMostTiles = int64_t(1) << 24;
// Blocks of the first pass over all matrices, four to an SM, and of the second over each: more of them, shorter, write faster (12 of
// 4096 x 1024 110 -> 94 us).
constexpr int kMostBlocks = 592, kMostStartBlocks = 2400;

struct Layout {
    int64_t side, ld, side_ld;   // the smaller side; row strides of X and of S and Q
    int64_t plane, side_plane;   // elements of a matrix
    int blocks, row_threads;     // of the start, for each matrix; for each row
    int64_t x, operand[2], s, q, partial, bytes;  // places in the workspace
};

inline int64_t up_to(int64_t n, int64_t m) { return (n + m - 1) / m * m; }

bool sizes_ok(int count, int64_t rows, int64_t cols) { return count >= 0 && count <= kMostMatrices && sides_ok(rows, cols); }

int layout_of(int count, int64_t rows, int64_t cols, Layout* l) {
    if (rows > kMostSide || cols > kMostSide) return SS_ERR_UNSUPPORTED;
    if (((rows + 255) / 256) * ((cols + 255) / 256) * count > kMostTiles) return SS_ERR_UNSUPPORTED;
    l->side = rows < cols ? rows : cols;
    l->ld = up_to(cols, 64), l->side_ld = up_to(l->side, 64);
    l->plane = rows * l->ld, l->side_plane = l->side * l->side_ld;
    l->row_threads = 1;
    while (l->row_threads < 256 && l->row_threads * 8 < cols) l->row_threads *= 2;
    const int64_t want = (rows + 256 / l->row_threads - 1) / (256 / l->row_threads), most = kMostBlocks / count > 1 ? kMostBlocks / count : 1;
    l->blocks = static_cast<int>(want < most ? want : most);
    int64_t at = 0;
    auto place = [&](int64_t bytes) {
        const int64_t p = at;
        at += up_to(bytes, 256);
        return p;
    };
    l->x = place(count * l->plane * 4), l->operand[0] = place(count * l->plane * 2), l->operand[1] = place(count * l->plane * 2);
    l->s = place(count * l->side_plane * 2), l->q = place(count * l->side_plane * 2);
    l->partial = place(static_cast<int64_t>(count) * l->blocks * 8);
    l->bytes = at;
    return SS_OK;
}

struct Call {
    Start start;
    Result<kToF32> result;
    int to;
    ss_dtype in_dt;
    int count;
    int64_t rows, cols;
    const float* coefficients;
    int steps;
};

template <typename T, bool TALL>
cudaError_t held_config(cudaLaunchConfig_t* cfg, cudaLaunchAttribute* at, int matrices, int blocks, cudaStream_t st) {
    struct Key {};
    const void* const kernel = reinterpret_cast<const void*>(ortho_held_kernel<T, TALL>);
    cudaError_t e = allow_shared<Key>(kernel, static_cast<int>(kHeldSmem));
    if (e == cudaSuccess && blocks > kPortableBlocks) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    at->id = cudaLaunchAttributeClusterDimension;
    at->val.clusterDim.x = blocks, at->val.clusterDim.y = 1, at->val.clusterDim.z = 1;
    cfg->gridDim = dim3(static_cast<unsigned>(matrices * blocks)), cfg->blockDim = dim3(kHeldThreads);
    cfg->dynamicSmemBytes = kHeldSmem, cfg->stream = st, cfg->attrs = at, cfg->numAttrs = 1;
    return e;
}

template <typename T, bool TALL>
int launch_held(const Held& h, int matrices, int blocks, cudaStream_t st) {
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at{};
    cudaError_t e = held_config<T, TALL>(&cfg, &at, matrices, blocks, st);
    if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, ortho_held_kernel<T, TALL>, h);
    return cuda_status_public(e);
}

// Whether the current device has place for a cluster of that many blocks, asked once for each device.
bool fits_on_device(int blocks) {
    if (blocks <= kPortableBlocks) return true;
    static std::atomic<int> known[64];  // 0: not asked, 1: no, 2: yes
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device >= 64) return false;
    int answer = known[device].load(std::memory_order_relaxed);
    if (answer == 0) {
        cudaLaunchConfig_t cfg{};
        cudaLaunchAttribute at{};
        int clusters = 0;
        answer = held_config<float, false>(&cfg, &at, 1, blocks, nullptr) == cudaSuccess &&
                         cudaOccupancyMaxActiveClusters(&clusters, ortho_held_kernel<float, false>, &cfg) == cudaSuccess && clusters > 0 ? 2 : 1;
        if (answer == 1) cudaGetLastError();
        known[device].store(answer, std::memory_order_relaxed);
    }
    return answer == 2;
}

// Blocks that hold a matrix of these sides, or 0: it is held only up to kHeldSide by kMostHeldBlocks * kHeldLong.
int held_blocks(int64_t rows, int64_t cols) {
    const int64_t small = rows < cols ? rows : cols, big = rows < cols ? cols : rows;
    if (small > kHeldSide || big > kMostHeldBlocks * kHeldLong) return 0;
    int blocks = 1;
    while (blocks * kHeldLong < big) blocks *= 2;
    return fits_on_device(blocks) ? blocks : 0;
}

int run_held(const Call& c, int blocks, float scale, float unscale, cudaStream_t st) {
    Held h{};
    h.start = c.start;
    h.start.rows = c.rows, h.start.cols = static_cast<int>(c.cols), h.start.scale = scale;
    h.in_vectors = c.start.vectors, h.out_vectors = c.result.vectors, h.out = c.result.out, h.param = c.result.param;
    h.out_stride = c.result.stride, h.to = c.to, h.steps = c.steps;
    h.unscale = unscale, h.lr = c.result.lr, h.scale = c.result.scale, h.decay = c.result.decay;
    for (int i = 0; i < 3 * c.steps; ++i) h.coefficients[i] = c.coefficients[i];
    const bool tall = c.rows > c.cols;
    if (c.in_dt == SS_F32) return tall ? launch_held<float, true>(h, c.count, blocks, st) : launch_held<float, false>(h, c.count, blocks, st);
    return tall ? launch_held<uint16_t, true>(h, c.count, blocks, st) : launch_held<uint16_t, false>(h, c.count, blocks, st);
}

int run(Call& c, const Layout& l, uint8_t* ws, cudaStream_t st) {
    const int64_t big = c.rows > c.cols ? c.rows : c.cols;
    int power = 0;  // 2^power: about the root of the larger side, so that X ends with values about 1
    while ((int64_t(1) << (2 * (power + 1))) <= big) ++power;
    const float scale = std::ldexp(1.0f, power), unscale = std::ldexp(1.0f, -power);
    const int held = held_blocks(c.rows, c.cols);
    if (held > 0) return run_held(c, held, scale, unscale, st);
    float* const xs = reinterpret_cast<float*>(ws + l.x);
    uint16_t* operand[2] = {reinterpret_cast<uint16_t*>(ws + l.operand[0]), reinterpret_cast<uint16_t*>(ws + l.operand[1])};
    uint16_t *const s = reinterpret_cast<uint16_t*>(ws + l.s), *const q = reinterpret_cast<uint16_t*>(ws + l.q);
    Start& a = c.start;
    a.plane = l.plane, a.rows = c.rows, a.cols = static_cast<int>(c.cols), a.ld = static_cast<int>(l.ld), a.blocks = l.blocks, a.row_threads = l.row_threads;
    a.scale = scale, a.partial = reinterpret_cast<double*>(ws + l.partial), a.x = xs, a.operand = operand[0];
    const dim3 grid(static_cast<unsigned>(l.blocks), static_cast<unsigned>(c.count));
    cudaError_t e;
    if (c.in_dt == SS_F32) e = launch_next(false, ortho_norm_kernel<float>, grid, 256, st, a);
    else e = launch_next(false, ortho_norm_kernel<uint16_t>, grid, 256, st, a);
    if (e != cudaSuccess) return cuda_status_public(e);
    const int64_t want = (c.rows + 256 / l.row_threads - 1) / (256 / l.row_threads);
    const dim3 many(static_cast<unsigned>(want < kMostStartBlocks ? want : kMostStartBlocks), static_cast<unsigned>(c.count));
    if (c.in_dt == SS_F32) e = launch_next(true, ortho_start_kernel<float>, many, 256, st, a);
    else e = launch_next(true, ortho_start_kernel<uint16_t>, many, 256, st, a);
    if (e != cudaSuccess) return cuda_status_public(e);

    const bool tall = c.rows > c.cols;
    const int64_t row_bytes = l.ld * 2, plane_bytes = l.plane * 2, side_row = l.side_ld * 2, side_bytes = l.side_plane * 2;
    CUtensorMap x_sum[2], x_prod[2], s_map, q_map;  // X as an operand of S and of Q X
    int status = SS_OK;
    auto map = [&](CUtensorMap* m, const void* p, int64_t fast, int64_t slow, int64_t rb, int64_t pb, bool mn) {
        if (status == SS_OK) status = map_operand(m, p, false, fast, slow, rb, c.count, pb, mn);
    };
    for (int i = 0; i < 2; ++i) {
        map(&x_sum[i], operand[i], c.cols, c.rows, row_bytes, plane_bytes, tall);
        map(&x_prod[i], operand[i], c.cols, c.rows, row_bytes, plane_bytes, !tall);
    }
    map(&s_map, s, l.side, l.side, side_row, side_bytes, false);
    map(&q_map, q, l.side, l.side, side_row, side_bytes, false);
    if (status != SS_OK) return status;

    const int sms = device_sm_count(&e);
    if (e != cudaSuccess) return cuda_status_public(e);
    Product ps = product_of(l.side, l.side, big, false, sms), pq = product_of(l.side, l.side, l.side, false, sms);
    Product px = product_of(c.rows, c.cols, l.side, false, sms);
    for (Product* p : {&ps, &pq, &px}) p->batches = c.count, p->bf16 = 0, p->follows = 1, p->m_fast = 1;
    ps.upper = pq.upper = 1;
    for (Product* p : {&ps, &pq, &px}) choose_small(p, sms);
    for (int k = 0; k < c.steps; ++k) {
        const float *const co = c.coefficients + 3 * k;
        const int from = k & 1;
        const Symmetric<false> es{s, nullptr, l.side_plane, static_cast<int>(l.side_ld), 0.0f, unscale * unscale};
        const Symmetric<true> eq{q, s, l.side_plane, static_cast<int>(l.side_ld), co[1], co[2]};
        const Carried x{xs, l.plane, static_cast<int>(l.ld), co[0]};
        status = tall ? launch_product<Symmetric<false>, true, true>(x_sum[from], x_sum[from], ps, es, st)
                      : launch_product<Symmetric<false>, false, false>(x_sum[from], x_sum[from], ps, es, st);
        if (status == SS_OK) status = launch_product<Symmetric<true>, false, false>(s_map, s_map, pq, eq, st);
        if (status != SS_OK) return status;
        if (k + 1 < c.steps) {
            const Next en{x, operand[from ^ 1]};
            status = tall ? launch_product<Next, false, false>(x_prod[from], q_map, px, en, st)
                          : launch_product<Next, false, true>(q_map, x_prod[from], px, en, st);
        } else {
            auto last = [&](auto r) {
                using R = decltype(r);
                r.x = x, r.unscale = unscale, r.cols = static_cast<int>(c.cols);
                r.stride = c.result.stride, r.vectors = c.result.vectors, r.lr = c.result.lr, r.scale = c.result.scale, r.decay = c.result.decay;
                r.out = c.result.out, r.param = c.result.param;
                return tall ? launch_product<R, false, false>(x_prod[from], q_map, px, r, st) : launch_product<R, false, true>(q_map, x_prod[from], px, r, st);
            };
            status = c.to == kToParam ? last(Result<kToParam>{}) : (c.to == kToBf16 ? last(Result<kToBf16>{}) : last(Result<kToF32>{}));
        }
        if (status != SS_OK) return status;
    }
    return SS_OK;
}

// The matrices of an argument, checked; a NULL array or pointer is refused.
struct Mats {
    Mat m[kMostMatrices];
    int status;
    bool vectors;  // every row starts on 16 bytes

    Mats(const void* const* p, int count, int64_t rows, int64_t cols, int64_t stride, size_t eb) : status(SS_OK), vectors(true) {
        if (p == nullptr || !stride_ok(rows, cols, stride)) {
            status = SS_ERR_INVALID_ARG;
            return;
        }
        for (int i = 0; i < count; ++i) {
            if (p[i] == nullptr) status = SS_ERR_INVALID_ARG;
            m[i] = mat(p[i], rows, cols, stride, eb);
            if (status == SS_OK && !addr_aligned(p[i], eb)) status = SS_ERR_MISALIGNED;
            vectors = vectors && m[i].row_aligned(16);
        }
    }
};

// Whether matrix i of `out` shares an element with any of `in`, but for in[i] in place where that is allowed.
bool overlaps(const Mats& out, const Mats& in, int count, bool in_place) {
    for (int i = 0; i < count; ++i)
        for (int j = 0; j < count; ++j)
            if (mats_overlap(out.m[i], in.m[j]) && !(in_place && i == j && same_mat(out.m[i], in.m[j]))) return true;
    return false;
}

bool overlaps_itself(const Mats& out, int count) {
    for (int i = 0; i < count; ++i)
        for (int j = 0; j < i; ++j)
            if (mats_overlap(out.m[i], out.m[j])) return true;
    return false;
}

bool overlaps_scratch(const Mats& a, int count, const void* p, size_t n) {
    for (int i = 0; i < count; ++i)
        if (mat_overlaps(a.m[i], p, n)) return true;
    return false;
}

// What the operands' range (fp16) asks of the coefficients, whatever the matrix. X_0 has singular values up to 1; `most` bounds those of each step's X, and
// so its elements, times 2^10 at the most (the power of two of the longest side): below 2^15 with singular values up to 32. Q's elements are below its
// largest singular value. And the linear term, which alone is not rounded, carries the small singular values: where it is nearly nothing beside the others, S, of their
// squares, falls below the range (two steps of (0, 1, 0) on 1000 x 2048 give nothing at all). With |a| a 64th of the others the model of the roundings is off
// by 2e-4 at most.
constexpr double kMostSingular = 32.0, kMostQ = 32768.0, kMostResult = 1e30, kLeastLinear = 1.0 / 64;

// Largest |f| on [0, end], f's extrema among `at`.
template <typename F>
double largest(F f, double end, const double* at, int n) {
    double m = std::fabs(f(end));
    for (int i = 0; i < n; ++i)
        if (at[i] > 0.0 && at[i] < end) m = std::fmax(m, std::fabs(f(at[i])));
    return m;
}

int check_coefficients(const float* co, int steps) {
    if (steps < 1 || steps > SS_ORTHO_MAX_STEPS || co == nullptr) return SS_ERR_INVALID_ARG;
    for (int i = 0; i < 3 * steps; ++i)
        if (!std::isfinite(co[i])) return SS_ERR_INVALID_ARG;
    double most = 1.0;
    for (int k = 0; k < steps; ++k) {
        const double a = co[3 * k], b = co[3 * k + 1], c = co[3 * k + 2];
        if (most > kMostSingular || std::fabs(a) < kLeastLinear * (std::fabs(b) + std::fabs(c))) return SS_ERR_UNSUPPORTED;
        const double q_at[1] = {c != 0.0 ? -b / (2.0 * c) : 0.0};
        if (largest([&](double t) { return b * t + c * t * t; }, most * most, q_at, 1) > kMostQ) return SS_ERR_UNSUPPORTED;
        double f_at[2] = {0.0, 0.0};  // squares: a + 3 b t + 5 c t^2 = 0
        const double root = 9.0 * b * b - 20.0 * a * c;
        if (c == 0.0) f_at[0] = b != 0.0 ? -a / (3.0 * b) : 0.0;
        else if (root >= 0.0) f_at[0] = (-3.0 * b + std::sqrt(root)) / (10.0 * c), f_at[1] = (-3.0 * b - std::sqrt(root)) / (10.0 * c);
        most = largest([&](double t) { return std::sqrt(t) * (a + b * t + c * t * t); }, most * most, f_at, 2);
    }
    return most > kMostResult ? SS_ERR_UNSUPPORTED : SS_OK;
}

int check_workspace(const Layout& l, const void* workspace, int64_t bytes) {
    if (workspace == nullptr || bytes < l.bytes) return SS_ERR_INVALID_ARG;
    return addr_aligned(workspace, 256) ? SS_OK : SS_ERR_MISALIGNED;
}

void fill(Table* t, const Mats& m, int count) {
    for (int i = 0; i < count; ++i) t->p[i] = m.m[i].p;
}

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" {
#pragma GCC visibility push(default)

int64_t ss_orthogonal_workspace(int count, int64_t rows, int64_t cols) {
    if (!sizes_ok(count, rows, cols)) return -1;
    if (count == 0 || rows == 0 || cols == 0) return 0;
    Layout l;
    return layout_of(count, rows, cols, &l) == SS_OK ? l.bytes : -1;
}

int ss_orthogonalise(const void* const* in, int64_t in_stride, ss_dtype in_dt, void* const* out, int64_t out_stride,
                     ss_dtype out_dt, int count, int64_t rows, int64_t cols, const float* coefficients, int steps,
                     void* workspace, int64_t workspace_bytes, void* cuda_stream) {
    if (!dtype_known(in_dt) || !dtype_known(out_dt) || !sizes_ok(count, rows, cols)) return SS_ERR_INVALID_ARG;
    int status = check_coefficients(coefficients, steps);
    if (status != SS_OK) return status;
    if (count == 0 || rows == 0 || cols == 0) return SS_OK;
    const Mats a(in, count, rows, cols, in_stride, dtype_bytes(in_dt)), b(out, count, rows, cols, out_stride, dtype_bytes(out_dt));
    for (const Mats* m : {&a, &b})
        if (m->status != SS_OK) return m->status;
    if (overlaps(b, a, count, true) || overlaps_itself(b, count)) return SS_ERR_INVALID_ARG;
    Layout l;
    status = layout_of(count, rows, cols, &l);
    if (status == SS_OK) status = check_workspace(l, workspace, workspace_bytes);
    if (status != SS_OK) return status;
    if (overlaps_scratch(a, count, workspace, l.bytes) || overlaps_scratch(b, count, workspace, l.bytes)) return SS_ERR_INVALID_ARG;
    Call c{};
    fill(&c.start.in, a, count);
    c.start.in_stride = a.m[0].stride, c.start.vectors = a.vectors;
    fill(&c.result.out, b, count);
    c.result.stride = b.m[0].stride, c.result.vectors = b.vectors, c.to = out_dt == SS_BF16 ? kToBf16 : kToF32;
    c.in_dt = in_dt, c.count = count, c.rows = rows, c.cols = cols, c.coefficients = coefficients, c.steps = steps;
    return run(c, l, static_cast<uint8_t*>(workspace), static_cast<cudaStream_t>(cuda_stream));
}

int ss_orthogonal_update(const void* const* grads, int64_t grad_stride, ss_dtype dt, const float* const* momenta,
                         float* const* momenta_out, int64_t momentum_stride, const float* const* params,
                         float* const* params_out, int64_t param_stride, int count, int64_t rows, int64_t cols,
                         float beta, int nesterov, const float* coefficients, int steps, float lr, float scale,
                         float weight_decay, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
    if (!dtype_known(dt) || !sizes_ok(count, rows, cols)) return SS_ERR_INVALID_ARG;
    if (!(beta >= 0.0f && beta < 1.0f) || !std::isfinite(lr) || !std::isfinite(scale) || !std::isfinite(weight_decay)) return SS_ERR_INVALID_ARG;
    int status = check_coefficients(coefficients, steps);
    if (status != SS_OK) return status;
    if (count == 0 || rows == 0 || cols == 0) return SS_OK;
    using P = const void* const*;
    const Mats g(grads, count, rows, cols, grad_stride, dtype_bytes(dt));
    const Mats v(reinterpret_cast<P>(momenta), count, rows, cols, momentum_stride, 4), vo(reinterpret_cast<P>(momenta_out), count, rows, cols, momentum_stride, 4);
    const Mats p(reinterpret_cast<P>(params), count, rows, cols, param_stride, 4), po(reinterpret_cast<P>(params_out), count, rows, cols, param_stride, 4);
    for (const Mats* m : {&g, &v, &vo, &p, &po})
        if (m->status != SS_OK) return m->status;
    if (overlaps_itself(vo, count) || overlaps_itself(po, count) || overlaps(vo, po, count, false)) return SS_ERR_INVALID_ARG;
    if (overlaps(vo, v, count, true) || overlaps(vo, g, count, false) || overlaps(vo, p, count, false)) return SS_ERR_INVALID_ARG;
    if (overlaps(po, p, count, true) || overlaps(po, g, count, false) || overlaps(po, v, count, false)) return SS_ERR_INVALID_ARG;
    Layout l;
    status = layout_of(count, rows, cols, &l);
    if (status == SS_OK) status = check_workspace(l, workspace, workspace_bytes);
    if (status != SS_OK) return status;
    for (const Mats* m : {&g, &v, &vo, &p, &po})
        if (overlaps_scratch(*m, count, workspace, l.bytes)) return SS_ERR_INVALID_ARG;
    Call c{};
    Start& s = c.start;
    fill(&s.in, g, count), fill(&s.momentum, v, count), fill(&s.momentum_out, vo, count);
    s.in_stride = g.m[0].stride, s.momentum_stride = v.m[0].stride, s.vectors = g.vectors && v.vectors && vo.vectors;
    s.update = 1, s.nesterov = nesterov != 0, s.beta = beta, s.rest = 1.0f - beta;
    Result<kToF32>& r = c.result;
    c.to = kToParam;
    fill(&r.param, p, count), fill(&r.out, po, count);
    r.stride = p.m[0].stride, r.vectors = p.vectors && po.vectors;
    r.lr = lr, r.scale = scale, r.decay = weight_decay;
    c.in_dt = dt, c.count = count, c.rows = rows, c.cols = cols, c.coefficients = coefficients, c.steps = steps;
    return run(c, l, static_cast<uint8_t*>(workspace), static_cast<cudaStream_t>(cuda_stream));
}

#pragma GCC visibility pop
}  // extern "C"
