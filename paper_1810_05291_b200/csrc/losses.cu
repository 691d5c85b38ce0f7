// Losses over a language model's logits, with their gradient: the clipped policy loss and the
// paired preference loss.
#include <cmath>
#include <type_traits>

#include "tcgen05.cuh"
#include "train.cuh"

namespace ss {

template <>
struct Elem<uint32_t> {  // fp32 by its bits
    static __device__ __forceinline__ float load(const uint32_t* p) { return __uint_as_float(*p); }
    static __device__ __forceinline__ void store(uint32_t* p, float v) { *p = __float_as_uint(v); }
};

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// Softmax statistics: s = sum of 2^(k (z - m)) over what was seen, m the largest z, k = c log2 e. The
// difference comes before the factor: k m itself would overflow for a row of the type's lowest value.
struct Stat {
    float m, s;
};

__device__ __forceinline__ float exp2_fast(float x) {  // 2^x to about 2 units in the last place
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// A maximum of -inf means that nothing but -inf was seen: its sum is 0, and 2^(-inf - -inf) must not be formed.
__device__ __forceinline__ Stat join(const Stat& a, const Stat& b, float k) {
    const float m = fmaxf(a.m, b.m);
    const float fa = a.m == -INFINITY ? 0.0f : exp2_fast((a.m - m) * k), fb = b.m == -INFINITY ? 0.0f : exp2_fast((b.m - m) * k);
    return Stat{m, a.s * fa + b.s * fb};
}

// Joined over the THREADS threads that share a row, in a fixed order; every one of them gets the result.
template <int THREADS>
__device__ __forceinline__ Stat row_join(Stat v, Stat* shared, float k) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = join(v, Stat{__shfl_xor_sync(0xFFFFFFFFu, v.m, o), __shfl_xor_sync(0xFFFFFFFFu, v.s, o)}, k);
    if constexpr (THREADS > 32) {
        if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
        __syncthreads();
        const int lane = threadIdx.x & 31;
        v = lane < THREADS / 32 ? shared[lane] : Stat{-INFINITY, 0.0f};
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v = join(v, Stat{__shfl_xor_sync(0xFFFFFFFFu, v.m, o), __shfl_xor_sync(0xFFFFFFFFu, v.s, o)}, k);
    }
    return v;
}

struct Logits {
    const void* z;
    void* dz;
    int64_t z_stride, dz_stride, vocab;
    const int64_t* targets;
    const float* weights;
    const float* grad_scale;
    float c;  // inverse temperature
    float* logp;
};

__device__ __forceinline__ bool row_live(const Logits& a, int64_t row, int64_t* target, float* w) {
    *target = a.targets[row];
    *w = a.weights[row];
    return *w != 0.0f && *target >= 0 && *target < a.vocab;
}

// ---- a row as vectors of 16 bytes -------------------------------------------------------------------
// The vectors are those of memory, so a row that starts off their grid has a first (and a last)
// one with elements that are not its own: those are never touched, and read as -inf.
template <typename T>
struct Row {
    static constexpr int kPer = 16 / sizeof(T);
    uintptr_t base;  // of vector 0
    int head;        // elements of vector 0 before the row
    int64_t end;     // head + vocab
    int64_t vectors;

    __device__ __forceinline__ Row(const void* p, int64_t vocab) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        base = at & ~static_cast<uintptr_t>(15);
        head = static_cast<int>((at & 15) / sizeof(T));
        end = head + vocab;
        vectors = (end + kPer - 1) / kPer;
    }
    __device__ __forceinline__ bool whole(int64_t j) const { return (j > 0 || head == 0) && (j + 1) * kPer <= end; }
    __device__ __forceinline__ bool own(int64_t i) const { return i >= head && i < end; }  // element i of the vectors
    __device__ __forceinline__ T* element(int64_t i) const { return reinterpret_cast<T*>(base) + i; }
    __device__ __forceinline__ uint4* vector(int64_t j) const { return reinterpret_cast<uint4*>(base) + j; }
};

template <typename T>
struct Vec {
    static constexpr int kPer = Row<T>::kPer;
    uint4 v;

    __device__ __forceinline__ const uint32_t* words() const { return &v.x; }
    __device__ __forceinline__ float get(int i) const {
        const uint32_t* w = &v.x;
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float((i & 1) ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
    }
    __device__ __forceinline__ void load(const Row<T>& r, int64_t j) {
        if (r.whole(j)) {
            v = *r.vector(j);
            return;
        }
        uint32_t w[4];
        constexpr uint32_t none = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;  // -inf
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = none;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (!r.own(j * kPer + i)) continue;
            const uint32_t x = *r.element(j * kPer + i);
            if constexpr (sizeof(T) == 4) w[i] = x;
            else w[i >> 1] = (i & 1) ? (w[i >> 1] & 0x0000FFFFu) | (x << 16) : (w[i >> 1] & 0xFFFF0000u) | x;
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void store(const Row<T>& r, int64_t j) const {
        if (r.whole(j)) {
            __stcs(r.vector(j), v);
            return;
        }
        const uint32_t* w = &v.x;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (!r.own(j * kPer + i)) continue;
            if constexpr (sizeof(T) == 4) *r.element(j * kPer + i) = w[i];
            else *r.element(j * kPer + i) = static_cast<T>(w[i >> 1] >> (16 * (i & 1)));
        }
    }
};

// Two fp32 operations at once.
__device__ __forceinline__ float2 sub_mul2(float a, float b, float minus, float k) {
    float2 r;
    asm("{\n\t.reg .b64 x, m, k;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 m, {%4, %4};\n\tmov.b64 k, {%5, %5};\n\t"
        "add.rn.f32x2 x, x, m;\n\tmul.rn.f32x2 x, x, k;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a), "f"(b), "f"(minus), "f"(k));
    return r;
}

template <typename T>
__device__ __forceinline__ void add_vector(Stat& v, const Vec<T>& x, float k) {
    constexpr int n = Vec<T>::kPer;
    float top = x.get(0);
#pragma unroll
    for (int i = 1; i < n; ++i) top = fmaxf(top, x.get(i));
    if (top > v.m) {
        v.s *= exp2_fast((v.m - top) * k);  // 0 where nothing was seen: m is -inf
        v.m = top;
    }
    const float minus = v.m == -INFINITY ? 0.0f : -v.m;  // nothing but -inf so far: their terms are 0
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < n; i += 2) {
        const float2 t = sub_mul2(x.get(i), x.get(i + 1), minus, k);
        sum[0] += exp2_fast(t.x), sum[1] += exp2_fast(t.y);
    }
    v.s += sum[0] + sum[1];
}

// coef ([v = y] - softmax_v) for the elements of vector j, `f` = -coef / s; target counted in the vectors' elements.
template <typename T>
__device__ __forceinline__ Vec<T> grad_vector(const Vec<T>& x, int64_t j, int64_t target, float m, float k, float f, float coef) {
    constexpr int n = Vec<T>::kPer;
    float g[n];
#pragma unroll
    for (int i = 0; i < n; i += 2) {
        const float2 t = sub_mul2(x.get(i), x.get(i + 1), -m, k);
        g[i] = f * exp2_fast(t.x), g[i + 1] = f * exp2_fast(t.y);
    }
    if (target / n == j) {
#pragma unroll
        for (int i = 0; i < n; ++i)
            if (target % n == i) g[i] += coef;
    }
    Vec<T> r;
    uint32_t* w = &r.v.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(g[i]);
        else w[i] = bf16_pair(g[2 * i], g[2 * i + 1]);
    }
    return r;
}

// Stores vector j of z's grid to dz, whose rows may lie differently against 16 bytes.
template <typename T>
__device__ __forceinline__ void store_vector(const Vec<T>& v, const Row<T>& z, const Row<T>& dz, int64_t j) {
    if (z.head == dz.head) {
        v.store(dz, j);
        return;
    }
    const uint32_t* w = v.words();
#pragma unroll
    for (int i = 0; i < Vec<T>::kPer; ++i) {
        const int64_t at = j * Vec<T>::kPer + i;
        if (!z.own(at)) continue;
        T* p = dz.element(at - z.head + dz.head);
        if constexpr (sizeof(T) == 4) *p = w[i];
        else *p = static_cast<T>(w[i >> 1] >> (16 * (i & 1)));
    }
}

// Vectors first, first + step, ... below last.
template <typename T>
__device__ __forceinline__ Stat stat_of(const Row<T>& r, int64_t first, int64_t last, int step, float k) {
    constexpr int kAhead = 4;  // loads of a thread under way at a time
    Stat v{-INFINITY, 0.0f};
    int64_t j = first;
    for (; j + (kAhead - 1) * step < last; j += kAhead * step) {
        Vec<T> x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) x[u].load(r, j + u * step);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) add_vector(v, x[u], k);
    }
    for (; j < last; j += step) {
        Vec<T> x;
        x.load(r, j);
        add_vector(v, x, k);
    }
    return v;
}

template <typename T>
__device__ __forceinline__ void grad_of(const Row<T>& z, const Row<T>& dz, int64_t first, int64_t last, int step, int64_t target,
                                        const Stat& s, float k, float coef) {
    constexpr int kAhead = 4;
    const float f = -coef / s.s;
    int64_t j = first;
    for (; j + (kAhead - 1) * step < last; j += kAhead * step) {
        Vec<T> x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) x[u].load(z, j + u * step);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) store_vector(grad_vector(x[u], j + u * step, target + z.head, s.m, k, f, coef), z, dz, j + u * step);
    }
    for (; j < last; j += step) {
        Vec<T> x;
        x.load(z, j);
        store_vector(grad_vector(x, j, target + z.head, s.m, k, f, coef), z, dz, j);
    }
}

template <typename T>
__device__ __forceinline__ void zero_of(const Row<T>& dz, int64_t first, int64_t last, int step) {
    Vec<T> zero;
    zero.v = make_uint4(0u, 0u, 0u, 0u);
    for (int64_t j = first; j < last; j += step) zero.store(dz, j);
}

struct Policy {
    const float *old_logp, *ref_logp, *advantages;
    float lo, hi, beta;
    float* terms;  // 3 * rows: what each position adds to the totals
};

struct PolicyTerm {
    float loss, kl, clipped, slope;
};

__device__ __forceinline__ PolicyTerm policy_term(const Policy& p, int64_t row, float logp, float w) {
    const float adv = p.advantages[row], r = expf(logp - p.old_logp[row]);
    const float gain = r * adv, held = fminf(fmaxf(r, p.lo), p.hi) * adv;
    const bool clipped = gain > held;
    float kl = 0.0f, dkl = 0.0f;
    if (p.ref_logp != nullptr) {
        const float back = p.ref_logp[row] - logp, u = expf(back);
        kl = u - back - 1.0f;
        dkl = 1.0f - u;
    }
    return PolicyTerm{w * (p.beta * kl - (clipped ? held : gain)), w * kl, clipped ? w : 0.0f,
                      w * ((clipped ? 0.0f : -gain) + p.beta * dkl)};
}

__device__ __forceinline__ void store_term(const Logits& a, const Policy& p, int64_t rows, int64_t row, float logp, const PolicyTerm& t) {
    a.logp[row] = logp;
    p.terms[row] = t.loss, p.terms[rows + row] = t.kl, p.terms[2 * rows + row] = t.clipped;
}

__device__ __forceinline__ float scale_of(const Logits& a) { return a.c * (a.grad_scale == nullptr ? 1.0f : *a.grad_scale); }

// ---- rows read straight from memory, THREADS threads (a warp or a block) to a row. With a
// gradient the row is read twice, the second time from the caches. ------------------------------------
template <int THREADS>
constexpr int block_of() { return THREADS > 256 ? THREADS : 256; }

template <typename T, int THREADS>
__global__ void __launch_bounds__(block_of<THREADS>()) policy_stream_kernel(const __grid_constant__ Logits a, const __grid_constant__ Policy p, int64_t rows) {
    __shared__ Stat shared[THREADS / 32];
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (blockDim.x / THREADS) + threadIdx.x / THREADS;
    const int t = threadIdx.x % THREADS;
    if (row >= rows) return;  // whole warps, or none of the block
    const Row<T> z(static_cast<const T*>(a.z) + row * a.z_stride, a.vocab);
    const Row<T> dz(a.dz == nullptr ? nullptr : static_cast<T*>(a.dz) + row * a.dz_stride, a.vocab);
    int64_t target;
    float w;
    if (!row_live(a, row, &target, &w)) {
        if (a.dz != nullptr) zero_of(dz, t, dz.vectors, THREADS);
        if (t == 0) store_term(a, p, rows, row, 0.0f, PolicyTerm{0.0f, 0.0f, 0.0f, 0.0f});
        return;
    }
    const float k = a.c * kLog2e, picked = Elem<T>::load(z.element(target + z.head));
    const Stat s = row_join<THREADS>(stat_of(z, t, z.vectors, THREADS, k), shared, k);
    const float logp = (picked - s.m) * a.c - logf(s.s);
    const PolicyTerm term = policy_term(p, row, logp, w);
    if (t == 0) store_term(a, p, rows, row, logp, term);
    if (a.dz != nullptr) grad_of(z, dz, t, z.vectors, THREADS, target, s, k, term.slope * scale_of(a));
}

// ---- rows held in shared memory between the sum and the gradient: one block to a row, or a cluster
// of up to 8 whose blocks hold a slice each and exchange their statistics. ------------------------------
constexpr int kSliceThreads = 256;
constexpr int kParts = 4;  // of a slice, so that summing starts when the first has arrived

template <typename T>
__global__ void __launch_bounds__(kSliceThreads) policy_slice_kernel(const __grid_constant__ Logits a, const __grid_constant__ Policy p, int64_t rows, int slice) {
    extern __shared__ __align__(128) uint8_t dynamic[];
    __shared__ Stat shared[kSliceThreads / 32], joined[8];
    __shared__ uint64_t arrived[kParts];
    __shared__ int abort;
    uint4* const held = reinterpret_cast<uint4*>(dynamic);
    uint32_t rank, size;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
    const int64_t row = blockIdx.x / size;
    const int t = threadIdx.x;
    const Row<T> z(static_cast<const T*>(a.z) + row * a.z_stride, a.vocab);
    const Row<T> dz(static_cast<T*>(a.dz) + row * a.dz_stride, a.vocab);
    const int64_t first = static_cast<int64_t>(rank) * slice;
    int64_t target;
    float w;
    if (!row_live(a, row, &target, &w)) {  // for every block of the cluster
        const int64_t most = dz.vectors > z.vectors ? dz.vectors : z.vectors;
        zero_of(dz, first + t, min(rank + 1 == size ? most : first + slice, dz.vectors), kSliceThreads);
        if (rank == 0 && t == 0) store_term(a, p, rows, row, 0.0f, PolicyTerm{0.0f, 0.0f, 0.0f, 0.0f});
        return;
    }
    // every block of the cluster must have begun before another writes to its memory
    if (size > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    const int n = static_cast<int>(max(min(z.vectors - first, static_cast<int64_t>(slice)), static_cast<int64_t>(0)));
    const int part = (n + kParts - 1) / kParts;
    if (t == 0) {
        for (int i = 0; i < kParts; ++i) mbar_init(smem_addr(&arrived[i]), 1);
        abort = 0;
        mbar_init_visible();
        // whole vectors by bulk copies; the first and the last of the row, if they are not, below
        const int lo = n > 0 && !z.whole(first) ? 1 : 0, hi = n > 0 && !z.whole(first + n - 1) ? n - 1 : n;
        for (int i = 0; i < kParts; ++i) {
            const int from = max(i * part, lo), to = min((i + 1) * part, hi);
            const uint32_t bytes = to > from ? (to - from) * 16 : 0;
            mbar_expect(smem_addr(&arrived[i]), bytes);
            if (bytes > 0) bulk_load(smem_addr(held + from), z.vector(first + from), smem_addr(&arrived[i]), bytes);
        }
    }
    if (t == 32 && n > 0) {
        Vec<T> x;
        if (!z.whole(first)) x.load(z, first), held[0] = x.v;
        if (!z.whole(first + n - 1)) x.load(z, first + n - 1), held[n - 1] = x.v;
    }
    const float k = a.c * kLog2e, picked = Elem<T>::load(z.element(target + z.head));
    __syncthreads();
    Stat s{-INFINITY, 0.0f};
    bool ok = true;
    for (int i = 0; i < kParts; ++i) {
        ok = mbar_wait(smem_addr(&arrived[i]), 0, &abort) && ok;
        for (int j = i * part + t; j < min((i + 1) * part, n); j += kSliceThreads) {
            Vec<T> x;
            x.v = held[j];
            add_vector(s, x, k);
        }
    }
    if (!ok) s.s = __uint_as_float(0x7FC00000u);  // a copy that did not arrive shows
    s = row_join<kSliceThreads>(s, shared, k);
    if (size > 1) {
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        if (t < static_cast<int>(size)) {
            uint32_t at;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_addr(&joined[rank])), "r"(t));
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(s.m), "f"(s.s) : "memory");
        }
        asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
        s = joined[0];
        for (uint32_t i = 1; i < size; ++i) s = join(s, joined[i], k);
    }
    const float logp = (picked - s.m) * a.c - logf(s.s);
    const PolicyTerm term = policy_term(p, row, logp, w);
    if (rank == 0 && t == 0) store_term(a, p, rows, row, logp, term);
    const float coef = term.slope * scale_of(a), f = -coef / s.s;
    for (int j = t; j < n; j += kSliceThreads) {
        Vec<T> x;
        x.v = held[j];
        store_vector(grad_vector(x, first + j, target + z.head, s.m, k, f, coef), z, dz, first + j);
    }
}

constexpr int kSumThreads = 1024;

// Sum over a block of 1024 threads in a fixed order.
__device__ __forceinline__ double block_sum(double v, double* shared) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = shared[threadIdx.x & 31];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

__global__ void __launch_bounds__(kSumThreads) totals_kernel(const float* terms, int64_t n, double scale, float* out) {
    __shared__ double shared[32];
    const float* x = terms + blockIdx.x * n;
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += kSumThreads) v += x[i];
    v = block_sum(v, shared);
    if (threadIdx.x == 0) out[blockIdx.x] = static_cast<float>(scale * v);
}

// ---- preference loss: statistics of every row, then every pair's coefficient, then the gradient -----
struct Rows {
    Stat* stat;
    float* coef;
};

template <typename T, int THREADS>
__global__ void __launch_bounds__(block_of<THREADS>()) row_stat_kernel(const __grid_constant__ Logits a, Rows r, int64_t rows) {
    __shared__ Stat shared[THREADS / 32];
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (blockDim.x / THREADS) + threadIdx.x / THREADS;
    const int t = threadIdx.x % THREADS;
    if (row >= rows) return;
    int64_t target;
    float w;
    Stat s{0.0f, 1.0f};
    float logp = 0.0f;
    if (row_live(a, row, &target, &w)) {
        const Row<T> z(static_cast<const T*>(a.z) + row * a.z_stride, a.vocab);
        const float k = a.c * kLog2e, picked = Elem<T>::load(z.element(target + z.head));
        s = row_join<THREADS>(stat_of(z, t, z.vectors, THREADS, k), shared, k);
        logp = (picked - s.m) * a.c - logf(s.s);
    }
    if (t == 0) {
        a.logp[row] = logp;
        r.stat[row] = s;
        r.coef[row] = 0.0f;  // of rows that belong to no sequence
    }
}

struct Preference {
    const int64_t* begin;
    const float* ref;
    int64_t pairs, rows;
    ss_pref kind;
    float beta, smoothing, scale;
    float *margins, *seq_logp, *pair_loss;
};

__global__ void __launch_bounds__(kSumThreads) pair_kernel(const __grid_constant__ Logits a, const __grid_constant__ Preference p, Rows r) {
    __shared__ double shared[32];
    const int64_t pair = blockIdx.x;
    int64_t at[3];
    for (int i = 0; i < 3; ++i) {
        const int64_t b = p.begin[2 * pair + i];
        at[i] = b < 0 ? 0 : (b > p.rows ? p.rows : b);
    }
    double sum[2];
    for (int i = 0; i < 2; ++i) {
        double v = 0.0;
        for (int64_t t = at[i] + threadIdx.x; t < at[i + 1]; t += kSumThreads) {
            int64_t target;
            float w;
            if (row_live(a, t, &target, &w)) v += static_cast<double>(w) * a.logp[t];
        }
        sum[i] = block_sum(v, shared);
    }
    const double h = (sum[0] - p.ref[2 * pair]) - (sum[1] - p.ref[2 * pair + 1]);
    const float m = static_cast<float>(p.beta * h);
    float loss, slope;  // of l_p, with respect to h
    if (p.kind == SS_PREF_SIGMOID) {
        const float lost = log1pf(expf(-fabsf(m)));  // -log sigma(|m|)
        const float plus = lost + fmaxf(-m, 0.0f), minus = lost + fmaxf(m, 0.0f);
        loss = (1.0f - p.smoothing) * plus + p.smoothing * minus;
        slope = p.beta * (p.smoothing / (1.0f + expf(-m)) - (1.0f - p.smoothing) / (1.0f + expf(m)));
    } else if (p.kind == SS_PREF_HINGE) {
        loss = 1.0f - m > 0.0f ? 1.0f - m : (m >= 1.0f ? 0.0f : m);
        slope = m >= 1.0f ? 0.0f : (m < 1.0f ? -p.beta : m);
    } else {
        const float off = static_cast<float>(h - 0.5 / p.beta);
        loss = off * off;
        slope = 2.0f * off;
    }
    if (threadIdx.x == 0) {
        p.margins[pair] = m;
        p.seq_logp[2 * pair] = static_cast<float>(sum[0]), p.seq_logp[2 * pair + 1] = static_cast<float>(sum[1]);
        p.pair_loss[pair] = loss;
    }
    slope *= p.scale * (a.grad_scale == nullptr ? 1.0f : *a.grad_scale);
    for (int i = 0; i < 2; ++i)
        for (int64_t t = at[i] + threadIdx.x; t < at[i + 1]; t += kSumThreads) {
            int64_t target;
            float w;
            if (row_live(a, t, &target, &w)) r.coef[t] = (i == 0 ? slope : -slope) * w * a.c;
        }
}

// In the order opposite to the statistics', so that it begins with the rows that the caches still hold.
template <typename T, int THREADS>
__global__ void __launch_bounds__(block_of<THREADS>()) row_grad_kernel(const __grid_constant__ Logits a, Rows r, int64_t rows) {
    const int64_t row = rows - 1 - (static_cast<int64_t>(blockIdx.x) * (blockDim.x / THREADS) + threadIdx.x / THREADS);
    const int t = threadIdx.x % THREADS;
    if (row < 0) return;
    const Row<T> z(static_cast<const T*>(a.z) + row * a.z_stride, a.vocab);
    const Row<T> dz(static_cast<T*>(a.dz) + row * a.dz_stride, a.vocab);
    const float coef = r.coef[row];
    if (coef == 0.0f) zero_of(dz, t, dz.vectors, THREADS);
    else grad_of(z, dz, t, z.vectors, THREADS, a.targets[row], r.stat[row], a.c * kLog2e, coef);
}

// ---- choices of a launch ------------------------------------------------------------------------------
constexpr int64_t kWarpRowBytes = 8192;     // rows up to this size: a warp each
constexpr int kFewRows = 296;               // fewer rows than two for each SM: a large block each
constexpr int64_t kSliceBytes = 72 * 1024;  // three such blocks on an SM
constexpr int64_t kMostSliceBytes = 208 * 1024;

template <typename F>
void pick_threads(int64_t rows, int64_t vocab, ss_dtype dt, F&& launch) {
    auto by_type = [&](auto t) {
        if (vocab * static_cast<int64_t>(sizeof(t)) <= kWarpRowBytes) launch(t, std::integral_constant<int, 32>{});
        else if (rows < kFewRows) launch(t, std::integral_constant<int, 1024>{});
        else launch(t, std::integral_constant<int, 256>{});
    };
    if (dt == SS_F32) by_type(uint32_t{}); else by_type(uint16_t{});
}

template <int THREADS>
unsigned rows_grid(int64_t rows) {
    constexpr int per = block_of<THREADS>() / THREADS;
    return static_cast<unsigned>((rows + per - 1) / per);
}

// Blocks that share a row in policy_slice_kernel, 0 if it does not fit (or is small): the fewest with which
// three blocks fit on an SM, more where there are not enough rows for all SMs.
int cluster_of(int64_t rows, int64_t vocab, size_t eb) {
    const int64_t bytes = vocab * static_cast<int64_t>(eb) + 16;
    if (bytes <= kWarpRowBytes || bytes > 8 * kMostSliceBytes) return 0;
    int size = 1;
    while (size < 8 && (bytes > size * kSliceBytes || (rows * size < 148 && bytes > size * 8192))) size *= 2;
    return size;
}

template <typename T>
cudaError_t launch_slices(const Logits& a, const Policy& p, int64_t rows, int size, cudaStream_t st) {
    const int64_t vectors = (a.vocab * static_cast<int64_t>(sizeof(T)) + 15 + 15) / 16;  // wherever the row starts
    const int slice = static_cast<int>((vectors + size - 1) / size);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(rows * size));
    cfg.blockDim = dim3(kSliceThreads);
    cfg.dynamicSmemBytes = static_cast<size_t>(slice) * 16;
    cfg.stream = st;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = size, at.val.clusterDim.y = 1, at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaFuncSetAttribute(policy_slice_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(cfg.dynamicSmemBytes));
    return e != cudaSuccess ? e : cudaLaunchKernelEx(&cfg, policy_slice_kernel<T>, a, p, rows, slice);
}

// ---- checks shared by the two losses ------------------------------------------------------------------
struct Buffer {
    const void* p;
    size_t bytes, align;
    bool written;
};

// Every buffer present and aligned, and none that is written over any other. `z` and `dz` are checked apart.
int buffers_check(const Buffer* b, int n, const Mat& z, const Mat& dz) {
    for (int i = 0; i < n; ++i) {
        if (b[i].bytes == 0) continue;
        if (b[i].p == nullptr) return SS_ERR_INVALID_ARG;
        if (!addr_aligned(b[i].p, b[i].align)) return SS_ERR_MISALIGNED;
    }
    for (int i = 0; i < n; ++i) {
        if (b[i].written && mat_overlaps(z, b[i].p, b[i].bytes)) return SS_ERR_INVALID_ARG;
        if (dz.p != nullptr && mat_overlaps(dz, b[i].p, b[i].bytes)) return SS_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if ((b[i].written || b[j].written) && bytes_overlap(b[i].p, b[i].bytes, b[j].p, b[j].bytes)) return SS_ERR_INVALID_ARG;
    }
    return SS_OK;
}

int logits_check(const Mat& z, int64_t z_stride, const Mat& dz, int64_t dz_stride) {
    if (!stride_ok(z.rows, z.cols, z_stride)) return SS_ERR_INVALID_ARG;
    if (z.rows > 0 && z.cols > 0 && z.p == nullptr) return SS_ERR_INVALID_ARG;
    if (!addr_aligned(z.p, z.eb)) return SS_ERR_MISALIGNED;
    if (dz.p == nullptr) return SS_OK;
    if (!stride_ok(dz.rows, dz.cols, dz_stride)) return SS_ERR_INVALID_ARG;
    if (!addr_aligned(dz.p, dz.eb)) return SS_ERR_MISALIGNED;
    return mats_overlap(z, dz) && !same_mat(z, dz) ? SS_ERR_INVALID_ARG : SS_OK;
}

inline int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" {
#pragma GCC visibility push(default)

int64_t ss_loss_workspace(int64_t rows, int64_t n_pairs) {
    if (rows < 0 || rows > kMaxSide || n_pairs < 0 || n_pairs > kMaxSide) return -1;
    return round_up(rows * 12, 256) + round_up(n_pairs * 4, 256);
}

int ss_policy_loss(const void* logits, int64_t logits_stride, ss_dtype dt, int64_t rows, int64_t vocab,
                   const int64_t* targets, const float* old_logp, const float* ref_logp, const float* advantages,
                   const float* weights, float inv_temperature, float clip_low, float clip_high, float kl_coef,
                   const float* grad_scale, float* totals, float* logp, void* dlogits, int64_t dlogits_stride,
                   void* workspace, int64_t workspace_bytes, void* cuda_stream) {
    if (!dtype_known(dt) || !sides_ok(rows, vocab)) return SS_ERR_INVALID_ARG;
    if (!(inv_temperature > 0.0f) || !std::isfinite(inv_temperature) || !std::isfinite(kl_coef)) return SS_ERR_INVALID_ARG;
    if (!(clip_low >= 0.0f && clip_low <= 1.0f) || !(clip_high >= 0.0f) || !std::isfinite(clip_high)) return SS_ERR_INVALID_ARG;
    if (ref_logp == nullptr && kl_coef != 0.0f) return SS_ERR_INVALID_ARG;
    const size_t n = static_cast<size_t>(rows) * 4;
    const Mat z = mat(logits, rows, vocab, logits_stride, dtype_bytes(dt));
    const Mat dz = mat(dlogits, rows, vocab, dlogits_stride, dtype_bytes(dt));
    int s = logits_check(z, logits_stride, dz, dlogits_stride);
    if (s != SS_OK) return s;
    if (totals == nullptr) return SS_ERR_INVALID_ARG;
    const int64_t need = ss_loss_workspace(rows, 0);
    if (workspace_bytes < need) return SS_ERR_INVALID_ARG;
    const Buffer bufs[] = {{targets, 2 * n, 8, false}, {old_logp, n, 4, false}, {ref_logp, ref_logp == nullptr ? 0 : n, 4, false},
                           {advantages, n, 4, false}, {weights, n, 4, false}, {grad_scale, grad_scale == nullptr ? 0u : 4u, 4, false},
                           {totals, 12, 4, true}, {logp, n, 4, true}, {workspace, static_cast<size_t>(need), 256, true}};
    s = buffers_check(bufs, sizeof(bufs) / sizeof(bufs[0]), z, dz);
    if (s != SS_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const Logits a{logits, dlogits, z.stride, dz.stride, vocab, targets, weights, grad_scale, inv_temperature, logp};
    const Policy p{old_logp, ref_logp, advantages, 1.0f - clip_low, 1.0f + clip_high, kl_coef, static_cast<float*>(workspace)};
    if (rows > 0) {
        const int size = dlogits == nullptr ? 0 : cluster_of(rows, vocab, dtype_bytes(dt));
        if (size > 0 && rows * size <= kMaxSide) {
            const cudaError_t e = dt == SS_F32 ? launch_slices<uint32_t>(a, p, rows, size, st) : launch_slices<uint16_t>(a, p, rows, size, st);
            if (e != cudaSuccess) return cuda_status_public(e);
        } else {
            pick_threads(rows, vocab, dt, [&](auto t, auto threads) {
                policy_stream_kernel<decltype(t), threads.value><<<rows_grid<threads.value>(rows), block_of<threads.value>(), 0, st>>>(a, p, rows);
            });
        }
    }
    totals_kernel<<<3, kSumThreads, 0, st>>>(p.terms, rows, 1.0, totals);
    return cuda_status_public(cudaGetLastError());
}

int ss_preference_loss(const void* logits, int64_t logits_stride, ss_dtype dt, int64_t rows, int64_t vocab,
                       const int64_t* targets, const float* weights, const int64_t* seq_begin, int64_t n_pairs,
                       const float* ref_seq_logp, float inv_temperature, ss_pref kind, float beta,
                       float label_smoothing, float scale, const float* grad_scale, float* loss, float* margins,
                       float* seq_logp, float* logp, void* dlogits, int64_t dlogits_stride, void* workspace,
                       int64_t workspace_bytes, void* cuda_stream) {
    if (!dtype_known(dt) || !sides_ok(rows, vocab) || n_pairs < 0 || n_pairs > kMaxSide) return SS_ERR_INVALID_ARG;
    if (kind != SS_PREF_SIGMOID && kind != SS_PREF_HINGE && kind != SS_PREF_SQUARED) return SS_ERR_INVALID_ARG;
    if (!(inv_temperature > 0.0f) || !std::isfinite(inv_temperature) || !std::isfinite(scale)) return SS_ERR_INVALID_ARG;
    if (!(beta > 0.0f) || !std::isfinite(beta) || !(label_smoothing >= 0.0f && label_smoothing <= 0.5f)) return SS_ERR_INVALID_ARG;
    if (kind != SS_PREF_SIGMOID && label_smoothing != 0.0f) return SS_ERR_INVALID_ARG;
    const size_t n = static_cast<size_t>(rows) * 4, np = static_cast<size_t>(n_pairs) * 4;
    const Mat z = mat(logits, rows, vocab, logits_stride, dtype_bytes(dt));
    const Mat dz = mat(dlogits, rows, vocab, dlogits_stride, dtype_bytes(dt));
    int s = logits_check(z, logits_stride, dz, dlogits_stride);
    if (s != SS_OK) return s;
    if (loss == nullptr) return SS_ERR_INVALID_ARG;
    const int64_t need = ss_loss_workspace(rows, n_pairs);
    if (workspace_bytes < need) return SS_ERR_INVALID_ARG;
    const Buffer bufs[] = {{targets, 2 * n, 8, false}, {weights, n, 4, false}, {seq_begin, n_pairs > 0 ? 4 * np + 8 : 0, 8, false},
                           {ref_seq_logp, 2 * np, 4, false}, {grad_scale, grad_scale == nullptr ? 0u : 4u, 4, false},
                           {loss, 4, 4, true}, {margins, np, 4, true}, {seq_logp, 2 * np, 4, true}, {logp, n, 4, true},
                           {workspace, static_cast<size_t>(need), 256, true}};
    s = buffers_check(bufs, sizeof(bufs) / sizeof(bufs[0]), z, dz);
    if (s != SS_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const Logits a{logits, dlogits, z.stride, dz.stride, vocab, targets, weights, grad_scale, inv_temperature, logp};
    const Rows r{static_cast<Stat*>(workspace), static_cast<float*>(workspace) + 2 * rows};
    float* pair_loss = reinterpret_cast<float*>(static_cast<char*>(workspace) + round_up(rows * 12, 256));
    const Preference p{seq_begin, ref_seq_logp, n_pairs, rows, kind, beta, label_smoothing, scale, margins, seq_logp, pair_loss};
    if (rows > 0) {
        pick_threads(rows, vocab, dt, [&](auto t, auto threads) {
            row_stat_kernel<decltype(t), threads.value><<<rows_grid<threads.value>(rows), block_of<threads.value>(), 0, st>>>(a, r, rows);
        });
    }
    if (n_pairs > 0) pair_kernel<<<static_cast<unsigned>(n_pairs), kSumThreads, 0, st>>>(a, p, r);
    totals_kernel<<<1, kSumThreads, 0, st>>>(pair_loss, n_pairs, scale, loss);
    if (rows > 0 && dlogits != nullptr) {
        pick_threads(rows, vocab, dt, [&](auto t, auto threads) {
            row_grad_kernel<decltype(t), threads.value><<<rows_grid<threads.value>(rows), block_of<threads.value>(), 0, st>>>(a, r, rows);
        });
    }
    return cuda_status_public(cudaGetLastError());
}

#pragma GCC visibility pop
}  // extern "C"
