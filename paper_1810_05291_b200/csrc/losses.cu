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
__device__ __forceinline__ float warp_max(float x) {  // NaNs are passed over
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}

// Joined over a warp's first N lanes (a power of two; the others hold nothing), in a fixed order;
// every lane gets the result. One maximum, one rescaling, then plain sums.
template <int N>
__device__ __forceinline__ Stat warp_join(Stat v, float k) {
    const float m = warp_max(v.m);
    float s = v.s * (v.m == -INFINITY ? 0.0f : exp2_fast((v.m - m) * k));  // a NaN stays one
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if constexpr (N < 32) s = __shfl_sync(0xFFFFFFFFu, s, 0);
    return Stat{m, s};
}

// Joined over the THREADS threads that share a row; every one of them gets the result.
template <int THREADS>
__device__ __forceinline__ Stat row_join(Stat v, Stat* shared, float k) {
    v = warp_join<32>(v, k);
    if constexpr (THREADS > 32) {
        if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
        __syncthreads();
        const int lane = threadIdx.x & 31;
        v = warp_join<THREADS / 32>(lane < THREADS / 32 ? shared[lane] : Stat{-INFINITY, 0.0f}, k);
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
// one with elements that are not its own: those are never touched, and read as -inf. Whole vectors
// are lo .. hi - 1; the loops run over them alone, and one thread each takes the partial ones.
template <typename T>
struct Row {
    static constexpr int kPer = 16 / sizeof(T);
    uintptr_t base;           // of vector 0
    uint32_t head, end;       // the row's elements, counted from there
    uint32_t lo, hi;
    bool first, last;         // partial vectors 0 and hi

    __device__ __forceinline__ Row(const void* p, int64_t vocab) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        base = at & ~static_cast<uintptr_t>(15);
        head = static_cast<uint32_t>(at & 15) / sizeof(T);
        end = head + static_cast<uint32_t>(vocab);
        lo = head > 0 ? 1 : 0;
        hi = max(end / kPer, lo);
        first = head > 0 && vocab > 0;
        last = end > hi * kPer;
    }
    __device__ __forceinline__ uint32_t vectors() const { return hi + (last ? 1 : 0); }
    __device__ __forceinline__ T* element(uint32_t i) const { return reinterpret_cast<T*>(base) + i; }
    __device__ __forceinline__ uint4* vector(uint32_t j) const { return reinterpret_cast<uint4*>(base) + j; }
    __device__ __forceinline__ bool own(uint32_t i) const { return i >= head && i < end; }
};

template <typename T>
struct Vec {
    static constexpr int kPer = Row<T>::kPer;
    uint4 v;

    __device__ __forceinline__ uint32_t word(int i) const { return i == 0 ? v.x : (i == 1 ? v.y : (i == 2 ? v.z : v.w)); }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(word(i));
        else return __uint_as_float((i & 1) ? word(i >> 1) & 0xFFFF0000u : word(i >> 1) << 16);
    }
    __device__ __forceinline__ void set(const float (&g)[kPer]) {
        if constexpr (sizeof(T) == 4) v = make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
        else v = make_uint4(bf16_pair(g[0], g[1]), bf16_pair(g[2], g[3]), bf16_pair(g[4 % kPer], g[5 % kPer]), bf16_pair(g[6 % kPer], g[7 % kPer]));
    }
    __device__ __forceinline__ void none() {  // nothing but -inf
        constexpr uint32_t w = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;
        v = make_uint4(w, w, w, w);
    }
    __device__ __forceinline__ void load_partial(const Row<T>& r, uint32_t j) {
        uint32_t w[4];
        none();
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = v.x;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (!r.own(j * kPer + i)) continue;
            const uint32_t x = *r.element(j * kPer + i);
            if constexpr (sizeof(T) == 4) w[i] = x;
            else w[i >> 1] = (i & 1) ? (w[i >> 1] & 0x0000FFFFu) | (x << 16) : (w[i >> 1] & 0xFFFF0000u) | x;
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    // The elements that vector j of z's grid has of the row, to the same elements of dz.
    __device__ __forceinline__ void store_partial(const Row<T>& z, const Row<T>& dz, uint32_t j) const {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (!z.own(j * kPer + i)) continue;
            T* p = dz.element(j * kPer + i - z.head + dz.head);
            if constexpr (sizeof(T) == 4) *p = word(i);
            else *p = static_cast<T>(word(i >> 1) >> (16 * (i & 1)));
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

__device__ __forceinline__ float2 mul2(float a, float b, float k) {
    float2 r;
    asm("{\n\t.reg .b64 x, k;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 k, {%4, %4};\n\tmul.rn.f32x2 x, x, k;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a), "f"(b), "f"(k));
    return r;
}

// Largest element of N vectors; NaNs are passed over (they reach the sum).
template <int N>
__device__ __forceinline__ float top_of(const Vec<uint32_t> (&x)[N]) {
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < N; ++u) top = fmaxf(top, fmaxf(fmaxf(x[u].get(0), x[u].get(1)), fmaxf(x[u].get(2), x[u].get(3))));
    return top;
}

__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

template <int N>
__device__ __forceinline__ float top_of(const Vec<uint16_t> (&x)[N]) {
    uint32_t top = 0xFF80FF80u;
#pragma unroll
    for (int u = 0; u < N; ++u) top = max_pair(top, max_pair(max_pair(x[u].v.x, x[u].v.y), max_pair(x[u].v.z, x[u].v.w)));
    return fmaxf(__uint_as_float(top << 16), __uint_as_float(top & 0xFFFF0000u));
}

// N vectors at once: one look at the maximum for all of them, and enough independent terms to keep
// the exponential unit busy.
template <typename T, int N>
__device__ __forceinline__ void add_vectors(Stat& v, const Vec<T> (&x)[N], float k) {
    const float top = top_of(x);
    if (top > v.m) {
        v.s *= exp2_fast((v.m - top) * k);  // 0 where nothing was seen: m is -inf
        v.m = top;
    }
    const float minus = v.m == -INFINITY ? 0.0f : -v.m;  // nothing but -inf so far: their terms are 0
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
        for (int i = 0; i < Vec<T>::kPer; i += 2) {
            const float2 t = sub_mul2(x[u].get(i), x[u].get(i + 1), minus, k);
            sum[i & 2] += exp2_fast(t.x), sum[(i & 2) + 1] += exp2_fast(t.y);
        }
    v.s += (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// f * 2^(k (z - m)): with f = -coef / s the gradient of a row, but for its target.
template <typename T>
__device__ __forceinline__ Vec<T> grad_vector(const Vec<T>& x, float m, float k, float f) {
    float g[Vec<T>::kPer];
#pragma unroll
    for (int i = 0; i < Vec<T>::kPer; i += 2) {
        const float2 t = sub_mul2(x.get(i), x.get(i + 1), -m, k), r = mul2(exp2_fast(t.x), exp2_fast(t.y), f);
        g[i] = r.x, g[i + 1] = r.y;
    }
    Vec<T> v;
    v.set(g);
    return v;
}

constexpr int kAhead = 4;  // vectors that a thread works on at a time

// Whole vectors lo + t, lo + t + THREADS, ...; the first partial vector by thread 0, the last by the last.
template <typename T, int THREADS>
__device__ __forceinline__ Stat stat_of(const Row<T>& r, uint32_t t, float k) {
    Stat v{-INFINITY, 0.0f};
    const uint32_t n = r.hi - r.lo;
    const uint4* p = r.vector(r.lo + t);
    uint32_t j = t;
    for (; j + (kAhead - 1) * THREADS < n; j += kAhead * THREADS, p += kAhead * THREADS) {
        Vec<T> x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) x[u].v = p[u * THREADS];
        add_vectors(v, x, k);
    }
    if (j < n) {  // the rest of them at once too
        Vec<T> x[kAhead - 1];
#pragma unroll
        for (int u = 0; u < kAhead - 1; ++u) {
            if (j + u * THREADS < n) x[u].v = p[u * THREADS];
            else x[u].none();
        }
        add_vectors(v, x, k);
    }
    if ((r.first && t == 0) || (r.last && t == THREADS - 1)) {
        Vec<T> x[1];
        if (r.first && t == 0) x[0].load_partial(r, 0), add_vectors(v, x, k);
        if (r.last && t == THREADS - 1) x[0].load_partial(r, r.hi), add_vectors(v, x, k);
    }
    return v;
}

// dz = coef ([v = y] - softmax_v). The target's element is written once more by the thread that
// wrote it (`picked`: its logit, read before anything is written: dz may be z).
template <typename T, int THREADS>
__device__ __forceinline__ void grad_of(const Row<T>& z, const Row<T>& dz, uint32_t t, uint32_t target, float picked, const Stat& s,
                                        float k, float coef) {
    const float f = -coef / s.s;
    const uint32_t n = z.hi - z.lo;
    const uint4* p = z.vector(z.lo + t);
    uint32_t j = t;
    if (z.head == dz.head) {
        uint4* q = dz.vector(z.lo + t);
        for (; j + (kAhead - 1) * THREADS < n; j += kAhead * THREADS, p += kAhead * THREADS, q += kAhead * THREADS) {
            Vec<T> x[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) x[u].v = p[u * THREADS];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) __stcs(q + u * THREADS, grad_vector(x[u], s.m, k, f).v);
        }
        Vec<T> x[kAhead - 1];
#pragma unroll
        for (int u = 0; u < kAhead - 1; ++u)
            if (j + u * THREADS < n) x[u].v = p[u * THREADS];
#pragma unroll
        for (int u = 0; u < kAhead - 1; ++u)
            if (j + u * THREADS < n) __stcs(q + u * THREADS, grad_vector(x[u], s.m, k, f).v);
    } else {  // rows of dz lie otherwise against 16 bytes: element by element
        for (; j < n; j += THREADS, p += THREADS) {
            Vec<T> x;
            x.v = *p;
            grad_vector(x, s.m, k, f).store_partial(z, dz, z.lo + j);
        }
    }
    if ((z.first && t == 0) || (z.last && t == THREADS - 1)) {
        Vec<T> x;
        if (z.first && t == 0) x.load_partial(z, 0), grad_vector(x, s.m, k, f).store_partial(z, dz, 0);
        if (z.last && t == THREADS - 1) x.load_partial(z, z.hi), grad_vector(x, s.m, k, f).store_partial(z, dz, z.hi);
    }
    const uint32_t at = (target + z.head) / Row<T>::kPer;  // the target's vector
    const uint32_t owner = at < z.lo ? 0 : (at >= z.hi ? THREADS - 1 : (at - z.lo) % THREADS);
    if (t == owner) Elem<T>::store(dz.element(target + dz.head), fmaf(f, exp2_fast((picked - s.m) * k), coef));
}

template <typename T>
__device__ __forceinline__ void zero_of(const Row<T>& dz, uint32_t from, uint32_t to, uint32_t t, uint32_t threads) {  // vectors
    for (uint32_t j = max(from, dz.lo) + t; j < min(to, dz.hi); j += threads) __stcs(dz.vector(j), make_uint4(0u, 0u, 0u, 0u));
    Vec<T> zero;
    zero.v = make_uint4(0u, 0u, 0u, 0u);
    if (dz.first && from == 0 && t == 0) zero.store_partial(dz, dz, 0);
    if (dz.last && from <= dz.hi && dz.hi < to && t == threads - 1) zero.store_partial(dz, dz, dz.hi);
}

struct Policy {
    const float *old_logp, *ref_logp, *advantages;
    float lo, hi, beta;
    float* terms;  // 3 * rows: what each position adds to the totals
};

struct PolicyTerm {
    float loss, kl, clipped, slope;
};

struct PolicyRow {
    float adv, old_logp, ref_logp;
    __device__ __forceinline__ PolicyRow(const Policy& p, int64_t row)
        : adv(p.advantages[row]), old_logp(p.old_logp[row]), ref_logp(p.ref_logp == nullptr ? 0.0f : p.ref_logp[row]) {}
};

// exp(x) - 1 and exp(x) - 1 - x. Near 0, where a policy still is its reference, the second is x^2 / 2 and next to
// nothing would be left of it after two differences; up to 1/2 it is its series, cut off below 2^-24 of it (x^7 / 9! of x^2).
__device__ __forceinline__ float2 exp_less_one(float x) {
    if (fabsf(x) < 0.5f) {
        float q = 1.0f / 40320.0f;
        q = fmaf(q, x, 1.0f / 5040.0f);
        q = fmaf(q, x, 1.0f / 720.0f);
        q = fmaf(q, x, 1.0f / 120.0f);
        q = fmaf(q, x, 1.0f / 24.0f);
        q = fmaf(q, x, 1.0f / 6.0f);
        q = fmaf(q, x, 0.5f);
        const float r = q * x * x;
        return make_float2(x + r, r);
    }
    const float e = expf(x) - 1.0f;
    return make_float2(e, e - x);
}

__device__ __forceinline__ PolicyTerm policy_term(const Policy& p, const PolicyRow& g, float logp, float w) {
    const float adv = g.adv, r = expf(logp - g.old_logp);
    const float gain = r * adv, held = fminf(fmaxf(r, p.lo), p.hi) * adv;
    const bool clipped = gain > held;
    float kl = 0.0f, dkl = 0.0f;
    if (p.ref_logp != nullptr) {
        const float back = g.ref_logp - logp;
        const float2 e = exp_less_one(back);
        kl = e.y;
        dkl = -e.x;
    }
    const bool penalty = p.beta != 0.0f;  // a coefficient of 0 leaves the term out, an infinite one too
    return PolicyTerm{w * ((penalty ? p.beta * kl : 0.0f) - (clipped ? held : gain)), w * kl, clipped ? w : 0.0f,
                      w * ((clipped ? 0.0f : -gain) + (penalty ? p.beta * dkl : 0.0f))};
}

__device__ __forceinline__ void store_term(const Logits& a, const Policy& p, int64_t rows, int64_t row, float logp, const PolicyTerm& t) {
    a.logp[row] = logp;
    p.terms[row] = t.loss, p.terms[rows + row] = t.kl, p.terms[2 * rows + row] = t.clipped;
}

__device__ __forceinline__ float scale_of(const Logits& a) { return a.c * (a.grad_scale == nullptr ? 1.0f : *a.grad_scale); }

// ---- rows read straight from memory, THREADS threads (a warp or a block) to a row. With a
// gradient the row is read twice, the second time from the caches. Bound by memory: the policy loss alone,
// 8192 x 131072 bf16, 332 us (6.5 TB/s). ---------------------------------------------------------------
template <int THREADS>
constexpr int block_of() { return THREADS > 32 ? THREADS : 256; }

template <typename T, int THREADS>
__global__ void __launch_bounds__(block_of<THREADS>()) policy_stream_kernel(const __grid_constant__ Logits a, const __grid_constant__ Policy p, int64_t rows) {
    next_may_begin();
    __shared__ Stat shared[THREADS / 32];
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (blockDim.x / THREADS) + threadIdx.x / THREADS;
    const int t = threadIdx.x % THREADS;
    if (row >= rows) return;  // whole warps, or none of the block
    const Row<T> z(static_cast<const T*>(a.z) + row * a.z_stride, a.vocab);
    const Row<T> dz(a.dz == nullptr ? nullptr : static_cast<T*>(a.dz) + row * a.dz_stride, a.vocab);
    int64_t target;
    float w;
    if (!row_live(a, row, &target, &w)) {
        if (a.dz != nullptr) zero_of(dz, 0, dz.vectors(), t, THREADS);
        if (t == 0) store_term(a, p, rows, row, 0.0f, PolicyTerm{0.0f, 0.0f, 0.0f, 0.0f});
        return;
    }
    const float k = a.c * kLog2e, picked = Elem<T>::load(z.element(static_cast<uint32_t>(target) + z.head));
    const PolicyRow given(p, row);
    const Stat s = row_join<THREADS>(stat_of<T, THREADS>(z, t, k), shared, k);
    const float logp = (picked - s.m) * a.c - logf(s.s);
    const PolicyTerm term = policy_term(p, given, logp, w);
    if (t == 0) store_term(a, p, rows, row, logp, term);
    if (a.dz != nullptr) grad_of<T, THREADS>(z, dz, t, static_cast<uint32_t>(target), picked, s, k, term.slope * scale_of(a));
}

// 16 bytes to the same place of block `to` of the cluster, and their arrival to its barrier.
__device__ __forceinline__ void tell(uint32_t at, uint32_t bar, int to, const float4& v) {
    asm volatile("{\n\t.reg .b32 x, y;\n\tmapa.shared::cluster.u32 x, %0, %2;\n\tmapa.shared::cluster.u32 y, %1, %2;\n\t"
                 "st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [x], {%3, %4, %5, %6}, [y];\n\t}"
                 ::"r"(at), "r"(bar), "r"(to), "r"(__float_as_uint(v.x)), "r"(__float_as_uint(v.y)), "r"(__float_as_uint(v.z)),
                 "r"(__float_as_uint(v.w)) : "memory");
}

// ---- rows read once: one block to a row, or a cluster of up to 8 whose blocks take a slice each. Slices
// come by bulk copies, a row or two ahead; a thread turns its 64 (or 128) logits of a row into exponentials
// relative to its own maximum, which stay in registers while the block, and the cluster, join their
// statistics. So the gradient needs one more factor and no second exponential: with two of them for
// each bf16 logit the exponential unit alone would take as long as the memory (8192 x 131072: 986 us).
//
// Bound by memory: a logit is read once and its gradient written once. 8192 x 131072 bf16 720 us
// (6.0 TB/s), 16384 x 32768 344 us (6.2), 30000 x 8000 165 us (5.8), 4096 x 131072 fp32 658 us (6.5). A row
// to a block of 512 threads with the row in shared memory: 986 us for the first, streaming it twice 957.
// Few rows are bound by the launches: 16 x 32768 takes 6.2 us with the totals.
constexpr int kSliceThreads = 128;
// Logits of a thread: 64, and where 8 blocks of that do not hold the row 128, at the price of two blocks fewer on an SM.
// (128 always: 2053 x 32001 fp32 112 us instead of 91, 4100 x 32001 bf16 136 instead of 112, 16384 x 32768 342
// instead of 344. Four blocks instead of five at 64: 820 us instead of 714 at 8192 x 131072, six the same.)
template <int HELD>
constexpr int kSliceBlocks = HELD == 64 ? 5 : 3;  // on an SM

template <typename T, int HELD>
constexpr int kSliceVectors = kSliceThreads * HELD / Row<T>::kPer;
template <typename T>
constexpr int kSliceSlots = sizeof(T) == 4 ? 1 : 2;

struct Slices {
    int64_t rows;
    int count;    // rows of a cluster, one after another
    int vectors;  // of a slice
};

// What a block has to know of a row before it can work on it.
struct Given {
    int target;  // -1: the row is left out
    float w;

    __device__ __forceinline__ Given(const Logits& a, int64_t row, bool in) : target(-1), w(0.0f) {
        int64_t y;
        if (in && row_live(a, row, &y, &w)) target = static_cast<int>(y);
    }
    __device__ __forceinline__ bool live() const { return target >= 0; }
};

// The end of a block in which a wait of thread 0 ran out, by that thread. (Where they were all met, every copy and message to the
// block has arrived.) Waits, with limits, for the copies that are still under way, and for the messages after every other
// block of the cluster has sent its own or has ended.
__device__ __noinline__ void drain(uint64_t* arrived, int slots, uint64_t* told, uint32_t size, uint32_t live_rows) {
    int own = 0;
    for (int i = 0; i < slots; ++i) {  // the phase that has not completed is the copy's, if there is one
        const uint32_t bar = smem_addr(&arrived[i]), parity = mbar_try(bar, 0) ? 1 : 0;
        mbar_wait(bar, parity, &own, kMaxTries >> 6);
    }
    if (size < 2) return;
    asm volatile("barrier.cluster.arrive.relaxed;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
    for (uint32_t i = 0; i < 2; ++i)
        if (const uint32_t rounds = (live_rows + 1 - i) >> 1) mbar_wait(smem_addr(&told[i]), (rounds - 1) & 1, &own);
}

template <typename T, int HELD>
__global__ void __launch_bounds__(kSliceThreads, kSliceBlocks<HELD>) policy_slice_kernel(const __grid_constant__ Logits a, const __grid_constant__ Policy p, const __grid_constant__ Slices c) {
    next_may_begin();
    extern __shared__ __align__(128) uint8_t dynamic[];
    constexpr int THREADS = kSliceThreads, kSlots = kSliceSlots<T>, kPer = Row<T>::kPer, kVectors = HELD / kPer;
    __shared__ Stat shared[2][THREADS / 32];  // two sets: a warp may be a row ahead of one that still reads
    __shared__ float4 joined[2][8];           // of the cluster's blocks: m, s, the target's logit
    __shared__ uint64_t arrived[kSlots], told[2];
    __shared__ int abort;
    uint32_t rank, size;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
    const uint32_t t = threadIdx.x;
    const int64_t row0 = blockIdx.x / size * static_cast<int64_t>(c.count);
    const int count = static_cast<int>(min(static_cast<int64_t>(c.count), c.rows - row0));
    const uint32_t begin = rank * c.vectors, stop = begin + c.vectors;  // this block's vectors of a row
    const float k = a.c * kLog2e;
    const T* const z0 = static_cast<const T*>(a.z);

    if (t == 0) {
        for (int i = 0; i < kSlots; ++i) mbar_init(smem_addr(&arrived[i]), 1);
        mbar_init(smem_addr(&told[0]), 1);
        mbar_init(smem_addr(&told[1]), 1);
        abort = 0;
        mbar_init_visible();
    }
    auto slot_of = [&](int i) { return reinterpret_cast<uint4*>(dynamic) + (kSlots == 2 ? i & 1 : 0) * c.vectors; };
    auto fetch = [&](int i) {  // by thread 0: the whole vectors of the slice
        const Row<T> z(z0 + (row0 + i) * a.z_stride, a.vocab);
        const uint32_t from = max(begin, z.lo), to = min(stop, z.hi), bytes = to > from ? (to - from) * 16 : 0;
        const uint32_t bar = smem_addr(&arrived[kSlots == 2 ? i & 1 : 0]);
        mbar_expect(bar, bytes);
        if (bytes > 0) bulk_load(smem_addr(slot_of(i) + (from - begin)), z.vector(from), bar, bytes);
    };

    Given now(a, row0, true), next(a, row0 + 1, count > 1);
    if (t == 0) {
        if (now.live()) fetch(0);
        if (kSlots == 2 && next.live()) fetch(1);
    }
    __syncthreads();
    // every block of the cluster must have begun, and its barriers be ready, before another writes to its memory
    // (the barriers' initialisation has a fence of its own)
    if (size > 1) asm volatile("barrier.cluster.arrive.relaxed;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
    uint32_t slot_parity = 0, live_rows = 0;  // slot_parity: a bit for each slot
    bool ok = true;
    for (int i = 0; i < count; ++i) {
        const int64_t row = row0 + i;
        const Row<T> z(z0 + row * a.z_stride, a.vocab);
        const Row<T> dz(static_cast<T*>(a.dz) + row * a.dz_stride, a.vocab);
        const Given later(a, row + 2, i + 2 < count);
        const bool fetch_next = kSlots == 2 ? later.live() : next.live();
        if (!now.live()) {  // for every block of the cluster
            zero_of(dz, begin, rank + 1 == size ? 0xFFFFFFFFu : stop, t, THREADS);
            if (rank == 0 && t == 0) store_term(a, p, c.rows, row, 0.0f, PolicyTerm{0.0f, 0.0f, 0.0f, 0.0f});
            if (fetch_next && t == 0 && ok) fetch(i + kSlots);  // once a wait ran out, nothing more is begun
        } else {
            const int slot = kSlots == 2 ? i & 1 : 0, set = live_rows & 1;
            const PolicyRow given(p, row);
            const uint32_t target = now.target + z.head, target_vector = target / kPer;
            const bool has_target = target_vector >= begin && target_vector < stop;
            float picked = has_target ? Elem<T>::load(z.element(target)) : 0.0f;
            if (size > 1 && t == 0) mbar_expect(smem_addr(&told[set]), size * 16);

            // this thread's vectors of the row are begin + t + u * THREADS; whole ones are below `whole`
            const uint4* const held = slot_of(i) + t;
            const uint32_t whole = min(stop, z.hi) > begin + t ? min(stop, z.hi) - begin - t : 0;
            const bool odd_first = z.first && begin == 0 && t == 0;
            const bool odd_last = z.last && z.hi >= begin && z.hi < stop && (z.hi - begin) % THREADS == t;
            ok = mbar_wait(smem_addr(&arrived[slot]), (slot_parity >> slot) & 1, &abort) && ok;
            slot_parity ^= 1u << slot;
            Vec<T> x[kVectors];
#pragma unroll
            for (int u = 0; u < kVectors; ++u) {
                if (u * THREADS < whole) x[u].v = held[u * THREADS];
                else x[u].none();
            }
            if (odd_first) x[0].load_partial(z, 0);
            if (odd_last) {
#pragma unroll
                for (int u = 0; u < kVectors; ++u)
                    if (begin + t + u * THREADS == z.hi) x[u].load_partial(z, z.hi);
            }
            const float top = top_of(x), minus = top == -INFINITY ? 0.0f : -top;
            float e[HELD], sum[2] = {0.0f, 0.0f};
#pragma unroll
            for (int u = 0; u < kVectors; ++u)
#pragma unroll
                for (int v = 0; v < kPer; v += 2) {
                    const float2 d = sub_mul2(x[u].get(v), x[u].get(v + 1), minus, k);
                    sum[0] += e[u * kPer + v] = exp2_fast(d.x);
                    sum[1] += e[u * kPer + v + 1] = exp2_fast(d.y);
                }
            Stat s{top, sum[0] + sum[1]};
            if (!ok) s.s = __uint_as_float(0x7FC00000u);  // a copy that did not arrive shows
            s = row_join<THREADS>(s, shared[set], k);
            // the block is past a barrier: its slot has been read
            if (fetch_next && t == 0 && ok) fetch(i + kSlots);  // once a wait ran out, nothing more is begun
            if (size > 1) {
                if (t < size) tell(smem_addr(&joined[set][rank]), smem_addr(&told[set]), t, make_float4(s.m, s.s, picked, 0.0f));
                ok = mbar_wait(smem_addr(&told[set]), (live_rows >> 1) & 1, &abort) && ok;
                const uint32_t lane = t & 31;
                const float4 o = lane < size ? joined[set][lane] : make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
                s = warp_join<8>(Stat{o.x, o.y}, k);
                float logit = o.z;  // 0 but for the block that has the target
#pragma unroll
                for (int d = 4; d > 0; d >>= 1) logit += __shfl_xor_sync(0xFFFFFFFFu, logit, d);
                picked = __shfl_sync(0xFFFFFFFFu, logit, 0);
                if (!ok) s.s = __uint_as_float(0x7FC00000u);
            }
            ++live_rows;
            const float logp = (picked - s.m) * a.c - logf(s.s);
            const PolicyTerm term = policy_term(p, given, logp, now.w);
            if (rank == 0 && t == 0) store_term(a, p, c.rows, row, logp, term);
            const float coef = term.slope * scale_of(a), all = -coef / s.s, f = all * exp2_fast((top - s.m) * k);
            auto grad = [&](int u) {
                float g[kPer];
#pragma unroll
                for (int v = 0; v < kPer; v += 2) {
                    const float2 r = mul2(e[u * kPer + v], e[u * kPer + v + 1], f);
                    g[v] = r.x, g[v + 1] = r.y;
                }
                Vec<T> v;
                v.set(g);
                return v;
            };
            if (z.head == dz.head) {
                uint4* const q = dz.vector(begin + t);
#pragma unroll
                for (int u = 0; u < kVectors; ++u)
                    if (u * THREADS < whole && !(u == 0 && odd_first)) __stcs(q + u * THREADS, grad(u).v);
            } else {
#pragma unroll
                for (int u = 0; u < kVectors; ++u)
                    if (u * THREADS < whole && !(u == 0 && odd_first)) grad(u).store_partial(z, dz, begin + t + u * THREADS);
            }
            if (odd_first) grad(0).store_partial(z, dz, 0);
            if (odd_last) {
#pragma unroll
                for (int u = 0; u < kVectors; ++u)
                    if (begin + t + u * THREADS == z.hi) grad(u).store_partial(z, dz, z.hi);
            }
            // once more, by the thread that wrote it
            if (has_target && (target_vector - begin) % THREADS == t)
                Elem<T>::store(dz.element(now.target + dz.head), fmaf(all, exp2_fast((picked - s.m) * k), coef));
        }
        now = next;
        next = later;
    }
    if (t == 0 && !ok) drain(arrived, kSlots, told, size, live_rows);
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

__global__ void __launch_bounds__(kSumThreads) totals_kernel(const float* terms, int64_t n, float* out) {
    after_previous();
    __shared__ double shared[32];
    const float* x = terms + blockIdx.x * n;
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += kSumThreads) v += x[i];
    v = block_sum(v, shared);
    if (threadIdx.x == 0) out[blockIdx.x] = static_cast<float>(v);
}

// ---- preference loss: statistics of every row, then every pair's coefficient, then the gradient -----
// A row's gradient has a factor that depends on every row of its pair, so the logits are read twice: three
// passes over memory with the write, and bound by it: 16384 rows of 65536 bf16, a quarter of them left out,
// 831 us (6.4 TB/s over the three; two passes alone would take 574). One kernel that forms the statistics of a pair while the
// pair before, still in the L2 cache, gets its gradient took 1045 us: the gradients that are written
// push the logits out, and what is under way at once is too little. Small calls wait for the three
// kernels to follow one another: 96 x 32768 fp32 in one pair 16.4 us.
struct Rows {
    Stat* stat;
    float* weight;  // what counts of weights[t]: 0 for rows left out
    float* coef;
};

template <typename T, int THREADS>
__global__ void __launch_bounds__(block_of<THREADS>()) row_stat_kernel(const __grid_constant__ Logits a, Rows r, int64_t rows) {
    next_may_begin();
    __shared__ Stat shared[THREADS / 32];
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (blockDim.x / THREADS) + threadIdx.x / THREADS;
    const int t = threadIdx.x % THREADS;
    if (row >= rows) return;
    int64_t target;
    float w;
    Stat s{0.0f, 1.0f};
    float logp = 0.0f;
    const bool live = row_live(a, row, &target, &w);
    if (live) {
        const Row<T> z(static_cast<const T*>(a.z) + row * a.z_stride, a.vocab);
        const float k = a.c * kLog2e, picked = Elem<T>::load(z.element(static_cast<uint32_t>(target) + z.head));
        s = row_join<THREADS>(stat_of<T, THREADS>(z, t, k), shared, k);
        logp = (picked - s.m) * a.c - logf(s.s);
    }
    if (t == 0) {
        a.logp[row] = logp;
        r.stat[row] = s;
        r.weight[row] = live ? w : 0.0f;
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
    next_may_begin();
    after_previous();
    __shared__ double shared[2][32];
    const int64_t pair = blockIdx.x;
    int64_t at[3];
    for (int i = 0; i < 3; ++i) {
        const int64_t b = p.begin[2 * pair + i];
        at[i] = b < 0 ? 0 : (b > p.rows ? p.rows : b);
    }
    // both sequences at once, each position to its own sum; the sums in a fixed order
    double sum[2] = {0.0, 0.0};
    for (int i = 0; i < 2; ++i)
        for (int64_t t = at[i] + threadIdx.x; t < at[i + 1]; t += kSumThreads) {
            const float w = r.weight[t];
            if (w != 0.0f) sum[i] += static_cast<double>(w) * a.logp[t];
        }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        sum[0] += __shfl_xor_sync(0xFFFFFFFFu, sum[0], o);
        sum[1] += __shfl_xor_sync(0xFFFFFFFFu, sum[1], o);
    }
    if ((threadIdx.x & 31) == 0) shared[0][threadIdx.x >> 5] = sum[0], shared[1][threadIdx.x >> 5] = sum[1];
    __syncthreads();
    sum[0] = shared[0][threadIdx.x & 31], sum[1] = shared[1][threadIdx.x & 31];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        sum[0] += __shfl_xor_sync(0xFFFFFFFFu, sum[0], o);
        sum[1] += __shfl_xor_sync(0xFFFFFFFFu, sum[1], o);
    }
    const double h = (sum[0] - p.ref[2 * pair]) - (sum[1] - p.ref[2 * pair + 1]);
    const float m = static_cast<float>(p.beta * h);
    float loss, slope;  // of l_p, with respect to h
    if (p.kind == SS_PREF_SIGMOID) {
        const float lost = log1pf(expf(-fabsf(m)));  // -log sigma(|m|)
        const float plus = lost + fmaxf(-m, 0.0f), minus = lost + fmaxf(m, 0.0f);
        loss = (1.0f - p.smoothing) * plus + (p.smoothing != 0.0f ? p.smoothing * minus : 0.0f);  // minus may be infinite
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
            const float w = r.weight[t];
            if (w != 0.0f) r.coef[t] = (i == 0 ? slope : -slope) * w * a.c;
        }
}

// Loss from the pairs' losses, by one warp in a fixed order.
struct Total {
    const float* pair_loss;
    int64_t pairs;
    double scale;
    float* loss;

    __device__ __forceinline__ void write() const {
        double v = 0.0;
        for (int64_t i = threadIdx.x & 31; i < pairs; i += 32) v += pair_loss[i];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
        if ((threadIdx.x & 31) == 0) *loss = static_cast<float>(scale * v);
    }
};

__global__ void __launch_bounds__(32) total_kernel(const __grid_constant__ Total total) {
    after_previous();
    total.write();
}

// In the order opposite to the statistics', so that it begins with the rows that the caches still hold.
// The first warp of the last block also writes the loss.
template <typename T, int THREADS>
__global__ void __launch_bounds__(block_of<THREADS>()) row_grad_kernel(const __grid_constant__ Logits a, Rows r, int64_t rows, const __grid_constant__ Total total) {
    after_previous();
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x < 32) total.write();
    const int64_t row = rows - 1 - (static_cast<int64_t>(blockIdx.x) * (blockDim.x / THREADS) + threadIdx.x / THREADS);
    const int t = threadIdx.x % THREADS;
    if (row < 0) return;
    const Row<T> z(static_cast<const T*>(a.z) + row * a.z_stride, a.vocab);
    const Row<T> dz(static_cast<T*>(a.dz) + row * a.dz_stride, a.vocab);
    const float coef = r.coef[row];
    if (coef == 0.0f) {
        zero_of(dz, 0, dz.vectors(), t, THREADS);
    } else {
        const uint32_t target = static_cast<uint32_t>(a.targets[row]);
        grad_of<T, THREADS>(z, dz, t, target, Elem<T>::load(z.element(target + z.head)), r.stat[row], a.c * kLog2e, coef);
    }
}

// ---- choices of a launch ------------------------------------------------------------------------------
// A warp to a row of up to 8 KB: both losses at 40000 x 3000 bf16 (6 KB) take 106 and 157 us, against 164
// (policy_slice_kernel) and 322 (256 threads); at 12 KB and 200 rows the warp takes 11.2 and 17.0 us,
// against 7.5 and 14.4.
constexpr int64_t kWarpRowBytes = 8192;
// Longer rows, fewer than two for each SM: 1024 threads each, so that there is enough under way (preference
// loss, 16 and 250 rows of 131072 bf16: 20.6 and 43 us, with 256 threads 27.7 and 55; 500 rows of 32768: 29.6
// against 22.3).
constexpr int kFewRows = 296;
// Else 128 threads up to 48 KB, so that a thread has a few rounds of vectors to a row, and 256 beyond
// (preference loss, 40000 x 8000 and x 20000 bf16: 373 and 779 us with 128, 471 and 838 with 256; 4000 x 32001:
// 147 against 140, 4000 x 65536: 271 against 258).
constexpr int64_t kSmallBlockRowBytes = 49152;
// Rows of a cluster in policy_slice_kernel, one after another (8192 x 131072 bf16, us: 1 row 738, 8 rows 714, 32 rows 749).
constexpr int kMostCount = 8;

template <typename F>
void pick_threads(int64_t rows, int64_t vocab, ss_dtype dt, F&& launch) {
    auto by_type = [&](auto t) {
        if (vocab * static_cast<int64_t>(sizeof(t)) <= kWarpRowBytes) launch(t, std::integral_constant<int, 32>{});
        else if (rows < kFewRows) launch(t, std::integral_constant<int, 1024>{});
        else if (vocab * static_cast<int64_t>(sizeof(t)) <= kSmallBlockRowBytes) launch(t, std::integral_constant<int, 128>{});
        else launch(t, std::integral_constant<int, 256>{});
    };
    if (dt == SS_F32) by_type(uint32_t{}); else by_type(uint16_t{});
}

template <int THREADS>
unsigned rows_grid(int64_t rows) {
    constexpr int per = block_of<THREADS>() / THREADS;
    return static_cast<unsigned>((rows + per - 1) / per);
}

// Blocks that share a row in policy_slice_kernel: the fewest that hold it, 0 if even 8 do not.
template <typename T, int HELD>
int cluster_of(int64_t vectors) {
    if (vectors > 8 * kSliceVectors<T, HELD>) return 0;
    int size = 1;
    while (vectors > size * kSliceVectors<T, HELD>) size *= 2;
    return size;
}

template <typename T, int HELD>
struct SliceKernel {};

template <typename T, int HELD>
cudaError_t launch_slices(const Logits& a, const Policy& p, int64_t rows, int64_t vectors, int size, int sms, cudaStream_t st) {
    constexpr int kSliceSmem = kSliceVectors<T, HELD> * 16 * kSliceSlots<T>;
    Slices c{rows, 1, static_cast<int>((vectors + size - 1) / size)};
    // As many rows to a cluster as leave three rounds of blocks for every SM (for one round, and for eight: 2053 x
    // 32001 fp32 100 and 92.5 us instead of 91, 4100 x 32001 bf16 108 and 113 instead of 112).
    const int64_t count = rows * size / (3 * kSliceBlocks<HELD> * sms);
    c.count = static_cast<int>(count < 1 ? 1 : (count > kMostCount ? kMostCount : count));
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>((rows + c.count - 1) / c.count * size));
    cfg.blockDim = dim3(kSliceThreads);
    cfg.dynamicSmemBytes = static_cast<size_t>(c.vectors) * 16 * kSliceSlots<T>;
    cfg.stream = st;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = size, at.val.clusterDim.y = 1, at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    const cudaError_t e = allow_shared<SliceKernel<T, HELD>>(reinterpret_cast<const void*>(policy_slice_kernel<T, HELD>), kSliceSmem);
    return e != cudaSuccess ? e : cudaLaunchKernelEx(&cfg, policy_slice_kernel<T, HELD>, a, p, c);
}

// Whether the rows were given to policy_slice_kernel.
template <typename T>
bool try_slices(const Logits& a, const Policy& p, const Mat& z, int sms, cudaStream_t st, cudaError_t* e) {
    const int64_t bytes = z.cols * static_cast<int64_t>(sizeof(T)), vectors = z.row_aligned(16) ? (bytes + 15) / 16 : (bytes + 30) / 16;
    if (bytes <= kWarpRowBytes) return false;
    if (const int size = cluster_of<T, 64>(vectors)) *e = launch_slices<T, 64>(a, p, z.rows, vectors, size, sms, st);
    else if (const int size = cluster_of<T, 128>(vectors)) *e = launch_slices<T, 128>(a, p, z.rows, vectors, size, sms, st);
    else return false;
    return true;
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
    return round_up(rows * 16, 256) + round_up(n_pairs * 4, 256);
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
        cudaError_t e;
        const int sms = device_sm_count(&e);
        if (e != cudaSuccess) return cuda_status_public(e);
        if (dlogits != nullptr && (dt == SS_F32 ? try_slices<uint32_t>(a, p, z, sms, st, &e) : try_slices<uint16_t>(a, p, z, sms, st, &e))) {
            if (e != cudaSuccess) return cuda_status_public(e);
        } else {
            pick_threads(rows, vocab, dt, [&](auto t, auto threads) {
                policy_stream_kernel<decltype(t), threads.value><<<rows_grid<threads.value>(rows), block_of<threads.value>(), 0, st>>>(a, p, rows);
            });
        }
    }
    const cudaError_t first = cudaGetLastError();
    if (first != cudaSuccess) return cuda_status_public(first);
    return cuda_status_public(launch_next(rows > 0, totals_kernel, 3, kSumThreads, st, p.terms, rows, totals));
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
    const Rows r{static_cast<Stat*>(workspace), static_cast<float*>(workspace) + 2 * rows, static_cast<float*>(workspace) + 3 * rows};
    float* pair_loss = reinterpret_cast<float*>(static_cast<char*>(workspace) + round_up(rows * 16, 256));
    const Preference p{seq_begin, ref_seq_logp, n_pairs, rows, kind, beta, label_smoothing, scale, margins, seq_logp, pair_loss};
    if (rows > 0) {
        pick_threads(rows, vocab, dt, [&](auto t, auto threads) {
            row_stat_kernel<decltype(t), threads.value><<<rows_grid<threads.value>(rows), block_of<threads.value>(), 0, st>>>(a, r, rows);
        });
    }
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess && n_pairs > 0) e = launch_next(rows > 0, pair_kernel, static_cast<unsigned>(n_pairs), kSumThreads, st, a, p, r);
    if (e != cudaSuccess) return cuda_status_public(e);
    const Total total{pair_loss, n_pairs, scale, loss};
    if (rows == 0 || dlogits == nullptr) {
        e = launch_next(rows > 0 || n_pairs > 0, total_kernel, 1, 32, st, total);
    } else {
        pick_threads(rows, vocab, dt, [&](auto t, auto threads) {
            e = launch_next(true, row_grad_kernel<decltype(t), threads.value>, rows_grid<threads.value>(rows), block_of<threads.value>(), st, a, r, rows, total);
        });
    }
    return cuda_status_public(e);
}

#pragma GCC visibility pop
}  // extern "C"
