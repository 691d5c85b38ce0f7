// Losses over a language model's logits, with their gradient: the clipped policy loss and the
// paired preference loss.
#include <cmath>

#include "train.cuh"

namespace ss {
namespace {

constexpr int kRowThreads = 256;
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

__device__ __forceinline__ Stat block_join(Stat v, Stat* shared, float k) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = join(v, Stat{__shfl_xor_sync(0xFFFFFFFFu, v.m, o), __shfl_xor_sync(0xFFFFFFFFu, v.s, o)}, k);
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = shared[0];
    for (int w = 1; w < kRowThreads / 32; ++w) v = join(v, shared[w], k);
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

template <typename T>
__device__ __forceinline__ Stat row_stat(const T* z, int64_t vocab, float k) {
    Stat v{-INFINITY, 0.0f};
    for (int64_t i = threadIdx.x; i < vocab; i += kRowThreads) {
        const float x = Elem<T>::load(z + i);
        if (x > v.m) {
            v.s *= exp2_fast((v.m - x) * k);
            v.m = x;
        }
        v.s += x == -INFINITY ? 0.0f : exp2_fast((x - v.m) * k);
    }
    return v;
}

// dz = coef c ([v = y] - softmax_v)
template <typename T>
__device__ __forceinline__ void row_grad(const T* z, T* dz, int64_t vocab, int64_t target, float k, const Stat& v, float coef) {
    const float f = -coef / v.s;
    for (int64_t i = threadIdx.x; i < vocab; i += kRowThreads) {
        const float p = f * exp2_fast((Elem<T>::load(z + i) - v.m) * k);
        Elem<T>::store(dz + i, i == target ? coef + p : p);
    }
}

template <typename T>
__device__ __forceinline__ void row_zero(T* dz, int64_t vocab) {
    for (int64_t i = threadIdx.x; i < vocab; i += kRowThreads) dz[i] = T(0);
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

template <typename T>
__global__ void __launch_bounds__(kRowThreads) policy_row_kernel(const __grid_constant__ Logits a, const __grid_constant__ Policy p, int64_t rows) {
    __shared__ Stat shared[kRowThreads / 32];
    const int64_t row = blockIdx.x;
    const T* z = static_cast<const T*>(a.z) + row * a.z_stride;
    T* dz = a.dz == nullptr ? nullptr : static_cast<T*>(a.dz) + row * a.dz_stride;
    int64_t target;
    float w;
    if (!row_live(a, row, &target, &w)) {
        if (dz != nullptr) row_zero(dz, a.vocab);
        if (threadIdx.x == 0) {
            a.logp[row] = 0.0f;
            for (int i = 0; i < 3; ++i) p.terms[i * rows + row] = 0.0f;
        }
        return;
    }
    const float k = a.c * kLog2e, picked = Elem<T>::load(z + target);
    const Stat v = block_join(row_stat(z, a.vocab, k), shared, k);
    const float logp = (picked - v.m) * a.c - logf(v.s);
    const PolicyTerm t = policy_term(p, row, logp, w);
    if (dz != nullptr) row_grad(z, dz, a.vocab, target, k, v, t.slope * a.c * (a.grad_scale == nullptr ? 1.0f : *a.grad_scale));
    if (threadIdx.x == 0) {
        a.logp[row] = logp;
        p.terms[row] = t.loss, p.terms[rows + row] = t.kl, p.terms[2 * rows + row] = t.clipped;
    }
}

// Sum over a block of 256 threads in a fixed order.
__device__ __forceinline__ double block_sum(double v, double* shared) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < kRowThreads / 32; ++w) v += shared[w];
    return v;
}

__global__ void __launch_bounds__(kRowThreads) totals_kernel(const float* terms, int64_t n, double scale, float* out) {
    __shared__ double shared[kRowThreads / 32];
    const float* x = terms + blockIdx.x * n;
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += kRowThreads) v += x[i];
    v = block_sum(v, shared);
    if (threadIdx.x == 0) out[blockIdx.x] = static_cast<float>(scale * v);
}

// ---- preference loss: statistics of every row, then every pair's coefficient, then the gradient -----
struct Rows {
    Stat* stat;
    float* coef;
};

template <typename T>
__global__ void __launch_bounds__(kRowThreads) row_stat_kernel(const __grid_constant__ Logits a, Rows r) {
    __shared__ Stat shared[kRowThreads / 32];
    const int64_t row = blockIdx.x;
    const T* z = static_cast<const T*>(a.z) + row * a.z_stride;
    int64_t target;
    float w;
    const bool live = row_live(a, row, &target, &w);
    Stat v{0.0f, 1.0f};
    float logp = 0.0f;
    if (live) {
        const float k = a.c * kLog2e, picked = Elem<T>::load(z + target);
        v = block_join(row_stat(z, a.vocab, k), shared, k);
        logp = (picked - v.m) * a.c - logf(v.s);
    }
    if (threadIdx.x == 0) {
        a.logp[row] = logp;
        r.stat[row] = v;
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

__global__ void __launch_bounds__(kRowThreads) pair_kernel(const __grid_constant__ Logits a, const __grid_constant__ Preference p, Rows r) {
    __shared__ double shared[kRowThreads / 32];
    const int64_t pair = blockIdx.x;
    int64_t at[3];
    for (int i = 0; i < 3; ++i) {
        const int64_t b = p.begin[2 * pair + i];
        at[i] = b < 0 ? 0 : (b > p.rows ? p.rows : b);
    }
    double sum[2];
    for (int i = 0; i < 2; ++i) {
        double v = 0.0;
        for (int64_t t = at[i] + threadIdx.x; t < at[i + 1]; t += kRowThreads) {
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
        for (int64_t t = at[i] + threadIdx.x; t < at[i + 1]; t += kRowThreads) {
            int64_t target;
            float w;
            if (row_live(a, t, &target, &w)) r.coef[t] = (i == 0 ? slope : -slope) * w * a.c;
        }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) row_grad_kernel(const __grid_constant__ Logits a, Rows r) {
    const int64_t row = blockIdx.x;
    T* dz = static_cast<T*>(a.dz) + row * a.dz_stride;
    const float coef = r.coef[row];
    if (coef == 0.0f) {
        row_zero(dz, a.vocab);
        return;
    }
    row_grad(static_cast<const T*>(a.z) + row * a.z_stride, dz, a.vocab, a.targets[row], a.c * kLog2e, r.stat[row], coef);
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
        if (dt == SS_F32) policy_row_kernel<float><<<static_cast<unsigned>(rows), kRowThreads, 0, st>>>(a, p, rows);
        else policy_row_kernel<uint16_t><<<static_cast<unsigned>(rows), kRowThreads, 0, st>>>(a, p, rows);
    }
    totals_kernel<<<3, kRowThreads, 0, st>>>(p.terms, rows, 1.0, totals);
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
    const unsigned grid = static_cast<unsigned>(rows);
    if (rows > 0) {
        if (dt == SS_F32) row_stat_kernel<float><<<grid, kRowThreads, 0, st>>>(a, r);
        else row_stat_kernel<uint16_t><<<grid, kRowThreads, 0, st>>>(a, r);
    }
    if (n_pairs > 0) pair_kernel<<<static_cast<unsigned>(n_pairs), kRowThreads, 0, st>>>(a, p, r);
    totals_kernel<<<1, kRowThreads, 0, st>>>(pair_loss, n_pairs, scale, loss);
    if (rows > 0 && dlogits != nullptr) {
        if (dt == SS_F32) row_grad_kernel<float><<<grid, kRowThreads, 0, st>>>(a, r);
        else row_grad_kernel<uint16_t><<<grid, kRowThreads, 0, st>>>(a, r);
    }
    return cuda_status_public(cudaGetLastError());
}

#pragma GCC visibility pop
}  // extern "C"
