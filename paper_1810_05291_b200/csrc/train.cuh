// Shared by the training operators (losses over logits, activations kept in 8 bits): checks of
// strided matrices, loads and stores of the two element types.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/signsgd_train.h"
#include "common.cuh"

namespace ss {

int cuda_status_public(cudaError_t e);  // abi.cu

constexpr int64_t kMaxSide = 0x7FFFFFFF;

inline bool addr_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline size_t dtype_bytes(ss_dtype dt) { return dt == SS_F32 ? 4 : 2; }

inline bool dtype_known(ss_dtype dt) { return dt == SS_F32 || dt == SS_BF16; }

// A matrix of a call: what a check needs to know of it.
struct Mat {
    const void* p;
    int64_t rows, cols, stride;  // elements
    size_t eb;

    size_t extent() const {  // bytes from the first element to the end of the last
        return rows == 0 || cols == 0 ? 0 : (static_cast<size_t>(rows - 1) * stride + cols) * eb;
    }
    bool row_aligned(size_t a) const { return addr_aligned(p, a) && (rows < 2 || (stride * eb) % a == 0); }
};

inline bool sides_ok(int64_t rows, int64_t cols) { return rows >= 0 && cols >= 0 && rows <= kMaxSide && cols <= kMaxSide; }

inline bool stride_ok(int64_t rows, int64_t cols, int64_t stride) {
    if (rows < 2) return true;
    return stride >= cols && stride <= SS_MAX_COORDS / rows;
}

// A stride that means nothing (fewer than two rows) is replaced, so that no product with it can wrap.
inline Mat mat(const void* p, int64_t rows, int64_t cols, int64_t stride, size_t eb) {
    return Mat{p, rows, cols, rows < 2 ? cols : stride, eb};
}

inline bool bytes_overlap(const void* p, size_t n, const void* q, size_t m) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return n != 0 && m != 0 && a < b + m && b < a + n;
}

// Whether two matrices share an element. Two of the same stride may interleave (columns of one
// wider matrix); for other strides the whole extents are compared.
inline bool mats_overlap(const Mat& a, const Mat& b) {
    if (!bytes_overlap(a.p, a.extent(), b.p, b.extent())) return false;
    const size_t sa = a.stride * a.eb, sb = b.stride * b.eb;
    if (sa != sb || (a.rows < 2 && b.rows < 2)) return true;
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
    const size_t ahead = (pb >= pa ? (pb - pa) % sa : (sa - (pa - pb) % sa) % sa);  // b's columns start this far into a's rows
    return ahead < a.cols * a.eb || sa - ahead < b.cols * b.eb;
}

inline bool mat_overlaps(const Mat& a, const void* p, size_t n) { return bytes_overlap(a.p, a.extent(), p, n); }

// An output that is an input in place: the same elements at the same places.
inline bool same_mat(const Mat& a, const Mat& b) {
    return a.p == b.p && a.rows == b.rows && a.cols == b.cols && a.stride == b.stride && a.eb == b.eb;
}

// Lets a kernel have `bytes` of dynamic shared memory on the current device: asked of the runtime once
// for each kernel (KEY: a type of its own) and device, and again only for more.
template <typename KEY>
cudaError_t allow_shared(const void* kernel, int bytes) {
    static std::atomic<int> allowed[64];
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const bool known = device < 64;
    if (known && allowed[device].load(std::memory_order_relaxed) >= bytes) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && known) allowed[device].store(bytes, std::memory_order_relaxed);
    return e;
}

// ---- kernels of one call that follow one another ---------------------------------------------------
// A kernel that another of the same call follows says so at its start; the other is launched with
// launch_next and begins with after_previous(), before it touches any memory. So its blocks are set up
// while the first kernel's last ones run, but it neither reads nor writes before the first has ended
// and its stores are seen. (`follows` is false where the call has launched nothing yet: such a kernel
// begins when all that the stream held before has ended, like any other.)
__device__ __forceinline__ void next_may_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename... P, typename... A>
cudaError_t launch_next(bool follows, void (*kernel)(P...), dim3 grid, dim3 block, cudaStream_t st, const A&... args) {
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid, cfg.blockDim = block, cfg.stream = st;
    cfg.attrs = &at, cfg.numAttrs = follows ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// ---- the two element types -------------------------------------------------------------------------
template <typename T>
struct Elem;  // T: float, or uint16_t for the bits of a bf16

template <>
struct Elem<float> {
    static __device__ __forceinline__ float load(const float* p) { return *p; }
    static __device__ __forceinline__ void store(float* p, float v) { *p = v; }
};

// Round to nearest even.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <>
struct Elem<uint16_t> {
    static __device__ __forceinline__ float load(const uint16_t* p) { return __uint_as_float(static_cast<uint32_t>(*p) << 16); }
    static __device__ __forceinline__ void store(uint16_t* p, float v) { *p = static_cast<uint16_t>(bf16_pair(v, 0.0f)); }
};

}  // namespace ss
