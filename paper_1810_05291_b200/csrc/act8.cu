// Activations kept in 8 bits: packing, unpacking, and the (gated) activation's two passes.
#include "act8.cuh"

namespace ss {
namespace {

// f and f' in fp32.
//   silu: s = 1 / (1 + exp(-x)), f = x s, f' = s (1 + x (1 - s))
//   gelu: f = x Phi(x), f' = Phi(x) + x phi(x), Phi(x) = (1 + erf(x / sqrt 2)) / 2
template <int ACT>
__device__ __forceinline__ float act_value(float x) {
    if constexpr (ACT == SS_ACT_SILU) return x / (1.0f + expf(-x));
    else return x * (0.5f + 0.5f * erff(x * 0.70710678118654752f));
}

template <int ACT>
__device__ __forceinline__ void act_value_slope(float x, float* f, float* slope) {
    if constexpr (ACT == SS_ACT_SILU) {
        const float s = 1.0f / (1.0f + expf(-x));
        *f = x * s;
        *slope = s * (1.0f + x * (1.0f - s));
    } else {
        const float cdf = 0.5f + 0.5f * erff(x * 0.70710678118654752f);
        *f = x * cdf;
        *slope = cdf + x * 0.39894228040143268f * expf(-0.5f * x * x);
    }
}

// One lane holds one column of a group, a warp the group.
__device__ __forceinline__ void keep_lane(const Ckpt& c, int64_t row, int64_t group, int lane, float x) {
    const uint32_t a = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(x) & 0x7FFFFFFFu);
    const uint32_t e = act8_exp_byte(a);
    const int64_t g = row * c.groups + group;
    c.values[g * SS_ACT8_GROUP + lane] = static_cast<uint8_t>(act8_code(x, act8_inverse(e)));
    if (lane == 0) c.exps[g] = static_cast<uint8_t>(e);
}

__device__ __forceinline__ float kept_lane(const Ckpt& c, int64_t g, int lane) {
    return act8_value(c.values[g * SS_ACT8_GROUP + lane], act8_unit(c.exps[g]));
}

// ---- one warp per group, one lane per column: any stride, any alignment -----------------------------
template <typename T>
__global__ void __launch_bounds__(256) act8_pack_kernel(const T* x, int64_t stride, int64_t rows, int64_t cols, Ckpt c) {
    const int lane = threadIdx.x & 31;
    const int64_t total = rows * c.groups, step = (static_cast<int64_t>(gridDim.x) * blockDim.x) >> 5;
    for (int64_t g = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) >> 5; g < total; g += step) {
        const int64_t row = g / c.groups, group = g - row * c.groups, col = group * SS_ACT8_GROUP + lane;
        const float v = col < cols ? Elem<T>::load(x + row * stride + col) : 0.0f;
        keep_lane(c, row, group, lane, v);
    }
}

template <typename T>
__global__ void __launch_bounds__(256) act8_unpack_kernel(Ckpt c, int64_t rows, int64_t cols, T* out, int64_t stride) {
    const int lane = threadIdx.x & 31;
    const int64_t total = rows * c.groups, step = (static_cast<int64_t>(gridDim.x) * blockDim.x) >> 5;
    for (int64_t g = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) >> 5; g < total; g += step) {
        const int64_t row = g / c.groups, col = (g - row * c.groups) * SS_ACT8_GROUP + lane;
        if (col < cols) Elem<T>::store(out + row * stride + col, kept_lane(c, g, lane));
    }
}

struct Forward {
    const void *x, *up;
    void* y;
    int64_t x_stride, up_stride, y_stride, rows, cols;
    Ckpt cx, cu, cy;
};

template <typename T, int ACT>
__global__ void __launch_bounds__(256) act8_forward_kernel(const __grid_constant__ Forward a) {
    const int lane = threadIdx.x & 31;
    const int64_t total = a.rows * a.cx.groups, step = (static_cast<int64_t>(gridDim.x) * blockDim.x) >> 5;
    const T* x = static_cast<const T*>(a.x);
    const T* up = static_cast<const T*>(a.up);
    T* y = static_cast<T*>(a.y);
    for (int64_t g = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) >> 5; g < total; g += step) {
        const int64_t row = g / a.cx.groups, group = g - row * a.cx.groups, col = group * SS_ACT8_GROUP + lane;
        const bool in = col < a.cols;
        const float v = in ? Elem<T>::load(x + row * a.x_stride + col) : 0.0f;
        float f = act_value<ACT>(v);
        keep_lane(a.cx, row, group, lane, v);
        if (up != nullptr) {
            const float u = in ? Elem<T>::load(up + row * a.up_stride + col) : 0.0f;
            f *= u;
            keep_lane(a.cu, row, group, lane, u);
        }
        if (a.cy.values != nullptr) {
            T stored;  // the checkpoint is of what the next layer reads
            Elem<T>::store(&stored, f);
            keep_lane(a.cy, row, group, lane, in ? Elem<T>::load(&stored) : 0.0f);
        }
        if (in) Elem<T>::store(y + row * a.y_stride + col, f);
    }
}

struct Backward {
    const void* dy;
    void *dx, *dup;
    int64_t dy_stride, dx_stride, dup_stride, rows, cols;
    Ckpt cx, cu;
};

template <typename T, int ACT>
__global__ void __launch_bounds__(256) act8_backward_kernel(const __grid_constant__ Backward a) {
    const int lane = threadIdx.x & 31;
    const int64_t total = a.rows * a.cx.groups, step = (static_cast<int64_t>(gridDim.x) * blockDim.x) >> 5;
    for (int64_t g = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) >> 5; g < total; g += step) {
        const int64_t row = g / a.cx.groups, col = (g - row * a.cx.groups) * SS_ACT8_GROUP + lane;
        if (col >= a.cols) continue;
        const float dy = Elem<T>::load(static_cast<const T*>(a.dy) + row * a.dy_stride + col);
        float f, slope;
        act_value_slope<ACT>(kept_lane(a.cx, g, lane), &f, &slope);
        float dx = dy * slope;
        if (a.dup != nullptr) {
            dx = dy * kept_lane(a.cu, g, lane) * slope;
            Elem<T>::store(static_cast<T*>(a.dup) + row * a.dup_stride + col, dy * f);
        }
        Elem<T>::store(static_cast<T*>(a.dx) + row * a.dx_stride + col, dx);
    }
}

// Grid of a kernel that strides over `warps` items, one to a warp of a 256-thread block.
cudaError_t warp_grid(int64_t warps, int* grid) {
    cudaError_t err = cudaSuccess;
    const int64_t sms = device_sm_count(&err);
    int64_t blocks = (warps + 7) / 8;
    if (blocks > sms * 8) blocks = sms * 8;
    *grid = static_cast<int>(blocks < 1 ? 1 : blocks);
    return err;
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
    int grid = 1;
    const cudaError_t e = warp_grid(rows * c.groups, &grid);
    if (e != cudaSuccess) return cuda_status_public(e);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (dt == SS_F32) act8_pack_kernel<float><<<grid, 256, 0, st>>>(static_cast<const float*>(x), mx.stride, rows, cols, c);
    else act8_pack_kernel<uint16_t><<<grid, 256, 0, st>>>(static_cast<const uint16_t*>(x), mx.stride, rows, cols, c);
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
    int grid = 1;
    const cudaError_t e = warp_grid(rows * c.groups, &grid);
    if (e != cudaSuccess) return cuda_status_public(e);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (dt == SS_F32) act8_unpack_kernel<float><<<grid, 256, 0, st>>>(c, rows, cols, static_cast<float*>(out), mo.stride);
    else act8_unpack_kernel<uint16_t><<<grid, 256, 0, st>>>(c, rows, cols, static_cast<uint16_t*>(out), mo.stride);
    return cuda_status_public(cudaGetLastError());
}

int ss_act8_forward(const void* x, int64_t x_stride, const void* up, int64_t up_stride, ss_dtype dt, ss_act act,
                    int64_t rows, int64_t cols, void* y, int64_t y_stride, uint8_t* ckpt_x, uint8_t* ckpt_up,
                    uint8_t* ckpt_y, void* cuda_stream) {
    if (!dtype_known(dt) || (act != SS_ACT_GELU && act != SS_ACT_SILU) || !sides_ok(rows, cols)) return SS_ERR_INVALID_ARG;
    if (!stride_ok(rows, cols, x_stride) || !stride_ok(rows, cols, y_stride)) return SS_ERR_INVALID_ARG;
    if ((up != nullptr) != (ckpt_up != nullptr) || (up != nullptr && !stride_ok(rows, cols, up_stride))) return SS_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return SS_OK;
    const size_t eb = dtype_bytes(dt), kept = ss_act8_bytes(rows, cols);
    const Mat mx = mat(x, rows, cols, x_stride, eb), my = mat(y, rows, cols, y_stride, eb);
    const Mat mu = mat(up, rows, cols, up_stride, eb);
    SS_TRY(mat_check(mx, x_stride));
    SS_TRY(mat_check(my, y_stride));
    if (up != nullptr) SS_TRY(mat_check(mu, up_stride));
    SS_TRY(ckpt_check(ckpt_x));
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
    const Forward a{x, up, y, mx.stride, mu.stride, my.stride, rows, cols, ckpt_of(ckpt_x, rows, cols),
                    ckpt_of(ckpt_up, rows, cols), ckpt_of(ckpt_y, rows, cols)};
    int grid = 1;
    const cudaError_t e = warp_grid(rows * a.cx.groups, &grid);
    if (e != cudaSuccess) return cuda_status_public(e);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (dt == SS_F32) {
        if (act == SS_ACT_GELU) act8_forward_kernel<float, SS_ACT_GELU><<<grid, 256, 0, st>>>(a);
        else act8_forward_kernel<float, SS_ACT_SILU><<<grid, 256, 0, st>>>(a);
    } else {
        if (act == SS_ACT_GELU) act8_forward_kernel<uint16_t, SS_ACT_GELU><<<grid, 256, 0, st>>>(a);
        else act8_forward_kernel<uint16_t, SS_ACT_SILU><<<grid, 256, 0, st>>>(a);
    }
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
    const Backward a{dy, dx, dup, my.stride, mx.stride, mu.stride, rows, cols,
                     ckpt_of(const_cast<uint8_t*>(ckpt_x), rows, cols), ckpt_of(const_cast<uint8_t*>(ckpt_up), rows, cols)};
    int grid = 1;
    const cudaError_t e = warp_grid(rows * a.cx.groups, &grid);
    if (e != cudaSuccess) return cuda_status_public(e);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (dt == SS_F32) {
        if (act == SS_ACT_GELU) act8_backward_kernel<float, SS_ACT_GELU><<<grid, 256, 0, st>>>(a);
        else act8_backward_kernel<float, SS_ACT_SILU><<<grid, 256, 0, st>>>(a);
    } else {
        if (act == SS_ACT_GELU) act8_backward_kernel<uint16_t, SS_ACT_GELU><<<grid, 256, 0, st>>>(a);
        else act8_backward_kernel<uint16_t, SS_ACT_SILU><<<grid, 256, 0, st>>>(a);
    }
    return cuda_status_public(cudaGetLastError());
}

#pragma GCC visibility pop
}  // extern "C"
