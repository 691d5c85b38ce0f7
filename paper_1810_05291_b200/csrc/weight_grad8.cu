// Weight gradient of a linear layer from its input kept in 8 bits: dW[n, k] (+)= sum_t dY[t, n] x^[t, k].
#include "act8.cuh"

namespace ss {
namespace {

struct WeightGrad {
    const void* dy;
    Ckpt x;
    float* dw;
    int64_t dy_stride, dw_stride, rows, n_out, n_in;
    int accumulate;
};

// Rows summed before a partial sum is added to the whole: a sum of 16384 rows one after the other
// would be off by a few 1e-6 of its size, in chunks of 512 by a few 1e-7.
constexpr int64_t kChunkRows = 512;

// A block forms a 64 x 64 tile of dW in fp32 from slices of 16 rows staged in shared memory, a
// thread 4 x 4 of it.
template <typename T>
__global__ void __launch_bounds__(256) weight_grad8_kernel(const __grid_constant__ WeightGrad a) {
    __shared__ float s_dy[16][64], s_x[16][64];
    const int tid = threadIdx.x, tn = (tid >> 4) * 4, tk = (tid & 15) * 4;
    const int64_t n0 = static_cast<int64_t>(blockIdx.y) * 64, k0 = static_cast<int64_t>(blockIdx.x) * 64;
    const T* dy = static_cast<const T*>(a.dy);
    float acc[4][4] = {}, whole[4][4] = {};
    for (int64_t t0 = 0; t0 < a.rows; t0 += 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (tid >> 6) + 4 * i, c = tid & 63;
            const int64_t t = t0 + r, n = n0 + c, k = k0 + c;
            s_dy[r][c] = t < a.rows && n < a.n_out ? Elem<T>::load(dy + t * a.dy_stride + n) : 0.0f;
            float v = 0.0f;
            if (t < a.rows && k < a.n_in) {
                const int64_t g = t * a.x.groups + k / SS_ACT8_GROUP;
                v = act8_value(a.x.values[t * a.x.groups * SS_ACT8_GROUP + k], act8_unit(a.x.exps[g]));
            }
            s_x[r][c] = v;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(s_dy[r][tn + i], s_x[r][tk + j], acc[i][j]);
        __syncthreads();
        if ((t0 + 16) % kChunkRows == 0 || t0 + 16 >= a.rows) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) whole[i][j] += acc[i][j], acc[i][j] = 0.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t n = n0 + tn + i, k = k0 + tk + j;
            if (n < a.n_out && k < a.n_in) {
                float* p = a.dw + n * a.dw_stride + k;
                *p = a.accumulate ? *p + whole[i][j] : whole[i][j];
            }
        }
}

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" {
#pragma GCC visibility push(default)

int64_t ss_weight_grad8_workspace(const void*, int64_t, ss_dtype dt, int64_t rows, int64_t n_out, int64_t n_in) {
    if (!dtype_known(dt) || !sides_ok(rows, n_out) || !sides_ok(rows, n_in)) return -1;
    return 0;
}

int ss_weight_grad8(const void* dy, int64_t dy_stride, ss_dtype dt, const uint8_t* ckpt_x, int64_t rows,
                    int64_t n_out, int64_t n_in, float* dw, int64_t dw_stride, int accumulate, void* workspace,
                    int64_t workspace_bytes, void* cuda_stream) {
    if (!dtype_known(dt) || !sides_ok(rows, n_out) || !sides_ok(rows, n_in)) return SS_ERR_INVALID_ARG;
    if (!stride_ok(rows, n_out, dy_stride) || !stride_ok(n_out, n_in, dw_stride)) return SS_ERR_INVALID_ARG;
    if (n_out == 0 || n_in == 0) return SS_OK;
    const size_t eb = dtype_bytes(dt);
    const Mat mw = mat(dw, n_out, n_in, dw_stride, 4), my = mat(dy, rows, n_out, dy_stride, eb);
    if (dw == nullptr || (rows > 0 && (dy == nullptr || ckpt_x == nullptr))) return SS_ERR_INVALID_ARG;
    if (!addr_aligned(dw, 4)) return SS_ERR_MISALIGNED;
    if (rows > 0) {
        if (!addr_aligned(dy, eb) || !addr_aligned(ckpt_x, 16)) return SS_ERR_MISALIGNED;
        const size_t kept = ss_act8_bytes(rows, n_in);
        if (mats_overlap(mw, my) || mat_overlaps(mw, ckpt_x, kept)) return SS_ERR_INVALID_ARG;
    }
    const int64_t need = ss_weight_grad8_workspace(dy, dy_stride, dt, rows, n_out, n_in);
    if (workspace_bytes < need || (need > 0 && workspace == nullptr)) return SS_ERR_INVALID_ARG;
    const WeightGrad a{dy, ckpt_of(const_cast<uint8_t*>(ckpt_x), rows, n_in), dw, my.stride, mw.stride, rows, n_out, n_in, accumulate};
    const dim3 grid(static_cast<unsigned>((n_in + 63) / 64), static_cast<unsigned>((n_out + 63) / 64));
    if (grid.y > 65535u) return SS_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (dt == SS_F32) weight_grad8_kernel<float><<<grid, 256, 0, st>>>(a);
    else weight_grad8_kernel<uint16_t><<<grid, 256, 0, st>>>(a);
    return cuda_status_public(cudaGetLastError());
}

#pragma GCC visibility pop
}  // extern "C"
