// Residual addition + root-mean-square norm + e4m3 quantisation in one pass, and quantisation alone.
//
// Norm: u = v / sqrt(mean v^2 + eps) * gamma needs the whole row before its first output, so a CTA keeps its row in
// registers (each thread CH chunks of 8 consecutive elements) and global memory sees every element once in and once out.
// Sixteen lanes hold one 128-column block: its largest magnitude is four shuffles away, and no shared memory is used but
// for the row's sum.  Bound: memory bytes for many rows, launch and one trip to memory and back for a few.
#include "fp8.cuh"

namespace monde {

namespace {

struct NormParams {
    int T, d;
    float eps;
    const void* x;
    const void* residual;
    const void* gamma;
    void* residual_out;
    void* y;
    uint8_t* q;
    float* scale;
    int64_t ld_x, ld_residual, ld_residual_out, ld_y, ld_q, ld_scale;
};

__device__ __forceinline__ float half_warp_max(float m) {      // over the 16 lanes that hold one block
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}

template <typename T, int CH, bool kVec>
__global__ void __launch_bounds__(1024) rmsnorm_quant_kernel(const NormParams P) {
    __shared__ float warp_sum[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t row = blockIdx.x;
    pdl_launch_dependents();
    pdl_wait();
    const T* x = static_cast<const T*>(P.x) + row * P.ld_x;
    const T* res = P.residual != nullptr ? static_cast<const T*>(P.residual) + row * P.ld_residual : nullptr;
    const T* gamma = static_cast<const T*>(P.gamma);
    float v[CH][8];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = (i * blockDim.x + tid) * 8;
        if (c < P.d) {
            load8<T, kVec>(x + c, P.d - c, v[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
        }
    }
    if (res != nullptr) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = (i * blockDim.x + tid) * 8;
            if (c >= P.d) continue;
            float r[8];
            load8<T, kVec>(res + c, P.d - c, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] += r[j];
        }
    }
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fmaf(v[i][j], v[i][j], sum);
    if (P.residual_out != nullptr) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = (i * blockDim.x + tid) * 8;
            if (c < P.d) store8<T, kVec>(static_cast<T*>(P.residual_out) + row * P.ld_residual_out + c, P.d - c, v[i]);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (blockDim.x > 32) {
        if (lane == 0) warp_sum[warp] = sum;
        __syncthreads();
        sum = lane < static_cast<int>(blockDim.x >> 5) ? warp_sum[lane] : 0.0f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    }
    const float rms = __frsqrt_rn(__fdiv_rn(sum, static_cast<float>(P.d)) + P.eps);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = (i * blockDim.x + tid) * 8;
        const bool in = c < P.d;
        float amax = 0.0f;
        if (in) {
            float g[8];
            if (gamma != nullptr) load8<T, kVec>(gamma + c, P.d - c, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[i][j] *= rms;
                if (gamma != nullptr) v[i][j] *= g[j];
                if (kVec || j < P.d - c) amax = max_nan(amax, fabsf(v[i][j]));
            }
            if (P.y != nullptr) store8<T, kVec>(static_cast<T*>(P.y) + row * P.ld_y + c, P.d - c, v[i]);
        }
        if (P.q != nullptr) {
            amax = half_warp_max(amax);
            const float s = block_scale(amax);
            if (in) {
                store8_e4m3<kVec>(P.q + row * P.ld_q + c, P.d - c, v[i], __fdiv_rn(1.0f, s));
                if ((lane & 15) == 0) P.scale[row * P.ld_scale + c / kFp8Block] = s;
            }
        }
    }
}

// ---- quantisation alone -----------------------------------------------------------------------
struct QuantParams {
    int64_t rows;               // all rows of the batch
    int rows_each, cols, blocks;    // rows of one matrix, columns, 128-column blocks of a row
    const void* x;
    uint8_t* q;
    float* scale;
    int64_t ld_x, ld_q, ld_scale;
};

// One row block: 16 lanes, 8 elements each.
template <typename T, bool kVec>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const QuantParams P) {
    const int lane = threadIdx.x & 15;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t total = P.rows * P.blocks;
    const int64_t groups = static_cast<int64_t>(gridDim.x) * (blockDim.x / 16);
    const int64_t first = static_cast<int64_t>(blockIdx.x) * (blockDim.x / 16) + threadIdx.x / 16;
    // every thread runs every round (the shuffles take whole warps); groups past the end do nothing in them
    for (int64_t b0 = 0; b0 < total; b0 += groups) {
        const int64_t b = b0 + first;
        const int64_t row = b / P.blocks;
        const int c = static_cast<int>(b - row * P.blocks) * kFp8Block + lane * 8;
        const bool in = b < total && c < P.cols;
        float v[8] = {};
        if (in) load8<T, kVec>(static_cast<const T*>(P.x) + row * P.ld_x + c, P.cols - c, v);
        float amax = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) amax = max_nan(amax, fabsf(v[j]));
        const float s = block_scale(half_warp_max(amax));
        if (in) {
            store8_e4m3<kVec>(P.q + row * P.ld_q + c, P.cols - c, v, __fdiv_rn(1.0f, s));
            if (lane == 0) P.scale[row * P.ld_scale + c / kFp8Block] = s;
        }
    }
}

// One 128 x 128 block per CTA of 256 threads: each holds 8 chunks of 8 elements, rows r, r + 16, ...
template <typename T, bool kVec>
__global__ void __launch_bounds__(256) quantize_blocks_kernel(const QuantParams P) {
    __shared__ float warp_max[8];
    const int tid = threadIdx.x;
    pdl_launch_dependents();
    pdl_wait();
    const int row_blocks = (P.rows_each + kFp8Block - 1) / kFp8Block;
    const int64_t tile = blockIdx.x;
    const int64_t rb = tile / P.blocks;                       // row block over the whole batch
    const int cb = static_cast<int>(tile - rb * P.blocks);
    const int64_t batch = rb / row_blocks;
    const int r0 = static_cast<int>(rb - batch * row_blocks) * kFp8Block;
    const int c = cb * kFp8Block + (tid & 15) * 8;
    float v[8][8];
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + (tid >> 4) + 16 * i;
        if (r < P.rows_each && c < P.cols) {
            load8<T, kVec>(static_cast<const T*>(P.x) + (batch * P.rows_each + r) * P.ld_x + c, P.cols - c, v[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) amax = max_nan(amax, fabsf(v[i][j]));
    amax = half_warp_max(amax);
    amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, 16));
    if ((tid & 31) == 0) warp_max[tid >> 5] = amax;
    __syncthreads();
    amax = warp_max[0];
#pragma unroll
    for (int w = 1; w < 8; ++w) amax = max_nan(amax, warp_max[w]);
    const float s = block_scale(amax), inv = __fdiv_rn(1.0f, s);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + (tid >> 4) + 16 * i;
        if (r < P.rows_each && c < P.cols)
            store8_e4m3<kVec>(P.q + (batch * P.rows_each + r) * P.ld_q + c, P.cols - c, v[i], inv);
    }
    if (tid == 0) P.scale[rb * P.ld_scale + cb] = s;
}

bool multiple_of(const void* p, int64_t ld_bytes, unsigned m) {     // null is fine: not accessed
    return p == nullptr || ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld_bytes)) & (m - 1)) == 0;
}
bool multiple_of(const void* p, unsigned m) { return multiple_of(p, 0, m); }

template <typename T, int CH, bool kVec>
cudaError_t launch_norm(const NormParams& P, int threads, cudaStream_t s) {
    return launch_pdl(rmsnorm_quant_kernel<T, CH, kVec>, dim3(P.T), dim3(threads), 0, s, P);
}
template <typename T, bool kVec>
cudaError_t launch_norm(const NormParams& P, cudaStream_t s) {
    const int chunks = (P.d + 7) / 8;
    const auto threads = [&](int ch) { return ((chunks + ch - 1) / ch + 31) / 32 * 32; };
    if (chunks <= 256) return launch_norm<T, 1, kVec>(P, threads(1), s);
    if (chunks <= 1024) return launch_norm<T, 2, kVec>(P, threads(2), s);
    return launch_norm<T, 4, kVec>(P, threads(4), s);
}

}  // namespace

}  // namespace monde

using namespace monde;

extern "C" {

int monde_rmsnorm_quant(int32_t dtype, int32_t T, int32_t d, float eps, const void* x, int64_t ld_x,
                        const void* residual, int64_t ld_residual, const void* gamma, void* residual_out,
                        int64_t ld_residual_out, void* y, int64_t ld_y, void* q, int64_t ld_q, float* scale,
                        int64_t ld_scale, void* stream) {
    if (T < 0 || d <= 0 || !(eps >= 0.0f) || isinf(eps)) return MONDE_ERR_INVALID_ARG;
    if (dtype != MONDE_F32 && dtype != MONDE_BF16) return MONDE_ERR_UNSUPPORTED;
    if (d > 32768) return MONDE_ERR_UNSUPPORTED;
    const int blocks = (d + kFp8Block - 1) / kFp8Block;
    if (ld_x < d || (residual && ld_residual < d) || (residual_out && ld_residual_out < d) || (y && ld_y < d) ||
        (q && (ld_q < d || ld_scale < blocks)))
        return MONDE_ERR_INVALID_ARG;
    if (T == 0) return MONDE_OK;
    if (!x || (q == nullptr) != (scale == nullptr) || (!residual_out && !y && !q)) return MONDE_ERR_INVALID_ARG;
    const int b = static_cast<int>(elem_bytes(dtype));
    if (!multiple_of(x, b) || !multiple_of(residual, b) || !multiple_of(gamma, b) || !multiple_of(residual_out, b) ||
        !multiple_of(y, b) || !multiple_of(scale, 4))
        return MONDE_ERR_INVALID_ARG;
    const int st = check_arch();
    if (st != MONDE_OK) return st;
    const NormParams P = {T, d, eps, x, residual, gamma, residual_out, y, static_cast<uint8_t*>(q), scale,
                          ld_x, ld_residual, ld_residual_out, ld_y, ld_q, ld_scale};
    const bool vec = d % 8 == 0 && multiple_of(x, ld_x * b, 16) && multiple_of(residual, ld_residual * b, 16) &&
                     multiple_of(gamma, 16) && multiple_of(residual_out, ld_residual_out * b, 16) &&
                     multiple_of(y, ld_y * b, 16) && multiple_of(q, ld_q, 8);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (dtype == MONDE_BF16)
        e = vec ? launch_norm<__nv_bfloat16, true>(P, s) : launch_norm<__nv_bfloat16, false>(P, s);
    else
        e = vec ? launch_norm<float, true>(P, s) : launch_norm<float, false>(P, s);
    if (e != cudaSuccess) return MONDE_ERR_CUDA;
    return launched();
}

int monde_quantize_fp8(int32_t dtype, int32_t batch, int32_t rows, int32_t cols, int32_t block_rows, const void* x,
                       int64_t ld_x, void* q, int64_t ld_q, float* scale, int64_t ld_scale, void* stream) {
    if (batch < 0 || rows < 0 || cols <= 0) return MONDE_ERR_INVALID_ARG;
    if (dtype != MONDE_F32 && dtype != MONDE_BF16) return MONDE_ERR_UNSUPPORTED;
    if (block_rows != 1 && block_rows != kFp8Block) return MONDE_ERR_UNSUPPORTED;
    const int blocks = (cols + kFp8Block - 1) / kFp8Block;
    if (ld_x < cols || ld_q < cols || ld_scale < blocks) return MONDE_ERR_INVALID_ARG;
    if (batch == 0 || rows == 0) return MONDE_OK;
    if (!x || !q || !scale) return MONDE_ERR_INVALID_ARG;
    const int b = static_cast<int>(elem_bytes(dtype));
    if (!multiple_of(x, b) || !multiple_of(scale, 4)) return MONDE_ERR_INVALID_ARG;
    const int64_t tiles = static_cast<int64_t>(batch) * ((rows + kFp8Block - 1) / kFp8Block) * blocks;
    if (block_rows != 1 && tiles > 0x7fffffff) return MONDE_ERR_UNSUPPORTED;
    const int st = check_arch();
    if (st != MONDE_OK) return st;
    const QuantParams P = {static_cast<int64_t>(batch) * rows, rows, cols, blocks, x, static_cast<uint8_t*>(q), scale,
                           ld_x, ld_q, ld_scale};
    const bool vec = cols % 8 == 0 && multiple_of(x, ld_x * b, 16) && multiple_of(q, ld_q, 8);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (block_rows == 1) {
        const int64_t want = (P.rows * blocks + 15) / 16;
        const dim3 grid(static_cast<unsigned>(want < 148 * 32 ? want : 148 * 32));
        if (dtype == MONDE_BF16)
            e = vec ? launch_pdl(quantize_rows_kernel<__nv_bfloat16, true>, grid, dim3(256), 0, s, P)
                    : launch_pdl(quantize_rows_kernel<__nv_bfloat16, false>, grid, dim3(256), 0, s, P);
        else
            e = vec ? launch_pdl(quantize_rows_kernel<float, true>, grid, dim3(256), 0, s, P)
                    : launch_pdl(quantize_rows_kernel<float, false>, grid, dim3(256), 0, s, P);
    } else {
        const dim3 grid(static_cast<unsigned>(tiles));
        if (dtype == MONDE_BF16)
            e = vec ? launch_pdl(quantize_blocks_kernel<__nv_bfloat16, true>, grid, dim3(256), 0, s, P)
                    : launch_pdl(quantize_blocks_kernel<__nv_bfloat16, false>, grid, dim3(256), 0, s, P);
        else
            e = vec ? launch_pdl(quantize_blocks_kernel<float, true>, grid, dim3(256), 0, s, P)
                    : launch_pdl(quantize_blocks_kernel<float, false>, grid, dim3(256), 0, s, P);
    }
    if (e != cudaSuccess) return MONDE_ERR_CUDA;
    return launched();
}

}  // extern "C"
