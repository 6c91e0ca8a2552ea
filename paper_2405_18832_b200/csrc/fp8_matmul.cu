// e4m3 matrix product with a scale per 128-block, dense and grouped by expert.
//
// out[r,n] = act(bias[n] + sum_b xs[r,b] ws[n/128,b] P_b[r,n]),  P_b[r,n] = sum_{k in block b} x[r,k] w[n,k].
#include "fp8.cuh"

namespace monde {

namespace {

struct MatmulParams {
    int rows, N, K, E, src_rows, row_div, act, out_dtype;
    int64_t ld_x, ld_x_scale, ld_out, ld_out_scale;
    const uint8_t* x;
    const float* x_scale;
    const uint8_t* w;
    const float* w_scale;
    const float* bias;
    const int32_t* offsets;     // null: one matrix, all rows
    const int32_t* row_ids;     // null: position r reads row r
    void* out;
    float* out_scale;
};

constexpr int kTileM = 32, kTileN = 128, kSubK = 32;
constexpr int kThreads = 256;

__device__ __forceinline__ float e4m3_to_float(uint8_t v) {
    const __half_raw h = __nv_cvt_fp8_to_halfraw(v, __NV_E4M3);
    return __half2float(__half(h));
}

// One 32 x 128 tile at a time on the CUDA cores: every warp holds four rows, every lane four columns of each.
__global__ void __launch_bounds__(kThreads) matmul_fp8_simt_kernel(const MatmulParams P) {
    __shared__ float sx[kTileM][kSubK + 1], sw[kTileN][kSubK + 1];
    __shared__ int src[kTileM];
    __shared__ int prefix[kMaxExperts + 1], first[kMaxExperts + 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_launch_dependents();
    pdl_wait();
    for (int e = tid; e <= P.E; e += kThreads)
        first[e] = P.offsets != nullptr ? min(max(P.offsets[e], 0), P.rows) : (e == 0 ? 0 : P.rows);
    __syncthreads();
    if (tid == 0) {
        int run = 0;
        for (int e = 0; e < P.E; ++e) {
            prefix[e] = run;
            run += max(0, first[e + 1] - first[e] + kTileM - 1) / kTileM;
        }
        prefix[P.E] = run;
    }
    __syncthreads();
    const int nb = (P.N + kTileN - 1) / kTileN, kb = (P.K + kFp8Block - 1) / kFp8Block;
    const int64_t total = static_cast<int64_t>(prefix[P.E]) * nb;
    for (int64_t tile = blockIdx.x; tile < total; tile += gridDim.x) {
        const int mt = static_cast<int>(tile / nb), nt = static_cast<int>(tile % nb);
        int e = 0;
        while (prefix[e + 1] <= mt) ++e;
        const int r0 = first[e] + (mt - prefix[e]) * kTileM;
        const int rows = min(kTileM, first[e + 1] - r0);
        const int n0 = nt * kTileN;
        __syncthreads();
        if (tid < kTileM) {
            int s = -1;
            if (tid < rows) {
                s = r0 + tid;
                if (P.row_ids != nullptr) {
                    const int id = P.row_ids[s];
                    s = id < 0 ? -1 : id / P.row_div;
                }
                if (s >= P.src_rows) s = -1;
            }
            src[tid] = s;
        }
        __syncthreads();
        const uint8_t* w = P.w + static_cast<int64_t>(e) * P.N * P.K;
        float acc[4][4] = {};
        for (int b = 0; b < kb; ++b) {
            float part[4][4] = {};
            for (int k0 = b * kFp8Block; k0 < min(P.K, (b + 1) * kFp8Block); k0 += kSubK) {
                for (int i = tid; i < kTileM * kSubK; i += kThreads) {
                    const int r = i / kSubK, k = k0 + i % kSubK;
                    sx[r][i % kSubK] = src[r] >= 0 && k < P.K ? e4m3_to_float(P.x[src[r] * P.ld_x + k]) : 0.0f;
                }
                for (int i = tid; i < kTileN * kSubK; i += kThreads) {
                    const int n = i / kSubK, k = k0 + i % kSubK;
                    sw[n][i % kSubK] = n0 + n < P.N && k < P.K
                        ? e4m3_to_float(w[static_cast<int64_t>(n0 + n) * P.K + k]) : 0.0f;
                }
                __syncthreads();
                for (int k = 0; k < kSubK; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            part[i][j] = fmaf(sx[warp * 4 + i][k], sw[lane + 32 * j][k], part[i][j]);
                __syncthreads();
            }
            const float ws = P.w_scale[(static_cast<int64_t>(e) * nb + nt) * kb + b];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int s = src[warp * 4 + i];
                const float f = s >= 0 ? P.x_scale[s * P.ld_x_scale + b] * ws : 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(f, part[i][j], acc[i][j]);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = warp * 4 + i;
            float amax = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = n0 + lane + 32 * j;
                if (n >= P.N) { acc[i][j] = 0.0f; continue; }
                if (P.bias != nullptr) acc[i][j] += P.bias[static_cast<int64_t>(e) * P.N + n];
                acc[i][j] = apply_act_nan(acc[i][j], P.act);
                amax = max_nan(amax, fabsf(acc[i][j]));
            }
            float inv = 0.0f;
            if (P.out_dtype == MONDE_E4M3) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, o));
                const float s = block_scale(amax);
                inv = __fdiv_rn(1.0f, s);
                if (r < rows && lane == 0) P.out_scale[(r0 + r) * P.ld_out_scale + nt] = s;
            }
            if (r >= rows) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = n0 + lane + 32 * j;
                if (n >= P.N) continue;
                const int64_t at = (r0 + r) * P.ld_out + n;
                if (P.out_dtype == MONDE_E4M3)
                    static_cast<uint8_t*>(P.out)[at] = static_cast<uint8_t>(pack_e4m3(acc[i][j] * inv, 0.f, 0.f, 0.f));
                else if (P.out_dtype == MONDE_BF16)
                    static_cast<__nv_bfloat16*>(P.out)[at] = __float2bfloat16_rn(acc[i][j]);
                else
                    static_cast<float*>(P.out)[at] = acc[i][j];
            }
        }
    }
}

int check_matmul(const monde_matmul_problem* p) {
    if (p == nullptr) return MONDE_ERR_INVALID_ARG;
    if (p->rows < 0 || p->N <= 0 || p->K <= 0 || p->E <= 0 || p->src_rows < 0 || p->row_div <= 0)
        return MONDE_ERR_INVALID_ARG;
    if (p->K % 16 != 0 || p->E > kMaxExperts) return MONDE_ERR_UNSUPPORTED;
    if (p->act != MONDE_ACT_NONE && p->act != MONDE_ACT_RELU && p->act != MONDE_ACT_GELU_ERF) return MONDE_ERR_UNSUPPORTED;
    if (p->out_dtype != MONDE_BF16 && p->out_dtype != MONDE_F32 && p->out_dtype != MONDE_E4M3) return MONDE_ERR_UNSUPPORTED;
    const int kb = (p->K + kFp8Block - 1) / kFp8Block, nb = (p->N + kFp8Block - 1) / kFp8Block;
    if (p->ld_x < p->K || p->ld_x_scale < kb || p->ld_out < p->N ||
        (p->out_dtype == MONDE_E4M3 && p->ld_out_scale < nb))
        return MONDE_ERR_INVALID_ARG;
    if (p->ld_x % 16 != 0) return MONDE_ERR_INVALID_ARG;
    return MONDE_OK;
}

bool aligned(const void* p, unsigned m) { return (reinterpret_cast<uintptr_t>(p) & (m - 1)) == 0; }

size_t matmul_ws_bytes(const monde_matmul_problem&) { return WsLayout::kHidden; }

int matmul(const monde_matmul_problem* p, const void* x, const float* x_scale, const void* w, const float* w_scale,
           const float* bias, bool grouped, const int32_t* offsets, const int32_t* row_ids, void* out, float* out_scale,
           void* ws, size_t ws_bytes, void* stream) {
    int st = check_matmul(p);
    if (st != MONDE_OK) return st;
    if (!grouped && p->E != 1) return MONDE_ERR_INVALID_ARG;
    if (row_ids == nullptr && p->src_rows != p->rows) return MONDE_ERR_INVALID_ARG;
    if (p->rows == 0) return MONDE_OK;
    if (!x || !x_scale || !w || !w_scale || !out || (grouped && !offsets) || p->src_rows == 0) return MONDE_ERR_INVALID_ARG;
    if (p->out_dtype == MONDE_E4M3 && !out_scale) return MONDE_ERR_INVALID_ARG;
    const unsigned ob = p->out_dtype == MONDE_E4M3 ? 1 : (p->out_dtype == MONDE_BF16 ? 2 : 4);
    if (!aligned(x, 16) || !aligned(w, 16) || !aligned(x_scale, 4) || !aligned(w_scale, 4) || !aligned(bias, 4) ||
        !aligned(offsets, 4) || !aligned(row_ids, 4) || !aligned(out, ob) ||
        (p->out_dtype == MONDE_E4M3 && !aligned(out_scale, 4)))
        return MONDE_ERR_INVALID_ARG;
    if (ws == nullptr || !aligned(ws, 16)) return MONDE_ERR_INVALID_ARG;
    if (ws_bytes < matmul_ws_bytes(*p)) return MONDE_ERR_WORKSPACE;
    if ((st = check_arch()) != MONDE_OK) return st;
    MatmulParams P;
    P.rows = p->rows; P.N = p->N; P.K = p->K; P.E = p->E;
    P.src_rows = p->src_rows; P.row_div = p->row_div; P.act = p->act; P.out_dtype = p->out_dtype;
    P.ld_x = p->ld_x; P.ld_x_scale = p->ld_x_scale; P.ld_out = p->ld_out; P.ld_out_scale = p->ld_out_scale;
    P.x = static_cast<const uint8_t*>(x);
    P.x_scale = x_scale;
    P.w = static_cast<const uint8_t*>(w);
    P.w_scale = w_scale;
    P.bias = bias;
    P.offsets = offsets;
    P.row_ids = row_ids;
    P.out = out;
    P.out_scale = out_scale;
    if (launch_pdl(matmul_fp8_simt_kernel, dim3(current_sm_count() * 4), dim3(kThreads), 0,
                   static_cast<cudaStream_t>(stream), P) != cudaSuccess)
        return MONDE_ERR_CUDA;
    return launched();
}

}  // namespace

}  // namespace monde

using namespace monde;

extern "C" {

size_t monde_matmul_workspace_bytes(const monde_matmul_problem* p) {
    return check_matmul(p) == MONDE_OK ? matmul_ws_bytes(*p) : 0;
}

int monde_matmul_fp8(const monde_matmul_problem* p, const void* x, const float* x_scale, const void* w,
                     const float* w_scale, const float* bias, void* out, float* out_scale, void* ws, size_t ws_bytes,
                     void* stream) {
    return matmul(p, x, x_scale, w, w_scale, bias, false, nullptr, nullptr, out, out_scale, ws, ws_bytes, stream);
}

int monde_grouped_matmul_fp8(const monde_matmul_problem* p, const void* x, const float* x_scale, const void* w,
                             const float* w_scale, const float* bias, const int32_t* offsets, const int32_t* row_ids,
                             void* out, float* out_scale, void* ws, size_t ws_bytes, void* stream) {
    return matmul(p, x, x_scale, w, w_scale, bias, true, offsets, row_ids, out, out_scale, ws, ws_bytes, stream);
}

}  // extern "C"
