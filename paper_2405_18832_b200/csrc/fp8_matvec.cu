// Block-scaled e4m3 product for a few rows: the decode step's form.
//
// With at most 32 rows in all the product is one pass over the weights of the experts that have rows, and what counts is how
// soon the first bytes are asked for and how many are in flight; the big kernel spends some 5 us on its way in and out
// (tensor memory, barriers, unit list, hand-overs).  Here every warp streams 16 weight rows straight into the registers of
// mma.sync (m16n8k32, weights as the 16 rows, x rows as the 8 columns): a lane's 16-byte loads hold four K slices each, and
// since a sum does not depend on the order of its terms, the K index is permuted so that they are used as they come.  Each
// 128-wide K block starts from zero and is added, scaled, to sums in registers.  Warps of a CTA split the K range and their
// sums are added in the order of K through shared memory, so results are bit-reproducible.
#include "fp8_matmul.cuh"

namespace monde {

namespace {

constexpr int kMaxTiles = kMatvecRows / 8;       // 8-row tiles of x

struct MatvecUnits {
    int n_active;                       // experts with rows
    int expert[kMatvecRows];            // at most one per row
    int first[kMatvecRows + 1], count[kMatvecRows + 1];
};

__device__ __forceinline__ uint4 load_weights(const uint8_t* p) {       // read once
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void mma_e4m3(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// kTiles: 8-row tiles of x that a warp carries at once.  kGroups of the warps take 16 weight rows each, the others share
// their K range.  An e4m3 output needs a block's 128 columns in one CTA (kGroups = 8).
template <int kTiles, int kGroups, int kThreads>
__global__ void __launch_bounds__(kThreads, kTiles == 1 ? 768 / kThreads : 512 / kThreads) matvec_fp8_kernel(const MatmulParams P, const uint8_t* __restrict__ w) {
    constexpr int kParts = kThreads / 32 / kGroups;             // K range of a weight row, split over so many warps
    constexpr int kCols = 16 * kGroups, kRows = 8 * kTiles;
    __shared__ MatvecUnits un;
    __shared__ alignas(16) float sums[kParts][kRows][kCols + 4];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int group = warp % kGroups, part = warp / kGroups, g = lane >> 2, t = lane & 3;
    pdl_launch_dependents();
    pdl_wait();
    // ---- experts with rows, in order (offsets clamped: a bad list may not reach outside the output) --------------------
    if (P.offsets == nullptr) {
        if (tid == 0) { un.n_active = 1; un.expert[0] = 0; un.first[0] = 0; un.count[0] = P.rows; }
    } else if (warp == 0) {
        int n = 0;
        for (int e0 = 0; e0 < P.E; e0 += 32) {
            const int e = e0 + lane;
            const int lo = e < P.E ? min(max(P.offsets[e], 0), P.rows) : 0;
            const int hi = e < P.E ? min(max(P.offsets[e + 1], 0), P.rows) : 0;
            const unsigned some = __ballot_sync(0xffffffffu, hi > lo);
            const int at = n + __popc(some & ((1u << lane) - 1));
            if (hi > lo && at < kMatvecRows) { un.expert[at] = e; un.first[at] = lo; un.count[at] = hi - lo; }
            n = min(n + __popc(some), kMatvecRows);
        }
        if (lane == 0) un.n_active = n;
    }
    __syncthreads();
    const int kb_all = (P.K + kFp8Block - 1) / kFp8Block, nb = (P.N + kFp8Block - 1) / kFp8Block;
    const int col_blocks = (P.N + kCols - 1) / kCols;
    const int total = un.n_active * col_blocks;
    const int kb_lo = kb_all * part / kParts, kb_hi = kb_all * (part + 1) / kParts;
    for (int u = blockIdx.x; u < total; u += gridDim.x) {
        const int j = u / col_blocks, c0 = (u - j * col_blocks) * kCols, n0 = c0 + group * 16;
        const int e = un.expert[j], first = un.first[j], count = un.count[j];
        // weight rows g and g + 8 of the group (past N the last row stands in; what comes of it is not stored)
        const uint8_t* w0 = w + (static_cast<int64_t>(e) * P.N + min(n0 + g, P.N - 1)) * P.K + 16 * t;
        const uint8_t* w1 = w + (static_cast<int64_t>(e) * P.N + min(n0 + g + 8, P.N - 1)) * P.K + 16 * t;
        const float* ws = P.w_scale + (static_cast<int64_t>(e) * nb + n0 / kFp8Block) * kb_all;
        const bool busy = n0 < P.N;
        for (int r0 = 0; r0 < count; r0 += kRows) {                   // (more than once only when an expert has more rows)
            const int rows = min(kRows, count - r0);
            // this lane's operand row of each tile, and the two rows whose sums it holds
            const uint8_t* xr[kTiles];
            const float* xs[kTiles][2];
#pragma unroll
            for (int i = 0; i < kTiles; ++i) {
                const int r = i * 8 + g;
                const int s = r < rows ? source_row(P, load_row_id(P, first + r0 + r)) : -1;
                xr[i] = s >= 0 ? P.x + s * P.ld_x : nullptr;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int c = __shfl_sync(0xffffffffu, s, (2 * t + h) * 4);
                    xs[i][h] = c >= 0 ? P.x_scale + c * P.ld_x_scale : nullptr;
                }
            }
            float acc[kTiles][4] = {};
            uint4 a[2][4];                     // weight rows g and g + 8, K bytes 16t and 64 + 16t of a block: two blocks in flight
            const auto fetch = [&](int kb, uint4 (&v)[4]) {
                if (kb >= kb_hi) return;
                const int k = kb * kFp8Block;
                if (k + kFp8Block <= P.K) {
                    v[0] = load_weights(w0 + k);
                    v[1] = load_weights(w0 + k + 64);
                    v[2] = load_weights(w1 + k);
                    v[3] = load_weights(w1 + k + 64);
                } else {                           // the last, shorter block: zeros past K
                    const bool lo = k + 16 * t < P.K, hi = k + 64 + 16 * t < P.K;
                    v[0] = lo ? load_weights(w0 + k) : make_uint4(0, 0, 0, 0);
                    v[1] = hi ? load_weights(w0 + k + 64) : make_uint4(0, 0, 0, 0);
                    v[2] = lo ? load_weights(w1 + k) : make_uint4(0, 0, 0, 0);
                    v[3] = hi ? load_weights(w1 + k + 64) : make_uint4(0, 0, 0, 0);
                }
            };
            const auto multiply = [&](int kb, const uint4 (&v)[4]) {
                const int k = kb * kFp8Block + 16 * t;
                const float wf = __ldg(ws + kb);
#pragma unroll
                for (int i = 0; i < kTiles; ++i) {
                    if (i * 8 >= rows) break;
                    uint4 x0 = make_uint4(0, 0, 0, 0), x1 = x0;
                    if (xr[i] != nullptr) {
                        if (k < P.K) x0 = __ldg(reinterpret_cast<const uint4*>(xr[i] + k));
                        if (k + 64 < P.K) x1 = __ldg(reinterpret_cast<const uint4*>(xr[i] + k + 64));
                    }
                    float f[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) f[h] = xs[i][h] != nullptr ? __ldg(xs[i][h] + kb) * wf : 0.0f;
                    float c[4] = {};
                    mma_e4m3(c, v[0].x, v[2].x, v[0].y, v[2].y, x0.x, x0.y);
                    mma_e4m3(c, v[0].z, v[2].z, v[0].w, v[2].w, x0.z, x0.w);
                    mma_e4m3(c, v[1].x, v[3].x, v[1].y, v[3].y, x1.x, x1.y);
                    mma_e4m3(c, v[1].z, v[3].z, v[1].w, v[3].w, x1.z, x1.w);
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[i][q] = fmaf(f[q & 1], c[q], acc[i][q]);
                }
            };
            if (busy) {
                fetch(kb_lo, a[0]);
                fetch(kb_lo + 1, a[1]);
                for (int kb = kb_lo; kb < kb_hi; kb += 2) {
                    multiply(kb, a[0]);
                    fetch(kb + 2, a[0]);
                    if (kb + 1 < kb_hi) multiply(kb + 1, a[1]);
                    fetch(kb + 3, a[1]);
                }
            }
            __syncthreads();                   // the sums of the unit before have been read
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) sums[part][i * 8 + 2 * t + (q & 1)][group * 16 + g + 8 * (q >> 1)] = acc[i][q];
            __syncthreads();
            // ---- a warp per row, four columns a lane --------------------------------------------------------------------
            const int col = 4 * lane, n = c0 + col;
            const bool mine = col < kCols;
            for (int r = warp; r < rows; r += kThreads / 32) {
                const int64_t row = first + r0 + r;
                float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (mine) {
#pragma unroll
                    for (int p = 0; p < kParts; ++p) {
                        const float4 s = *reinterpret_cast<const float4*>(&sums[p][r][col]);
                        v[0] += s.x; v[1] += s.y; v[2] += s.z; v[3] += s.w;
                    }
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (!mine || n + q >= P.N) { v[q] = 0.0f; continue; }
                    if (P.bias != nullptr) v[q] += __ldg(P.bias + static_cast<int64_t>(e) * P.N + n + q);
                    if (P.act == MONDE_ACT_RELU) v[q] = max_nan(v[q], 0.0f);
                }
                if (P.act == MONDE_ACT_GELU_ERF) {
                    const float2 p = gelu2(make_float2(v[0], v[1])), q = gelu2(make_float2(v[2], v[3]));
                    v[0] = p.x; v[1] = p.y; v[2] = q.x; v[3] = q.y;
                }
                const bool whole = mine && n + 4 <= P.N && P.out_vec;
                if (P.out_dtype == MONDE_E4M3) {
                    float amax = max_nan(max_nan(fabsf(v[0]), fabsf(v[1])), max_nan(fabsf(v[2]), fabsf(v[3])));
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, o));
                    const float s = block_scale(amax), inv = __fdiv_rn(1.0f, s);
                    if (lane == 0) P.out_scale[row * P.ld_out_scale + c0 / kFp8Block] = s;
                    const uint32_t packed = pack_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
                    uint8_t* out = static_cast<uint8_t*>(P.out) + row * P.ld_out + n;
                    if (whole) *reinterpret_cast<uint32_t*>(out) = packed;
                    else
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            if (mine && n + q < P.N) out[q] = static_cast<uint8_t>(packed >> (8 * q));
                } else if (P.out_dtype == MONDE_BF16) {
                    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(P.out) + row * P.ld_out + n;
                    if (whole) {
                        const __nv_bfloat162 p = __floats2bfloat162_rn(v[0], v[1]), q = __floats2bfloat162_rn(v[2], v[3]);
                        *reinterpret_cast<uint2*>(out) = make_uint2(*reinterpret_cast<const uint32_t*>(&p), *reinterpret_cast<const uint32_t*>(&q));
                    } else {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            if (mine && n + q < P.N) out[q] = __float2bfloat16_rn(v[q]);
                    }
                } else {
                    float* out = static_cast<float*>(P.out) + row * P.ld_out + n;
                    if (whole) *reinterpret_cast<float4*>(out) = make_float4(v[0], v[1], v[2], v[3]);
                    else
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            if (mine && n + q < P.N) out[q] = v[q];
                }
            }
        }
    }
}

template <int kTiles, int kGroups, int kThreads>
cudaError_t launch(const MatmulParams& P, const uint8_t* w, cudaStream_t s) {
    const int64_t blocks = (P.N + 16 * kGroups - 1) / (16 * kGroups);
    const int64_t units = blocks * (P.offsets == nullptr ? 1 : (P.E < P.rows ? P.E : P.rows));    // at most
    const int64_t most = static_cast<int64_t>(current_sm_count()) * ((kTiles == 1 ? 768 : 512) / kThreads);
    return launch_pdl(matvec_fp8_kernel<kTiles, kGroups, kThreads>, dim3(static_cast<unsigned>(units < most ? units : most)),
                      dim3(kThreads), 0, s, P, w);
}

// An e4m3 output has eight groups of warps in a CTA (a scale's 128 columns); the K range is split in two besides when that
// leaves SMs without a CTA.  Other outputs: 32 columns, K in four parts.
template <int kTiles>
cudaError_t launch(const MatmulParams& P, const uint8_t* w, cudaStream_t s) {
    if (P.out_dtype != MONDE_E4M3) return launch<kTiles, 2, 256>(P, w, s);
    const int64_t units = static_cast<int64_t>((P.N + kFp8Block - 1) / kFp8Block) * (P.offsets == nullptr ? 1 : (P.E < P.rows ? P.E : P.rows));
    return units > 2 * current_sm_count() ? launch<kTiles, 8, 256>(P, w, s) : launch<kTiles, 8, 512>(P, w, s);
}

}  // namespace

int launch_matvec_fp8(const MatmulParams& P, const void* w, cudaStream_t s) {
    const uint8_t* weights = static_cast<const uint8_t*>(w);
    // Few experts of a decode batch have more than eight rows; those read their weights again (from L2) for the next eight.
    const cudaError_t e = P.offsets != nullptr || P.rows <= 8 ? launch<1>(P, weights, s)
                          : P.rows <= 16 ? launch<2>(P, weights, s) : launch<kMaxTiles>(P, weights, s);
    if (e != cudaSuccess) return MONDE_ERR_CUDA;
    return launched();
}

}  // namespace monde
