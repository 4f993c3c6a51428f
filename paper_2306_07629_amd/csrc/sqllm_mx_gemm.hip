// Product of two packed matrices of the microscaled 4-bit format on the matrix cores -- device code for gfx950 (wave64).
//
// y[t][i] = sum_j X[t][j] W[i][j].  v_mfma_scale_f32_32x32x64 multiplies A (32 rows of W x 64 j) by B (64 j x 32 rows of X) and takes codes
// and scale bytes as they lie in memory: lane (r, h) = (l % 32, l / 32) supplies one block of 32 codes (16 bytes) of row r and that block's
// scale, and keeps of the result column r (a row of X) the rows 8 (e / 4) + 4 h + e % 4 of W, e = 0..15.  Which blocks of a row the two
// halves of a wave take at which step is free as long as both operands agree: half h takes blocks 4 h + s of every eight at step
// s = 0..3, so its four scale bytes are one dword and its codes 64 neighbouring bytes.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sqllm_mx.h"
#include "sqllm_mx_device.h"

namespace sqllm {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int S>
__device__ __forceinline__ f32x16 mma(const i32x4& a, const i32x4& b, const f32x16& c, u32 sa, u32 sb) {
    const i32x8 A = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, B = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(A, B, c, 4, 4, S, (int)sa, S, (int)sb);
}

// Four waves share a tile of 64 rows of W x 64 rows of X and deal its steps of 256 columns out among themselves; their sums meet in LDS.
constexpr int kGemmWaves = 4;

template <int TYPE>
__global__ void __launch_bounds__(kGemmWaves * 64) mx_gemm_kernel(MxGemmArgs g, int tiles_m, int K) {
    __shared__ float part[kGemmWaves][16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, h = lane >> 5;
    const long long m0 = 64ll * (blockIdx.x % tiles_m), t0 = 64ll * (blockIdx.x / tiles_m);
    const size_t cp = K / 2, sp = K / kMxBlock;
    const char *ac[2], *bc[2], *as[2], *bs[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) {                                    // rows past the end repeat the last one; their results are not stored
        const size_t m = min(m0 + 32 * f + r, (long long)g.M - 1), t = min(t0 + 32 * f + r, (long long)g.T - 1);
        ac[f] = static_cast<const char*>(g.w_codes) + m * cp; as[f] = static_cast<const char*>(g.w_scales) + m * sp;
        bc[f] = static_cast<const char*>(g.x_codes) + t * cp; bs[f] = static_cast<const char*>(g.x_scales) + t * sp;
    }
    f32x16 acc[2][2] = {};
    for (int k = 256 * wave; k + 256 <= K; k += 256 * kGemmWaves) {
        i32x4 a[2][4], b[2][4];
        u32 sa[2], sb[2];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                a[f][s] = *reinterpret_cast<const i32x4*>(ac[f] + k / 2 + 64 * h + 16 * s);
                b[f][s] = *reinterpret_cast<const i32x4*>(bc[f] + k / 2 + 64 * h + 16 * s);
            }
            sa[f] = *reinterpret_cast<const u32*>(as[f] + k / 32 + 4 * h);
            sb[f] = *reinterpret_cast<const u32*>(bs[f] + k / 32 + 4 * h);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                acc[i][j] = mma<0>(a[i][0], b[j][0], acc[i][j], sa[i], sb[j]);
                acc[i][j] = mma<1>(a[i][1], b[j][1], acc[i][j], sa[i], sb[j]);
                acc[i][j] = mma<2>(a[i][2], b[j][2], acc[i][j], sa[i], sb[j]);
                acc[i][j] = mma<3>(a[i][3], b[j][3], acc[i][j], sa[i], sb[j]);
            }
    }
    if (K % 256 != 0 && (K / 256) % kGemmWaves == wave) {            // the last 128 columns: half h takes blocks 2 h + s
        const int k = K - 128;
        i32x4 a[2][2], b[2][2];
        u32 sa[2], sb[2];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                a[f][s] = *reinterpret_cast<const i32x4*>(ac[f] + k / 2 + 32 * h + 16 * s);
                b[f][s] = *reinterpret_cast<const i32x4*>(bc[f] + k / 2 + 32 * h + 16 * s);
            }
            sa[f] = *reinterpret_cast<const u32*>(as[f] + k / 32) >> (16 * h);
            sb[f] = *reinterpret_cast<const u32*>(bs[f] + k / 32) >> (16 * h);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                acc[i][j] = mma<0>(a[i][0], b[j][0], acc[i][j], sa[i], sb[j]);
                acc[i][j] = mma<1>(a[i][1], b[j][1], acc[i][j], sa[i], sb[j]);
            }
    }
    typedef typename MxType<TYPE>::value value;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 16; ++e) part[wave][e][lane] = acc[i][j][e];
            __syncthreads();
#pragma unroll
            for (int e = wave; e < 16; e += kGemmWaves) {
                const float sum = (part[0][e][lane] + part[1][e][lane]) + (part[2][e][lane] + part[3][e][lane]);
                const long long m = m0 + 32 * i + 8 * (e / 4) + 4 * h + e % 4, t = t0 + 32 * j + r;
                if (m < g.M && t < g.T) {
                    value* y = static_cast<value*>(g.y) + t * g.ldy + m;
                    *y = (value)(g.accumulate ? (float)*y + sum : sum);
                }
            }
        }
}

hipError_t launch_mx_gemm(const MxGemmArgs& g, hipStream_t s) {
    const int K = mx_padded(g.N), tiles_m = (int)(((long long)g.M + 63) / 64), tiles_t = (int)(((long long)g.T + 63) / 64);
    const dim3 grid((unsigned)((long long)tiles_m * tiles_t));
    if (g.type == SQLLM_F16) mx_gemm_kernel<SQLLM_F16><<<grid, kGemmWaves * 64, 0, s>>>(g, tiles_m, K);
    else if (g.type == SQLLM_BF16) mx_gemm_kernel<SQLLM_BF16><<<grid, kGemmWaves * 64, 0, s>>>(g, tiles_m, K);
    else mx_gemm_kernel<SQLLM_F32><<<grid, kGemmWaves * 64, 0, s>>>(g, tiles_m, K);
    return hipGetLastError();
}

}  // namespace sqllm
