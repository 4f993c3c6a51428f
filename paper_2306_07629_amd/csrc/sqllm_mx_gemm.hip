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

// ---------------------------------------------------------------------------------------------- many rows on both sides
constexpr int kTileRows = 256;                                       // of W and of X
constexpr int kStageBytes = 2 * kTileRows * 64;                      // 128 columns of both
constexpr int kScaleGroupBytes = 2 * kTileRows * 16;                 // scales of 512 columns of both

__device__ __forceinline__ u32 chunk_swizzle(u32 row) { return ((row >> 1) ^ (row >> 3)) & 3u; }

// What a lane holds of a result tile of 32 rows of W x 32 rows of X goes to y: four neighbouring elements of row t, four times.
template <int TYPE, bool VEC>
__device__ __forceinline__ void store_block(const MxGemmArgs& g, const f32x16& acc, long long m, long long t) {
    typedef typename MxType<TYPE>::value value;
    typedef value value4 __attribute__((ext_vector_type(4)));
    if (t >= g.T) return;
    value* y = static_cast<value*>(g.y) + t * g.ldy + m;
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
        const long long left = g.M - (m + 2 * e);
        if (VEC && left >= 4) {
            value4* d = reinterpret_cast<value4*>(y + 2 * e);
            value4 v;
            if (g.accumulate) {
                const value4 old = *d;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = (value)((float)old[i] + acc[e + i]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = (value)acc[e + i];
            }
            *d = v;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < left) y[2 * e + i] = (value)(g.accumulate ? (float)y[2 * e + i] + acc[e + i] : acc[e + i]);
        }
    }
}

template <int TYPE, bool VEC>
__global__ void __launch_bounds__(256, 1) mx_gemm_tile_kernel(MxGemmArgs g, int tiles_m, int tiles_t, int K) {
    __shared__ __align__(16) char stage[2 * kStageBytes];
    __shared__ __align__(16) char scale[2 * kScaleGroupBytes];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 31, h = lane >> 5;
    const int n = tiles_m * tiles_t, xcd = blockIdx.x & 7, q8 = n >> 3, r8 = n & 7;
    const int p = xcd * q8 + min(xcd, r8) + (int)(blockIdx.x >> 3);
    const int per = 8 * tiles_t, grp = p / per, in = p % per, gsz = min(tiles_m - 8 * grp, 8);
    const int tm = 8 * grp + in % gsz, tt = in / gsz;
    const long long m0 = (long long)tm * kTileRows, t0 = (long long)tt * kTileRows;
    const u32 cp = K / 2, sp = K / kMxBlock;
    const int nst = K / 128;
    // waves 0, 1 fetch the rows of W, 2, 3 those of X: 128 rows each, 16 rows of 64 bytes to an instruction
    const bool mine_w = wave < 2;
    const char* codes = static_cast<const char*>(mine_w ? g.w_codes : g.x_codes) + (size_t)(mine_w ? m0 : t0) * cp;
    const char* scales = static_cast<const char*>(mine_w ? g.w_scales : g.x_scales) + (size_t)(mine_w ? m0 : t0) * sp;
    const int last = (int)min((mine_w ? (long long)g.M - m0 : (long long)g.T - t0) - 1, (long long)kTileRows - 1);
    u32 off[8], wr[8], soff[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const u32 row = 128 * (wave & 1) + 16 * i + (lane >> 2), rc = (u32)min((int)row, last);
        off[i] = rc * cp + 16 * (lane & 3);
        soff[i] = rc * sp;
        wr[i] = wave * 8192 + 1024 * i + 64 * (lane >> 2) + 16 * ((lane & 3) ^ chunk_swizzle(row));
    }
    const int wm = wave & 1, wt = wave >> 1;
    const u32 rd0 = r * 64 + 16 * ((2 * h) ^ chunk_swizzle(r)), rd1 = rd0 ^ 16;
    const u32 rda = wm * 8192, rdb = 16384 + wt * 8192;
    f32x16 acc[4][4] = {};
    i32x4 a0[4], b0[4], a1[4], b1[4], pre[2][8];
    u32 ua[4], ub[4], va[4], vb[4], spre[2][2];
    auto fetch = [&](int s, i32x4 (&d)[8]) {
        const char* base = codes + (size_t)min(s, nst - 1) * 64;
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = *reinterpret_cast<const i32x4*>(base + off[i]);
    };
    auto put = [&](int s, const i32x4 (&d)[8]) {
        char* b = stage + (s & 1) * kStageBytes;
#pragma unroll
        for (int i = 0; i < 8; ++i) *reinterpret_cast<i32x4*>(b + wr[i]) = d[i];
    };
    // quarter q of the scales of 512 columns: 32 rows of the wave's 128, four dwords each
    auto fetch_scales = [&](int grp4, int q, u32 (&d)[2]) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int dw = 4 * grp4 + (lane & 3);
            const u32 row = 128 * (wave & 1) + 32 * q + 16 * k + (lane >> 2), rc = (u32)min((int)row, last);
            d[k] = *reinterpret_cast<const u32*>(scales + (size_t)(rc * sp + 4 * (u32)min(dw, nst - 1)));
        }
    };
    auto put_scales = [&](int grp4, int q, const u32 (&d)[2]) {
        char* b = scale + (grp4 & 1) * kScaleGroupBytes;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const u32 row = 32 * q + 16 * k + (lane >> 2);
            *reinterpret_cast<u32*>(b + wave * 2048 + 16 * row + 4 * ((lane ^ (row >> 3)) & 3)) = 4 * grp4 + (lane & 3) < nst ? d[k] : 0u;
        }
    };
    auto read = [&](int s, u32 rd, i32x4 (&a)[4], i32x4 (&b)[4]) {
        const char* base = stage + (s & 1) * kStageBytes;
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            a[f] = *reinterpret_cast<const i32x4*>(base + rda + rd + 2048 * f);
            b[f] = *reinterpret_cast<const i32x4*>(base + rdb + rd + 2048 * f);
        }
    };
    auto read_scales = [&](int s, u32 (&a)[4], u32 (&b)[4]) {
        const char* base = scale + ((s >> 2) & 1) * kScaleGroupBytes + 16 * r + 4 * ((s ^ (r >> 3)) & 3) + 2 * h;
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            a[f] = *reinterpret_cast<const uint16_t*>(base + wm * 2048 + 512 * f);
            b[f] = *reinterpret_cast<const uint16_t*>(base + 4096 + wt * 2048 + 512 * f);
        }
    };
    // before the first stage: stage 0 and the scales of the first 512 columns in LDS, stages 1 and 2 and the quarters to be written in stages 0 and 1 on the way
    {
        u32 s4[4][2];
#pragma unroll
        for (int q = 0; q < 4; ++q) fetch_scales(0, q, s4[q]);
        fetch(0, pre[0]);
        put(0, pre[0]);
#pragma unroll
        for (int q = 0; q < 4; ++q) put_scales(0, q, s4[q]);
        __builtin_amdgcn_sched_barrier(0);
        fetch(1, pre[1]);
        fetch_scales(1, 0, spre[0]);
        __builtin_amdgcn_sched_barrier(0);
        fetch(2, pre[0]);
        fetch_scales(1, 1, spre[1]);
    }
    __syncthreads();
    read(0, rd0, a0, b0);
    read_scales(0, ua, ub);
    for (int s2 = 0; s2 < nst; s2 += 2) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int s = s2 + j;
            put(s + 1, pre[1 - j]);
            put_scales(s / 4 + 1, s & 3, spre[j]);
            fetch(s + 3, pre[1 - j]);
            fetch_scales((s + 2) / 4 + 1, (s + 2) & 3, spre[j]);
            read(s, rd1, a1, b1);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[i][k] = mma<0>(a0[i], b0[k], acc[i][k], ua[i], ub[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x200, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x020, 2, 0);
            __builtin_amdgcn_sched_barrier(0);
            __syncthreads();
            __builtin_amdgcn_sched_barrier(0);
            read(s + 1, rd0, a0, b0);
            read_scales(s + 1, va, vb);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[i][k] = mma<1>(a1[i], b1[k], acc[i][k], ua[i], ub[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
                __builtin_amdgcn_sched_group_barrier(0x008, 2, 1);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int f = 0; f < 4; ++f) { ua[f] = va[f]; ub[f] = vb[f]; }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) store_block<TYPE, VEC>(g, acc[i][k], m0 + 128 * wm + 32 * i + 4 * h, t0 + 128 * wt + 32 * k + r);
}

namespace {

template <int TYPE>
hipError_t gemm(const MxGemmArgs& g, hipStream_t s) {
    const int K = mx_padded(g.N);
    const long long big_m = ((long long)g.M + kTileRows - 1) / kTileRows, big_t = ((long long)g.T + kTileRows - 1) / kTileRows;
    if (big_m * big_t >= 128 && K <= 1 << 24) {
        const bool vec = (reinterpret_cast<uintptr_t>(g.y) & (4 * mx_type_size(TYPE) - 1)) == 0 && g.ldy % 4 == 0;
        const dim3 grid((unsigned)(big_m * big_t));
        if (vec) mx_gemm_tile_kernel<TYPE, true><<<grid, 256, 0, s>>>(g, (int)big_m, (int)big_t, K);
        else mx_gemm_tile_kernel<TYPE, false><<<grid, 256, 0, s>>>(g, (int)big_m, (int)big_t, K);
    } else {
        const int tiles_m = (int)(((long long)g.M + 63) / 64), tiles_t = (int)(((long long)g.T + 63) / 64);
        mx_gemm_kernel<TYPE><<<dim3((unsigned)((long long)tiles_m * tiles_t)), kGemmWaves * 64, 0, s>>>(g, tiles_m, K);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_gemm(const MxGemmArgs& g, hipStream_t s) {
    return g.type == SQLLM_F16 ? gemm<SQLLM_F16>(g, s) : g.type == SQLLM_BF16 ? gemm<SQLLM_BF16>(g, s) : gemm<SQLLM_F32>(g, s);
}

}  // namespace sqllm
