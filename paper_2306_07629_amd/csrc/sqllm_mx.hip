// Microscaled 4-bit floating point: quantisation along the rows and along the columns, expansion, and the product with a few fp16
// columns -- device code for gfx950 (wave64).
//
// A block is 32 neighbouring elements of a packed row.  With a = max |v| of the block its scale is 2^e, e = floor(log2 a) - 2 (so that a / 2^e
// lies in [4, 8)), held as the byte e + 127; an element is v / 2^e rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even code,
// what is above 6 becomes 6) with its sign.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <algorithm>

#include "sqllm_mx.h"
#include "sqllm_mx_device.h"

namespace sqllm {

constexpr int kThreads = 256;

// ---------------------------------------------------------------------------------------------- rows: quantise, expand
// Eight elements to a thread, a quad of threads to a block.  A workgroup is 256 / tpr rows of tpr threads, tpr a power of two, so short rows do not
// leave most of it idle; rows beyond the grid are walked in steps of it.
struct RowShape {
    int log_tpr, chunks;    // threads per row, eights per row
};
inline RowShape row_shape(long long chunks) {
    RowShape r;
    r.chunks = (int)chunks;
    r.log_tpr = 4;
    while (r.log_tpr < 8 && (1 << r.log_tpr) < chunks) ++r.log_tpr;
    return r;
}
inline dim3 row_grid(const RowShape& r, int M) {
    const long long groups = ((long long)M + (kThreads >> r.log_tpr) - 1) / (kThreads >> r.log_tpr);
    return dim3((unsigned)((r.chunks + (1 << r.log_tpr) - 1) >> r.log_tpr), (unsigned)(groups < 65535 ? groups : 65535));
}

template <int TYPE, bool VEC>
__global__ void __launch_bounds__(kThreads) mx_quantize_rows_kernel(MxQuantArgs a, RowShape rs, size_t code_pitch, size_t scale_pitch) {
    const int chunk = (int)(blockIdx.x << rs.log_tpr) + (int)(threadIdx.x & ((1u << rs.log_tpr) - 1));
    if (chunk >= rs.chunks) return;                                  // whole quads: chunks is a multiple of 16
    const int rows = kThreads >> rs.log_tpr, j0 = 8 * chunk, left = a.N - j0;
    typedef typename MxType<TYPE>::value value;
    for (long long r = (long long)blockIdx.y * rows + (threadIdx.x >> rs.log_tpr); r < a.M; r += (long long)gridDim.y * rows) {
        const value* src = static_cast<const value*>(a.w) + r * a.ldw + j0;
        MxEight<TYPE> e;
        if (VEC && left >= 8) e.load(src);
        else e.load_some(src, min(max(left, 0), 8));
        const u32 byte = mx_scale_byte(mx_magnitude<TYPE>(quad_max(e.top())));
        reinterpret_cast<u32*>(static_cast<char*>(a.codes) + r * code_pitch)[chunk] = e.pack(byte);
        if ((chunk & 3) == 0) (static_cast<uint8_t*>(a.scales) + r * scale_pitch)[chunk >> 2] = (uint8_t)byte;
    }
}

template <int TYPE, bool VEC>
__global__ void __launch_bounds__(kThreads) mx_dequantize_kernel(MxDequantArgs a, RowShape rs, size_t code_pitch, size_t scale_pitch) {
    const int chunk = (int)(blockIdx.x << rs.log_tpr) + (int)(threadIdx.x & ((1u << rs.log_tpr) - 1));
    if (chunk >= rs.chunks) return;
    const int rows = kThreads >> rs.log_tpr, j0 = 8 * chunk, left = a.N - j0;
    typedef typename MxType<TYPE>::value value;
    for (long long r = (long long)blockIdx.y * rows + (threadIdx.x >> rs.log_tpr); r < a.M; r += (long long)gridDim.y * rows) {
        const u32 codes = reinterpret_cast<const u32*>(static_cast<const char*>(a.codes) + r * code_pitch)[chunk];
        const u32 byte = (static_cast<const uint8_t*>(a.scales) + r * scale_pitch)[chunk >> 2];
        MxEight<TYPE> e;
        e.unpack(codes, byte);
        value* dst = static_cast<value*>(a.w) + r * a.ldw + j0;
        if (VEC && left >= 8) e.store(dst);
        else e.store_some(dst, min(left, 8));
    }
}

// ---------------------------------------------------------------------------------------------- columns: quantise the transpose
// A workgroup takes a tile of 128 x 128 elements through LDS: eights of the rows go in as they are loaded (and, where the row direction is
// asked for too, are quantised on the way, so w is read once for both), then every thread walks down 32 rows of a column.
constexpr int kTile = 128;

template <int TYPE, bool VEC, bool ROWS>
__global__ void __launch_bounds__(kThreads) mx_quantize_tile_kernel(MxQuantArgs a, int tiles_n, size_t code_pitch, size_t scale_pitch, size_t code_pitch_t, size_t scale_pitch_t) {
    typedef typename MxType<TYPE>::value value;
    constexpr int D = MxEight<TYPE>::kDwords, kPitch = kTile / 8 * D;   // dwords of a row
    extern __shared__ __align__(16) u32 tile[];
    const int tid = threadIdx.x;
    const int tm = blockIdx.x / tiles_n, tn = blockIdx.x % tiles_n;
    const long long m0 = (long long)tm * kTile;
    const int n0 = tn * kTile, chunk = tid & 15;
#pragma unroll
    for (int p = 0; p < kTile / 16; ++p) {
        const int row = 16 * p + (tid >> 4), left = m0 + row < a.M ? a.N - (n0 + 8 * chunk) : 0;
        MxEight<TYPE> e;
        const value* src = static_cast<const value*>(a.w) + (m0 + row) * a.ldw + n0 + 8 * chunk;
        if (VEC && left >= 8) e.load(src);
        else e.load_some(src, min(max(left, 0), 8));
        e.store(tile + row * kPitch + chunk * D);
        if (ROWS) {
            const u32 byte = mx_scale_byte(mx_magnitude<TYPE>(quad_max(e.top())));
            const u32 packed = e.pack(byte);
            if (m0 + row < a.M) {
                reinterpret_cast<u32*>(static_cast<char*>(a.codes) + (m0 + row) * code_pitch)[n0 / 8 + chunk] = packed;
                if ((chunk & 3) == 0) (static_cast<uint8_t*>(a.scales) + (m0 + row) * scale_pitch)[n0 / 32 + (chunk >> 2)] = (uint8_t)byte;
            }
        }
    }
    __syncthreads();
    auto put = [&](int col, int b, const MxEight<TYPE> (&e)[4]) {     // block b of the tile's column
        const u32 byte = mx_scale_byte(mx_magnitude<TYPE>(max(max(e[0].top(), e[1].top()), max(e[2].top(), e[3].top()))));
        if (n0 + col < a.N) {
            *reinterpret_cast<u32x4*>(static_cast<char*>(a.codes_t) + (size_t)(n0 + col) * code_pitch_t + m0 / 2 + 16 * b) =
                u32x4{e[0].pack(byte), e[1].pack(byte), e[2].pack(byte), e[3].pack(byte)};
            (static_cast<uint8_t*>(a.scales_t) + (size_t)(n0 + col) * scale_pitch_t)[m0 / 32 + b] = (uint8_t)byte;
        }
    };
    if constexpr (TYPE == SQLLM_F32) {
        const int col = tid & 127;
#pragma unroll
        for (int b = tid >> 7; b < 4; b += 2) {
            MxEight<TYPE> e[4];
#pragma unroll
            for (int k = 0; k < 32; ++k) e[k >> 3].v[k & 7] = tile[(32 * b + k) * kPitch + col];
            put(col, b, e);
        }
    } else {
        const int b = tid >> 6, pair = tid & 63;                     // two neighbouring columns
        MxEight<TYPE> lo[4], hi[4];
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
            const u32 r0 = tile[(32 * b + k) * kPitch + pair], r1 = tile[(32 * b + k + 1) * kPitch + pair];
            lo[k >> 3].v[(k & 7) >> 1] = __builtin_amdgcn_perm(r1, r0, 0x05040100u);
            hi[k >> 3].v[(k & 7) >> 1] = __builtin_amdgcn_perm(r1, r0, 0x07060302u);
        }
        put(2 * pair, b, lo);
        put(2 * pair + 1, b, hi);
    }
}

// ---------------------------------------------------------------------------------------------- a few fp16 columns
// One column: wave w of a workgroup owns columns [2048 w, 2048 w + 2048), lane l block 64 w + l of every row, and keeps the 32 activations of its
// block in 16 registers while it walks down the workgroup's rows, four at a time with the next four requested.  The codes are converted
// without their scale (every code is an fp16 number), so a block's sum is formed as for fp16 weights, and enters the row's sum times the scale in
// fp32: no scale byte leaves a range.
struct FourRows {
    u32x4 codes[4];
    u32 scale[4];
};

__device__ __forceinline__ float block_dot(const u32x4& c, const u32 (&x)[16]) {
    float a0 = 0.f, a1 = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const half2_t w0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c[d], 1.f, 0), w1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c[d], 1.f, 1);
        const half2_t w2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c[d], 1.f, 2), w3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c[d], 1.f, 3);
        a0 = __builtin_amdgcn_fdot2(w0, __builtin_bit_cast(half2_t, x[4 * d]), a0, false);
        a1 = __builtin_amdgcn_fdot2(w1, __builtin_bit_cast(half2_t, x[4 * d + 1]), a1, false);
        a0 = __builtin_amdgcn_fdot2(w2, __builtin_bit_cast(half2_t, x[4 * d + 2]), a0, false);
        a1 = __builtin_amdgcn_fdot2(w3, __builtin_bit_cast(half2_t, x[4 * d + 3]), a1, false);
    }
    return a0 + a1;
}

// scale byte -> fp32 factor: 2^(byte - 127), NaN for 255
__device__ __forceinline__ float scale_factor(u32 byte) {
    const u32 bits = byte == 0u ? 0x00400000u : byte << 23;
    return __uint_as_float(byte == 255u ? 0x7FC00000u : bits);
}

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}

// Sums of four values over the wave; lanes 16 k .. 16 k + 15 end up with that of value 0, 2, 1, 3 for k = 0, 1, 2, 3.
__device__ __forceinline__ float wave_sums(const float (&v)[4]) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[0]), __float_as_uint(v[1]), false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[2]), __float_as_uint(v[3]), false, false);
    const float s01 = __uint_as_float(a[0]) + __uint_as_float(a[1]), s23 = __uint_as_float(b[0]) + __uint_as_float(b[1]);
    const auto c = __builtin_amdgcn_permlane16_swap(__float_as_uint(s01), __float_as_uint(s23), false, false);
    float s = __uint_as_float(c[0]) + __uint_as_float(c[1]);
    s = dpp_add<0xB1>(s);                                            // lane ^ 1
    s = dpp_add<0x4E>(s);                                            // lane ^ 2
    s = dpp_add<0x141>(s);                                           // half mirror: the other quad of the eight
    return dpp_add<0x140>(s);                                        // mirror: the other eight
}

constexpr int kGemvMaxWaves = 14, kGemvMaxRows = 64;                 // rows of a workgroup

__global__ void __launch_bounds__(kGemvMaxWaves * 64) mx_gemv_kernel(MxGemvArgs a, int rows) {
    __shared__ float part[kGemvMaxWaves * kGemvMaxRows];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), nw = blockDim.x >> 6;
    const long long r0 = (long long)blockIdx.x * rows;
    const int n = (int)min((long long)rows, a.M - r0);
    const int nb = a.N / kMxBlock, block = 64 * wave + lane;
    const bool inside = block < nb;
    const int b = min(block, nb - 1);                                // surplus lanes read the last block and multiply with zeros
    u32 x[16];
    {
        const u32x4* src = reinterpret_cast<const u32x4*>(static_cast<const half_t*>(a.x) + 32 * (size_t)b);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const u32x4 v = src[k];
            x[4 * k] = v.x; x[4 * k + 1] = v.y; x[4 * k + 2] = v.z; x[4 * k + 3] = v.w;
        }
    }
    const char* codes = static_cast<const char*>(a.codes) + (size_t)r0 * (a.N / 2);
    const uint8_t* scales = static_cast<const uint8_t*>(a.scales) + (size_t)r0 * nb;
    auto load = [&](int r, FourRows& f) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int row = min(r + k, n - 1);
            f.codes[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(codes + (size_t)row * (a.N / 2)) + b);
            f.scale[k] = __builtin_nontemporal_load(scales + (size_t)row * nb + b);
        }
    };
    FourRows now, next;
    load(0, now);
    const int group = lane >> 4, slot = (group >> 1) | (group & 1) << 1;   // whose sum the lane holds after wave_sums
    for (int r = 0; r < n; r += 4) {
        if (r + 4 < n) load(r + 4, next);
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = inside ? block_dot(now.codes[k], x) * scale_factor(now.scale[k]) : 0.f;
        const float s = wave_sums(v);
        if ((lane & 15) == 0) part[(r + slot) * nw + wave] = s;
        now = next;
    }
    __syncthreads();
    if (tid < n) {
        float s = 0.f;
        for (int w = 0; w < nw; ++w) s += part[tid * nw + w];
        half_t* y = static_cast<half_t*>(a.y) + r0 + tid;
        *y = (half_t)(a.accumulate ? (float)*y + s : s);
    }
}

// A wave to a row, lane l takes blocks l, l + 64, ...  The codes are converted without their scale (every code is an fp16 number), so the block's
// sum is formed exactly as for fp16 weights, and enters the row's sum times the scale in fp32: no scale byte leaves the range.
__global__ void __launch_bounds__(kThreads) mx_gemv_columns_kernel(MxGemvArgs a) {
    const int lane = threadIdx.x & 63;
    const long long row = (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (row >= a.M) return;
    const u32x4* codes = reinterpret_cast<const u32x4*>(static_cast<const char*>(a.codes) + row * (size_t)(a.N / 2));
    const uint8_t* scales = static_cast<const uint8_t*>(a.scales) + row * (size_t)(a.N / kMxBlock);
    const half_t* x = static_cast<const half_t*>(a.x);
    for (int t = 0; t < a.B; ++t) {
        float sum = 0.f;
        for (int b = lane; b < a.N / kMxBlock; b += 64) {
            const u32x4 c = codes[b];
            float part = 0.f;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const u32 w[4] = {MxType<SQLLM_F16>::unpack<0>(c[d], 1.f), MxType<SQLLM_F16>::unpack<1>(c[d], 1.f), MxType<SQLLM_F16>::unpack<2>(c[d], 1.f), MxType<SQLLM_F16>::unpack<3>(c[d], 1.f)};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const size_t j = (size_t)(32 * b + 8 * d + 2 * k) * a.B + t;
                    part = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2_t, w[k]), half2_t{x[j], x[j + a.B]}, part, false);
                }
            }
            const u32 s = scales[b];
            sum = __builtin_fmaf(s == 255u ? __builtin_nanf("") : __builtin_ldexpf(1.f, (int)s - 127), part, sum);
        }
#pragma unroll
        for (int m = 32; m; m >>= 1) sum += __shfl_xor(sum, m);
        if (lane == 0) {
            half_t* y = static_cast<half_t*>(a.y) + row * a.B + t;
            *y = (half_t)(a.accumulate ? (float)*y + sum : sum);
        }
    }
}

// ---------------------------------------------------------------------------------------------- launchers
namespace {

bool vector_rows(const void* p, long long ld, int size) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * size % 16 == 0; }

template <int TYPE>
hipError_t quantize(const MxQuantArgs& a, hipStream_t s) {
    const bool vec = vector_rows(a.w, a.ldw, mx_type_size(TYPE));
    const size_t cp = mx_row_code_bytes(a.N), sp = mx_row_scale_bytes(a.N);
    if (a.codes_t) {
        const int tiles_n = mx_padded(a.N) / kTile, tiles_m = mx_padded(a.M) / kTile;
        const size_t cpt = mx_row_code_bytes(a.M), spt = mx_row_scale_bytes(a.M);
        const unsigned lds = kTile * (kTile / 8) * MxEight<TYPE>::kDwords * 4;
        const dim3 grid((unsigned)((long long)tiles_m * tiles_n));
        if (vec && a.codes) mx_quantize_tile_kernel<TYPE, true, true><<<grid, kThreads, lds, s>>>(a, tiles_n, cp, sp, cpt, spt);
        else if (vec) mx_quantize_tile_kernel<TYPE, true, false><<<grid, kThreads, lds, s>>>(a, tiles_n, cp, sp, cpt, spt);
        else if (a.codes) mx_quantize_tile_kernel<TYPE, false, true><<<grid, kThreads, lds, s>>>(a, tiles_n, cp, sp, cpt, spt);
        else mx_quantize_tile_kernel<TYPE, false, false><<<grid, kThreads, lds, s>>>(a, tiles_n, cp, sp, cpt, spt);
    } else {
        const RowShape rs = row_shape(mx_padded(a.N) / 8);
        if (vec) mx_quantize_rows_kernel<TYPE, true><<<row_grid(rs, a.M), kThreads, 0, s>>>(a, rs, cp, sp);
        else mx_quantize_rows_kernel<TYPE, false><<<row_grid(rs, a.M), kThreads, 0, s>>>(a, rs, cp, sp);
    }
    return hipGetLastError();
}

template <int TYPE>
hipError_t dequantize(const MxDequantArgs& a, hipStream_t s) {
    const RowShape rs = row_shape(((long long)a.N + 7) / 8);
    const size_t cp = mx_row_code_bytes(a.N), sp = mx_row_scale_bytes(a.N);
    if (vector_rows(a.w, a.ldw, mx_type_size(TYPE))) mx_dequantize_kernel<TYPE, true><<<row_grid(rs, a.M), kThreads, 0, s>>>(a, rs, cp, sp);
    else mx_dequantize_kernel<TYPE, false><<<row_grid(rs, a.M), kThreads, 0, s>>>(a, rs, cp, sp);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quantize(const MxQuantArgs& a, hipStream_t s) {
    return a.type == SQLLM_F16 ? quantize<SQLLM_F16>(a, s) : a.type == SQLLM_BF16 ? quantize<SQLLM_BF16>(a, s) : quantize<SQLLM_F32>(a, s);
}

hipError_t launch_mx_dequantize(const MxDequantArgs& a, hipStream_t s) {
    return a.type == SQLLM_F16 ? dequantize<SQLLM_F16>(a, s) : a.type == SQLLM_BF16 ? dequantize<SQLLM_BF16>(a, s) : dequantize<SQLLM_F32>(a, s);
}

hipError_t launch_mx_gemv(const MxGemvArgs& a, hipStream_t s) {
    if (a.B == 1) {
        const int waves = (a.N + 2047) / 2048;
        const int resident = 256 * (24 / waves);                     // workgroups that run side by side
        const int rows = (int)std::min<long long>(kGemvMaxRows, std::max<long long>(1, ((long long)a.M + 4ll * resident - 1) / (4ll * resident)) * 4);
        mx_gemv_kernel<<<dim3((unsigned)(((long long)a.M + rows - 1) / rows)), waves * 64, 0, s>>>(a, rows);
    } else {
        mx_gemv_columns_kernel<<<dim3((unsigned)(((long long)a.M + 3) / 4)), kThreads, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace sqllm
