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
// Two to sixteen columns, on the matrix cores.  v_mfma_f32_16x16x32_f16 multiplies 16 rows of W x 32 columns by 32 rows of x x 16 columns: lane
// (r, q) = (l % 16, l / 16) supplies eight neighbouring weights of row r and the same eight rows of x in column r, and keeps rows 4 q + e of column r.
// A workgroup owns 16 RG rows; its waves deal the windows of 128 columns out among themselves.  Lane (r, q) holds block q of row r of a window
// (16 bytes and one scale), converted with its scale to fp16, eights 0..3 for instructions 0..3; the window's 128 rows of x go through the wave's own
// LDS, where they are padded to a multiple of four columns and read back transposed.  What columns past B hold reaches columns that are not stored.
//
// With its scale a code is an fp16 number for scale bytes 114 .. 140 (0.5 x 2^-13 .. 6 x 2^13).  A block with a byte of 60 or less adds less than
// 28672 x 65504 x 6 x 2^(60 - 127) < 2^-32 to any result, far below half the smallest fp16 number, and becomes zeros.  Other bytes
// (weights of other magnitudes, NaN) send the window to a slower form: one instruction per block with the codes alone, its result times the scale in fp32.
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int kWindow = 128, kBatchMaxWaves = 16;

constexpr int batch_pitch(int B) { return (B + 3) / 4 * 4; }                     // halves of a row of x in LDS
constexpr int batch_stage_bytes(int B) { return kWindow * batch_pitch(B) * 2 + (batch_pitch(B) < 16 ? 32 : 0); }   // short rows are read as if they had 16 columns
static_assert(kBatchMaxWaves * batch_stage_bytes(16) <= 65536 && batch_stage_bytes(12) <= batch_stage_bytes(16), "the staging areas fit a launch's LDS");

template <int B, int RG>
__global__ void __launch_bounds__(kBatchMaxWaves * 64) mx_gemv_batch_kernel(MxGemvArgs a) {
    constexpr int P = batch_pitch(B), L = (B + 3) / 4;               // 16-byte pieces of a window per lane
    constexpr int PER = B % 4 == 0 ? 1 : B % 2 == 0 ? 4 : 8;          // LDS writes a piece takes
    extern __shared__ __align__(16) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), nw = blockDim.x >> 6;
    const int r = lane & 15, q = lane >> 4;
    const long long r0 = (long long)blockIdx.x * (16 * RG);
    const int nwin = a.N / kWindow;
    char* stage = smem + wave * batch_stage_bytes(B);
    const u32x4* codes[RG];
    const uint8_t* scales[RG];
#pragma unroll
    for (int g = 0; g < RG; ++g) {
        const size_t row = (size_t)min(r0 + 16 * g + r, (long long)a.M - 1);
        codes[g] = reinterpret_cast<const u32x4*>(static_cast<const char*>(a.codes) + row * (a.N / 2)) + q;
        scales[g] = static_cast<const uint8_t*>(a.scales) + row * (a.N / kMxBlock) + q;
    }
    const u32x4* x = static_cast<const u32x4*>(a.x);
    int piece[L];
    u32 at[L][PER];
#pragma unroll
    for (int i = 0; i < L; ++i) {
        piece[i] = min(lane + 64 * i, 16 * B - 1);                   // surplus lanes repeat the last piece
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const u32 e = 8u * piece[i] + j * (8 / PER);
            at[i][j] = 2 * (e / B * P + e % B);
        }
    }
    u32x4 next_codes[RG], next_x[L];
    u32 next_scale[RG];
    auto fetch = [&](int t) {
#pragma unroll
        for (int g = 0; g < RG; ++g) {
            next_codes[g] = __builtin_nontemporal_load(codes[g] + 4 * t);
            next_scale[g] = __builtin_nontemporal_load(scales[g] + 4 * t);
        }
#pragma unroll
        for (int i = 0; i < L; ++i) next_x[i] = x[(size_t)t * (16 * B) + piece[i]];
    };
    f32x4 acc[RG] = {};
    const u32 from = 2 * ((32 * q + (r >> 2)) * P + 4 * (r & 3));
    if (wave < nwin) fetch(wave);
    for (int t = wave; t < nwin; t += nw) {
        u32x4 c[RG];
        u32 s[RG];
        bool plain = true;
#pragma unroll
        for (int g = 0; g < RG; ++g) {
            c[g] = next_codes[g];
            s[g] = next_scale[g];
            plain = plain && (s[g] <= 60u || s[g] - 114u <= 26u);
        }
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const u32x4 v = next_x[i];
            if constexpr (PER == 1) {
                *reinterpret_cast<u32x4*>(stage + at[i][0]) = v;
            } else if constexpr (PER == 4) {
#pragma unroll
                for (int j = 0; j < 4; ++j) *reinterpret_cast<u32*>(stage + at[i][j]) = v[j];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) *reinterpret_cast<uint16_t*>(stage + at[i][j]) = (uint16_t)(v[j >> 1] >> (16 * (j & 1)));
            }
        }
        fetch(min(t + nw, nwin - 1));
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        half8_t xb[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(stage + from + 16 * m * P));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(stage + from + 16 * m * P + 8 * P));
            xb[m] = __builtin_bit_cast(half8_t, (__attribute__((ext_vector_type(8))) short){lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w});
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        auto weights = [&](u32 codes8, float scale) {
            const u32x4 w = {MxType<SQLLM_F16>::unpack<0>(codes8, scale), MxType<SQLLM_F16>::unpack<1>(codes8, scale), MxType<SQLLM_F16>::unpack<2>(codes8, scale),
                             MxType<SQLLM_F16>::unpack<3>(codes8, scale)};
            return __builtin_bit_cast(half8_t, w);
        };
        if (__builtin_amdgcn_ballot_w64(!plain) == 0) {
#pragma unroll
            for (int g = 0; g < RG; ++g)
#pragma unroll
                for (int m = 0; m < 4; ++m) acc[g] = __builtin_amdgcn_mfma_f32_16x16x32_f16(weights(c[g][m], mx_scale(s[g])), xb[m], acc[g], 0, 0, 0);
        } else {
#pragma unroll
            for (int g = 0; g < RG; ++g)
                for (int b = 0; b < 4; ++b) {                        // the lanes that hold block b of their rows; the others supply zeros
                    f32x4 d = {};
#pragma unroll
                    for (int m = 0; m < 4; ++m) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(weights(q == b ? c[g][m] : 0u, 1.f), xb[m], d, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[g][e] = __builtin_fmaf(scale_factor(__shfl(s[g], 16 * b + 4 * q + e)), d[e], acc[g][e]);
                }
        }
    }
    __syncthreads();
    float* part = reinterpret_cast<float*>(smem);                    // [wave][row][column]
#pragma unroll
    for (int g = 0; g < RG; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[wave * (RG * 256) + (16 * g + 4 * q + e) * 16 + r] = acc[g][e];
    __syncthreads();
    for (int i = tid; i < 16 * RG * 16; i += blockDim.x) {
        const long long row = r0 + (i >> 4);
        if ((i & 15) < B && row < a.M) {
            float sum = 0.f;
            for (int w = 0; w < nw; ++w) sum += part[w * (RG * 256) + i];
            half_t* y = static_cast<half_t*>(a.y) + row * B + (i & 15);
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

namespace {

template <int B, int RG>
hipError_t gemv_batch(const MxGemvArgs& a, hipStream_t s) {
    const long long groups = ((long long)a.M + 16 * RG - 1) / (16 * RG);
    int waves = (int)std::min<long long>(kBatchMaxWaves, std::max<long long>(4, 4096 / groups));   // sixteen waves to a compute unit
    waves = std::min(waves, std::max(1, a.N / kWindow));
    const size_t lds = (size_t)waves * std::max(batch_stage_bytes(B), RG * 1024);
    mx_gemv_batch_kernel<B, RG><<<dim3((unsigned)groups), waves * 64, lds, s>>>(a);
    return hipGetLastError();
}

template <int B>
hipError_t gemv_batch(const MxGemvArgs& a, hipStream_t s) {
    if constexpr (B > 1) {
        if (a.B < B) return gemv_batch<B - 1>(a, s);
        return a.M > 16 * 256 ? gemv_batch<B, 2>(a, s) : gemv_batch<B, 1>(a, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_mx_gemv(const MxGemvArgs& a, hipStream_t s) {
    if (a.B > 1) return gemv_batch<SQLLM_MAX_BATCH>(a, s);
    const int waves = (a.N + 2047) / 2048;
    const int resident = 256 * (24 / waves);                         // workgroups that run side by side
    const int rows = (int)std::min<long long>(kGemvMaxRows, std::max<long long>(1, ((long long)a.M + 4ll * resident - 1) / (4ll * resident)) * 4);
    mx_gemv_kernel<<<dim3((unsigned)(((long long)a.M + rows - 1) / rows)), waves * 64, 0, s>>>(a, rows);
    return hipGetLastError();
}

}  // namespace sqllm
