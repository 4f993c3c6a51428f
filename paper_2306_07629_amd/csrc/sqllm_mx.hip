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
inline dim3 row_grid(const RowShape& r, long long M) {
    const long long groups = (M + (kThreads >> r.log_tpr) - 1) / (kThreads >> r.log_tpr);
    return dim3((unsigned)((r.chunks + (1 << r.log_tpr) - 1) >> r.log_tpr), (unsigned)(groups < 65535 ? groups : 65535));
}

// AHEAD: rows a thread requests before it quantises the first.
template <int TYPE, int AHEAD>
__global__ void __launch_bounds__(kThreads) mx_quantize_rows_kernel(MxQuantArgs a, RowShape rs, size_t code_pitch, size_t scale_pitch) {
    const int chunk = (int)(blockIdx.x << rs.log_tpr) + (int)(threadIdx.x & ((1u << rs.log_tpr) - 1));
    if (chunk >= rs.chunks) return;                                  // whole quads: chunks is a multiple of 16
    const int rows = kThreads >> rs.log_tpr, j0 = 8 * chunk;
    typedef typename MxType<TYPE>::value value;
    const long long step = (long long)gridDim.y * rows;
    for (long long r = (long long)blockIdx.y * rows + (threadIdx.x >> rs.log_tpr); r < a.M; r += AHEAD * step) {
        MxEight<TYPE> e[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (r + k * step < a.M) e[k].load(static_cast<const value*>(a.w) + (r + k * step) * a.ldw, j0, a.N);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (r + k * step >= a.M) break;
            e[k].settle(j0, a.N);
            const u32 byte = mx_scale_byte(mx_magnitude<TYPE>(quad_max(e[k].top())));
            reinterpret_cast<u32*>(static_cast<char*>(a.codes) + (r + k * step) * code_pitch)[chunk] = e[k].pack(byte);
            if ((chunk & 3) == 0) (static_cast<uint8_t*>(a.scales) + (r + k * step) * scale_pitch)[chunk >> 2] = (uint8_t)byte;
        }
    }
}

// Sixteen bytes of the result to a thread: eight elements, or four in fp32, so that neighbouring lanes write whole lines with one store.
template <int TYPE>
__global__ void __launch_bounds__(kThreads) mx_dequantize_kernel(MxDequantArgs a, RowShape rs, size_t code_pitch, size_t scale_pitch) {
    constexpr int E = TYPE == SQLLM_F32 ? 4 : 8;
    const int chunk = (int)(blockIdx.x << rs.log_tpr) + (int)(threadIdx.x & ((1u << rs.log_tpr) - 1));
    if (chunk >= rs.chunks) return;
    const int rows = kThreads >> rs.log_tpr, j0 = E * chunk, left = a.N - j0;
    typedef typename MxType<TYPE>::value value;
    for (long long r = (long long)blockIdx.y * rows + (threadIdx.x >> rs.log_tpr); r < a.M; r += (long long)gridDim.y * rows) {
        const char* codes = static_cast<const char*>(a.codes) + r * code_pitch;
        const u32 byte = (static_cast<const uint8_t*>(a.scales) + r * scale_pitch)[j0 / kMxBlock];
        value* dst = static_cast<value*>(a.w) + r * a.ldw + j0;
        MxEight<TYPE> e;
        if constexpr (TYPE == SQLLM_F32) {
            e.unpack(reinterpret_cast<const uint16_t*>(codes)[chunk], byte);
            if (left >= 4) __builtin_nontemporal_store(u32x4{e.v[0], e.v[1], e.v[2], e.v[3]}, reinterpret_cast<u32x4_a4*>(dst));
            else e.store_some(dst, left);
        } else {
            e.unpack(reinterpret_cast<const u32*>(codes)[chunk], byte);
            if (left >= 8) e.store(dst);
            else e.store_some(dst, left);
        }
    }
}

// ---------------------------------------------------------------------------------------------- columns: quantise the transpose
// A workgroup takes a tile of 128 x 128 elements through LDS: eights of the rows go in as they are loaded (and, where the row direction is
// asked for too, are quantised on the way, so w is read once for both), then every thread walks down 32 rows of a column, or of two.  Codes and
// scales of the columns, and scales of the rows, are gathered in LDS and leave four neighbouring bytes, or sixteen, to a lane: a byte of a row of
// its own from every lane took longer (5120 x 5120 fp16, both directions: 28.0
// against 24.8 us; with the loads past the caches 21.8).  Within a sixth of the copy rate for 4096 x 11008 (bf16 32.9 us, fp32, of whose tiles two fit a compute unit, 51.2);
// below some tiles to a compute unit one tile's chain shows (1999 x 5120: 10.3 for 6.4 us in bf16, 16.4 for 10.6 in fp32).
constexpr int kTile = 128;

template <int TYPE, bool ROWS>
__global__ void __launch_bounds__(kThreads) mx_quantize_tile_kernel(MxQuantArgs a, int tiles_m, int tiles_n, int first, size_t code_pitch, size_t scale_pitch, size_t code_pitch_t, size_t scale_pitch_t) {
    typedef typename MxType<TYPE>::value value;
    constexpr int D = MxEight<TYPE>::kDwords, kPitch = kTile / 8 * D;   // dwords of a row
    extern __shared__ __align__(16) u32 tile[];
    __shared__ u32 row_scales[kTile], column_scales[kTile];          // the four scale bytes of a row, of a column
    const int tid = threadIdx.x;
    // the XCDs, to which workgroups are handed in turn, take contiguous ranges of the tiles in bands of eight columns of them: neighbours, whose outputs
    // share cache lines, write through the same L2
    const int tiles = tiles_m * tiles_n, xcd = blockIdx.x & 7;
    const int p = (int)((long long)tiles * xcd >> 3) + first + (int)(blockIdx.x >> 3);
    if (p >= (int)((long long)tiles * (xcd + 1) >> 3)) return;
    const int band = p / (8 * tiles_m), at = p % (8 * tiles_m), wide = min(tiles_n - 8 * band, 8);
    const long long m0 = (long long)(at / wide) * kTile;
    const int n0 = (8 * band + at % wide) * kTile, chunk = tid & 15;
    MxEight<TYPE> in[kTile / 16];                                    // all of a thread's share on its way before the first is used
    const value* const w = static_cast<const value*>(a.w);
    if (a.N >= 8) {
        const int j = min(n0 + 8 * chunk, a.N - 8);
#pragma unroll
        for (int p = 0; p < kTile / 16; ++p) in[p].load(w + min(m0 + 16 * p + (tid >> 4), (long long)a.M - 1) * a.ldw + j);
    } else {
#pragma unroll
        for (int p = 0; p < kTile / 16; ++p) in[p].load_some(w + min(m0 + 16 * p + (tid >> 4), (long long)a.M - 1) * a.ldw, chunk == 0 ? a.N : 0);
    }
#pragma unroll
    for (int p = 0; p < kTile / 16; ++p) {
        const int row = 16 * p + (tid >> 4);
        in[p].settle(n0 + 8 * chunk, a.N);
        if (m0 + row >= a.M) in[p].clear();
        in[p].to_lds(tile + row * kPitch + chunk * D);
        if (ROWS) {
            const u32 byte = mx_scale_byte(mx_magnitude<TYPE>(quad_max(in[p].top())));
            const u32 packed = in[p].pack(byte);
            if (m0 + row < a.M) reinterpret_cast<u32*>(static_cast<char*>(a.codes) + (m0 + row) * code_pitch)[n0 / 8 + chunk] = packed;
            if ((chunk & 3) == 0) reinterpret_cast<uint8_t*>(row_scales)[4 * row + (chunk >> 2)] = (uint8_t)byte;
        }
    }
    __syncthreads();
    u32x4 out[2];                                                    // codes of block b of two columns
    int column[2], block[2];
    auto take = [&](int k, int col, int b, const MxEight<TYPE> (&e)[4]) {
        const u32 byte = mx_scale_byte(mx_magnitude<TYPE>(max(max(e[0].top(), e[1].top()), max(e[2].top(), e[3].top()))));
        out[k] = u32x4{e[0].pack(byte), e[1].pack(byte), e[2].pack(byte), e[3].pack(byte)};
        column[k] = col; block[k] = b;
        reinterpret_cast<uint8_t*>(column_scales)[4 * col + b] = (uint8_t)byte;
    };
    if constexpr (TYPE == SQLLM_F32) {
        const int col = tid & 127;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int b = (tid >> 7) + 2 * k;
            MxEight<TYPE> e[4];
#pragma unroll
            for (int i = 0; i < 32; ++i) e[i >> 3].v[i & 7] = tile[(32 * b + i) * kPitch + col];
            take(k, col, b, e);
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
        take(0, 2 * pair, b, lo);
        take(1, 2 * pair + 1, b, hi);
    }
    __syncthreads();                                                 // the tile is read: its place takes the codes of the columns, 64 bytes each
    // block b of column c at position b ^ (c / 2): neighbouring lanes write and read different banks
#pragma unroll
    for (int k = 0; k < 2; ++k) *reinterpret_cast<u32x4*>(tile + 16 * column[k] + 4 * (block[k] ^ ((column[k] >> 1) & 3))) = out[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int col = (tid >> 2) + 64 * k, b = tid & 3;
        if (n0 + col < a.N)
            *reinterpret_cast<u32x4*>(static_cast<char*>(a.codes_t) + (size_t)(n0 + col) * code_pitch_t + m0 / 2 + 16 * b) = *reinterpret_cast<const u32x4*>(tile + 16 * col + 4 * (b ^ ((col >> 1) & 3)));
    }
    if (tid < kTile) {
        if (n0 + tid < a.N) *reinterpret_cast<u32*>(static_cast<char*>(a.scales_t) + (size_t)(n0 + tid) * scale_pitch_t + m0 / 32) = column_scales[tid];
    } else if (ROWS) {
        const int row = tid - kTile;
        if (m0 + row < a.M) *reinterpret_cast<u32*>(static_cast<char*>(a.scales) + (m0 + row) * scale_pitch + n0 / 32) = row_scales[row];
    }
}

// ---------------------------------------------------------------------------------------------- a few fp16 columns
// One or two columns: wave w of a workgroup owns columns [2048 w, 2048 w + 2048) of W, lane l block 64 w + l of every row, and keeps the 32 rows of x of
// its block in 16 registers per column of x while it walks down the workgroup's rows, R at a time with the next R requested.  The codes are converted
// without their scale (every code is an fp16 number), so a block's sum is formed as for fp16 weights, and enters the row's sum times the scale in
// fp32: no scale byte leaves a range.  Bound by reads: 22016 x 8192 from HBM 21.6 us (4.4 TB/s; its bytes at the rate of a copy 19.6), from a warm last-level cache 20.1; two
// columns, with twice the dot products to a row's bytes, 25.5 and 24.6.
template <int R>
struct BlockRows {
    u32x4 codes[R];
    u32 scale[R];
};

template <int B>
__device__ __forceinline__ void block_dot(const u32x4& c, const u32 (&x)[B][16], float (&sum)[B]) {
    float odd[B];
#pragma unroll
    for (int t = 0; t < B; ++t) sum[t] = odd[t] = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const half2_t w[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c[d], 1.f, 0), __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c[d], 1.f, 1),
                              __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c[d], 1.f, 2), __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c[d], 1.f, 3)};
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int t = 0; t < B; ++t) {
                float& s = k & 1 ? odd[t] : sum[t];
                s = __builtin_amdgcn_fdot2(w[k], __builtin_bit_cast(half2_t, x[t][4 * d + k]), s, false);
            }
    }
#pragma unroll
    for (int t = 0; t < B; ++t) sum[t] += odd[t];
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

constexpr int kGemvMaxWaves = 14, kGemvMaxSums = 128;                 // sums of a workgroup: rows x columns of x
constexpr int kGemvColumns = 2;

template <int B, int R>
__global__ void __launch_bounds__(kGemvMaxWaves * 64) mx_gemv_kernel(MxGemvArgs a, int rows) {
    __shared__ float part[kGemvMaxWaves * kGemvMaxSums];             // [row][column][wave]
    constexpr int V = (R * B + 3) / 4 * 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), nw = blockDim.x >> 6;
    const long long r0 = (long long)blockIdx.x * rows;
    const int n = (int)min((long long)rows, a.M - r0);
    const int nb = a.N / kMxBlock, block = 64 * wave + lane;
    const bool inside = block < nb;
    const int b = min(block, nb - 1);                                // surplus lanes read the last block and multiply with zeros
    const char* codes = static_cast<const char*>(a.codes) + (size_t)r0 * (a.N / 2);
    const uint8_t* scales = static_cast<const uint8_t*>(a.scales) + (size_t)r0 * nb;
    auto load = [&](int r, BlockRows<R>& f) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int row = min(r + k, n - 1);
            f.codes[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(codes + (size_t)row * (a.N / 2)) + b);
            f.scale[k] = __builtin_nontemporal_load(scales + (size_t)row * nb + b);
        }
    };
    u32 x[B][16];                                                    // rows 2 k, 2 k + 1 of column t as a pair
    {
        const u32x4* src = reinterpret_cast<const u32x4*>(static_cast<const half_t*>(a.x) + (size_t)(32 * B) * b);
        u32 v[16 * B];
#pragma unroll
        for (int k = 0; k < 4 * B; ++k) {
            const u32x4 t = src[k];
            v[4 * k] = t.x; v[4 * k + 1] = t.y; v[4 * k + 2] = t.z; v[4 * k + 3] = t.w;
        }
#pragma unroll
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int t = 0; t < B; ++t) {
                const int lo = 2 * k * B + t, hi = lo + B;           // positions among the lane's halves
                x[t][k] = B == 1 ? v[k] : __builtin_amdgcn_perm(v[hi / 2], v[lo / 2], (hi & 1 ? 0x07060000u : 0x05040000u) | (lo & 1 ? 0x0302u : 0x0100u));
            }
    }
    BlockRows<R> now, next;
    load(0, now);
    const int group = lane >> 4, slot = (group >> 1) | (group & 1) << 1;   // whose sum the lane holds after wave_sums
    for (int r = 0; r < n; r += R) {
        if (r + R < n) load(r + R, next);
        float v[V];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            float sum[B];
            block_dot<B>(now.codes[k], x, sum);
            const float f = scale_factor(now.scale[k]);
#pragma unroll
            for (int t = 0; t < B; ++t) v[k * B + t] = inside ? sum[t] * f : 0.f;
        }
#pragma unroll
        for (int k = R * B; k < V; ++k) v[k] = 0.f;
#pragma unroll
        for (int k = 0; k < V; k += 4) {
            const float four[4] = {v[k], v[k + 1], v[k + 2], v[k + 3]};
            const float s = wave_sums(four);
            if ((lane & 15) == 0 && k + slot < R * B) part[(r * B + k + slot) * nw + wave] = s;
        }
        now = next;
    }
    __syncthreads();
    for (int i = tid; i < n * B; i += blockDim.x) {
        float s = 0.f;
        for (int w = 0; w < nw; ++w) s += part[i * nw + w];
        half_t* y = static_cast<half_t*>(a.y) + r0 * B + i;
        *y = (half_t)(a.accumulate ? (float)*y + s : s);
    }
}

// Three to sixteen columns, on the matrix cores.  v_mfma_f32_16x16x32_f16 multiplies 16 rows of W x 32 columns by 32 rows of x x 16 columns: lane
// (r, q) = (l % 16, l / 16) supplies eight neighbouring weights of row r and the same eight rows of x in column r, and keeps rows 4 q + e of column r.
// A workgroup owns 16 G rows, each of its eight waves an equal share of the columns: n <= NS steps of 128 (in rounds of 8 x 8 steps where there are more).
// Lane (r, q) takes block q of row r of every step, converted with its scale to fp16, eights 0..3 for instructions 0..3; the scales of a step are fetched
// four lanes to a row and change lanes when they are used.  The wave's rows of x are read once per round, go through the wave's own LDS (padded there to a multiple of four columns) to
// be transposed, and stay in 16 NS registers while the wave walks down the groups of 16 rows, RING of them ahead of itself with its requests.
// What columns past B hold reaches columns that are not stored.  8192 x 8192 times 16 takes 15.4 us with weights from HBM and 11.4 from the last-level cache, times 3 13.2
// and 8.9 (the bytes at the rate of a copy: 7.4): launch and x in place, then reads.
//
// With its scale a code is an fp16 number for scale bytes 114 .. 140 (0.5 x 2^-13 .. 6 x 2^13).  A block with a byte of 60 or less adds less than
// 28672 x 65504 x 6 x 2^(60 - 127) < 2^-32 to any result, far below half the smallest fp16 number, and becomes zeros.  Other bytes
// (weights of other magnitudes, NaN) send the window to a slower form: one instruction per block with the codes alone, its result times the scale in fp32.
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int kBatchWaves = 8;

constexpr int batch_pitch(int B) { return (B + 3) / 4 * 4; }                     // halves of a row of x in LDS
constexpr int batch_stage_bytes(int B) { return 128 * batch_pitch(B) * 2 + (batch_pitch(B) < 16 ? 32 : 0); }   // short rows are read as if they had 16 columns

__device__ __forceinline__ void wave_fence() {                       // orders the LDS accesses of one wave
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <int NS>
struct BatchCodes {                                                  // a lane's blocks of one group of rows
    u32x4 c[NS];
    u32 scale[(NS + 3) / 4];                                         // row lane / 4, scales of steps lane % 4, lane % 4 + 4
};

__device__ __forceinline__ half8_t fp16_weights(u32 codes, float scale) {
    const u32x4 w = {MxType<SQLLM_F16>::unpack<0>(codes, scale), MxType<SQLLM_F16>::unpack<1>(codes, scale), MxType<SQLLM_F16>::unpack<2>(codes, scale),
                     MxType<SQLLM_F16>::unpack<3>(codes, scale)};
    return __builtin_bit_cast(half8_t, w);
}

// acc += 16 rows x 128 n columns of W times x
template <int NS>
__device__ __forceinline__ f32x4 batch_product(const BatchCodes<NS>& w, const half8_t (&xb)[NS][4], f32x4 acc, int n, int r, int q) {
    u32 byte[NS];
    bool plain = true;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        byte[s] = ((u32)__shfl((int)w.scale[s >> 2], 4 * r + (s & 3)) >> (8 * q)) & 255u;
        plain = plain && (byte[s] <= 60u || byte[s] - 114u <= 26u);
    }
    if (__builtin_amdgcn_ballot_w64(!plain) == 0) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            if (s >= n) continue;                                    // uniform
            const float scale = mx_scale(byte[s]);
#pragma unroll
            for (int m = 0; m < 4; ++m) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(fp16_weights(w.c[s][m], scale), xb[s][m], acc, 0, 0, 0);
        }
    } else {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            if (s >= n) continue;
#pragma unroll 1
            for (int b = 0; b < 4; ++b) {                            // the lanes with q = b; the others supply zeros
                f32x4 d = {};
#pragma unroll
                for (int m = 0; m < 4; ++m) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(fp16_weights(q == b ? w.c[s][m] : 0u, 1.f), xb[s][m], d, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(scale_factor(__shfl(byte[s], 16 * b + 4 * q + e)), d[e], acc[e]);
            }
        }
    }
    return acc;
}

template <int B, int NS, int RING>
__global__ void __launch_bounds__(kBatchWaves * 64, 2) mx_gemv_batch_kernel(MxGemvArgs a, int G, int share) {
    constexpr int P = batch_pitch(B);
    extern __shared__ __align__(16) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, q = lane >> 4;
    const long long r0 = (long long)blockIdx.x * (16 * G);
    const int groups = (int)min((long long)G, (a.M - r0 + 15) / 16);
    const int nb = a.N / kMxBlock, total = nb / 4;                   // blocks of a row, steps of a row (and dwords of its scales)
    char* const stage = smem + wave * batch_stage_bytes(B);
    float* const part = reinterpret_cast<float*>(smem + kBatchWaves * batch_stage_bytes(B)) + wave * (G * 256) + 64 * q + r;   // [wave][row][column]
    for (int round = 0; round * kBatchWaves * share < total; ++round) {
        const int first = min((round * kBatchWaves + wave) * share, total);   // the wave's first step
        const int n = min(share, total - first);                     // uniform; may be 0
        long long top = r0;
        asm volatile("" : "+s"(top));                                // rows' addresses made anew each round: kept, they were spilled, and waited for x on their way back (8192 x 8192 times 5, weights from HBM: 15.3 us, now 13.4)
        auto fetch = [&](int g, BatchCodes<NS>& d) {
            const size_t row = (size_t)min(top + 16 * g + r, (long long)a.M - 1);
            const u32x4* codes = reinterpret_cast<const u32x4*>(static_cast<const char*>(a.codes) + row * (a.N / 2)) + 4 * first + q;
#pragma unroll
            for (int s = 0; s < NS; ++s)
                if (s < n) d.c[s] = codes[4 * s];
            const size_t srow = (size_t)min(top + 16 * g + (lane >> 2), (long long)a.M - 1);
            const u32* scales = reinterpret_cast<const u32*>(static_cast<const char*>(a.scales) + srow * nb);
#pragma unroll
            for (int k = 0; k < (NS + 3) / 4; ++k) d.scale[k] = scales[min(first + min(4 * k + (lane & 3), max(n, 1) - 1), total - 1)];
        };
        BatchCodes<NS> ring[RING];
        half8_t xb[NS][4];
        {
            // x: lane l fetches rows 2 l and 2 l + 1 of a step (B dwords); rows of 4, 8, 12 or 16 need no padding, and the step goes to LDS as it lies, sixteen
            // neighbouring bytes to a lane (weights from HBM: 8192 x 8192 times 16 17.1 us, now 15.4; 4096 x 14336 20.7, now 17.0)
            constexpr bool kWhole = P == B;
            const u32* x = static_cast<const u32*>(a.x) + (size_t)B * (64 * min(first, total - 1) + lane);
            constexpr int C = NS * B <= 36 ? NS : 4, EARLY = NS == 8 ? 1 : RING;   // steps of x requested ahead, groups of codes before x is in place: what 256 registers hold
            u32 v[NS][B];
            auto fetch_x = [&](int s) {
                const int step = min(s, max(n, 1) - 1);
                if constexpr (kWhole) {
#pragma unroll
                    for (int i = 0; i < B; i += 4) {
                        const u32x4 t = reinterpret_cast<const u32x4*>(a.x)[(size_t)(16 * B) * (min(first, total - 1) + step) + 16 * i + lane];
                        v[s][i] = t.x; v[s][i + 1] = t.y; v[s][i + 2] = t.z; v[s][i + 3] = t.w;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < B; ++i) v[s][i] = x[(size_t)B * (64 * step) + i];
                }
            };
#pragma unroll
            for (int s = 0; s < C && s < NS; ++s) fetch_x(s);
            asm volatile("" ::: "memory");                           // keeps the requests in this order: x, whose transposition the codes outlast, then these
#pragma unroll
            for (int i = 0; i < EARLY; ++i)
                if (i < groups) fetch(i, ring[i]);
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                asm volatile("" ::: "memory");
                if constexpr (kWhole) {
#pragma unroll
                    for (int i = 0; i < B; i += 4) *reinterpret_cast<u32x4*>(stage + 16 * (16 * i + lane)) = u32x4{v[s][i], v[s][i + 1], v[s][i + 2], v[s][i + 3]};
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        u32 row[P / 2];
#pragma unroll
                        for (int i = 0; i < P / 2; ++i) {
                            const int at = h * B + 2 * i;                // halves from the lane's first on
                            row[i] = 2 * i >= B ? 0u : at % 2 == 0 ? v[s][at / 2] : __builtin_amdgcn_alignbyte(at / 2 + 1 < B ? v[s][at / 2 + 1] : 0u, v[s][at / 2], 2);
                        }
#pragma unroll
                        for (int i = 0; i < P / 4; ++i) *reinterpret_cast<u32x2*>(stage + 2 * P * (2 * lane + h) + 8 * i) = u32x2{row[2 * i], row[2 * i + 1]};
                    }
                }
                wave_fence();
                const u32 from = 2 * ((32 * q + (r >> 2)) * P + 4 * (r & 3));
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(stage + from + 16 * m * P));
                    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(stage + from + 16 * m * P + 8 * P));
                    xb[s][m] = __builtin_bit_cast(half8_t, (__attribute__((ext_vector_type(8))) short){lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w});
                }
                wave_fence();
                if (s + C < NS) fetch_x(s + C);
            }
#pragma unroll
            for (int i = EARLY; i < RING; ++i)
                if (i < groups) fetch(i, ring[i]);
        }
#pragma unroll 1
        for (int g0 = 0; g0 < groups; g0 += RING) {
#pragma unroll
            for (int j = 0; j < RING; ++j) {
                const int g = g0 + j;
                if (g < groups) {                                    // uniform
                    float* out = part + 256 * g;
                    f32x4 acc;
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[e] = round == 0 ? 0.f : out[16 * e];
                    acc = batch_product<NS>(ring[j], xb, acc, n, r, q);
                    if (g + RING < groups) fetch(g + RING, ring[j]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) out[16 * e] = acc[e];
                }
            }
        }
    }
    __syncthreads();
    const float* all = reinterpret_cast<const float*>(smem + kBatchWaves * batch_stage_bytes(B));
    for (int i = tid; i < 16 * G * 16; i += kBatchWaves * 64) {
        const long long row = r0 + (i >> 4);
        if ((i & 15) < B && row < a.M) {
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < kBatchWaves; ++w) sum += all[w * (G * 256) + i];
            half_t* y = static_cast<half_t*>(a.y) + row * B + (i & 15);
            *y = (half_t)(a.accumulate ? (float)*y + sum : sum);
        }
    }
}

// ---------------------------------------------------------------------------------------------- launchers
namespace {

template <int TYPE>
hipError_t quantize(const MxQuantArgs& a, hipStream_t s) {
    const size_t cp = mx_row_code_bytes(a.N), sp = mx_row_scale_bytes(a.N);
    if (a.codes_t) {
        const int tiles_n = mx_padded(a.N) / kTile, tiles_m = mx_padded(a.M) / kTile;
        const size_t cpt = mx_row_code_bytes(a.M), spt = mx_row_scale_bytes(a.M);
        const unsigned lds = kTile * (kTile / 8) * MxEight<TYPE>::kDwords * 4;
        if (lds > 65536 - 2048) {                                    // with the scales above what a launch gets without asking
            const hipError_t e = hipFuncSetAttribute(a.codes ? reinterpret_cast<const void*>(&mx_quantize_tile_kernel<TYPE, true>) : reinterpret_cast<const void*>(&mx_quantize_tile_kernel<TYPE, false>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (e != hipSuccess) return e;
        }
        constexpr int kMost = 1 << 20;                               // tiles of an XCD in a launch, whose threads are counted in 32 bits
        const int share = (int)(((long long)tiles_m * tiles_n + 7) / 8);
        for (int first = 0; first < share; first += kMost) {
            const unsigned grid = 8u * std::min(share - first, kMost);
            if (a.codes) mx_quantize_tile_kernel<TYPE, true><<<grid, kThreads, lds, s>>>(a, tiles_m, tiles_n, first, cp, sp, cpt, spt);
            else mx_quantize_tile_kernel<TYPE, false><<<grid, kThreads, lds, s>>>(a, tiles_m, tiles_n, first, cp, sp, cpt, spt);
        }
    } else {
        // Four rows ahead where that leaves eight workgroups to a compute unit: 11008 x 4096 fp16 25.2 -> 21.8 us, but 301 x 5120 3.2 -> 3.7.  Not in fp32, where a
        // row is two loads already: 40 -> 43 us.
        const RowShape rs = row_shape(mx_padded(a.N) / 8);
        const dim3 few = row_grid(rs, (a.M + 3ll) / 4);
        if (TYPE != SQLLM_F32 && (long long)few.x * few.y >= 2048) mx_quantize_rows_kernel<TYPE, 4><<<few, kThreads, 0, s>>>(a, rs, cp, sp);
        else mx_quantize_rows_kernel<TYPE, 1><<<row_grid(rs, a.M), kThreads, 0, s>>>(a, rs, cp, sp);
    }
    return hipGetLastError();
}

template <int TYPE>
hipError_t dequantize(const MxDequantArgs& a, hipStream_t s) {
    constexpr int E = TYPE == SQLLM_F32 ? 4 : 8;
    const RowShape rs = row_shape(((long long)a.N + E - 1) / E);
    mx_dequantize_kernel<TYPE><<<row_grid(rs, a.M), kThreads, 0, s>>>(a, rs, mx_row_code_bytes(a.N), mx_row_scale_bytes(a.N));
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

template <int B, int R>
hipError_t gemv_few(const MxGemvArgs& a, hipStream_t s) {
    const int waves = (a.N + 2047) / 2048;
    const long long resident = 256ll * (24 / waves);                 // workgroups that run side by side
    const int most = kGemvMaxSums / B / R * R;
    const int rows = (int)std::min<long long>(most, std::max<long long>(1, (a.M + R * resident - 1) / (R * resident)) * R);
    mx_gemv_kernel<B, R><<<dim3((unsigned)(((long long)a.M + rows - 1) / rows)), waves * 64, 0, s>>>(a, rows);
    return hipGetLastError();
}

template <int B, int NS, int RING>
hipError_t gemv_batch(const MxGemvArgs& a, int share, hipStream_t s) {
    // one workgroup to a compute unit, as long as the partial sums of its rows fit
    const long long groups = ((long long)a.M + 15) / 16;
    constexpr int kMostGroups = 8;
    const int G = (int)std::min<long long>(kMostGroups, (groups + 255) / 256);
    auto lds_of = [](int G) { return (size_t)kBatchWaves * (batch_stage_bytes(B) + G * 1024); };
    const size_t lds = lds_of(G);
    if (lds > 65536) {                                               // above what a launch gets without asking; always the most, as another thread may be between this and its launch
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&mx_gemv_batch_kernel<B, NS, RING>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds_of(kMostGroups));
        if (e != hipSuccess) return e;
    }
    mx_gemv_batch_kernel<B, NS, RING><<<dim3((unsigned)((groups + G - 1) / G)), kBatchWaves * 64, lds, s>>>(a, G, share);
    return hipGetLastError();
}

template <int B>
hipError_t gemv_batch(const MxGemvArgs& a, hipStream_t s) {
    if constexpr (B > kGemvColumns) {
        if (a.B < B) return gemv_batch<B - 1>(a, s);
        const int steps = a.N / 128, rounds = (steps + 8 * kBatchWaves - 1) / (8 * kBatchWaves), share = (steps + rounds * kBatchWaves - 1) / (rounds * kBatchWaves);
        return share <= 4 ? gemv_batch<B, 4, 4>(a, share, s) : share <= 6 ? gemv_batch<B, 6, 3>(a, share, s) : gemv_batch<B, 8, 2>(a, share, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_mx_gemv(const MxGemvArgs& all, hipStream_t s) {
    constexpr int kMostRows = 1 << 28;                               // of a launch, whose threads are counted in 32 bits
    for (long long r0 = 0; r0 < all.M; r0 += kMostRows) {
        MxGemvArgs a = all;
        a.M = (int)std::min<long long>(all.M - r0, kMostRows);
        a.codes = static_cast<const char*>(all.codes) + r0 * mx_row_code_bytes(a.N);
        a.scales = static_cast<const char*>(all.scales) + r0 * mx_row_scale_bytes(a.N);
        a.y = static_cast<half_t*>(all.y) + r0 * a.B;
        const hipError_t e = a.B == 1 ? gemv_few<1, 4>(a, s) : a.B == 2 ? gemv_few<2, 4>(a, s) : gemv_batch<SQLLM_MAX_BATCH>(a, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace sqllm
