// Product of two packed matrices of the microscaled 4-bit format on the matrix cores -- device code for gfx950 (wave64).
//
// y[t][i] = sum_j X[t][j] W[i][j].  v_mfma_scale_f32_32x32x64 multiplies A (32 rows of W x 64 j) by B (64 j x 32 rows of X) and takes codes
// and scale bytes as they lie in memory: lane (r, h) = (l % 32, l / 32) supplies one block of 32 codes (16 bytes) of row r and that block's
// scale, and keeps of the result column r (a row of X) the rows 8 (e / 4) + 4 h + e % 4 of W, e = 0..15.  Which blocks of a row the two
// halves of a wave take at which step is free as long as both operands agree: half h takes blocks 4 h + s of every eight at step
// s = 0..3, so its four scale bytes are one dword and its codes 64 neighbouring bytes.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "sqllm_mx.h"
#include "sqllm_mx_device.h"

namespace sqllm {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <int S>
__device__ __forceinline__ f32x16 mma(const i32x4& a, const i32x4& b, const f32x16& c, u32 sa, u32 sb) {
    const i32x8 A = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, B = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(A, B, c, 4, 4, S, (int)sa, S, (int)sb);
}

// ---------------------------------------------------------------------------------------------- few rows of X
// The waves of a workgroup share a tile of 32 rows of W x 32 FT rows of X and deal its units of 256 columns out among themselves; their sums meet
// in LDS.  A wave requests its next unit (eight lanes to the 128 bytes of a row) while it multiplies the present one, which changes lanes in the
// wave's own part of LDS: chunk c of row r lies at position c ^ g(r) of the row's 128 bytes, so that neither 8 nor 16 neighbouring lanes, which read
// the same chunk of different rows, meet in a bank.  Fetched by the lanes that use it, neighbouring lanes on different rows, every 16 bytes were an access of
// the vector L1 of their own (33 x 11008 x 4096: 14.8 us).
__device__ __forceinline__ u32 chunk_swizzle(u32 row) { return (row & 7u) ^ ((row >> 3) & 1u); }

__device__ __forceinline__ void wave_fence() {                       // orders the LDS accesses of one wave
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int kFewMaxWaves = 8;

template <int TYPE, int FT>
__global__ void __launch_bounds__(kFewMaxWaves * 64, 2) mx_gemm_few_kernel(MxGemmArgs g, int tiles_m, int K) {
    constexpr int F = 1 + FT, kOwn = 32 * F * 128;                   // 32-row operands; bytes of a unit of them
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6, r = lane & 31, h = lane >> 5;
    const long long m0 = 32ll * (blockIdx.x % tiles_m), t0 = (32ll * FT) * (blockIdx.x / tiles_m);
    const size_t cp = K / 2, sp = K / kMxBlock;
    const int ndw = K / 128, units = mx_units(K);
    char* const own = lds + wave * kOwn;
    const char *codes[F][4], *scales[F];                             // rows past the end repeat the last one; their results are not stored
#pragma unroll
    for (int f = 0; f < F; ++f) {
        const char* c = static_cast<const char*>(f == 0 ? g.w_codes : g.x_codes);
        const char* s = static_cast<const char*>(f == 0 ? g.w_scales : g.x_scales);
        const long long first = f == 0 ? m0 : t0 + 32 * (f - 1), last = (f == 0 ? g.M : g.T) - 1;
#pragma unroll
        for (int i = 0; i < 4; ++i) codes[f][i] = c + (size_t)min(first + 8 * i + (lane >> 3), last) * cp + 16 * (lane & 7);
        scales[f] = s + (size_t)min(first + r, last) * sp;
    }
    i32x4 next[F][4];
    u32 next_scale[F];
    // K is a multiple of 128: the upper half of the last unit may lie behind the rows, and repeats the lower one with scales of 2^-127, whose products
    // vanish against every fp32 number
    auto fetch = [&](int u) {
        const bool behind = 2 * u + 1 >= ndw;
        const size_t at = (size_t)u * 128 - (behind && (lane & 4) ? 64 : 0);
#pragma unroll
        for (int f = 0; f < F; ++f) {
#pragma unroll
            for (int i = 0; i < 4; ++i) next[f][i] = *reinterpret_cast<const i32x4*>(codes[f][i] + at);
            next_scale[f] = *reinterpret_cast<const u32*>(scales[f] + 4 * (size_t)min(2 * u + h, ndw - 1));
        }
    };
    f32x16 acc[FT] = {};
    if (wave < units) fetch(wave);
    for (int u = wave; u < units; u += nw) {
        u32 scale[F];
#pragma unroll
        for (int f = 0; f < F; ++f) {
            scale[f] = 2 * u + h < ndw ? next_scale[f] : 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const u32 row = 8 * i + (lane >> 3);
                *reinterpret_cast<i32x4*>(own + 4096 * f + 128 * row + 16 * ((lane & 7) ^ chunk_swizzle(row))) = next[f][i];
            }
        }
        if (u + nw < units) fetch(u + nw);
        wave_fence();
        i32x4 op[F][4];
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int s = 0; s < 4; ++s) op[f][s] = *reinterpret_cast<const i32x4*>(own + 4096 * f + 128 * r + 16 * ((4 * h + s) ^ chunk_swizzle(r)));
        wave_fence();
#pragma unroll
        for (int t = 0; t < FT; ++t) {
            acc[t] = mma<0>(op[0][0], op[1 + t][0], acc[t], scale[0], scale[1 + t]);
            acc[t] = mma<1>(op[0][1], op[1 + t][1], acc[t], scale[0], scale[1 + t]);
            acc[t] = mma<2>(op[0][2], op[1 + t][2], acc[t], scale[0], scale[1 + t]);
            acc[t] = mma<3>(op[0][3], op[1 + t][3], acc[t], scale[0], scale[1 + t]);
        }
    }
    // sums: [row of X][row of W], rows of 36 so that a wave's writes and the reads of rows spread over the banks
    typedef typename MxType<TYPE>::value value;
    constexpr int kRow = 36;
    static_assert(32 * kRow * 4 * FT <= kOwn, "a wave's sums fit its part");
    __syncthreads();
#pragma unroll
    for (int t = 0; t < FT; ++t)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<f32x4*>(own + 4 * (kRow * (32 * t + r) + 4 * h + 2 * e)) = f32x4{acc[t][e], acc[t][e + 1], acc[t][e + 2], acc[t][e + 3]};
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * FT * 32; i += blockDim.x) {
        const long long t = t0 + (i >> 5), m = m0 + (i & 31);
        if (t < g.T && m < g.M) {
            const char* s = lds + 4 * (kRow * (i >> 5) + (i & 31));
            float sum = 0.f;
            for (int w = 0; w < nw; ++w) sum += *reinterpret_cast<const float*>(s + w * kOwn);
            value* y = static_cast<value*>(g.y) + t * g.ldy + m;
            *y = (value)(g.accumulate ? (float)*y + sum : sum);
        }
    }
}

// ---------------------------------------------------------------------------------------------- many rows on both sides
// A workgroup of four waves makes a tile of R rows of W x R rows of X, R = 64 F, each wave a quarter of it in 16 F^2 accumulator registers: F = 4, one wave
// to a SIMD, or F = 2, two workgroups to a compute unit.  Stages of 256 columns: a wave requests its share of the stage after next into 16 F registers (128
// bytes of a row to eight lanes, whole cache lines), writes the next stage to the LDS buffer that is not being read, and feeds the matrix
// instructions from the other; one barrier a stage.  Operands are read a step (64 columns) ahead.  Scales go the same way in groups of 1024 columns, half
// the rows every second stage: a request is an access of the vector L1 for every row it touches, so two lanes take 32 bytes of a row (in groups of 512, a lane
// to a row, 2047 x 4096 x 11008 took 7 % longer).  Chunk c (16 bytes) of row r lies at position c ^ g(r) of the row's 128 bytes, so that neither 8 nor
// 16 neighbouring lanes, which read the same chunk of different rows, meet in a bank.
//
// What bounds it (4096 x 22016 x 8192 to bf16: 434 us, 3.4 PFLOP/s): 850 000 cycles, on zeros as on random data, in 41 % of which the matrix pipes are busy; with one
// wave to a SIMD the traffic through LDS, the requests and the results take the rest.  Power takes the clock from 2.35 GHz (zeros: 363 us) to 1.97.  The
// instructions alone, operands in registers, make 6.6 PFLOP/s on random data and 9.8 on zeros.  Left out one by one (zeros): scales' way to LDS a tenth, codes' way
// to LDS a tenth, their requests a sixth of the time.
//
// Registers: the 256-row forms need all 512 and spill 47 to 76 more (and 37 to 109 scalar ones, to vector registers).  In those that write, every reload lies outside the loop
// over the stages; in those that add to y, four or five lie in it, one set for each two stages.  The 128-row forms spill no vector registers.
template <int F>
struct TileShape {
    static constexpr int kRows = 64 * F;                             // of W and of X
    static constexpr int kStageBytes = 2 * kRows * 128;              // 256 columns of both
    static constexpr int kScaleGroupBytes = 2 * kRows * 32;          // scales of 1024 columns of both
    static constexpr int kPieces = 4 * F;                            // 16-byte pieces of a stage per lane
    static constexpr int kPitch = kRows * 4 + 16;                    // of a row of sums in LDS: neighbouring rows four banks apart
    static constexpr int kLds = 2 * kStageBytes + 2 * kScaleGroupBytes;
    static_assert(kRows / 2 * kPitch <= kLds, "half a tile of sums fits");
};

// Where tile p of the order lies.  Workgroups are handed to the eight XCDs in turn: each takes a contiguous range of the order, which goes through bands of
// eight tiles of W, so that the tiles in flight on an XCD share rows in its L2.
struct TileOrder {
    int tiles_m, tiles_t, rows;
    __device__ void at(int p, long long& m0, long long& t0) const {
        const int per = 8 * tiles_t, band = p / per, in = p % per, wide = min(tiles_m - 8 * band, 8);
        m0 = (long long)(8 * band + in % wide) * rows;
        t0 = (long long)(in / wide) * rows;
    }
};

// R / 2 rows of R sums in LDS added to y, a quarter of them by each of four waves.
template <int TYPE, int R>
__device__ __forceinline__ void add_rows(const MxGemmArgs& g, const char* lds, int pitch, long long m0, long long t0, int wave, int lane) {
    typedef typename MxType<TYPE>::value value;
    constexpr int E = 16 / sizeof(value), kLanes = R / E;     // elements of 16 bytes, lanes to a row
    if (m0 + R <= g.M) {
        typedef value vec __attribute__((ext_vector_type(E)));
        const int row0 = R / 8 * wave + lane / kLanes, col = E * (lane % kLanes);
#pragma unroll 4
        for (int i = 0; i < R / 8; i += 64 / kLanes) {
            const int row = row0 + i;
            if (t0 + row >= g.T) continue;
            value* y = static_cast<value*>(g.y) + (t0 + row) * g.ldy + m0 + col;
            const float* s = reinterpret_cast<const float*>(lds + row * pitch) + col;
            vec v;
            if constexpr (E == 8) v = __builtin_bit_cast(vec, (u32x4)*reinterpret_cast<const u32x4_a2*>(y));
            else v = __builtin_bit_cast(vec, (u32x4)*reinterpret_cast<const u32x4_a4*>(y));
#pragma unroll
            for (int k = 0; k < E; k += 4) {
                const f32x4 t = *reinterpret_cast<const f32x4*>(s + k);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[k + j] = (value)((float)v[k + j] + t[j]);
            }
            if constexpr (E == 8) *reinterpret_cast<u32x4_a2*>(y) = __builtin_bit_cast(u32x4, v);
            else *reinterpret_cast<u32x4_a4*>(y) = __builtin_bit_cast(u32x4, v);
        }
    } else {
        constexpr int kAhead = 8;                                    // rows read before the first is written (one: 4096 x 8191 of 1000 in fp32, y from HBM, 169 us, now 92; bytes 56)
        for (int i = 0; i < R / 8; i += kAhead) {
            const int row0 = R / 8 * wave + i;
            value* const y = static_cast<value*>(g.y) + (t0 + row0) * g.ldy + m0;
            value v[kAhead][R / 64];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
#pragma unroll
                for (int c = 0; c < R / 64; ++c)
                    if (t0 + row0 + k < g.T && m0 + 64 * c + lane < g.M) v[k][c] = y[k * g.ldy + 64 * c + lane];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
#pragma unroll
                for (int c = 0; c < R / 64; ++c)
                    if (t0 + row0 + k < g.T && m0 + 64 * c + lane < g.M)
                        y[k * g.ldy + 64 * c + lane] = (value)((float)v[k][c] + reinterpret_cast<const float*>(lds + (row0 + k) * pitch)[64 * c + lane]);
        }
    }
}

// d[4 p + w] of lane c of four, swapped to d[4 c + w] of lane p.
__device__ __forceinline__ void quad_transpose(u32 (&d)[16], int c) {
    auto swap = [&](auto ctrl, int bit) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            if (e >> 2 & bit) continue;
            u32 &a = d[e], &b = d[e + 4 * bit];
            const u32 from_a = __builtin_amdgcn_mov_dpp((int)a, decltype(ctrl)::value, 0xf, 0xf, true), from_b = __builtin_amdgcn_mov_dpp((int)b, decltype(ctrl)::value, 0xf, 0xf, true);
            const u32 new_a = c & bit ? from_b : a, new_b = c & bit ? b : from_a;
            a = new_a;
            b = new_b;
        }
    };
    swap(std::integral_constant<int, 0xb1>{}, 1);                    // lanes 1 0 3 2
    swap(std::integral_constant<int, 0x4e>{}, 2);                    // lanes 2 3 0 1
}

// What becomes of the sums: added to y, or written to it, past the caches or through them.  Rows of y that are not aligned to 16 bytes share
// lines, which gather in the caches: 4096 x 8191 results, bf16 of 4096 columns 105 us, past the caches 114, fp32 of 1024 60 and 78; tiles of 128 in 16 bits write
// shorter pieces sooner after one another and do not gain, of 1024 columns 50 and 44.  Through LDS an element at a time they took 129, 65 and 59.
enum Out { kAdd, kStream, kCached };

// SHORT: fewer than 512 columns, so four dwords of scales are more than a row holds and are fetched one by one (5120 x 5120 results of 384 columns in fp32:
// 30 us, 58 with the kernel for few rows).
template <int TYPE, int F, Out OUT, bool SHORT>
__global__ void __launch_bounds__(256, F == 4 ? 1 : 2) mx_gemm_tile_kernel(MxGemmArgs g, TileOrder order, int K) {
    typedef TileShape<F> S;
    constexpr int R = S::kRows, kStageBytes = S::kStageBytes, kScaleGroupBytes = S::kScaleGroupBytes, NP = S::kPieces;
    __shared__ __align__(16) char lds[S::kLds];
    char* const stage = lds;
    char* const scale = lds + 2 * kStageBytes;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 31, h = lane >> 5;
    // the workgroups of an XCD take its range of tiles in turn
    const int tiles = order.tiles_m * order.tiles_t, xcd = blockIdx.x & 7, step = gridDim.x >> 3;
    const int end = (int)((long long)tiles * (xcd + 1) >> 3);
    int p = (int)((long long)tiles * xcd >> 3) + (int)(blockIdx.x >> 3);
    if (p >= end) return;
    long long m0, t0;
    order.at(p, m0, t0);
    const u32 cp = K / 2, sp = K / kMxBlock;
    const int ndw = K / 128, nst = mx_units(K);   // dwords of scales of a row, stages
    // waves 0, 1 fetch the rows of W, 2, 3 those of X: R / 2 each, eight of them to an instruction; rows past the end repeat the last one
    const bool mine_w = wave < 2;
    const u32 row0 = R / 2 * (wave & 1);
    const char *codes, *scales;
    u32 off[NP], wr[2];
    int last;
    // Position 32 block + at of an operand's part of LDS holds that row of it, and for W the row for which a lane's 16 sums of a 32-row operand are neighbours in
    // y, and beside those of the other half of the wave (fp32) or of the next operand (16 bits): 64 bytes.
    constexpr bool kPairs = sizeof(typename MxType<TYPE>::value) == 2;
    auto row_at = [&](int block, int at) {
        const int base = kPairs ? 64 * (block >> 1) + 16 * (block & 1) : 32 * block;
        return mine_w ? base + (kPairs ? 32 : 16) * (at >> 2 & 1) + 4 * (at >> 3) + (at & 3) : 32 * block + at;
    };
    auto aim = [&]() {                                               // the fetches at the tile (m0, t0)
        codes = static_cast<const char*>(mine_w ? g.w_codes : g.x_codes) + (size_t)(mine_w ? m0 : t0) * cp;
        scales = static_cast<const char*>(mine_w ? g.w_scales : g.x_scales) + (size_t)(mine_w ? m0 : t0) * sp;
        last = (int)min((mine_w ? (long long)g.M - m0 : (long long)g.T - t0) - 1, (long long)R - 1);
#pragma unroll
        for (int i = 0; i < NP; ++i) off[i] = (u32)min((int)row0 + row_at(i >> 2, 8 * (i & 3)) + row_at(0, lane >> 3), last) * cp + 16 * (lane & 7);
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) wr[i] = wave * (64 * R) + 128 * (8 * i + (lane >> 3)) + 16 * ((lane & 7) ^ chunk_swizzle(8 * i + (lane >> 3)));
    const int wm = wave & 1, wt = wave >> 1;
    const u32 rda = wm * (64 * R) + r * 128, rdb = 128 * R + wt * (64 * R) + r * 128, swz = chunk_swizzle(r);
    f32x16 acc[F][F];
    i32x4 a0[F], b0[F], a1[F], b1[F], pre[NP];
    u32 ua[F], ub[F], va[F], vb[F];
    u32x4 spre[F / 2], spre1[F / 2];
    const int quad = 4 * (lane & 1);                                 // of a row's eight dwords of a group a lane moves four
    // K is a multiple of 128: the upper half of the last stage may lie behind the rows, and repeats the lower one with scales of 2^-127, whose products
    // vanish against every fp32 number
    auto fetch = [&](int st, int i) { pre[i] = *reinterpret_cast<const i32x4*>(codes + (size_t)min(st, nst - 1) * 128 + off[i] - ((lane & 4) && 2 * min(st, nst - 1) + 1 >= ndw ? 64 : 0)); };
    auto put = [&](int st, int i) { *reinterpret_cast<i32x4*>(stage + (st & 1) * kStageBytes + 2048 * (i >> 1) + wr[i & 1]) = pre[i]; };
    // Part g of the scales: half the rows (g even: the first) of group g / 2.
    auto fetch_scales = [&](int g, u32x4 (&spre)[F / 2]) {
        const int d = 8 * (g >> 1) + quad;
        int end = last;
        asm volatile("" : "+s"(end));                                // offsets made anew each time: kept, they would be spilled
#pragma unroll
        for (int i = 0; i < F / 2; ++i) {
            const u32 row = __umul24(min((int)row0 + row_at(F / 2 * (g & 1) + i, 0) + row_at(0, lane >> 1), end), sp);
            if constexpr (SHORT) {
#pragma unroll
                for (int j = 0; j < 4; ++j) spre[i][j] = *reinterpret_cast<const u32*>(scales + (size_t)(row + 4 * (u32)min(d + j, ndw - 1)));
            } else {
                spre[i] = *reinterpret_cast<const u32x4_a4*>(scales + (size_t)(row + 4 * (u32)min(d, ndw - 4)));
            }
        }
    };
    auto put_scales = [&](int g, const u32x4 (&spre)[F / 2]) {
        char* b = scale + ((g >> 1) & 1) * kScaleGroupBytes + wave * (16 * R) + (g & 1) * (8 * R);
        const int d = 8 * (g >> 1) + quad, over = max(d + 4 - ndw, 0);   // dwords behind the row's end: so much earlier they were fetched
        const bool drop1 = over & 1, drop2 = over & 2, drop4 = over >= 4;
#pragma unroll
        for (int i = 0; i < F / 2; ++i) {
            u32x4 v = spre[i];
            if constexpr (SHORT) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = d + j < ndw ? v[j] : 0u;
            } else {
                v = u32x4{drop1 ? v.y : v.x, drop1 ? v.z : v.y, drop1 ? v.w : v.z, drop1 ? 0u : v.w};
                v = u32x4{drop2 ? v.z : v.x, drop2 ? v.w : v.y, drop2 ? 0u : v.z, drop2 ? 0u : v.w};
                v = u32x4{drop4 ? 0u : v.x, drop4 ? 0u : v.y, drop4 ? 0u : v.z, drop4 ? 0u : v.w};
            }
            const u32 row = 32 * i + (lane >> 1);
#pragma unroll
            for (int j = 0; j < 2; ++j) *reinterpret_cast<u32x2*>(b + 32 * row + 8 * (((quad >> 1) + j) ^ ((row >> 3) & 3))) = u32x2{v[2 * j], v[2 * j + 1]};
        }
    };
    auto read = [&](int st, int s, i32x4 (&a)[F], i32x4 (&b)[F]) {
        const char* base = stage + (st & 1) * kStageBytes + 16 * ((4 * h + s) ^ swz);
#pragma unroll
        for (int f = 0; f < F; ++f) {
            a[f] = *reinterpret_cast<const i32x4*>(base + rda + 4096 * f);
            b[f] = *reinterpret_cast<const i32x4*>(base + rdb + 4096 * f);
        }
    };
    auto read_scales = [&](int st) {
        const char* base = scale + ((st >> 2) & 1) * kScaleGroupBytes + 32 * r + 4 * ((2 * (st & 3) + h) ^ (2 * ((r >> 3) & 3)));
#pragma unroll
        for (int f = 0; f < F; ++f) {
            va[f] = *reinterpret_cast<const u32*>(base + wm * (16 * R) + 1024 * f);
            vb[f] = *reinterpret_cast<const u32*>(base + 32 * R + wt * (16 * R) + 1024 * f);
        }
    };
    auto multiply = [&](auto s, const i32x4 (&a)[F], const i32x4 (&b)[F]) {
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
            for (int k = 0; k < F; ++k) acc[i][k] = mma<decltype(s)::value>(a[i], b[k], acc[i][k], ua[i], ub[k]);
    };
    // The order of a step's instructions: the reads of the next step's operands as early as they fit, a write to LDS and a request between two matrix
    // instructions (reads spread over the whole step take 3 % longer at 301 x 5120 x 5120, 1.3 % at 4096 x 22016 x 8192).
    auto arrange = [&](auto group, auto writes) {
        constexpr int G = decltype(group)::value;
        if constexpr (F == 2) {
            __builtin_amdgcn_sched_group_barrier(0x100, 4, G);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, G);
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x200, decltype(writes)::value, G);
                __builtin_amdgcn_sched_group_barrier(0x020, 1, G);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, G);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i < 4) __builtin_amdgcn_sched_group_barrier(0x100, 2, G);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, G);
                __builtin_amdgcn_sched_group_barrier(0x200, decltype(writes)::value, G);
                __builtin_amdgcn_sched_group_barrier(0x020, 1, G);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, G);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto one_stage = [&](int st, auto odd) {
        constexpr bool kOdd = decltype(odd)::value;
#pragma unroll
        for (int f = 0; f < F; ++f) { ua[f] = va[f]; ub[f] = vb[f]; }
        // the pieces of the next stage go to LDS and those of the one after are requested in the first three steps
        read(st, 1, a1, b1);
#pragma unroll
        for (int i = 0; i < 3 * F / 2; ++i) { put(st + 1, i); fetch(st + 2, i); }
        multiply(std::integral_constant<int, 0>{}, a0, b0);
        arrange(std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{});
        read(st, 2, a0, b0);
#pragma unroll
        for (int i = 3 * F / 2; i < 3 * F; ++i) { put(st + 1, i); fetch(st + 2, i); }
        multiply(std::integral_constant<int, 1>{}, a1, b1);
        arrange(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{});
        read(st, 3, a1, b1);
#pragma unroll
        for (int i = 3 * F; i < NP; ++i) { put(st + 1, i); fetch(st + 2, i); }
        if (kOdd) {
            put_scales((st >> 1) + 2, spre);
            fetch_scales((st >> 1) + 3, spre);
        }
        multiply(std::integral_constant<int, 2>{}, a0, b0);
        arrange(std::integral_constant<int, 2>{}, std::integral_constant<int, kOdd ? 2 : 1>{});
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
        read(st + 1, 0, a0, b0);
        read_scales(st + 1);
        multiply(std::integral_constant<int, 3>{}, a1, b1);
        if constexpr (F == 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 3);
#pragma unroll
        for (int i = 0; i < 2 * F; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 3);
            __builtin_amdgcn_sched_group_barrier(0x008, F / 2, 3);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto request = [&]() {                                           // the first stage and group of scales of the tile aimed at
#pragma unroll
        for (int i = 0; i < NP; ++i) fetch(0, i);
        fetch_scales(0, spre);
        fetch_scales(1, spre1);
    };
    aim();
    request();
    while (true) {
#pragma unroll
        for (int i = 0; i < NP; ++i) put(0, i);
#pragma unroll
        for (int i = 0; i < NP; ++i) fetch(1, i);
        put_scales(0, spre);
        put_scales(1, spre1);
        fetch_scales(2, spre);
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
            for (int k = 0; k < F; ++k) acc[i][k] = f32x16{};
        __syncthreads();
        read(0, 0, a0, b0);
        read_scales(0);
        for (int st = 0; st < nst; st += 2) {                        // an odd number of stages is filled up by one whose scales are all 2^-127
            one_stage(st, std::false_type{});
            one_stage(st + 1, std::true_type{});
        }
        // The next tile's first stage is requested before this one's result goes out.
        const long long m_out = m0, t_out = t0;
        p += step;
        const bool more = p < end;
        if (more) {
            order.at(p, m0, t0);
            aim();
            request();
        }
        if constexpr (OUT != kAdd) {
            // Four lanes exchange their 64 bytes of four rows, so that each instruction writes eight whole lines, with no barrier and while the next
            // tile's stage is on its way (4096 x 22016 results of 8192 columns: 6 % longer through LDS).
            const int c = lane & 3;
            typedef typename MxType<TYPE>::value value;
            typedef value pair __attribute__((ext_vector_type(2)));
            constexpr int E = 16 / sizeof(value);                    // of a store
            long long t = t_out + R / 2 * wt + (r & ~3);
            const long long m = m_out + R / 2 * wm + (kPairs ? 32 : 16) * h + E * c;
            value* y = static_cast<value*>(g.y) + t * g.ldy + m;
#pragma unroll
            for (int k = 0; k < F; ++k, t += 32, y += 32 * g.ldy) {
#pragma unroll
                for (int i = 0; i < F; i += 2) {
#pragma unroll
                    for (int s = 0; s < (kPairs ? 1 : 2); ++s) {
                        u32 d[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            if constexpr (!kPairs) d[e] = __float_as_uint(acc[i + s][k][e]);
                            else d[e] = __builtin_bit_cast(u32, pair{(value)acc[i + (e >> 3)][k][2 * (e & 7)], (value)acc[i + (e >> 3)][k][2 * (e & 7) + 1]});
                        }
                        quad_transpose(d, c);
                        const int at = 32 * (i + s);
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (t + j < g.T) {
                                value* dst = y + j * g.ldy + at;
                                u32x4 v = {d[4 * j], d[4 * j + 1], d[4 * j + 2], d[4 * j + 3]};
                                const long long left = g.M - (m + at);
                                if (left >= E) {
                                    if constexpr (OUT == kStream && kPairs) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_a2*>(dst));
                                    else if constexpr (OUT == kStream) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_a4*>(dst));
                                    else if constexpr (kPairs) *reinterpret_cast<u32x4_a2*>(dst) = v;
                                    else *reinterpret_cast<u32x4_a4*>(dst) = v;
                                } else {
#pragma unroll 1
                                    for (int e = 0; e < left; ++e) {
                                        dst[e] = __builtin_bit_cast(value, (typename std::conditional<kPairs, uint16_t, u32>::type)v.x);
                                        constexpr int kShift = 8 * sizeof(value) % 32;
                                        if constexpr (kPairs) v = u32x4{__builtin_amdgcn_alignbit(v.y, v.x, kShift), __builtin_amdgcn_alignbit(v.z, v.y, kShift), __builtin_amdgcn_alignbit(v.w, v.z, kShift), v.w >> kShift};
                                        else v = u32x4{v.y, v.z, v.w, 0u};
                                    }
                                }
                            }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        } else {
            // Through LDS, half the rows of X at a time, so that y is read and written in whole lines.
            constexpr int kPitch = S::kPitch;
            for (int half = 0; half < 2; ++half) {
                __syncthreads();
                if (wt == half) {
#pragma unroll
                    for (int i = 0; i < F; ++i)
#pragma unroll
                        for (int k = 0; k < F; ++k)
#pragma unroll
                            for (int e = 0; e < 16; e += 4)
                                *reinterpret_cast<f32x4*>(lds + (32 * k + r) * kPitch + 4 * (R / 2 * wm + (kPairs ? 64 * (i >> 1) + 32 * h + 16 * (i & 1) : 32 * i + 16 * h) + e)) = f32x4{acc[i][k][e], acc[i][k][e + 1], acc[i][k][e + 2], acc[i][k][e + 3]};
                }
                __syncthreads();
                add_rows<TYPE, R>(g, lds, kPitch, m_out, t_out + R / 2 * half, wave, lane);
            }
        }
        if (!more) break;
        __syncthreads();
    }
}

namespace {

constexpr int kTileShort = 512, kTileMost = 1 << 24;                 // columns: below, rows of SHORT's form; above, offsets inside a tile leave 32 bits

template <int TYPE, int F, bool SHORT>
hipError_t gemm_tiles(const MxGemmArgs& g, int K, hipStream_t s) {
    if ((K < kTileShort) != SHORT || K > kTileMost) return hipErrorInvalidValue;   // the kernel would read scales or codes that are not there
    constexpr int R = TileShape<F>::kRows;
    const TileOrder order = {(int)(((long long)g.M + R - 1) / R), (int)(((long long)g.T + R - 1) / R), R};
    const unsigned grid = F == 4 ? 256 : 512;                        // one workgroup to a compute unit, or two
    constexpr int e = 16 / (TYPE == SQLLM_F32 ? 4 : 2);
    constexpr Out kUnaligned = F == 2 && TYPE != SQLLM_F32 ? kStream : kCached;
    if (g.accumulate) mx_gemm_tile_kernel<TYPE, F, kAdd, SHORT><<<grid, 256, 0, s>>>(g, order, K);
    else if ((reinterpret_cast<uintptr_t>(g.y) & 15) == 0 && g.ldy % e == 0) mx_gemm_tile_kernel<TYPE, F, kStream, SHORT><<<grid, 256, 0, s>>>(g, order, K);
    else mx_gemm_tile_kernel<TYPE, F, kUnaligned, SHORT><<<grid, 256, 0, s>>>(g, order, K);
    return hipGetLastError();
}

template <int TYPE, int FT>
hipError_t gemm_few(const MxGemmArgs& g, int K, hipStream_t s) {
    const long long tiles_m = ((long long)g.M + 31) / 32, tiles = tiles_m * (((long long)g.T + 32 * FT - 1) / (32 * FT));
    const int waves = std::min(tiles > 256 ? 4 : kFewMaxWaves, mx_units(K));
    const size_t lds = (size_t)waves * (1 + FT) * 4096;
    if (lds > 65536) {                                               // above what a launch gets without asking; always the most, as another thread may be between this and its launch
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&mx_gemm_few_kernel<TYPE, FT>), hipFuncAttributeMaxDynamicSharedMemorySize, kFewMaxWaves * (1 + FT) * 4096);
        if (e != hipSuccess) return e;
    }
    mx_gemm_few_kernel<TYPE, FT><<<dim3((unsigned)tiles), waves * 64, lds, s>>>(g, (int)tiles_m, K);
    return hipGetLastError();
}

// Which kernel: the one whose estimate is lowest.  An estimate, in microseconds, is a part for the result (size bytes an element) and a part per 1024 columns (k)
// for each round of tiles over the compute units, fitted to measured times.  Tiles of 256 / 128, bf16: 4096 x 16384 results of 1024 columns take 79 / 70 us,
// of 2048 112 / 104, of 8192 313 / 358; 2048 x 16384 of 4096 94 / 100; 2047 x 4096 of 11008 78 / 64; fp32: 4096 x 11008 of 2047 102 / 91.  128 / few rows: 301 x
// 5120 of 5120 15 / 22, 128 x 4096 of 11008 29 / 15, 33 x 11008 of 4096 13.4 / 12.
double cost_of_256(double rows, double others, double k, int size) { return std::ceil(std::ceil(rows / 256) * std::ceil(others / 256) / 256) * (4.8 + 3.3 * size + 8.3 * k); }
double cost_of_128(double rows, double others, double k, int size) {
    const double tiles = std::ceil(rows / 128) * std::ceil(others / 128);
    return tiles <= 256 ? 4.0 + 2.5 * k : std::ceil(tiles / 512) * (1.6 + 0.9 * size + 5.15 * k);
}
double cost_of_few(double rows, double others, double k) { return 5.8 + (0.0026 + 0.0039 * k) * std::ceil(rows / 32) * std::ceil(others / (others <= 32 ? 32 : 64)); }

template <int TYPE>
hipError_t gemm(const MxGemmArgs& g, hipStream_t s) {
    const int K = mx_padded(g.N);
    const int size = mx_type_size(TYPE);
    const double k = K / 1024.0, cost2 = cost_of_128(g.M, g.T, k, size), few = cost_of_few(g.M, g.T, k);
    if (K <= kTileMost) {
        if (K < kTileShort) {
            if (cost2 < few) return gemm_tiles<TYPE, 2, true>(g, K, s);
        } else {
            const double cost4 = cost_of_256(g.M, g.T, k, size);
            if (std::min(cost4, cost2) < few) return cost4 < cost2 ? gemm_tiles<TYPE, 4, false>(g, K, s) : gemm_tiles<TYPE, 2, false>(g, K, s);
        }
    }
    return g.T <= 32 ? gemm_few<TYPE, 1>(g, K, s) : gemm_few<TYPE, 2>(g, K, s);
}

}  // namespace

hipError_t launch_mx_gemm(const MxGemmArgs& g, hipStream_t s) {
    return g.type == SQLLM_F16 ? gemm<SQLLM_F16>(g, s) : g.type == SQLLM_BF16 ? gemm<SQLLM_BF16>(g, s) : gemm<SQLLM_F32>(g, s);
}

}  // namespace sqllm
