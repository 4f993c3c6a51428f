// Device code shared by the kernels of the microscaled 4-bit format: values of the three element types and their conversions.
//
// gfx950 converts pairs between the format and fp16, bf16 and fp32 in one instruction each, taking the exponent field of an fp32 operand
// as the scale: round to nearest even, saturation at 6, and every scale byte s passed as the bits s << 23 (0 stands for 2^-127, 255 gives
// NaN).  Checked on the GPU for all fp16 and bf16 values and all scales, and for fp32 around every border.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sqllm_mx.h"

namespace sqllm {

typedef uint32_t u32;
typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32 u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef _Float16 half_t;
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16_t;
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float mx_scale(u32 byte) { return __uint_as_float(byte << 23); }

// largest magnitude of a block (bits of an fp32 number) -> scale byte: 2^(byte - 127) puts it into [4, 8); Inf and NaN -> 255
__device__ __forceinline__ u32 mx_scale_byte(u32 top_bits) {
    const u32 field = top_bits >> 23;
    return field == 255u ? 255u : field < 2u ? 0u : field - 2u;
}

template <int TYPE>
struct MxType;

template <>
struct MxType<SQLLM_F16> {
    typedef half_t value;
    static constexpr int kPairDwords = 1;
    __device__ static u32 magnitude(u32 bits) { return __float_as_uint((float)__builtin_bit_cast(half_t, (uint16_t)bits)); }   // of non-negative bits
    template <int S>
    __device__ static u32 pack(u32 old, u32 pair, float scale) { return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, __builtin_bit_cast(half2_t, pair), scale, S); }
    template <int S>
    __device__ static u32 unpack(u32 codes, float scale) { return __builtin_bit_cast(u32, (half2_t)__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, S)); }
};
template <>
struct MxType<SQLLM_BF16> {
    typedef bf16_t value;
    static constexpr int kPairDwords = 1;
    __device__ static u32 magnitude(u32 bits) { return bits << 16; }
    template <int S>
    __device__ static u32 pack(u32 old, u32 pair, float scale) { return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2_t, pair), scale, S); }
    template <int S>
    __device__ static u32 unpack(u32 codes, float scale) { return __builtin_bit_cast(u32, (bf16x2_t)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, S)); }
};
template <>
struct MxType<SQLLM_F32> {
    typedef float value;
    static constexpr int kPairDwords = 2;
};

// Eight neighbouring elements: four dwords of 16-bit pairs, or eight dwords.
template <int TYPE>
struct MxEight {
    static constexpr int kDwords = 4 * MxType<TYPE>::kPairDwords;
    u32 v[kDwords];

    __device__ void load(const void* p) {                            // eight elements from any element's address
        if constexpr (TYPE == SQLLM_F32) {
            const u32x4_a4* s = static_cast<const u32x4_a4*>(p);
            const u32x4 t = s[0], u = s[1];                          // two loads to a line: through the caches
            v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w; v[4] = u.x; v[5] = u.y; v[6] = u.z; v[7] = u.w;
        } else {
            // gfx950 takes sixteen bytes at any address (dwords that were shifted together: 11008 x 4095 bf16 in both directions 65 us, so 52)
            const u32x4 t = __builtin_nontemporal_load(static_cast<const u32x4_a2*>(p));
            v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
        }
    }
    // Eight elements of a row of n from element j on.  Where the row ends before, its last eight are fetched, and settle() moves them: a lane that fetched its few
    // one by one made its wave wait for all its requests (1999 x 5118 fp16 in both directions 20.2 us, now 10.8).
    typedef typename MxType<TYPE>::value value;
    __device__ void load(const value* row, int j, int n) {
        if (n >= 8) load(row + min(j, n - 8));
        else load_some(row + j, max(n - j, 0));                      // j = 0 or behind the row
    }
    __device__ void settle(int j, int n) {
        const int by = n >= 8 ? j - (n - 8) : 0;                     // elements too early
        if (by > 0) {
            constexpr int kPer = TYPE == SQLLM_F32 ? 1 : 2;          // elements of a dword
            if (kPer == 2 && (by & 1)) {
#pragma unroll
                for (int i = 0; i < kDwords; ++i) v[i] = __builtin_amdgcn_alignbyte(i + 1 < kDwords ? v[i + 1] : 0u, v[i], 2);
            }
#pragma unroll
            for (int s = 1; s < kDwords; s *= 2) {
                const bool move = by / kPer & s;
#pragma unroll
                for (int i = 0; i < kDwords; ++i) v[i] = move ? (i + s < kDwords ? v[i + s] : 0u) : v[i];
            }
            if (by >= 8) clear();
        }
    }
    __device__ void clear() {
#pragma unroll
        for (int i = 0; i < kDwords; ++i) v[i] = 0u;
    }
    __device__ void load_some(const void* p, int n) {                // the first n (0..8) elements, any alignment; the rest is zero
        if constexpr (TYPE == SQLLM_F32) {
            const u32* s = static_cast<const u32*>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < n ? s[i] : 0u;
        } else {
            const uint16_t* s = static_cast<const uint16_t*>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = (2 * i < n ? (u32)s[2 * i] : 0u) | (2 * i + 1 < n ? (u32)s[2 * i + 1] << 16 : 0u);
        }
    }
    __device__ void to_lds(u32* d) const {                           // 16-byte aligned
#pragma unroll
        for (int i = 0; i < kDwords / 4; ++i) reinterpret_cast<u32x4*>(d)[i] = u32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
    }
    // Past the caches: neighbouring lanes write whole lines with one store (13824 x 5120 to fp16: 41 -> 28 us).
    __device__ void store(void* p) const {                           // 16-bit types, to any element's address
        __builtin_nontemporal_store(u32x4{v[0], v[1], v[2], v[3]}, static_cast<u32x4_a2*>(p));
    }
    __device__ void store_some(void* p, int n) const {
        if constexpr (TYPE == SQLLM_F32) {
            u32* d = static_cast<u32*>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) d[i] = v[i];
        } else {
            uint16_t* d = static_cast<uint16_t*>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) d[i] = (uint16_t)(v[i >> 1] >> (16 * (i & 1)));
        }
    }
    // bits of the largest magnitude; order of magnitudes is order of their bits, NaN above Inf above the numbers
    __device__ u32 top() const {
        if constexpr (TYPE == SQLLM_F32) {
            u32 m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, v[i] & 0x7FFFFFFFu);
            return m;
        } else {
            u16x2 m = __builtin_bit_cast(u16x2, v[0] & 0x7FFF7FFFu);
#pragma unroll
            for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i] & 0x7FFF7FFFu));
            return max((u32)m.x, (u32)m.y);
        }
    }
    __device__ u32 pack(u32 byte) const {                            // eight codes; a block without a number scale holds zeros
        const float s = mx_scale(byte);
        u32 r = 0;
        if constexpr (TYPE == SQLLM_F32) {
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(v[0]), __uint_as_float(v[1]), s, 0);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(v[2]), __uint_as_float(v[3]), s, 1);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(v[4]), __uint_as_float(v[5]), s, 2);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(v[6]), __uint_as_float(v[7]), s, 3);
        } else {
            r = MxType<TYPE>::template pack<0>(r, v[0], s);
            r = MxType<TYPE>::template pack<1>(r, v[1], s);
            r = MxType<TYPE>::template pack<2>(r, v[2], s);
            r = MxType<TYPE>::template pack<3>(r, v[3], s);
        }
        return byte == 255u ? 0u : r;
    }
    __device__ void unpack(u32 codes, u32 byte) {
        const float s = mx_scale(byte);
        if constexpr (TYPE == SQLLM_F32) {
            const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1);
            const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 3);
            v[0] = __float_as_uint(a.x); v[1] = __float_as_uint(a.y); v[2] = __float_as_uint(b.x); v[3] = __float_as_uint(b.y);
            v[4] = __float_as_uint(c.x); v[5] = __float_as_uint(c.y); v[6] = __float_as_uint(d.x); v[7] = __float_as_uint(d.y);
        } else {
            v[0] = MxType<TYPE>::template unpack<0>(codes, s);
            v[1] = MxType<TYPE>::template unpack<1>(codes, s);
            v[2] = MxType<TYPE>::template unpack<2>(codes, s);
            v[3] = MxType<TYPE>::template unpack<3>(codes, s);
        }
    }
};

// bits of a magnitude in the type -> bits of the same number in fp32
template <int TYPE>
__device__ __forceinline__ u32 mx_magnitude(u32 bits) {
    if constexpr (TYPE == SQLLM_F32) return bits;
    else return MxType<TYPE>::magnitude(bits);
}

__device__ __forceinline__ u32 quad_max(u32 v) {                     // over the four lanes of a quad
    v = max(v, (u32)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));   // lane ^ 1
    return max(v, (u32)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));   // lane ^ 2
}

}  // namespace sqllm
