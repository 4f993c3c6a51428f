// Internal interface of the microscaled 4-bit format: element types, geometry of a packed matrix, launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>

#include "sqllm.h"

namespace sqllm {

constexpr int kMxBlock = 32;        // elements that share a scale
constexpr int kMxRowUnit = 128;     // elements a packed row is padded to: four blocks, whose scales are a dword, and one to four matrix instructions
constexpr int kMxMaxN = 0x7FFFFF80; // longest row: its padded length is still an int

inline int mx_padded(int n) { return (int)(((long long)n + kMxRowUnit - 1) / kMxRowUnit * kMxRowUnit); }
// units (or stages) of 256 columns that a packed row of K columns takes; K + 255 leaves an int
__host__ __device__ inline int mx_units(int K) { return K / 256 + (K % 256 != 0); }
inline size_t mx_row_code_bytes(int n) { return (size_t)mx_padded(n) / 2; }
inline size_t mx_row_scale_bytes(int n) { return (size_t)mx_padded(n) / kMxBlock; }
inline int mx_type_size(int type) { return type == SQLLM_F32 ? 4 : 2; }

struct MxQuantArgs {
    int M, N, type;
    const void* w;
    long long ldw;          // elements
    void *codes, *scales;       // blocks along the rows, or both NULL
    void *codes_t, *scales_t;   // the transpose, blocks along the columns, or both NULL
};
struct MxDequantArgs {
    int M, N, type;
    const void *codes, *scales;
    void* w;
    long long ldw;
};
struct MxGemvArgs {
    int M, N, B, accumulate;
    const void *codes, *scales, *x;
    void* y;
};
struct MxGemmArgs {
    int T, M, N, type, accumulate;
    const void *x_codes, *x_scales, *w_codes, *w_scales;
    void* y;
    long long ldy;          // elements
};
hipError_t launch_mx_quantize(const MxQuantArgs& a, hipStream_t s);
hipError_t launch_mx_dequantize(const MxDequantArgs& a, hipStream_t s);
hipError_t launch_mx_gemv(const MxGemvArgs& a, hipStream_t s);
hipError_t launch_mx_gemm(const MxGemmArgs& a, hipStream_t s);

}  // namespace sqllm
