// 8-bit operands with block scales: e4m3 values (the finite-only OCP format, largest value 448) under a power-of-two scale for
// every 128 columns of a token row and every 128 x 128 block of a weight matrix, held as the byte s of 2^(s - 127).
#pragma once
#include "zeda_internal.h"

namespace zeda {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

constexpr int kFp8Block = 128;       // columns (and weight rows) under one scale
constexpr int kFp8Unit = 2048;       // bytes of a packed unit: 32 rows x 64 columns
constexpr int kFp8MaxWidth = 16384;  // H, I: a token tile's scales are kept in LDS

__host__ __device__ inline int fp8_cols(int n) { return (n + kFp8Block - 1) / kFp8Block * kFp8Block; }
// scale bytes of a row of n columns, whole words
__host__ __device__ inline int fp8_pitch(int n) { return (fp8_cols(n) / kFp8Block + 3) / 4 * 4; }

__device__ __forceinline__ float finite_abs(float v) { return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u ? 0.f : fabsf(v); }
// The byte of the least power of two that keeps amax (finite) within 448 = 1.75 * 2^8, at least 2^-126: a power of two, so that
// dividing by it is exact, and so that the matrix instruction can apply it.  What it costs against amax / 448 is at most one
// binade of the values' range below 448 * 2^-15, whose elements are rounded to multiples of a fixed step.
__device__ __forceinline__ int scale_byte(float amax) { return max((int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 8, 1); }
__device__ __forceinline__ float scale_inverse(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }
// four values, already divided by their scale, to the nearest e4m3 values, ties to even (no-numbers and infinities give 0x7f or 0xff)
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d)
{
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}

// launchers (arguments are validated)
int launch_quantize_rows(int rows, int cols, int dtype, const void *x, void *q, int ldq, uint8_t *scales, int pitch, hipStream_t s);
int launch_quantize_weights(int count, int rows, int cols, int dtype, const void *w, void *q, uint8_t *scales, hipStream_t s);
int launch_pack_fp8(const zeda_layer_desc *d, const uint8_t *q_gate, const uint8_t *s_gate, const uint8_t *q_up, const uint8_t *s_up,
                    const uint8_t *q_down, const uint8_t *s_down, const zeda_fp8_experts *out, hipStream_t s);
size_t fp8_ffn_ws_bytes(const zeda_layer_desc *d);
// y_exp: NULL (y_slot receives bf16), or receives where the exponents of the rows' 128-column blocks are (y_slot: fp16, for
// launch_combine_scaled)
int launch_ffn_fp8(const zeda_layer_desc *d, const void *x, const zeda_fp8_experts *e, const int32_t *offsets, const int32_t *sorted_slot,
                   void *y_slot, const int16_t **y_exp, void *ws, const TilePlace *tp, hipStream_t s);
// the same for small batches; act: fp32 scratch [T*K][I]
int64_t fp8_few_slots(const zeda_layer_desc *d);  // T * K up to which these are the better ones; 0: never
inline bool fp8_few(const zeda_layer_desc *d) { return (int64_t)d->T * d->K <= fp8_few_slots(d); }
bool fp8_places(const zeda_layer_desc *d);   // its gate/up kernel places the slots (tp is given; offsets and sorted_slot are then outputs)
bool fp8_selects(const zeda_layer_desc *d);  // ... and selects, from the partial logits of the router's first kernel
int launch_ffn_fp8_few(const zeda_layer_desc *d, const void *x, const zeda_fp8_experts *e, const int32_t *offsets, const int32_t *sorted_slot,
                       void *y_slot, int16_t *y_exp, float *act, int log_terms, const TilePlace *tp, hipStream_t s);

}  // namespace zeda
