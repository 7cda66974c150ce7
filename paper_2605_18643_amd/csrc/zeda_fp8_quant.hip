// Quantisation to 8 bits with block scales (see zeda_fp8.h) and the packed layout of the 8-bit expert weights.
#include "zeda_fp8.h"
#include "zeda_select.h"

namespace zeda {

template <typename T> __device__ __forceinline__ void load8(const T *p, float (&v)[8]);
template <> __device__ __forceinline__ void load8<bf16_t>(const bf16_t *p, float (&v)[8])
{
    const bf16x8 t = *reinterpret_cast<const bf16x8 *>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)t[i];
}
template <> __device__ __forceinline__ void load8<float>(const float *p, float (&v)[8])
{
    const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[i + 4] = b[i]; }
}

// Rows: 16 lanes take the 128 columns of one scale, eight each, and agree on their largest finite magnitude inside the lane row.
// HBM-bound: 2 or 4 bytes in, 1 out per element.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T *__restrict__ x, int rows, int cols, uint8_t *__restrict__ q, int ldq,
                                                            uint8_t *__restrict__ scales, int pitch)
{
    const int nb = (cols + kFp8Block - 1) / kFp8Block, l16 = threadIdx.x & 15;
    const int64_t g = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (g >= (int64_t)rows * nb) return;  // (whole lane rows leave together)
    const int r = (int)(g / nb), b = (int)(g - (int64_t)r * nb), col = b * kFp8Block + l16 * 8;
    float v[8] = {};
    if (col < cols) load8<T>(x + (size_t)r * cols + col, v);
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_abs(v[i]));
    const int sb = scale_byte(row_max(m));
    const float inv = scale_inverse(sb);
    u32x2_t o;
    o[0] = to_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
    o[1] = to_e4m3(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
    if (col < cols) *reinterpret_cast<u32x2_t *>(q + (size_t)r * ldq + col) = o;
    if (l16 == 0) scales[(size_t)r * pitch + b] = (uint8_t)sb;
}

int launch_quantize_rows(int rows, int cols, int dtype, const void *x, void *q, int ldq, uint8_t *scales, int pitch, hipStream_t s)
{
    const int64_t groups = (int64_t)rows * ceil_div(cols, kFp8Block), grid = (groups + 15) / 16;
    if (grid > 0x7fffffff) return ZEDA_EUNSUPPORTED;
    if (dtype == ZEDA_BF16) quantize_rows_kernel<bf16_t><<<(unsigned)grid, 256, 0, s>>>((const bf16_t *)x, rows, cols, (uint8_t *)q, ldq, scales, pitch);
    else quantize_rows_kernel<float><<<(unsigned)grid, 256, 0, s>>>((const float *)x, rows, cols, (uint8_t *)q, ldq, scales, pitch);
    return last_launch_status();
}

// Weights: a workgroup takes a block of 128 x 128, sixteen lanes a row, eight rows a thread; the block stays in registers
// between its largest magnitude and the conversion.
template <typename T>
__global__ __launch_bounds__(256) void quantize_weights_kernel(const T *__restrict__ w, int rows, int cols, uint8_t *__restrict__ q,
                                                               uint8_t *__restrict__ scales)
{
    __shared__ float s_max[4];
    const int rb = (rows + kFp8Block - 1) / kFp8Block, cb = (cols + kFp8Block - 1) / kFp8Block;
    const int b = blockIdx.x, c = b % cb, r = b / cb % rb;
    const size_t base = (size_t)(b / cb / rb) * rows * cols;
    const int col = c * kFp8Block + (threadIdx.x & 15) * 8, row0 = r * kFp8Block + (threadIdx.x >> 4);
    float v[8][8];
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[i][k] = 0.f;
        if (row0 + 16 * i < rows && col < cols) load8<T>(w + base + (size_t)(row0 + 16 * i) * cols + col, v[i]);
#pragma unroll
        for (int k = 0; k < 8; ++k) m = fmaxf(m, finite_abs(v[i][k]));
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
    if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = m;
    __syncthreads();
    const int sb = scale_byte(fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3])));
    const float inv = scale_inverse(sb);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        u32x2_t o;
        o[0] = to_e4m3(v[i][0] * inv, v[i][1] * inv, v[i][2] * inv, v[i][3] * inv);
        o[1] = to_e4m3(v[i][4] * inv, v[i][5] * inv, v[i][6] * inv, v[i][7] * inv);
        if (row0 + 16 * i < rows && col < cols) *reinterpret_cast<u32x2_t *>(q + base + (size_t)(row0 + 16 * i) * cols + col) = o;
    }
    if (threadIdx.x == 0) scales[b] = (uint8_t)sb;
}

int launch_quantize_weights(int count, int rows, int cols, int dtype, const void *w, void *q, uint8_t *scales, hipStream_t s)
{
    const int64_t grid = (int64_t)count * ceil_div(rows, kFp8Block) * ceil_div(cols, kFp8Block);
    if (grid > 0x7fffffff) return ZEDA_EUNSUPPORTED;
    if (dtype == ZEDA_BF16) quantize_weights_kernel<bf16_t><<<(unsigned)grid, 256, 0, s>>>((const bf16_t *)w, rows, cols, (uint8_t *)q, scales);
    else quantize_weights_kernel<float><<<(unsigned)grid, 256, 0, s>>>((const float *)w, rows, cols, (uint8_t *)q, scales);
    return last_launch_status();
}

// Packed weights: units of 32 rows x 64 columns, piece p (0, 1) of lane l = the 16 bytes at row l % 32, columns 32 p + 16 (l / 32) of
// the unit, at byte 1024 p + 16 l: the order in which the lanes of a wave hold a 32x32x64 matrix operand, so that a wave fetches
// one with two contiguous KiB.  The units of a row block follow each other along the columns.  gate and up share units: rows 0..15
// of unit row block ib are gate rows 16 ib .., rows 16..31 the up rows 16 ib .., so that a lane ends up with both factors of the
// same activation.  The intermediate dimension is filled up with zeros to whole blocks of 128.
// DOWN: q = q_down [N, H, I], else q = q_gate, q2 = q_up [N, I, H].  One thread per 16 bytes.
template <bool DOWN>
__global__ __launch_bounds__(256) void pack_fp8_kernel(const uint8_t *__restrict__ q, const uint8_t *__restrict__ q2, int N, int H, int I,
                                                       uint8_t *__restrict__ out)
{
    const int Ip = fp8_cols(I), rbs = DOWN ? H / 32 : Ip / 16, kbs = (DOWN ? Ip : H) / 64;
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, n = (size_t)N * rbs * kbs * (kFp8Unit / 16);
    if (i >= n) return;
    const int lane = (int)(i & 63), p = (int)(i >> 6) & 1;
    const size_t u = i >> 7;
    const int kb = (int)(u % kbs), rb = (int)(u / kbs % rbs), e = (int)(u / kbs / rbs);
    const int row = lane & 31, col = kb * 64 + 32 * p + 16 * (lane >> 5);
    u32x4_t v = {0u, 0u, 0u, 0u};
    if (DOWN) {
        if (col < I) v = *reinterpret_cast<const u32x4_t *>(q + ((size_t)e * H + rb * 32 + row) * I + col);
    } else {
        const int r = rb * 16 + (row & 15);
        if (r < I) v = *reinterpret_cast<const u32x4_t *>((row < 16 ? q : q2) + ((size_t)e * I + r) * H + col);
    }
    reinterpret_cast<u32x4_t *>(out)[i] = v;
}

// Scales beside them: gateup [N][Ip / 128][gate, up][pitch(H)], down [N][H / 128][pitch(I)], rows of whole words (padding: 1).
template <bool DOWN>
__global__ __launch_bounds__(256) void pack_fp8_scales_kernel(const uint8_t *__restrict__ s, const uint8_t *__restrict__ s2, int N, int H, int I,
                                                              uint8_t *__restrict__ out)
{
    const int Ib = fp8_cols(I) / kFp8Block, Hb = H / kFp8Block, pitch = fp8_pitch(DOWN ? I : H), cols = DOWN ? Ib : Hb;
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, rows = (size_t)N * (DOWN ? Hb : 2 * Ib);
    if (i >= rows * pitch) return;
    const int c = (int)(i % pitch);
    const size_t r = i / pitch;
    uint8_t v = 127;
    if (c < cols) v = DOWN ? s[r * cols + c] : ((r & 1) ? s2 : s)[(r >> 1) * cols + c];
    out[i] = v;
}

int launch_pack_fp8(const zeda_layer_desc *d, const uint8_t *q_gate, const uint8_t *s_gate, const uint8_t *q_up, const uint8_t *s_up,
                    const uint8_t *q_down, const uint8_t *s_down, const zeda_fp8_experts *out, hipStream_t s)
{
    const size_t Ip = fp8_cols(d->I), ng = (size_t)d->N * 2 * Ip * d->H / 16, nd = ng / 2;
    const size_t sg = (size_t)d->N * 2 * (Ip / kFp8Block) * fp8_pitch(d->H), sd = (size_t)d->N * (d->H / kFp8Block) * fp8_pitch(d->I);
    if ((ng + 255) / 256 > 0x7fffffffu) return ZEDA_EUNSUPPORTED;
    pack_fp8_kernel<false><<<(unsigned)((ng + 255) / 256), 256, 0, s>>>(q_gate, q_up, d->N, d->H, d->I, (uint8_t *)out->w_gateup);
    pack_fp8_kernel<true><<<(unsigned)((nd + 255) / 256), 256, 0, s>>>(q_down, nullptr, d->N, d->H, d->I, (uint8_t *)out->w_down);
    pack_fp8_scales_kernel<false><<<(unsigned)((sg + 255) / 256), 256, 0, s>>>(s_gate, s_up, d->N, d->H, d->I, (uint8_t *)out->s_gateup);
    pack_fp8_scales_kernel<true><<<(unsigned)((sd + 255) / 256), 256, 0, s>>>(s_down, nullptr, d->N, d->H, d->I, (uint8_t *)out->s_down);
    return last_launch_status();
}

}  // namespace zeda
