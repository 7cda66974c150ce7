// 8-bit expert FFN of small batches (see zeda_fp8_ffn.hip for the formulas), where nothing but the streaming of the weights counts or
// where there are too few weight tiles to give every CU one: a tile of 256 weight rows makes 24 workgroups of 512 KiB each for one
// decoded token with four real slots.  Here a workgroup owns one unit row block (16 activations; 32 output columns) and up to 16
// token rows; its four waves split the reduction and fetch their units, all in flight at once, straight into the registers of
// the matrix instruction.  The token rows are rounded to 8 bits by every workgroup for itself, into LDS, while its weights are
// on their way: x in gate/up, the fp32 activations that gate/up leaves in down, whose 128-column blocks span eight workgroups.
// No launch for a quantisation is left, and for short calls none for placement and selection (zeda_place.h).
// HBM-bound: N=128, I=768, H=2048, 64 tokens (106 experts hit): gate/up 62.8 us = 5.3 TB/s, down 37.6 us = 4.4 TB/s; one token with four real
// slots 10.0 and 5.1 us, a chain of latencies (placement, weights, join of the waves' sums).
#include <type_traits>

#include "zeda_fp8.h"
#include "zeda_tile_select.h"

namespace zeda {

constexpr int kF8FewThreads = 256, kF8FewWaves = 4, kF8FewRows = 16;
constexpr int kF8FewDepth = 4;  // units in flight of a wave and row block (gate/up: eight leave room for three waves a SIMD, 126.1 us for the layer of 64 tokens; four 115.0)

template <typename T> __device__ __forceinline__ void few_load8(const T *p, float (&v)[8]);
template <> __device__ __forceinline__ void few_load8<bf16_t>(const bf16_t *p, float (&v)[8])
{
    const bf16x8 t = *reinterpret_cast<const bf16x8 *>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)t[i];
}
template <> __device__ __forceinline__ void few_load8<float>(const float *p, float (&v)[8])
{
    const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[i + 4] = b[i]; }
}

// LDS: a row's columns at row * (cols + 16) (16 rows' pieces then start in different banks), its scales behind all rows
__host__ __device__ constexpr int few_row(int cols) { return cols + 16; }
// (and behind them gate/up's weight scales)
__host__ __device__ constexpr int few_rows_bytes(int cols) { return kF8FewRows * (few_row(cols) + cols / kFp8Block) + 2 * (cols / kFp8Block); }
// ... and when the rows have been multiplied, the waves' sums of nf unit row blocks
__host__ __device__ constexpr int few_lds(int cols, int nf)
{
    return few_rows_bytes(cols) > nf * kF8FewWaves * 4096 ? few_rows_bytes(cols) : nf * kF8FewWaves * 4096;
}

// rows x src_cols of a matrix, filled up with zeros to cols columns, as e4m3 in LDS.  row_of(r): the row's address.
template <typename T, typename RowOf>
__device__ __forceinline__ void few_quantize(uint8_t *lds, int rows, int src_cols, int cols, const RowOf &row_of)
{
    const int nb = cols / kFp8Block, l16 = threadIdx.x & 15;
    uint8_t *scales = lds + kF8FewRows * few_row(cols);
    for (int g = threadIdx.x >> 4; g < rows * nb; g += kF8FewThreads / 16) {
        const int r = g / nb, b = g - r * nb, col = b * kFp8Block + l16 * 8;
        float v[8] = {};
        if (col < src_cols) few_load8<T>(row_of(r) + col, v);
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_abs(v[i]));
        const int sb = scale_byte(row_max(m));
        const float inv = scale_inverse(sb);
        u32x2_t o;
        o[0] = to_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
        o[1] = to_e4m3(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
        *reinterpret_cast<u32x2_t *>(lds + r * few_row(cols) + col) = o;
        if (l16 == 0) scales[r * nb + b] = (uint8_t)sb;
    }
}

// eight e4m3 values (two words) as bf16, exactly
__device__ __forceinline__ bf16x8 few_widen(uint32_t a, uint32_t b)
{
    bf16x8 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const auto t = k & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)(k < 2 ? a : b), 1.0f, true)
                             : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)(k < 2 ? a : b), 1.0f, false);
        v[2 * k] = t[0];
        v[2 * k + 1] = t[1];
    }
    return v;
}

// This wave's units of NF unit row blocks that follow each other (wave, wave + 4, ... along the columns; w: the first one's first
// bytes plus the lane's), in flight.
template <int NF>
struct FewUnits {
    static constexpr int DEPTH = kF8FewDepth;
    u32x4_t u[DEPTH][NF][2];
    const uint8_t *w;
    size_t block;  // bytes of a row block
    int n, wave;
    __device__ __forceinline__ void load(int d, int i)
    {
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const u32x4_t *p = reinterpret_cast<const u32x4_t *>(w + f * block + (size_t)(wave + kF8FewWaves * i) * kFp8Unit);
            u[d][f][0] = __builtin_nontemporal_load(p);
            u[d][f][1] = __builtin_nontemporal_load(p + 64);
        }
    }
    __device__ __forceinline__ void begin(const uint8_t *at, int units, int wv)
    {
        w = at;
        block = (size_t)units * kFp8Unit;
        wave = wv;
        n = (units - wave + kF8FewWaves - 1) / kF8FewWaves;
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (d < n) load(d, d);
    }
    // As multiply below, for one gate/up row block, with the products' sums as exact as fp32 sums are (ts: token scales, ws: gate scales, then
    // up scales, in LDS).  The activations are rounded to 8 bits afterwards: an error of the sums moves some of them across the middle
    // between two e4m3 values, by 6 to 12 % of the value.  The 8-bit instruction leaves 1.4e-5 (it adds products to 13 bits below the largest
    // one of a group), which did that to one activation in 5000: layer errors of 1.8e-3 to 6.6e-3 with few tokens where the formula in fp32 has
    // 1.7e-3.  So here the values are widened to bf16, which is exact, as are their products: 5e-8.  The weights' streaming hides it
    // (layer of 64 tokens, N=128, I=768, H=2048: 115.0 us, with the 8-bit instruction 116.7; one token 21.3 and 20.3).
    __device__ __forceinline__ void multiply_widened(uint8_t *lds, int cols, int rows)
    {
        static_assert(NF == 1, "");
        const int lane = threadIdx.x & 63, r = min(lane & (kF8FewRows - 1), rows - 1), half = lane >> 5, nb = cols / kFp8Block;
        const uint8_t *row = lds + r * few_row(cols) + 16 * half, *ts = lds + kF8FewRows * few_row(cols) + r * nb;
        const uint8_t *ws = lds + kF8FewRows * (few_row(cols) + nb);
        f32x16 acc = {};
        for (int i = 0; i < n; i += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (i + d >= n) break;
                const int kb = wave + kF8FewWaves * (i + d);
                const u32x4_t t[2] = {*reinterpret_cast<const u32x4_t *>(row + kb * 64), *reinterpret_cast<const u32x4_t *>(row + kb * 64 + 32)};
                f32x16 p = {};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const u32x4_t wq = u[d][0][q >> 1], tq = t[q >> 1];
                    const int o = 2 * (q & 1);
                    p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(few_widen(wq[o], wq[o + 1]), few_widen(tq[o], tq[o + 1]), p, 0, 0, 0);
                }
                const int s = (int)ts[kb >> 1] - 254, sg = s + ws[kb >> 1], su = s + ws[nb + (kb >> 1)];
#pragma unroll
                for (int k = 0; k < 16; ++k) acc[k] += __builtin_amdgcn_ldexpf(p[k], k < 8 ? sg : su);  // (unit rows 8 (k / 4) ..: gate, then up)
                if (i + d + DEPTH < n) load(d, i + d + DEPTH);
            }
        }
        leave(lds, &acc);
    }
    // Their products with the LDS rows (those past `rows` repeat the last one); ws: the weights' scales of this lane's row.  The waves'
    // sums take the rows' place: part[block][wave][q][l] = unit rows 8 q + 4 (l / 32) .. + 3, token row l % 32.
    __device__ __forceinline__ void multiply(uint8_t *lds, int cols, int rows, const uint8_t *ws)
    {
        const int lane = threadIdx.x & 63, r = min(lane & (kF8FewRows - 1), rows - 1), half = lane >> 5;
        const uint8_t *row = lds + r * few_row(cols) + 16 * half, *ts = lds + kF8FewRows * few_row(cols) + r * (cols / kFp8Block);
        f32x16 acc[NF];
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[f][i] = 0.f;
        for (int i = 0; i < n; i += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (i + d >= n) break;
                const int kb = wave + kF8FewWaves * (i + d);
                const u32x4_t t0 = *reinterpret_cast<const u32x4_t *>(row + kb * 64), t1 = *reinterpret_cast<const u32x4_t *>(row + kb * 64 + 32);
                const i32x8 b = __builtin_bit_cast(i32x8, __builtin_shufflevector(t0, t1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int f = 0; f < NF; ++f) {
                    const i32x8 a = __builtin_bit_cast(i32x8, __builtin_shufflevector(u[d][f][0], u[d][f][1], 0, 1, 2, 3, 4, 5, 6, 7));
                    acc[f] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc[f], 0, 0, 0, (int)ws[kb >> 1], 0, (int)ts[kb >> 1]);
                }
                if (i + d + DEPTH < n) load(d, i + d + DEPTH);
            }
        }
        leave(lds, acc);
    }
    __device__ __forceinline__ void leave(uint8_t *lds, const f32x16 *acc)
    {
        const int lane = threadIdx.x & 63;
        __syncthreads();
        f32x4 *part = reinterpret_cast<f32x4 *>(lds);
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                part[((f * kF8FewWaves + wave) * 4 + q) * 64 + lane] = f32x4{acc[f][4 * q], acc[f][4 * q + 1], acc[f][4 * q + 2], acc[f][4 * q + 3]};
        __syncthreads();
    }
    static __device__ __forceinline__ f32x4 total(const uint8_t *lds, int f, int q, int l)
    {
        const f32x4 *part = reinterpret_cast<const f32x4 *>(lds) + (f * kF8FewWaves * 4 + q) * 64 + l;
        f32x4 v = part[0];
#pragma unroll
        for (int w = 1; w < kF8FewWaves; ++w) v += part[w * 256];
        return v;
    }
};
struct FewArgs {
    const bf16_t *x;
    const uint8_t *w, *ws;
    const int32_t *offsets, *sorted_slot;
    float *act;  // [rows][I]: what gate/up leaves
    void *y;
    int16_t *y_exp;
    int T, N, K, H, I, Ip, log_terms;
    TilePlace tp;
};

template <int FROM>
__global__ __launch_bounds__(kF8FewThreads, 4) void fp8_few_gateup_kernel(FewArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ TilePlaceLds<kF8FewRows> s_place;
    constexpr int NF = 1;  // (two: 64 tokens, 106 experts hit, no faster: 64.5 us)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n_ft = a.Ip / (16 * NF);
    const int tile = blockIdx.x / n_ft, ft = blockIdx.x - tile * n_ft;
    int4 loc;
    if constexpr (FROM == kFromTables) {
        loc = locate_rows<kF8FewRows>(a.offsets, a.N, tile);
    } else if constexpr (FROM == kFromIds) {
        loc = place_tile<kF8FewRows>([&](int slot) { return a.tp.ids[slot]; }, a.T * a.K, a.N, tile, ft == 0, blockIdx.x == 0, s_place, a.tp.out);
    } else {
        __shared__ float s_lg[kTileSelTokens][kMaxExperts];
        __shared__ int s_ids[kTileSelTokens * kMaxK];
        select_tokens(a.tp, a.T, a.N, a.K, blockIdx.x == 0, s_lg, s_ids);
        loc = place_tile<kF8FewRows>([&](int slot) { return s_ids[slot]; }, a.T * a.K, a.N, tile, ft == 0, blockIdx.x == 0, s_place, a.tp.out);
    }
    if (loc.z == 0) return;
    FewUnits<NF> units;
    units.begin(a.w + ((size_t)loc.x * n_ft + ft) * NF * (a.H / 64) * kFp8Unit + lane * 16, a.H / 64, wave);
    few_quantize<bf16_t>(lds, loc.z, a.H, a.H, [&](int r) {
        const int slot = FROM != kFromTables ? s_place.list[r] : a.sorted_slot[loc.y + r];
        return a.x + (size_t)min(max(slot / a.K, 0), a.T - 1) * a.H;  // (a bad index must not fault)
    });
    const int nb = a.H / kFp8Block;
    for (int i = threadIdx.x; i < 2 * nb; i += kF8FewThreads)  // scales of the gate rows, of the up rows
        lds[kF8FewRows * (few_row(a.H) + nb) + i] = a.ws[(((size_t)loc.x * (a.Ip / kFp8Block) + (ft * NF >> 3)) * 2 + i / nb) * fp8_pitch(a.H) + i % nb];
    __syncthreads();
    units.multiply_widened(lds, a.H, loc.z);
    if (threadIdx.x < 4 * NF * kF8FewRows) {  // a thread: activations 4 f .. + 3 of a token row
        const int r = threadIdx.x / (4 * NF), f = threadIdx.x % (4 * NF), l = r + 32 * (f & 1), q = (f & 3) >> 1;
        const f32x4 g = units.total(lds, f >> 2, q, l), u = units.total(lds, f >> 2, q + 2, l);
        f32x4 h;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = g[i] / (1.0f + __expf(-g[i])) * u[i];
        const int col = ft * 16 * NF + 4 * f;
        if (r < loc.z && col < a.I) *reinterpret_cast<f32x4 *>(a.act + (size_t)(loc.y + r) * a.I + col) = h;
    }
}

template <bool SCALED>
__global__ __launch_bounds__(kF8FewThreads) void fp8_few_down_kernel(FewArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    constexpr int NF = 2;  // (64 tokens, I = 768: one 47 us, two 37, four 39)
    __shared__ int s_k[kF8FewRows];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n_ft = a.H / (32 * NF);
    const int tile = blockIdx.x / n_ft, ft = blockIdx.x - tile * n_ft, nb = a.Ip / kFp8Block;
    const int4 loc = locate_rows<kF8FewRows>(a.offsets, a.N, tile);
    if (loc.z == 0) return;
    FewUnits<NF> units;
    units.begin(a.w + ((size_t)loc.x * (a.H / 32) + ft * NF) * (a.Ip / 64) * kFp8Unit + lane * 16, a.Ip / 64, wave);
    few_quantize<float>(lds, loc.z, a.I, a.Ip, [&](int r) { return a.act + (size_t)(loc.y + r) * a.I; });
    __syncthreads();
    const uint8_t *ws = a.ws + ((size_t)loc.x * (a.H / kFp8Block) + ft * NF / 4) * fp8_pitch(a.Ip);
    if (SCALED && threadIdx.x < loc.z) {
        const uint8_t *ts = lds + kF8FewRows * few_row(a.Ip) + threadIdx.x * nb;
        int k = 0;
        for (int c = 0; c < nb; ++c) k = max(k, (int)ts[c] + (int)ws[c]);
        k += a.log_terms - 254 - 15;
        s_k[threadIdx.x] = k;
        if (ft * NF % 4 == 0) a.y_exp[(size_t)(loc.y + threadIdx.x) * (a.H / kFp8Block) + ft * NF / 4] = (int16_t)k;
    }
    units.multiply(lds, a.Ip, loc.z, ws);
    typedef std::conditional_t<SCALED, _Float16, bf16_t> out_t;
    typedef out_t out4 __attribute__((ext_vector_type(4)));
    for (int i = threadIdx.x; i < loc.z * 8 * NF; i += kF8FewThreads) {  // columns 4 f .. + 3 of a row
        const int f = i % (8 * NF), r = i / (8 * NF);
        const f32x4 v = units.total(lds, f >> 3, (f & 7) >> 1, r + 32 * (f & 1));
        out4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = (out_t)(SCALED ? ldexpf(v[j], -s_k[r]) : v[j]);
        *reinterpret_cast<out4 *>((out_t *)a.y + (size_t)(loc.y + r) * a.H + ft * 32 * NF + 4 * f) = o;
    }
}

// at most this many tiles of 16 rows
static int64_t few_tiles(const zeda_layer_desc *d)
{
    const int64_t slots = (int64_t)d->T * d->K;
    return (slots < d->N ? slots : d->N) + slots / kF8FewRows;
}

// Up to how many slots these kernels beat the tile kernels, which quantise the tokens in a launch of their own and take a workgroup per 128
// activations.  Every workgroup rounds the rows of its tile for itself, slots * Ip / 16 * H values in gate/up alone, and has a fixed cost like
// that of some 256 columns more in both directions: at slots * (Ip + 256) * (H + 256) of about 2.8e8 that is what the launches saved and a chip
// filled with more workgroups are worth, whatever the number of experts.  Where the layer's weights are past the last-level cache
// (256 MiB) twice over, their streaming hides the rounding as long as tiles of 16 rows seldom fetch an expert's weights twice and a
// workgroup's weights (32 H bytes) are more than its latency: up to 3.25 slots per expert if they fell evenly on all N + Z.
// Whole layer, us, tiles / here, weights from HBM (half of the slots on zero experts), up to the slots in brackets here:
//   N=16, I=1024, H=4096 (50): 16 slots 49.0 / 35.5, 48 55.2 / 55.2, 80 59.6 / 62.7;  I=256 (125): 120 46.6 / 38.4, 800 52.3 / 79.6
//   N=24, I=448, H=4096 (83): 60 53.6 / 44.7, 288 57.9 / 62.4;  H=1152 (258): 192 32.4 / 27.0, 480 33.2 / 34.0
//   N=64, I=512, H=1024 (284): 160 40.0 / 39.3, 320 41.9 / 45.0;  N=30, I=256, H=256 (1068): 400 22.9 / 20.5, 1200 23.8 / 23.9
//   N=200, I=64, H=128 (1898): 2000 25.7 / 27.9, 8800 29.4 / 39.7;  N=1, I=2048, H=2048 (52): 35 41.4 / 34.4, 60 41.7 / 39.2
//   N=128, I=768, H=2048 (520): 8 32.7 / 26.3, 128 67.4 / 58.6, 512 114.0 / 115.1, 640 119.5 / 126.1
//   N=64, I=1536, H=2048 (312): 4 31.8 / 23.8, 128 85.1 / 79.6, 256 111.0 / 113.9, 384 123.1 / 127.2
// Over 485 other shapes (N 4 to 220, I 128 to 2176, H 384 to 4480, 0.4 to 35 slots per expert) what is chosen is 0.6 % behind the better kernels on
// average and 41 % at worst; 1.5 and 51 % where one layer's weights stay in the cache from call to call.
// Above 45 slots per expert the tile kernels keep every call that they have had (one to three small experts would gain: N=3, I=512, H=512,
// 400 slots 29.2 / 22.8).
int64_t fp8_few_slots(const zeda_layer_desc *d)
{
    if (few_rows_bytes(d->H) > 72 * 1024 || few_rows_bytes(fp8_cols(d->I)) > 72 * 1024) return 0;  // (two workgroups to a CU)
    const int64_t H = d->H, Ip = fp8_cols(d->I), NE = (int64_t)d->N + d->Z;
    const int64_t rounded = 280000000 / ((H + 256) * (Ip + 256)), most = rounded < 45 * NE ? rounded : 45 * NE;
    const int64_t hidden = d->N * 3 * H * Ip >= 500000000 && H > 1024 ? 13 * NE / 4 : 0;
    return most > hidden ? most : hidden;
}
bool fp8_places(const zeda_layer_desc *d) { return fp8_few(d) && (int64_t)d->T * d->K <= kTileMaxSlots && few_tiles(d) * (fp8_cols(d->I) / 16) <= 7168; }
bool fp8_selects(const zeda_layer_desc *d)
{
    return d->T <= kTileSelTokens && fp8_places(d) && few_tiles(d) * (fp8_cols(d->I) / 16) <= 1024 && route_splits(d);
}

template <typename Kernel>
static int few_launch(Kernel kernel, bool (&done)[kMaxDevices], int64_t grid, int lds, const FewArgs &a, hipStream_t s)
{
    const int dev = current_device();
    if (dev < 0) return ZEDA_EHIP;
    if (!done[dev]) {  // per kernel and device (idempotent)
        if (hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 72 * 1024) != hipSuccess) return ZEDA_EHIP;
        done[dev] = true;
    }
    if (grid > 0x7fffffff) return ZEDA_EUNSUPPORTED;
    kernel<<<(unsigned)grid, kF8FewThreads, lds, s>>>(a);
    return last_launch_status();
}

int launch_ffn_fp8_few(const zeda_layer_desc *d, const void *x, const zeda_fp8_experts *e, const int32_t *offsets, const int32_t *sorted_slot,
                       void *y_slot, int16_t *y_exp, float *act, int log_terms, const TilePlace *tp, hipStream_t s)
{
    const int Ip = fp8_cols(d->I);
    FewArgs a = {(const bf16_t *)x, (const uint8_t *)e->w_gateup, (const uint8_t *)e->s_gateup, offsets, sorted_slot, act, y_slot, y_exp,
                 d->T, d->N, d->K, d->H, d->I, Ip, log_terms, tp ? *tp : TilePlace{}};
    static bool done[5][kMaxDevices] = {};
    const int64_t up = few_tiles(d) * (Ip / 16), down = few_tiles(d) * (d->H / 64);
    const int lds = few_lds(d->H, 1);
    const int rc = !tp           ? few_launch(fp8_few_gateup_kernel<kFromTables>, done[0], up, lds, a, s)
                   : tp->partial ? few_launch(fp8_few_gateup_kernel<kFromLogits>, done[1], up, lds, a, s)
                                 : few_launch(fp8_few_gateup_kernel<kFromIds>, done[2], up, lds, a, s);
    if (rc != ZEDA_OK) return rc;
    a.w = (const uint8_t *)e->w_down;
    a.ws = (const uint8_t *)e->s_down;
    return y_exp ? few_launch(fp8_few_down_kernel<true>, done[3], down, few_lds(Ip, 2), a, s)
                 : few_launch(fp8_few_down_kernel<false>, done[4], down, few_lds(Ip, 2), a, s);
}

}  // namespace zeda
