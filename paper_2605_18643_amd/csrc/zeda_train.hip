// Training of the router (Section 2.2: the balance losses L_A, Eq. 4, and L_GA, Eq. 5-6) and of the routing weights of Eq. 1:
//   zeda_route_train      logits -> softmax, top-K, gates; per-expert counts, mean probabilities and the losses
//   zeda_route_backward   gradients of losses and gates -> logits -> x, w_router, router_bias
//   zeda_combine_backward gradient of the layer output -> gates, expert outputs
#include <limits.h>

#include <type_traits>

#include "zeda_internal.h"
#include "zeda_select.h"

namespace zeda {

// ---------------------------------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------------------------------
// 16 tokens a workgroup, four a wave: adds the logit tables and the bias, selects (select_rows, as the router), keeps the
// probabilities, and leaves for the batch sums: part_p[block][NE] = sum of the probabilities of the tokens that count,
// part_c[block][NE + 1] = their slots on every expert, and their number.
constexpr int kTrainTokens = 16;

template <int NB>
__global__ __launch_bounds__(256) void train_select_kernel(const float *__restrict__ tables, int slices, int Tpad,
                                                           const float *__restrict__ bias, const uint8_t *__restrict__ mask, int T, int N,
                                                           int NE, int K, int gate_norm, int32_t *__restrict__ ids, float *__restrict__ gates,
                                                           float *__restrict__ probs, float *__restrict__ part_p, int32_t *__restrict__ part_c)
{
    constexpr int E = NB * 32, LD = E + 1;
    __shared__ float lg[kTrainTokens * LD];
    __shared__ int s_cnt[kMaxExperts], s_on[kTrainTokens];
    const int t0 = blockIdx.x * kTrainTokens, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nt = min(kTrainTokens, T - t0);
    for (int i = tid; i < kTrainTokens * E / 4; i += 256) {
        const int tk = i / (E / 4), e = (i - tk * (E / 4)) * 4;
        f32x4 v = *reinterpret_cast<const f32x4 *>(tables + (size_t)(t0 + tk) * E + e);
        for (int q = 1; q < slices; ++q) v += *reinterpret_cast<const f32x4 *>(tables + ((size_t)q * Tpad + t0 + tk) * E + e);
#pragma unroll
        for (int k = 0; k < 4; ++k) lg[tk * LD + e + k] = v[k] + (bias ? bias[min(e + k, NE - 1)] : 0.f);
    }
    if (tid < kMaxExperts) s_cnt[tid] = 0;
    if (tid < kTrainTokens) s_on[tid] = tid < nt && (!mask || mask[t0 + tid]);
    __syncthreads();
    const float no_bias[2 * NB] = {};
    const int id = select_rows<2 * NB, 1>(lg, LD, 0, no_bias, 4 * wave, kTrainTokens, t0, T, NE, N, K, gate_norm, ids, gates, lg, LD);
    if ((unsigned)id < (unsigned)kMaxExperts && s_on[4 * wave + (lane >> 4)]) atomicAdd(&s_cnt[id], 1);
    __syncthreads();
    for (int i = tid; i < nt * NE; i += 256) probs[(size_t)t0 * NE + i] = lg[(i / NE) * LD + i % NE];
    if (tid < NE) {
        float p = 0.f;
#pragma unroll
        for (int tk = 0; tk < kTrainTokens; ++tk) p += s_on[tk] ? lg[tk * LD + tid] : 0.f;
        part_p[(size_t)blockIdx.x * NE + tid] = p;
        part_c[(size_t)blockIdx.x * (NE + 1) + tid] = s_cnt[tid];
    }
    if (tid == 0) {
        int n = 0;
        for (int tk = 0; tk < kTrainTokens; ++tk) n += s_on[tk];
        part_c[(size_t)blockIdx.x * (NE + 1) + NE] = n;
    }
}

// The batch sums and the losses, by one workgroup; sums over blocks in 64 bits and in a fixed order.
constexpr int kTrainFinalThreads = 1024;
__global__ __launch_bounds__(kTrainFinalThreads) void train_final_kernel(const float *__restrict__ part_p, const int32_t *__restrict__ part_c, int nblk,
                                                                         int N, int NE, int K, float alpha, float w, int32_t *__restrict__ counts,
                                                                         float *__restrict__ P, float *__restrict__ summary)
{
    __shared__ double s_p[kTrainFinalThreads];
    __shared__ int s_c[kTrainFinalThreads], s_n[kTrainFinalThreads];
    __shared__ double s_f[kMaxExperts], s_P[kMaxExperts];
    const int tid = threadIdx.x, parts = kTrainFinalThreads / NE, e = tid % NE, part = tid / NE;
    double p = 0.;
    int c = 0, n = 0;
    if (part < parts)
        for (int b = part; b < nblk; b += parts) {
            p += (double)part_p[(size_t)b * NE + e];
            c += part_c[(size_t)b * (NE + 1) + e];
        }
    for (int b = tid; b < nblk; b += kTrainFinalThreads) n += part_c[(size_t)b * (NE + 1) + NE];
    s_p[tid] = p;
    s_c[tid] = c;
    s_n[tid] = n;
    __syncthreads();
    for (int h = kTrainFinalThreads / 2; h >= 1; h >>= 1) {
        if (tid < h) s_n[tid] += s_n[tid + h];
        __syncthreads();
    }
    if (tid < NE) {
        for (int q = 1; q < parts; ++q) { p += s_p[q * NE + tid]; c += s_c[q * NE + tid]; }
        const double all = s_n[0] > 0 ? s_n[0] : 1;  // nothing counts: f = P = 0
        s_f[tid] = c / all;
        s_P[tid] = p / all;
        counts[tid] = c;
        P[tid] = (float)(p / all);
    }
    __syncthreads();
    if (tid == 0) {
        double fE = 0., PE = 0., fZ = 0., PZ = 0., fP = 0.;
        for (int i = 0; i < NE; ++i) {
            fP += s_f[i] * s_P[i];
            (i < N ? fE : fZ) += s_f[i];
            (i < N ? PE : PZ) += s_P[i];
        }
        const double Zw = (double)(NE - N) * w;
        summary[0] = (float)fE; summary[1] = (float)PE; summary[2] = (float)fZ; summary[3] = (float)PZ;
        summary[4] = (float)(fZ / K);
        summary[5] = (float)((double)alpha * NE / K * fP);                                                  // Eq. 4
        summary[6] = (float)((double)alpha * (N + Zw) / K * (fE * PE / N + (NE > N ? fZ * PZ / Zw : 0.)));  // Eq. 5-6
    }
}

struct TrainWs {
    size_t tables, part_p, part_c, total;
};
static TrainWs train_ws(const zeda_layer_desc *d)
{
    const size_t nblk = ceil_div(d->T, kTrainTokens), NE = d->N + d->Z;
    TrainWs w;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes ? bytes : 1, 256); return at; };
    w.tables = take(route_tables(d).bytes());
    w.part_p = take(nblk * NE * 4);
    w.part_c = take(nblk * (NE + 1) * 4);
    w.total = o;
    return w;
}
size_t route_train_ws_bytes(const zeda_layer_desc *d) { return train_ws(d).total; }

int launch_route_train(const zeda_layer_desc *d, const void *x, const void *wr, const float *bias, const uint8_t *mask, float alpha, float w,
                       int32_t *ids, float *gates, float *probs, int32_t *counts, float *P, float *summary, void *ws, hipStream_t s)
{
    const TrainWs L = train_ws(d);
    const RouteTables t = route_tables(d);
    float *tables = (float *)((char *)ws + L.tables), *part_p = (float *)((char *)ws + L.part_p);
    int32_t *part_c = (int32_t *)((char *)ws + L.part_c);
    const int NE = d->N + d->Z, nblk = ceil_div(d->T, kTrainTokens);
    if (d->T > 0) {
        const int rc = launch_route_tables(d, x, wr, tables, s);
        if (rc != ZEDA_OK) return rc;
#define ZEDA_TRAIN(NB) train_select_kernel<NB><<<nblk, 256, 0, s>>>(tables, t.slices, t.Tpad, bias, mask, d->T, d->N, NE, d->K, d->gate_norm, ids, gates, probs, part_p, part_c)
        switch (t.E / 32) {
            case 1: ZEDA_TRAIN(1); break; case 2: ZEDA_TRAIN(2); break; case 3: ZEDA_TRAIN(3); break; case 4: ZEDA_TRAIN(4); break;
            case 5: ZEDA_TRAIN(5); break; case 6: ZEDA_TRAIN(6); break; case 7: ZEDA_TRAIN(7); break; default: ZEDA_TRAIN(8); break;
        }
#undef ZEDA_TRAIN
        if (hipGetLastError() != hipSuccess) return ZEDA_EHIP;
    }
    train_final_kernel<<<1, kTrainFinalThreads, 0, s>>>(part_p, part_c, nblk, d->N, NE, d->K, alpha, w, counts, P, summary);
    return last_launch_status();
}

// ---------------------------------------------------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------------------------------------------------
// The gradient of the logits,
//   dl_e = p_e (a_e - sum_j p_j a_j) + the gates' part,   a_e = (dL_A alpha (N+Z)/K f_e + dL_GA alpha (N + Z w)/K f_E/N or f_Z/(Z w)) / n,
// does not change when a constant is added to a: the slopes' mean is taken off in 64 bits, so that the difference keeps what the
// slopes differ by.  Gates: SOFTMAX adds dg_j to a at the selected experts; the normalised forms add g_j (dg_j - s), s = sum_l dg_l g_l,
// on the experts of the denominator and g_j dg_j on a selected expert outside it.
constexpr int kBackTokens = 64;

// bf16 parts by truncation: v = v0 + v1 + v2 exactly (24 bits)
__device__ __forceinline__ uint16_t top_bits(float v) { return (uint16_t)(__float_as_uint(v) >> 16); }
__device__ __forceinline__ float top_part(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }

struct LogitGrad {
    const float *probs, *gates, *d_loss, *d_gates;
    const int32_t *ids, *counts;
    const uint8_t *mask;
    int T, N, NE, K, gate_norm;
    float alpha, w;
    void *rows, *cols;    // dl as [parts][Tp][NEp] and [parts][NEp][Tp]
    float *part_b;        // [blocks][NE]: sums over the block's tokens
    int Tp, NEp;
};

// A wave takes a token at a time, lane l the experts l, l + 64, ...  F32: both copies in fp32; else the rows as two bf16 parts (their
// product is rounded to bf16), the columns as three (theirs stays fp32: nothing of dl is lost).
template <bool F32>
__global__ __launch_bounds__(256) void logit_grad_kernel(LogitGrad a)
{
    extern __shared__ float s_dl[];  // [kBackTokens][LD]
    __shared__ float s_a[kMaxExperts];
    __shared__ double s_red[2][4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, t0 = blockIdx.x * kBackTokens, NE = a.NE, N = a.N, LD = a.NEp + 1;
    {
        // slopes: thread e expert e
        const double c = tid < NE ? (double)a.counts[tid] : 0.;
        auto block_sum = [&](double v, int k) {
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
            if (lane == 0) s_red[k][wave] = v;
            __syncthreads();
            const double r = (s_red[k][0] + s_red[k][1]) + (s_red[k][2] + s_red[k][3]);
            __syncthreads();
            return r;
        };
        const double cE = block_sum(tid < N ? c : 0., 0), cZ = block_sum(tid < N ? 0. : c, 1);
        const double n = fmax(1., (cE + cZ) / a.K);
        const double Zw = (double)(NE - N) * a.w, lA = a.d_loss ? (double)a.d_loss[0] : 0., lG = a.d_loss ? (double)a.d_loss[1] : 0.;
        double v = tid < NE ? (double)a.alpha / a.K * (lA * NE * c + lG * (N + Zw) * (tid < N ? cE / N : cZ / Zw)) / n / n : 0.;
        const double mean = block_sum(v, 0) / NE;
        if (tid < NE) s_a[tid] = (float)(v - mean);
        __syncthreads();
    }
    for (int k = wave; k < kBackTokens; k += 4) {
        const int t = t0 + k;
        const bool on = t < a.T && (!a.mask || a.mask[t]);
        float dl[4] = {0.f, 0.f, 0.f, 0.f};
        if (on) {
            float p[4], u[4], g_of[4] = {}, v_of[4] = {};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int e = lane + 64 * q;
                p[q] = e < NE ? a.probs[(size_t)t * NE + e] : 0.f;
                u[q] = e < NE ? s_a[e] : 0.f;
            }
            float s = 0.f;
            if (a.d_gates) {
                int id = -1;
                float g = 0.f, dg = 0.f;
                if (lane < a.K) {
                    id = a.ids[(size_t)t * a.K + lane];
                    g = a.gates[(size_t)t * a.K + lane];
                    dg = a.d_gates[(size_t)t * a.K + lane];
                    if ((unsigned)id >= (unsigned)NE) id = -1, g = dg = 0.f;
                }
                for (int j = 0; j < a.K; ++j) {
                    const int ej = __builtin_amdgcn_readlane(id, j);
                    const float gj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(g), j));
                    const float dj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(dg), j));
                    s = fmaf(gj, dj, s);
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (ej == lane + 64 * q) {
                            if (a.gate_norm == ZEDA_GATE_SOFTMAX) {
                                u[q] += dj;
                            } else {
                                v_of[q] = fmaf(gj, dj, v_of[q]);
                                if (a.gate_norm == ZEDA_GATE_TOPK_NORM || ej < N) g_of[q] += gj;
                            }
                        }
                }
            }
            float pa = 0.f;
#pragma unroll
            for (int q = 0; q < 4; ++q) pa = fmaf(p[q], u[q], pa);
            pa = wave_sum(pa);
#pragma unroll
            for (int q = 0; q < 4; ++q) dl[q] = lane + 64 * q < NE ? p[q] * (u[q] - pa) + (v_of[q] - s * g_of[q]) : 0.f;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (lane + 64 * q < a.NEp) s_dl[k * LD + lane + 64 * q] = dl[q];
    }
    __syncthreads();
    if (tid < NE) {
        double b = 0.;
        for (int k = 0; k < kBackTokens; ++k) b += (double)s_dl[k * LD + tid];
        a.part_b[(size_t)blockIdx.x * NE + tid] = (float)b;
    }
    const int Tp = a.Tp, NEp = a.NEp;
    for (int i = tid; i < kBackTokens * NEp; i += 256) {
        const int k = i / NEp, e = i - k * NEp;
        const float v = s_dl[k * LD + e];
        const size_t at = (size_t)(t0 + k) * NEp + e;
        if (F32) {
            ((float *)a.rows)[at] = v;
        } else {
            ((uint16_t *)a.rows)[at] = top_bits(v);
            ((uint16_t *)a.rows)[(size_t)Tp * NEp + at] = top_bits(v - top_part(v));
        }
    }
    for (int i = tid; i < kBackTokens * NEp; i += 256) {
        const int e = i / kBackTokens, k = i - e * kBackTokens;
        const float v = s_dl[k * LD + e];
        const size_t at = (size_t)e * Tp + t0 + k;
        if (F32) {
            ((float *)a.cols)[at] = v;
        } else {
            const float m = v - top_part(v);
            ((uint16_t *)a.cols)[at] = top_bits(v);
            ((uint16_t *)a.cols)[(size_t)Tp * NEp + at] = top_bits(m);
            ((uint16_t *)a.cols)[(size_t)2 * Tp * NEp + at] = top_bits(m - top_part(m));
        }
    }
}

// Four columns of eight rows of a bf16 matrix, two words a row, to the rows' bf16 of each column: the operand of a product whose
// reduction runs along the rows.
__device__ __forceinline__ void turn8x4(const uint2 (&r)[8], bf16x8 (&c)[4])
{
    uint32_t o[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o[0][i] = __builtin_amdgcn_perm(r[2 * i + 1].x, r[2 * i].x, 0x05040100u);
        o[1][i] = __builtin_amdgcn_perm(r[2 * i + 1].x, r[2 * i].x, 0x07060302u);
        o[2][i] = __builtin_amdgcn_perm(r[2 * i + 1].y, r[2 * i].y, 0x05040100u);
        o[3][i] = __builtin_amdgcn_perm(r[2 * i + 1].y, r[2 * i].y, 0x07060302u);
    }
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = __builtin_bit_cast(bf16x8, u32x4{o[k][0], o[k][1], o[k][2], o[k][3]});
}

// dx[T, H] = dl w_router.  A wave keeps its 64 columns of w_router (all experts) in registers and walks over 16-token blocks.
// Lane (l16, kq) of a 16x16x32 product: columns 4 l16 .. + 3 as four operands, experts 8 kq .. + 7 of the step.
constexpr int kDxTokens = 128;
template <int KS>  // steps of 32 experts
__global__ __launch_bounds__(256) void router_dx_bf16_kernel(const uint16_t *__restrict__ dl, const bf16_t *__restrict__ wr, int T, int H, int NE,
                                                             int Tp, bf16_t *__restrict__ dx)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, kq = lane >> 4;
    const int h0 = (blockIdx.y * 4 + wave) * 64;
    if (h0 >= H) return;
    bf16x8 wf[KS][4];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        uint2 r[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = 32 * k + 8 * kq + i;
            r[i] = e < NE ? *reinterpret_cast<const uint2 *>(wr + (size_t)e * H + h0 + 4 * l16) : make_uint2(0, 0);
        }
        turn8x4(r, wf[k]);
    }
    constexpr int NEp = KS * 32;
    for (int t0 = blockIdx.x * kDxTokens; t0 < min(T, (int)(blockIdx.x + 1) * kDxTokens); t0 += 16) {
        f32x4 acc[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
        bf16x8 df[2][KS];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int k = 0; k < KS; ++k)
                df[q][k] = *reinterpret_cast<const bf16x8 *>(dl + ((size_t)q * Tp + t0 + l16) * NEp + 32 * k + 8 * kq);
#pragma unroll
        for (int q = 1; q >= 0; --q)
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(df[q][k], wf[k][c], acc[c], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + 4 * kq + i;
            bf16x4 v;
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = (bf16_t)acc[c][i];
            if (t < T) *reinterpret_cast<bf16x4 *>(dx + (size_t)t * H + h0 + 4 * l16) = v;
        }
    }
}

// The same in fp32 on the fp32 matrix instruction: a wave has 64 tokens and 64 columns, 16 experts a step (lane (l16, kq): experts
// 4 kq .. + 3, one to each of four products).  Columns past H (H % 4 == 0) are left out.
__global__ __launch_bounds__(256) void router_dx_f32_kernel(const float *__restrict__ dl, const float *__restrict__ wr, int T, int H, int NE, int NEp,
                                                            float *__restrict__ dx)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, kq = lane >> 4;
    const int h0 = (blockIdx.y * 4 + wave) * 64, t0 = blockIdx.x * kBackTokens, h = h0 + 4 * l16;
    if (h0 >= H) return;
    f32x4 acc[4][4];  // [token block][column operand]
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[b][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int e0 = 0; e0 < NEp; e0 += 16) {
        f32x4 wf[4], df[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = e0 + 4 * kq + i;
            wf[i] = e < NE && h < H ? *reinterpret_cast<const f32x4 *>(wr + (size_t)e * H + h) : f32x4{0.f, 0.f, 0.f, 0.f};
            df[i] = *reinterpret_cast<const f32x4 *>(dl + (size_t)(t0 + 16 * i + l16) * NEp + e0 + 4 * kq);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[b][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(df[b][i], wf[i][c], acc[b][c], 0, 0, 0);
    }
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + 16 * b + 4 * kq + i;
            if (t < T && h < H) *reinterpret_cast<f32x4 *>(dx + (size_t)t * H + h) = f32x4{acc[b][0][i], acc[b][1][i], acc[b][2][i], acc[b][3][i]};
        }
}

// dw_router[NE, H] = dl^T x, split over the tokens: part[split][NE16][H], added up by reduce_dw_kernel.  A wave has 64 columns and EB
// blocks of 16 experts.  Rows of tokens that do not count are taken as zero whatever they hold.
template <int EB, bool F32>
__global__ __launch_bounds__(256) void router_dw_kernel(const void *__restrict__ dlT, const void *__restrict__ xv, const uint8_t *__restrict__ mask, int T,
                                                        int H, int Tp, int NEp, int per, float *__restrict__ part, int NE16)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, kq = lane >> 4;
    const int h0 = (blockIdx.x * 4 + wave) * 64, h = h0 + 4 * l16, e0 = blockIdx.z * EB * 16, ta = blockIdx.y * per, tb = min(ta + per, T);
    if (h0 >= H) return;
    f32x4 acc[EB][4];
#pragma unroll
    for (int b = 0; b < EB; ++b)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[b][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto counts = [&](int t) { return t < T && (!mask || mask[t]); };
    if constexpr (F32) {
        const float *x = (const float *)xv, *dl = (const float *)dlT;
        for (int t = ta; t < tb; t += 16) {
            f32x4 xf[4], df[EB];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                xf[i] = h < H && counts(t + 4 * kq + i) ? *reinterpret_cast<const f32x4 *>(x + (size_t)(t + 4 * kq + i) * H + h) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = 0; b < EB; ++b) df[b] = *reinterpret_cast<const f32x4 *>(dl + (size_t)min(e0 + 16 * b + l16, NEp - 1) * Tp + t + 4 * kq);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int b = 0; b < EB; ++b)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[b][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(df[b][i], xf[i][c], acc[b][c], 0, 0, 0);
        }
    } else {
        const bf16_t *x = (const bf16_t *)xv;
        const uint16_t *dl = (const uint16_t *)dlT;
        for (int t = ta; t < tb; t += 32) {
            uint2 r[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                r[i] = counts(t + 8 * kq + i) ? *reinterpret_cast<const uint2 *>(x + (size_t)(t + 8 * kq + i) * H + h) : make_uint2(0, 0);
            bf16x8 xf[4];
            turn8x4(r, xf);
#pragma unroll
            for (int q = 2; q >= 0; --q) {
                bf16x8 df[EB];
#pragma unroll
                for (int b = 0; b < EB; ++b)
                    df[b] = *reinterpret_cast<const bf16x8 *>(dl + ((size_t)q * NEp + min(e0 + 16 * b + l16, NEp - 1)) * Tp + t + 8 * kq);
#pragma unroll
                for (int b = 0; b < EB; ++b)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[b][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(df[b], xf[c], acc[b][c], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int b = 0; b < EB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = e0 + 16 * b + 4 * kq + i;
            if (e < NE16 && h < H)
                *reinterpret_cast<f32x4 *>(part + ((size_t)blockIdx.y * NE16 + e) * H + h) = f32x4{acc[b][0][i], acc[b][1][i], acc[b][2][i], acc[b][3][i]};
        }
}

// dw = the splits' sums, dbias = the token blocks' sums (last workgroup); in a fixed order
__global__ __launch_bounds__(256) void reduce_dw_kernel(const float *__restrict__ part, int splits, int NE, int NE16, int H, float *__restrict__ dw,
                                                        const float *__restrict__ part_b, int nblk, float *__restrict__ dbias)
{
    if (blockIdx.x == gridDim.x - 1) {
        if (dbias && threadIdx.x < NE) {
            double b = 0.;
            for (int k = 0; k < nblk; ++k) b += (double)part_b[(size_t)k * NE + threadIdx.x];
            dbias[threadIdx.x] = (float)b;
        }
        return;
    }
    const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (!dw || i >= (size_t)NE * H) return;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int q = 0; q < splits; ++q) v += *reinterpret_cast<const f32x4 *>(part + (size_t)q * NE16 * H + i);
    *reinterpret_cast<f32x4 *>(dw + i) = v;
}

struct BackWs {
    size_t rows, cols, part_b, part, total;
    int Tp, NEp, NE16, splits, per, nblk;
};
static BackWs back_ws(const zeda_layer_desc *d)
{
    const int NE = d->N + d->Z;
    const size_t es = d->dtype == ZEDA_BF16 ? 2 : 4;
    BackWs w;
    w.nblk = ceil_div(d->T, kBackTokens);
    w.Tp = w.nblk * kBackTokens;
    w.NEp = ceil_div(NE, 32) * 32;
    w.NE16 = ceil_div(NE, 16) * 16;
    // token ranges: enough workgroups for the chip, whole blocks of 64 tokens
    const int cols = ceil_div(d->H, 256) * ceil_div(w.NE16 / 16, 8);
    int splits = ceil_div(512, cols);
    if (splits > w.nblk) splits = w.nblk;
    if (splits < 1) splits = 1;
    w.per = ceil_div(w.nblk, splits) * kBackTokens;
    w.splits = w.nblk ? ceil_div(w.Tp, w.per) : 0;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes ? bytes : 1, 256); return at; };
    const size_t n = (size_t)w.Tp * w.NEp * es;
    w.rows = take(n * (es == 2 ? 2 : 1));
    w.cols = take(n * (es == 2 ? 3 : 1));
    w.part_b = take((size_t)w.nblk * NE * 4);
    w.part = take((size_t)w.splits * w.NE16 * d->H * 4);
    w.total = o;
    return w;
}
size_t route_backward_ws_bytes(const zeda_layer_desc *d) { return back_ws(d).total; }

template <bool F32>
static int launch_logit_grad(const LogitGrad &g, int nblk, hipStream_t s)
{
    static bool done[kMaxDevices] = {};  // (more LDS than a launch gets by default) per instantiation and device, idempotent
    const int dev = current_device();
    if (dev < 0) return ZEDA_EHIP;
    if (!done[dev]) {
        if (hipFuncSetAttribute((const void *)logit_grad_kernel<F32>, hipFuncAttributeMaxDynamicSharedMemorySize, kBackTokens * (kMaxExperts + 1) * 4) != hipSuccess)
            return ZEDA_EHIP;
        done[dev] = true;
    }
    logit_grad_kernel<F32><<<nblk, 256, kBackTokens * (g.NEp + 1) * 4, s>>>(g);
    return last_launch_status();
}

int launch_route_backward(const zeda_layer_desc *d, const void *x, const void *wr, const float *probs, const int32_t *ids, const float *gates,
                          const uint8_t *mask, const int32_t *counts, float alpha, float w, const float *d_loss, const float *d_gates, void *dx,
                          float *dw, float *dbias, void *ws, hipStream_t s)
{
    const BackWs L = back_ws(d);
    const int NE = d->N + d->Z, H = d->H;
    const bool f32 = d->dtype != ZEDA_BF16;
    char *b = (char *)ws;
    float *part_b = (float *)(b + L.part_b), *part = (float *)(b + L.part);
    if (d->T > 0) {
        const LogitGrad g = {probs, gates, d_loss, d_gates, ids, counts, mask, d->T, d->N, NE, d->K, d->gate_norm, alpha, w,
                             b + L.rows, b + L.cols, part_b, L.Tp, L.NEp};
        int rc = f32 ? launch_logit_grad<true>(g, L.nblk, s) : launch_logit_grad<false>(g, L.nblk, s);
        if (rc != ZEDA_OK) return rc;
        if (dx) {
            if (f32) {
                router_dx_f32_kernel<<<dim3(L.nblk, ceil_div(H, 256)), 256, 0, s>>>((const float *)(b + L.rows), (const float *)wr, d->T, H, NE, L.NEp,
                                                                                   (float *)dx);
            } else {
                const dim3 grid(ceil_div(d->T, kDxTokens), ceil_div(H, 256));
#define ZEDA_DX(KS) router_dx_bf16_kernel<KS><<<grid, 256, 0, s>>>((const uint16_t *)(b + L.rows), (const bf16_t *)wr, d->T, H, NE, L.Tp, (bf16_t *)dx)
                switch (L.NEp / 32) {
                    case 1: ZEDA_DX(1); break; case 2: ZEDA_DX(2); break; case 3: ZEDA_DX(3); break; case 4: ZEDA_DX(4); break;
                    case 5: ZEDA_DX(5); break; case 6: ZEDA_DX(6); break; case 7: ZEDA_DX(7); break; default: ZEDA_DX(8); break;
                }
#undef ZEDA_DX
            }
            if (hipGetLastError() != hipSuccess) return ZEDA_EHIP;
        }
        if (dw) {
            const int blocks = L.NE16 / 16, groups = ceil_div(blocks, 8), eb = ceil_div(blocks, groups);
            const dim3 grid(ceil_div(H, 256), L.splits, groups);
#define ZEDA_DW(EB)                                                                                                                        \
    if (f32) router_dw_kernel<EB, true><<<grid, 256, 0, s>>>(b + L.cols, x, mask, d->T, H, L.Tp, L.NEp, L.per, part, L.NE16);                  \
    else router_dw_kernel<EB, false><<<grid, 256, 0, s>>>(b + L.cols, x, mask, d->T, H, L.Tp, L.NEp, L.per, part, L.NE16)
            switch (eb) {
                case 1: ZEDA_DW(1); break; case 2: ZEDA_DW(2); break; case 3: ZEDA_DW(3); break; case 4: ZEDA_DW(4); break;
                case 5: ZEDA_DW(5); break; case 6: ZEDA_DW(6); break; case 7: ZEDA_DW(7); break; default: ZEDA_DW(8); break;
            }
#undef ZEDA_DW
            if (hipGetLastError() != hipSuccess) return ZEDA_EHIP;
        }
    }
    if (dw || dbias) {
        reduce_dw_kernel<<<ceil_div(NE * H / 4, 256) + 1, 256, 0, s>>>(part, L.splits, NE, L.NE16, H, dw, part_b, L.nblk, dbias);
        return last_launch_status();
    }
    return ZEDA_OK;
}

// ---------------------------------------------------------------------------------------------------------------------
// combine backward
// ---------------------------------------------------------------------------------------------------------------------
// out[t] = sum_j g_j y[row_j] (+ sum over free experts g_j x[t], copy experts):  d_g_j = <d_out[t], y[row_j]> (<d_out[t], x[t]>, or 0),
// d_y[row_j] = g_j d_out[t],  dx[t] = (sum over free experts g_j) d_out[t].  A workgroup a token, its waves take slots in turn.
// HBM-bound: reads d_out and a row of y a slot, writes a row of d_y a slot.
template <typename T, bool COPY>
__global__ __launch_bounds__(256) void combine_backward_kernel(const T *__restrict__ d_out, const T *__restrict__ y_slot, const int32_t *__restrict__ ids,
                                                               const float *__restrict__ gates, const int32_t *__restrict__ slot_to_row,
                                                               const T *__restrict__ x, float *__restrict__ d_gates, T *__restrict__ d_y,
                                                               T *__restrict__ dx, int H, int N, int NE, int K, int rows_cap)
{
    constexpr int VN = 16 / sizeof(T);
    typedef T vec_t __attribute__((ext_vector_type(VN)));
    const int t = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const T *d = d_out + (size_t)t * H;
    for (int j = wave; j < K; j += 4) {
        const size_t slot = (size_t)t * K + j;
        const int e = ids[slot], row = slot_to_row[slot];
        const float g = gates[slot];
        const bool real = e >= 0 && e < N && row >= 0 && row < rows_cap, free = COPY && e >= N && e < NE;
        float sum = 0.f;
        if (real || free) {
            const T *y = real ? y_slot + (size_t)row * H : x + (size_t)t * H;
            for (int v = lane * VN; v < H; v += 64 * VN) {
                const vec_t a = *reinterpret_cast<const vec_t *>(d + v), b = *reinterpret_cast<const vec_t *>(y + v);
                vec_t o;
#pragma unroll
                for (int i = 0; i < VN; ++i) {
                    sum = fmaf((float)a[i], (float)b[i], sum);
                    o[i] = (T)(g * (float)a[i]);
                }
                if (real && d_y) *reinterpret_cast<vec_t *>(d_y + (size_t)row * H + v) = o;
            }
            sum = wave_sum(sum);
        }
        if (lane == 0) d_gates[slot] = sum;
    }
    if (COPY && dx) {
        float gz = 0.f;
        for (int j = 0; j < K; ++j) {
            const int e = ids[(size_t)t * K + j];
            gz += e >= N && e < NE ? gates[(size_t)t * K + j] : 0.f;
        }
        for (int v = threadIdx.x * VN; v < H; v += 256 * VN) {
            const vec_t a = *reinterpret_cast<const vec_t *>(d + v);
            vec_t o;
#pragma unroll
            for (int i = 0; i < VN; ++i) o[i] = (T)(gz * (float)a[i]);
            *reinterpret_cast<vec_t *>(dx + (size_t)t * H + v) = o;
        }
    }
}

template <typename T>
static void launch_combine_backward_t(const zeda_layer_desc *d, const void *d_out, const void *y_slot, const int32_t *ids, const float *gates,
                                      const int32_t *slot_to_row, const void *x, float *d_gates, void *d_y, void *dx, hipStream_t s)
{
    const int NE = d->N + d->Z, S = d->T * d->K;
    if (d->free_expert == ZEDA_EXPERT_COPY)
        combine_backward_kernel<T, true><<<d->T, 256, 0, s>>>((const T *)d_out, (const T *)y_slot, ids, gates, slot_to_row, (const T *)x, d_gates,
                                                             (T *)d_y, (T *)dx, d->H, d->N, NE, d->K, S);
    else
        combine_backward_kernel<T, false><<<d->T, 256, 0, s>>>((const T *)d_out, (const T *)y_slot, ids, gates, slot_to_row, nullptr, d_gates,
                                                              (T *)d_y, nullptr, d->H, d->N, NE, d->K, S);
}

int launch_combine_backward(const zeda_layer_desc *d, const void *d_out, const void *y_slot, const int32_t *ids, const float *gates,
                            const int32_t *slot_to_row, const void *x, float *d_gates, void *d_y_slot, void *dx, hipStream_t s)
{
    if (d->dtype == ZEDA_BF16) launch_combine_backward_t<bf16_t>(d, d_out, y_slot, ids, gates, slot_to_row, x, d_gates, d_y_slot, dx, s);
    else launch_combine_backward_t<float>(d, d_out, y_slot, ids, gates, slot_to_row, x, d_gates, d_y_slot, dx, s);
    return last_launch_status();
}

}  // namespace zeda
