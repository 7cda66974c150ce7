// Training of the router (Section 2.2: the balance losses L_A, Eq. 4, and L_GA, Eq. 5-6) and of the routing weights of Eq. 1:
//   zeda_route_train      logits -> softmax, top-K, gates; per-expert counts, mean probabilities and the losses
//   zeda_route_backward   gradients of losses and gates -> logits -> x, w_router, router_bias
//   zeda_combine_backward gradient of the layer output -> gates, expert outputs
#include <limits.h>

#include <type_traits>

#include "zeda_place.h"
#include "zeda_select.h"

namespace zeda {

// ---------------------------------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------------------------------
// In bf16, where the router covers the hidden dimension in one kernel, that kernel does all of this (route_bf16_kernel<.., TRAIN>, 8192 tokens, 160
// experts, H = 2048: 24.6 us; apart 17.7 + 11.0).  Otherwise, with split sums or in fp32, where a workgroup of the router has too few tokens:
// 16 tokens a workgroup, four a wave: adds the logit tables and the bias, selects (select_rows, as the router), keeps the
// probabilities, and leaves for the batch sums: part_p[block][NE] = sum of the probabilities of the tokens that count,
// part_c[block][NE + 1] = their slots on every expert, and their number.
constexpr int kTrainTokens = 16;

template <int NB>
__global__ __launch_bounds__(256) void train_select_kernel(const float *__restrict__ tables, int slices, int Tpad,
                                                           const float *__restrict__ bias, const uint8_t *__restrict__ mask, int T, int N,
                                                           int NE, int K, int gate_norm, int32_t *__restrict__ ids, float *__restrict__ gates,
                                                           float *__restrict__ probs, float *__restrict__ part_p, int32_t *__restrict__ part_c,
                                                           int32_t *__restrict__ done)
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
        if (blockIdx.x == 0) *done = 0;
    }
}

// The batch sums: a workgroup adds up kFinalExperts experts' partial sums (in 64 bits and in a fixed order), and the last one to
// finish, found by a counter that the selecting kernel has cleared, does the losses.  One workgroup for everything took 34 us at 8192
// tokens and 160 experts (655 KB through one CU), these 20 workgroups 6.0.
constexpr int kFinalThreads = 1024, kFinalExperts = 8;
__global__ __launch_bounds__(kFinalThreads) void train_final_kernel(const float *__restrict__ part_p, const int32_t *__restrict__ part_c, int nblk,
                                                                    int N, int NE, int K, float alpha, float w, int32_t *counts, float *P,
                                                                    float *__restrict__ summary, int32_t *__restrict__ done)
{
    constexpr int PARTS = kFinalThreads / kFinalExperts, W = kFinalThreads / 64;
    __shared__ double s_p[W][kFinalExperts];
    __shared__ int s_c[W][kFinalExperts], s_n[W], s_last;
    const int tid = threadIdx.x, wave = tid >> 6, e = blockIdx.x * kFinalExperts + tid % kFinalExperts;
    double p = 0.;
    int c = 0, n = 0;
    if (e < NE) {
#pragma unroll 4
        for (int b = tid / kFinalExperts; b < nblk; b += PARTS) {
            p += (double)part_p[(size_t)b * NE + e];
            c += part_c[(size_t)b * (NE + 1) + e];
        }
    }
    for (int b = tid; b < nblk; b += kFinalThreads) n += part_c[(size_t)b * (NE + 1) + NE];
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        n += __shfl_xor(n, off);
        if (off >= kFinalExperts) {
            p += __shfl_xor(p, off);
            c += __shfl_xor(c, off);
        }
    }
    if ((tid & 63) < kFinalExperts) {
        s_p[wave][tid & 63] = p;
        s_c[wave][tid & 63] = c;
        if ((tid & 63) == 0) s_n[wave] = n;
    }
    __syncthreads();
    n = 0;
#pragma unroll
    for (int q = 0; q < W; ++q) n += s_n[q];
    n = max(1, n);  // nothing counts: f = P = 0
    if (tid < kFinalExperts && e < NE) {
        p = 0.;
        c = 0;
#pragma unroll
        for (int q = 0; q < W; ++q) { p += s_p[q][tid]; c += s_c[q][tid]; }
        __hip_atomic_store(counts + e, c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(P + e, (float)(p / n), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    // (the stores above and this are one wave's: one release covers them)
    if (tid == 0) s_last = __hip_atomic_fetch_add(done, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
    __syncthreads();
    if (!s_last) return;
    double v[5] = {0., 0., 0., 0., 0.};  // f_E, P_E, f_Z, P_Z, sum of f P
    if (tid < 64) {
        for (int i = tid; i < NE; i += 64) {
            const double f = (double)__hip_atomic_load(counts + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) / n;
            const double q = (double)__hip_atomic_load(P + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            v[4] += f * q;
            v[i < N ? 0 : 2] += f;
            v[i < N ? 1 : 3] += q;
        }
#pragma unroll
        for (int q = 0; q < 5; ++q)
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) v[q] += __shfl_xor(v[q], off);
        if (tid == 0) {
            const double Zw = (double)(NE - N) * w;
            for (int q = 0; q < 4; ++q) summary[q] = (float)v[q];
            summary[4] = (float)(v[2] / K);
            summary[5] = (float)((double)alpha * NE / K * v[4]);                                                               // Eq. 4
            summary[6] = (float)((double)alpha * (N + Zw) / K * (v[0] * v[1] / N + (NE > N ? v[2] * v[3] / Zw : 0.)));  // Eq. 5-6
        }
    }
}

// no token: everything is zero
__global__ __launch_bounds__(256) void train_nothing_kernel(int NE, int32_t *__restrict__ counts, float *__restrict__ P, float *__restrict__ summary)
{
    if (threadIdx.x < NE) { counts[threadIdx.x] = 0; P[threadIdx.x] = 0.f; }
    if (threadIdx.x < 7) summary[threadIdx.x] = 0.f;
}

struct TrainWs {
    size_t tables, part_p, part_c, done, total;
};
static TrainWs train_ws(const zeda_layer_desc *d)
{
    const size_t nblk = ceil_div(d->T, kTrainTokens), NE = d->N + d->Z;
    TrainWs w;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes ? bytes : 1, 256); return at; };
    w.tables = take(route_tables_most(d));
    w.part_p = take(nblk * NE * 4);
    w.part_c = take(nblk * (NE + 1) * 4);
    w.done = take(4);
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
    int32_t *part_c = (int32_t *)((char *)ws + L.part_c), *done = (int32_t *)((char *)ws + L.done);
    const int NE = d->N + d->Z, nblk = ceil_div(d->T, kTrainTokens);
    const TrainOut to = {mask, probs, part_p, part_c, done};
    if (d->T == 0) {
        train_nothing_kernel<<<1, 256, 0, s>>>(NE, counts, P, summary);
        return last_launch_status();
    }
    const bool fused = route_train_fused(d);
    if (!fused && t.bytes() > L.part_p - L.tables) return ZEDA_EWORKSPACE;  // (no plan is past route_tables_most)
    const int rows = fused ? ceil_div(d->T, t.tokens) : nblk;  // workgroups that select
    const int rc = fused ? launch_route_train_fused(d, x, wr, bias, ids, gates, to, s) : launch_route_tables(d, x, wr, tables, s);
    if (rc != ZEDA_OK) return rc;
    if (!fused) {
#define ZEDA_TRAIN(NB) train_select_kernel<NB><<<nblk, 256, 0, s>>>(tables, t.slices, t.Tpad, bias, mask, d->T, d->N, NE, d->K, d->gate_norm, ids, gates, probs, part_p, part_c, done)
        switch (t.E / 32) {
            case 1: ZEDA_TRAIN(1); break; case 2: ZEDA_TRAIN(2); break; case 3: ZEDA_TRAIN(3); break; case 4: ZEDA_TRAIN(4); break;
            case 5: ZEDA_TRAIN(5); break; case 6: ZEDA_TRAIN(6); break; case 7: ZEDA_TRAIN(7); break; default: ZEDA_TRAIN(8); break;
        }
#undef ZEDA_TRAIN
        if (hipGetLastError() != hipSuccess) return ZEDA_EHIP;
    }
    train_final_kernel<<<ceil_div(NE, kFinalExperts), kFinalThreads, 0, s>>>(part_p, part_c, rows, d->N, NE, d->K, alpha, w, counts, P, summary, done);
    return last_launch_status();
}

// ---------------------------------------------------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------------------------------------------------
// The gradient of the logits,
//   dl_e = p_e (a_e - sum_j p_j a_j) + the gates' part,   a_e = (dL_A alpha (N+Z)/K f_e + dL_GA alpha (N + Z w)/K f_E/N or f_Z/(Z w)) / n,
// does not change when a constant is added to a: the slopes' mean is taken off, in 64 bits, so that what they differ
// by is kept.  Gates: SOFTMAX adds dg_j to a at the selected experts; the normalised forms add g_j (dg_j - s), s = sum_l dg_l g_l,
// on the experts of the denominator and g_j dg_j on a selected expert outside it.
constexpr int kBackTokens = 32, kBackThreads = 1024;

// bf16 parts by truncation: v = v0 + v1 + v2 exactly (24 bits)
__device__ __forceinline__ uint16_t top_bits(float v) { return (uint16_t)(__float_as_uint(v) >> 16); }
__device__ __forceinline__ float top_part(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }

struct LogitGrad {
    const float *probs, *gates, *d_loss, *d_gates;
    const int32_t *ids, *counts;
    const uint8_t *mask;
    int T, N, NE, K, gate_norm;
    float alpha, w;
    // dl twice, as tiles in the order in which the products fetch them: rows [part][t / 16][e / 32][t % 16][e % 32] and
    // cols [part][t / 32][e][t % 32]
    void *rows, *cols;
    float *part_b;        // [blocks][NE]: sums over the block's tokens
    uint32_t *on;         // [blocks]
    int Tp, NEp;
};

// A wave takes two tokens, lane l the experts l, l + 64, ...  F32: both copies in fp32; else the rows as two bf16 parts (their
// product is rounded to bf16), the columns as three (theirs stays fp32: nothing of dl is lost).  8192 tokens, 160 experts: 11.9 us (reads
// 5 MB, writes 13), bound by the latency of its steps, one workgroup a CU.  on[block]: which of the block's
// tokens count, a bit each.
template <bool F32>
__global__ __launch_bounds__(kBackThreads) void logit_grad_kernel(LogitGrad a)
{
    constexpr int W = kBackThreads / 64, PER = kBackTokens / W;
    extern __shared__ float s_dl[];  // [kBackTokens][LD]
    __shared__ float s_a[kMaxExperts];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, t0 = blockIdx.x * kBackTokens, NE = a.NE, N = a.N, LD = a.NEp + 1;
    bool on[PER];
    float p[PER][4], g[PER], dg[PER];
    int id[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int t = t0 + wave * PER + k;
        const size_t at = min(t, a.T - 1);
        on[k] = t < a.T && (!a.mask || a.mask[at]);
        id[k] = -1;
        g[k] = dg[k] = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) p[k][q] = lane + 64 * q < NE ? a.probs[at * NE + lane + 64 * q] : 0.f;
        if (a.d_gates && lane < a.K) {
            id[k] = a.ids[at * a.K + lane];
            g[k] = a.gates[at * a.K + lane];
            dg[k] = a.d_gates[at * a.K + lane];
            if ((unsigned)id[k] >= (unsigned)NE) id[k] = -1, g[k] = dg[k] = 0.f;
        }
    }
    if (wave == 0) {  // the slopes: lane l experts l, l + 64, ...
        int c[4], cE = 0, cZ = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int e = lane + 64 * q;
            c[q] = e < NE ? a.counts[e] : 0;
            (e < N ? cE : cZ) += c[q];
        }
        cE = __builtin_amdgcn_readlane(wave_scan(cE), 63);
        cZ = __builtin_amdgcn_readlane(wave_scan(cZ), 63);
        const double n = fmax(1., (double)(cE + cZ) / a.K), Zw = (double)(NE - N) * a.w, unit = (double)a.alpha / a.K / (n * n);
        const double kA = a.d_loss ? unit * a.d_loss[0] * NE : 0., kG = a.d_loss ? unit * a.d_loss[1] * (N + Zw) : 0.;
        // without their mean: c_e - sum c / NE, and the groups' slopes share their difference
        const double apart = NE > N ? kG * (cE * Zw - (double)cZ * N) / (N * Zw) / NE : 0.;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            s_a[lane + 64 * q] = (float)(kA / NE * ((double)c[q] * NE - (cE + cZ)) + (lane + 64 * q < N ? apart * (NE - N) : -apart * N));
    }
    __syncthreads();
    // (a wave's tokens side by side: each step is a broadcast from one lane and four comparisons)
    float u[PER][4], g_of[PER][4] = {}, v_of[PER][4] = {}, sum[PER] = {};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float slope = lane + 64 * q < NE ? s_a[lane + 64 * q] : 0.f;
#pragma unroll
        for (int k = 0; k < PER; ++k) u[k][q] = slope;
    }
    if (a.d_gates) {
        const bool softmax = a.gate_norm == ZEDA_GATE_SOFTMAX;
        const int within = a.gate_norm == ZEDA_GATE_TOPK_NORM ? NE : N;
        for (int j = 0; j < a.K; ++j) {
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const int ej = __builtin_amdgcn_readlane(id[k], j);
                const float gj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(g[k]), j));
                const float dj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(dg[k]), j));
                const float direct = softmax ? dj : 0.f, shared = softmax ? 0.f : gj, in = ej < within ? shared : 0.f;
                sum[k] = fmaf(gj, dj, sum[k]);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const bool mine = ej == lane + 64 * q;
                    u[k][q] += mine ? direct : 0.f;
                    v_of[k][q] += mine ? shared * dj : 0.f;
                    g_of[k][q] += mine ? in : 0.f;
                }
            }
        }
    }
    float pa[PER] = {};
#pragma unroll
    for (int k = 0; k < PER; ++k) {
#pragma unroll
        for (int q = 0; q < 4; ++q) pa[k] = fmaf(p[k][q], u[k][q], pa[k]);
        pa[k] = wave_sum(pa[k]);
    }
#pragma unroll
    for (int k = 0; k < PER; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float dl = on[k] && lane + 64 * q < NE ? p[k][q] * (u[k][q] - pa[k]) + (v_of[k][q] - (g_of[k][q] != 0.f ? sum[k] * g_of[k][q] : 0.f)) : 0.f;
            if (lane + 64 * q < a.NEp) s_dl[(wave * PER + k) * LD + lane + 64 * q] = dl;
        }
    __syncthreads();
    if (tid < NE) {
        double b = 0.;
#pragma unroll 8
        for (int k = 0; k < kBackTokens; ++k) b += (double)s_dl[k * LD + tid];
        a.part_b[(size_t)blockIdx.x * NE + tid] = (float)b;
    }
    if (wave == W - 1) {
        const int t = t0 + lane;
        const unsigned long long bits = __ballot(lane < kBackTokens && t < a.T && (!a.mask || a.mask[t]));
        if (lane == 0) a.on[blockIdx.x] = (uint32_t)bits;
    }
    const int Tp = a.Tp, NEp = a.NEp;
    typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
    const size_t plane = (size_t)Tp * NEp;
    auto store = [&](void *to, size_t at, const float (&v)[4], int parts) {
        if (F32) {
            *reinterpret_cast<f32x4 *>((float *)to + at) = f32x4{v[0], v[1], v[2], v[3]};
            return;
        }
        float r[4] = {v[0], v[1], v[2], v[3]};
        for (int q = 0; q < parts; ++q) {
            u16x4 o;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[i] = top_bits(r[i]);
                r[i] -= top_part(r[i]);
            }
            *reinterpret_cast<u16x4 *>((uint16_t *)to + q * plane + at) = o;
        }
    };
    for (int i = tid; i < kBackTokens * NEp / 4; i += kBackThreads) {
        const int k = i / (NEp / 4), e = (i - k * (NEp / 4)) * 4;
        const float v[4] = {s_dl[k * LD + e], s_dl[k * LD + e + 1], s_dl[k * LD + e + 2], s_dl[k * LD + e + 3]};
        store(a.rows, ((size_t)((t0 + k) >> 4) * (NEp >> 5) + (e >> 5)) * 512 + (k & 15) * 32 + (e & 31), v, 2);
    }
    for (int i = tid; i < kBackTokens * NEp / 4; i += kBackThreads) {
        const int e = i / (kBackTokens / 4), k = (i - e * (kBackTokens / 4)) * 4;
        const float v[4] = {s_dl[k * LD + e], s_dl[(k + 1) * LD + e], s_dl[(k + 2) * LD + e], s_dl[(k + 3) * LD + e]};
        store(a.cols, ((size_t)(t0 >> 5) * NEp + e) * 32 + k, v, 3);
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
// Lane (l16, kq) of a 16x16x32 product: columns 4 l16 .. + 3 as four operands, experts 8 kq .. + 7 of the step.  8192 tokens, 160 experts,
// H = 2048: 18-19 us, 33 MB written; every CU pulls w_router's and dl's pieces out of L2 (84 MB in all).
template <int KS>  // steps of 32 experts
__global__ __launch_bounds__(256) void router_dx_bf16_kernel(const uint16_t *__restrict__ dl, const bf16_t *__restrict__ wr, int T, int H, int NE,
                                                             int Tp, int per, bf16_t *__restrict__ dx)
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
    const int ta = blockIdx.x * per, tb = min(T, ta + per);
    const size_t plane = (size_t)Tp * KS * 32;
    // dl of the next two token blocks is on its way while one is multiplied
    bf16x8 df[2][2][KS];
    auto fetch = [&](bf16x8 (&to)[2][KS], int t0) {
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int k = 0; k < KS; ++k) to[q][k] = *reinterpret_cast<const bf16x8 *>(dl + q * plane + ((size_t)(t0 >> 4) * KS + k) * 512 + l16 * 32 + 8 * kq);
    };
    auto block = [&](bf16x8 (&d)[2][KS], int t0) {
        f32x4 acc[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 1; q >= 0; --q)
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(d[q][k], wf[k][c], acc[c], 0, 0, 0);
        if (t0 + 32 < tb) fetch(d, t0 + 32);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + 4 * kq + i;
            bf16x4 v;
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = (bf16_t)acc[c][i];
            if (t < T) *reinterpret_cast<bf16x4 *>(dx + (size_t)t * H + h0 + 4 * l16) = v;
        }
    };
    fetch(df[0], ta);
    if (ta + 16 < tb) fetch(df[1], ta + 16);
    for (int t0 = ta; t0 < tb; t0 += 32) {
        block(df[0], t0);
        if (t0 + 16 < tb) block(df[1], t0 + 16);
    }
}

// The same in fp32 on the fp32 matrix instruction: a wave has 64 tokens and 64 columns, 16 experts a step (lane (l16, kq): experts
// 4 kq .. + 3, one to each of four products).  Columns past H (H % 4 == 0) are left out.
__global__ __launch_bounds__(256) void router_dx_f32_kernel(const float *__restrict__ dl, const float *__restrict__ wr, int T, int H, int NE, int NEp,
                                                            float *__restrict__ dx)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, kq = lane >> 4;
    const int h0 = (blockIdx.y * 4 + wave) * 64, t0 = blockIdx.x * 64, h = h0 + 4 * l16;
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
            df[i] = *reinterpret_cast<const f32x4 *>(dl + ((size_t)(t0 / 16 + i) * (NEp >> 5) + (e0 >> 5)) * 512 + l16 * 32 + (e0 & 31) + 4 * kq);
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

// dw_router[NE, H] = dl^T x, split over the tokens: part[split][NE16][H], added up by reduce_dw_kernel.  A workgroup has 128 columns,
// EB blocks of 16 experts and a range of tokens; of its eight waves four share 64 columns and take 32 tokens (fp32: 16) in turn,
// and their sums meet in LDS.  Rows of tokens that do not count are taken as zero whatever they hold.  8192 tokens, 160 experts, H = 2048: 25 us
// + 5 for the splits' sums (16 GFLOP as three products, 12 us at the rate of a large bf16 product; the rest is the latency of the
// loads, one step ahead).
constexpr int kDwThreads = 512, kDwTurns = 4, kDwMaxBlocks = 6;
template <int EB, bool F32>
__global__ __launch_bounds__(kDwThreads) void router_dw_kernel(const void *__restrict__ dlT, const void *__restrict__ xv, const uint32_t *__restrict__ on,
                                                               int H, int Tp, int NEp, int per, float *__restrict__ part, int NE16)
{
    __shared__ f32x4 s_sum[2][kDwTurns][16][32];  // [buffer][turn][expert][column / 4]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, kq = lane >> 4;
    const int turn = wave >> 1, h0 = blockIdx.x * 128, h = h0 + (wave & 1) * 64 + 4 * l16, e0 = blockIdx.z * EB * 16, ta = blockIdx.y * per, tb = min(ta + per, Tp);
    f32x4 acc[EB][4];
#pragma unroll
    for (int b = 0; b < EB; ++b)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[b][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (F32) {
        const float *x = (const float *)xv, *dl = (const float *)dlT;
        for (int t = ta + 16 * turn; t < tb; t += 16 * kDwTurns) {
            const uint32_t bits = on[t >> 5] >> (t & 31);
            f32x4 xf[4], df[EB];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                xf[i] = h < H && (bits >> (4 * kq + i) & 1) ? *reinterpret_cast<const f32x4 *>(x + (size_t)(t + 4 * kq + i) * H + h) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = 0; b < EB; ++b) df[b] = *reinterpret_cast<const f32x4 *>(dl + ((size_t)(t >> 5) * NEp + min(e0 + 16 * b + l16, NEp - 1)) * 32 + (t & 31) + 4 * kq);
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
        const size_t plane = (size_t)NEp * Tp;
        uint2 r[8];
        bf16x8 df[3][EB];
        auto load_x = [&](int t) {
            const uint32_t bits = on[t >> 5] >> (8 * kq);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                r[i] = bits >> i & 1 ? *reinterpret_cast<const uint2 *>(x + (size_t)(t + 8 * kq + i) * H + h) : make_uint2(0, 0);
        };
        auto load_dl = [&](int q, int t) {
#pragma unroll
            for (int b = 0; b < EB; ++b)
                df[q][b] = *reinterpret_cast<const bf16x8 *>(dl + q * plane + ((size_t)(t >> 5) * NEp + min(e0 + 16 * b + l16, NEp - 1)) * 32 + 8 * kq);
        };
        int t = ta + 32 * turn;
        if (t < tb) {
            load_x(t);
#pragma unroll
            for (int q = 2; q >= 0; --q) load_dl(q, t);
        }
        for (; t < tb; t += 32 * kDwTurns) {  // a part's registers are filled again as soon as its products are issued
            const bool more = t + 32 * kDwTurns < tb;
            bf16x8 xf[4];
            turn8x4(r, xf);
            if (more) load_x(t + 32 * kDwTurns);
#pragma unroll
            for (int q = 2; q >= 0; --q) {
#pragma unroll
                for (int b = 0; b < EB; ++b)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[b][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(df[q][b], xf[c], acc[b][c], 0, 0, 0);
                if (more) load_dl(q, t + 32 * kDwTurns);
            }
        }
    }
#pragma unroll
    for (int b = 0; b < EB; ++b) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            s_sum[b & 1][turn][4 * kq + i][(wave & 1) * 16 + l16] = f32x4{acc[b][0][i], acc[b][1][i], acc[b][2][i], acc[b][3][i]};
        __syncthreads();
        const int row = threadIdx.x >> 5, q = threadIdx.x & 31, e = e0 + 16 * b + row;
        if (e < NE16 && h0 + 4 * q < H)
            *reinterpret_cast<f32x4 *>(part + ((size_t)blockIdx.y * NE16 + e) * H + h0 + 4 * q) =
                (s_sum[b & 1][0][row][q] + s_sum[b & 1][1][row][q]) + (s_sum[b & 1][2][row][q] + s_sum[b & 1][3][row][q]);
    }
}

// dw = the splits' sums; dbias = the token blocks' sums, eight experts to each of the last workgroups.  In a fixed order.
constexpr int kBiasExperts = 8;
__global__ __launch_bounds__(256) void reduce_dw_kernel(const float *__restrict__ part, int splits, int NE, int NE16, int H, int nw, float *__restrict__ dw,
                                                        const float *__restrict__ part_b, int nblk, float *__restrict__ dbias)
{
    if ((int)blockIdx.x >= nw) {
        __shared__ double s_b[256];
        const int e = (blockIdx.x - nw) * kBiasExperts + threadIdx.x % kBiasExperts;
        double b = 0.;
        if (e < NE) {
#pragma unroll 4
            for (int k = threadIdx.x / kBiasExperts; k < nblk; k += 256 / kBiasExperts) b += (double)part_b[(size_t)k * NE + e];
        }
        s_b[threadIdx.x] = b;
        __syncthreads();
        if (threadIdx.x < kBiasExperts && e < NE) {
            for (int k = 1; k < 256 / kBiasExperts; ++k) b += s_b[k * kBiasExperts + threadIdx.x];
            dbias[e] = (float)b;
        }
        return;
    }
    const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= (size_t)NE * H) return;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int q = 0; q < splits; ++q) v += *reinterpret_cast<const f32x4 *>(part + (size_t)q * NE16 * H + i);
    *reinterpret_cast<f32x4 *>(dw + i) = v;
}

struct BackWs {
    size_t rows, cols, part_b, on, part, total;
    int Tp, NEp, NE16, splits, per, nblk, groups, eb;
};
static BackWs back_ws(const zeda_layer_desc *d)
{
    const int NE = d->N + d->Z;
    const size_t es = d->dtype == ZEDA_BF16 ? 2 : 4;
    BackWs w;
    w.Tp = ceil_div(d->T, 64) * 64;
    w.nblk = w.Tp / kBackTokens;
    w.NEp = ceil_div(NE, 32) * 32;
    w.NE16 = ceil_div(NE, 16) * 16;
    w.groups = ceil_div(w.NE16 / 16, kDwMaxBlocks);
    w.eb = ceil_div(w.NE16 / 16, w.groups);
    // token ranges, multiples of 128, so that some 256 workgroups share the product
    int splits = ceil_div(256, ceil_div(d->H, 128) * w.groups);
    const int most = ceil_div(w.Tp, 128);
    if (splits > most) splits = most;
    w.per = splits ? ceil_div(most, splits) * 128 : 128;
    w.splits = ceil_div(w.Tp, w.per);  // (at most `splits`, which does not fall as T grows: the scratch is sized by that)
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes ? bytes : 1, 256); return at; };
    const size_t n = (size_t)w.Tp * w.NEp * es;
    w.rows = take(n * (es == 2 ? 2 : 1));
    w.cols = take(n * (es == 2 ? 3 : 1));
    w.part_b = take((size_t)w.nblk * NE * 4);
    w.on = take((size_t)w.nblk * 4);
    w.part = take((size_t)splits * w.NE16 * d->H * 4);
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
    logit_grad_kernel<F32><<<nblk, kBackThreads, kBackTokens * (g.NEp + 1) * 4, s>>>(g);
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
    uint32_t *on = (uint32_t *)(b + L.on);
    if (d->T > 0) {
        const LogitGrad g = {probs, gates, d_loss, d_gates, ids, counts, mask, d->T, d->N, NE, d->K, d->gate_norm, alpha, w,
                             b + L.rows, b + L.cols, part_b, on, L.Tp, L.NEp};
        int rc = f32 ? launch_logit_grad<true>(g, L.nblk, s) : launch_logit_grad<false>(g, L.nblk, s);
        if (rc != ZEDA_OK) return rc;
        if (dx) {
            if (f32) {
                router_dx_f32_kernel<<<dim3(L.Tp / 64, ceil_div(H, 256)), 256, 0, s>>>((const float *)(b + L.rows), (const float *)wr, d->T, H, NE, L.NEp,
                                                                                   (float *)dx);
            } else {
                // Tokens of a workgroup: as many workgroups as run at once (two to a CU), from 32 up (each fetches its part of w_router), and no more
                // than 128 to a workgroup, which leaves the last round fuller.  H = 2048, us, always 128 / so: 200 tokens 10.8 / 4.4, 997 8.9 / 4.4,
                // 2048 11.2 / 8.6, 4096 12.8 / 12.6, 8192 18.1 / 18.2 (twice as many workgroups there: 21.0)
                const int even = ceil_div((int)((int64_t)d->T * ceil_div(H, 256) / 512), 32) * 32, per = even < 32 ? 32 : even > 128 ? 128 : even;
                const dim3 grid(ceil_div(d->T, per), ceil_div(H, 256));
#define ZEDA_DX(KS) router_dx_bf16_kernel<KS><<<grid, 256, 0, s>>>((const uint16_t *)(b + L.rows), (const bf16_t *)wr, d->T, H, NE, L.Tp, per, (bf16_t *)dx)
                switch (L.NEp / 32) {
                    case 1: ZEDA_DX(1); break; case 2: ZEDA_DX(2); break; case 3: ZEDA_DX(3); break; case 4: ZEDA_DX(4); break;
                    case 5: ZEDA_DX(5); break; case 6: ZEDA_DX(6); break; case 7: ZEDA_DX(7); break; default: ZEDA_DX(8); break;
                }
#undef ZEDA_DX
            }
            if (hipGetLastError() != hipSuccess) return ZEDA_EHIP;
        }
        if (dw) {
            const dim3 grid(ceil_div(H, 128), L.splits, L.groups);
#define ZEDA_DW(EB)                                                                                                                        \
    if (f32) router_dw_kernel<EB, true><<<grid, kDwThreads, 0, s>>>(b + L.cols, x, on, H, L.Tp, L.NEp, L.per, part, L.NE16);                  \
    else router_dw_kernel<EB, false><<<grid, kDwThreads, 0, s>>>(b + L.cols, x, on, H, L.Tp, L.NEp, L.per, part, L.NE16)
            switch (L.eb) {
                case 1: ZEDA_DW(1); break; case 2: ZEDA_DW(2); break; case 3: ZEDA_DW(3); break;
                case 4: ZEDA_DW(4); break; case 5: ZEDA_DW(5); break; default: ZEDA_DW(6); break;
            }
#undef ZEDA_DW
            if (hipGetLastError() != hipSuccess) return ZEDA_EHIP;
        }
    }
    if (dw || dbias) {
        const int nw = dw ? ceil_div(NE * H / 4, 256) : 0, nb = dbias ? ceil_div(NE, kBiasExperts) : 0;
        reduce_dw_kernel<<<nw + nb, 256, 0, s>>>(part, L.splits, NE, L.NE16, H, nw, dw, part_b, L.nblk, dbias);
        return last_launch_status();
    }
    return ZEDA_OK;
}

// ---------------------------------------------------------------------------------------------------------------------
// combine backward
// ---------------------------------------------------------------------------------------------------------------------
// out[t] = sum_j g_j y[row_j] (+ sum over free experts g_j x[t], copy experts):  d_g_j = <d_out[t], y[row_j]> (<d_out[t], x[t]>, or 0),
// d_y[row_j] = g_j d_out[t],  dx[t] = (sum over free experts g_j) d_out[t].  A workgroup a token, its waves take slots in turn.
// HBM-bound: reads d_out and a row of y a slot, writes a row of d_y a slot.  4096 tokens, K = 8, H = 2048: 151 MB in 37-39 us (3.9-4.1 TB/s).
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
