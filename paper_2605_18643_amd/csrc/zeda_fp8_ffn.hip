// Grouped SwiGLU expert FFN over the real slots with 8-bit operands (Section 2.1; Appendix D, Eq. 10):
//   xq = Q(x), h = silu(G xq) .* (U xq), y = D Q(h),
// Q = rounding to e4m3 under a power-of-two scale for every 128 columns, G, U, D e4m3 under one for every 128 x 128 block.
//
// Tiles of up to 160 token rows x 256 weight rows.  Every weight byte is used by one wave only, so weights go straight into the registers
// of the matrix instruction (their layout is its operand's, 2 KiB a fetch), half a chunk of 128 columns at a time into the registers that
// the products before have freed; token rows, which all four waves use, go through a ring of three chunks in LDS.  The scales ride
// along as operands of the instruction (bytes of powers of two).  Two workgroups to a CU: one's prologue and epilogue run under the
// other's products.
// What bounds it: with up to 128 rows an expert the weights from HBM (997 tokens, N=64, I=1536, H=2048: gate/up 403 MB in 77 us = 5.2 TB/s, the
// rate of a large copy).  4096 tokens of N=128, I=768 have 128 rows an expert on average, so every second expert of its tiles of 128 needs a
// second one: gate/up 103 us, down 64 (with tiles of 160, which hardly need one, the same, in 1.5 rounds of workgroups instead of 2.2).  16381 skewed
// tokens with 51318 slots on normal experts: 164-207 and 123-146 us, with 72983 212-288 and 165-208, the matrix pipes busy 53 and 33 % of the
// cycles (down writes 16 bits a product of 768 terms).
// What the compiler must not see as flat: token rows fetched by global loads into LDS made it wait for everything in flight before the first
// product of every chunk (4096 tokens, whole layer, 205 us against 202; 8192 tokens 283 against 270; 16381 470 against 444).
// Tried and slower: one workgroup of eight waves with 192-row tiles and two chunks ahead (16381 tokens: gate/up 258 -> 305 us), one of four
// waves with twice the accumulators (4096 tokens, whole layer: 219 -> 320 us).
//
// Sums: the matrix instruction adds its products with the bits down to 2^-13 of the largest of a group: 1.4e-5 of a sum's root mean square.
// That moves one activation in 5000 to the next 8-bit value and puts the layer's result 2.0e-3 off where fp32 sums and the rounding of the
// result give 1.7e-3.  (The kernels of few rows, where it would show more, pay for exact products: zeda_fp8_few.hip.  Here that would
// double the matrix instructions.)
#include <type_traits>
#include <utility>

#include "zeda_fp8.h"
#include "zeda_lds.h"
#include "zeda_place.h"

namespace zeda {

constexpr int kF8Tok = 160;      // token rows of a tile at most
constexpr int kF8Threads = 256;  // four waves, each two units (64 rows) of the weights against all token rows of the tile

// One wave: {expert, first row, rows} of token tile `tile` of the expert-sorted rows, and the number of tiles of all experts.
struct F8Tiles {
    int off[5], nt[4], excl, total, tok;
    __device__ __forceinline__ void count(const int32_t *__restrict__ offsets, int N, int rows)
    {
        const int lane = threadIdx.x & 63;
        int local = 0;
        tok = rows;
#pragma unroll
        for (int q = 0; q < 5; ++q) off[q] = offsets[min(4 * lane + q, N)];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            nt[q] = (off[q + 1] - off[q] + tok - 1) / tok;
            local += nt[q];
        }
        const int incl = wave_scan(local);
        excl = incl - local;
        total = __builtin_amdgcn_readlane(incl, 63);
    }
    __device__ __forceinline__ int3 locate(int tile) const
    {
        int e = 0, row0 = 0, rows = 0, at = excl;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (tile >= at && tile < at + nt[q]) {
                e = 4 * (threadIdx.x & 63) + q;
                row0 = off[q] + (tile - at) * tok;
                rows = min(tok, off[q + 1] - row0);
            }
            at += nt[q];
        }
        const int src = __ffsll((long long)__ballot(rows > 0)) - 1;
        return make_int3(__builtin_amdgcn_readlane(e, src), __builtin_amdgcn_readlane(row0, src), __builtin_amdgcn_readlane(rows, src));
    }
};

struct F8Args {
    const uint8_t *src, *src_s;  // operand rows of ld bytes and their scales
    const uint8_t *w, *ws;       // packed weights and scales
    const int32_t *offsets, *sorted_slot;
    uint8_t *act, *act_s;  // gate/up's result
    void *y;               // down's
    int16_t *y_exp;
    int T, N, K, H, Ip, tok, nft;  // token rows of a tile, feature tiles
    int log_terms;         // down: 2^log_terms >= Ip * 448 * 448
};

// What a launch leaves: activations, expert outputs in bf16, or (whole layer) expert outputs for the combine in the same 16 bits
// but with 11 significant ones: fp16 under a power of two for every row and 128 columns that bounds the sum whatever its terms,
// 2^k with k = the largest exponent of the blocks' scale products + log2(terms * 448^2) - 15.  bf16's 8 bits would cost the layer's
// output a second rounding of the size of its own (2.6e-3 off in all, against 1.7e-3 for the rounding of the result alone).
enum { kF8GateUp = 0, kF8Down = 1, kF8DownScaled = 2 };

constexpr int kF8Slot = kF8Tok * kFp8Block, kF8Ring = 3 * kF8Slot;

// Gate/up: 128 activations (256 weight rows, eight units) a workgroup; down: 256 output columns.
template <typename F, int... S>
__device__ __forceinline__ void for_steps(F &f, std::integer_sequence<int, S...>) { (f(std::integral_constant<int, S>{}), ...); }

template <int KIND, bool ONE, bool BIG>  // ONE: a single chunk; BIG: token rows past 4 GiB
struct F8Kernel {
    static constexpr bool GATEUP = KIND == kF8GateUp;
    const F8Args &a;
    uint8_t *ring, *tab;  // LDS: three chunks of token rows; the rows' scales and the weights'
    int e, row0, rows, ft;

    __device__ __forceinline__ int src_row(int r) const { return GATEUP ? min(max(a.sorted_slot[r] / a.K, 0), a.T - 1) : r; }  // (a bad index must not fault)

    template <int NB>
    __device__ __forceinline__ void run() const
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
        const int ld = GATEUP ? a.H : a.Ip, nk = ld / kFp8Block, pitch = fp8_pitch(ld);
        // the wave's two units: along the packed row blocks, clamped where the last feature tile is narrower
        const int rbs = GATEUP ? a.Ip / 16 : a.H / 32, rb = ft * 8 + wave * 2;
        const uint8_t *wp[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) wp[u] = a.w + ((size_t)e * rbs + min(rb + u, rbs - 1)) * (2 * nk) * kFp8Unit;
        u32x4 w[2][4];
        auto load_w = [&](int c, int m) {  // half m of chunk c's columns
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int q = 2 * m; q < 2 * m + 2; ++q) w[u][q] = *reinterpret_cast<const u32x4 *>(wp[u] + (size_t)c * (2 * kFp8Unit) + q * 1024 + lane * 16);
        };
        load_w(0, 0);
        load_w(0, 1);  // (what an item starts from is asked for before anything waits: weights, token rows, scales)
        // This thread's piece of the token rows of every 32-row block: row tid / 8, and the ring's position tid % 8 of that row, where
        // the row's 16-byte pieces stand permuted by the row: 16 lanes that read one piece of 16 rows touch all banks once.
        // They are fetched by buffer loads with 32-bit offsets (gate/up: into all tokens; down: into the tile's rows): a global load into LDS
        // counts as flat with the compiler, which then waits for everything in flight wherever it needs a weight.
        std::conditional_t<BIG, size_t, uint32_t> tp[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int r = min(32 * b + (tid >> 3), rows - 1);
            tp[b] = (std::conditional_t<BIG, size_t, uint32_t>)(GATEUP ? src_row(row0 + r) : r) * ld + (((tid & 7) ^ ((tid >> 4) & 7)) << 4);
        }
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(GATEUP ? a.src : a.src + (size_t)row0 * ld), 0, 0xffffffff, 0x00027000);
        uint8_t *wtab = tab + kF8Tok * pitch;
        const uint32_t my_ws = lds_addr(wtab + (GATEUP ? l32 >> 4 : wave >> 1) * pitch), my_ts = lds_addr(tab + l32 * pitch);

        f32x16 acc[2][NB];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[u][b][i] = 0.f;

        // Per chunk of 128 columns a wave fetches a quarter of the token rows into the ring, two chunks ahead, and its weights into registers
        // half a chunk at a time, as soon as the half before them in the same registers is used.
        auto load_t = [&](int c, int slot) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const auto to = (__attribute__((address_space(3))) void *)(ring + slot * kF8Slot + b * 4096 + wave * 1024);
                if constexpr (BIG) __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(a.src + tp[b] + (size_t)c * kFp8Block), to, 16, 0, 0);
                else __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, to, 16, tp[b], c * kFp8Block, 0, 0);
            }
        };
        const uint32_t ring0 = lds_addr(ring), sw = (l32 >> 1) & 7;
        uint32_t ts[NB], wsc = 0;  // four chunks' scales
        auto multiply = [&](int c, int slot, bool more) {
            if ((c & 3) == 0) {
                wsc = lds_read_b32(my_ws + c);
#pragma unroll
                for (int b = 0; b < NB; ++b) ts[b] = lds_read_b32(my_ts + 32 * b * pitch + c);
                lds_wait(wsc);
#pragma unroll
                for (int b = 0; b < NB; ++b) lds_wait(ts[b]);
            }
            const int sa = (int)(wsc >> (8 * (c & 3)));
            uint32_t at = ring0 + slot * kF8Slot + l32 * kFp8Block;
            asm volatile("" : "+v"(at));  // (four addresses a chunk; those of all chunks would stay in registers)
            const uint32_t at4[4] = {at + ((half ^ sw) << 4), at + (((2 + half) ^ sw) << 4), at + (((4 + half) ^ sw) << 4), at + (((6 + half) ^ sw) << 4)};
            u32x4 t[2][2];
            // Step s: half s / NB of the chunk's columns of token block s % NB.  (The other way round, the two halves' products into the
            // same accumulators would follow each other.)
            auto fetch = [&](auto step) {
                constexpr int s = decltype(step)::value, b = s % NB, m = s / NB;
                t[s & 1][0] = lds_read_b128_at<b * 4096>(at4[2 * m]);
                t[s & 1][1] = lds_read_b128_at<b * 4096>(at4[2 * m + 1]);
            };
            fetch(std::integral_constant<int, 0>{});
            auto step = [&](auto sc) {
                constexpr int s = decltype(sc)::value, b = s % NB, m = s / NB;
                if constexpr (s + 1 < 2 * NB) {
                    fetch(std::integral_constant<int, s + 1>{});
                    lds_wait_but<2>(t[s & 1][0], t[s & 1][1]);
                } else {
                    lds_wait(t[s & 1][0], t[s & 1][1]);
                }
                const i32x8 tb = __builtin_bit_cast(i32x8, __builtin_shufflevector(t[s & 1][0], t[s & 1][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const i32x8 wu = __builtin_bit_cast(i32x8, __builtin_shufflevector(w[u][2 * m], w[u][2 * m + 1], 0, 1, 2, 3, 4, 5, 6, 7));
                    acc[u][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wu, tb, acc[u][b], 0, 0, 0, sa, 0, (int)(ts[b] >> (8 * (c & 3))));
                }
                asm volatile("" : "+v"(acc[0][b]), "+v"(acc[1][b]));  // (here and not after later reads, whose fragments would all stay in registers)
                if (b == NB - 1 && more) load_w(c + 1, m);
            };
            for_steps(step, std::make_integer_sequence<int, 2 * NB>{});
        };
        int slot = 0;
        // LEFT: chunks that follow this one, two at most; nothing is asked for past the last one
        auto chunk = [&](int c, auto left) {
            constexpr int LEFT = decltype(left)::value;
            // chunk c's token rows (asked for behind them: chunk c's weights and chunk c + 1's rows; of the first chunk see below)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((LEFT >= 1 ? NB : 0) + 8) : "memory");
            asm volatile("s_barrier" ::: "memory");  // everyone's; and everyone is done with chunk c - 1
            if constexpr (LEFT >= 2) load_t(c + 2, slot == 0 ? 2 : slot - 1);
            multiply(c, slot, LEFT >= 1);
            slot = slot == 2 ? 0 : slot + 1;
        };
        constexpr std::integral_constant<int, 0> none{};
        constexpr std::integral_constant<int, 1> one{};
        constexpr std::integral_constant<int, 2> two{};
        load_t(0, 0);
        if constexpr (!ONE) load_t(1, 1);
        // scales: one LDS row per token row, then one (two: gate, up) for the weights
        for (int i = tid; i < NB * 32 * (pitch / 4); i += kF8Threads) {
            const int r = i / (pitch / 4), c = i - r * (pitch / 4), rr = row0 + min(r, rows - 1);
            reinterpret_cast<uint32_t *>(tab)[i] =
                reinterpret_cast<const uint32_t *>(a.src_s + (size_t)src_row(rr) * pitch)[c];
        }
        {
            // (down: a workgroup's 256 rows are two blocks of 128)
            const size_t r0 = GATEUP ? ((size_t)e * (a.Ip / kFp8Block) + ft) * 2 : (size_t)e * (a.H / kFp8Block) + ft * 2;
            const int last = GATEUP ? 1 : min(1, a.H / kFp8Block - 1 - ft * 2);
            for (int i = tid; i < 2 * (pitch / 4); i += kF8Threads) {
                const int r = i / (pitch / 4), c = i - r * (pitch / 4);
                reinterpret_cast<uint32_t *>(wtab)[i] = reinterpret_cast<const uint32_t *>(a.ws + (r0 + min(r, last)) * pitch)[c];
            }
        }
        // The first chunk's weights were asked for before its token rows, so the count that a chunk waits for does not cover these: all but the
        // second chunk's rows are awaited here (a wave that fetches no scales has nothing else that waits).  And the scale tables are
        // written.  Both are met by the first barrier.
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(ONE ? 0 : NB) : "memory");
        int c = 0;
        for (; c + 2 < nk; ++c) chunk(c, two);
        if constexpr (!ONE) chunk(c++, one);
        chunk(c, none);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();  // everyone is done with the ring
        // acc[u][b][i]: unit row 8 (i / 4) + 4 half + i % 4, token row 32 b + l32
        if constexpr (GATEUP) {
            float *s_max = reinterpret_cast<float *>(tab);  // [4][kF8Tok]
            float h[2][NB][8], mx[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                mx[b] = 0.f;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float g = acc[u][b][i];
                        h[u][b][i] = g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * acc[u][b][i + 8];
                        mx[b] = fmaxf(mx[b], finite_abs(h[u][b][i]));
                    }
                mx[b] = fmaxf(mx[b], __shfl_xor(mx[b], 32));
                if (half == 0) s_max[wave * kF8Tok + 32 * b + l32] = mx[b];
            }
            __syncthreads();
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int r = 32 * b + l32;
                const int sb = scale_byte(fmaxf(fmaxf(s_max[r], s_max[kF8Tok + r]), fmaxf(s_max[2 * kF8Tok + r], s_max[3 * kF8Tok + r])));
                const float inv = scale_inverse(sb);
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const float *v = &h[u][b][4 * q];
                        *reinterpret_cast<uint32_t *>(ring + r * kFp8Block + (((wave * 2 + u) ^ ((r >> 1) & 7)) << 4) + 8 * q + 4 * half) =
                            to_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
                    }
                if (wave == 0 && half == 0 && r < rows) a.act_s[(size_t)(row0 + r) * fp8_pitch(a.Ip) + ft] = (uint8_t)sb;
            }
            __syncthreads();
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int r = 32 * b + (tid >> 3);
                if (r < rows)
                    *reinterpret_cast<u32x4_t *>(a.act + (size_t)(row0 + r) * a.Ip + ft * kFp8Block + (tid & 7) * 16) =
                        *reinterpret_cast<const u32x4_t *>(ring + r * kFp8Block + (((tid & 7) ^ ((r >> 1) & 7)) << 4));
            }
        } else {
            // a wave's 64 columns of 32 rows turn through 4 KiB of its own: whole cache lines leave
            if (rb >= rbs) return;
            uint8_t *buf = ring + wave * 4096;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                int k = 0;
                if constexpr (KIND == kF8DownScaled) {
                    int most = 0;
                    for (int c = 0; c < nk; ++c) most = max(most, (int)tab[(32 * b + l32) * pitch + c] + (int)wtab[(wave >> 1) * pitch + c]);
                    k = most - 254 + a.log_terms - 15;
                    if ((wave & 1) == 0 && half == 0 && 32 * b + l32 < rows)
                        a.y_exp[(size_t)(row0 + 32 * b + l32) * (a.H / kFp8Block) + ft * 2 + (wave >> 1)] = (int16_t)k;
                }
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        typedef std::conditional_t<KIND == kF8DownScaled, _Float16, bf16_t> out_t;
                        typedef out_t out4 __attribute__((ext_vector_type(4)));
                        out4 v;
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = (out_t)(KIND == kF8DownScaled ? ldexpf(acc[u][b][4 * q + i], -k) : acc[u][b][4 * q + i]);
                        *reinterpret_cast<out4 *>(buf + l32 * 128 + (((4 * u + q) ^ ((l32 >> 1) & 7)) << 4) + 8 * half) = v;
                    }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = 8 * i + (lane >> 3);
                    const u32x4_t v = *reinterpret_cast<const u32x4_t *>(buf + r * 128 + (((lane & 7) ^ ((r >> 1) & 7)) << 4));
                    if (32 * b + r < rows) *reinterpret_cast<u32x4_t *>((uint16_t *)a.y + (size_t)(row0 + 32 * b + r) * a.H + rb * 32 + (lane & 7) * 8) = v;
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
        }
    }
};

template <int KIND, bool ONE, bool BIG>
__global__ __launch_bounds__(kF8Threads, 2) void ffn_fp8_kernel(F8Args a)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    F8Tiles t;
    t.count(a.offsets, a.N, a.tok);
    // the chip hands workgroups to its eight XCDs in turn: each takes a contiguous eighth of the items, so that the feature tiles of a
    // token tile and the token tiles of an expert meet in one L2
    const int items = t.total * a.nft, per = (items + 7) / 8, idx = blockIdx.x >> 3, item = (blockIdx.x & 7) * per + idx;
    if (idx >= per || item >= items) return;
    const int tile = item / a.nft, ft = item - tile * a.nft;
    const int3 at = t.locate(tile);
    const F8Kernel<KIND, ONE, BIG> k = {a, lds, lds + kF8Ring, at.x, at.y, at.z, ft};
    const int nb = (at.z + 31) >> 5;
    if (nb == 1) k.template run<1>();
    else if (nb == 2) k.template run<2>();
    else if (nb == 3) k.template run<3>();
    else if (nb == 4) k.template run<4>();
    else k.template run<5>();
}

// scratch: token rows and scales, activations and scales, exponents of the expert outputs
struct F8Ws {
    size_t x, xs, act, act_s, y_exp, total;
};
static F8Ws fp8_ws(const zeda_layer_desc *d)
{
    const size_t S = (size_t)d->T * d->K;
    F8Ws w;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes ? bytes : 1, 256); return at; };
    w.x = take((size_t)d->T * d->H);
    w.xs = take((size_t)d->T * fp8_pitch(d->H));
    // (fp32 for small batches; never less for a longer batch: callers size workspaces once, for their longest)
    const size_t few = fp8_few_slots(d), most = S < few ? S : few;
    w.act = take(S * fp8_cols(d->I) > most * 4 * d->I ? S * fp8_cols(d->I) : most * 4 * d->I);
    w.act_s = take(S * fp8_pitch(d->I));
    w.y_exp = take(S * (d->H / kFp8Block) * 2);
    w.total = o;
    return w;
}
size_t fp8_ffn_ws_bytes(const zeda_layer_desc *d) { return fp8_ws(d).total; }

template <int KIND, bool ONE, bool BIG = false>
static int launch_f8_chunks(const F8Args &a, int S, hipStream_t s)
{
    const int pitch = fp8_pitch(KIND == kF8GateUp ? a.H : a.Ip), tab = (kF8Tok + 2) * pitch, bytes = kF8Ring + (tab > 4 * kF8Tok * 4 ? tab : 4 * kF8Tok * 4);
    static bool done[kMaxDevices] = {};  // per instantiation and device (idempotent)
    const int dev = current_device();
    if (dev < 0) return ZEDA_EHIP;
    if (!done[dev]) {
        constexpr int most = kF8Ring + (kF8Tok + 2) * (kFp8MaxWidth / kFp8Block);
        if (hipFuncSetAttribute((const void *)ffn_fp8_kernel<KIND, ONE, BIG>, hipFuncAttributeMaxDynamicSharedMemorySize, most) != hipSuccess) return ZEDA_EHIP;
        done[dev] = true;
    }
    const int64_t items = ((int64_t)S / a.tok + (a.N < S ? a.N : S)) * a.nft, grid = (items + 7) / 8 * 8;
    if (grid > 0x7fffffff) return ZEDA_EUNSUPPORTED;
    ffn_fp8_kernel<KIND, ONE, BIG><<<(unsigned)grid, kF8Threads, bytes, s>>>(a);
    return last_launch_status();
}

template <int KIND>
static int launch_f8(const F8Args &a, int S, hipStream_t s)
{
    // (a single chunk's token rows never pass 4 GiB: T * K < 2^24)
    if (KIND == kF8GateUp && (int64_t)a.T * a.H >= (int64_t)1 << 32) return launch_f8_chunks<kF8GateUp, false, true>(a, S, s);
    return (KIND == kF8GateUp ? a.H : a.Ip) == kFp8Block ? launch_f8_chunks<KIND, true>(a, S, s) : launch_f8_chunks<KIND, false>(a, S, s);
}

int launch_ffn_fp8(const zeda_layer_desc *d, const void *x, const zeda_fp8_experts *e, const int32_t *offsets, const int32_t *sorted_slot,
                   void *y_slot, const int16_t **y_exp, void *ws, const TilePlace *tp, hipStream_t s)
{
    const F8Ws L = fp8_ws(d);
    uint8_t *w = (uint8_t *)ws;
    const int S = d->T * d->K, Ip = fp8_cols(d->I);
    int log_terms = 18;
    while ((1 << (log_terms - 18)) < Ip) ++log_terms;  // (448 * 448 < 2^18)
    if (y_exp) *y_exp = (int16_t *)(w + L.y_exp);
    if (fp8_few(d))
        return launch_ffn_fp8_few(d, x, e, offsets, sorted_slot, y_slot, y_exp ? (int16_t *)(w + L.y_exp) : nullptr, (float *)(w + L.act), log_terms, tp, s);
    int rc = launch_quantize_rows(d->T, d->H, d->dtype, x, w + L.x, d->H, w + L.xs, fp8_pitch(d->H), s);
    if (rc != ZEDA_OK) return rc;
    F8Args a = {};
    a.offsets = offsets; a.sorted_slot = sorted_slot;
    a.T = d->T; a.N = d->N; a.K = d->K; a.H = d->H; a.Ip = Ip;
    a.src = w + L.x; a.src_s = w + L.xs;
    a.w = (const uint8_t *)e->w_gateup; a.ws = (const uint8_t *)e->s_gateup;
    a.act = w + L.act; a.act_s = w + L.act_s;
    a.nft = Ip / kFp8Block;
    // Tiles of up to 160 rows use each weight more often, tiles of up to 128 make more workgroups; by the work items that all slots would make.
    // Whole layer, us, 128 / 160 rows: N=24, I=448, H=1152, 3000 tokens (280 items) 44.7 / 48.1; N=64, I=1536, H=2048, 2048 tokens (768) 149.3 /
    // 150.9, 8192 skewed (3072) 225.1 / 226.9, 16384 (6144) 422.4 / 417.9; N=128, I=768, H=2048, 2048 tokens (768) 159.1 / 160.9, 4096 (1536) 202.3 /
    // 202.3, 8192 (3072) 280.5 / 270.5, 16381 skewed (6144) 453.8 / 443.9
    a.tok = (int64_t)S * a.nft < 128 * 3072 ? 128 : kF8Tok;
    if ((rc = launch_f8<kF8GateUp>(a, S, s)) != ZEDA_OK) return rc;
    a.src = a.act; a.src_s = a.act_s;
    a.w = (const uint8_t *)e->w_down; a.ws = (const uint8_t *)e->s_down;
    a.y = y_slot;
    a.nft = ceil_div(d->H, 256);
    if (!y_exp) return launch_f8<kF8Down>(a, S, s);
    a.y_exp = (int16_t *)(w + L.y_exp);
    a.log_terms = log_terms;
    return launch_f8<kF8DownScaled>(a, S, s);
}

}  // namespace zeda
