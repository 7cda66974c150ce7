// The routing of a few tokens by the workgroups of the gate/up kernels themselves.
#pragma once
#include "zeda_place.h"
#include "zeda_select.h"

namespace zeda {

// The routing of up to kTileSelTokens tokens from their partial logits, a token per wave; s_ids receives the ids.  The same
// additions and the same selection as in the router's second kernel, of four waves or of sixteen (tp.by_rows).
__device__ __forceinline__ void select_tokens(const TilePlace &tp, int T, int N, int K, bool lead, float (*lg)[kMaxExperts], int *s_ids)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (wave < T) {
        // (all loads in flight together: each is a trip to another XCD's results)
        constexpr int NC = kMaxExperts / 64, MAXQ = 16;
        float v[MAXQ][NC], bias[NC] = {};
#pragma unroll
        for (int q = 0; q < MAXQ; ++q)
            if (q < tp.slices) {
#pragma unroll
                for (int c = 0; c < NC; ++c) v[q][c] = tp.partial[((size_t)q * tp.Tpad + wave) * tp.E + min(lane + 64 * c, tp.E - 1)];
            }
        if (tp.bias) {
#pragma unroll
            for (int c = 0; c < NC; ++c) bias[c] = tp.bias[min(lane + 64 * c, tp.NE - 1)];
        }
#pragma unroll
        for (int q = 1; q < MAXQ; ++q)
            if (q < tp.slices) {
#pragma unroll
                for (int c = 0; c < NC; ++c) v[0][c] += v[q][c];
            }
#pragma unroll
        for (int c = 0; c < NC; ++c) lg[wave][lane + 64 * c] = v[0][c] + bias[c];
        // (a wave reads what it wrote; experts past NE are left out)
        const int id = select_wave<kMaxExperts / 64>(lg[wave], true, wave, tp.NE, N, K, tp.gate_norm, lead ? tp.ids : nullptr, tp.gates, nullptr, tp.by_rows);
        if (lane < K) s_ids[wave * K + lane] = id;
    }
    __syncthreads();
}

// Where a tile's rows come from: the tables of a placement, the ids of all slots, or the logits of all tokens (tp).
enum FewFrom { kFromTables, kFromIds, kFromLogits };

}  // namespace zeda
