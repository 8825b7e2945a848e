// Top-k router with balance and z loss: one pass over the logits forward, one backward.
//
// A token belongs to a group of kGroup lanes, each with kMine of its logits in registers (eight experts or fewer: one
// thread; 256 or more: a warp), read as 16-byte vectors where rows allow it, the next token's while this one is worked on.
// The passes are bound by instructions, not by HBM: a round of the choice costs a few dozen, and with many experts in fp32
// the k rounds give way to one count.
//
// Forward: softmax, choice and weights are local to a token; the losses need the sums over tokens of p_te, of lse^2 and
// the counts.  Every lane keeps the sums of its own experts in registers over all its tokens, the block adds them up in a
// fixed order and leaves one partial row in the workspace, and the blocks that finish last add the rows, again in a fixed
// order.  One launch, and no floating-point atomics.
// Backward: with the counts known the gradient of a token's logits is local to the token again; it is recomputed from
// the logits, which are the only thing both passes have to read.
#include <cfloat>

#include "layer_common.h"

namespace loco_layer {

constexpr int kMaxExperts = 512;
constexpr int kMaxChoice = 16;
constexpr int kTeam = 16;                           // blocks whose rows are added first; also the most teams
constexpr int kMaxBlocks = kTeam * kTeam;           // partial rows the workspace holds
constexpr uint64_t kTicketBytes = 256;
constexpr unsigned kAll = 0xffffffffu;
constexpr float kLog2e = 1.4426950408889634f;

struct RouterParams {
    const void *logits;
    int64_t row_stride;
    const uint8_t *mask;
    int32_t *index;
    float *weight;
    int32_t *counts;
    float *mean, *losses;
    unsigned *ticket;                                // the teams', then each team's; zero between calls
    float *part;                                     // [block][E + 1][2]: sum of p and count (an integer) of an expert; sum of lse^2, active tokens
    double2 *team_part;                              // the same of a team
    // backward
    const int32_t *in_index, *in_counts;
    const float *dlosses, *dweight;
    void *dlogits;
    int64_t drow_stride;
    int64_t tokens;
    int32_t experts, top_k, normalize;
    float balance_coef, z_coef;
};

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(kAll, x, o);
    return x;
}
__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(kAll, x, o);
    return x;
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Which expert the lane's i-th value belongs to: vectors of 16 bytes go round the group, single values otherwise.
template <typename T, int kGroup, bool kWide> __device__ __forceinline__ int expert_of(int lane, int i) {
    constexpr int kV = kWide ? 16 / static_cast<int>(sizeof(T)) : 1;
    return (i / kV * kGroup + lane) * kV + i % kV;
}

// The lane's part of a row as it lies in memory; what is past the last expert reads as -inf.
template <typename T, int kGroup, int kMine, bool kWide> struct Row {
    static constexpr int kV = kWide ? 16 / static_cast<int>(sizeof(T)) : 1;
    Pack<T, kV> v[kMine / kV];
    __device__ __forceinline__ void load(const T *row, int lane, int experts) {
#pragma unroll
        for (int i = 0; i < kMine / kV; ++i) {
            const int e = (i * kGroup + lane) * kV;
            if (e < experts) {
                v[i] = *reinterpret_cast<const Pack<T, kV> *>(row + e);
            } else {
#pragma unroll
                for (int x = 0; x < kV; ++x) v[i].v[x] = from_f32<T>(-INFINITY);
            }
        }
    }
    __device__ __forceinline__ float operator[](int i) const { return to_f32(v[i / kV].v[i % kV]); }
};

template <int kGroup> __device__ __forceinline__ float group_sum(float x) {
#pragma unroll
    for (int o = kGroup / 2; o; o >>= 1) x += __shfl_xor_sync(kAll, x, o);
    return x;
}
template <int kGroup> __device__ __forceinline__ float group_max(float x) {
#pragma unroll
    for (int o = kGroup / 2; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(kAll, x, o));
    return x;
}

// p[i] = exp(z[i] - top), their sum and log-sum-exp over the group; false where no expert is available.
template <int kGroup, int kMine> __device__ __forceinline__ bool softmax(const float *z, float *p, float &top, float &total, float &lse) {
    top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kMine; ++i) top = fmaxf(top, z[i]);
    top = group_max<kGroup>(top);
    const bool some = top != -INFINITY;
    const float from = some ? top : 0.0f;
    total = 0.0f;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        p[i] = exp2_fast((z[i] - from) * kLog2e);   // -inf gives 0
        total += p[i];
    }
    total = group_sum<kGroup>(total);
    lse = logf(total) + from;
    return some || total != total;
}

// Adds the blocks' partial rows once all of them are written; called by every thread with the block's own row in shared
// memory: sums[E], tally[E], the sum of lse^2 and the active tokens.  In two levels, a team of 16 blocks and the teams: the last
// block of a team adds its rows, the last team's block the teams'.  One block adding 148 rows of 160 experts alone took 16 us.
__device__ void finish(const RouterParams &P, const float *sums, const int *tally, float zsq, int active) {
    __shared__ bool last;
    __shared__ double fold[32];
    __shared__ double sum[kMaxExperts + 1];          // the last place: lse^2, active tokens
    __shared__ int count[kMaxExperts + 1];
    const int E = P.experts, tid = threadIdx.x, threads = blockDim.x;
    const int blocks = static_cast<int>(gridDim.x), team = static_cast<int>(blockIdx.x) / kTeam, teams = (blocks + kTeam - 1) / kTeam;
    for (int c = tid; c <= E; c += threads) {
        sum[c] = c < E ? sums[c] : zsq;
        count[c] = c < E ? tally[c] : active;
    }
    if (blocks > 1) {
        float *const mine = P.part + static_cast<int64_t>(blockIdx.x) * 2 * (E + 1);
        for (int c = tid; c <= E; c += threads) {
            mine[2 * c] = static_cast<float>(sum[c]);
            mine[2 * c + 1] = __int_as_float(count[c]);
        }
        const int rows = min(kTeam, blocks - team * kTeam);
        __threadfence();
        __syncthreads();
        if (tid == 0) last = atomicAdd(P.ticket + 1 + team, 1u) == static_cast<unsigned>(rows) - 1;
        __syncthreads();
        if (!last) return;
        __threadfence();
        if (tid == 0) P.ticket[1 + team] = 0;
        const float2 *from = reinterpret_cast<const float2 *>(P.part) + static_cast<int64_t>(team) * kTeam * (E + 1);
        for (int c = tid; c <= E; c += threads) {
            float2 r[kTeam];
#pragma unroll
            for (int b = 0; b < kTeam; ++b) r[b] = b < rows ? __ldcg(from + static_cast<int64_t>(b) * (E + 1) + c) : make_float2(0.0f, 0.0f);
            double a = 0.0;
            int k = 0;
#pragma unroll
            for (int b = 0; b < kTeam; ++b) {
                a += static_cast<double>(r[b].x);
                k += __float_as_int(r[b].y);
            }
            sum[c] = a;
            count[c] = k;
        }
    }
    if (teams > 1) {
        double2 *const mine = P.team_part + static_cast<int64_t>(team) * (E + 1);
        for (int c = tid; c <= E; c += threads) mine[c] = make_double2(sum[c], static_cast<double>(count[c]));
        __threadfence();
        __syncthreads();
        if (tid == 0) last = atomicAdd(P.ticket, 1u) == static_cast<unsigned>(teams) - 1;
        __syncthreads();
        if (!last) return;
        __threadfence();
        if (tid == 0) P.ticket[0] = 0;
        for (int c = tid; c <= E; c += threads) {
            double2 r[kTeam];
#pragma unroll
            for (int b = 0; b < kTeam; ++b) r[b] = b < teams ? __ldcg(P.team_part + static_cast<int64_t>(b) * (E + 1) + c) : make_double2(0.0, 0.0);
            double a = 0.0, k = 0.0;
#pragma unroll
            for (int b = 0; b < kTeam; ++b) {
                a += r[b].x;
                k += r[b].y;
            }
            sum[c] = a;
            count[c] = static_cast<int>(k);
        }
    }
    __syncthreads();
    const double zz = sum[E];
    const int n = count[E];
    const double per = n > 0 ? 1.0 / n : 0.0;
    double load = 0.0;
    for (int e = tid; e < E; e += threads) {
        P.mean[e] = static_cast<float>(sum[e] * per);
        P.counts[e] = count[e];
        load += static_cast<double>(count[e]) * (sum[e] * per);
    }
    load = warp_sum(load);
    if (tid % 32 == 0) fold[tid / 32] = load;
    __syncthreads();
    if (tid == 0) {
        double all = 0.0;
        for (int w = 0; w < threads / 32; ++w) all += fold[w];
        P.counts[E] = n;
        P.losses[0] = static_cast<float>(static_cast<double>(P.balance_coef) * E * all * per / P.top_k);
        // logits of the type's lowest value have squares past fp32: infinite in the sum, and nothing without a coefficient
        P.losses[1] = P.z_coef == 0.0f && zz == INFINITY ? 0.0f : static_cast<float>(static_cast<double>(P.z_coef) * zz * per);
    }
}

// The choice among a token's logits: next() gives the group's largest one left, lowest expert first, and takes it out.
// fp32: the largest value, then the lowest expert that has it, one reduction over the group each.  NaN counts as +inf.
template <typename T, int kGroup, int kMine, bool kWide> struct Chooser {
    float z[kMine];
    __device__ __forceinline__ Chooser(const float *from, int) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) z[i] = from[i] != from[i] ? INFINITY : from[i];
    }
    __device__ __forceinline__ int next(int lane, float &value) {
        float best = z[0];
#pragma unroll
        for (int i = 1; i < kMine; ++i) best = fmaxf(best, z[i]);
        best = group_max<kGroup>(best);
        value = best;
        int mine = kMine;
#pragma unroll
        for (int i = kMine - 1; i >= 0; --i) mine = z[i] == best ? i : mine;
        // the lane's first place with it, as an expert
        constexpr int kV = kWide ? 16 / static_cast<int>(sizeof(T)) : 1;
        const int own = mine < kMine ? (mine / kV * kGroup + lane) * kV + mine % kV : 0x7fffffff;
        int at = own;
#pragma unroll
        for (int o = kGroup / 2; o; o >>= 1) at = min(at, __shfl_xor_sync(kAll, at, o));
        mine = own == at ? mine : kMine;
#pragma unroll
        for (int i = 0; i < kMine; ++i) z[i] = i == mine ? -INFINITY : z[i];
        return best == -INFINITY ? -1 : at;
    }
};
// bfloat16: value and expert fit one integer whose order is the choice's (order of the value in the upper half, 0xffff -
// expert in the lower), so that one reduction finds both.  Adding 0 makes -0 plain and NaN the largest integer, which then
// counts as +infinity's.
template <int kGroup, int kMine, bool kWide> struct Chooser<__nv_bfloat16, kGroup, kMine, kWide> {
    unsigned key[kMine];
    __device__ __forceinline__ Chooser(const float *from, int lane) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int u = min(__float_as_int(from[i] + 0.0f), 0x7f800000);
            key[i] = ((u ^ (u >> 31 | 0x80000000u)) & 0xffff0000u) | (0xffffu - expert_of<__nv_bfloat16, kGroup, kWide>(lane, i));
        }
    }
    __device__ __forceinline__ int next(int, float &value) {
        unsigned best = key[0];
#pragma unroll
        for (int i = 1; i < kMine; ++i) best = max(best, key[i]);
        if constexpr (kGroup == 32) {
            best = __reduce_max_sync(kAll, best);
        } else {
#pragma unroll
            for (int o = kGroup / 2; o; o >>= 1) best = max(best, __shfl_xor_sync(kAll, best, o));
        }
#pragma unroll
        for (int i = 0; i < kMine; ++i) key[i] = key[i] == best ? 0u : key[i];
        const unsigned v = best & 0xffff0000u;
        value = __uint_as_float(v & 0x80000000u ? v ^ 0x80000000u : ~v & 0xffff0000u);
        return v <= 0x007f0000u ? -1 : static_cast<int>(0xffffu - (best & 0xffffu));
    }
};

// The choice in one go, for fp32 and 16 or 32 lanes (65 experts and more).  `bar` is the k-th largest of the lanes' largest
// values: k values at least reach it, so the choice is among those that do.  They are few (to meet k of G lanes takes G (1/G +
// ... + 1/(G-k+1)) draws of a random order: 7.2 for 6 of 16, 9.0 for 8 of 32); they are laid side by side, and each lane counts
// those before its own.  False, for the whole warp, where more than G reach `bar` for one of its tokens (equal logits): the
// rounds of Chooser make the same choice.  Choice j comes back in lane j.
// Forward, 50021 tokens, fp32, by rounds and so: 160 experts, k = 2: 26.5, 28.9 us; 3: 30.4, 28.9; 6: 41.5, 29.0; 8: 49.4, 31.5;
// 256 experts, k = 2: 32.9, 34.3; 3: 38.3, 35.0; 8: 65.7, 38.7; 16: 110.0, 47.3; 512 experts, k = 8: 116.4, 56.1.  8 lanes gain 0.7 us
// at most.  From k = 3, then; with 16 lanes to 8, beyond which more than 16 values often reach `bar` (9 would take 12.7 draws,
// 10 take 14.9).
constexpr int kRankFrom = 3;
template <int kGroup> __host__ __device__ constexpr int rank_most() { return kGroup == 16 ? 8 : 16; }
template <int kGroup> struct alignas(16) Candidates {
    float value[kGroup];
    int expert[kGroup];
};
template <int kGroup, int kMine, bool kWide>
__device__ __forceinline__ bool rank_choice(const float *from, int lane, int k, Candidates<kGroup> &C, float &value, int &pick) {
    float z[kMine], most = -INFINITY;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        z[i] = from[i] != from[i] ? INFINITY : from[i];
        most = fmaxf(most, z[i]);
    }
    float bar;
    if constexpr (kGroup == 32) {                    // one at a time, as integers of the same order
        const int u = __float_as_int(most + 0.0f);
        unsigned left = u ^ (u >> 31 | 0x80000000u), best = 0;
#pragma unroll 1
        for (int j = 0; j < k; ++j) {
            best = __reduce_max_sync(kAll, left);
            left = left == best ? 0u : left;
        }
        bar = __uint_as_float(best & 0x80000000u ? best ^ 0x80000000u : ~best);      // 0, none left: NaN
    } else {
        int before = 0;
#pragma unroll
        for (int o = 1; o < kGroup; ++o) before += __shfl_xor_sync(kAll, most, o) > most;
        bar = before < k ? most : INFINITY;
#pragma unroll
        for (int o = kGroup / 2; o; o >>= 1) bar = fminf(bar, __shfl_xor_sync(kAll, bar, o));
    }
    bar = fmaxf(bar, -FLT_MAX);                      // what is not available is never chosen
    int at = 0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) at += z[i] >= bar;
    const int own = at;
#pragma unroll
    for (int o = 1; o < kGroup; o <<= 1) {
        const int x = __shfl_up_sync(kAll, at, o, kGroup);
        at += lane >= o ? x : 0;
    }
    const int n = __shfl_sync(kAll, at, kGroup - 1, kGroup);
    if (__any_sync(kAll, n > kGroup)) return false;
    at -= own;
    __syncwarp();                                    // the token before has been read
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        if (z[i] >= bar) {
            C.value[at] = z[i];             // at < n <= kGroup
            C.expert[at] = expert_of<float, kGroup, kWide>(lane, i);
            ++at;
        }
    }
    if (lane >= n) {
        C.value[lane] = -INFINITY;
        C.expert[lane] = -1;
    }
    __syncwarp();
    const float mine = C.value[lane];
    const int expert = C.expert[lane];
    int rank = 0;
    const int to = kGroup == 32 ? n : kGroup;
#pragma unroll kGroup == 32 ? 1 : kGroup / 4
    for (int j = 0; j < to; j += 4) {
        const float4 x = *reinterpret_cast<const float4 *>(C.value + j);
        rank += (x.x > mine) + (x.y > mine) + (x.z > mine) + (x.w > mine);
    }
    // equal values share a rank: lowest expert first
    const unsigned taken = __reduce_or_sync(kAll, lane < n ? 1u << (rank + threadIdx.x % 32 / kGroup * kGroup) : 0u);
    if (__popc(taken) != __popc(__ballot_sync(kAll, lane < n)))
        for (int j = 0; j < kGroup; ++j) rank += C.value[j] == mine && C.expert[j] < expert;
    if (lane >= n) rank = lane;
    __syncwarp();
    C.value[rank] = mine;
    C.expert[rank] = expert;
    __syncwarp();
    value = C.value[lane];
    pick = C.expert[lane];
    return true;
}

// Where a lane keeps the group's choices: choice j in lane j % kGroup, place j / kGroup.
template <int kGroup, int kMine> __host__ __device__ constexpr int choice_places() {
    return ((kGroup * kMine < kMaxChoice ? kGroup * kMine : kMaxChoice) + kGroup - 1) / kGroup;
}
template <int kMine> __host__ __device__ constexpr int forward_threads() { return kMine > 12 ? 512 : 1024; }

template <typename T, int kGroup, int kMine, bool kWide>
__global__ void __launch_bounds__(forward_threads<kMine>()) router_forward(const __grid_constant__ RouterParams P) {
    extern __shared__ float sums[];                  // [warp][experts of all places]
    __shared__ int tally[kMaxExperts];
    __shared__ float extra[32];
    __shared__ int active[32];
    constexpr int kPlaces = choice_places<kGroup, kMine>(), kRow = kGroup * kMine;
    constexpr bool kRank = kGroup >= 16 && sizeof(T) == 4;
    __shared__ Candidates<kGroup> candidates[kRank ? forward_threads<kMine>() / kGroup : 1];
    const int E = P.experts, tid = threadIdx.x, warp = tid / 32, lane = tid % kGroup, warps = blockDim.x / 32, k = P.top_k;
    const bool rank = k >= kRankFrom && k <= rank_most<kGroup>();
    for (int e = tid; e < E; e += blockDim.x) tally[e] = 0;
    wait_for_previous();
    let_next_start();
    __syncthreads();
    float sum[kMine], zsq = 0.0f;
    int act = 0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) sum[i] = 0.0f;
    const int64_t step = static_cast<int64_t>(gridDim.x) * blockDim.x / kGroup;
    int64_t t = (static_cast<int64_t>(blockIdx.x) * blockDim.x + tid) / kGroup;
    const T *logits = static_cast<const T *>(P.logits);
    Row<T, kGroup, kMine, kWide> next;
    const auto fetch = [&](int64_t at) { next.load(logits + at * P.row_stride, lane, at < P.tokens && (!P.mask || P.mask[at] != 0) ? E : 0); };
    fetch(t);
    // every lane of a warp goes round as often as the warp's first group
    for (int64_t lead = t - (tid % 32) / kGroup; lead < P.tokens; lead += step, t += step) {
        float z[kMine], p[kMine];
#pragma unroll
        for (int i = 0; i < kMine; ++i) z[i] = next[i];
        if (lead + step < P.tokens) fetch(t + step);
        float top, total, lse;
        const bool some = softmax<kGroup, kMine>(z, p, top, total, lse);
        const float inv = some ? 1.0f / total : 0.0f;
        if (some) {
            act += lane == 0;
            zsq = lane == 0 ? fmaf(lse, lse, zsq) : zsq;
#pragma unroll
            for (int i = 0; i < kMine; ++i) sum[i] = fmaf(p[i], inv, sum[i]);
        }
        const float from = top != -INFINITY ? top : 0.0f;
        float share = 0.0f, w[kPlaces];
        int pick[kPlaces];
        bool chosen = false;
        if constexpr (kRank)
            if (rank) chosen = rank_choice<kGroup, kMine, kWide>(z, lane, k, candidates[tid / kGroup], w[0], pick[0]);
        if (!chosen) {
            Chooser<T, kGroup, kMine, kWide> choose(z, lane);
#pragma unroll
            for (int place = 0; place < kPlaces; ++place) {
                pick[place] = -1;
                w[place] = 0.0f;
#pragma unroll 1
                for (int j = place * kGroup; j < k && j < (place + 1) * kGroup; ++j) {
                    float value;
                    const int at = choose.next(lane, value);
                    if (lane == j % kGroup) {
                        pick[place] = at;
                        w[place] = value;
                    }
                }
            }
        }
#pragma unroll
        for (int place = 0; place < kPlaces; ++place) {
            w[place] = place * kGroup + lane < k && pick[place] >= 0 ? exp2_fast((w[place] - from) * kLog2e) : 0.0f;
            share += w[place];
        }
        share = group_sum<kGroup>(share);
        const float by = P.normalize ? (share != 0.0f ? 1.0f / share : 1.0f) : inv;
        if (t < P.tokens) {
#pragma unroll
            for (int place = 0; place < kPlaces; ++place) {
                const int j = place * kGroup + lane;
                if (j < k) {
                    P.index[t * k + j] = pick[place];
                    P.weight[t * k + j] = w[place] * by;
                    if (pick[place] >= 0) atomicAdd(&tally[pick[place]], 1);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kMine; ++i) {                // over the groups of the warp
#pragma unroll
        for (int o = 16; o >= kGroup; o >>= 1) sum[i] += __shfl_xor_sync(kAll, sum[i], o);
        if (tid % 32 < kGroup) sums[warp * kRow + expert_of<T, kGroup, kWide>(lane, i)] = sum[i];
    }
    zsq = warp_sum(zsq);
    act = __reduce_add_sync(kAll, act);
    if (tid % 32 == 0) { extra[warp] = zsq; active[warp] = act; }
    __syncthreads();
    for (int e = tid; e < E; e += blockDim.x)
        for (int v = 1; v < warps; ++v) sums[e] += sums[v * kRow + e];
    zsq = 0.0f;
    act = 0;
    for (int v = 0; v < warps; ++v) { zsq += extra[v]; act += active[v]; }
    __syncthreads();
    finish(P, sums, tally, zsq, act);
}

constexpr int kBackwardThreads = 256;
// Blocks of an SM, and the grid is as many as run at once (50021 x 160 in fp32, 131072 x 64 and 40000 x 256 in bfloat16: 17.6,
// 20.1, 22.2 us with eight blocks an SM in the grid; with three that run at once 15.1, 18.2, 23.6, with four 17.0, 17.1, 20.6;
// sixteen values a lane, 20000 x 512 in bfloat16, with two, three, four: 17.2, 16.5, 19.3).
template <int kMine> __host__ __device__ constexpr int backward_blocks() { return kMine > 8 ? 3 : 4; }

// dz_e = p_e (g_e - sum_j p_j g_j) + 2 b lse p_e / N + the chosen weights' part, g_e = d balance / d p_e.  All experts are
// written as if unchosen, then the lanes that hold the choices write theirs.
template <typename T, int kGroup, int kMine, bool kWide>
__global__ void __launch_bounds__(kBackwardThreads, backward_blocks<kMine>()) router_backward(const __grid_constant__ RouterParams P) {
    __shared__ float slope[kMaxExperts];
    constexpr int kPlaces = choice_places<kGroup, kMine>();
    constexpr int kV = kWide ? 16 / static_cast<int>(sizeof(T)) : 1;
    const int E = P.experts, tid = threadIdx.x, lane = tid % kGroup, k = P.top_k;
    wait_for_previous();
    let_next_start();
    const int n = P.in_counts[E];
    const float per = n > 0 ? 1.0f / static_cast<float>(n) : 0.0f;
    const float scale = P.dlosses ? P.dlosses[0] * P.balance_coef * static_cast<float>(E) / static_cast<float>(k) * per * per : 0.0f;
    const float zc = P.dlosses ? P.dlosses[1] * P.z_coef * 2.0f * per : 0.0f;
    for (int e = tid; e < E; e += kBackwardThreads) slope[e] = scale * static_cast<float>(P.in_counts[e]);
    const int64_t step = static_cast<int64_t>(gridDim.x) * kBackwardThreads / kGroup;
    int64_t t = (static_cast<int64_t>(blockIdx.x) * kBackwardThreads + tid) / kGroup;
    const T *logits = static_cast<const T *>(P.logits);
    Row<T, kGroup, kMine, kWide> next;
    const auto fetch = [&](int64_t at) { next.load(logits + at * P.row_stride, lane, at < P.tokens && (!P.mask || P.mask[at] != 0) ? E : 0); };
    fetch(t);
    __syncthreads();
    float g[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int e = expert_of<T, kGroup, kWide>(lane, i);
        g[i] = e < E ? slope[e] : 0.0f;
    }
    for (int64_t lead = t - (tid % 32) / kGroup; lead < P.tokens; lead += step, t += step) {
        float z[kMine], p[kMine];
#pragma unroll
        for (int i = 0; i < kMine; ++i) z[i] = next[i];
        int e[kPlaces];
        float x[kPlaces], pe[kPlaces];
#pragma unroll
        for (int place = 0; place < kPlaces; ++place) {
            const int j = place * kGroup + lane;
            e[place] = P.dweight && j < k && t < P.tokens ? P.in_index[t * k + j] : -1;
            if (e[place] >= E) e[place] = -1;        // whatever the caller's indices hold, accesses stay in the row
            x[place] = e[place] >= 0 ? P.dweight[t * k + j] : 0.0f;
            pe[place] = e[place] >= 0 ? to_f32(logits[t * P.row_stride + e[place]]) : -INFINITY;      // the logit for now
        }
        if (lead + step < P.tokens) fetch(t + step);
        float top, total, lse;
        const bool some = softmax<kGroup, kMine>(z, p, top, total, lse);
        const float inv = some ? 1.0f / total : 0.0f, from = top != -INFINITY ? top : 0.0f;
        float dot = 0.0f, wd = 0.0f, share = 0.0f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            p[i] *= inv;
            dot = fmaf(p[i], g[i], dot);
        }
        dot = group_sum<kGroup>(dot);
        if (P.dweight) {
#pragma unroll
            for (int place = 0; place < kPlaces; ++place) {
                pe[place] = exp2_fast((pe[place] - from) * kLog2e) * inv;
                share += pe[place];
                wd = fmaf(pe[place], x[place], wd);
            }
            share = group_sum<kGroup>(share);
            wd = group_sum<kGroup>(wd);
        }
        const float common = (some ? zc * lse - dot : 0.0f), all = P.normalize ? common : common - wd;
        const float norm = share != 0.0f ? 1.0f / share : 1.0f;
        if (t < P.tokens) {
            T *out = static_cast<T *>(P.dlogits) + t * P.drow_stride;
#pragma unroll
            for (int i = 0; i < kMine / kV; ++i) {
                const int first = (i * kGroup + lane) * kV;
                if (first < E) {
                    Pack<T, kV> v;
#pragma unroll
                    for (int y = 0; y < kV; ++y) v.v[y] = from_f32<T>(p[i * kV + y] * (g[i * kV + y] + all));
                    *reinterpret_cast<Pack<T, kV> *>(out + first) = v;
                }
            }
        }
        if (P.dweight) {
            __syncwarp();                            // the choices' values come after the row's
            if (t < P.tokens) {
                T *out = static_cast<T *>(P.dlogits) + t * P.drow_stride;
#pragma unroll
                for (int place = 0; place < kPlaces; ++place)
                    if (e[place] >= 0)
                        out[e[place]] = from_f32<T>(pe[place] * (slope[e[place]] + all) +
                                                    (P.normalize ? pe[place] * norm * (x[place] - wd * norm) : pe[place] * x[place]));
            }
        }
    }
}

// Lanes and values a lane by the number of experts: eight values a lane, twelve (three vectors) from 129 to 192 in fp32,
// sixteen above 256.
using RouterKernel = void (*)(const RouterParams);
struct RouterShape {
    RouterKernel forward, backward;
    int group, row, threads, backward_blocks;
};
template <typename T, int kGroup, int kMine, bool kWide> RouterShape shape_of() {
    return RouterShape{router_forward<T, kGroup, kMine, kWide>, router_backward<T, kGroup, kMine, kWide>, kGroup, kGroup * kMine, forward_threads<kMine>(),
                       backward_blocks<kMine>()};
}
template <typename T, bool kWide> RouterShape router_shape(int E) {
    if (E <= 8) return shape_of<T, 1, 8, kWide>();
    if (E <= 16) return shape_of<T, 2, 8, kWide>();
    if (E <= 32) return shape_of<T, 4, 8, kWide>();
    if (E <= 64) return shape_of<T, 8, 8, kWide>();
    if (E <= 128) return shape_of<T, 16, 8, kWide>();
    if constexpr (sizeof(T) == 4)
        if (E <= 192) return shape_of<T, 16, 12, kWide>();
    if (E <= 256) return shape_of<T, 32, 8, kWide>();
    return shape_of<T, 32, 16, kWide>();
}
RouterShape pick_router(const loco_router_t *c, bool wide) {
    if (c->dtype == LOCO_BF16) return wide ? router_shape<__nv_bfloat16, true>(c->experts) : router_shape<__nv_bfloat16, false>(c->experts);
    return wide ? router_shape<float, true>(c->experts) : router_shape<float, false>(c->experts);
}

// Dynamic shared memory above the default limit (32 KB beside the 19 KB of static arrays).
bool allow_shared(RouterKernel fn) {
    if (cudaFuncSetAttribute(reinterpret_cast<const void *>(fn), cudaFuncAttributeMaxDynamicSharedMemorySize, 65536) == cudaSuccess) return true;
    cudaGetLastError();
    return false;
}

int check_router(const loco_router_t *c) {
    if (!c) return LOCO_ERR_ARG;
    if (c->dtype != LOCO_F32 && c->dtype != LOCO_BF16) return LOCO_ERR_ARG;
    if (c->experts < 1 || c->experts > kMaxExperts) return LOCO_ERR_ARG;
    if (c->top_k < 1 || c->top_k > kMaxChoice || c->top_k > c->experts) return LOCO_ERR_ARG;
    if (!std::isfinite(c->balance_coef) || !std::isfinite(c->z_coef)) return LOCO_ERR_ARG;
    return LOCO_OK;
}

}  // namespace loco_layer

using namespace loco_layer;

extern "C" {

uint64_t loco_router_workspace_bytes(const loco_router_t *c) {
    if (check_router(c) != LOCO_OK) return 0;
    return kTicketBytes + (static_cast<uint64_t>(kMaxBlocks) * 8 + static_cast<uint64_t>(kTeam) * 16) * (c->experts + 1);
}

int loco_router_forward(const loco_router_t *c, int64_t tokens, const void *d_logits, int64_t row_stride, const uint8_t *d_mask,
                        int32_t *d_index, float *d_weight, int32_t *d_counts, float *d_mean, float *d_losses, void *d_work,
                        uint64_t d_work_bytes, void *stream) {
    const int rc = check_router(c);
    if (rc != LOCO_OK) return rc;
    if (tokens < 0 || tokens > 0x7fffffff / c->top_k) return LOCO_ERR_ARG;
    if (!d_counts || !d_mean || !d_losses || !d_work || (tokens > 0 && (!d_logits || !d_index || !d_weight))) return LOCO_ERR_ARG;
    const uintptr_t size = c->dtype == LOCO_BF16 ? 2 : 4;
    if (!aligned(d_logits, size) || !aligned(d_index, 4) || !aligned(d_weight, 4) || !aligned(d_counts, 4) || !aligned(d_mean, 4) ||
        !aligned(d_losses, 4) || !aligned(d_work, 16)) return LOCO_ERR_ALIGN;
    if (d_work_bytes < loco_router_workspace_bytes(c)) return LOCO_ERR_SIZE;
    const int sms = sm_count();
    if (sms == 0) return LOCO_ERR_CUDA;
    RouterParams P{};
    P.logits = d_logits;
    P.row_stride = row_stride;
    P.mask = d_mask;
    P.index = d_index;
    P.weight = d_weight;
    P.counts = d_counts;
    P.mean = d_mean;
    P.losses = d_losses;
    P.ticket = static_cast<unsigned *>(d_work);
    P.team_part = reinterpret_cast<double2 *>(static_cast<uint8_t *>(d_work) + kTicketBytes);
    P.part = reinterpret_cast<float *>(P.team_part + static_cast<int64_t>(kTeam) * (c->experts + 1));
    P.tokens = tokens;
    P.experts = c->experts;
    P.top_k = c->top_k;
    P.normalize = c->normalize;
    P.balance_coef = c->balance_coef;
    P.z_coef = c->z_coef;
    // rows that are whole 16-byte vectors on 16-byte boundaries are read as such
    const int vec = 16 / static_cast<int>(size);
    const bool wide = aligned(d_logits, 16) && row_stride % vec == 0 && c->experts % vec == 0;
    const RouterShape R = pick_router(c, wide);
    // one block to an SM (every block leaves a partial row to be added), as wide as the tokens need
    const int64_t warps = (tokens * R.group + 31) / 32;
    const int most = sms < kMaxBlocks ? sms : kMaxBlocks;
    int64_t per = (warps + most - 1) / most;
    per = per < 4 ? 4 : (per > R.threads / 32 ? R.threads / 32 : per);
    int64_t blocks = (warps + per - 1) / per;
    blocks = blocks < 1 ? 1 : (blocks > most ? most : blocks);
    const size_t shared = static_cast<size_t>(per) * R.row * sizeof(float);
    if (shared > 28672 && !allow_shared(R.forward)) return LOCO_ERR_CUDA;
    return launch_kernel(R.forward, dim3(static_cast<unsigned>(blocks)), static_cast<unsigned>(per * 32), shared, stream, P);
}

int loco_router_backward(const loco_router_t *c, int64_t tokens, const void *d_logits, int64_t row_stride, const uint8_t *d_mask,
                         const int32_t *d_index, const int32_t *d_counts, const float *d_dlosses, const float *d_dweight,
                         void *d_dlogits, int64_t drow_stride, void *stream) {
    const int rc = check_router(c);
    if (rc != LOCO_OK) return rc;
    if (tokens < 0 || tokens > 0x7fffffff / c->top_k) return LOCO_ERR_ARG;
    if (tokens == 0) return LOCO_OK;
    if (!d_logits || !d_index || !d_counts || !d_dlogits || (tokens > 1 && drow_stride == 0)) return LOCO_ERR_ARG;
    const uintptr_t size = c->dtype == LOCO_BF16 ? 2 : 4;
    if (!aligned(d_logits, size) || !aligned(d_dlogits, size) || !aligned(d_index, 4) || !aligned(d_counts, 4) ||
        !aligned(d_dlosses, 4) || !aligned(d_dweight, 4)) return LOCO_ERR_ALIGN;
    const int sms = sm_count();
    if (sms == 0) return LOCO_ERR_CUDA;
    RouterParams P{};
    P.logits = d_logits;
    P.row_stride = row_stride;
    P.mask = d_mask;
    P.in_index = d_index;
    P.in_counts = d_counts;
    P.dlosses = d_dlosses;
    P.dweight = d_dweight;
    P.dlogits = d_dlogits;
    P.drow_stride = drow_stride;
    P.tokens = tokens;
    P.experts = c->experts;
    P.top_k = c->top_k;
    P.normalize = c->normalize;
    P.balance_coef = c->balance_coef;
    P.z_coef = c->z_coef;
    const int vec = 16 / static_cast<int>(size);
    const bool wide = aligned(d_logits, 16) && aligned(d_dlogits, 16) && row_stride % vec == 0 && drow_stride % vec == 0 && c->experts % vec == 0;
    const RouterShape R = pick_router(c, wide);
    int64_t blocks = (tokens * R.group + kBackwardThreads - 1) / kBackwardThreads;
    if (blocks > sms * R.backward_blocks) blocks = sms * R.backward_blocks;
    return launch_kernel(R.backward, dim3(static_cast<unsigned>(blocks)), kBackwardThreads, 0, stream, P);
}

}  // extern "C"
