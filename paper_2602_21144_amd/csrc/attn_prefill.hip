// Attention of prompt chunks: the plan of the work, and the choice of the padded width.
#include "attn_cut.h"
#include "attn_prefill.h"

namespace ssm {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kBins = 32;

// The steps of one tile: tokens [k0, k1) that its rows see
struct TileRange { int k0, k1, steps; };
__device__ __forceinline__ TileRange tile_range(const KvArgs& a, const KvSeq& s, int g, int row0, int height) {
    const int rows = s.m * g, last = min(row0 + height, rows) - 1;
    const int before = s.n - s.m, lo = before + row0 / g;
    TileRange r;
    r.k1 = before + last / g + 1;
    r.k0 = a.window > 0 && lo >= a.window ? (lo - a.window + 1) & ~(kStep - 1) : 0;
    r.steps = (r.k1 - r.k0 + kStep - 1) / kStep;
    return r;
}

// One workgroup: tiles of every sequence, the length that no item exceeds, and the items in bins of
// falling length. Places inside a bin come from LDS atomics: they settle which item runs first and
// where partial results lie, never what is added to what.
__global__ __launch_bounds__(kPlanThreads) void attn_plan_kernel(KvArgs a, AttnPlan p, bool bf16_act) {
    __shared__ int s_wave[kPlanThreads / 64];
    __shared__ int32_t s_prefix[kPlanThreads];
    __shared__ int s_len[512];
    __shared__ int s_bin[kBins], s_items, s_part, s_join;
    __shared__ unsigned long long s_steps;
    const int tid = threadIdx.x, lane = tid & 63, g = a.Hq / a.Hkv;
    kv_check_seqs(a, tid, kPlanThreads);
    if (tid < kBins) s_bin[tid] = 0;
    if (tid == 0) {
        s_steps = 0;
        s_part = s_join = 0;
    }
    const int per = (a.nseq + kPlanThreads - 1) / kPlanThreads;
    auto tiles_of = [&](int i) {
        const KvSeq s = kv_seq(a, i);
        return s.ok ? tiles_of_rows(s.m, g, p.rows) : 0;
    };
    int sum = 0;
    for (int k = 0; k < per; ++k)
        if (tid * per + k < a.nseq) sum = add_tiles(sum, tiles_of(tid * per + k));
    int incl = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int o = __shfl_up(incl, off, 64);
        if (lane >= off) incl = add_tiles(incl, o);
    }
    if (lane == 63) s_wave[tid >> 6] = incl;
    __syncthreads();
    int at = __shfl_up(incl, 1, 64), total = 0;
    if (lane == 0) at = 0;
    for (int k = 0; k < kPlanThreads / 64; ++k) {
        if (k < (tid >> 6)) at = add_tiles(at, s_wave[k]);
        total = add_tiles(total, s_wave[k]);
    }
    // the tiles before every sequence: in LDS where they fit
    int32_t* prefix = a.nseq <= kPlanThreads ? s_prefix : p.prefix;
    for (int k = 0; k < per; ++k) {
        const int i = tid * per + k;
        if (i < a.nseq) {
            prefix[i] = at;
            at = add_tiles(at, tiles_of(i));
        }
    }
    if (total > p.max_tiles) {   // sequences that overlap hold more rows than the call has
        if (tid == 0) atomicOr(a.status, SSM_STATUS_BAD_SEQLENS);
        total = p.max_tiles;
    }
    __syncthreads();
    struct Tile { int seq, row0; KvSeq s; TileRange r; };
    auto tile = [&](int t) {   // its sequence is the last one whose tiles begin at or before t
        int i = 0, e = a.nseq;
        while (e - i > 1) {
            const int mid = (i + e) >> 1;
            if (prefix[mid] <= t) i = mid;
            else e = mid;
        }
        const int row0 = (t - prefix[i]) * p.rows;
        const KvSeq s = kv_seq(a, i);
        return Tile{i, row0, s, tile_range(a, s, g, row0, p.rows)};
    };
    // a thread keeps its first tile over the three passes
    Tile first{};
    if (tid < total) first = tile(tid);
    auto each = [&](auto f) {
        if (tid < total) f(first);
        for (int t = tid + kPlanThreads; t < total; t += kPlanThreads) f(tile(t));
    };
    unsigned long long steps = 0;
    each([&](const Tile& x) { steps += x.r.steps; });
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) steps += __shfl_xor(steps, off, 64);
    if (lane == 0 && steps) atomicAdd(&s_steps, steps);
    __syncthreads();
    int most = longest_item(s_steps, a.Hkv, p.places, p.min_steps);   // steps of the longest item
    // If every tile has a place of its own at once, the cut is such that every item has: the first of 16 lengths,
    // from an equal share to twice that (float32: one and a half times), at which the items are no more than the
    // places. Float32 is otherwise cut to half a share, in two rounds: its steps are long, and what the rounds add
    // costs less than places without work (16 heads of 112, 2048 rows: 131 us and 13 for the join, uncut 160 and 4;
    // three prompts, one behind 4096 tokens: 146 and 10, in one round 140 and 6).
    if ((int64_t)total * a.Hkv <= p.places) {
        if (tid < total) s_len[tid] = first.r.steps;
        __syncthreads();
        const int c = tid >> 6, len = most + most * c / 16;
        int items = 0;
        for (int t = lane; t < total; t += 64) items += (s_len[t] + len - 1) / len;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) items += __shfl_xor(items, off, 64);
        if (lane == 0) s_wave[c] = (int64_t)items * a.Hkv <= p.places && (bf16_act || c <= 8) ? len : 0;
        __syncthreads();
        int found = 0;
        for (int k = kPlanThreads / 64 - 1; k >= 0; --k) found = s_wave[k] ? s_wave[k] : found;
        if (found) most = found;
        else if (!bf16_act) most = max(p.min_steps, (most + 1) / 2);
    }
    each([&](const Tile& x) {
        const TileCut c = cut_tile(x.r.steps, most);
        atomicAdd(&s_bin[item_bin(c.len, most, kBins)], c.pieces);
    });
    __syncthreads();
    if (tid < 64) {
        const int c = tid < kBins ? s_bin[tid] : 0;
        int n = c;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int o = __shfl_up(n, off, 64);
            if (lane >= off) n += o;
        }
        if (tid < kBins) s_bin[tid] = n - c;
        if (tid == 63) s_items = n;
    }
    __syncthreads();
    for (int k = s_items + tid; k < p.max_items; k += kPlanThreads) p.items[k].part = -2;
    each([&](const Tile& x) {
        const auto [pieces, len] = cut_tile(x.r.steps, most);
        const int pos = atomicAdd(&s_bin[item_bin(len, most, kBins)], pieces);
        int part = -1;
        if (pieces > 1) {
            part = atomicAdd(&s_part, pieces);
            p.joins[atomicAdd(&s_join, 1)] = AttnJoin{x.row0, part, pieces, x.s.lo, x.s.m, {0, 0, 0}};
        }
        for (int k = 0; k < pieces; ++k) {
            const int k0 = x.r.k0 + k * len * kStep;
            p.items[pos + k] = AttnItem{x.seq, x.row0, k0, min(x.r.k1, k0 + len * kStep), pieces > 1 ? part + k : -1, x.s.lo, x.s.m, x.s.n};
        }
    });
    __syncthreads();
    if (tid == 0) p.count[0] = s_join;
}

// The width that a head's values are padded to in the products. Float32 has one above 128.
int padded_dim(bool bf16_act, int D) {
    if (bf16_act) return D <= 64 ? 64 : (D + 31) / 32 * 32;
    return D <= 64 ? 64 : D <= 128 ? (D + 31) / 32 * 32 : 256;
}

template <typename T, int FMT> hipError_t prefill_dim(const AttnArgs& p, const AttnPlan& pl, int dp, hipStream_t s) {
    if constexpr (sizeof(T) == 2) {
        switch (dp) {
            case 160: return launch_attn_prefill_tile<T, FMT, 160>(p, pl, s);
            case 192: return launch_attn_prefill_tile<T, FMT, 192>(p, pl, s);
            case 224: return launch_attn_prefill_tile<T, FMT, 224>(p, pl, s);
        }
    }
    switch (dp) {
        case 64: return launch_attn_prefill_tile<T, FMT, 64>(p, pl, s);
        case 96: return launch_attn_prefill_tile<T, FMT, 96>(p, pl, s);
        case 128: return launch_attn_prefill_tile<T, FMT, 128>(p, pl, s);
        default: return launch_attn_prefill_tile<T, FMT, 256>(p, pl, s);
    }
}
template <typename T> hipError_t prefill_fmt(const AttnArgs& p, const AttnPlan& pl, int dp, hipStream_t s) {
    switch (p.kv.fmt) {
        case SSM_KV_ACT: return prefill_dim<T, SSM_KV_ACT>(p, pl, dp, s);
        case SSM_KV_FP8_E4M3: return prefill_dim<T, SSM_KV_FP8_E4M3>(p, pl, dp, s);
        default: return prefill_dim<T, SSM_KV_INT8>(p, pl, dp, s);
    }
}

}  // namespace

size_t attn_prefill_scratch_bytes(bool bf16_act, int Hq, int Hkv, int D, int64_t T, int nseq) {
    return T > 0 ? attn_plan(bf16_act, Hq, Hkv, padded_dim(bf16_act, D), T, nseq, nullptr).total : 0;
}
hipError_t launch_attn_prefill(const AttnArgs& p, bool bf16_act, hipStream_t s) {
    const KvArgs& a = p.kv;
    const int dp = padded_dim(bf16_act, a.D);
    const AttnPlan pl = attn_plan(bf16_act, a.Hq, a.Hkv, dp, a.T, a.nseq, p.scratch);
    KernelTimer kt("attn.prefill_plan", s);
    SSM_LAUNCH(attn_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a, pl, bf16_act);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return bf16_act ? prefill_fmt<bf16>(p, pl, dp, s) : prefill_fmt<float>(p, pl, dp, s);
}

}  // namespace ssm
