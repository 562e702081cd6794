// The kernels over the plan of attn_prefill.h: the items, and the join of cut tiles. One source file per
// padded width instantiates them.
#pragma once
#include <utility>

#include "attn_prefill.h"

namespace ssm {

// ---------------------------------------------------------------- the main kernel
// Float32 products on the bf16 matrix cores: a value is the sum of three bf16 (8 bits each, to nearest, the
// rest going on: the 24 bits of the value), and a product that of the six pairs that count. What is left out, two
// products of a middle and a low part, is below 2^-23 of |a b|, where the float32 sum of D products is good to
// D 2^-24; every product of parts is exact and summed in float32. Six MFMAs of 16 values take 192 cycles, the
// eight float32 ones that they stand for 512 (32 heads of 128, 8192 tokens: 2.7 ms, 4.1 by float32 MFMAs, 201 and
// 133 TF/s; three prompts of 2048 tokens in all, 16 heads of 112: 151 and 207 us with plan and join). An 8-bit
// cache's codes are one part, 3 products. Infinite values have no such parts: they give NaN. Wider heads than 128
// have no room for the parts in LDS and take the float32 MFMAs.
template <typename T, int FMT, int DP, int WAVES> struct PrefillShape {
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr bool SPLIT = !BF && DP <= 128;
    static constexpr int QP = SPLIT ? 3 : 1, KP = SPLIT && FMT == SSM_KV_ACT ? 3 : 1;   // parts of q and p, of k and v
    using S = std::conditional_t<BF || SPLIT, bf16, float>;                             // what LDS and the products hold
    static constexpr int TOK = BF ? 64 : 32, MT = TOK / 32, DT = DP / 32;
    static constexpr int PE = 16 / (int)sizeof(T);        // values per staged piece
    static constexpr int NP = DP / 32;                     // pieces of 16 bytes per lane, step and source
    // row strides in LDS: k rows 16 bytes apart modulo 256 (16 lanes read 16 rows), v rows 64 or 192
    // bytes (bf16: a half wave reads 4 rows of 64 bytes) or 32 bytes (float32) apart
    static constexpr int KS = DP + 16 / (int)sizeof(S);
    static constexpr int VS = sizeof(S) == 2 ? ((DP * 2) % 256 == 64 || (DP * 2) % 256 == 192 ? DP : DP + 32) : DP + 8;
    // workgroups of a compute unit, by registers and LDS (tile_places; float32 heads of 96, 24 of them, 8192 tokens:
    // two 1.44 ms, one with registers to spare 1.67)
    static constexpr int PER_CU = BF ? (DP <= 128 && WAVES == 4 ? 2 : 1) : (DP <= 96 ? 2 : 1);
};
// The next part of two values, which are left with what goes on: two bf16 of a word
__device__ __forceinline__ uint32_t take_part(float (&r)[2]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const uint32_t w = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{r[0], r[1]}, bf16x2));
    r[0] -= __builtin_bit_cast(float, w << 16);
    r[1] -= __builtin_bit_cast(float, w & 0xffff0000u);
    return w;
}

constexpr float kLag = 8.0f;

// f(integral_constant<int, 0>), .., f(integral_constant<int, n - 1>): places in register arrays that are
// constants from the start
template <typename F, int... I> __device__ __forceinline__ void static_each(std::integer_sequence<int, I...>, F f) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int n, typename F> __device__ __forceinline__ void static_for(F f) { static_each(std::make_integer_sequence<int, n>{}, f); }

// f over a value of the lane and of its partner in the other half of the wave
template <typename F> __device__ __forceinline__ float over_halves(float x, F f) {
    const uint32_t v = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return f(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

template <typename T, int FMT, int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, (PrefillShape<T, FMT, DP, WAVES>::PER_CU * WAVES / 4))
void attn_prefill_kernel(AttnArgs p, AttnPlan plan) {
    using Sh = PrefillShape<T, FMT, DP, WAVES>;
    using S = typename Sh::S;
    using E = typename KvElem<T, FMT>::type;
    constexpr bool BF = Sh::BF, SPLIT = Sh::SPLIT, RUN = BF || SPLIT;
    constexpr int PER_CU = Sh::PER_CU, QP = Sh::QP, KP = Sh::KP;
    constexpr int TOK = Sh::TOK, MT = Sh::MT, DT = Sh::DT, PE = Sh::PE, NP = Sh::NP, KS = Sh::KS, VS = Sh::VS;
    constexpr int ROWS = 32 * WAVES;
    constexpr int GW = PE * (int)sizeof(E) / 4;            // 32-bit words of a piece in the cache
    __shared__ __align__(16) S s_k[2][KP * TOK * KS];
    __shared__ __align__(16) S s_v[2][KP * TOK * VS];
    __shared__ __align__(16) float s_ks[4][FMT == SSM_KV_ACT ? 4 : TOK], s_vs[4][FMT == SSM_KV_ACT ? 4 : TOK];
    __shared__ int s_bad;

    const KvArgs& a = p.kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, col = lane & 31;
    const int it = (int)blockIdx.x / a.Hkv, head = (int)blockIdx.x % a.Hkv;
    const AttnItem item = plan.items[it];
    if (item.part == -2) return;
    const struct { int lo, m, n; } sq = {item.lo, item.m, item.n};
    const int g = a.Hq / a.Hkv, n = sq.n, before = sq.n - sq.m;
    // the first token that a row of the tile sees, and the step that the item begins with: not one wholly before it
    const int front = __builtin_amdgcn_readfirstlane(a.window > 0 ? max(before + item.row0 / g - a.window + 1, 0) : 0);
    const int k0 = item.k0 + (max(front - item.k0, 0) & ~(TOK - 1));
    const int32_t* table = a.table + (int64_t)item.seq * a.max_pages;

    if (tid == 0) s_bad = 0;
    __syncthreads();

    // this lane's query
    const int row = item.row0 + wave * 32 + col;
    const bool on = row < sq.m * g;
    const int tok = (on ? row : item.row0) / g, hq = head * g + (on ? row : item.row0) % g;
    const int pos = on ? before + tok : -1;
    const int row_w = item.row0 + wave * 32;              // the wave's first and last position
    const bool wave_on = row_w < sq.m * g;
    const int pos_lo = before + (wave_on ? row_w : item.row0) / g;
    const int pos_hi = before + min(row_w + 31, sq.m * g - 1) / g;
    constexpr int QN = RUN ? DP / 16 : DP / 8;             // q operands: 8 values per lane per 16 dims, 4 per 8
    S q[QN][QP][RUN ? 8 : 4];
    {
        const T* qp = (const T*)p.q + (int64_t)(sq.lo + tok) * p.ld_q + (int64_t)hq * a.D;
#pragma unroll
        for (int s = 0; s < QN; ++s) {
            const int d = RUN ? s * 16 + half * 8 : s * 8 + half * 4;
            T x[RUN ? 8 : 4];
            if (on && d < a.D) {
                load16(qp + d, x);
            } else {
#pragma unroll
                for (int e = 0; e < (RUN ? 8 : 4); ++e) x[e] = from_f32<T>(0.0f);
            }
            if constexpr (SPLIT) {
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    float y[2] = {x[2 * h], x[2 * h + 1]};
#pragma unroll
                    for (int k = 0; k < QP; ++k) {
                        const uint32_t w = take_part(y);
                        __builtin_memcpy(&q[s][k][2 * h], &w, 4);
                    }
                }
            } else {
                __builtin_memcpy(q[s][0], x, sizeof x);
            }
        }
    }

    // Staging: a wave brings the step's tokens of one block of 16 (two waves share a block of a float32
    // step), which lie on one page, through buffer resources that end behind the sequence's last token:
    // what is not there reads as zero, and a lane's offsets never change. Of 8 waves four bring k and four
    // v (one source each), of 4 waves each brings both. k is staged one step ahead of v (below).
    constexpr bool PINGPONG = WAVES == 8;
    static_assert(WAVES == 4 || (PINGPONG && BF), "four waves, or eight of bf16");
    constexpr int NB = PINGPONG ? 1 : 2;                   // sources of a wave: 0 (k, or v in the second half), 1 (v)
    constexpr int PR = DP / PE;                            // pieces per row
    const int blk = BF ? wave & 3 : wave >> 1;             // the wave's block of the step
    const bool second = PINGPONG && wave >= 4;             // the half of the workgroup that brings v
    uint32_t off[NP];                                      // byte offset of piece i in its block
    int at[NB][NP];                                        // its place in a buffer
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int pc = ((BF ? 0 : (wave & 1) * NP) + i) * 64 + lane, t = pc / PR, d = (pc % PR) * PE;
        off[i] = d < a.D ? (uint32_t)((t * a.D + d) * (int)sizeof(E)) : kOffOutOfRange;
        at[0][i] = (16 * blk + t) * (second ? VS : KS) + d;
        if constexpr (NB == 2) at[1][i] = (16 * blk + t) * VS + d;
    }
    uint32_t held[NB][NP][GW];                             // pieces on their way
    uint32_t held_ks = 0, held_vs = 0;
    const char* src[NB];
    src[0] = (const char*)(second ? a.v : a.k);
    if constexpr (NB == 2) src[1] = (const char*)a.v;
    __amdgpu_buffer_rsrc_t from[NB], from_ks, from_vs;
    auto page_at = [&](int step) {                         // the table entry of the wave's block
        return table[max(min(k0 + step * TOK + 16 * blk, n - 1), 0) >> a.page_log2];
    };
    // a page is page_bytes long, the head's part of it begins at head_bytes (both below 2^30)
    const uint32_t row_bytes = (uint32_t)(a.D * (int)sizeof(E)), page_mask = (1u << a.page_log2) - 1;
    const uint32_t head_row = (uint32_t)head << a.page_log2, page_rows = (uint32_t)a.Hkv << a.page_log2;
    const uint32_t head_bytes = head_row * row_bytes, page_bytes = page_rows * row_bytes;
    auto locate = [&](auto b, int step, int page) {         // where the block's tokens of source b are
        const int pg = __builtin_amdgcn_readfirstlane(page), j = k0 + step * TOK + 16 * blk;
        const bool there = (uint32_t)pg < (uint32_t)a.num_pages && j < n;
        const uint32_t tokens = there ? (uint32_t)min(n - j, 16) : 0u, in_page = (uint32_t)j & page_mask;
        const uint32_t page0 = there ? (uint32_t)pg : 0u;
        const uint64_t o = (uint64_t)page0 * page_bytes + (head_bytes + in_page * row_bytes);
        from[b] = buffer_rsrc(src[b] + o, tokens * row_bytes);
        if constexpr (FMT != SSM_KV_ACT) {
            if constexpr (b == 0) {
                const uint64_t r = (uint64_t)page0 * page_rows + (head_row + in_page);
                from_ks = buffer_rsrc(a.ks + r, 4 * tokens);
                from_vs = buffer_rsrc(a.vs + r, 4 * tokens);
            }
        }
    };
    auto load_piece = [&](auto b, auto i) {
        uint32_t (&x)[GW] = held[b][i];
        if constexpr (GW == 4) {
            const u32x4 w = buffer_load16(from[b], off[i]);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = w[e];
        } else if constexpr (GW == 2) {
            const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(from[b], (int)off[i], 0, 0);
            x[0] = w[0];
            x[1] = w[1];
        } else {
            x[0] = __builtin_amdgcn_raw_buffer_load_b32(from[b], (int)off[i], 0, 0);
        }
    };
    // Lanes 0 .. 15 of the waves that bring k bring the block's scales, of k and of v
    auto load_scales = [&] {
        if constexpr (FMT != SSM_KV_ACT) {
            const uint32_t so = lane < 16 && !second ? 4 * lane : kOffOutOfRange;
            held_ks = __builtin_amdgcn_raw_buffer_load_b32(from_ks, (int)so, 0, 0);
            held_vs = __builtin_amdgcn_raw_buffer_load_b32(from_vs, (int)so, 0, 0);
        }
    };
    auto load_all = [&](auto b, int step) {
        locate(b, step, page_at(step));
        static_for<NP>([&](auto i) { load_piece(b, i); });
        if constexpr (b == 0) load_scales();
    };
    constexpr int kTurns = KP == 3 ? 4 : 1;                // that a piece is staged in
    float rest[2];
    u32x2 parts[KP];
    auto stage_piece = [&](auto b, int step, auto i, auto turn) {
        const uint32_t (&w)[GW] = held[b][i];
        S* to = (b == 1 || second ? &s_v[step & 1][0] : &s_k[step & 1][0]) + at[b][i];
        if constexpr (SPLIT && FMT == SSM_KV_ACT) {   // four values in 4 turns: a pair's first part, then its others
            constexpr int pair = turn / 2, at0 = 2 * pair;
            static_assert(KP == 3 && kTurns == 4);
            if constexpr (turn % 2 == 0) {
                rest[0] = __builtin_bit_cast(float, w[at0]);
                rest[1] = __builtin_bit_cast(float, w[at0 + 1]);
                parts[0][pair] = take_part(rest);
            } else {
                parts[1][pair] = take_part(rest);
                parts[2][pair] = take_part(rest);
            }
            if constexpr (turn == kTurns - 1) {
#pragma unroll
                for (int k = 0; k < KP; ++k) *(u32x2*)(to + k * TOK * (b == 1 ? VS : KS)) = parts[k];
            }
            return;
        }
        if constexpr (SPLIT && FMT != SSM_KV_ACT) {
            *(u32x2*)to = kv_decode4_bf16<FMT>(w[0]);
            return;
        }
        u32x4 x;                                           // 16 bytes of T
        if constexpr (FMT == SSM_KV_ACT) {
            x = u32x4{w[0], w[1], w[2], w[3]};
        } else if constexpr (BF) {   // codes are exact in bf16; their scales wait for the scores
            const u32x2 lo = kv_decode4_bf16<FMT>(w[0]), hi = kv_decode4_bf16<FMT>(w[GW - 1]);
            x = u32x4{lo[0], lo[1], hi[0], hi[1]};
        } else {
            float f[4];
            kv_decode4<FMT>(w[0], f);
            __builtin_memcpy(&x, f, 16);
        }
        *(u32x4*)to = x;
    };
    // Tokens of step 0 before `front` are seen by no row, and what the cache holds there must not reach the product with
    // v (0 * infinity): its values and scales become zeros. Scores of such tokens are masked one by one.
    auto clear_front = [&](auto b) {
        if (front <= k0) return;
        const int gone = front - k0 - 16 * blk;            // leading tokens of the wave's block
        if (b == 1 || second) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int t = (((BF ? 0 : (wave & 1) * NP) + i) * 64 + lane) / PR;
#pragma unroll
                for (int e = 0; e < GW; ++e) held[b][i][e] = t < gone ? 0u : held[b][i][e];
            }
        }
        if constexpr (FMT != SSM_KV_ACT && b == 0) held_vs = lane < gone ? 0u : held_vs;
    };
    auto stage_scales = [&](int step) {
        if constexpr (FMT != SSM_KV_ACT) {
            if (lane < 16 && !second) {
                s_ks[step & 3][16 * blk + lane] = __builtin_bit_cast(float, held_ks);
                s_vs[step & 3][16 * blk + lane] = __builtin_bit_cast(float, held_vs);
            }
        }
    };
    auto stage_all = [&](auto b, int step) {
        static_for<NP * kTurns>([&](auto i) {
            stage_piece(b, step, std::integral_constant<int, i / kTurns>{}, std::integral_constant<int, i % kTurns>{});
        });
        if constexpr (b == 0) stage_scales(step);
    };
    constexpr std::integral_constant<int, 0> b0{};
    constexpr std::integral_constant<int, NB - 1> b1{};

    // pages that the table does not name: their tokens are masked one by one (below)
    auto check_pages = [&] {
        for (int i = (max(k0, front) >> a.page_log2) + tid; i <= ((min(item.k1, n) - 1) >> a.page_log2); i += 64 * WAVES) {
            const int pg = table[i];
            if (pg < 0 || pg >= a.num_pages) {
                s_bad = 1;
                atomicOr(a.status, SSM_STATUS_BAD_PAGE);
            }
        }
    };

    const float c2 = a.scale * kLog2e;
    float m = -3.0e38f, l = 0.0f;   // finite, so that differences are numbers before any token is seen
    f32x16 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;

    f32x16 s[MT];                                          // the step's scores, then its probabilities
    bf16x8 pf[QP][RUN ? TOK / 16 : 1];                     // and those as the operand of the product with v
    auto seen = [&](int tb) {
        return wave_on && tb <= pos_hi && (a.window <= 0 || tb + TOK - 1 > pos_lo - a.window);
    };
    bool bad = false;
    auto scale_scores = [&](f32x16 (&s)[MT], int step) {
        if constexpr (FMT != SSM_KV_ACT) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const f32x4 sc = *(const f32x4*)&s_ks[step & 3][t * 32 + 8 * w + 4 * half];
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[t][4 * w + e] *= sc[e];
                    if (w == 3) __builtin_amdgcn_sched_barrier(0);
                }
        }
    };
    auto mask_scores = [&](f32x16 (&s)[MT], int tb) {
        const bool edge = tb + TOK - 1 > pos_lo || (a.window > 0 && tb <= pos_hi - a.window);
        if (edge) {   // the token of s[t][r] is a constant behind tb + 4 half
            const int last = pos - tb - 4 * half, first = a.window > 0 ? last - a.window : -1;
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int j = t * 32 + 8 * (r >> 2) + (r & 3);
                    s[t][r] = j <= last && j > first ? s[t][r] : -__builtin_inff();
                }
        }
        if (bad) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int j = tb + t * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
                    const int pg = j < n ? table[j >> a.page_log2] : -1;
                    s[t][r] = pg >= 0 && pg < a.num_pages ? s[t][r] : -__builtin_inff();
                }
        }
    };
    // Empty statements that have the sums in the same registers on both ways of the branch below, a wave that is
    // alone on its SIMD in the matrix cores' own (the branch then moves them out and back): without them the
    // compiler copies four tiles of them in every step, and spills with 8-bit caches
    constexpr bool ALONE = RUN && DP <= 128 && PER_CU * WAVES == 4;
    auto keep_sums = [&] {
        if constexpr (RUN && DP <= 128) {
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                if constexpr (ALONE) asm volatile("" : "+a"(o[t]));
                else asm volatile("" : "+v"(o[t]));
            }
        }
    };
    auto follow_max = [&](float mx) {                      // mx: of the lane's scores
        mx = over_halves(mx, [](float x, float y) { return fmaxf(x, y); });
        const float mn = fmaxf(m, mx * c2);
        // The sums are kept relative to m, which need not be the maximum itself: it follows once the
        // maximum is kLag powers of two above it (then no p is above 2^kLag, and no digit is lost)
        if constexpr (ALONE) keep_sums();
        if (__any(mn > m + kLag)) {
            const float al = fast_exp2(m - mn);
            l *= al;
#pragma unroll
            for (int t = 0; t < DT; ++t) o[t] *= al;
            if constexpr (ALONE) keep_sums();
            m = mn;
        }
        keep_sums();
    };
    auto soften = [&](int tb, int step) {
        scale_scores(s, step);
        mask_scores(s, tb);
        float mx = s[0][0];
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[t][r]);
        follow_max(mx);
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[t][r] = fast_exp2(__builtin_fmaf(s[t][r], c2, -m));
                if constexpr (!BF || FMT != SSM_KV_ACT) l += s[t][r];
            }
        if constexpr (FMT != SSM_KV_ACT) {
            __builtin_amdgcn_sched_barrier(0);   // (the scales are read when the scores' registers are free)
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const f32x4 sc = *(const f32x4*)&s_vs[step & 3][t * 32 + 8 * w + 4 * half];
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[t][4 * w + e] *= sc[e];
                }
        }
        if constexpr (BF) {
            // The probabilities enter the product in bf16, up to half a step (2^-8 of the value)
            // off each, as v itself is stored. Their sum l is of the rounded ones where no scale of v is in them: two to an
            // instruction, in float32, and the weights p / l add up to one.
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            const bf16x2 one = {(bf16)1.0f, (bf16)1.0f};
            float ls[2] = {0.0f, 0.0f};
#pragma unroll
            for (int ks = 0; ks < TOK / 16; ++ks) {
#pragma unroll
                for (int e = 0; e < 8; ++e) pf[0][ks][e] = (bf16)s[ks >> 1][8 * (ks & 1) + e];
                if constexpr (FMT == SSM_KV_ACT) {
#pragma unroll
                    for (int e = 0; e < 8; e += 2)
                        ls[ks & 1] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pf[0][ks][e], pf[0][ks][e + 1]}, one, ls[ks & 1], false);
                }
            }
            if constexpr (FMT == SSM_KV_ACT) l += ls[0] + ls[1];
        }
    };
    const int steps = (item.k1 - k0 + TOK - 1) / TOK;
    if constexpr (RUN) {
        // The products of step i are one run of MFMAs, K(i) Q and then V(i-1) P(i-1), each fragment read
        // from LDS kLead MFMAs ahead of its own (a wave alone: 69 cycles per MFMA as the compiler orders it,
        // 41 so; the MFMA takes 32). Meanwhile K(i+1) and V(i) go from registers to LDS and the loads of the
        // step behind them start, one piece to an MFMA. The run never branches: P is zero where a step is
        // not seen or not there, and its scores are not used.
        //
        // Eight waves: two share a SIMD, one of each half of the workgroup, and while one half is in its
        // products the other is in its softmax, half a step behind. In phase 2 i the first half has the
        // products of step i and stages K(i+1), the second has softmax i - 1; in phase 2 i + 1 the second half
        // has the products of step i and stages V(i), the first has softmax i. K(i) is read in phases
        // 2 i - 1 (its first fragments) to 2 i + 1, V(i) in 2 i + 2 and 2 i + 3: two buffers of each do. The
        // scales of step i + 1 come with K(i+1) in phase 2 i and are read in 2 i + 3 and 2 i + 4, when those of
        // the step behind it are there already: three buffers, taken as four.
        // Four waves, where two halves of 8 would not have registers enough or few rows would leave most of
        // them without work: one barrier per step, and the other workgroup of the compute unit (up to 128
        // values per head) fills the softmax.
        //
        // Float32: the parts of a fragment of k or v one after the other, each for the parts of q or p that it is
        // paired with. One wave on each SIMD, whose softmax i - 1 is dealt out over the products K(i) Q, in front
        // of V(i-1) P(i-1) that needs it.
        constexpr int MF = KP == 3 ? 6 : QP;               // MFMAs of a fragment's parts
        constexpr int FK = QN * MT * KP, F = FK + DT * (TOK / 16) * KP;   // fragments of k; and of v
        constexpr int NK = FK / KP * MF, N = F / KP * MF, NV = N - NK;
        constexpr int kAfter = SPLIT ? MF * 3 / KP : 0;    // MFMAs of the last kLead fragments
        constexpr int kLead = SPLIT ? 3 : 4, kSlots = NB * (NP * kTurns + NP + 1) + 1, kSoft = 37;
        static_assert(BF || F % (kLead + 1) == 0, "a step's first fragments follow the last ones");
        static_assert(BF ? N >= kSlots : NV > kAfter, "the run is long enough for what it brings");
        const int lead = second ? 0 : 1;                   // source 0 is staged for step i + lead
        for (int i = tid; i < KP * TOK * VS * 2 / 16; i += 64 * WAVES) ((u32x4*)&s_v[1][0])[i] = u32x4{0, 0, 0, 0};   // V(-1)
        if constexpr (SPLIT && FMT != SSM_KV_ACT) {
            if (tid < TOK) s_vs[3][tid] = 0.0f;            // and its scales
        }
        auto no_probabilities = [&] {
#pragma unroll
            for (int k = 0; k < QP; ++k)
#pragma unroll
                for (int ks = 0; ks < TOK / 16; ++ks) pf[k][ks] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
        };
        no_probabilities();
        int page[NB];
        load_all(b0, 0);
        clear_front(b0);
        if constexpr (NB == 2) {
            load_all(b1, 0);
            clear_front(b1);
            page[1] = page_at(1);
        }
        if (!second) {
            page[0] = page_at(1);
            stage_all(b0, 0);
            locate(b0, 1, page[0]);
            static_for<NP>([&](auto i) { load_piece(b0, i); });
            load_scales();
        }
        page[0] = page_at(1 + lead);
        check_pages();

        const S* v_at = &s_v[0][(4 * half + ((lane & 15) >> 2)) * VS + ((lane >> 4) & 1) * 16 + (lane & 3) * 4];
        const S* k_at = &s_k[0][col * KS + half * 8];
        bf16x8 fr[kLead + 1];
        auto read = [&](auto f, int i) {
            constexpr int part = f % KP;
            if constexpr (f < FK) {
                constexpr int x = f / KP;
                fr[f % (kLead + 1)] = *(const bf16x8*)(k_at + ((i & 1) * KP + part) * TOK * KS + (x % MT) * 32 * KS + (x / MT) * 16);
            } else {
                typedef short s16x4 __attribute__((ext_vector_type(4)));
                typedef __attribute__((address_space(3))) s16x4* lds4;
                constexpr int x = (f - FK) / KP;
                const S* q = v_at + (((i - 1) & 1) * KP + part) * TOK * VS + (x / DT) * 16 * VS + (x % DT) * 32;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)q);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(q + 8 * VS));
                fr[f % (kLead + 1)] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        };
        auto read_first = [&](int i) { static_for<kLead>([&](auto f) { read(f, i); }); };
        auto bring = [&](auto slot, int i) {               // slot of kSlots: stage, then locate and load by source
            if constexpr (slot < NB * NP * kTurns) {
                constexpr int piece = slot / kTurns;
                constexpr std::integral_constant<int, piece / NP> b{};
                stage_piece(b, i + (b == 0 ? lead : 0), std::integral_constant<int, piece % NP>{}, std::integral_constant<int, slot % kTurns>{});
            } else {
                constexpr int r = slot - NB * NP * kTurns, x = r % (NP + 1);
                constexpr std::integral_constant<int, r / (NP + 1)> b{};
                if constexpr (r == 0) stage_scales(i + lead);
                if constexpr (b < NB) {
                    const int step = i + 1 + (b == 0 ? lead : 0);
                    if constexpr (x == 0) locate(b, step, page[b]);
                    else load_piece(b, std::integral_constant<int, x - 1>{});
                    if constexpr (x == NP) page[b] = page_at(step + 1);
                } else {
                    load_scales();
                }
            }
        };
        // A turn of float32's softmax: scales, masks, maximum, then the probabilities by pairs, each value, a first
        // part and the others in a turn of their own: six instructions fit beside an MFMA
        f32x4 sc_v;
        float rest_p[2], top = 0.0f;
        auto put = [](bf16x8& x, int word, uint32_t v) {
            u32x4 y = __builtin_bit_cast(u32x4, x);
            y[word] = v;
            x = __builtin_bit_cast(bf16x8, y);
        };
        auto soften_turn = [&](f32x16 (&s)[MT], auto k, int i) {
            const int tb = k0 + i * TOK;
            if constexpr (k == 0) {
                scale_scores(s, i);
            } else if constexpr (k == 1) {
                if (i >= 0 && i < steps && seen(tb)) {
                    mask_scores(s, tb);
                } else {
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[0][r] = -__builtin_inff();
                }
            } else if constexpr (k == 2 || k == 3) {
                if constexpr (k == 2) top = s[0][0];
#pragma unroll
                for (int r = 8 * (k - 2); r < 8 * (k - 1); ++r) top = fmaxf(top, s[0][r]);
            } else if constexpr (k == 4) {
                if constexpr (FMT != SSM_KV_ACT) sc_v = *(const f32x4*)&s_vs[i & 3][4 * half];
                follow_max(top);
            } else {
                constexpr int w = (k - 5) / 4, ks = w / 4, turn = (k - 5) % 4;
                if constexpr (turn < 2) {
                    float y = fast_exp2(__builtin_fmaf(s[0][2 * w + turn], c2, -m));
                    l += y;
                    if constexpr (FMT != SSM_KV_ACT) y *= sc_v[(2 * w + turn) & 3];
                    rest_p[turn] = y;
                    if constexpr (FMT != SSM_KV_ACT && turn == 1 && w % 2 == 1 && w < 7)
                        sc_v = *(const f32x4*)&s_vs[i & 3][8 * (w / 2 + 1) + 4 * half];
                } else if constexpr (turn == 2) {
                    put(pf[0][ks], w % 4, take_part(rest_p));
                } else {
                    put(pf[1][ks], w % 4, take_part(rest_p));
                    put(pf[2][ks], w % 4, take_part(rest_p));
                }
            }
        };
        // K(i) Q into sk; sp: the scores of step i - 1 (float32)
        auto products = [&](int i, f32x16 (&sk)[MT], f32x16 (&sp)[MT]) {
            if constexpr (BF) __builtin_amdgcn_s_setprio(1);
            static_for<F>([&](auto f) {
                if constexpr (SPLIT && f + kLead == F) __syncthreads();   // all of the step is read, all of the next one there
                if constexpr (f + kLead < F) read(std::integral_constant<int, f + kLead>{}, i);
                else if constexpr (SPLIT) read(std::integral_constant<int, f + kLead - F>{}, i + 1);
                constexpr int part = f % KP, first = f / KP * MF + (part == 0 ? 0 : part == 1 ? QP : 2 * QP - 1);
                static_for<(KP == 3 ? QP - part : QP)>([&](auto x) {   // the parts of q or p
                    constexpr int at = first + x;          // this MFMA's place in the run
                    if constexpr (f < FK) {
                        constexpr int t = f / KP % MT;
                        if constexpr (f / KP / MT == 0 && part == 0 && x == 0) {
#pragma unroll
                            for (int r = 0; r < 16; ++r) sk[t][r] = 0.0f;
                        }
                        sk[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[f % (kLead + 1)], __builtin_bit_cast(bf16x8, q[f / KP / MT][x]), sk[t], 0, 0, 0);
                    } else {
                        constexpr int t = (f - FK) / KP % DT;
                        o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[f % (kLead + 1)], pf[x][(f - FK) / KP / DT], o[t], 0, 0, 0);
                    }
                    if constexpr (SPLIT) {
                        static_for<kSoft>([&](auto k) {
                            if constexpr (k * NK / kSoft == at) soften_turn(sp, k, i - 1);
                        });
                    }
                    static_for<kSlots>([&](auto slot) {
                        if constexpr ((BF ? N - kSlots + slot : NK + slot * (NV - kAfter) / kSlots) == at) bring(slot, i);
                    });
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
            if constexpr (BF) __builtin_amdgcn_s_setprio(0);
            if constexpr (ALONE) keep_sums();
        };
        auto softmax = [&](int i) {
            if (i < steps && seen(k0 + i * TOK)) soften(k0 + i * TOK, i);
            else no_probabilities();
        };
        __syncthreads();
        bad = s_bad != 0;
        if (!wave_on) {                                    // no rows: what the wave brings, and the barriers
            if (second) __syncthreads();
            for (int i = 0; i <= steps; ++i) {
                static_for<kSlots>([&](auto slot) { bring(slot, i); });
                __syncthreads();
                if constexpr (PINGPONG) {
                    if (!second || i < steps) __syncthreads();
                }
            }
            return;
        }
        read_first(0);
        if constexpr (SPLIT) {
            f32x16 next[MT];
            int i = 0;
            for (; i < steps; i += 2) {
                products(i, next, s);
                products(i + 1, s, next);
            }
            if (i == steps) products(i, next, s);
        } else {
            if (second) __syncthreads();
            for (int i = 0; i <= steps; ++i) {
                products(i, s, s);
                if constexpr (PINGPONG) __syncthreads();
                softmax(i);
                if constexpr (PINGPONG) {
                    read_first(i + 1);
                    if (!second || i < steps) __syncthreads();
                } else {
                    __syncthreads();
                    read_first(i + 1);
                }
            }
        }
    } else {
        load_all(b0, 0);
        load_all(b1, 0);
        check_pages();
        clear_front(b0);
        stage_all(b0, 0);
        stage_all(b1, 0);
        if (front > k0) {                                  // as clear_front(b1), by what the lane staged
#pragma unroll 1
            for (int i = 0; i < NP; ++i) {
                const int pc = ((wave & 1) * NP + i) * 64 + lane, t = 16 * blk + pc / PR;
                if (k0 + t < front) *(u32x4*)&s_v[0][t * VS + (pc % PR) * PE] = u32x4{0, 0, 0, 0};
            }
        }
        __syncthreads();
        bad = s_bad != 0;
        for (int i = 0; i < steps; ++i) {
            const int tb = k0 + i * TOK;
            if (i + 1 < steps) {
                load_all(b0, i + 1);
                load_all(b1, i + 1);
            }
            if (seen(tb)) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[0][r] = 0.0f;
#pragma unroll
                for (int k = 0; k < QN; ++k) {
                    if (k * 8 >= a.D) break;
                    const f32x4 kf = *(const f32x4*)&s_k[i & 1][col * KS + k * 8 + half * 4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], q[k][0][e], s[0], 0, 0, 0);
                }
                soften(tb, i);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const S* vp = &s_v[i & 1][(8 * (r >> 2) + 4 * half + (r & 3)) * VS + col];
#pragma unroll
                    for (int t = 0; t < DT; ++t) o[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(vp[t * 32], s[0][r], o[t], 0, 0, 0);
                }
            }
            if (i + 1 < steps) {
                stage_all(b0, i + 1);
                stage_all(b1, i + 1);
            }
            __syncthreads();
        }
    }

    l = over_halves(l, [](float x, float y) { return x + y; });
    if (item.part < 0) {
        if (!on) return;
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;   // nothing visible: zeros
        T* out = (T*)p.o + (int64_t)(sq.lo + tok) * p.ld_o + (int64_t)hq * a.D;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int d = t * 32 + 8 * w + 4 * half;
                if (d < a.D) {
                    T y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = from_f32<T>(o[t][4 * w + e] * inv);
                    __builtin_memcpy(__builtin_assume_aligned(out + d, 4 * sizeof(T)), y, sizeof y);
                }
            }
    } else if (wave_on) {
        float* part = plan.parts + ((int64_t)head * plan.max_parts + item.part) * ROWS * (DP + 2);
        const int r0 = wave * 32 + col;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int w = 0; w < 4; ++w)
                *(float4*)(part + (int64_t)r0 * DP + t * 32 + 8 * w + 4 * half) =
                    make_float4(o[t][4 * w], o[t][4 * w + 1], o[t][4 * w + 2], o[t][4 * w + 3]);
        if (half == 0) {
            part[ROWS * DP + r0] = m;
            part[ROWS * (DP + 1) + r0] = l;
        }
    }
}

// The partial results of cut tiles, in order: four rows of a (tile, kv head) per workgroup and turn, one to
// a wave, two partials on their way (5 partials of 8000 rows, 32 of 1056: 7.7 and 7.1 us; four 9.2 and 6.5, eight
// 12.3 and 6.5)
constexpr int kJoinWorkgroups = 2048;
template <typename T, int DP, int ROWS> __global__ __launch_bounds__(256) void attn_prefill_join_kernel(AttnArgs p, AttnPlan plan) {
    const KvArgs& a = p.kv;
    constexpr int64_t stride = (int64_t)ROWS * (DP + 2);
    constexpr int turns = ROWS / 4;
    const int g = a.Hq / a.Hkv, total = plan.count[0] * a.Hkv * turns;
    for (int i = (int)blockIdx.x; i < total; i += (int)gridDim.x) {
        const int r = (i % turns) * 4 + (threadIdx.x >> 6), head = i / turns % a.Hkv;
        const AttnJoin jn = plan.joins[i / turns / a.Hkv];
        const int row = jn.row0 + r;
        if (row >= jn.m * g) continue;
        const float* part = plan.parts + ((int64_t)head * plan.max_parts + jn.part) * stride;
        join_row<T, 2>(jn.pieces, [&](int v) { return part + v * stride; }, (int64_t)r * DP, ROWS * DP + r, ROWS * (DP + 1) + r, a.D,
                    (T*)p.o + (int64_t)(jn.lo + row / g) * p.ld_o + (int64_t)(head * g + row % g) * a.D);
    }
}

template <typename T, int FMT, int DP, int WAVES> hipError_t launch_attn_prefill_waves(const AttnArgs& p, const AttnPlan& pl, hipStream_t s) {
    KernelTimer kt("attn.prefill", s);
    SSM_LAUNCH((attn_prefill_kernel<T, FMT, DP, WAVES>), dim3((unsigned)pl.max_items * p.kv.Hkv), dim3(64 * WAVES), 0, s, p, pl);
    hipError_t e = hipGetLastError();
    const int64_t longest = (int64_t)p.kv.max_pages << p.kv.page_log2;
    if (e != hipSuccess || longest <= pl.min_steps * kStep) return e;   // no tile is ever cut
    KernelTimer kj("attn.prefill_join", s);
    const int64_t most = (int64_t)pl.max_joins * p.kv.Hkv * (8 * WAVES);
    SSM_LAUNCH((attn_prefill_join_kernel<T, DP, 32 * WAVES>), dim3((unsigned)(most < kJoinWorkgroups ? most : kJoinWorkgroups)), dim3(256),
               0, s, p, pl);
    return hipGetLastError();
}
template <typename T, int FMT, int DP>
hipError_t launch_attn_prefill_tile(const AttnArgs& p, const AttnPlan& pl, hipStream_t s) {
    if constexpr (sizeof(T) == 2 && DP == 128) {
        if (pl.rows == 256) return launch_attn_prefill_waves<T, FMT, DP, 8>(p, pl, s);
    }
    return launch_attn_prefill_waves<T, FMT, DP, 4>(p, pl, s);
}

// the instances of one padded width, one file each
#define SSM_ATTN_PREFILL_BF16(DP)                                                                             \
    template hipError_t launch_attn_prefill_tile<bf16, SSM_KV_ACT, DP>(const AttnArgs&, const AttnPlan&, hipStream_t);      \
    template hipError_t launch_attn_prefill_tile<bf16, SSM_KV_FP8_E4M3, DP>(const AttnArgs&, const AttnPlan&, hipStream_t); \
    template hipError_t launch_attn_prefill_tile<bf16, SSM_KV_INT8, DP>(const AttnArgs&, const AttnPlan&, hipStream_t);
#define SSM_ATTN_PREFILL_F32(DP)                                                                              \
    template hipError_t launch_attn_prefill_tile<float, SSM_KV_ACT, DP>(const AttnArgs&, const AttnPlan&, hipStream_t);      \
    template hipError_t launch_attn_prefill_tile<float, SSM_KV_FP8_E4M3, DP>(const AttnArgs&, const AttnPlan&, hipStream_t); \
    template hipError_t launch_attn_prefill_tile<float, SSM_KV_INT8, DP>(const AttnArgs&, const AttnPlan&, hipStream_t);

}  // namespace ssm
