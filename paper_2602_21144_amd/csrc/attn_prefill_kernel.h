// The kernels over the plan of attn_prefill.h: the items, and the join of cut tiles. One source file per
// padded width instantiates them.
#pragma once
#include "attn_prefill.h"

namespace ssm {

// ---------------------------------------------------------------- the main kernel
template <typename T, int DP, int WAVES> struct PrefillShape {
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int TOK = BF ? 64 : 32, MT = TOK / 32, DT = DP / 32;
    static constexpr int PE = 16 / (int)sizeof(T);        // values per staged piece
    static constexpr int NP = DP / 32;                     // pieces of 1 KB per wave and step, of k and of v (8 waves: of one)
    // row strides in LDS: k rows 16 bytes apart modulo 256 (16 lanes read 16 rows), v rows 64 or 192
    // bytes (bf16: a half wave reads 4 rows of 64 bytes) or 32 bytes (float32) apart
    static constexpr int KS = DP + PE;
    static constexpr int VS = BF ? ((DP * 2) % 256 == 64 || (DP * 2) % 256 == 192 ? DP : DP + 32) : DP + 8;
};

constexpr float kLag = 8.0f;

// f over a value of the lane and of its partner in the other half of the wave
template <typename F> __device__ __forceinline__ float over_halves(float x, F f) {
    const uint32_t v = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return f(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

template <typename T, int FMT, int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, (sizeof(T) == 2 && DP <= 128 ? 2 : 1))
void attn_prefill_kernel(AttnArgs p, AttnPlan plan) {
    using Sh = PrefillShape<T, DP, WAVES>;
    using E = typename KvElem<T, FMT>::type;
    constexpr bool BF = Sh::BF;
    constexpr int TOK = Sh::TOK, MT = Sh::MT, DT = Sh::DT, PE = Sh::PE, NP = Sh::NP, KS = Sh::KS, VS = Sh::VS;
    constexpr int ROWS = 32 * WAVES;
    constexpr int GW = PE * (int)sizeof(E) / 4;            // 32-bit words of a piece in the cache
    __shared__ __align__(16) T s_k[2][TOK * KS];
    __shared__ __align__(16) T s_v[2][TOK * VS];
    __shared__ __align__(16) float s_ks[4][FMT == SSM_KV_ACT ? 4 : TOK], s_vs[4][FMT == SSM_KV_ACT ? 4 : TOK];
    __shared__ int s_bad;

    const KvArgs& a = p.kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, col = lane & 31;
    const int it = (int)blockIdx.x / a.Hkv, head = (int)blockIdx.x % a.Hkv;
    if (it >= plan.count[0]) return;
    const AttnItem item = plan.items[it];
    const KvSeq sq = kv_seq(a, item.seq);
    const int g = a.Hq / a.Hkv, n = sq.n, before = sq.n - sq.m;
    const int32_t* table = a.table + (int64_t)item.seq * a.max_pages;

    if (tid == 0) s_bad = 0;
    __syncthreads();
    // pages that the table does not name: their tokens are masked one by one (below)
    for (int i = (item.k0 >> a.page_log2) + tid; i <= ((min(item.k1, n) - 1) >> a.page_log2); i += 64 * WAVES) {
        const int pg = table[i];
        if (pg < 0 || pg >= a.num_pages) {
            s_bad = 1;
            atomicOr(a.status, SSM_STATUS_BAD_PAGE);
        }
    }

    // this lane's query
    const int row = item.row0 + wave * 32 + col;
    const bool on = row < sq.m * g;
    const int tok = (on ? row : item.row0) / g, hq = head * g + (on ? row : item.row0) % g;
    const int pos = on ? before + tok : -1;
    const int row_w = item.row0 + wave * 32;              // the wave's first and last position
    const bool wave_on = row_w < sq.m * g;
    const int pos_lo = before + (wave_on ? row_w : item.row0) / g;
    const int pos_hi = before + min(row_w + 31, sq.m * g - 1) / g;
    constexpr int QN = BF ? DP / 16 : DP / 8;              // q operands: 8 values per lane per 16 dims, 4 per 8
    T q[QN][BF ? 8 : 4];
    {
        const T* qp = (const T*)p.q + (int64_t)(sq.lo + tok) * p.ld_q + (int64_t)hq * a.D;
#pragma unroll
        for (int s = 0; s < QN; ++s) {
            const int d = BF ? s * 16 + half * 8 : s * 8 + half * 4;
            if (on && d < a.D) {
                load16(qp + d, q[s]);
            } else {
#pragma unroll
                for (int e = 0; e < (BF ? 8 : 4); ++e) q[s][e] = from_f32<T>(0.0f);
            }
        }
    }

    // Staging: a wave brings the step's tokens of one block of 16 (two waves share a block of a float32
    // step; of 8 waves, four bring k and four v), which lie on one page, through a buffer resource that
    // ends behind the sequence's last token: what is not there reads as zero, and a lane's offsets never
    // change. The block's page is looked up one step before its loads are issued.
    constexpr int PR = DP / PE;                            // pieces per row
    constexpr bool SPLIT = WAVES == 8;
    static_assert(WAVES == 4 || (SPLIT && BF), "four waves, or eight of bf16");
    const int blk = BF ? wave & 3 : wave >> 1;             // the wave's block of the step
    const bool brings_v = SPLIT && __builtin_amdgcn_readfirstlane(wave) >= 4;
    uint32_t off[NP];                                      // byte offset of piece i in its block
    int at_k[NP], at_v[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int pc = ((BF ? 0 : (wave & 1) * NP) + i) * 64 + lane, t = pc / PR, d = (pc % PR) * PE;
        off[i] = d < a.D ? (uint32_t)((t * a.D + d) * (int)sizeof(E)) : kOffOutOfRange;
        at_k[i] = (16 * blk + t) * (brings_v ? VS : KS) + d;
        at_v[i] = (16 * blk + t) * VS + d;
    }
    uint32_t rk[NP][GW], rv[SPLIT ? 1 : NP][GW];           // SPLIT: rk holds what the wave brings
    uint32_t rks = 0, rvs = 0;
    auto page_at = [&](int tb) {                           // the table entry of the wave's block
        return table[max(min(tb + 16 * blk, n - 1), 0) >> a.page_log2];
    };
    // a page is page_bytes long, the head's part of it begins at head_bytes (both below 2^30)
    const uint32_t row_bytes = (uint32_t)(a.D * (int)sizeof(E)), page_mask = (1u << a.page_log2) - 1;
    const uint32_t head_row = (uint32_t)head << a.page_log2, page_rows = (uint32_t)a.Hkv << a.page_log2;
    const uint32_t head_bytes = head_row * row_bytes, page_bytes = page_rows * row_bytes;
    const char* src = (const char*)(brings_v ? a.v : a.k);
    // where the block's tokens are: the descriptor of what the wave brings
    __amdgpu_buffer_rsrc_t from, from_v, from_s, from_vs;
    auto locate = [&](int tb, int page) {
        const int pg = __builtin_amdgcn_readfirstlane(page), j = tb + 16 * blk;
        const bool there = (uint32_t)pg < (uint32_t)a.num_pages && j < n;
        const uint32_t tokens = there ? (uint32_t)min(n - j, 16) : 0u, in_page = (uint32_t)j & page_mask;
        const uint32_t page_at0 = there ? (uint32_t)pg : 0u;
        const uint64_t o = (uint64_t)page_at0 * page_bytes + (head_bytes + in_page * row_bytes);
        from = buffer_rsrc(src + o, tokens * row_bytes);
        if constexpr (!SPLIT) from_v = buffer_rsrc((const char*)a.v + o, tokens * row_bytes);
        if constexpr (FMT != SSM_KV_ACT) {
            const uint64_t r = (uint64_t)page_at0 * page_rows + (head_row + in_page);
            from_s = buffer_rsrc(a.ks + r, 4 * tokens);
            from_vs = buffer_rsrc(a.vs + r, 4 * tokens);
        }
    };
    auto load = [&](__amdgpu_buffer_rsrc_t r, uint32_t o, uint32_t (&x)[GW]) {
        if constexpr (GW == 4) {
            const u32x4 w = buffer_load16(r, o);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = w[e];
        } else if constexpr (GW == 2) {
            const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(r, (int)o, 0, 0);
            x[0] = w[0];
            x[1] = w[1];
        } else {
            x[0] = __builtin_amdgcn_raw_buffer_load_b32(r, (int)o, 0, 0);
        }
    };
    // Lanes 0 .. 15 of the waves that bring k bring the block's scales, of k and of v: four buffers of them,
    // by the step, since a softmax half a step behind reads them later than the codes (below)
    auto load_scales = [&] {
        const uint32_t so = lane < 16 && !brings_v ? 4 * lane : kOffOutOfRange;
        rks = __builtin_amdgcn_raw_buffer_load_b32(from_s, (int)so, 0, 0);
        rvs = __builtin_amdgcn_raw_buffer_load_b32(from_vs, (int)so, 0, 0);
    };
    auto fetch = [&](int tb, int page) {
        locate(tb, page);
#pragma unroll
        for (int i = 0; i < NP; ++i) load(from, off[i], rk[i]);
        if constexpr (!SPLIT) {
#pragma unroll
            for (int i = 0; i < NP; ++i) load(from_v, off[i], rv[i]);
        }
        if constexpr (FMT != SSM_KV_ACT) load_scales();
    };
    auto piece = [&](const uint32_t (&w)[GW]) {            // 16 bytes of T
        u32x4 x;
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
        return x;
    };
    auto stage_piece = [&](int b, int i) {
        *(u32x4*)((brings_v ? &s_v[b][0] : &s_k[b][0]) + at_k[i]) = piece(rk[i]);
        if constexpr (!SPLIT) *(u32x4*)&s_v[b][at_v[i]] = piece(rv[i]);
    };
    auto stage_scales = [&](int step) {
        if constexpr (FMT != SSM_KV_ACT) {
            if (lane < 16 && !brings_v) {
                s_ks[step & 3][16 * blk + lane] = __builtin_bit_cast(float, rks);
                s_vs[step & 3][16 * blk + lane] = __builtin_bit_cast(float, rvs);
            }
        }
    };
    auto stage = [&](int step) {
#pragma unroll
        for (int i = 0; i < NP; ++i) stage_piece(step & 1, i);
        stage_scales(step);
    };

    const float c2 = a.scale * kLog2e;
    float m = -3.0e38f, l = 0.0f;   // finite, so that differences are numbers before any token is seen
    f32x16 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;

    f32x16 s[MT];                                          // the step's scores, then its probabilities
    bf16x8 pf[BF ? TOK / 16 : 1];                          // and those as the operand of the product with v
    auto seen = [&](int tb) {
        return wave_on && tb <= pos_hi && (a.window <= 0 || tb + TOK - 1 > pos_lo - a.window);
    };
    auto scores = [&](int b) {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[t][r] = 0.0f;
        if constexpr (BF) {
            // fragments kLead ahead of the products that take them
            constexpr int kLead = 6, N = QN * MT;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < QN; ++k)
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const bf16x8 kf = *(const bf16x8*)&s_k[b][(t * 32 + col) * KS + k * 16 + half * 8];
                    s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, __builtin_bit_cast(bf16x8, q[k]), s[t], 0, 0, 0);
                }
            __builtin_amdgcn_sched_group_barrier(0x100, kLead, 0);
#pragma unroll
            for (int i = 0; i < N - kLead; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x8, kLead, 0);
            __builtin_amdgcn_sched_barrier(0);
        } else {
#pragma unroll
            for (int k = 0; k < QN; ++k)
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const f32x4 kf = *(const f32x4*)&s_k[b][(t * 32 + col) * KS + k * 8 + half * 4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], q[k][e], s[t], 0, 0, 0);
                }
        }
    };
    bool bad = false;
    auto soften = [&](int tb, int step) {
        if constexpr (FMT != SSM_KV_ACT) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const f32x4 sc = *(const f32x4*)&s_ks[step & 3][t * 32 + 8 * w + 4 * half];
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[t][4 * w + e] *= sc[e];
                }
        }
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
        float mx = s[0][0];
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[t][r]);
        mx = over_halves(mx, [](float x, float y) { return fmaxf(x, y); });
        const float mn = fmaxf(m, mx * c2);
        // The sums are kept relative to m, which need not be the maximum itself: it follows once the
        // maximum is kLag powers of two above it (then no p is above 2^kLag, and no digit is lost)
        if (__any(mn > m + kLag)) {
            const float al = fast_exp2(m - mn);
            l *= al;
#pragma unroll
            for (int t = 0; t < DT; ++t) o[t] *= al;
            m = mn;
        }
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[t][r] = fast_exp2(__builtin_fmaf(s[t][r], c2, -m));
                if constexpr (!BF || FMT != SSM_KV_ACT) l += s[t][r];
            }
        if constexpr (FMT != SSM_KV_ACT) {
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
            // The probabilities enter the product in bf16, half a step (2^-9) off each, as v itself is
            // stored. Their sum l is of the rounded ones where no scale of v is in them: two to an
            // instruction, in float32, and the weights p / l add up to one.
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            const bf16x2 one = {(bf16)1.0f, (bf16)1.0f};
            float ls[2] = {0.0f, 0.0f};
#pragma unroll
            for (int ks = 0; ks < TOK / 16; ++ks) {
#pragma unroll
                for (int e = 0; e < 8; ++e) pf[ks][e] = (bf16)s[ks >> 1][8 * (ks & 1) + e];
                if constexpr (FMT == SSM_KV_ACT) {
#pragma unroll
                    for (int e = 0; e < 8; e += 2)
                        ls[ks & 1] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pf[ks][e], pf[ks][e + 1]}, one, ls[ks & 1], false);
                }
            }
            if constexpr (FMT == SSM_KV_ACT) l += ls[0] + ls[1];
        }
    };
    auto values = [&](int b) {
        if constexpr (BF) {
#pragma unroll
            for (int ks = 0; ks < TOK / 16; ++ks) {
                const T* vp = &s_v[b][(16 * ks + 4 * half + ((lane & 15) >> 2)) * VS + ((lane >> 4) & 1) * 16 + (lane & 3) * 4];
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    typedef short s16x4 __attribute__((ext_vector_type(4)));
                    typedef __attribute__((address_space(3))) s16x4* lds4;
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(vp + t * 32));
                    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(vp + 8 * VS + t * 32));
                    const auto vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf), pf[ks], o[t], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const T* vp = &s_v[b][(8 * (r >> 2) + 4 * half + (r & 3)) * VS + col];
#pragma unroll
                for (int t = 0; t < DT; ++t) o[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(vp[t * 32], s[0][r], o[t], 0, 0, 0);
            }
        }
    };

    if constexpr (SPLIT) {
        // Two waves share a SIMD, one of each half of the workgroup: while one half is in its products,
        // the other is in its softmax, half a step behind. In phase 2 i the first half has the products
        // V(i-1) P(i-1) and K(i) Q and stages K(i+1), the second half has softmax i - 1; in phase 2 i + 1
        // the second half has the same products and stages V(i), the first half has softmax i. K(i) is
        // read in phases 2 i and 2 i + 1, V(i) in 2 i + 2 and 2 i + 3, so two buffers of each do. The
        // scales of step i + 1 come with K(i+1) in phase 2 i and are read in 2 i + 3 and 2 i + 4, when those
        // of the step behind it are there already: three buffers, taken as four.
        //
        // The products of a phase are one run of MFMAs, each fragment read kLead MFMAs ahead of its own
        // (one wave alone: 69 cycles per MFMA as the compiler orders it, 41 so; the MFMA takes 32). The
        // run never branches: P is zero where a step is not seen or not there, and its scores are not used.
        constexpr int kLead = 4, NV = DT * TOK / 16, NK = QN * MT;
        const int steps = (item.k1 - item.k0 + TOK - 1) / TOK;
        const int lead = brings_v ? 0 : 1;                 // products(i) stages step i + lead
        fetch(item.k0, page_at(item.k0));
        int page = page_at(item.k0 + TOK);
        for (int i = tid; i < TOK * VS * 2 / 16; i += 64 * WAVES) ((u32x4*)&s_v[1][0])[i] = u32x4{0, 0, 0, 0};   // V(-1)
#pragma unroll
        for (int ks = 0; ks < TOK / 16; ++ks)
#pragma unroll
            for (int e = 0; e < 8; ++e) pf[ks][e] = (bf16)0.0f;
        const T* v_at = &s_v[0][(4 * half + ((lane & 15) >> 2)) * VS + ((lane >> 4) & 1) * 16 + (lane & 3) * 4];
        const T* k_at = &s_k[0][col * KS + half * 8];
        bf16x8 fr[kLead + 1];
        auto read = [&](int f, int i) {
            if (f < NK) {
                fr[f % (kLead + 1)] = *(const bf16x8*)(k_at + (i & 1) * TOK * KS + (f % MT) * 32 * KS + (f / MT) * 16);
            } else {
                typedef short s16x4 __attribute__((ext_vector_type(4)));
                typedef __attribute__((address_space(3))) s16x4* lds4;
                const T* q = v_at + ((i - 1) & 1) * TOK * VS + ((f - NK) / DT) * 16 * VS + ((f - NK) % DT) * 32;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)q);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(q + 8 * VS));
                fr[f % (kLead + 1)] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        };
        auto read_first = [&](int i) {
#pragma unroll
            for (int f = 0; f < kLead; ++f) read(f, i);
        };
        auto products = [&](int i) {
            constexpr int kStage = NK + 2, kFetch = kStage + NP + 1;
            static_assert(kFetch + NP + 1 <= NV + NK, "the run is long enough");
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int f = 0; f < NV + NK; ++f) {
                if (f + kLead < NV + NK) read(f + kLead, i);
                if (f < NK) {
                    const int t = f % MT;
                    if (f / MT == 0) {
#pragma unroll
                        for (int r = 0; r < 16; ++r) s[t][r] = 0.0f;
                    }
                    s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[f % (kLead + 1)], __builtin_bit_cast(bf16x8, q[f / MT]), s[t], 0, 0, 0);
                } else {
                    const int t = (f - NK) % DT;
                    o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[f % (kLead + 1)], pf[(f - NK) / DT], o[t], 0, 0, 0);
                }
                // what the wave brings, one piece to an MFMA
                if (f >= kStage && f < kStage + NP) stage_piece((i + lead) & 1, f - kStage);
                if (f == kStage + NP) {
                    stage_scales(i + lead);
                    locate(item.k0 + (i + lead + 1) * TOK, page);
                }
                if (f >= kFetch && f < kFetch + NP) load(from, off[f - kFetch], rk[f - kFetch]);
                if (f == kFetch + NP) {
                    if constexpr (FMT != SSM_KV_ACT) load_scales();
                    page = page_at(item.k0 + (i + lead + 2) * TOK);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
        };
        if (!brings_v) {                                   // K(0); the second half's V(0) waits for its first products
            stage(0);
            fetch(item.k0 + TOK, page);
            page = page_at(item.k0 + 2 * TOK);
        }
        __syncthreads();
        bad = s_bad != 0;
        read_first(0);
        if (brings_v) __syncthreads();
        for (int i = 0; i <= steps; ++i) {
            products(i);
            __syncthreads();
            if (i < steps && seen(item.k0 + i * TOK)) {
                soften(item.k0 + i * TOK, i);
            } else {
#pragma unroll
                for (int ks = 0; ks < TOK / 16; ++ks)
#pragma unroll
                    for (int e = 0; e < 8; ++e) pf[ks][e] = (bf16)0.0f;
            }
            read_first(i + 1);
            if (!brings_v || i < steps) __syncthreads();
        }
    } else {
        fetch(item.k0, page_at(item.k0));
        int page = page_at(item.k0 + TOK);
        stage(0);
        __syncthreads();
        bad = s_bad != 0;
        int step = 0;
        for (int tb = item.k0; tb < item.k1; tb += TOK, ++step) {
            const bool more = tb + TOK < item.k1;
            if (more) {
                fetch(tb + TOK, page);
                page = page_at(tb + 2 * TOK);
            }
            if (seen(tb)) {
                scores(step & 1);
                soften(tb, step);
                values(step & 1);
            }
            if (more) stage(step + 1);
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

// Four rows of a cut tile per workgroup, one to a wave: the partial results of its items, in order
template <typename T, int DP, int ROWS> __global__ __launch_bounds__(256) void attn_prefill_join_kernel(AttnArgs p, AttnPlan plan) {
    const KvArgs& a = p.kv;
    const int ji = (int)blockIdx.x / a.Hkv, head = (int)blockIdx.x % a.Hkv;
    if (ji >= plan.count[1]) return;
    const AttnJoin jn = plan.joins[ji];
    const KvSeq sq = kv_seq(a, jn.seq);
    const int g = a.Hq / a.Hkv, r = (int)blockIdx.y * 4 + (threadIdx.x >> 6), row = jn.row0 + r;
    if (row >= sq.m * g) return;
    constexpr int64_t stride = (int64_t)ROWS * (DP + 2);
    const float* part = plan.parts + ((int64_t)head * plan.max_parts + jn.part) * stride;
    join_row<T>(jn.pieces, [&](int v) { return part + v * stride; }, (int64_t)r * DP, ROWS * DP + r,
                ROWS * (DP + 1) + r, a.D, (T*)p.o + (int64_t)(sq.lo + row / g) * p.ld_o + (int64_t)(head * g + row % g) * a.D);
}

template <typename T, int FMT, int DP>
hipError_t launch_attn_prefill_tile(const AttnArgs& p, const AttnPlan& pl, hipStream_t s) {
    constexpr int WAVES = tile_rows(sizeof(T) == 2, DP) / 32;
    KernelTimer kt("attn.prefill", s);
    SSM_LAUNCH((attn_prefill_kernel<T, FMT, DP, WAVES>), dim3((unsigned)pl.max_items * p.kv.Hkv), dim3(64 * WAVES), 0, s, p, pl);
    hipError_t e = hipGetLastError();
    const int64_t longest = (int64_t)p.kv.max_pages << p.kv.page_log2;
    if (e != hipSuccess || longest <= kMinSteps * kStep) return e;   // no tile is ever cut
    KernelTimer kj("attn.prefill_join", s);
    SSM_LAUNCH((attn_prefill_join_kernel<T, DP, 32 * WAVES>), dim3((unsigned)pl.max_joins * p.kv.Hkv, 32 * WAVES / 4), dim3(256), 0,
               s, p, pl);
    return hipGetLastError();
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
