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
    __shared__ __align__(16) float s_ks[2][FMT == SSM_KV_ACT ? 4 : TOK], s_vs[2][FMT == SSM_KV_ACT ? 4 : TOK];
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
    auto page_at = [&](int tb) {                           // the table entry of the wave's block, if there is one
        const int j = tb + 16 * blk;
        return j < n ? table[j >> a.page_log2] : -1;
    };
    auto fetch = [&](int tb, int page) {
        const int pg = __builtin_amdgcn_readfirstlane(page), j = tb + 16 * __builtin_amdgcn_readfirstlane(blk);
        const bool there = pg >= 0 && pg < a.num_pages;
        const int tokens = there ? min(n - j, 16) : 0;     // pg -1 where n <= j
        const int64_t r = there ? kv_pool_row(a, pg, head, j) : 0;
        const uint32_t bytes = (uint32_t)(tokens * a.D * (int)sizeof(E));
        const auto k_src = buffer_rsrc((const E*)(brings_v ? a.v : a.k) + r * a.D, bytes);
        auto load = [&](__amdgpu_buffer_rsrc_t src, uint32_t o, uint32_t (&x)[GW]) {
            if constexpr (GW == 4) {
                const u32x4 w = buffer_load16(src, o);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = w[e];
            } else if constexpr (GW == 2) {
                const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(src, (int)o, 0, 0);
                x[0] = w[0];
                x[1] = w[1];
            } else {
                x[0] = __builtin_amdgcn_raw_buffer_load_b32(src, (int)o, 0, 0);
            }
        };
#pragma unroll
        for (int i = 0; i < NP; ++i) load(k_src, off[i], rk[i]);
        if constexpr (!SPLIT) {
            const auto v_src = buffer_rsrc((const E*)a.v + r * a.D, bytes);
#pragma unroll
            for (int i = 0; i < NP; ++i) load(v_src, off[i], rv[i]);
        }
        if constexpr (FMT != SSM_KV_ACT) {                 // lanes 0 .. 15 bring the block's scales
            const uint32_t so = lane < 16 ? 4 * lane : kOffOutOfRange;
            rks = __builtin_amdgcn_raw_buffer_load_b32(buffer_rsrc((brings_v ? a.vs : a.ks) + r, 4 * tokens), (int)so, 0, 0);
            if constexpr (!SPLIT) rvs = __builtin_amdgcn_raw_buffer_load_b32(buffer_rsrc(a.vs + r, 4 * tokens), (int)so, 0, 0);
        }
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
    auto stage = [&](int b) {
        T* to = brings_v ? &s_v[b][0] : &s_k[b][0];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            *(u32x4*)(to + at_k[i]) = piece(rk[i]);
            if constexpr (!SPLIT) *(u32x4*)&s_v[b][at_v[i]] = piece(rv[i]);
        }
        if constexpr (FMT != SSM_KV_ACT) {
            if (lane < 16) {
                (brings_v ? s_vs : s_ks)[b][16 * blk + lane] = __builtin_bit_cast(float, rks);
                if constexpr (!SPLIT) s_vs[b][16 * blk + lane] = __builtin_bit_cast(float, rvs);
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
    auto soften = [&](int tb, int b) {
        if constexpr (FMT != SSM_KV_ACT) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const f32x4 sc = *(const f32x4*)&s_ks[b][t * 32 + 8 * w + 4 * half];
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[t][4 * w + e] *= sc[e];
                }
        }
        const bool edge = tb + TOK - 1 > pos_lo || (a.window > 0 && tb <= pos_hi - a.window);
        if (edge) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int j = tb + t * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
                    const bool see = j <= pos && (a.window <= 0 || j > pos - a.window);
                    s[t][r] = see ? s[t][r] : -__builtin_inff();
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
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
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
                l += s[t][r];
            }
        if constexpr (FMT != SSM_KV_ACT) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const f32x4 sc = *(const f32x4*)&s_vs[b][t * 32 + 8 * w + 4 * half];
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[t][4 * w + e] *= sc[e];
                }
        }
        if constexpr (BF) {
            // the probabilities enter the product in bf16, half a step (2^-9) off each, as v itself
            // is stored; the sum l is of the unrounded ones
#pragma unroll
            for (int ks = 0; ks < TOK / 16; ++ks)
#pragma unroll
                for (int e = 0; e < 8; ++e) pf[ks][e] = (bf16)s[ks >> 1][8 * (ks & 1) + e];
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
        // V(i-1) P(i-1) and K(i) Q, the second half softmax i - 1 and the staging of V(i); in phase 2 i + 1
        // the second half has its products and the first softmax i and the staging of K(i+1). K(i) is
        // read in phases 2 i and 2 i + 1, V(i) in 2 i + 2 and 2 i + 3, so two buffers of each do.
        const int steps = (item.k1 - item.k0 + TOK - 1) / TOK;
        fetch(item.k0, page_at(item.k0));
        int page = page_at(item.k0 + TOK);
        auto bring = [&](int i) {                          // step i from registers to LDS, step i + 1 on its way
            if (i < steps) {
                stage(i & 1);
                if (i + 1 < steps) {
                    fetch(item.k0 + (i + 1) * TOK, page);
                    page = page_at(item.k0 + (i + 2) * TOK);
                }
            }
        };
        auto products = [&](int i) {
            __builtin_amdgcn_s_setprio(1);
            if (i > 0 && seen(item.k0 + (i - 1) * TOK)) values((i - 1) & 1);
            if (i < steps && seen(item.k0 + i * TOK)) scores(i & 1);
            __builtin_amdgcn_s_setprio(0);
        };
        auto softmax = [&](int i) {
            if (i < steps && seen(item.k0 + i * TOK)) soften(item.k0 + i * TOK, i & 1);
        };
        if (!brings_v) bring(0);
        __syncthreads();
        bad = s_bad != 0;
        if (brings_v) {
            bring(0);
            __syncthreads();
        }
        for (int i = 0; i <= steps; ++i) {
            products(i);
            __syncthreads();
            bring(i + 1);
            softmax(i);
            if (!brings_v || i < steps) __syncthreads();
        }
    } else {
        fetch(item.k0, page_at(item.k0));
        int page = page_at(item.k0 + TOK);
        stage(0);
        __syncthreads();
        bad = s_bad != 0;
        int b = 0;
        for (int tb = item.k0; tb < item.k1; tb += TOK, b ^= 1) {
            const bool more = tb + TOK < item.k1;
            if (more) {
                fetch(tb + TOK, page);
                page = page_at(tb + 2 * TOK);
            }
            if (seen(tb)) {
                scores(b);
                soften(tb, b);
                values(b);
            }
            if (more) stage(b ^ 1);
            __syncthreads();
        }
    }

    l += __shfl_xor(l, 32, 64);
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
