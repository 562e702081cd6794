// Attention of one new token per sequence over the paged cache.
//
// For query head h of sequence i: o = sum_j softmax_j(scale q . k_j) v_j over the visible cached
// tokens j, in one pass with a running maximum m and sum l of the softmax. The g = q_heads / kv_heads
// query heads that share a kv head are the columns of one matrix product, so every cached value is
// read once per 16 of them.
//
// Work split: a unit is 128 tokens of one (sequence, kv head, 16 query heads). The units of the whole
// batch, in that order, are cut into as many equal runs as there are workgroups, whatever the
// sequences' lengths. A workgroup's run may end inside a row of units: what it has of that row is a
// partial result (m, l and the unnormalised o, float32), and a second kernel joins the partials of
// each row in order. Every sum's order follows from the lengths alone.
//
// A wave takes 32 tokens of a unit on its own, straight from global memory into the matrix cores'
// operand layout (16x16 tiles: lane = (quad, i), quad = lane / 16):
//   S^T = K Q^T   row i of tile t is token 8 (i / 4) + 4 t + i % 4, so that the scores a lane ends up
//                 with (rows 4 quad + r) are tokens 8 quad + 4 t + r: eight neighbours;
//   O^T = V^T P^T those eight scores are the lane's operand as they stand. The lane loads
//                 D / 16 neighbouring values of each of the same eight tokens and pairs them up
//                 in registers (one byte permute per two values); row i of product c is dim i D / 16 + c.
// The contraction over D may run in any order that q shares, so k is loaded in whole 16-byte pieces.
// The next tile's loads are issued before the present one is computed. Eight-bit codes become bf16
// exactly; their scales multiply the scores and the probabilities.
//
// Bound by memory: one sequence of 131072 tokens, 8 kv heads of 128 in bf16, 95 us and 7 for the join (5.7 TB/s in the
// main kernel), 256 sequences of 513 to 1025 tokens, 16 heads of 112, 250 us (5.6), 64 of 200 to 8192 tokens in fp8
// 111 us (5.1, the decoding beside it). One of 391 tokens in float32 is one chain of loads, 10 us, and the join's 4.
#include "kv.h"

namespace ssm {
namespace {

constexpr int kUnit = 128;      // tokens per unit: 4 waves x 32
constexpr int kWaveTok = 32;
constexpr int kRows = 16;       // query heads of a unit
constexpr float kNoMax = -3.0e38f;   // running maximum before any token: finite, so differences are numbers

__host__ __device__ constexpr int part_floats(int DP) { return kRows * DP + 2 * kRows; }

// The first visible token of a sequence of n, rounded down to the tile's alignment
__device__ __forceinline__ int first_token(const KvArgs& a, int n) {
    return a.window > 0 && n > a.window ? ((n - a.window) & ~(kWaveTok - 1)) : 0;
}
// units of a row of sequence i: at least one where the sequence is well formed (a row without tokens
// is written as zeros)
__device__ __forceinline__ int row_units(const KvArgs& a, int i) {
    const KvSeq s = kv_seq(a, i);
    if (!s.ok) return 0;
    const int u = (s.n - first_token(a, s.n) + kUnit - 1) / kUnit;
    return u > 0 ? u : 1;
}

// `total` units in `cut` runs that differ by one unit at most: run w is [begin(w), begin(w + 1))
struct Runs {
    int64_t per, rem;
    int cut;
    __device__ __forceinline__ Runs(int64_t total, int workers) {
        cut = total < workers ? (int)total : workers;
        if (cut == 0) {
            per = rem = 0;
        } else if (total <= 0x7fffffff) {   // 32-bit division: a tenth of the 64-bit one's instructions
            per = (uint32_t)total / (uint32_t)cut;
            rem = (uint32_t)total % (uint32_t)cut;
        } else {
            per = total / cut;
            rem = total % cut;
        }
    }
    __device__ __forceinline__ int64_t begin(int w) const { return w * per + (w < rem ? w : rem); }
};
// A value that is the same in every lane, known to be so
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
    return (int64_t)(((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32) | (uint32_t)uniform((int)v));
}

// Prefix over the sequences by a workgroup of 256: the number of units in runs, and the sequence that holds
// the first unit of run w with the units before it (undefined for w >= runs.cut).
struct Place { Runs runs; int seq; int64_t base; };
__device__ __forceinline__ Place find_run(const KvArgs& a, int rows_per_seq, int workers, int w, int64_t* sh) {
    const int tid = threadIdx.x;
    const int per = (a.nseq + 255) / 256;
    int64_t sum = 0;
    for (int k = 0; k < per; ++k) {
        const int i = tid * per + k;
        if (i < a.nseq) sum += (int64_t)row_units(a, i) * rows_per_seq;
    }
    int64_t incl = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int64_t o = __shfl_up(incl, off, 64);
        if ((tid & 63) >= off) incl += o;
    }
    if ((tid & 63) == 63) sh[tid >> 6] = incl;
    __syncthreads();
    int64_t before = 0;
    for (int k = 0; k < (tid >> 6); ++k) before += sh[k];
    const Runs runs(uniform(sh[0] + sh[1] + sh[2] + sh[3]), workers);
    const int64_t u = runs.begin(w), lo = before + incl - sum;
    if (w < runs.cut && u >= lo && u < lo + sum) {   // exactly one thread
        int64_t b = lo;
        for (int k = 0; k < per; ++k) {
            const int64_t c = (int64_t)row_units(a, tid * per + k) * rows_per_seq;
            if (u < b + c) {
                sh[4] = tid * per + k;
                sh[5] = b;
                break;
            }
            b += c;
        }
    }
    __syncthreads();
    return Place{runs, uniform((int)sh[4]), uniform(sh[5])};
}

// Runs, in all forms: two for each of the 256 compute units, which take two workgroups at once up to 128 values a head
// (one of float32 rows of 65 to 128 values) and one above. 768, 1024 and 512 of them: 104, 115 and 102 us for one
// sequence of 131072 tokens with its join, 128, 116 and 115 for the 64 in fp8. 256 and 512 where one workgroup
// fills a unit: 16 heads of 224, 16 sequences of 1000 to 4000 tokens 112 and 115, 16 of 256 over 2 kv heads, 116
// sequences 57 and 60 (float32 161 and 161), one of 65536 tokens 52 and 74 (its join has half the partials then);
// 16 of 112 in float32, 64 sequences 346 and 330, one of 20000 tokens 57 and 64; over fp8 pages 241 and 188.
constexpr int kWorkers = 512;
// The join of a row that is cut: its first query head, how many of them, and the partial results
struct RowJoin { int32_t seq, q_head, rows, pieces; };
constexpr size_t kJoinBytes = kWorkers * sizeof(RowJoin);

// Raw registers of one 32-token tile: a k row in 16-byte pieces of CH values
template <typename T, int FMT, int DP> struct Tile {
    using E = typename KvElem<T, FMT>::type;
    static constexpr int CH = 16 / (int)sizeof(E), NC = DP / (4 * CH), VEC = DP / 16;
    static constexpr int VW = VEC * (int)sizeof(E) / 4;   // 32-bit words of a lane's piece of a v row
    u32x4 k[2][NC];
    uint32_t v[8][VW];
    float ks[8], vs[8];
    int first, last;   // tokens [first, last) of the lane's eight are visible
};

template <int n> __device__ __forceinline__ void load_words(const void* p, uint32_t (&o)[n]) {
    if constexpr (n % 4 == 0) {
#pragma unroll
        for (int i = 0; i < n / 4; ++i) {
            const u32x4 w = ((const u32x4*)p)[i];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[4 * i + e] = w[e];
        }
    } else if constexpr (n == 2) {
        const u32x2 w = *(const u32x2*)p;
        o[0] = w[0];
        o[1] = w[1];
    } else {
        static_assert(n == 1, "a lane's piece of a v row is 4, 8 or a multiple of 16 bytes");
        o[0] = *(const uint32_t*)p;
    }
}

// The table's entries for the wave's 32 tokens from tb: of the eight tokens whose k rows the lane loads, and
// of those whose v rows. Tokens past the sequence's last group of eight are read from that group and masked.
// The entries are fetched a tile ahead of the loads that need them: loads come back in their order, so a
// wait for an entry fetched later would be a wait for the whole tile before it.
struct Pages { int k, v; };
__device__ __forceinline__ Pages tile_pages(const KvArgs& a, const int32_t* table, int n, int tb, int lane) {
    const int end = (n - 1) & ~7;
    return Pages{table[min(tb + 8 * ((lane & 15) >> 2), end) >> a.page_log2], table[min(tb + 8 * (lane >> 4), end) >> a.page_log2]};
}
// The loads of the wave's 32 tokens from tb. Groups whose page the table does not name are read from a
// place that exists and masked.
template <typename T, int FMT, int DP>
__device__ __forceinline__ void load_tile(const KvArgs& a, Tile<T, FMT, DP>& x, Pages pg, int head, int n, int lo, int tb, int lane) {
    using L = Tile<T, FMT, DP>;
    using E = typename L::E;
    const int quad = lane >> 4, i = lane & 15;
    const int end = (n - 1) & ~7;
    const int gk = min(tb + 8 * (i >> 2), end), gv = min(tb + 8 * quad, end);
    const bool named = pg.v >= 0 && pg.v < a.num_pages;
    if (!named && gv + 7 >= lo) atomicOr(a.status, SSM_STATUS_BAD_PAGE);   // a page wholly in front of the window may be gone
    const int pk = pg.k >= 0 && pg.k < a.num_pages ? pg.k : 0, pv = named ? pg.v : 0;
    const int64_t rk = kv_pool_row(a, pk, head, gk), rv = kv_pool_row(a, pv, head, gv);
    const E* kp = (const E*)a.k + rk * a.D;
    const E* vp = (const E*)a.v + rv * a.D;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < L::NC; ++u) {
            int d = u * 4 * L::CH + quad * L::CH;
            d = d < a.D ? d : 0;   // q is zero there
            x.k[t][u] = *(const u32x4*)(kp + (4 * t + (i & 3)) * a.D + d);
        }
    int d = i * L::VEC;
    d = d < a.D ? d : 0;       // dims that are not stored
#pragma unroll
    for (int e = 0; e < 8; ++e) load_words<L::VW>(vp + e * a.D + d, x.v[e]);
    if constexpr (FMT != SSM_KV_ACT) {
        const float4* s0 = (const float4*)(a.ks + rv);
        const float4* s1 = (const float4*)(a.vs + rv);
        const float4 p = s0[0], q = s0[1], r = s1[0], s = s1[1];
        x.ks[0] = p.x; x.ks[1] = p.y; x.ks[2] = p.z; x.ks[3] = p.w; x.ks[4] = q.x; x.ks[5] = q.y; x.ks[6] = q.z; x.ks[7] = q.w;
        x.vs[0] = r.x; x.vs[1] = r.y; x.vs[2] = r.z; x.vs[3] = r.w; x.vs[4] = s.x; x.vs[5] = s.y; x.vs[6] = s.z; x.vs[7] = s.w;
    }
    const int g = tb + 8 * quad;
    x.first = max(lo - g, 0);
    x.last = named ? min(n - g, 8) : 0;
}

// q in the order of the k pieces: bf16 [NC][CH] values per lane, or float32
template <typename T, int FMT, int DP> struct Query {
    using L = Tile<T, FMT, DP>;
    T q[L::NC][L::CH];
    __device__ __forceinline__ void load(const T* p, bool on, int D, int quad) {
#pragma unroll
        for (int u = 0; u < L::NC; ++u) {
            const int d = u * 4 * L::CH + quad * L::CH;
            if (on && d < D) {
                load16(p + d, q[u]);
            } else {
#pragma unroll
                for (int e = 0; e < L::CH; ++e) q[u][e] = from_f32<T>(0.0f);
            }
        }
    }
};

template <int DP> struct Acc {
    f32x4 o[DP / 16];   // product c: rows 4 quad + r are dims (4 quad + r) VEC + c
    float m, l;         // of the lane's query (i); l: the lane's own tokens only
};

__device__ __forceinline__ f32x4 mfma_bf16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_f32(float a, float b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

template <typename T, int FMT, int DP>
__device__ __forceinline__ void attend_tile(Tile<T, FMT, DP>& x, const Query<T, FMT, DP>& q, Acc<DP>& acc, float c2) {
    using L = Tile<T, FMT, DP>;
    constexpr bool BF = sizeof(T) == 2;
    f32x4 s[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
#pragma unroll
    for (int u = 0; u < L::NC; ++u) {
        if constexpr (BF && FMT == SSM_KV_ACT) {
            const bf16x8 b = __builtin_bit_cast(bf16x8, q.q[u]);
#pragma unroll
            for (int t = 0; t < 2; ++t) s[t] = mfma_bf16(__builtin_bit_cast(bf16x8, x.k[t][u]), b, s[t]);
        } else if constexpr (BF) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bf16x8 b;
#pragma unroll
                for (int e = 0; e < 8; ++e) b[e] = q.q[u][8 * h + e];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const u32x2 w0 = kv_decode4_bf16<FMT>(x.k[t][u][2 * h]), w1 = kv_decode4_bf16<FMT>(x.k[t][u][2 * h + 1]);
                    s[t] = mfma_bf16(__builtin_bit_cast(bf16x8, u32x4{w0[0], w0[1], w1[0], w1[1]}), b, s[t]);
                }
            }
        } else {
#pragma unroll
            for (int w = 0; w < L::CH / 4; ++w)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    float k[4];
                    if constexpr (FMT == SSM_KV_ACT) {
                        const f32x4 kv = __builtin_bit_cast(f32x4, x.k[t][u]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) k[e] = kv[e];
                    } else {
                        kv_decode4<FMT>(x.k[t][u][w], k);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[t] = mfma_f32(k[e], q.q[u][4 * w + e], s[t]);
                }
        }
    }
    // scores of tokens 8 quad + e for query i
    float z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = s[e >> 2][e & 3];
    if constexpr (FMT != SSM_KV_ACT) {
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] *= x.ks[e];
    }
    if (!__all(x.first == 0 && x.last == 8)) {   // the tile holds tokens that are not to be seen
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool see = e >= x.first && e < x.last;
            z[e] = see ? z[e] : -__builtin_inff();
            if constexpr (FMT != SSM_KV_ACT) x.vs[e] = see ? x.vs[e] : 0.0f;
            // whatever the cache holds there: 0 * infinity must not reach the sum
#pragma unroll
            for (int w = 0; w < L::VW; ++w) x.v[e][w] = see ? x.v[e][w] : 0u;
        }
    }
    float mx = z[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) mx = fmaxf(mx, z[e]);
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float mn = fmaxf(acc.m, mx * c2);
    if (__any(mn > acc.m)) {
        const float al = fast_exp2(acc.m - mn);
        acc.l *= al;
#pragma unroll
        for (int c = 0; c < L::VEC; ++c) acc.o[c] *= al;
        acc.m = mn;
    }
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        p[e] = fast_exp2(__builtin_fmaf(z[e], c2, -mn));
        acc.l += p[e];
        if constexpr (FMT != SSM_KV_ACT) p[e] *= x.vs[e];
    }
    if constexpr (BF) {
        // the probabilities enter the product in bf16, up to half a step (2^-8 of the value) off
        // each, as v itself is stored; the sum l is of the unrounded ones
        bf16x8 b;
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = (bf16)p[e];
        constexpr int W2 = L::VEC / 2;
        uint32_t r[8][W2];   // bf16 pairs of the lane's dims
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (FMT == SSM_KV_ACT) {
#pragma unroll
                for (int w = 0; w < W2; ++w) r[e][w] = x.v[e][w];
            } else {
#pragma unroll
                for (int w = 0; w < L::VW; ++w) {
                    const u32x2 d = kv_decode4_bf16<FMT>(x.v[e][w]);
                    r[e][2 * w] = d[0];
                    r[e][2 * w + 1] = d[1];
                }
            }
        }
#pragma unroll
        for (int c = 0; c < L::VEC; ++c) {
            u32x4 av;
#pragma unroll
            for (int h = 0; h < 4; ++h)
                av[h] = __builtin_amdgcn_perm(r[2 * h + 1][c >> 1], r[2 * h][c >> 1], (c & 1) ? 0x07060302u : 0x05040100u);
            acc.o[c] = mfma_bf16(__builtin_bit_cast(bf16x8, av), b, acc.o[c]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v[L::VEC];
            if constexpr (FMT == SSM_KV_ACT) {
#pragma unroll
                for (int c = 0; c < L::VEC; ++c) v[c] = __builtin_bit_cast(float, x.v[e][c]);
            } else {
#pragma unroll
                for (int w = 0; w < L::VW; ++w) {
                    float d[4];
                    kv_decode4<FMT>(x.v[e][w], d);
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[4 * w + k] = d[k];
                }
            }
#pragma unroll
            for (int c = 0; c < L::VEC; ++c) acc.o[c] = mfma_f32(v[c], p[e], acc.o[c]);
        }
    }
}

// waves per SIMD that the tile's registers leave room for
template <typename T, int DP> constexpr int min_waves() { return DP <= 128 && sizeof(T) == 2 ? 2 : 1; }

// whether two tiles fit beside the sums: not for float32 rows of 256 values (256 registers a tile)
template <typename T, int FMT, int DP> constexpr bool loads_ahead() { return sizeof(Tile<T, FMT, DP>) <= 768; }

template <typename T, int FMT, int DP>
__global__ __launch_bounds__(256, (min_waves<T, DP>())) void attn_decode_kernel(AttnArgs p, int workers) {
    using L = Tile<T, FMT, DP>;
    constexpr int LD = DP + 4;
    __shared__ int64_t sh[8];
    __shared__ float s_m[4][kRows], s_l[4][kRows];
    __shared__ __align__(16) float s_o[4][kRows][LD];
    const KvArgs& a = p.kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, quad = lane >> 4, i = lane & 15;
    const int g = a.Hq / a.Hkv, rt = (g + kRows - 1) / kRows, rows = a.Hkv * rt;
    if (blockIdx.x == 0) kv_check_seqs(a, tid, 256);
    const int w = (int)blockIdx.x;
    const Place pl = find_run(a, rows, workers, w, sh);
    RowJoin join{};
    RowJoin* joins = (RowJoin*)p.scratch;
    if (w >= pl.runs.cut) {
        if (tid == 0) joins[w] = join;
        return;
    }
    int64_t u = pl.runs.begin(w);
    const int64_t u1 = pl.runs.begin(w + 1);
    const float c2 = a.scale * kLog2e;
    float* part = (float*)(p.scratch + kJoinBytes);
    int seq = pl.seq;
    int64_t base = pl.base;
    while (u < u1) {
        const int nt = row_units(a, seq);
        const int64_t cnt = (int64_t)nt * rows;   // below 2^32: nt at most 2^24, rows at most 128 (checked by the caller)
        if (u >= base + cnt) {
            base += cnt;
            ++seq;
            continue;
        }
        const int n = a.kv_len[seq];
        const int start = first_token(a, n), lo = a.window > 0 && n > a.window ? n - a.window : 0;
        const int row = (int)((uint32_t)(u - base) / (uint32_t)nt), t0 = (int)((uint32_t)(u - base) % (uint32_t)nt);
        const int t1 = (int)((int64_t)nt < t0 + (u1 - u) ? nt : t0 + (u1 - u));
        const int head = row / rt, q0 = (row % rt) * kRows;
        const int nq = g - q0 < kRows ? g - q0 : kRows;

        Query<T, FMT, DP> q;
        q.load((const T*)p.q + (int64_t)seq * p.ld_q + (int64_t)(head * g + q0 + (i < nq ? i : 0)) * a.D, i < nq, a.D, quad);
        Acc<DP> acc;
        acc.m = kNoMax;
        acc.l = 0.0f;
#pragma unroll
        for (int c = 0; c < L::VEC; ++c) acc.o[c] = f32x4{0, 0, 0, 0};
        int tb = start + t0 * kUnit + wave * kWaveTok;
        const int te = min(n, start + t1 * kUnit);
        if (tb < te) {
            const int32_t* table = a.table + (int64_t)seq * a.max_pages;
            Tile<T, FMT, DP> x;
            Pages pg = tile_pages(a, table, n, tb, lane);
            Pages next = tile_pages(a, table, n, tb + kUnit, lane);
            load_tile<T, FMT, DP>(a, x, pg, head, n, lo, tb, lane);
            while (true) {
                const int nb = tb + kUnit;
                if (nb >= te) {
                    attend_tile<T, FMT, DP>(x, q, acc, c2);
                    break;
                }
                pg = next;
                next = tile_pages(a, table, n, nb + kUnit, lane);
                if constexpr (loads_ahead<T, FMT, DP>()) {
                    Tile<T, FMT, DP> y;
                    load_tile<T, FMT, DP>(a, y, pg, head, n, lo, nb, lane);
                    attend_tile<T, FMT, DP>(x, q, acc, c2);
                    x = y;
                } else {
                    attend_tile<T, FMT, DP>(x, q, acc, c2);
                    load_tile<T, FMT, DP>(a, x, pg, head, n, lo, nb, lane);
                }
                tb = nb;
            }
        }
        // join the four waves
        float l = acc.l;
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        if (quad == 0) {
            s_m[wave][i] = acc.m;
            s_l[wave][i] = l;
        }
        if (i < nq) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float* o = &s_o[wave][i][(4 * quad + r) * L::VEC];
#pragma unroll
                for (int c = 0; c < L::VEC; c += 4)
                    *(float4*)(o + c) = make_float4(acc.o[c][r], acc.o[c + 1][r], acc.o[c + 2][r], acc.o[c + 3][r]);
            }
        }
        __syncthreads();
        const bool whole = t0 == 0 && t1 == nt;
        // slot 2 w: a row that began in an earlier workgroup; 2 w + 1: one that goes on in the next
        float* slot = part + (2 * (int64_t)w + (t0 == 0 ? 1 : 0)) * part_floats(DP);
        const int d4 = a.D / 4;
        for (int k = tid; k < nq * d4; k += 256) {
            const int r = k / d4, d = (k % d4) * 4;
            const float M = fmaxf(fmaxf(s_m[0][r], s_m[1][r]), fmaxf(s_m[2][r], s_m[3][r]));
            float o[4] = {0, 0, 0, 0}, ls = 0.0f;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float f = fast_exp2(s_m[v][r] - M);
                const float4 x = *(const float4*)&s_o[v][r][d];
                ls += f * s_l[v][r];
                o[0] += f * x.x; o[1] += f * x.y; o[2] += f * x.z; o[3] += f * x.w;
            }
            if (whole) {
                const float inv = ls > 0.0f ? 1.0f / ls : 0.0f;   // nothing visible: zeros
                T y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = from_f32<T>(o[e] * inv);
                T* out = (T*)p.o + (int64_t)seq * p.ld_o + (int64_t)(head * g + q0 + r) * a.D + d;
                __builtin_memcpy(__builtin_assume_aligned(out, 4 * sizeof(T)), y, sizeof y);
            } else {
                *(float4*)(slot + r * DP + d) = make_float4(o[0], o[1], o[2], o[3]);
                if (d == 0) {
                    slot[kRows * DP + r] = M;
                    slot[kRows * DP + kRows + r] = ls;
                }
            }
        }
        __syncthreads();
        if (t0 == 0 && t1 < nt) {   // the row goes on: this workgroup's record says what its join will be
            const int64_t end = u + nt;
            int last = w + 1;
            while (last + 1 < pl.runs.cut && pl.runs.begin(last + 1) < end) ++last;
            join = RowJoin{seq, head * g + q0, nq, last - w + 1};
        }
        u += t1 - t0;
    }
    if (tid == 0) joins[w] = join;
}

// The rows that the workgroups' runs cut, by the records of the workgroups that began them
template <typename T>
__global__ __launch_bounds__(256) void attn_decode_join_kernel(AttnArgs p, int DP) {
    const int w = (int)blockIdx.x;
    const RowJoin jn = ((const RowJoin*)p.scratch)[w];
    const float* part = (const float*)(p.scratch + kJoinBytes);
    auto slot = [&](int v) { return part + (2 * (int64_t)w + (v == 0 ? 1 : 2 * v)) * part_floats(DP); };
    for (int r = (int)blockIdx.y * 4 + (threadIdx.x >> 6); r < jn.rows; r += 4 * (int)gridDim.y)
        join_row<T, 8>(jn.pieces, slot, r * DP, kRows * DP + r, kRows * DP + kRows + r, p.kv.D,
                    (T*)p.o + (int64_t)jn.seq * p.ld_o + (int64_t)(jn.q_head + r) * p.kv.D);
}

int padded_dim(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

template <typename T, int FMT> hipError_t decode_launch(const AttnArgs& p, hipStream_t s) {
    const KvArgs& a = p.kv;
    const int g = a.Hq / a.Hkv;
    const int64_t rows = (int64_t)a.Hkv * ((g + kRows - 1) / kRows) * a.nseq;
    const int64_t cached = (int64_t)a.max_pages << a.page_log2, seen = (int64_t)a.window + kWaveTok;
    const int64_t longest = a.window > 0 && seen < cached ? seen : cached;
    const int64_t most = rows * ((longest + kUnit - 1) / kUnit);
    const int workers = (int)(most < kWorkers ? most : kWorkers);
    const dim3 grid((unsigned)workers), block(256);
    {
        KernelTimer kt("attn.decode", s);
        switch (padded_dim(a.D)) {
            case 64: SSM_LAUNCH((attn_decode_kernel<T, FMT, 64>), grid, block, 0, s, p, workers); break;
            case 128: SSM_LAUNCH((attn_decode_kernel<T, FMT, 128>), grid, block, 0, s, p, workers); break;
            default: SSM_LAUNCH((attn_decode_kernel<T, FMT, 256>), grid, block, 0, s, p, workers); break;
        }
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || longest <= kUnit || workers < 2) return e;   // no row is ever cut
    KernelTimer kj("attn.decode_join", s);
    SSM_LAUNCH((attn_decode_join_kernel<T>), dim3((unsigned)workers - 1, (unsigned)((g < kRows ? g : kRows) + 3) / 4), block, 0, s, p,
               padded_dim(a.D));
    return hipGetLastError();
}
template <typename T> hipError_t decode_fmt(const AttnArgs& p, hipStream_t s) {
    switch (p.kv.fmt) {
        case SSM_KV_ACT: return decode_launch<T, SSM_KV_ACT>(p, s);
        case SSM_KV_FP8_E4M3: return decode_launch<T, SSM_KV_FP8_E4M3>(p, s);
        default: return decode_launch<T, SSM_KV_INT8>(p, s);
    }
}

}  // namespace

size_t attn_decode_scratch_bytes(int D, int64_t batch) {
    return batch > 0 ? kJoinBytes + (size_t)kWorkers * 2 * part_floats(padded_dim(D)) * 4 : 0;
}
hipError_t launch_attn_decode(const AttnArgs& p, bool bf16_act, hipStream_t s) {
    return bf16_act ? decode_fmt<bf16>(p, s) : decode_fmt<float>(p, s);
}

}  // namespace ssm
