// Prompts of the gated delta rule, in chunks of 64 tokens on the matrix cores. Per value head, with the state S
// (dk x dv here), G the running sum of log alpha in the chunk, K the keys as they are staged and kappa_i what makes row i
// of them the token's key:
//   A_ij = beta_i e^(Gi - Gj) kappa_i kappa_j k_i . k_j (j < i),  T = kappa (I + A)^-1 beta        no state in it
//   R = V - kappa e^G (K S),  U = T R,  O = c e^G (Q S) + (c_i e^(Gi - Gj) q_i . k_j)_{j <= i} U
//   S <- e^(G_C) S + K^T (e^(G_C - Gj) U)
// (c: the queries' lengths and the output's scale.) Pass 1 (delta_chunk_kernel) has a workgroup per chunk and q/k head:
// T and the masked products of queries and keys of its value heads. Pass 2 (delta_split_kernel) walks a sequence's chunks with
// the state in accumulators: columns of S need nothing of each other, so a wave owns 16 of them and waits for no sum of
// another; the outputs are formed by waves of their own. Longer chunks than 64 tokens would have fewer steps in the
// chain, but more work in the inversion and in the products with T; shorter ones more steps, each with the same waits.
//
// Operands are bf16, sums float32. A float32 value is the sum of three bf16 ones, each the rounding of what those in front
// of it leave: 8 bits and a sign each, in float32's range, so nothing has a scale that another value could set. Of
// the products of two such values the six largest are formed; the others are below 2^-26 of the whole. q, k and v in
// bf16 are one value. f16 pairs with a scale by row or column are faster (three MFMAs for a product of two, three vector
// instructions to split a pair of values for eleven, a third less to write and read: prompts of 16 bf16 heads of 128 x 128
// took 53 us for 59, 142 for 185 and 643 for 860), but what lies far below the largest value of its scale loses its bits:
// tokens whose write gate is nearly closed, all that follows a reset.
#include <algorithm>

#include "gate.h"

namespace ssm {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kC = 64;           // tokens per chunk
constexpr int kFrags = 6;        // 16 x 32 pieces of a lower triangular 64 x 64 matrix
// factors by token: e^G kappa, e^(G_C - G), e^G, c; e^(G_C) is the last token's e^G (behind a sequence G stays)
constexpr int kFacDecay = 3 * kC - 1;
constexpr size_t kFacBytes = 4 * kC * 4;
constexpr int kFindSeqs = 256;   // more sequences are laid out by a launch of its own

constexpr int kSplit = 3;        // bf16 values that hold a float32 one
// the parts of a stored q or k
template <typename T> constexpr int kParts = sizeof(T) == 4 ? kSplit : 1;

// Piece (row tile it, k step s) of a lower triangle: rows 16 it .., columns 32 s ..
__host__ __device__ constexpr int frag_of(int it, int s) { return it < 2 ? it : 2 * it - 2 + s; }
// Operand layout of a 16 x 32 piece: lane l holds row l % 16 and, with hh = l / 16, columns 4 hh .. 4 hh + 3 and
// 16 + 4 hh .. 16 + 4 hh + 3: the order in which two stacked accumulator tiles hold their rows. Pieces of q and k
// have their rows rotated by 4 hh, so that the transposing reads of k meet every bank once.
__device__ __forceinline__ int qk_unit(int row, int hh) { return 16 * hh + ((row + 4 * hh) & 15); }

// Sizes of the workspace. Per chunk and q/k head: pieces of k, then of q; per chunk and value head: kappa T beta and the
// factors, then the products of queries and keys.
constexpr size_t qk_bytes(int NS, int parts) { return (size_t)4 * NS * parts * 1024; }   // k or q
constexpr size_t t_bytes() { return (size_t)kFrags * kSplit * 1024 + kFacBytes; }        // for the state
constexpr size_t p_bytes() { return (size_t)kFrags * kSplit * 1024; }                    // for the outputs
constexpr size_t v_bytes() { return t_bytes() + p_bytes(); }

struct DeltaWs {
    int32_t* base;     // [nseq] first chunk of every sequence
    int32_t* count;    // chunks of the call (launch of its own)
    int2* plan;        // [slots] sequence and chunk (launch of its own)
    char* qk; char* v;
    int slots;         // chunks there is room for
};

struct Args {
    DeltaArgs d;
    DeltaWs w;
};

struct SeqRows {
    int lo, n;
    bool ok;
};
__device__ __forceinline__ SeqRows seq_rows(const DeltaArgs& p, int i) {
    const int lo = p.cu[i], hi = p.cu[i + 1];
    const bool ok = lo >= 0 && hi >= lo && (int64_t)hi <= p.T;
    return SeqRows{lo, ok ? hi - lo : 0, ok};
}
__device__ __forceinline__ int chunks_of(int rows) { return (rows + kC - 1) / kC; }

// Inclusive running sums over the wave's lanes, in the vector unit: from the lanes 1, 2, 4 and 8 before in a row of 16,
// then the row before's last lane to rows 1 and 3, then row 1's to rows 2 and 3
template <int CTRL, int ROWS> __device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false); }
template <int CTRL, int ROWS> __device__ __forceinline__ int64_t dpp64(int64_t v) {
    return (int64_t)(((uint64_t)(uint32_t)dpp<CTRL, ROWS>((int)(v >> 32)) << 32) | (uint32_t)dpp<CTRL, ROWS>((int)v));
}
__device__ __forceinline__ int wave_scan32(int c) {
    c += dpp<0x111, 0xF>(c);
    c += dpp<0x112, 0xF>(c);
    c += dpp<0x114, 0xF>(c);
    c += dpp<0x118, 0xF>(c);
    c += dpp<0x142, 0xA>(c);
    return c + dpp<0x143, 0xC>(c);
}
__device__ __forceinline__ int64_t wave_scan64(int64_t c) {
    c += dpp64<0x111, 0xF>(c);
    c += dpp64<0x112, 0xF>(c);
    c += dpp64<0x114, 0xF>(c);
    c += dpp64<0x118, 0xF>(c);
    c += dpp64<0x142, 0xA>(c);
    return c + dpp64<0x143, 0xC>(c);
}

// over four neighbouring lanes
__device__ __forceinline__ float quad_sum(float v) {
    v += __builtin_bit_cast(float, dpp<0xB1, 0xF>(__builtin_bit_cast(int, v)));
    return v + __builtin_bit_cast(float, dpp<0x4E, 0xF>(__builtin_bit_cast(int, v)));
}
__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, __builtin_bit_cast(float, dpp<0xB1, 0xF>(__builtin_bit_cast(int, v))));
    return fmaxf(v, __builtin_bit_cast(float, dpp<0x4E, 0xF>(__builtin_bit_cast(int, v))));
}

// exclusive running sum of v over the 256 threads; total: the whole sum
__device__ __forceinline__ int block_scan(int v, int* lds, int* total) {
    const int tid = threadIdx.x;
    const int c = wave_scan32(v);
    if ((tid & 63) == 63) lds[tid >> 6] = c;
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < (tid >> 6)) before += lds[w];
    }
    *total = (lds[0] + lds[1]) + (lds[2] + lds[3]);
    __syncthreads();
    return before + c - v;
}

// Lays out the chunks of a call of more than 256 sequences
__global__ __launch_bounds__(256) void delta_plan_kernel(Args a) {
    __shared__ int lds[4];
    int start = 0;
    for (int i0 = 0; i0 < a.d.nseq; i0 += 256) {
        const int i = i0 + threadIdx.x;
        const int n = i < a.d.nseq ? chunks_of(seq_rows(a.d, i).n) : 0;
        int total;
        const int at = start + block_scan(n, lds, &total);
        if (i < a.d.nseq) a.w.base[i] = at;
        for (int k = 0; k < n && at + k < a.w.slots; ++k) a.w.plan[at + k] = make_int2(i, k);
        start = min(start + total, 1 << 30);   // sequences that overlap may name any number of rows
    }
    if (threadIdx.x == 0) *a.w.count = min(start, a.w.slots);
}

__device__ __forceinline__ float pow2(int e) { return __builtin_bit_cast(float, (uint32_t)(127 + e) << 23); }
// The exponent that takes a row's largest value m to [1, 2); 0 and what is too small or not finite get one that keeps all
// factors finite
__device__ __forceinline__ int row_exp(float m) {
    const int e = (int)((__builtin_bit_cast(uint32_t, m) >> 23) & 255u);
    return 127 - min(max(e, 40), 230);
}

// The next bf16 values of eight that are left, rounded to nearest; v: what they leave.
__device__ __forceinline__ bf16x8 take8(float (&v)[8]) {
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const bf16x2 h = __builtin_convertvector((f32x2){v[e], v[e + 1]}, bf16x2);
        o[e] = h[0];
        o[e + 1] = h[1];
        v[e] -= (float)h[0];
        v[e + 1] -= (float)h[1];
    }
    return o;
}
template <int N> __device__ __forceinline__ void split8(float (&v)[8], bf16x8 (&o)[N]) {
#pragma unroll
    for (int part = 0; part < N; ++part) o[part] = take8(v);
}

__device__ __forceinline__ f32x4 mma(const bf16x8& a, const bf16x8& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// The products of two values in parts, the largest first: part first(n) of the one and second(n) of the other
constexpr int kProducts = 6;
constexpr int first(int n) { return n == 2 || n == 4 ? 1 : n == 5 ? 2 : 0; }
constexpr int second(int n) { return n == 1 || n == 4 ? 1 : n == 3 ? 2 : 0; }
__device__ __forceinline__ f32x4 mma4(float a, float b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// ---------------------------------------------------------------- pass 1
constexpr int kLdA = kC + 4;   // row stride of the 64 x 64 float32 matrix

template <typename T> struct Piece {   // eight values of a row
    u32x4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t& r, uint32_t off) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = buffer_load16(r, off + 16 * i);
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        T x[8];
        __builtin_memcpy(x, w, sizeof x);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = to_f32(x[k]);
    }
};

// Of a row of q or k that four threads hold: the sum of squares, and the exponent of its scale
template <typename T, int NS> __device__ __forceinline__ float row_sizes(const Piece<T> (&x)[NS], int* e) {
    float ss = 0.0f, m = 0.0f;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        float v[8];
        x[s].values(v);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            ss = __builtin_fmaf(v[k], v[k], ss);
            m = fmaxf(m, fabsf(v[k]));
        }
    }
    *e = row_exp(quad_max(m));
    return quad_sum(ss);
}
// N pieces of the row that this thread (c4 of four) holds, from s0 on, times f: in operand layout, to LDS
template <typename T, int N, int NS>
__device__ __forceinline__ void stage_row(const Piece<T> (&x)[NS], int s0, int row, int c4, float f, char* lds) {
#pragma unroll
    for (int s = 0; s < N; ++s) {
        float v[8];
        x[s0 + s].values(v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= f;
#pragma unroll
        for (int part = 0; part < kParts<T>; ++part) {
            const bf16x8 h = take8(v);
            // values 0..3 of the piece are (hh, half) = (2 (c4 & 1), c4 / 2), values 4..7 the next hh
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                bf16x4 o;
#pragma unroll
                for (int k = 0; k < 4; ++k) o[k] = h[4 * q + k];
                const int at = (((part * 4 + (row >> 4)) * N + s) * 64 + qk_unit(row & 15, 2 * (c4 & 1) + q)) * 16 + (c4 >> 1) * 8;
                *(bf16x4*)(lds + at) = o;
            }
        }
    }
}

template <int NS> __device__ __forceinline__ bf16x8 qk_piece(const char* lds, int part, int it, int s, int lane) {
    return *(const bf16x8*)(lds + (((part * 4 + it) * NS + s) * 64 + qk_unit(lane & 15, lane >> 4)) * 16);
}

// One workgroup per chunk and q/k head; its value heads two at a time, each inverted by two waves. What bounds it is the
// chain of its phases (rows to LDS, products, inversion by blocks, output), half of whose time is waits, and with many
// chunks HBM: 8 prompts of 2048 tokens, 16 bf16 value heads of 128 over 8, 60 us for 222 MB written, 4 of 16384 tokens,
// 889 MB, 222 us; three workgroups to a compute unit for two took the first from 63 to 55 when it wrote 147 MB. A chunk of
// its own per value head read and multiplied the rows twice (then 274 us for 222 of the second).
// HB: value heads a pass, 1 where a q/k head has one. What a pass of two computes for a second head that is not there
// is not stored.
template <typename T, int NS, int HB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(kParts<T> * NS <= 12 ? 2 : 1))) void delta_chunk_kernel(Args a) {
    constexpr int PA = kParts<T>, kQk = (int)qk_bytes(NS, PA);
    // pieces in LDS at a time: float32 rows come in two halves
    constexpr int kTurns = PA > 1 && NS >= 4 ? 2 : 1, NH = NS / kTurns, kTurn = kQk / kTurns;
    // q's pieces, and once they are used the heads' matrices in their place
    constexpr int kMat = HB * kC * kLdA * 4;
    __shared__ __attribute__((aligned(16))) char s_k[kTurn], s_q[kTurn > kMat ? kTurn : kMat];
    float(*s_t)[kC * kLdA] = (float(*)[kC * kLdA])s_q;
    __shared__ __attribute__((aligned(16))) float s_gh[HB][kC], s_gl[HB][kC], s_beta[HB][kC], s_kap[kC], s_c[kC];
    __shared__ int s_find[8];
    const DeltaArgs& p = a.d;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), slot = blockIdx.x, hk = blockIdx.y;
    int seq = -1, chunk = 0;
    if (p.nseq <= kFindSeqs) {
        int n = 0, total;
        if (tid < p.nseq) {
            const SeqRows r = seq_rows(p, tid);
            n = chunks_of(r.n);
            if (!r.ok && slot == 0 && hk == 0) atomicOr(p.status, SSM_STATUS_BAD_SEQLENS);
        }
        if (tid == 0) s_find[4] = -1;
        const int at = block_scan(n, s_find, &total);
        if (slot == 0 && hk == 0 && tid < p.nseq) a.w.base[tid] = at;
        if (slot >= at && slot < at + n) {
            s_find[4] = tid;
            s_find[5] = slot - at;
        }
        __syncthreads();
        seq = s_find[4];
        chunk = s_find[5];
    } else if (slot < *a.w.count) {
        const int2 pl = a.w.plan[slot];
        seq = pl.x;
        chunk = pl.y;
    }
    seq = __builtin_amdgcn_readfirstlane(seq);
    chunk = __builtin_amdgcn_readfirstlane(chunk);
    if (seq < 0) return;
    const SeqRows sr = seq_rows(p, seq);
    const int64_t t0 = (int64_t)__builtin_amdgcn_readfirstlane(sr.lo) + (int64_t)chunk * kC;
    const int nq = min(__builtin_amdgcn_readfirstlane(sr.n) - chunk * kC, kC);

    // the gates of a value head by wave 2 or 3, a token a lane; into place b. Asked for in front of the rows and worked out
    // while these are on their way
    T av{}, bv{};
    float la = 0.0f, db = 0.0f;
    auto gate_loads = [&](int h) {
        if (lane < nq) {
            av = ((const T*)p.a)[(t0 + lane) * p.ld_ab + h];
            bv = ((const T*)p.b)[(t0 + lane) * p.ld_ab + h];
        }
        la = p.A_log[h];
        db = p.dt_bias[h];
    };
    if (wave >= 2 && wave - 2 < HB) gate_loads(hk * p.rep + wave - 2);

    // rows of q and k: four threads to a row
    const __amdgpu_buffer_rsrc_t rx = buffer_rsrc((const T*)p.qkv + t0 * p.ld, (uint32_t)((nq - 1) * p.ld + 2 * p.Hk * p.dk) * sizeof(T));
    const int row = tid >> 2, c4 = tid & 3;
    Piece<T> xq[NS], xk[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const int n = 32 * s + 8 * c4;
        const uint32_t off = row < nq && n < p.dk ? (uint32_t)(row * p.ld + hk * p.dk + n) * (uint32_t)sizeof(T) : kOffOutOfRange;
        xk[s].load(rx, off + (uint32_t)(p.Hk * p.dk) * (uint32_t)sizeof(T));
        xq[s].load(rx, off);
    }
    auto gates = [&](int b) {
        // log2 of alpha; below -1000 it is 0 in float32 either way, and the sums of what follows stay exact. The running
        // sum in 64 bits of 2^-40 (its absolute error is what counts), kept as two float32 values: what comes
        // after a reset is as exact as without one
        float g = -fast_exp2(la * kLog2e) * kLog2e * softplus_f(to_f32(av) + db);
        const bool nan = g != g;
        g = lane < nq ? (g < -1000.0f ? -1000.0f : g) : 0.0f;
        const int64_t c = wave_scan64(nan ? 0 : (int64_t)((double)g * 1099511627776.0));
        const double d = (double)c * (1.0 / 1099511627776.0);
        // a decay that is no number leaves none from its token on
        const bool bad = (__ballot(nan && lane < nq) & (~0ull >> (63 - lane))) != 0;
        s_gh[b][lane] = bad ? __builtin_nanf("") : (float)d;
        s_gl[b][lane] = (float)(d - (double)(float)d);
        s_beta[b][lane] = lane < nq ? p.beta_max * sigmoid_f(to_f32(bv)) : 0.0f;
    };
    if (wave >= 2 && wave - 2 < HB) gates(wave - 2);
    int eq, ek;
    const float sk = row_sizes<T, NS>(xk, &ek), sq = row_sizes<T, NS>(xq, &eq);
    if (c4 == 0) {
        s_c[row] = p.scale * (p.qk_norm ? 1.0f / sqrtf(fmaxf(sq + p.eps, 1.2e-38f)) : 1.0f) * pow2(-eq);
        s_kap[row] = (p.qk_norm ? 1.0f / sqrtf(fmaxf(sk + p.eps, 1.2e-38f)) : 1.0f) * pow2(-ek);
    }

    // K K^T and K Q^T: wave w has columns i = 16 w + lane % 16, pieces n of rows j = 32 n + 16 q + 4 hh + r up to the
    // diagonal: one piece for waves 0 and 1, two for the others
    const int it = wave, pieces = 1 + it / 2;
    // The lane's place in a tile, worked out anew in every phase: addresses kept from one to the next cost a third of the
    // registers and with them a workgroup per compute unit
    auto place = [&] {
        int l = lane;
        asm volatile("" : "+v"(l));
        return l;
    };
    const bool odd = (it & 1) != 0;                    // the second tile of the last piece reaches the diagonal
    f32x4 kk[2][2], kq[2][2];
#pragma unroll
    for (int n = 0; n < 2; ++n) kk[n][0] = kk[n][1] = kq[n][0] = kq[n][1] = f32x4{};
    char* qk = a.w.qk + ((int64_t)slot * p.Hk + hk) * (2 * kQk);
#pragma unroll
    for (int turn = 0; turn < kTurns; ++turn) {
        if (turn > 0) __syncthreads();
        stage_row<T, NH, NS>(xk, NH * turn, row, c4, pow2(ek), s_k);
        stage_row<T, NH, NS>(xq, NH * turn, row, c4, pow2(eq), s_q);
        __syncthreads();
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            if (n >= pieces) break;
#pragma unroll
            for (int s = 0; s < NH; ++s) {
                bf16x8 y[PA], z[PA];
#pragma unroll
                for (int part = 0; part < PA; ++part) {
                    y[part] = qk_piece<NH>(s_k, part, it, s, lane);
                    z[part] = qk_piece<NH>(s_q, part, it, s, lane);
                }
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    if (q == 1 && n + 1 == pieces && !odd) break;
                    bf16x8 x[PA];
#pragma unroll
                    for (int part = 0; part < PA; ++part) x[part] = qk_piece<NH>(s_k, part, 2 * n + q, s, lane);
#pragma unroll
                    for (int m = 0; m < kProducts; ++m) {
                        if (first(m) >= PA || second(m) >= PA) continue;
                        kk[n][q] = mma(x[first(m)], y[second(m)], kk[n][q]);
                        kq[n][q] = mma(x[first(m)], z[second(m)], kq[n][q]);
                    }
                }
            }
        }
#pragma unroll
        for (int n = 0; n < kTurn / 4096; ++n) {
            const int b = n * 4 + wave, from = (b * 64 + lane) * 16, to = ((b / NH * NS + turn * NH + b % NH) * 64 + lane) * 16;
            *(u32x4*)(qk + to) = *(const u32x4*)(s_k + from);
            *(u32x4*)(qk + kQk + to) = *(const u32x4*)(s_q + from);
        }
    }
    const float kap = s_kap[16 * it + (lane & 15)];
    __syncthreads();

    for (int r0 = 0; r0 < p.rep; r0 += HB) {
        const int heads = min(HB, p.rep - r0);
        auto vout = [&](int b) { return a.w.v + ((int64_t)slot * p.Hv + hk * p.rep + r0 + b) * v_bytes(); };
        if (r0 > 0) {
            __syncthreads();
            if (wave >= 2 && wave - 2 < heads) {
                gate_loads(hk * p.rep + r0 + wave - 2);
                gates(wave - 2);
            }
            __syncthreads();
        }
        {
        const int l = place(), hh = l >> 4, i = 16 * it + (l & 15);
        float gh[HB], gl[HB], bk[HB];
#pragma unroll
        for (int b = 0; b < HB; ++b) {
            gh[b] = s_gh[b][i];
            gl[b] = s_gl[b][i];
            bk[b] = s_beta[b][i] * kap;
        }
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            if (n >= pieces) break;
            float x[HB][8];
            f32x4 jh[HB][2], jl[HB][2], jk[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int j = 32 * n + 16 * q + 4 * hh;
                jk[q] = *(const f32x4*)&s_kap[j];
#pragma unroll
                for (int b = 0; b < HB; ++b) {
                    jh[b][q] = *(const f32x4*)&s_gh[b][j];
                    jl[b][q] = *(const f32x4*)&s_gl[b][j];
                }
            }
#pragma unroll
            for (int b = 0; b < HB; ++b)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int j = 32 * n + 16 * q + 4 * hh;
                    f32x4 m;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float ex = fast_exp2((gh[b] - jh[b][q][r]) + (gl[b] - jl[b][q][r]));
                        m[r] = j + r < i ? kk[n][q][r] * ex * (bk[b] * jk[q][r]) : 0.0f;
                        x[b][4 * q + r] = j + r <= i ? kq[n][q][r] * ex : 0.0f;
                    }
                    *(f32x4*)&s_t[b][i * kLdA + j] = m;   // zeros above the diagonal, where this piece has them
                }
#pragma unroll
            for (int b = 0; b < HB; ++b) {
                if (b >= heads) break;
                char* to = vout(b) + t_bytes() + (frag_of(it, n) * 1024 + l * 16);
#pragma unroll
                for (int part = 0; part < kSplit; ++part) *(bf16x8*)(to + part * kFrags * 1024) = take8(x[b]);
            }
        }
        }
        __syncthreads();
        // T = (I + A)^-1 in place, in float32: the diagonal 16 x 16 blocks by substitution (lane: block and column), then
        // [T1 0; -T2 A21 T1 T2] for blocks of 16 and of 32. One wave per head, then two, then all for each
        if (wave < HB) {
            const int l = place(), hh = l >> 4, col = l & 15;
            float* t = s_t[wave] + 16 * hh * kLdA + 16 * hh;
            // row r in pieces of four, asked for in three lots in front of their use
            f32x4 m[16][4];
            float x[16];
            auto ask = [&](int r0, int r1) {
#pragma unroll
                for (int r = r0; r < r1; ++r)
#pragma unroll
                    for (int j = 0; 4 * j < r; ++j) m[r][j] = *(const f32x4*)&t[r * kLdA + 4 * j];
                __builtin_amdgcn_sched_barrier(0);
            };
            auto solve = [&](int r0, int r1) {
#pragma unroll
                for (int r = r0; r < r1; ++r) {
                    float s = r == col ? 1.0f : 0.0f;
#pragma unroll
                    for (int j = 0; j < r; ++j) s = __builtin_fmaf(-m[r][j / 4][j % 4], x[j], s);
                    x[r] = s;
                }
            };
            ask(1, 8);
            solve(0, 8);
            ask(8, 12);
            solve(8, 12);
            ask(12, 16);
            solve(12, 16);
#pragma unroll
            for (int r = 0; r < 16; ++r) t[r * kLdA + col] = x[r];
        }
        // the tokens' factors, by waves 2 and 3
        if (wave >= 2 && wave - 2 < heads) {
            const int b = wave - 2;
            float* fac = (float*)(vout(b) + t_bytes() - kFacBytes);
            const float gh = s_gh[b][lane], gl = s_gl[b][lane], ch = s_gh[b][kC - 1], cl = s_gl[b][kC - 1];
            const float eg = fast_exp2(gh + gl);
            fac[lane] = eg * s_kap[lane];
            fac[kC + lane] = fast_exp2((ch - gh) + (cl - gl));
            fac[2 * kC + lane] = eg;
            fac[3 * kC + lane] = s_c[lane];
        }
        __syncthreads();
        // a row piece (this lane's row, columns 4 hh ..) of a block, and its column entries 4 hh + r of this lane's column;
        // l: the lane
        auto row4 = [&](const float* t, int y, int x, int l) { return *(const f32x4*)&t[(y + (l & 15)) * kLdA + x + 4 * (l >> 4)]; };
        auto col4 = [&](const float* t, int y, int x, int l) {
            f32x4 v;
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = t[(y + 4 * (l >> 4) + r) * kLdA + x + (l & 15)];
            return v;
        };
        auto times = [&](const f32x4& m, const f32x4& x, f32x4 acc) {
#pragma unroll
            for (int r = 0; r < 4; ++r) acc = mma4(m[r], x[r], acc);
            return acc;
        };
        auto put = [&](float* t, int y, int x, const f32x4& v, int l) {
#pragma unroll
            for (int r = 0; r < 4; ++r) t[(y + 4 * (l >> 4) + r) * kLdA + x + (l & 15)] = -v[r];
        };
        if (wave < 2 * HB) {
            float* t = s_t[wave >> 1];
            const int c0 = 32 * (wave & 1), y0 = c0 + 16, l = place();
            const f32x4 x = times(row4(t, y0, c0, l), col4(t, c0, c0, l), f32x4{});
            put(t, y0, c0, times(row4(t, y0, y0, l), x, f32x4{}), l);
        }
        __syncthreads();
        {
            const int r2 = wave >> 1, c0 = 16 * (wave & 1), l = place();
            // [T1 0; T21 T2] again, in 16 x 16 blocks; what lies above the diagonal is not stored and counts as zero
            f32x4 y[HB];
#pragma unroll
            for (int b = 0; b < HB; ++b) {
                const float* t = s_t[b];
                const f32x4 zero{}, t0 = col4(t, 0, 0, l), t1 = col4(t, 16, c0, l);
                const f32x4 u0 = (wave & 1) == 0 ? t0 : zero;
                f32x4 x[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) x[k] = times(row4(t, 32 + 16 * k, 16, l), t1, times(row4(t, 32 + 16 * k, 0, l), u0, zero));
                const f32x4 m1 = r2 == 1 ? row4(t, 48, 48, l) : zero;
                y[b] = times(m1, x[1], times(row4(t, 32 + 16 * r2, 32, l), x[0], zero));
            }
            __syncthreads();
#pragma unroll
            for (int b = 0; b < HB; ++b) put(s_t[b], 32 + 16 * r2, c0, y[b], l);
        }
        __syncthreads();
        // kappa T beta: wave w has row tile w
        const int l = place(), hh = l >> 4;
#pragma unroll
        for (int b = 0; b < HB; ++b) {
            if (b >= heads) break;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                if (n >= pieces) break;
                const f32x4 v0 = row4(s_t[b], 16 * it, 32 * n, l), v1 = row4(s_t[b], 16 * it, 32 * n + 16, l);
                const f32x4 b0 = *(const f32x4*)&s_beta[b][32 * n + 4 * hh], b1 = *(const f32x4*)&s_beta[b][32 * n + 16 + 4 * hh];
                const bool two = odd || n + 1 < pieces;
                float x[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = v0[e] * b0[e] * kap;
                    x[4 + e] = two ? v1[e] * b1[e] * kap : 0.0f;
                }
                char* to = vout(b) + (frag_of(it, n) * 1024 + l * 16);
#pragma unroll
                for (int part = 0; part < kSplit; ++part) *(bf16x8*)(to + part * kFrags * 1024) = take8(x);
            }
        }
    }
}

// ---------------------------------------------------------------- pass 2
// Two stacked tiles as an operand: the bf16 values of each
template <int N> __device__ __forceinline__ void split2(const f32x4& x0, const f32x4& x1, bf16x8 (&o)[N]) {
    float v[8];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        v[r] = x0[r];
        v[4 + r] = x1[r];
    }
    split8(v, o);
}

// Asks for an order of what lies between two sched_barriers: M times an MFMA and V vector instructions
template <int M, int V> __device__ __forceinline__ void interleave() {
#pragma unroll
    for (int i = 0; i < M; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, V, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
}

constexpr size_t kLds = 160 * 1024;

// `bytes` (a multiple of 1 KB) from a buffer to LDS, dealt out over the workgroup's waves
template <int WAVES, int BYTES> __device__ __forceinline__ void dma_pieces(const __amdgpu_buffer_rsrc_t& r, uint32_t from, uint32_t lds, int wave, int lane) {
    constexpr int N = BYTES / 1024;
#pragma unroll
    for (int i = 0; i < (N + WAVES - 1) / WAVES; ++i) {
        const int j = wave + WAVES * i;
        if (N % WAVES == 0 || j < N)
            dma16(r, (uint32_t)lane * 16, from + (uint32_t)j * 1024, __builtin_amdgcn_readfirstlane(lds + (uint32_t)j * 1024));
    }
}
// Pieces that a wave holds in registers: of q, k step s, and the products of queries and keys
template <int NS, int PA>
__device__ __forceinline__ void load_q(bf16x8 (&q)[PA][4], const __amdgpu_buffer_rsrc_t& r, uint32_t from, int s, int lane) {
    const int off = qk_unit(lane & 15, lane >> 4) * 16;
#pragma unroll
    for (int part = 0; part < PA; ++part)
#pragma unroll
        for (int it = 0; it < 4; ++it)
            q[part][it] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(r, off, (int)from + ((part * 4 + it) * NS + s) * 1024, 0));
}
__device__ __forceinline__ void load_p(bf16x8 (&x)[kSplit][kFrags], const __amdgpu_buffer_rsrc_t& r, uint32_t from, int lane) {
#pragma unroll
    for (int part = 0; part < kSplit; ++part)
#pragma unroll
        for (int f = 0; f < kFrags; ++f)
            x[part][f] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(r, lane * 16, (int)from + (part * kFrags + f) * 1024, 0));
}
// Rows dk = 16 t + lane % 16 of K^T, tokens 32 s + 4 hh .. and 32 s + 16 + 4 hh ..: four rows of 16 values of k, transposed
// as they are read
template <int NS> __device__ __forceinline__ bf16x8 kt_piece(const char* s_k, int part, int s, int t, int lane) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds4;
    s16x4 k2[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const char* at = s_k + (((part * 4 + 2 * s + q) * NS + t / 2) * 64 + qk_unit(4 * (lane >> 4) + ((lane & 15) >> 2), lane & 3)) * 16 + (t & 1) * 8;
        k2[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)at);
    }
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(k2[0], k2[1], 0, 1, 2, 3, 4, 5, 6, 7));
}

// Workgroups are dealt out to the XCDs in turn: item (sequence, q/k head) u runs on XCD u % 8, whose L2 then holds the
// pieces that its value heads and column blocks share. Grid: 8 rep blocks by every eighth item, in rows of kGridRow.
constexpr int kGridRow = 1 << 15;
struct WorkItem {
    int seq, head, block;   // seq may be past the last
};
__device__ __forceinline__ WorkItem work_item(const DeltaArgs& p, int blocks) {
    const int u = ((int)blockIdx.z * kGridRow + (int)blockIdx.y) * 8 + (int)(blockIdx.x & 7), in = (int)(blockIdx.x >> 3);
    return WorkItem{u / p.Hk, u % p.Hk * p.rep + in / blocks, in % blocks};
}
dim3 work_grid(const DeltaArgs& p, int blocks) {
    const unsigned rows = (unsigned)(((int64_t)p.nseq * p.Hk + 7) / 8);
    return dim3((unsigned)(8 * p.rep * blocks), std::min<unsigned>(rows, kGridRow), (rows + kGridRow - 1) / kGridRow);
}

// A workgroup has W waves that carry the state, 16 columns each, and W that form the outputs of the chunk before from what
// the first left in LDS: the chain from chunk to chunk is that much shorter, and both kinds run beside each other.
// 317, 1130 and 601 tokens, 16 heads of 128 x 128: 45.6 us in bf16 (2.5 a chunk of the longest), 68 in float32 (3.8). Bound
// by a chunk's chain: a wave that carries the state has 132 MFMAs and 420 vector instructions, which share its issue port (8
// and 4 cycles each), and waits for what it reads from LDS in between; with four waves of columns by those of the outputs
// beside them on the same SIMD: 8 prompts of 2048 tokens 140 us (4.4 a chunk), the matrix pipe 36% busy, vector
// instructions 40%, LDS 32%. Each stretch of a chunk asks the compiler for vector instructions between its MFMAs that are
// for those of the next. Tried: taking a half of a pair off by a dot product with (-1, 0), one instruction for two, which is
// exact too, but runs in the matrix pipe (float32 76 us for 68); DMA spread over the products instead of in bursts (173 us
// for 158 of the 8 prompts); a higher priority for either kind of wave (nothing).
//
// What it has in LDS. Two barriers a chunk, at its begin and in its middle, tell what is free. Read by the middle: the
// factors and values of the chunk, and what is handed over; k and T are needed until the end and have two stages where
// there is room (else they arrive by the middle). For the outputs, q arrives by the middle and is read behind it, and
// the products of queries and keys are read by it; where these do not fit, each wave has its own in registers (kDirect). Where
// values do not fit, so has each wave that carries the state.
template <typename T, int NS, int W> struct SplitLds {
    static constexpr int kQk = (int)qk_bytes(NS, kParts<T>), kT = (int)(t_bytes() - kFacBytes), kFac = (int)kFacBytes, kP = (int)p_bytes();
    static constexpr int kRow = 16 * W * (int)sizeof(T);                      // the workgroup's values of a token
    // S and U of 16 columns; with four waves of columns, where the waves of the outputs are late, S as operands, which they
    // then need not form (8 prompts of 2048 tokens 177 us for 184; two waves of columns lose by it, 62.4 us for 59.5)
    static constexpr bool kFormed = W == 4;
    static constexpr int kHandS = (kFormed ? kSplit * NS : 2 * NS) * 1024, kHand = kHandS + 4 * 1024;
    static constexpr int k_stages(int mode) { return mode < 4 ? 2 : 1; }
    static constexpr int t_stages(int mode) { return mode == 0 || mode == 2 ? 2 : 1; }
    static constexpr int row_bytes(int mode) { return mode < 5 ? kC * kRow : 0; }
    static constexpr int bytes(int mode) {
        return k_stages(mode) * kQk + t_stages(mode) * kT + kFac + row_bytes(mode) + W * kHand + (mode < 2 ? kQk + kFac + kP : 0);
    }
    static constexpr int pick(int mode) { return mode == 6 || bytes(mode) <= (int)kLds ? mode : pick(mode + 1); }
    static constexpr int kMode = pick(0), kBytes = bytes(kMode), kKStages = k_stages(kMode), kTStages = t_stages(kMode);
    static constexpr bool kDirect = kMode >= 2, kOwnRows = kMode >= 5;
    static constexpr int kTAt = kKStages * kQk, kFacAt = kTAt + kTStages * kT, kRowsAt = kFacAt + kFac, kHandAt = kRowsAt + row_bytes(kMode);
    static constexpr int kQAt = kHandAt + W * kHand, kOutFacAt = kQAt + kQk, kPAt = kOutFacAt + kFac;
};

// Where 256 registers are enough the kernel is held to them: beyond, the compiler keeps half where only MFMAs reach them (391
// float32 tokens, heads of 64: 30.7 us for 32.4, bf16 heads of 192: 72.8 for 77.7)
template <typename T, int NS, int W>
__global__ __launch_bounds__(128 * W) __attribute__((amdgpu_waves_per_eu(NS * kParts<T> <= 6 ? 2 : 1))) void delta_split_kernel(Args a) {
    constexpr int PA = kParts<T>, NT = 2 * NS;
    using L = SplitLds<T, NS, W>;
    static_assert(L::kMode < 6, "pass 2 does not fit into LDS");
    constexpr int kQk = L::kQk, kT = L::kT, kRow = L::kRow, kHandS = L::kHandS, kHand = L::kHand, kP = L::kP;
    constexpr uint32_t sz = sizeof(T);
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const DeltaArgs& p = a.d;
    const int tid = threadIdx.x, lane = tid & 63, hh = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const WorkItem it0 = work_item(p, (p.dv + 16 * W - 1) / (16 * W));
    if (it0.seq >= p.nseq) return;
    const int seq = it0.seq, h = it0.head, hk = h / p.rep;
    const bool carries = wave < W;
    const int wc = carries ? wave : wave - W;
    const int c0 = (it0.block * W + wc) * 16;          // this wave's columns
    const bool on = c0 < p.dv;
    const SeqRows sr = seq_rows(p, seq);
    const int lo = __builtin_amdgcn_readfirstlane(sr.lo), rows = __builtin_amdgcn_readfirstlane(sr.n);
    const int slot = p.slot[seq], n = chunks_of(rows), base = rows > 0 ? __builtin_amdgcn_readfirstlane(a.w.base[seq]) : 0;
    const bool fits = sr.ok && base + n <= a.w.slots, ok = slot >= 0 && slot < p.S;
    if (h == 0 && it0.block == 0 && tid == 0 && (!fits || !ok))
        atomicOr(p.status, (fits ? 0 : SSM_STATUS_BAD_SEQLENS) | (ok ? 0 : SSM_STATUS_BAD_SLOT));
    if (!fits) return;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
    auto qk_buf = [&](int c) { return buffer_rsrc(a.w.qk + ((int64_t)(base + c) * p.Hk + hk) * (2 * kQk), 2 * kQk); };
    auto v_buf = [&](int c) { return buffer_rsrc(a.w.v + ((int64_t)(base + c) * p.Hv + h) * (int64_t)v_bytes(), (uint32_t)v_bytes()); };
    const uint32_t ldv = (uint32_t)p.ld * sz;
    auto rows_buf = [&](int c) {                       // this head's values
        const int nq = min(rows - c * kC, kC);
        return buffer_rsrc((const T*)p.qkv + ((int64_t)lo + (int64_t)c * kC) * p.ld + 2 * p.Hk * p.dk + h * p.dv,
                           (uint32_t)(nq - 1) * ldv + (uint32_t)p.dv * sz);
    };
    // What comes by DMA, a wave's share: k; the factors and values; T. A wave waits long at a burst of these: T in two
    // stages is asked for by the waves that carry the state, the rest by those of the outputs
    auto k_at = [&](int c) { return L::kKStages == 2 ? (c & 1) * kQk : 0; };
    auto bring_k = [&](int c) { dma_pieces<W, kQk>(qk_buf(c), 0, lds0 + k_at(c), wc, lane); };
    auto bring_state = [&](int c) {
        dma_pieces<W, L::kFac>(v_buf(c), kT, lds0 + L::kFacAt, wc, lane);
        if constexpr (!L::kOwnRows) {
            constexpr int kPer = 1024 / kRow;          // rows in 1 KB
            const __amdgpu_buffer_rsrc_t r = rows_buf(c);
            const uint32_t off = (uint32_t)(lane / (kRow / 16)) * ldv + (uint32_t)(it0.block * kRow + lane % (kRow / 16) * 16);
#pragma unroll
            for (int i = 0; i < kC / kPer / W; ++i) {
                const uint32_t q = (uint32_t)(wc + W * i);
                dma16(r, off + q * kPer * ldv, 0, __builtin_amdgcn_readfirstlane(lds0 + L::kRowsAt + q * 1024));
            }
        }
    };
    auto t_at = [&](int c) { return L::kTAt + (L::kTStages == 2 ? (c & 1) * kT : 0); };
    auto bring_t = [&](int c) { dma_pieces<W, kT>(v_buf(c), 0, lds0 + t_at(c), wc, lane); };
    // For the outputs, q and the factors again
    auto bring_q = [&](int c) {
        if (L::kDirect) return;
        dma_pieces<W, kQk>(qk_buf(c), kQk, lds0 + L::kQAt, wc, lane);
        dma_pieces<W, L::kFac>(v_buf(c), kT, lds0 + L::kOutFacAt, wc, lane);
    };
    // and the products of queries and keys
    auto bring_p = [&](int c) {
        if (!L::kDirect) dma_pieces<W, kP>(v_buf(c), kT + L::kFac, lds0 + L::kPAt, wc, lane);
    };
    char* hand = lds + L::kHandAt + wc * kHand;
    auto barrier = [&] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto meet = [&] {
        wait_lgkm0();
        barrier();
    };
    if (!carries) {
        if (n == 0) return;
        // behind the middle of chunk c, for the next one and c's outputs; behind the begin of c, for itself and the outputs of
        // the one before
        auto bring_next = [&](int c) {
            if (c + 1 < n) {
                if (L::kKStages == 2) bring_k(c + 1);
                bring_state(c + 1);
            }
            if (c < n) bring_p(c);
        };
        auto bring_now = [&](int c) {
            if (c < n) {
                if (L::kKStages == 1) bring_k(c);
                if (L::kTStages == 1) bring_t(c);
            }
            bring_q(c - 1);
        };
        bring_k(0);
        bring_state(0);
        bring_t(0);
        wait_vm<0>();
        meet();
        barrier();
        if (!on) {
            for (int c = 1; c <= n; ++c) {
                bring_next(c - 1);
                wait_vm<0>();
                meet();
                bring_now(c);
                wait_vm<0>();
                barrier();
            }
            return;
        }
        // O^T of 16 columns: rows are columns of the state, a lane's token is its column of the product
        const uint32_t ldo = (uint32_t)p.ld_out * sz;
        const uint32_t o0 = (uint32_t)(lane & 15) * ldo + (uint32_t)(c0 + 4 * hh) * sz;
        const char *s_q = lds + L::kQAt, *s_p = lds + L::kPAt;
        const float* s_fac = (const float*)(lds + L::kOutFacAt) + 2 * kC + (lane & 15);
        constexpr bool kDirect = L::kDirect;
        // steps of q that a wave holds from one chunk to the next, the others two steps in front of their use
        constexpr int kHold = !kDirect ? 0 : NS * PA <= 12 ? NS : 2, kRing = !kDirect ? 2 : kHold == NS ? NS : 3;
        constexpr int kAskQ = kHold * PA * 4, kAskP = kDirect ? kSplit * kFrags + 8 : 0;   // loads of them
        bf16x8 q[kRing][PA][4], P[kSplit][kFrags];
        float eg[4], cc[4];
        auto ask_q = [&](int c) {
#pragma unroll
            for (int s = 0; s < kHold; ++s) load_q<NS, PA>(q[s], qk_buf(c), kQk, s, lane);
        };
        auto ask_p = [&](int c) {
            if constexpr (kDirect) {
                load_p(P, v_buf(c), kT + L::kFac, lane);
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const int at = kT + (2 * kC + 16 * it) * 4;
                    eg[it] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(v_buf(c), (lane & 15) * 4, at, 0));
                    cc[it] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(v_buf(c), (lane & 15) * 4, at + kC * 4, 0));
                }
            }
        };
        ask_p(0);
        bring_next(0);
        ask_q(0);
        wait_vm<kAskQ>();
        for (int c = 1; c <= n; ++c) {
            wait_vm<kAskQ + 4>();                      // the next q, and the stores of the outputs, may be out
            meet();
            const int d = c - 1, nq = min(rows - d * kC, kC), next = min(c, n - 1);
            bring_now(c);
            f32x4 S[NT], U[4], Y[4], O[4];
            bf16x8 Sp[L::kFormed ? NS : 2][kSplit];
#pragma unroll
            for (int it = 0; it < 4; ++it) U[it] = *(const f32x4*)(hand + kHandS + it * 1024 + lane * 16);
            if constexpr (!kDirect) {
#pragma unroll
                for (int part = 0; part < kSplit; ++part)
#pragma unroll
                    for (int f = 0; f < kFrags; ++f) P[part][f] = *(const bf16x8*)(s_p + (part * kFrags + f) * 1024 + lane * 16);
            }
#pragma unroll
            for (int i = 0; i < kHandS / 1024; ++i) {
                if constexpr (L::kFormed) Sp[i / kSplit][i % kSplit] = *(const bf16x8*)(hand + i * 1024 + lane * 16);
                else S[i] = *(const f32x4*)(hand + i * 1024 + lane * 16);
            }
#pragma unroll
            for (int it = 0; it < 4; ++it) Y[it] = O[it] = f32x4{};
            // P U, and beside it the first operands of Q S
            bf16x8 Up[2][kSplit];
            split2(U[0], U[1], Up[0]);
            __builtin_amdgcn_sched_barrier(0);
            auto times_p = [&](int s) {
#pragma unroll
                for (int m = 0; m < kProducts; ++m)
#pragma unroll
                    for (int it = 2 * s; it < 4; ++it) Y[it] = mma(Up[s][first(m)], P[second(m)][frag_of(it, s)], Y[it]);
            };
            split2(U[2], U[3], Up[1]);
            times_p(0);
            interleave<kProducts * 4, 2>();
            if constexpr (!L::kFormed) split2(S[0], S[1], Sp[0]);
            times_p(1);
            interleave<kProducts * 2, 4>();
            float ce[4], co[4];
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                ce[it] = eg[it];
                co[it] = cc[it];
            }
            __builtin_amdgcn_sched_barrier(0);
            ask_p(next);
            if (!kDirect || L::kTStages == 1) wait_vm<kAskP>();
            meet();
            __builtin_amdgcn_sched_barrier(0);
            bring_next(c);
            const __amdgpu_buffer_rsrc_t ro = buffer_rsrc((T*)p.out + ((int64_t)lo + (int64_t)d * kC) * p.ld_out + h * p.dv,
                                                          (uint32_t)(nq - 1) * ldo + (uint32_t)p.dv * sz);
            if constexpr (!kDirect) {
#pragma unroll
                for (int part = 0; part < PA; ++part)
#pragma unroll
                    for (int it = 0; it < 4; ++it) q[0][part][it] = qk_piece<NS>(s_q, part, it, 0, lane);
            }
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                if (!kDirect && s + 1 < NS) {
#pragma unroll
                    for (int part = 0; part < PA; ++part)
#pragma unroll
                        for (int it = 0; it < 4; ++it) q[(s + 1) % kRing][part][it] = qk_piece<NS>(s_q, part, it, s + 1, lane);
                }
                if (kDirect && s + 2 >= kHold && s + 2 < NS) load_q<NS, PA>(q[(s + 2) % kRing], qk_buf(d), kQk, s + 2, lane);
                constexpr int kS = L::kFormed ? NS : 2;   // steps of S that there is room for
                if constexpr (!L::kFormed) {
                    if (s + 1 < NS) split2(S[2 * (s + 1 < NS ? s + 1 : s)], S[2 * (s + 1 < NS ? s + 1 : s) + 1], Sp[(s + 1) % kS]);
                }
                auto& qs = q[s % kRing];
#pragma unroll
                for (int m = 0; m < kProducts; ++m) {
                    if (second(m) >= PA) continue;
#pragma unroll
                    for (int it = 0; it < 4; ++it) O[it] = mma(Sp[s % kS][first(m)], qs[second(m)][it], O[it]);
                }
                interleave<(PA == 1 ? 12 : 24), (PA == 1 ? 4 : 2)>();
            }
            ask_q(next);
            asm volatile("" ::: "memory");
            if constexpr (!kDirect) {
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    ce[it] = s_fac[16 * it];
                    co[it] = s_fac[kC + 16 * it];
                }
            }
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                T o[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = from_f32<T>(co[it] * __builtin_fmaf(ce[it], O[it][r], Y[it][r]));
                if constexpr (sz == 4) {
                    u32x4 w;
                    __builtin_memcpy(&w, o, 16);
                    __builtin_amdgcn_raw_buffer_store_b128(w, ro, (int)(o0 + (uint32_t)(16 * it) * ldo), 0, 0);
                } else {
                    u32x2 w;
                    __builtin_memcpy(&w, o, 8);
                    __builtin_amdgcn_raw_buffer_store_b64(w, ro, (int)(o0 + (uint32_t)(16 * it) * ldo), 0, 0);
                }
            }
        }
        return;
    }
    float* state = p.pool + (((int64_t)(ok ? slot : 0) * p.Hv + h) * p.dv + (on ? c0 + (lane & 15) : 0)) * p.dk + 4 * hh;
    f32x4 S[NT];
    const bool carry = ok && p.has_init[seq];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        S[t] = f32x4{};
        if (carry && on && 16 * t < p.dk) S[t] = *(const f32x4*)(state + 16 * t);
    }
    // Steps whose operands are formed beside the products of the others; the others' behind the barrier, beside the first
    // reads
    constexpr int kEarly = 1;
    bf16x8 Sp[NS][kSplit];
    auto form = [&](int s0, int s1) {
#pragma unroll
        for (int s = s0; s < s1; ++s) split2(S[2 * s], S[2 * s + 1], Sp[s]);
    };
    form(0, kEarly);
    // the values of this lane's column, where they are not in LDS
    float own[4][4];
    auto ask_own = [&](int c) {
        if constexpr (L::kOwnRows) {
            static_assert(sz == 4, "float32 rows");
            const uint32_t at = (uint32_t)(4 * hh) * ldv + (uint32_t)(c0 + (lane & 15)) * sz;
#pragma unroll
            for (int it = 0; it < 4; ++it)
#pragma unroll
                for (int r = 0; r < 4; ++r) own[it][r] = buffer_load_f32(rows_buf(c), at + (uint32_t)(16 * it + r) * ldv);
        }
    };
    if (n > 0 && on) ask_own(0);
    for (int c = 0; c < n; ++c) {
        wait_vm<0>();
        meet();
        if (!on) {
            barrier();
            if (L::kTStages == 2 && c + 1 < n) bring_t(c + 1);
            continue;
        }
        const char *s_k = lds + k_at(c), *s_t = lds + t_at(c);
        const float* fac = (const float*)(lds + L::kFacAt);
        // What is read from LDS is asked for well in front of its use, as nothing else hides its way: two k steps of k
        // ahead of their products, T behind the last of them, k transposed in front of the products with T
        bf16x8 K[2][PA][4], Tr[kSplit][kFrags];
        f32x4 bg[4], wg[4];
        auto read_k = [&](int s) {
#pragma unroll
            for (int part = 0; part < PA; ++part)
#pragma unroll
                for (int it = 0; it < 4; ++it) K[s & 1][part][it] = qk_piece<NS>(s_k, part, it, s, lane);
        };
        auto first_k = [&] {
            read_k(0);
            read_k(1);
        };
        if constexpr (L::kKStages == 2) first_k();
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            bg[it] = *(const f32x4*)&fac[16 * it + 4 * hh];
            wg[it] = *(const f32x4*)&fac[kC + 16 * it + 4 * hh];
        }
        const float decay = fac[kFacDecay];
        // V of this lane's column, tokens 16 it + 4 hh + r
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4* lds4;
        const char* s_v = lds + L::kRowsAt + wc * 16 * (int)sizeof(T);
        float v[4][4];
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            if constexpr (L::kOwnRows) {
#pragma unroll
                for (int r = 0; r < 4; ++r) v[it][r] = own[it][r];
            } else if constexpr (PA == 1) {
                const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds4)(s_v + (16 * it + 4 * hh + ((lane & 15) >> 2)) * kRow + (lane & 3) * 8));
#pragma unroll
                for (int r = 0; r < 4; ++r) v[it][r] = (float)__builtin_bit_cast(bf16, (short)x[r]);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) v[it][r] = *(const float*)(s_v + (16 * it + 4 * hh + r) * kRow + (lane & 15) * 4);
            }
        }
        if (c == n - 1) {                              // what lies behind the sequence is no value of it
#pragma unroll
            for (int it = 0; it < 4; ++it)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (16 * it + 4 * hh + r >= rows - c * kC) v[it][r] = 0.0f;
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (L::kKStages == 1) {              // k arrives by now
            meet();
            __builtin_amdgcn_sched_barrier(0);
            first_k();
        }

        // K S, and beside it the operands of the next step, at last of the first half of R
        f32x4 R[4];
        bf16x8 Rp[2][kSplit];
        constexpr int kN = PA == 1 ? 3 : kProducts;    // products of a value of k and one in parts
#pragma unroll
        for (int it = 0; it < 4; ++it) R[it] = f32x4{};
        auto times_s = [&](int s, int i0, int i1) {
#pragma unroll
            for (int m = 0; m < kProducts; ++m) {
                if (first(m) >= PA) continue;
#pragma unroll
                for (int it = i0; it < i1; ++it) R[it] = mma(K[s & 1][first(m)][it], Sp[s][second(m)], R[it]);
            }
        };
        auto part_r = [&](int s) {
#pragma unroll
            for (int it = 2 * s; it < 2 * s + 2; ++it)
#pragma unroll
                for (int r = 0; r < 4; ++r) R[it][r] = __builtin_fmaf(-bg[it][r], R[it][r], v[it][r]);
            split2(R[2 * s], R[2 * s + 1], Rp[s]);
        };
#pragma unroll
        for (int s = 0; s + 1 < NS; ++s) {
            form(s + 1, s + 2);
            times_s(s, 0, 4);
            interleave<4 * kN, (PA == 1 ? 4 : 2)>();
            if (s + 2 < NS) read_k(s + 2);
        }
        auto read_t = [&] {
#pragma unroll
            for (int part = 0; part < kSplit; ++part)
#pragma unroll
                for (int f = 0; f < kFrags; ++f) Tr[part][f] = *(const bf16x8*)(s_t + (part * kFrags + f) * 1024 + lane * 16);
        };
        if constexpr (L::kTStages == 2) read_t();
        times_s(NS - 1, 0, 2);
        __builtin_amdgcn_sched_barrier(0);
        times_s(NS - 1, 2, 4);
        part_r(0);
        interleave<2 * kN, (PA == 1 ? 8 : 4)>();
        if constexpr (L::kKStages == 2) barrier();
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (L::kTStages == 1) read_t();
        // k transposed, in groups of tiles, for tokens 0 .. 31 and then the others
        constexpr int kG = PA == 1 ? NT : NT % 4 == 0 ? 4 : 2, kGroups = NT / kG;
        bf16x8 Kt[2][PA][kG];
        auto read_kt = [&](int i) {
#pragma unroll
            for (int part = 0; part < PA; ++part)
#pragma unroll
                for (int t = 0; t < kG; ++t) Kt[i & 1][part][t] = kt_piece<NS>(s_k, part, i / kGroups, i % kGroups * kG + t, lane);
        };
#pragma unroll
        for (int i = 0; i < kHandS / 1024; ++i) {
            if constexpr (L::kFormed) *(bf16x8*)(hand + i * 1024 + lane * 16) = Sp[i / kSplit][i % kSplit];
            else *(f32x4*)(hand + i * 1024 + lane * 16) = S[i];
        }
        read_kt(0);
        __builtin_amdgcn_sched_barrier(0);
        // U = T R, W = e^(G_C - G) U. Tokens 0 .. 31 run ahead of the others
        f32x4 U[4];
        bf16x8 Wp[2][kSplit];
#pragma unroll
        for (int it = 0; it < 4; ++it) U[it] = f32x4{};
        auto times_r = [&](int s) {
#pragma unroll
            for (int m = 0; m < kProducts; ++m)
#pragma unroll
                for (int it = 2 * s; it < 4; ++it) U[it] = mma(Tr[first(m)][frag_of(it, s)], Rp[s][second(m)], U[it]);
        };
        auto part_w = [&](int s) {
            f32x4 x[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                *(f32x4*)(hand + kHandS + (2 * s + i) * 1024 + lane * 16) = U[2 * s + i];
#pragma unroll
                for (int r = 0; r < 4; ++r) x[i][r] = U[2 * s + i][r] * wg[2 * s + i][r];
            }
            split2(x[0], x[1], Wp[s]);
        };
        // S <- e^(G_C) S + K^T W, tiles t0 .. t1 of a group
        auto grow = [&](int i, int t0, int t1) {
#pragma unroll
            for (int m = 0; m < kProducts; ++m) {
                if (first(m) >= PA) continue;
#pragma unroll
                for (int t = t0; t < t1; ++t)
                    S[i % kGroups * kG + t] = mma(Kt[i & 1][first(m)][t], Wp[i / kGroups][second(m)], S[i % kGroups * kG + t]);
            }
        };
        part_r(1);
        if (c + 1 < n) ask_own(c + 1);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] *= decay;
        times_r(0);
        interleave<4 * kProducts, 4>();
        part_w(0);
        times_r(1);
        interleave<2 * kProducts, 4>();
        if (L::kTStages == 2 && c + 1 < n) bring_t(c + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 2 * kGroups; ++i) {
            constexpr int kM = kG * kN, kRest = kG > 2 ? kM - 2 * kN : 1;
            if (i + 1 < 2 * kGroups) read_kt(i + 1);
            if (i == 0) part_w(1);
            if (kGroups == 1 && i == 1) {              // the first operands of the next chunk beside the last products
                grow(1, 0, 2);
                __builtin_amdgcn_sched_barrier(0);
                form(0, 1);
                grow(1, 2, kG);
                interleave<kRest, (50 + kRest - 1) / kRest>();
            } else {
                if (i == kGroups + 1) form(0, 1);
                grow(i, 0, kG);
                interleave<kM, (60 + kM - 1) / kM>();
            }
        }
    }
    if (n > 0) {
        meet();
        barrier();
    }
    if (ok && on) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (16 * t >= p.dk) break;
            *(f32x4*)(state + 16 * t) = S[t];
        }
    }
}

// k steps of 32 that the kernels are built for
int steps_of(int dk) {
    const int n = (dk + 31) / 32;
    return n <= 2 ? 2 : n <= 4 ? n : n <= 6 ? 6 : 8;
}

DeltaWs layout(char* scratch, bool bf16_act, int Hk, int Hv, int dk, int64_t T, int nseq, size_t* total) {
    DeltaWs w{};
    const int parts = bf16_act ? kParts<bf16> : kParts<float>;
    w.slots = (int)(T / kC) + nseq;
    size_t off = 0;
    auto take = [&](size_t bytes) { char* q = scratch ? scratch + off : nullptr; off += align256(bytes); return q; };
    w.base = (int32_t*)take((size_t)nseq * 4);
    w.count = (int32_t*)take(4);
    w.plan = (int2*)take((size_t)w.slots * 8);
    w.qk = take((size_t)w.slots * Hk * 2 * qk_bytes(steps_of(dk), parts));
    w.v = take((size_t)w.slots * Hv * v_bytes());
    *total = off;
    return w;
}

template <typename T, int NS, int W> void split_launch(const Args& a, hipStream_t s) {
    const dim3 grid = work_grid(a.d, (a.d.dv + 16 * W - 1) / (16 * W));
    // LDS is asked for at the launch: a kernel that the compiler sees to fill it alone has half of its registers where only
    // MFMAs reach them, and a move for every value that goes between the two
    SSM_LAUNCH((delta_split_kernel<T, NS, W>), grid, dim3(128 * W), (SplitLds<T, NS, W>::kBytes), s, a);
}
template <typename T, int NS> hipError_t prefill_launch(const Args& a, hipStream_t s) {
    const DeltaArgs& p = a.d;
    if (p.nseq > kFindSeqs) {
        KernelTimer kt("delta.plan", s);
        SSM_LAUNCH(delta_plan_kernel, dim3(1), dim3(256), 0, s, a);
    }
    {
        KernelTimer kt("delta.chunk", s);
        const dim3 grid((unsigned)a.w.slots, (unsigned)p.Hk);
        if (p.rep == 1) SSM_LAUNCH((delta_chunk_kernel<T, NS, 1>), grid, dim3(256), 0, s, a);
        else SSM_LAUNCH((delta_chunk_kernel<T, NS, 2>), grid, dim3(256), 0, s, a);
    }
    // Two waves of columns to a workgroup where all of these run at once, a compute unit each; else in bf16 four, which share
    // what they read (float32 stages leave no LDS for four). 16 heads of 128 x 128 over prompts of 1024 tokens, whole call:
    // 4 prompts (256 workgroups of two) 63 us by twos and 80 by fours, 6 prompts 96 and 81, 24 prompts 360 and 285
    KernelTimer kt("delta.main", s);
    const int64_t pairs = (int64_t)p.nseq * p.Hv, by_two = pairs * ((p.dv + 31) / 32);
    constexpr bool by_four = sizeof(T) == 2 && SplitLds<T, NS, 4>::kMode < 2;
    if constexpr (by_four) {
        if (by_two > 256 && p.dv > 32) {
            split_launch<T, NS, 4>(a, s);
            return hipGetLastError();
        }
    }
    split_launch<T, NS, 2>(a, s);
    return hipGetLastError();
}
template <typename T> hipError_t prefill_steps(const Args& a, hipStream_t s) {
    switch (steps_of(a.d.dk)) {
        case 2: return prefill_launch<T, 2>(a, s);
        case 3: return prefill_launch<T, 3>(a, s);
        case 4: return prefill_launch<T, 4>(a, s);
        case 6: return prefill_launch<T, 6>(a, s);
        default: return prefill_launch<T, 8>(a, s);
    }
}

}  // namespace

size_t delta_prefill_scratch_bytes(bool bf16_act, int Hk, int Hv, int dk, int, int64_t T, int nseq) {
    size_t total;
    layout(nullptr, bf16_act, Hk, Hv, dk, T, nseq, &total);
    return total;
}

hipError_t launch_delta_prefill(const DeltaArgs& p, bool bf16_act, hipStream_t s) {
    if (p.nseq <= 0) return hipSuccess;
    size_t total;
    const Args a{p, layout(p.scratch, bf16_act, p.Hk, p.Hv, p.dk, p.T, p.nseq, &total)};
    return bf16_act ? prefill_steps<bf16>(a, s) : prefill_steps<float>(a, s);
}

}  // namespace ssm
