// Prompts of the gated delta rule, in chunks of 64 tokens on the matrix cores. Per value head, with the state S
// (dk x dv here), G the running sum of log alpha in the chunk, K the keys as they are staged and kappa_i what makes row i
// of them the token's key:
//   A_ij = beta_i e^(Gi - Gj) kappa_i kappa_j k_i . k_j (j < i),  T = kappa (I + A)^-1 beta        no state in it
//   R = V - kappa e^G (K S),  U = T R,  O = c e^G (Q S) + (c_i e^(Gi - Gj) q_i . k_j)_{j <= i} U
//   S <- e^(G_C) S + K^T (e^(G_C - Gj) U)
// (c: the queries' lengths and the output's scale.) Pass 1 (delta_chunk_kernel) has a workgroup per chunk and q/k head:
// T and the masked products of queries and keys of its value heads. Pass 2 walks a sequence's chunks with the state in
// accumulators: columns of S need nothing of each other, so a wave owns 16 of them and waits for no sum of another.
// delta_split_kernel gives the outputs waves of their own where its LDS suffices, delta_main_kernel has one kind of wave.
// Longer chunks than 64 tokens would have fewer steps in the chain, but more work in the inversion and in the products
// with T; shorter ones more steps, each with the same waits.
//
// Operands are f16, sums float32. A row of k or q is scaled by the power of two that takes its largest value to 1
// or to 2^12, which holds bf16 values exactly (those of k down to 2^-14 of the row's largest, smaller ones to 2^-25 of
// it); float32 ones are two f16 values, 22 bits or 2^-25 of the largest. What is computed (S, R, U) is scaled by column
// in the same way and split in two where it carries the state on; a product of two splits is three MFMAs, off by 2^-22.
// Where only an output that will be rounded to bf16 depends on it, the first f16 value alone (2^-11) stands for S, U and
// the products of queries and keys.
#include <algorithm>

#include "gate.h"

namespace ssm {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr int kC = 64;           // tokens per chunk
constexpr int kFrags = 6;        // 16 x 32 pieces of a lower triangular 64 x 64 matrix
// factors for the state, by token: e^G kappa, e^(G_C - G); then e^(G_C), the scale of T, a bound of e^G |k|
constexpr int kFacDecay = 2 * kC, kFacT = 2 * kC + 1, kFacMax = 2 * kC + 2;
constexpr size_t kFacBytes = 1024, kOutFacBytes = 1024;   // and for the outputs: c e^G, c 2^8
constexpr int kFindSeqs = 256;   // more sequences are laid out by a launch of its own

// the parts of a stored q, k or product: float32 activations take two f16 values
template <typename T> constexpr int kParts = sizeof(T) == 4 ? 2 : 1;

// Piece (row tile it, k step s) of a lower triangle: rows 16 it .., columns 32 s ..
__host__ __device__ constexpr int frag_of(int it, int s) { return it < 2 ? it : 2 * it - 2 + s; }
// Operand layout of a 16 x 32 piece: lane l holds row l % 16 and, with hh = l / 16, columns 4 hh .. 4 hh + 3 and
// 16 + 4 hh .. 16 + 4 hh + 3: the order in which two stacked accumulator tiles hold their rows. Pieces of q and k
// have their rows rotated by 4 hh, so that the transposing reads of k meet every bank once.
__device__ __forceinline__ int qk_unit(int row, int hh) { return 16 * hh + ((row + 4 * hh) & 15); }

// Sizes of the workspace. Per chunk and q/k head: pieces of k, then of q; per chunk and value head: kappa T beta (two
// parts) and the state's factors, then the products of queries and keys and the outputs' factors.
constexpr size_t qk_bytes(int NS, int parts) { return (size_t)4 * NS * parts * 1024; }   // k or q
constexpr size_t t_bytes() { return (size_t)kFrags * 2 * 1024 + kFacBytes; }                            // for the state
constexpr size_t p_bytes(int parts) { return (size_t)kFrags * parts * 1024 + kOutFacBytes; }           // for the outputs
constexpr size_t v_bytes(int parts) { return t_bytes() + p_bytes(parts); }

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

// The largest of the wave's values, none of them negative (their bits compare like they do)
__device__ __forceinline__ float wave_max(float v) {
    int c = __builtin_bit_cast(int, v);
    c = max(c, dpp<0x111, 0xF>(c));
    c = max(c, dpp<0x112, 0xF>(c));
    c = max(c, dpp<0x114, 0xF>(c));
    c = max(c, dpp<0x118, 0xF>(c));
    c = max(c, dpp<0x142, 0xA>(c));
    c = max(c, dpp<0x143, 0xC>(c));
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(c, 63));
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
// The exponent of m's scale: m pow2(scale_exp(m)) lies in [2^12, 2^13); 0 and what is too small or not finite get one
// that keeps all factors finite
__device__ __forceinline__ int scale_exp(float m) {
    const int e = (int)((__builtin_bit_cast(uint32_t, m) >> 23) & 255u);
    return 12 + 127 - min(max(e, 40), 230);
}

template <int N> __device__ __forceinline__ f16x8 pair_f16(const float (&v)[N], int at) {
    f16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (_Float16)v[at + e];
    return o;
}

__device__ __forceinline__ f32x4 mma(const f16x8& a, const f16x8& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
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

// The pieces of a row of q or k that this thread (c4 of four) holds: scaled to f16 parts in operand layout, to LDS. The
// row's largest value comes to 2^top. Returns the sum of squares of the row; e: the exponent of its scale.
template <typename T, int NS>
__device__ __forceinline__ float stage_row(const Piece<T> (&x)[NS], int row, int c4, int top, char* lds, int* e) {
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
    ss = quad_sum(ss);
    *e = scale_exp(quad_max(m)) - 12 + top;
    const float f = pow2(*e);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        float v[8];
        x[s].values(v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= f;
#pragma unroll
        for (int part = 0; part < kParts<T>; ++part) {
            const f16x8 h = pair_f16(v, 0);
            // values 0..3 of the piece are (hh, half) = (2 (c4 & 1), c4 / 2), values 4..7 the next hh
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                f16x4 o;
#pragma unroll
                for (int k = 0; k < 4; ++k) o[k] = h[4 * q + k];
                const int at = (((part * 4 + (row >> 4)) * NS + s) * 64 + qk_unit(row & 15, 2 * (c4 & 1) + q)) * 16 + (c4 >> 1) * 8;
                *(f16x4*)(lds + at) = o;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] -= (float)h[k];
        }
    }
    return ss;
}

template <int NS> __device__ __forceinline__ f16x8 qk_piece(const char* lds, int part, int it, int s, int lane) {
    return *(const f16x8*)(lds + (((part * 4 + it) * NS + s) * 64 + qk_unit(lane & 15, lane >> 4)) * 16);
}

// One workgroup per chunk and q/k head; its value heads two at a time, each inverted by two waves. What bounds it is the
// chain of its phases (rows to LDS, products, inversion by blocks, output), half of whose time is waits: 8 prompts of
// 2048 tokens, 16 bf16 value heads of 128 over 8, 53 us for 147 MB written, the matrix pipe 12% busy, LDS 18%; three
// workgroups to a compute unit for two took 63 us to 55. 4 x 16384 tokens, 924 MB, 180 us: HBM. A chunk of its own per value head read and multiplied the
// rows twice (4 x 16384 tokens: 274 us for 222).
// HB: value heads a pass, 1 where a q/k head has one. What a pass of two computes for a second head that is not there
// is not stored.
template <typename T, int NS, int HB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(kParts<T> * NS <= 8 ? 2 : 1))) void delta_chunk_kernel(Args a) {
    constexpr int PA = kParts<T>, kQk = (int)qk_bytes(NS, PA);
    // q's pieces, and once they are used the heads' matrices in their place
    constexpr int kMat = HB * kC * kLdA * 4;
    __shared__ __attribute__((aligned(16))) char s_k[kQk], s_q[kQk > kMat ? kQk : kMat];
    float(*s_t)[kC * kLdA] = (float(*)[kC * kLdA])s_q;
    __shared__ __attribute__((aligned(16))) float s_gh[HB][kC], s_gl[HB][kC], s_beta[HB][kC], s_kap[kC], s_c[kC], s_len[kC];
    __shared__ float s_max[HB][4];
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
    const float sk = stage_row<T, NS>(xk, row, c4, 0, s_k, &ek);
    const float sq = stage_row<T, NS>(xq, row, c4, 12, s_q, &eq);
    if (c4 == 0) {
        s_len[row] = sqrtf(sk) * pow2(ek);
        s_c[row] = p.scale * (p.qk_norm ? 1.0f / sqrtf(fmaxf(sq + p.eps, 1.2e-38f)) : 1.0f) * pow2(-eq);
        s_kap[row] = (p.qk_norm ? 1.0f / sqrtf(fmaxf(sk + p.eps, 1.2e-38f)) : 1.0f) * pow2(-ek);
    }
    __syncthreads();

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
    const float kap = s_kap[16 * it + (lane & 15)];
    f32x4 kk[2][2], kq[2][2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        if (n >= pieces) break;
        kk[n][0] = kk[n][1] = kq[n][0] = kq[n][1] = f32x4{};
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const f16x8 y = qk_piece<NS>(s_k, 0, it, s, lane), z = qk_piece<NS>(s_q, 0, it, s, lane);
            f16x8 yl{}, zl{};
            if constexpr (PA == 2) {
                yl = qk_piece<NS>(s_k, 1, it, s, lane);
                zl = qk_piece<NS>(s_q, 1, it, s, lane);
            }
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                if (q == 1 && n + 1 == pieces && !odd) break;
                const f16x8 x = qk_piece<NS>(s_k, 0, 2 * n + q, s, lane);
                kk[n][q] = mma(x, y, kk[n][q]);
                kq[n][q] = mma(x, z, kq[n][q]);
                if constexpr (PA == 2) {
                    const f16x8 xl = qk_piece<NS>(s_k, 1, 2 * n + q, s, lane);
                    kk[n][q] = mma(xl, y, kk[n][q]);
                    kq[n][q] = mma(xl, z, kq[n][q]);
                    kk[n][q] = mma(x, yl, kk[n][q]);
                    kq[n][q] = mma(x, zl, kq[n][q]);
                }
            }
        }
    }
    char* qk = a.w.qk + ((int64_t)slot * p.Hk + hk) * (2 * kQk);
#pragma unroll
    for (int n = 0; n < kQk / 4096; ++n) {
        const int u = (n * 256 + tid) * 16;
        *(u32x4*)(qk + u) = *(const u32x4*)(s_k + u);
        *(u32x4*)(qk + kQk + u) = *(const u32x4*)(s_q + u);
    }
    __syncthreads();

    for (int r0 = 0; r0 < p.rep; r0 += HB) {
        const int heads = min(HB, p.rep - r0);
        auto vout = [&](int b) { return a.w.v + ((int64_t)slot * p.Hv + hk * p.rep + r0 + b) * v_bytes(PA); };
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
                        x[b][4 * q + r] = j + r <= i ? kq[n][q][r] * ex * pow2(-8) : 0.0f;
                    }
                    *(f32x4*)&s_t[b][i * kLdA + j] = m;   // zeros above the diagonal, where this piece has them
                }
#pragma unroll
            for (int b = 0; b < HB; ++b) {
                if (b >= heads) break;
                char* to = vout(b) + t_bytes() + (frag_of(it, n) * 1024 + l * 16);
#pragma unroll
                for (int part = 0; part < PA; ++part) {
                    const f16x8 o = pair_f16(x[b], 0);
                    *(f16x8*)(to + part * kFrags * 1024) = o;
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[b][e] -= (float)o[e];
                }
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
            float *fac = (float*)(vout(b) + t_bytes() - kFacBytes), *f = (float*)(vout(b) + v_bytes(PA) - kOutFacBytes);
            const float gh = s_gh[b][lane], gl = s_gl[b][lane], ch = s_gh[b][kC - 1], cl = s_gl[b][kC - 1];
            const float eg = fast_exp2(gh + gl), bg = eg * s_kap[lane];
            fac[lane] = bg;
            fac[kC + lane] = fast_exp2((ch - gh) + (cl - gl));
            const float m = wave_max(bg * s_len[lane] * 1.001f);
            if (lane == 0) {
                fac[kFacDecay] = fast_exp2(ch + cl);
                fac[kFacMax] = m;
            }
            f[lane] = s_c[lane] * eg;
            f[kC + lane] = s_c[lane] * pow2(8);
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
        // kappa T beta, scaled by the power of two that takes its largest value to 2^12; wave w has row tile w
        float x[HB][2][8];
        const int l = place(), hh = l >> 4;
#pragma unroll
        for (int b = 0; b < HB; ++b) {
            float m = 0.0f;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                if (n >= pieces) break;
                const f32x4 v0 = row4(s_t[b], 16 * it, 32 * n, l), v1 = row4(s_t[b], 16 * it, 32 * n + 16, l);
                const f32x4 b0 = *(const f32x4*)&s_beta[b][32 * n + 4 * hh], b1 = *(const f32x4*)&s_beta[b][32 * n + 16 + 4 * hh];
                const bool two = odd || n + 1 < pieces;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[b][n][e] = v0[e] * b0[e] * kap;
                    x[b][n][4 + e] = two ? v1[e] * b1[e] * kap : 0.0f;
                    m = fmaxf(m, fmaxf(fabsf(x[b][n][e]), fabsf(x[b][n][4 + e])));
                }
            }
            m = wave_max(m);
            if (lane == 0) s_max[b][wave] = m;
        }
        __syncthreads();
#pragma unroll
        for (int b = 0; b < HB; ++b) {
            if (b >= heads) break;
            const int et = scale_exp(fmaxf(fmaxf(s_max[b][0], s_max[b][1]), fmaxf(s_max[b][2], s_max[b][3])));
            const float f = pow2(et);
            if (tid == 0) ((float*)(vout(b) + t_bytes() - kFacBytes))[kFacT] = pow2(-et);
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                if (n >= pieces) break;
                char* to = vout(b) + (frag_of(it, n) * 1024 + l * 16);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[b][n][e] *= f;
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    const f16x8 o = pair_f16(x[b][n], 0);
                    *(f16x8*)(to + part * kFrags * 1024) = o;
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[b][n][e] -= (float)o[e];
                }
            }
        }
    }
}

// ---------------------------------------------------------------- pass 2
// Values of this lane's column: their largest magnitude over the column's four lanes
__device__ __forceinline__ float column_max(float m) {
    const uint32_t v = __builtin_bit_cast(uint32_t, m);
    const auto x = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    const uint32_t w = __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, (uint32_t)x[0]), __builtin_bit_cast(float, (uint32_t)x[1])));
    const auto y = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)y[0]), __builtin_bit_cast(float, (uint32_t)y[1]));
}
template <int N> __device__ __forceinline__ float largest(const f32x4 (&v)[N]) {
    float m = 0.0f;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) m = fmaxf(m, fabsf(v[t][r]));
    return m;
}
// Two stacked tiles, times f (a power of two), as an operand: its first f16 values, and what they leave. SCALED false: f is
// one, though the compiler does not know it. Of two values that are left the first goes through an empty statement, which
// makes one instruction of each (a product, a difference and a rounding), where their conversion as a pair would
// take three
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
template <bool LO, bool SCALED = true>
__device__ __forceinline__ void split2(const f32x4& x0, const f32x4& x1, float f, f16x8& hi, f16x8& lo) {
#pragma unroll
    for (int r = 0; r < 8; r += 2) {
        const float a = r < 4 ? x0[r] : x1[r - 4], b = r < 4 ? x0[r + 1] : x1[r - 3];
        const f16x2 h = __builtin_convertvector((f32x2){SCALED ? a * f : a, SCALED ? b * f : b}, f16x2);
        hi[r] = h[0];
        hi[r + 1] = h[1];
        if constexpr (LO) {
            _Float16 l = (_Float16)__builtin_fmaf(a, f, -(float)h[0]);
            asm("" : "+v"(l));
            lo[r] = l;
            lo[r + 1] = (_Float16)__builtin_fmaf(b, f, -(float)h[1]);
        }
    }
}

// What pass 2 holds in LDS: two stages of a chunk's k, masked products and factors, and of its q where they fit
// (kQStages 2); else one of q (1); else a single stage of everything, waited for in full (0).
constexpr size_t kLds = 160 * 1024;
template <typename T, int NS> struct MainLds {
    static constexpr int kQk = (int)qk_bytes(NS, kParts<T>), kV = (int)v_bytes(kParts<T>);
    static constexpr int kQStages = 2 * (2 * kQk + kV) <= (int)kLds ? 2 : 2 * (kQk + kV) + kQk <= (int)kLds ? 1 : 0;
    static constexpr int kStages = kQStages > 0 ? 2 : 1;
    static constexpr int kBytes = kStages * (kQk + kV) + (kQStages == 2 ? 2 : 1) * kQk;
    static_assert(kBytes <= (int)kLds, "pass 2 does not fit into LDS");
};

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

// One value of a row of T, zero (and nothing stored) behind the buffer's end
template <typename T> struct Raw;
template <> struct Raw<float> {
    typedef uint32_t type;
    static __device__ __forceinline__ type load(const __amdgpu_buffer_rsrc_t& r, uint32_t off) { return __builtin_amdgcn_raw_buffer_load_b32(r, (int)off, 0, 0); }
    static __device__ __forceinline__ void store(const __amdgpu_buffer_rsrc_t& r, uint32_t off, float v) {
        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), r, (int)off, 0, 0);
    }
    static __device__ __forceinline__ float value(type v) { return __builtin_bit_cast(float, v); }
};
template <> struct Raw<bf16> {
    typedef uint16_t type;
    static __device__ __forceinline__ type load(const __amdgpu_buffer_rsrc_t& r, uint32_t off) { return __builtin_amdgcn_raw_buffer_load_b16(r, (int)off, 0, 0); }
    static __device__ __forceinline__ void store(const __amdgpu_buffer_rsrc_t& r, uint32_t off, float v) {
        __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, (bf16)v), r, (int)off, 0, 0);
    }
    static __device__ __forceinline__ float value(type v) { return (float)__builtin_bit_cast(bf16, v); }
};

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

// While a chunk is computed the next one's pieces and values are on their way, and the stores of its outputs stay out
// at the wait in front of the next: every wave waits for its own share, then the barrier stands for the others'.
// Bound by a chunk's chain of products and of the vector instructions that scale and split between them: 317, 1130 and
// 601 float32 tokens, 16 heads of 128 x 128, 73 us, 4.0 us a chunk of the longest; with staging in front of each
// chunk instead of beside it bf16 took 185 us for 62.
template <typename T, int NS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(NS <= 4 ? 2 : 1))) void delta_main_kernel(Args a) {
    constexpr int PA = kParts<T>, NT = 2 * NS;
    using L = MainLds<T, NS>;
    constexpr int kQk = L::kQk, kV = L::kV;
    constexpr uint32_t sz = sizeof(T);
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const DeltaArgs& p = a.d;
    const int tid = threadIdx.x, lane = tid & 63, hh = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const WorkItem it0 = work_item(p, (p.dv + 16 * WAVES - 1) / (16 * WAVES));
    if (it0.seq >= p.nseq) return;
    const int seq = it0.seq, h = it0.head, hk = h / p.rep, c0 = (it0.block * WAVES + wave) * 16;   // this wave's columns
    const bool on = c0 < p.dv;
    const SeqRows sr = seq_rows(p, seq);
    const int lo = __builtin_amdgcn_readfirstlane(sr.lo), rows = __builtin_amdgcn_readfirstlane(sr.n);
    const int slot = p.slot[seq], n = chunks_of(rows), base = rows > 0 ? __builtin_amdgcn_readfirstlane(a.w.base[seq]) : 0;
    const bool fits = sr.ok && base + n <= a.w.slots, ok = slot >= 0 && slot < p.S;
    if (h == 0 && it0.block == 0 && tid == 0 && (!fits || !ok))
        atomicOr(p.status, (fits ? 0 : SSM_STATUS_BAD_SEQLENS) | (ok ? 0 : SSM_STATUS_BAD_SLOT));
    if (!fits) return;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
    // places of a stage: k and the masked products by stage, q behind them
    auto k_at = [&](int c) { return (L::kStages == 2 ? (c & 1) : 0) * (kQk + kV); };
    auto q_at = [&](int c) { return L::kStages * (kQk + kV) + (L::kQStages == 2 ? (c & 1) : 0) * kQk; };
    auto qk_buf = [&](int c) { return buffer_rsrc(a.w.qk + ((int64_t)(base + c) * p.Hk + hk) * (2 * kQk), 2 * kQk); };
    auto bring = [&](int c) {
        dma_pieces<WAVES, kQk>(qk_buf(c), 0, lds0 + k_at(c), wave, lane);
        dma_pieces<WAVES, kV>(buffer_rsrc(a.w.v + ((int64_t)(base + c) * p.Hv + h) * kV, kV), 0, lds0 + k_at(c) + kQk, wave, lane);
    };
    auto bring_q = [&](int c) { dma_pieces<WAVES, kQk>(qk_buf(c), kQk, lds0 + q_at(c), wave, lane); };
    // V of this lane's column, tokens 16 it + 4 hh + r
    typename Raw<T>::type raw[4][4];
    const uint32_t ldv = (uint32_t)p.ld * sz, ldo = (uint32_t)p.ld_out * sz;
    const uint32_t v0 = on ? (uint32_t)(4 * hh) * ldv + (uint32_t)(c0 + (lane & 15)) * sz : kOffOutOfRange;
    const uint32_t o0 = (uint32_t)(4 * hh) * ldo + (uint32_t)(c0 + (lane & 15)) * sz;
    auto bring_v = [&](int c) {
        const int nq = min(rows - c * kC, kC);
        const __amdgpu_buffer_rsrc_t r = buffer_rsrc((const T*)p.qkv + ((int64_t)lo + (int64_t)c * kC) * p.ld + 2 * p.Hk * p.dk + h * p.dv,
                                                     (uint32_t)(nq - 1) * ldv + (uint32_t)p.dv * sz);
#pragma unroll
        for (int it = 0; it < 4; ++it)
#pragma unroll
            for (int k = 0; k < 4; ++k) raw[it][k] = Raw<T>::load(r, v0 + (uint32_t)(16 * it + k) * ldv);
    };
    if (n > 0) {
        bring(0);
        bring_q(0);
        bring_v(0);
    }
    float* state = p.pool + (((int64_t)(ok ? slot : 0) * p.Hv + h) * p.dv + (on ? c0 + (lane & 15) : 0)) * p.dk + 4 * hh;
    f32x4 S[NT];
    const bool carry = ok && p.has_init[seq];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        S[t] = f32x4{};
        if (carry && on && 16 * t < p.dk) S[t] = *(const f32x4*)(state + 16 * t);
    }
    float unit = 1.0f;                                 // S times this power of two is the state
    for (int c = 0; c < n; ++c) {
        // the outputs' 16 stores are the youngest where everything of this chunk was asked for in front of them
        if (L::kQStages == 2 && on && c > 0) wait_vm<16>();
        else wait_vm<0>();
        wait_lgkm0();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        float v[4][4];
#pragma unroll
        for (int it = 0; it < 4; ++it)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[it][k] = Raw<T>::value(raw[it][k]);
                asm volatile("" : "+v"(v[it][k]));     // taken here, in front of the loads for the next chunk
            }
        if (L::kStages == 2 && c + 1 < n) {
            bring(c + 1);
            if (L::kQStages == 2) bring_q(c + 1);
            bring_v(c + 1);
        }
        const char* s_k = lds + k_at(c);
        const char* s_v = s_k + kQk;
        const char* s_q = lds + q_at(c);
        if (on) {
            const int nq = min(rows - c * kC, kC);
            const float *fac = (const float*)(s_v + t_bytes() - kFacBytes), *ofac = (const float*)(s_v + v_bytes(PA) - kOutFacBytes);
            auto tok4 = [&](const float* f, int k, int it) { return *(const f32x4*)&f[k * kC + 16 * it + 4 * hh]; };
            auto tri = [&](const char* m, int part, int it, int s) { return *(const f16x8*)(m + (part * kFrags + frag_of(it, s)) * 1024 + lane * 16); };

            // K S, and Q S for the outputs, whose products run while R is formed
            f16x8 Sh[NS], Sl[NS];
            const float ms = column_max(largest(S));
            const int es = scale_exp(ms);
#pragma unroll
            for (int s = 0; s < NS; ++s) split2<true>(S[2 * s], S[2 * s + 1], pow2(es), Sh[s], Sl[s]);
            const float fs = unit * pow2(-es);
            f32x4 R[4], O[4];
#pragma unroll
            for (int it = 0; it < 4; ++it) R[it] = O[it] = f32x4{};
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                f16x8 k[PA][4];
#pragma unroll
                for (int part = 0; part < PA; ++part)
#pragma unroll
                    for (int it = 0; it < 4; ++it) k[part][it] = qk_piece<NS>(s_k, part, it, s, lane);
#pragma unroll
                for (int it = 0; it < 4; ++it) R[it] = mma(k[0][it], Sh[s], R[it]);
#pragma unroll
                for (int it = 0; it < 4; ++it) R[it] = mma(k[0][it], Sl[s], R[it]);
                if constexpr (PA == 2) {
#pragma unroll
                    for (int it = 0; it < 4; ++it) R[it] = mma(k[PA - 1][it], Sh[s], R[it]);
                }
            }
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                f16x8 q[PA][4];
#pragma unroll
                for (int part = 0; part < PA; ++part)
#pragma unroll
                    for (int it = 0; it < 4; ++it) q[part][it] = qk_piece<NS>(s_q, part, it, s, lane);
#pragma unroll
                for (int it = 0; it < 4; ++it) O[it] = mma(q[0][it], Sh[s], O[it]);
                if constexpr (PA == 2) {
#pragma unroll
                    for (int it = 0; it < 4; ++it) O[it] = mma(q[0][it], Sl[s], O[it]);
#pragma unroll
                    for (int it = 0; it < 4; ++it) O[it] = mma(q[PA - 1][it], Sh[s], O[it]);
                }
            }
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const f32x4 bg = tok4(fac, 0, it);
#pragma unroll
                for (int r = 0; r < 4; ++r) R[it][r] = v[it][r] - bg[r] * (R[it][r] * fs);
            }
            // U = T R
            const int er = scale_exp(column_max(largest(R)));
            f16x8 Rh[2], Rl[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) split2<true>(R[2 * s], R[2 * s + 1], pow2(er), Rh[s], Rl[s]);
            f32x4 U[4], W[4];
            const float fr = pow2(-er) * fac[kFacT];
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                f32x4 x{};
#pragma unroll
                for (int s = 0; s <= it / 2; ++s) {
                    const f16x8 th = tri(s_v, 0, it, s), tl = tri(s_v, 1, it, s);
                    x = mma(th, Rh[s], x);
                    x = mma(th, Rl[s], x);
                    x = mma(tl, Rh[s], x);
                }
                const f32x4 w = tok4(fac, 1, it);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    U[it][r] = x[r] * fr;
                    W[it][r] = U[it][r] * w[r];
                }
            }
            // S <- decay S + K^T W, in the units of W's scale; a state far above W keeps the scale in range
            const float decay = fac[kFacDecay];
            const float mw = column_max(largest(W));
            const int ew = scale_exp(fmaxf(mw, ms * unit * decay * pow2(-10)));
            f16x8 Wh[2], Wl[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) split2<true>(W[2 * s], W[2 * s + 1], pow2(ew), Wh[s], Wl[s]);
            const float keep = decay * unit * pow2(ew);
            unit = pow2(-ew);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int r = 0; r < 4; ++r) S[t][r] *= keep;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    // rows dk = 16 t + lane % 16 of K^T, tokens 32 s + 4 hh .. and 32 s + 16 + 4 hh ..: four rows of
                    // 16 values of k, transposed as they are read
                    typedef short s16x4 __attribute__((ext_vector_type(4)));
                    typedef __attribute__((address_space(3))) s16x4* lds4;
#pragma unroll
                    for (int part = 0; part < PA; ++part) {
                        s16x4 k2[2];
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const char* at = s_k + (((part * 4 + 2 * s + q) * NS + t / 2) * 64 +
                                                    qk_unit(4 * hh + ((lane & 15) >> 2), lane & 3)) * 16 + (t & 1) * 8;
                            k2[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)at);
                        }
                        const f16x8 k = __builtin_bit_cast(f16x8, __builtin_shufflevector(k2[0], k2[1], 0, 1, 2, 3, 4, 5, 6, 7));
                        S[t] = mma(k, Wh[s], S[t]);
                        if (part == 0) S[t] = mma(k, Wl[s], S[t]);
                    }
                }
            }
            // O = Q S + P U
            const int eu = scale_exp(column_max(largest(U)));
            f16x8 Uh[2], Ul[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) split2<PA == 2>(U[2 * s], U[2 * s + 1], pow2(eu), Uh[s], Ul[s]);
            const __amdgpu_buffer_rsrc_t ro = buffer_rsrc((T*)p.out + ((int64_t)lo + (int64_t)c * kC) * p.ld_out + h * p.dv,
                                                          (uint32_t)(nq - 1) * ldo + (uint32_t)p.dv * sz);
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                f32x4 y{};
#pragma unroll
                for (int s = 0; s <= it / 2; ++s) {
                    const f16x8 q = tri(s_v + t_bytes(), 0, it, s);
                    y = mma(q, Uh[s], y);
                    if constexpr (PA == 2) {
                        y = mma(q, Ul[s], y);
                        y = mma(tri(s_v + t_bytes(), 1, it, s), Uh[s], y);
                    }
                }
                const f32x4 ce = tok4(ofac, 0, it), cc = tok4(ofac, 1, it);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    Raw<T>::store(ro, o0 + (uint32_t)(16 * it + r) * ldo, ce[r] * (O[it][r] * fs) + cc[r] * (y[r] * pow2(-eu)));
            }
        }
        if (L::kQStages < 2 && c + 1 < n) {            // q (and, with one stage, everything) is read by now
            wait_lgkm0();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            bring_q(c + 1);
            if (L::kStages == 1) {
                bring(c + 1);
                bring_v(c + 1);
            }
        }
    }
    if (ok && on) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (16 * t >= p.dk) break;
            f32x4 o;
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = S[t][r] * unit;
            *(f32x4*)(state + 16 * t) = o;
        }
    }
}

// As delta_main_kernel, with the outputs by waves of their own: W waves carry the state, W more form the outputs of the
// chunk before from the operands that the first left in LDS. The chain from chunk to chunk is that much shorter, and
// both kinds run beside each other. Scales that need not be exact are bounds, known before what they scale:
// a bound loses headroom (f16 pairs hold 39 bits, 22 are used), not precision.
// 317, 1130 and 601 bf16 tokens, 16 heads of 128 x 128: 37.5 us, 2.1 us a chunk of the longest sequence (51 when it was
// built, 62 by delta_main_kernel then); 8 x 2048 tokens 98 us for 294 MB. Bound by the instructions of a chunk's chain
// (480 vector ones and 82 MFMAs of a wave that carries the state) with the next chunk's 55 KB on their way; matrix pipe
// 24% busy, LDS 34%. Touching the chunk after next for L2, loads by the waves that carry the state and other orders of
// the products gave nothing or cost time.
template <typename T, int NS, int W> struct SplitLds {
    static constexpr int kQk = (int)qk_bytes(NS, kParts<T>), kT = (int)t_bytes(), kP = (int)p_bytes(kParts<T>);
    static constexpr int kRow = 16 * W * (int)sizeof(T), kRows = kC * kRow;   // the workgroup's values of a token, of a chunk
    static constexpr int kHand = (NS + 2) * kParts<T> * 1024 + 256;           // S, U and their scales of 16 columns
    static constexpr int kStage = 2 * kQk + kT + kRows + (int)kOutFacBytes, kBytes = 2 * (kStage + W * kHand);
    static constexpr bool kFits = kBytes <= (int)kLds;
};

template <typename T, int NS, int W>
__global__ __launch_bounds__(128 * W) __attribute__((amdgpu_waves_per_eu(2))) void delta_split_kernel(Args a) {
    constexpr int PA = kParts<T>, NT = 2 * NS;
    using L = SplitLds<T, NS, W>;
    constexpr int kQk = L::kQk, kT = L::kT, kP = L::kP, kRow = L::kRow, kRows = L::kRows, kHand = L::kHand, kStage = L::kStage;
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
    // a stage: k, T and the state's factors, values; q and the outputs' factors; then what the waves hand over
    auto qk_buf = [&](int c) { return buffer_rsrc(a.w.qk + ((int64_t)(base + c) * p.Hk + hk) * (2 * kQk), 2 * kQk); };
    auto v_at = [&](int c) { return a.w.v + ((int64_t)(base + c) * p.Hv + h) * (kT + kP); };
    const uint32_t ldv = (uint32_t)p.ld * sz;
    // All that comes by DMA is asked for by the waves of the outputs: beside a burst of it a wave waits long to issue a load
    auto bring_state = [&](int c) {
        const uint32_t to = lds0 + (c & 1) * kStage;
        dma_pieces<W, kQk>(qk_buf(c), 0, to, wc, lane);
        dma_pieces<W, kT>(buffer_rsrc(v_at(c), kT), 0, to + kQk, wc, lane);
        const int nq = min(rows - c * kC, kC);
        const __amdgpu_buffer_rsrc_t r = buffer_rsrc((const T*)p.qkv + ((int64_t)lo + (int64_t)c * kC) * p.ld + 2 * p.Hk * p.dk + h * p.dv,
                                                     (uint32_t)(nq - 1) * ldv + (uint32_t)p.dv * sz);
        constexpr int kPer = 1024 / kRow;              // rows in 1 KB
        const uint32_t off = (uint32_t)(lane / (kRow / 16)) * ldv + (uint32_t)(it0.block * kRow + lane % (kRow / 16) * 16);
#pragma unroll
        for (int i = 0; i < kRows / 1024 / W; ++i) {
            const uint32_t q = (uint32_t)(wc + W * i);
            dma16(r, off + q * kPer * ldv, 0, __builtin_amdgcn_readfirstlane(to + kQk + kT + q * 1024));
        }
    };
    auto bring_out = [&](int c) {
        const uint32_t to = lds0 + (c & 1) * kStage + kQk + kT + kRows;
        dma_pieces<W, kQk>(qk_buf(c), kQk, to, wc, lane);
        dma_pieces<W, (int)kOutFacBytes>(buffer_rsrc(v_at(c) + kT + kP - kOutFacBytes, kOutFacBytes), 0, to + kQk, wc, lane);
    };
    auto hand = [&](int c) { return lds + 2 * kStage + ((c & 1) * W + wc) * kHand; };
    auto meet = [&] {
        wait_lgkm0();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    if (!carries) {
        if (n > 0) bring_state(0);
        // O^T of 16 columns: rows are columns of the state, a lane's token is its column of the product
        const uint32_t ldo = (uint32_t)p.ld_out * sz;
        const uint32_t o0 = (uint32_t)(lane & 15) * ldo + (uint32_t)(c0 + 4 * hh) * sz;
        f16x8 Pn[PA][kFrags];                          // the next products of queries and keys
        for (int c = 0; c <= n && n > 0; ++c) {
            if (on && c > 1) wait_vm<4>();             // but for the stores of the outputs
            else wait_vm<0>();
            f16x8 P[PA][kFrags];
#pragma unroll
            for (int part = 0; part < PA; ++part)
#pragma unroll
                for (int f = 0; f < kFrags; ++f) P[part][f] = Pn[part][f];
            meet();
            if (c + 1 < n) bring_state(c + 1);
            if (c < n) {
                bring_out(c);
                const char* from = v_at(c) + kT;
#pragma unroll
                for (int part = 0; part < PA; ++part)
#pragma unroll
                    for (int f = 0; f < kFrags; ++f) Pn[part][f] = *(const f16x8*)(from + (part * kFrags + f) * 1024 + lane * 16);
            }
            if (c == 0 || !on) continue;
            const int d = c - 1, nq = min(rows - d * kC, kC);
            const char *s_q = lds + (d & 1) * kStage + kQk + kT + kRows, *from = hand(d);
            const float *fac = (const float*)(s_q + kQk), *sc = (const float*)(from + (NS + 2) * PA * 1024);
            f16x8 S[PA][NS], U[PA][2];
#pragma unroll
            for (int part = 0; part < PA; ++part) {
#pragma unroll
                for (int s = 0; s < NS; ++s) S[part][s] = *(const f16x8*)(from + (part * NS + s) * 1024 + lane * 16);
#pragma unroll
                for (int s = 0; s < 2; ++s) U[part][s] = *(const f16x8*)(from + (PA * NS + part * 2 + s) * 1024 + lane * 16);
            }
            const f32x4 fs = *(const f32x4*)&sc[4 * hh], fu = *(const f32x4*)&sc[16 + 4 * hh];
            const __amdgpu_buffer_rsrc_t ro = buffer_rsrc((T*)p.out + ((int64_t)lo + (int64_t)d * kC) * p.ld_out + h * p.dv,
                                                          (uint32_t)(nq - 1) * ldo + (uint32_t)p.dv * sz);
            f32x4 O[4], Y[4];
#pragma unroll
            for (int it = 0; it < 4; ++it) O[it] = Y[it] = f32x4{};
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                f16x8 q[PA][4];
#pragma unroll
                for (int part = 0; part < PA; ++part)
#pragma unroll
                    for (int it = 0; it < 4; ++it) q[part][it] = qk_piece<NS>(s_q, part, it, s, lane);
#pragma unroll
                for (int it = 0; it < 4; ++it) O[it] = mma(S[0][s], q[0][it], O[it]);
                if constexpr (PA == 2) {
#pragma unroll
                    for (int it = 0; it < 4; ++it) O[it] = mma(S[PA - 1][s], q[0][it], O[it]);
#pragma unroll
                    for (int it = 0; it < 4; ++it) O[it] = mma(S[0][s], q[PA - 1][it], O[it]);
                }
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int it = 2 * s; it < 4; ++it) {
                    Y[it] = mma(U[0][s], P[0][frag_of(it, s)], Y[it]);
                    if constexpr (PA == 2) {
                        Y[it] = mma(U[PA - 1][s], P[0][frag_of(it, s)], Y[it]);
                        Y[it] = mma(U[0][s], P[PA - 1][frag_of(it, s)], Y[it]);
                    }
                }
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const float ce = fac[16 * it + (lane & 15)], cc = fac[kC + 16 * it + (lane & 15)];
                T o[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = from_f32<T>(ce * (O[it][r] * fs[r]) + cc * (Y[it][r] * fu[r]));
                if constexpr (PA == 2) {
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
    // S times unit (a power of two) is the state; |S| stays below 2^15, so that S itself is the pair of operands.
    // Tiles of which these are formed beside the products of the others; the others' behind the barrier, beside the first
    // reads
    constexpr int kEarly = NT / 4 * 2;
    float one = 1.0f;
    asm volatile("" : "+s"(one));
    float unit;
    {
        const int e = scale_exp(column_max(largest(S))) + 2;
        unit = pow2(-e);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] *= pow2(e);
    }
    f16x8 Sh[NS], Sl[NS];
    auto form = [&](int t0, int t1) {
#pragma unroll
        for (int t = t0; t < t1; t += 2) split2<true, false>(S[t], S[t + 1], one, Sh[t / 2], Sl[t / 2]);
    };
    form(0, kEarly);
    for (int c = 0; c <= n && n > 0; ++c) {
        meet();
        if (c == n || !on) continue;
        const char *s_k = lds + (c & 1) * kStage, *s_t = s_k + kQk;
        const float* fac = (const float*)(s_t + kT - kFacBytes);
        char* to = hand(c);
        // What is read from LDS is asked for well in front of its use, as nothing else hides its way: two k steps of k
        // ahead of their products, T behind the last of them, k transposed in front of the products with T
        f16x8 K[2][PA][4], Tr[2][kFrags];
        f32x4 bg[4], wg[4];
        auto read_k = [&](int s) {
#pragma unroll
            for (int part = 0; part < PA; ++part)
#pragma unroll
                for (int it = 0; it < 4; ++it) K[s & 1][part][it] = qk_piece<NS>(s_k, part, it, s, lane);
        };
        read_k(0);
        if (NS > 1) read_k(1);
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            bg[it] = *(const f32x4*)&fac[16 * it + 4 * hh];
            wg[it] = *(const f32x4*)&fac[kC + 16 * it + 4 * hh];
        }
        const float decay = fac[kFacDecay], tscale = fac[kFacT], gmax = fac[kFacMax];
        // V of this lane's column, tokens 16 it + 4 hh + r
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4* lds4;
        const char* s_v = s_t + kT + wc * 16 * (int)sizeof(T);
        float v[4][4];
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            if constexpr (PA == 1) {
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
        form(kEarly, NT);

        // K S beside all that does not wait for it
        f32x4 R[4];
#pragma unroll
        for (int it = 0; it < 4; ++it) R[it] = f32x4{};
        const float fs = unit;
        constexpr float kRoot = NS <= 2 ? 8.0f : NS <= 4 ? 11.4f : 16.0f;   // of 32 NS, or above it
        float ms, fu;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
#pragma unroll
            for (int it = 0; it < 4; ++it) R[it] = mma(K[s & 1][0][it], Sh[s], R[it]);
#pragma unroll
            for (int it = 0; it < 4; ++it) R[it] = mma(K[s & 1][0][it], Sl[s], R[it]);
            if constexpr (PA == 2) {
#pragma unroll
                for (int it = 0; it < 4; ++it) R[it] = mma(K[s & 1][PA - 1][it], Sh[s], R[it]);
            }
            if (s + 2 < NS) read_k(s + 2);
            if (s >= NS - 2) {
                const int part = s - (NS - 2);
#pragma unroll
                for (int f = 0; f < kFrags; ++f) Tr[part][f] = *(const f16x8*)(s_t + (part * kFrags + f) * 1024 + lane * 16);
            }
            *(f16x8*)(to + s * 1024 + lane * 16) = Sh[s];
            if constexpr (PA == 2) *(f16x8*)(to + (NS + s) * 1024 + lane * 16) = Sl[s];
            if (s == 0) {
                float vmax = 0.0f;
#pragma unroll
                for (int it = 0; it < 4; ++it)
#pragma unroll
                    for (int k = 0; k < 4; ++k) vmax = fmaxf(vmax, fabsf(v[it][k]));
                ms = column_max(largest(S));
                // a bound of R = V - e^G K S: |k . S| <= |k| sqrt(dk) max |S|
                const int er = scale_exp(column_max(vmax) + gmax * kRoot * (ms * unit));
                const float gr = pow2(er), cr = fs * gr;
                fu = pow2(-er) * tscale;
#pragma unroll
                for (int it = 0; it < 4; ++it)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        v[it][r] *= gr;
                        bg[it][r] *= -cr;
                    }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        // rows dk = 16 t + lane % 16 of K^T, tokens 32 s + 4 hh .. and 32 s + 16 + 4 hh ..: four rows of 16 values of k,
        // transposed as they are read
        f16x8 Kt[PA][2][NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int part = 0; part < PA; ++part) {
                    s16x4 k2[2];
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const char* at = s_k + (((part * 4 + 2 * s + q) * NS + t / 2) * 64 +
                                                qk_unit(4 * hh + ((lane & 15) >> 2), lane & 3)) * 16 + (t & 1) * 8;
                        k2[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)at);
                    }
                    Kt[part][s][t] = __builtin_bit_cast(f16x8, __builtin_shufflevector(k2[0], k2[1], 0, 1, 2, 3, 4, 5, 6, 7));
                }
        __builtin_amdgcn_sched_barrier(0);
        // From here tokens 0 .. 31 run ahead of the others: while the one half is in the matrix cores the other is formed.
        // U = kappa T beta R times 1 / fu, W = e^(G_C - G) U
        f16x8 Rh[2], Rl[2], Wh[2], Wl[2];
        f32x4 U[4], X[4];
#pragma unroll
        for (int it = 0; it < 4; ++it) U[it] = f32x4{};
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int it = 2 * s; it < 2 * s + 2; ++it)
#pragma unroll
                for (int r = 0; r < 4; ++r) R[it][r] = __builtin_fmaf(bg[it][r], R[it][r], v[it][r]);
            split2<true, false>(R[2 * s], R[2 * s + 1], one, Rh[s], Rl[s]);
#pragma unroll
            for (int it = 2 * s; it < 4; ++it) U[it] = mma(Tr[0][frag_of(it, s)], Rh[s], U[it]);
#pragma unroll
            for (int it = 2 * s; it < 4; ++it) U[it] = mma(Tr[0][frag_of(it, s)], Rl[s], U[it]);
#pragma unroll
            for (int it = 2 * s; it < 4; ++it) U[it] = mma(Tr[1][frag_of(it, s)], Rh[s], U[it]);
        }
        // The state's units: what is left of it and 64 products of W with values of k below 2 come to 2^15 at most. In bf16
        // W's largest value follows from R's (times the 64 of a row of T below 2^13) while the products run; in
        // float32, where a token's own precision is asked for, it is W's own
        float keep;
        auto units = [&](float most) {                 // of W
            const int ew = scale_exp(__builtin_fmaf(decay * ms, unit, most * pow2(7))) + 2;
            keep = decay * unit * pow2(ew);
            unit = pow2(-ew);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[t][r] *= keep;
            return pow2(ew);
        };
        float wc = fu;
        if constexpr (PA == 1) wc *= units(fu * pow2(19) * column_max(largest(R)));
#pragma unroll
        for (int it = 0; it < 4; ++it)
#pragma unroll
            for (int r = 0; r < 4; ++r) wg[it][r] *= wc;
        auto weigh = [&](int s) {
#pragma unroll
            for (int it = 2 * s; it < 2 * s + 2; ++it)
#pragma unroll
                for (int r = 0; r < 4; ++r) X[it][r] = U[it][r] * wg[it][r];
        };
        if constexpr (PA == 2) {
            weigh(0);
            weigh(1);
            const float f = units(column_max(largest(X)));
#pragma unroll
            for (int it = 0; it < 4; ++it)
#pragma unroll
                for (int r = 0; r < 4; ++r) X[it][r] *= f;
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if constexpr (PA == 1) weigh(s);
            split2<true, false>(X[2 * s], X[2 * s + 1], one, Wh[s], Wl[s]);
            if (s == 0) {
                // S <- decay S + K^T W, the first half's products
#pragma unroll
                for (int t = 0; t < NT; ++t) S[t] = mma(Kt[0][0][t], Wh[0], S[t]);
#pragma unroll
                for (int t = 0; t < NT; ++t) S[t] = mma(Kt[0][0][t], Wl[0], S[t]);
                if constexpr (PA == 2) {
#pragma unroll
                    for (int t = 0; t < NT; ++t) S[t] = mma(Kt[PA - 1][0][t], Wh[0], S[t]);
                }
            }
        }
        auto second = [&](int t0, int t1) {
#pragma unroll
            for (int t = t0; t < t1; ++t) S[t] = mma(Kt[0][1][t], Wh[1], S[t]);
#pragma unroll
            for (int t = t0; t < t1; ++t) S[t] = mma(Kt[0][1][t], Wl[1], S[t]);
            if constexpr (PA == 2) {
#pragma unroll
                for (int t = t0; t < t1; ++t) S[t] = mma(Kt[PA - 1][1][t], Wh[1], S[t]);
            }
        };
        second(0, kEarly);
        second(kEarly, NT);
        // U for the outputs
        const int eu = scale_exp(column_max(largest(U)));
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            f16x8 uh, ul;
            split2<PA == 2>(U[2 * s], U[2 * s + 1], pow2(eu), uh, ul);
            *(f16x8*)(to + (PA * NS + s) * 1024 + lane * 16) = uh;
            if constexpr (PA == 2) *(f16x8*)(to + (PA * NS + 2 + s) * 1024 + lane * 16) = ul;
        }
        if (hh == 0) {
            float* sc = (float*)(to + (NS + 2) * PA * 1024);
            sc[lane] = fs;
            sc[16 + lane] = fu * pow2(-eu);
        }
        form(0, kEarly);
    }
    if (ok && on) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (16 * t >= p.dk) break;
            f32x4 o;
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = S[t][r] * unit;
            *(f32x4*)(state + 16 * t) = o;
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
    const int parts = bf16_act ? 1 : 2;
    w.slots = (int)(T / kC) + nseq;
    size_t off = 0;
    auto take = [&](size_t bytes) { char* q = scratch ? scratch + off : nullptr; off += align256(bytes); return q; };
    w.base = (int32_t*)take((size_t)nseq * 4);
    w.count = (int32_t*)take(4);
    w.plan = (int2*)take((size_t)w.slots * 8);
    w.qk = take((size_t)w.slots * Hk * 2 * qk_bytes(steps_of(dk), parts));
    w.v = take((size_t)w.slots * Hv * v_bytes(parts));
    *total = off;
    return w;
}

template <typename T, int NS, int WAVES> void main_launch(const Args& a, hipStream_t s) {
    const dim3 grid = work_grid(a.d, (a.d.dv + 16 * WAVES - 1) / (16 * WAVES));
    // LDS is asked for at the launch: a kernel that the compiler sees to fill it alone has half of its registers where only
    // MFMAs reach them, and a move for every value that goes between the two
    constexpr bool split = SplitLds<T, NS, WAVES>::kFits;
    constexpr int bytes = split ? SplitLds<T, NS, WAVES>::kBytes : MainLds<T, NS>::kBytes;
    if constexpr (split) SSM_LAUNCH((delta_split_kernel<T, NS, WAVES>), grid, dim3(128 * WAVES), bytes, s, a);
    else SSM_LAUNCH((delta_main_kernel<T, NS, WAVES>), grid, dim3(64 * WAVES), bytes, s, a);
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
    // Two waves of columns to a workgroup where all of these run at once, a compute unit each; else four, which share what
    // they read. 16 heads of 128 x 128 over prompts of 1024 tokens, whole call: 4 prompts (256 workgroups of two) 53.5 us
    // by twos and 61 by fours, 6 prompts (384) 92 and 72, 24 prompts 285 and 232; float32 4 prompts 103 and 108, 6
    // 190 and 123
    KernelTimer kt("delta.main", s);
    const int64_t pairs = (int64_t)p.nseq * p.Hv, by_two = pairs * ((p.dv + 31) / 32);
    if (by_two <= 256 || p.dv <= 32) main_launch<T, NS, 2>(a, s);
    else main_launch<T, NS, 4>(a, s);
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
