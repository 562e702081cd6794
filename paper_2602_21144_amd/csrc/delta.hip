// Gated delta rule of one shard's value heads. Per head, with the state S (dv x dk, float32):
//   k, q over their length; alpha = exp(-exp(A_log) softplus(a + dt_bias)); beta = beta_max sigmoid(b)
//   u = beta (v - alpha S k);  S <- alpha S + u k^T;  o = scale S q
// A row of S needs nothing of the others: 8 lanes hold one, lane q the float4 groups at
// n = 32 j + 4 q, so that a load or store instruction of a wave covers whole lines.
#include "gate.h"

namespace ssm {
namespace {

// four values of this lane in a head row of n values, zeros behind its end
template <typename T> __device__ __forceinline__ f32x4 head4(const T* row, int at, int n) {
    f32x4 v{};
    if (at < n) {
        typedef T T4 __attribute__((ext_vector_type(4)));
        const T4 x = *(const T4*)(row + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = to_f32(x[e]);
    }
    return v;
}
__device__ __forceinline__ float dot4(const f32x4& x, const f32x4& y, float s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) s = __builtin_fmaf(x[e], y[e], s);
    return s;
}
// over eight neighbouring lanes, complete in each: by DPP within four, then from the mirrored lane of the eight
template <int CTRL> __device__ __forceinline__ float dpp_f32(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float sum8(float v) {
    v += dpp_f32<0xB1>(v);    // quad_perm: lane ^ 1
    v += dpp_f32<0x4E>(v);    // lane ^ 2
    return v + dpp_f32<0x141>(v);   // row_half_mirror: lane ^ 7, whose quad holds the other sum
}

// one token's q and k of a head (q scaled, both normalised where the descriptor says so) and its
// decay and write strength: asked for, then worked out
template <typename T, int NJ> struct Token {
    f32x4 q[NJ], k[NJ];
    float alpha, beta;
    __device__ __forceinline__ void load(const DeltaArgs& p, const T* row, int64_t t, int h, int lane8) {
        const T* pq = row + (h / p.rep) * p.dk;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            q[j] = head4(pq, 32 * j + 4 * lane8, p.dk);
            k[j] = head4(pq + p.Hk * p.dk, 32 * j + 4 * lane8, p.dk);
        }
        alpha = to_f32(((const T*)p.a)[t * p.ld_ab + h]) + p.dt_bias[h];
        beta = to_f32(((const T*)p.b)[t * p.ld_ab + h]);
    }
    __device__ __forceinline__ void form(const DeltaArgs& p, float a_log) {
        alpha = fast_exp2(-fast_exp2(a_log * kLog2e) * kLog2e * softplus_f(alpha));
        beta = p.beta_max * sigmoid_f(beta);
        float rq = p.scale, rk = 1.0f;
        if (p.qk_norm) {
            float sq = 0.0f, sk = 0.0f;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                sq = dot4(q[j], q[j], sq);
                sk = dot4(k[j], k[j], sk);
            }
            rq = p.scale / sqrtf(fmaxf(sum8(sq) + p.eps, 1.2e-38f));
            rk = 1.0f / sqrtf(fmaxf(sum8(sk) + p.eps, 1.2e-38f));
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            q[j] *= rq;
            k[j] *= rk;
        }
    }
};

// one token on one row of the state; the row's output, complete in every of its 8 lanes
template <typename T, int NJ>
__device__ __forceinline__ float row_step(f32x4 (&S)[NJ], const Token<T, NJ>& x, float v) {
    float sk = 0.0f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) sk = dot4(S[j], x.k[j], sk);
    const float u = x.beta * (v - x.alpha * sum8(sk));
    float o = 0.0f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
#pragma unroll
        for (int e = 0; e < 4; ++e) S[j][e] = __builtin_fmaf(u, x.k[j][e], x.alpha * S[j][e]);
        o = dot4(S[j], x.q[j], o);
    }
    return sum8(o);
}

// PAST: past the caches, for states that they would not keep until the next step
template <bool PAST, int NJ> __device__ __forceinline__ void row_load(f32x4 (&S)[NJ], const float* row, int lane8, int dk) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const f32x4* at = (const f32x4*)(row + 32 * j + 4 * lane8);
        S[j] = f32x4{};
        if (32 * j + 4 * lane8 < dk) S[j] = PAST ? __builtin_nontemporal_load(at) : *at;
    }
}
template <bool PAST, int NJ> __device__ __forceinline__ void row_store(const f32x4 (&S)[NJ], float* row, int lane8, int dk) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        f32x4* at = (f32x4*)(row + 32 * j + 4 * lane8);
        if (32 * j + 4 * lane8 >= dk) continue;
        if constexpr (PAST) __builtin_nontemporal_store(S[j], at);
        else *at = S[j];
    }
}

// ---------------------------------------------------------------- single tokens
// One workgroup per (head, sequence): 32 rows a pass, NP passes' rows in flight together, what needs no state worked out
// meanwhile. Bound by the states' traffic: 256 sequences of 16 heads of 128 x 128 (537 MB) 104 us, 5.2 TB/s; one sequence
// 5.5 us, a launch and two round trips (slot, then state).
template <typename T, int NJ, int NP, bool PAST> __global__ __launch_bounds__(256) void delta_decode_kernel(DeltaArgs p) {
    __shared__ float s_o[512], s_sum[4];
    const int h = blockIdx.x, tid = threadIdx.x, lane8 = tid & 7;
    const int64_t i = blockIdx.y;
    const int slot = p.slot[i];
    const T* x = (const T*)p.qkv + i * p.ld;
    Token<T, NJ> tok;
    tok.load(p, x, i, h, lane8);
    const float a_log = p.A_log[h];
    const bool ok = slot >= 0 && slot < p.S;
    T* out = (T*)p.out + i * p.ld_out + h * p.dv;
    if (!ok) {
        for (int c = tid; c < p.dv; c += 256) out[c] = from_f32<T>(0.0f);
        if (h == 0 && tid == 0) atomicOr(p.status, SSM_STATUS_BAD_SLOT);
        return;
    }
    float* head = p.pool + ((int64_t)slot * p.Hv + h) * p.dv * p.dk;
    bool formed = false;
    for (int r0 = 0; r0 < p.dv; r0 += 32 * NP) {
        f32x4 S[NP][NJ];
        float v[NP];
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            const int r = min(r0 + 32 * n + (tid >> 3), p.dv - 1);
            row_load<PAST>(S[n], head + (int64_t)r * p.dk, lane8, p.dk);
            v[n] = to_f32(x[2 * p.Hk * p.dk + h * p.dv + r]);
        }
        if (!formed) tok.form(p, a_log);
        formed = true;
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            const int r = r0 + 32 * n + (tid >> 3);
            const float o = row_step(S[n], tok, v[n]);
            if (r >= p.dv) continue;   // whole groups of 8 lanes
            row_store<PAST>(S[n], head + (int64_t)r * p.dk, lane8, p.dk);
            if (lane8 == 0) s_o[r] = o;
        }
    }
    __syncthreads();
    const GatedNormArgs& n = p.norm;
    float y[2], g[2], ss = 0.0f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int c = tid + 256 * e;
        if (c >= p.dv) continue;
        y[e] = s_o[c];
        g[e] = n.w && n.z ? gate_f(to_f32(((const T*)n.z)[i * n.ld_z + h * p.dv + c]), n.gate) : 1.0f;
        if (n.gate_first) y[e] *= g[e];
        ss += y[e] * y[e];
    }
    if (n.w) {
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) ss += __shfl_xor(ss, off, 64);
        if ((tid & 63) == 0) s_sum[tid >> 6] = ss;
        __syncthreads();
        const float inv = 1.0f / sqrtf(((s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3])) / (float)p.dv + n.eps);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int c = tid + 256 * e;
            if (c < p.dv) y[e] = y[e] * inv * n.w[(n.per_head ? h * p.dv : 0) + c] * (n.gate_first ? 1.0f : g[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
        if (tid + 256 * e < p.dv) out[tid + 256 * e] = from_f32<T>(y[e]);
}

template <typename T, bool PAST> hipError_t decode_launch(const DeltaArgs& p, hipStream_t s) {
    const dim3 grid((unsigned)p.Hv, (unsigned)p.nseq);
    if (p.dk <= 64) SSM_LAUNCH((delta_decode_kernel<T, 2, 4, PAST>), grid, dim3(256), 0, s, p);
    else if (p.dk <= 128) SSM_LAUNCH((delta_decode_kernel<T, 4, 4, PAST>), grid, dim3(256), 0, s, p);
    else SSM_LAUNCH((delta_decode_kernel<T, 8, 2, PAST>), grid, dim3(256), 0, s, p);
    return hipGetLastError();
}
// States of more than 96 MB are read and written past the caches: 128 sequences of 1 MB 60 -> 54 us, 256 112 -> 104; below
// that the 256 MB cache can keep them from step to step (64 sequences 22.9, past the caches 26.8)
template <typename T> hipError_t decode_launch(const DeltaArgs& p, hipStream_t s) {
    const bool past = (int64_t)p.nseq * p.Hv * p.dv * p.dk * 4 > (96ll << 20);
    return past ? decode_launch<T, true>(p, s) : decode_launch<T, false>(p, s);
}

}  // namespace

hipError_t launch_delta_decode(const DeltaArgs& p, bool bf16_act, hipStream_t s) {
    if (p.nseq <= 0) return hipSuccess;
    KernelTimer kt("delta.decode", s);
    return bf16_act ? decode_launch<bf16>(p, s) : decode_launch<float>(p, s);
}

}  // namespace ssm
