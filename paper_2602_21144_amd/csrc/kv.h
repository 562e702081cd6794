// Device helpers of the paged attention cache: a call's sequences, pages, and the 8-bit codes.
#pragma once
#include "common.h"

namespace ssm {

// One sequence of a call: rows [lo, lo + m) of the packed batch are its tokens n - m .. n - 1.
// ok false: the metadata does not fit the call, and the sequence's work is left out.
struct KvSeq {
    int lo, m, n;
    bool ok;
};
__device__ __forceinline__ KvSeq kv_seq(const KvArgs& a, int i) {
    KvSeq s;
    s.n = a.kv_len[i];
    if (a.cu) {
        const int lo = a.cu[i], hi = a.cu[i + 1];
        s.lo = lo;
        s.m = hi - lo;
        s.ok = lo >= 0 && hi >= lo && (int64_t)hi <= a.T && s.n >= s.m;
    } else {
        // one row per sequence; a length of 0 marks a row without a token (a padded batch)
        s.lo = i;
        s.m = 1;
        s.ok = s.n >= 0;
    }
    s.ok = s.ok && (int64_t)s.n <= ((int64_t)a.max_pages << a.page_log2);
    return s;
}
// Sets the status bit where any sequence's metadata is bad; called by the threads of one workgroup.
__device__ __forceinline__ void kv_check_seqs(const KvArgs& a, int tid, int threads) {
    for (int i = tid; i < a.nseq; i += threads)
        if (!kv_seq(a, i).ok) atomicOr(a.status, SSM_STATUS_BAD_SEQLENS);
}
// The sequence of packed row t and its place in it; seq -1: no sequence has this row.
struct KvRow {
    int seq, pos;   // pos: the token's index in the sequence; -1: a row without a token
};
__device__ __forceinline__ KvRow kv_row(const KvArgs& a, int64_t t) {
    int i = (int)t;
    if (a.cu) {
        int e = a.nseq;   // the last sequence that starts at or before t: empty ones end before it
        i = 0;
        while (e - i > 1) {
            const int mid = (i + e) >> 1;
            if (a.cu[mid] <= t) i = mid;
            else e = mid;
        }
    }
    const KvSeq s = kv_seq(a, i);
    if (!s.ok || t < s.lo || t >= (int64_t)s.lo + s.m) return KvRow{-1, -1};
    return KvRow{i, s.n - s.m + (int)(t - s.lo)};
}

// The page of a sequence's token; -1 (and the status bit) when the table names none
__device__ __forceinline__ int kv_page(const KvArgs& a, int seq, int pos) {
    const int p = a.table[(int64_t)seq * a.max_pages + (pos >> a.page_log2)];
    if (p >= 0 && p < a.num_pages) return p;
    atomicOr(a.status, SSM_STATUS_BAD_PAGE);
    return -1;
}
// index of (page, head, token of the page) among the pool's rows of D values
__device__ __forceinline__ int64_t kv_pool_row(const KvArgs& a, int page, int head, int pos) {
    return (((int64_t)page * a.Hkv + head) << a.page_log2) + (pos & ((1 << a.page_log2) - 1));
}

template <int FMT> constexpr float kv_code_max() { return FMT == SSM_KV_FP8_E4M3 ? 448.0f : 127.0f; }
// Rows whose largest magnitude is below this are stored as zeros: 448 / max stays finite.
constexpr float kKvTiny = 1e-30f;

// four values -> four codes of a 32-bit word (round to nearest even), x already scaled to the codes' range
template <int FMT> __device__ __forceinline__ uint32_t kv_encode4(const float (&x)[4]) {
    constexpr float Q = kv_code_max<FMT>();
    float q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = fminf(fmaxf(x[i], -Q), Q);
    if constexpr (FMT == SSM_KV_FP8_E4M3) {
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], p, true);
    } else {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w |= ((uint32_t)(int32_t)__builtin_rintf(q[i]) & 0xFFu) << (8 * i);
        return w;
    }
}
// four codes -> float32
template <int FMT> __device__ __forceinline__ void kv_decode4(uint32_t w, float (&v)[4]) {
    if constexpr (FMT == SSM_KV_FP8_E4M3) {
        v[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
        v[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
        v[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
        v[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (float)(int8_t)((w >> (8 * k)) & 0xFF);
    }
}
// four codes -> two words of two bf16 each, exactly: e4m3 has 4 significant bits, int8 at most 7
// (|code| <= 127), bf16 has 8
template <int FMT> __device__ __forceinline__ u32x2 kv_decode4_bf16(uint32_t w) {
    u32x2 r;
    if constexpr (FMT == SSM_KV_FP8_E4M3) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        r[0] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, false));
        r[1] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, true));
    } else {
        float v[4];
        kv_decode4<FMT>(w, v);   // exact in bf16: the high half of the float32
        r[0] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, v[1]), __builtin_bit_cast(uint32_t, v[0]), 0x07060302u);
        r[1] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, v[3]), __builtin_bit_cast(uint32_t, v[2]), 0x07060302u);
    }
    return r;
}

// The stored element of a cache: act type T, or the codes of a format
template <typename T, int FMT> struct KvElem { using type = uint8_t; };
template <typename T> struct KvElem<T, SSM_KV_ACT> { using type = T; };

// Joins the partial results of one row: o = sum_v f_v o_v / sum_v f_v l_v with f_v = 2^(m_v - max m). One
// wave; slot(v) is partial v, which holds the row's D values at o_at and its statistics at m_at and l_at.
// Lanes take 4 values each; what is left of the wave splits the partials, every lane's share in order and
// then the shares. The first values are on their way before the statistics are there.
template <typename T, int kBatch, typename F>
__device__ __forceinline__ void join_row(int pieces, F slot, int64_t o_at, int64_t m_at, int64_t l_at, int D, T* out) {
    const int lane = threadIdx.x & 63;
    const int lpr = D <= 64 ? 16 : D <= 128 ? 32 : 64, subs = 64 / lpr;
    const int sub = lane / lpr, d = (lane % lpr) * 4;
    f32x4 x[kBatch];
    auto fetch = [&](int v0) {   // partials v0 + sub, v0 + sub + subs, ..
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int v = v0 + k * subs + sub;
            x[k] = f32x4{0, 0, 0, 0};
            if (v < pieces && d < D) x[k] = *(const f32x4*)(slot(v) + o_at + d);
        }
    };
    fetch(0);
    float M = -3.0e38f;
    for (int v = lane; v < pieces; v += 64) M = fmaxf(M, slot(v)[m_at]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
    float ls = 0.0f, f = 0.0f, o[4] = {0, 0, 0, 0};
    for (int v0 = 0; v0 < pieces; v0 += kBatch * subs) {
        if (v0 % 64 == 0) {   // the factors of the next 64 (a batch is at most 32 of them)
            f = 0.0f;
            if (v0 + lane < pieces) {
                f = fast_exp2(slot(v0 + lane)[m_at] - M);
                ls += f * slot(v0 + lane)[l_at];
            }
        }
        f32x4 y[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) y[k] = x[k];
        if (v0 + kBatch * subs < pieces) fetch(v0 + kBatch * subs);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const float fv = __shfl(f, (v0 + k * subs + sub) & 63, 64);   // 0 past the last partial
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += fv * y[k][e];
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) ls += __shfl_xor(ls, off, 64);
    for (int off = lpr; off < 64; off <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], off, 64);
    if (sub == 0 && d < D) {
        const float inv = ls > 0.0f ? 1.0f / ls : 0.0f;   // nothing visible: zeros
        T y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = from_f32<T>(o[e] * inv);
        __builtin_memcpy(__builtin_assume_aligned(out + d, 4 * sizeof(T)), y, sizeof y);
    }
}

}  // namespace ssm
