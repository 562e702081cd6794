// The paged attention cache: what writes it and what reads it back.
//
// kv_append: one token's [q | k | v] projection. Every q and k head of D values is divided by its
// RMS and weighted (if wanted), its first `rot` values are rotated in pairs by the token's position,
// and k and v are written to the token's page; q goes on to the attention. With the 8-bit formats a
// row of D values is stored as codes of x * (Q / max|x|) and the float32 scale max|x| / Q.
//
// The rotation's angle is position * frequency. Frequencies come as turns per token in 64-bit fixed
// point, so the product's fraction of a turn is exact in integer arithmetic (it wraps where the
// angle does), at any position; sine and cosine are polynomials on an eighth of a turn to either side.
#include "kv.h"

namespace ssm {
namespace {

// four values as they are stored
__device__ __forceinline__ f32x4 kv_load4(const float* p) { return *(const f32x4*)p; }
__device__ __forceinline__ bf16x4 kv_load4(const bf16* p) { return *(const bf16x4*)p; }
template <typename T> __device__ __forceinline__ void kv_store4(T* p, const float (&v)[4]);
template <> __device__ __forceinline__ void kv_store4<float>(float* p, const float (&v)[4]) {
    *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
}
template <> __device__ __forceinline__ void kv_store4<bf16>(bf16* p, const float (&v)[4]) {
    bf16x4 a;
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = (bf16)v[e];
    *(bf16x4*)p = a;
}

// cos and sin of x turns / 2^64. The nearest quarter turn comes off exactly; the rest, at most an
// eighth of a turn, is within 2^-28 turns (2.3e-8 radians) of its float32 form (24 of the 32 bits that
// are taken of it), where the Taylor sums to theta^9 and theta^10 leave less than 2e-9.
__device__ __forceinline__ void cos_sin_turns(uint64_t x, float& c, float& s) {
    const uint32_t quarter = (uint32_t)((x + (1ull << 61)) >> 62);
    const int64_t rest = (int64_t)(x - ((uint64_t)quarter << 62));
    const float th = (float)(int32_t)(rest >> 30) * 3.6572952e-10f;   // 2 pi / 2^34
    const float t2 = th * th;
    const float sn = th + th * t2 * (-1.6666667e-1f + t2 * (8.3333333e-3f + t2 * (-1.9841270e-4f + t2 * 2.7557319e-6f)));
    const float cs = 1.0f + t2 * (-0.5f + t2 * (4.1666667e-2f + t2 * (-1.3888889e-3f + t2 * (2.4801587e-5f + t2 * -2.7557319e-7f))));
    const float a = (quarter & 1) ? sn : cs, b = (quarter & 1) ? cs : sn;
    c = (quarter == 1 || quarter == 2) ? -a : a;
    s = (quarter >= 2) ? -b : b;
}

// 1 / sqrt(x), one step of 2^-23 off; the instruction takes no subnormal numbers: 1.2e-38 stands for them
__device__ __forceinline__ float inv_root(float x) { return __builtin_amdgcn_rsqf(x < 1.2e-38f ? 1.2e-38f : x); }

// max|row| / Q and Q / max|row|, the nearest float32 values: a quotient near the true one, and what it leaves (exact in
// one fma) put right. With a reciprocal up to one step off, as the instruction's is, that gives the nearest value for
// every float32 from 1e-30 to the largest (all of them tried; int8 after a step on the reciprocal). With the compiler's
// divisions 2048 tokens of 48 heads of 112 take 0.4 us more.
template <int FMT> __device__ __forceinline__ float row_scale(float amax) {
    constexpr float Q = kv_code_max<FMT>(), part = 1.0f / Q;
    const float s = amax * part;
    return __builtin_fmaf(__builtin_fmaf(-Q, s, amax), part, s);
}
template <int FMT> __device__ __forceinline__ float row_factor(float amax, float scale) {
    constexpr float Q = kv_code_max<FMT>(), part = 1.0f / Q;
    float y = __builtin_amdgcn_rcpf(scale);   // of the scale: above 2^-120, where max|row| itself may have a subnormal one
    if constexpr (FMT == SSM_KV_INT8) y = __builtin_fmaf(__builtin_fmaf(-scale, y, 1.0f), y, y);
    return __builtin_fmaf(__builtin_fmaf(-amax, y, Q) * part, y, y);
}

// The result of op over groups of LPH neighbouring lanes, in each of them. Every step pairs lanes whose
// partial results are of different values: neighbours, pairs, then mirrored quads and eights.
template <int LPH, typename F> __device__ __forceinline__ float group_reduce(float v, F op) {
    auto moved = [&](auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    v = op(v, moved(std::integral_constant<int, 0xB1>{}));    // quad_perm 1 0 3 2
    v = op(v, moved(std::integral_constant<int, 0x4E>{}));    // quad_perm 2 3 0 1
    v = op(v, moved(std::integral_constant<int, 0x141>{}));   // row_half_mirror
    if constexpr (LPH >= 16) v = op(v, moved(std::integral_constant<int, 0x140>{}));   // row_mirror
    if constexpr (LPH >= 32) v = op(v, __shfl_xor(v, 16, 64));
    return v;
}

// A group of LPH lanes holds one head's D values, 8 per lane in two pieces of 4: the pieces that a
// rotation pairs (4 values at 4 j and 4 at rot / 2 + 4 j), or 8 neighbours. One workgroup per token:
// its angles are worked out once, and each group goes through every 256 / LPH-th head with the next
// head's values on their way.
//
// A chunk of 2048 tokens of 48 heads of 112 into fp8 (37 MB in and out, 6 us at 6.2 TB/s) takes
// 10.6 us, of which 4 are an empty launch's. It was bound by instructions, not bytes: 15.4 us with the angles in
// every lane, library root and divisions and sums by way of shared memory. Splitting a token's heads over
// workgroups is no faster at any number of tokens (2048: 14.8 us, the lookups are repeated; 1 to 256: alike, 4 to 5).
//
// Workgroups go to the 8 XCDs in turn. Of each 128 an XCD takes 16 neighbouring tokens, so that the parts of a line that
// they write (rows of 224 bytes or of codes, four bytes of scale) meet in one L2: 4792 tokens of 48 heads of 112 in bf16
// 31.4 -> 28.6 us, 2048 in fp8 10.9 -> 10.6 (an eighth of all tokens to each XCD: 27.9 and 10.7, but 42.8 for 41.8
// where rows are whole lines).
__device__ __forceinline__ int64_t token_of(uint32_t b, int64_t T) {
    return b < (T & ~(int64_t)127) ? (b & ~127u) + (b & 7) * 16 + ((b >> 3) & 15) : b;
}
template <typename T, int FMT, int LPH>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendArgs a) {
    using E = typename KvElem<T, FMT>::type;
    const KvArgs& kv = a.kv;
    const int64_t t = token_of(blockIdx.x, kv.T);
    const int D = kv.D, j = threadIdx.x % LPH;
    const bool on = 8 * j < D;
    const bool half = !a.inter && 8 * j < a.rot;          // the two pieces are a rotation's two halves
    const int d0 = half ? 4 * j : 8 * j, d1 = half ? a.rot / 2 + 4 * j : 8 * j + 4;
    const int heads = kv.Hq + 2 * kv.Hkv;
    constexpr int step = 256 / LPH;
    const float inv_d = 1.0f / (float)D;
    const T* in = (const T*)a.qkv + t * a.ld;
    int h = threadIdx.x / LPH;
    // the first head and the norms' weights are on their way while the row's place is looked up
    using Piece = decltype(kv_load4(in));
    Piece x0, x1;
    auto fetch = [&](int head) {
        x0 = x1 = Piece{};
        if (on && head < heads) {
            x0 = kv_load4(in + (int64_t)head * D + d0);
            x1 = kv_load4(in + (int64_t)head * D + d1);
        }
    };
    fetch(h);
    float4 qw[2] = {}, kw[2] = {};
    if (on && a.q_w) qw[0] = *(const float4*)(a.q_w + d0), qw[1] = *(const float4*)(a.q_w + d1);
    if (on && a.k_w) kw[0] = *(const float4*)(a.k_w + d0), kw[1] = *(const float4*)(a.k_w + d1);

    if (t == 0) kv_check_seqs(kv, threadIdx.x, 256);
    const KvRow row = kv_row(kv, t);
    if (row.seq < 0) return;   // the whole workgroup
    const int pos = row.pos < 0 ? 0 : row.pos;
    const int page = row.pos < 0 ? -1 : kv_page(kv, row.seq, pos);

    __shared__ __align__(16) float s_cs[128], s_sn[128];
    float cs[4], sn[4];
    const bool turn = on && 8 * j < a.rot;
    if (a.rot > 0) {
        if ((int)threadIdx.x < a.rot / 2) cos_sin_turns(a.turns[threadIdx.x] * (uint64_t)pos, s_cs[threadIdx.x], s_sn[threadIdx.x]);
        __syncthreads();
        if (turn) {
            const f32x4 c4 = kv_load4(s_cs + 4 * j), s4 = kv_load4(s_sn + 4 * j);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                cs[e] = c4[e];
                sn[e] = s4[e];
            }
        }
    }
    for (; h < heads; h += step) {
        float x[4], y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = (float)x0[e];
            y[e] = (float)x1[e];
        }
        fetch(h + step);   // the next head, while this one is worked on
        const bool is_v = h >= kv.Hq + kv.Hkv;
        if (!is_v && (h < kv.Hq ? a.q_w : a.k_w)) {
            float ss = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) ss += x[e] * x[e] + y[e] * y[e];
            ss = group_reduce<LPH>(ss, [](float p, float q) { return p + q; });
            const float inv = inv_root(ss * inv_d + a.eps);
            const float4 w0 = h < kv.Hq ? qw[0] : kw[0], w1 = h < kv.Hq ? qw[1] : kw[1];
            const float u[4] = {w0.x, w0.y, w0.z, w0.w}, v[4] = {w1.x, w1.y, w1.z, w1.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = x[e] * inv * u[e];
                y[e] = y[e] * inv * v[e];
            }
        }
        if (turn && !is_v) {
            if (a.inter) {   // pairs (0, 1), (2, 3) of x take angles 0, 1; those of y angles 2, 3
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float p = x[2 * e], q = x[2 * e + 1], u = y[2 * e], v = y[2 * e + 1];
                    x[2 * e] = p * cs[e] - q * sn[e];
                    x[2 * e + 1] = q * cs[e] + p * sn[e];
                    y[2 * e] = u * cs[2 + e] - v * sn[2 + e];
                    y[2 * e + 1] = v * cs[2 + e] + u * sn[2 + e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = x[e], q = y[e];
                    x[e] = p * cs[e] - q * sn[e];
                    y[e] = q * cs[e] + p * sn[e];
                }
            }
        }
        if (h < kv.Hq) {
            if (on) {
                T* o = (T*)a.q + t * a.ld_q + (int64_t)h * D;
                kv_store4(o + d0, x);
                kv_store4(o + d1, y);
            }
            continue;
        }
        const int64_t r = page < 0 ? 0 : kv_pool_row(kv, page, is_v ? h - kv.Hq - kv.Hkv : h - kv.Hq, pos);
        E* o = (E*)(is_v ? kv.v : kv.k) + r * D;
        if constexpr (FMT == SSM_KV_ACT) {
            if (on && page >= 0) {
                kv_store4(o + d0, x);
                kv_store4(o + d1, y);
            }
        } else {
            constexpr float Q = kv_code_max<FMT>();
            // The largest magnitude, by the order of the bits: infinity lies above all numbers, NaN above that
            auto larger = [](float p, float q) {
                return __builtin_bit_cast(float, max(__builtin_bit_cast(uint32_t, p), __builtin_bit_cast(uint32_t, q)));
            };
            float amax = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) amax = larger(amax, larger(fabsf(x[e]), fabsf(y[e])));
            amax = group_reduce<LPH>(amax, larger);
            const bool finite = amax < __builtin_inff();
            // Both quotients are the nearest ones. A row's factor is often a power of two (its largest value 1.75 2^k), and
            // then values of few bits lie on ties, which a factor one step off would send the wrong way.
            // A row with a value that is no number, for which int8 has no code, is lost as a whole: its scale is NaN.
            const bool held = finite && amax >= kKvTiny;
            const float scale = held ? row_scale<FMT>(amax) : finite ? 0.0f : __builtin_nanf("");
            const float inv = held ? row_factor<FMT>(amax, scale) : 0.0f;
            float u[4], v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                u[e] = x[e] * inv;
                v[e] = y[e] * inv;
            }
            if (on && page >= 0) {
                *(uint32_t*)(o + d0) = kv_encode4<FMT>(u);
                *(uint32_t*)(o + d1) = kv_encode4<FMT>(v);
                if (j == 0) (is_v ? kv.vs : kv.ks)[r] = scale;
            }
        }
    }
}

// kv_read: kReadRows packed rows per workgroup. A page holds a head's tokens next to each other, so
// the threads walk (k or v, head, row, 8 values) with the row inside the head: neighbouring threads
// read one stretch of a page. A thread's next kReadAhead loads are in flight together.
//
// Bound by memory: 24000 rows of 16 heads of 128 from fp8 (149 MB in and out, 24 us at 6.2 TB/s)
// in 25.3 us, 5.9 TB/s. The packed rows are stored past the caches (42.4 us without, where the cache is not
// there from an earlier call: what is written takes the place of what is to be read). Few rows are split over
// gridDim.y workgroups (391 rows of bf16: 4.5 us, 12 by 25 workgroups alone).
template <typename T> __device__ __forceinline__ void store_through(T* p, const T (&v)[8]) {
    f32x4 w[sizeof(T) / 2];
    __builtin_memcpy(w, v, sizeof w);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) __builtin_nontemporal_store(w[i], (f32x4*)p + i);
}
constexpr int kReadRows = 16, kReadAhead = 4, kReadGroups = 4096;
template <typename T, int FMT>
__global__ __launch_bounds__(256) void kv_read_kernel(KvArgs a, T* k_out, int64_t ld_k, T* v_out, int64_t ld_v) {
    using E = typename KvElem<T, FMT>::type;
    struct alignas(sizeof(E) == 1 ? 8 : 16) Codes { E e[8]; };
    __shared__ int s_page[kReadRows], s_pos[kReadRows];
    if (blockIdx.x == 0 && blockIdx.y == 0) kv_check_seqs(a, threadIdx.x, 256);
    const int64_t t0 = (int64_t)blockIdx.x * kReadRows;
    if (threadIdx.x < kReadRows) {
        const int64_t t = t0 + threadIdx.x;
        int page = -1, pos = 0;
        if (t < a.T) {
            const KvRow row = kv_row(a, t);
            if (row.pos >= 0) {
                pos = row.pos;
                page = kv_page(a, row.seq, pos);
            }
        }
        s_page[threadIdx.x] = page;
        s_pos[threadIdx.x] = pos;
    }
    __syncthreads();
    const int D = a.D, pieces = D / 8, per = pieces * kReadRows, all = 2 * a.Hkv * per;
    const int step = 256 * (int)gridDim.y;
    for (int i0 = (int)blockIdx.y * 256 + threadIdx.x; i0 < all; i0 += kReadAhead * step) {
        Codes c[kReadAhead];
        float sc[kReadAhead];
        T* o[kReadAhead];
#pragma unroll
        for (int b = 0; b < kReadAhead; ++b) {
            const int i = i0 + b * step;
            o[b] = nullptr;
            if (i >= all) continue;
            const int hh = i / per, r = (i % per) / pieces, d = (i % pieces) * 8;
            const int page = s_page[r];
            if (page < 0) continue;
            const bool is_v = hh >= a.Hkv;
            const int h = is_v ? hh - a.Hkv : hh;
            const int64_t row = kv_pool_row(a, page, h, s_pos[r]);
            c[b] = *(const Codes*)((const E*)(is_v ? a.v : a.k) + row * D + d);
            if constexpr (FMT != SSM_KV_ACT) sc[b] = (is_v ? a.vs : a.ks)[row];
            o[b] = (is_v ? v_out + (t0 + r) * ld_v : k_out + (t0 + r) * ld_k) + (int64_t)h * D + d;
        }
#pragma unroll
        for (int b = 0; b < kReadAhead; ++b) {
            if (!o[b]) continue;
            if constexpr (FMT == SSM_KV_ACT) {
                store_through(o[b], c[b].e);
            } else {
                const uint2 w = __builtin_bit_cast(uint2, c[b]);
                float x[4], y[4];
                kv_decode4<FMT>(w.x, x);
                kv_decode4<FMT>(w.y, y);
                T v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = from_f32<T>(x[e] * sc[b]);
                    v[4 + e] = from_f32<T>(y[e] * sc[b]);
                }
                store_through(o[b], v);
            }
        }
    }
}

template <typename T, int FMT> hipError_t append_launch(const KvAppendArgs& a, hipStream_t s) {
    const int lph = a.kv.D <= 64 ? 8 : a.kv.D <= 128 ? 16 : 32;
    const dim3 grid((unsigned)a.kv.T), block(256);
    if (lph == 8) SSM_LAUNCH((kv_append_kernel<T, FMT, 8>), grid, block, 0, s, a);
    else if (lph == 16) SSM_LAUNCH((kv_append_kernel<T, FMT, 16>), grid, block, 0, s, a);
    else SSM_LAUNCH((kv_append_kernel<T, FMT, 32>), grid, block, 0, s, a);
    return hipGetLastError();
}
template <typename T> hipError_t append_fmt(const KvAppendArgs& a, hipStream_t s) {
    switch (a.kv.fmt) {
        case SSM_KV_ACT: return append_launch<T, SSM_KV_ACT>(a, s);
        case SSM_KV_FP8_E4M3: return append_launch<T, SSM_KV_FP8_E4M3>(a, s);
        default: return append_launch<T, SSM_KV_INT8>(a, s);
    }
}
template <typename T> hipError_t read_fmt(const KvArgs& a, T* k, int64_t ld_k, T* v, int64_t ld_v, hipStream_t s) {
    // few rows: split until there are kReadGroups workgroups or each thread has one piece
    const int64_t groups = (a.T + kReadRows - 1) / kReadRows, rounds = (2LL * a.Hkv * (a.D / 8) * kReadRows + 255) / 256;
    const int64_t want = (kReadGroups + groups - 1) / groups, slices = want < rounds ? want : rounds;
    const dim3 grid((unsigned)groups, (unsigned)slices), block(256);
    switch (a.fmt) {
        case SSM_KV_ACT: SSM_LAUNCH((kv_read_kernel<T, SSM_KV_ACT>), grid, block, 0, s, a, k, ld_k, v, ld_v); break;
        case SSM_KV_FP8_E4M3: SSM_LAUNCH((kv_read_kernel<T, SSM_KV_FP8_E4M3>), grid, block, 0, s, a, k, ld_k, v, ld_v); break;
        default: SSM_LAUNCH((kv_read_kernel<T, SSM_KV_INT8>), grid, block, 0, s, a, k, ld_k, v, ld_v); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_append(const KvAppendArgs& a, bool bf16_act, hipStream_t s) {
    return bf16_act ? append_fmt<bf16>(a, s) : append_fmt<float>(a, s);
}
hipError_t launch_kv_read(const KvArgs& a, void* k, int64_t ld_k, void* v, int64_t ld_v, bool bf16_act, hipStream_t s) {
    return bf16_act ? read_fmt<bf16>(a, (bf16*)k, ld_k, (bf16*)v, ld_v, s)
                    : read_fmt<float>(a, (float*)k, ld_k, (float*)v, ld_v, s);
}

}  // namespace ssm
