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

template <typename T> __device__ __forceinline__ void kv_load4(const T* p, float (&v)[4]);
template <> __device__ __forceinline__ void kv_load4<float>(const float* p, float (&v)[4]) {
    const float4 a = *(const float4*)p;
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
template <> __device__ __forceinline__ void kv_load4<bf16>(const bf16* p, float (&v)[4]) {
    const bf16x4 a = *(const bf16x4*)p;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)a[e];
}
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
// eighth of a turn, is within 2^-34 turns (3.7e-10 radians) of its float32 form, where the Taylor
// sums to theta^9 and theta^10 leave less than 2e-9.
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

// A group of LPH lanes holds one head's D values, 8 per lane in two pieces of 4: the pieces that a
// rotation pairs (4 values at 4 j and 4 at rot / 2 + 4 j), or 8 neighbours. One workgroup per token
// and slice of its heads: a lane's four angles serve every head that its group takes.
template <typename T, int FMT, int LPH>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendArgs a) {
    using E = typename KvElem<T, FMT>::type;
    const KvArgs& kv = a.kv;
    const int64_t t = blockIdx.x;
    const int D = kv.D, j = threadIdx.x % LPH;
    if (t == 0 && blockIdx.y == 0) kv_check_seqs(kv, threadIdx.x, 256);
    const KvRow row = kv_row(kv, t);
    if (row.seq < 0) return;   // the whole workgroup
    const int pos = row.pos < 0 ? 0 : row.pos;
    const int page = row.pos < 0 ? -1 : kv_page(kv, row.seq, pos);

    const bool on = 8 * j < D;
    const bool half = !a.inter && 8 * j < a.rot;          // the two pieces are a rotation's two halves
    const int d0 = half ? 4 * j : 8 * j, d1 = half ? a.rot / 2 + 4 * j : 8 * j + 4;
    float cs[4], sn[4];
    const bool turn = on && 8 * j < a.rot;
    if (turn) {
#pragma unroll
        for (int e = 0; e < 4; ++e) cos_sin_turns(a.turns[4 * j + e] * (uint64_t)pos, cs[e], sn[e]);
    }
    const int heads = kv.Hq + 2 * kv.Hkv;
    const int step = (256 / LPH) * gridDim.y;
    const T* in = (const T*)a.qkv + t * a.ld;
    for (int h = (int)blockIdx.y * (256 / LPH) + threadIdx.x / LPH; h < heads; h += step) {
        float x[4] = {}, y[4] = {};
        if (on) {
            kv_load4(in + (int64_t)h * D + d0, x);
            kv_load4(in + (int64_t)h * D + d1, y);
        }
        const bool is_v = h >= kv.Hq + kv.Hkv;
        const float* w = is_v ? nullptr : (h < kv.Hq ? a.q_w : a.k_w);
        if (w) {
            float ss = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) ss += x[e] * x[e] + y[e] * y[e];
#pragma unroll
            for (int off = LPH / 2; off > 0; off >>= 1) ss += __shfl_xor(ss, off, 64);
            const float inv = 1.0f / sqrtf(ss / (float)D + a.eps);
            if (on) {
                float w0[4], w1[4];
                kv_load4(w + d0, w0);
                kv_load4(w + d1, w1);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = x[e] * inv * w0[e];
                    y[e] = y[e] * inv * w1[e];
                }
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
            float amax = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) amax = fmaxf(amax, fmaxf(fabsf(x[e]), fabsf(y[e])));
#pragma unroll
            for (int off = LPH / 2; off > 0; off >>= 1) amax = fmaxf(amax, __shfl_xor(amax, off, 64));
            amax = amax >= kKvTiny ? amax : 0.0f;
            const float inv = amax > 0.0f ? Q / amax : 0.0f;
            float u[4], v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                u[e] = x[e] * inv;
                v[e] = y[e] * inv;
            }
            if (on && page >= 0) {
                *(uint32_t*)(o + d0) = kv_encode4<FMT>(u);
                *(uint32_t*)(o + d1) = kv_encode4<FMT>(v);
                if (j == 0) (is_v ? kv.vs : kv.ks)[r] = amax / Q;
            }
        }
    }
}

// kv_read: kReadRows packed rows per workgroup. A page holds a head's tokens next to each other, so
// the threads walk (k or v, head, row, 8 values) with the row inside the head: neighbouring threads
// read one stretch of a page.
constexpr int kReadRows = 16;
template <typename T, int FMT>
__global__ __launch_bounds__(256) void kv_read_kernel(KvArgs a, T* k_out, int64_t ld_k, T* v_out, int64_t ld_v) {
    using E = typename KvElem<T, FMT>::type;
    __shared__ int s_page[kReadRows], s_pos[kReadRows];
    if (blockIdx.x == 0) kv_check_seqs(a, threadIdx.x, 256);
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
    const int D = a.D, pieces = D / 8, per = pieces * kReadRows;
    for (int i = threadIdx.x; i < 2 * a.Hkv * per; i += 256) {
        const int hh = i / per, r = (i % per) / pieces, d = (i % pieces) * 8;
        const int page = s_page[r];
        if (page < 0) continue;
        const bool is_v = hh >= a.Hkv;
        const int h = is_v ? hh - a.Hkv : hh;
        const int64_t row = kv_pool_row(a, page, h, s_pos[r]);
        const E* p = (const E*)(is_v ? a.v : a.k) + row * D + d;
        T* o = (is_v ? v_out + (t0 + r) * ld_v : k_out + (t0 + r) * ld_k) + (int64_t)h * D + d;
        if constexpr (FMT == SSM_KV_ACT) {
            T v[8];
            load16(p, v);
            store16(o, v);
        } else {
            const float sc = (is_v ? a.vs : a.ks)[row];
            const uint2 w = *(const uint2*)p;
            float x[4], y[4];
            kv_decode4<FMT>(w.x, x);
            kv_decode4<FMT>(w.y, y);
            T v[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = from_f32<T>(x[e] * sc);
                v[4 + e] = from_f32<T>(y[e] * sc);
            }
            store16(o, v);
        }
    }
}

template <typename T, int FMT> hipError_t append_launch(const KvAppendArgs& a, hipStream_t s) {
    const int lph = a.kv.D <= 64 ? 8 : a.kv.D <= 128 ? 16 : 32;
    const int rounds = (a.kv.Hq + 2 * a.kv.Hkv + 256 / lph - 1) / (256 / lph);
    // few tokens: the heads spread over workgroups; many: one workgroup takes a token's heads
    const int slices = (int)(a.kv.T >= 1024 ? 1 : rounds);
    const dim3 grid((unsigned)a.kv.T, (unsigned)slices), block(256);
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
    const dim3 grid((unsigned)((a.T + kReadRows - 1) / kReadRows)), block(256);
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
