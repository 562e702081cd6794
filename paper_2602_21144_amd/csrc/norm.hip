// The norms around a gated block.
//
// gated_rmsnorm: per row and head, y = x / rms(x) w f(z), or the norm of x f(z). A head is read
// once, by 1 to 64 lanes of 8 values (4 times 8 above 512 values), and written once: HBM-bound,
// 16384 rows of 16 bf16 heads of 128 (201 MB) 40 us, 5.0 TB/s.
//
// block_rmsnorm: y = sum of the parts, normed with post_w, gated and scaled; r = base + y;
// RMSNorm(r) w. As residual_rmsnorm, with a second reduction in front of the add: one workgroup
// per row, whose values stay in registers between being read and written. HBM-bound: 2048 x 3584 with two bf16 parts
// and a gate (117 MB) 24 us; by 256 threads in passes of 2048 values 29, as most of the second pass is empty. The
// residual is stored past the caches, since the block between reads only the normed row (26.5 -> 24.2).
#include <algorithm>

#include "gate.h"

namespace ssm {
namespace {

template <typename T, int P>
__global__ __launch_bounds__(256) void gated_rmsnorm_kernel(const T* x, int64_t ld_x, uint32_t items, int heads, int dim,
                                                            int lanes, GatedNormArgs n, T* out, int64_t ld_out) {
    const int li = threadIdx.x & (lanes - 1);
    const uint32_t per = 256 / lanes;
    const float inv_dim = 1.0f / (float)dim;
    for (uint64_t item = (uint64_t)blockIdx.x * per + threadIdx.x / lanes; item < items; item += (uint64_t)gridDim.x * per) {
        const uint32_t row = (uint32_t)item / (uint32_t)heads, head = (uint32_t)item % (uint32_t)heads;
        const T* px = x + (int64_t)row * ld_x + (int64_t)head * dim;
        const T* pz = (const T*)n.z + (int64_t)row * n.ld_z + (int64_t)head * dim;
        const float* pw = n.w + (n.per_head ? (int64_t)head * dim : 0);
        float v[P][8], g[P][8], ss = 0.0f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int c = (p * lanes + li) * 8;
            if (c >= dim) continue;
            read8(px + c, v[p]);
            if (n.z) read8(pz + c, g[p]);
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if ((p * lanes + li) * 8 >= dim) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                g[p][e] = n.z ? gate_f(g[p][e], n.gate) : 1.0f;
                if (n.gate_first) v[p][e] *= g[p][e];
                ss += v[p][e] * v[p][e];
            }
        }
        for (int off = lanes >> 1; off > 0; off >>= 1) ss += __shfl_xor(ss, off, 64);
        const float inv = 1.0f / sqrtf(ss * inv_dim + n.eps);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int c = (p * lanes + li) * 8;
            if (c >= dim) continue;
            float w[8];
            read8(pw + c, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[p][e] = v[p][e] * inv * w[e] * (n.gate_first ? 1.0f : g[p][e]);
            write8(out + (int64_t)row * ld_out + (int64_t)head * dim + c, v[p]);
        }
    }
}

template <typename T> hipError_t gated_launch(const void* x, int64_t ld_x, int64_t rows, int heads, int dim,
                                              const GatedNormArgs& n, void* out, int64_t ld_out, hipStream_t s) {
    int lanes = 1;
    while (lanes < 64 && lanes * 8 < dim) lanes *= 2;
    const uint32_t items = (uint32_t)(rows * heads), per = 256 / lanes;
    const unsigned blocks = (unsigned)std::min<uint64_t>(((uint64_t)items + per - 1) / per, 1u << 20);
    if (dim <= 512)
        SSM_LAUNCH((gated_rmsnorm_kernel<T, 1>), dim3(blocks), dim3(256), 0, s, (const T*)x, ld_x, items, heads, dim, lanes, n,
                   (T*)out, ld_out);
    else
        SSM_LAUNCH((gated_rmsnorm_kernel<T, 4>), dim3(blocks), dim3(256), 0, s, (const T*)x, ld_x, items, heads, dim, lanes, n,
                   (T*)out, ld_out);
    return hipGetLastError();
}

constexpr int kThreads = 512, kPasses = 2;   // d <= 8 * 512 * 2

__device__ __forceinline__ float block_sum(float v, float* lds) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.0f;
    for (unsigned w = 0; w < blockDim.x / 64; ++w) s += lds[w];
    return s;
}

// P passes of 8 values per thread, by as many threads as a row then needs
template <typename BT, typename PT, typename GT, typename OT, int P>
// base may be the residual itself (in place): neither is restrict
__global__ __launch_bounds__(kThreads) void block_rmsnorm_kernel(BlockNormArgs a) {
    __shared__ float sums[2][kThreads / 64];
    const int64_t row = (int64_t)blockIdx.x * a.d;
    const int tid = threadIdx.x, d = a.d;
    const float inv_d = 1.0f / (float)d;
    float y[P][8], r[P][8], g[P][8], w[P][8], ss = 0.0f;
#pragma unroll
    for (int q = 0; q < P; ++q) {
        const int c = (q * (int)blockDim.x + tid) * 8;
        if (c >= d) continue;
        read8((const BT*)a.base + row + c, r[q]);
        if (a.gate) read8((const GT*)a.gate + (int64_t)blockIdx.x * a.ld_gate + c, g[q]);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[q][e] = 0.0f;
#pragma unroll
        for (int k = 0; k < kMaxNormParts; ++k) {
            if (k >= a.parts.n) break;
            float o[8];
            read8((const PT*)a.parts.p[k] + row + c, o);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[q][e] = k == 0 ? o[e] : y[q][e] + o[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += y[q][e] * y[q][e];
    }
    const float inv1 = a.post_w ? 1.0f / sqrtf(block_sum(ss, sums[0]) * inv_d + a.post_eps) : 1.0f;
    ss = 0.0f;
#pragma unroll
    for (int q = 0; q < P; ++q) {
        const int c = (q * (int)blockDim.x + tid) * 8;
        if (c >= d) continue;
        read8(a.w + c, w[q]);
        if (a.post_w) {
            float v[8];
            read8(a.post_w + c, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[q][e] = y[q][e] * inv1 * v[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (a.gate) y[q][e] *= gate_f(g[q][e], a.gate_fn);
            r[q][e] += a.scale * y[q][e];
            ss += r[q][e] * r[q][e];
        }
        write8_past(a.resid + row + c, r[q]);
    }
    const float inv = 1.0f / sqrtf(block_sum(ss, sums[1]) * inv_d + a.eps);
#pragma unroll
    for (int q = 0; q < P; ++q) {
        const int c = (q * (int)blockDim.x + tid) * 8;
        if (c >= d) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) r[q][e] = r[q][e] * inv * w[q][e];
        write8((OT*)a.out + row + c, r[q]);
    }
}

template <typename BT, typename PT, typename GT, typename OT> hipError_t block_launch_o(const BlockNormArgs& a, int64_t T, hipStream_t s) {
    const int passes = a.d <= 8 * kThreads ? 1 : kPasses, threads = ((a.d / 8 + passes - 1) / passes + 63) / 64 * 64;
    if (passes == 1) SSM_LAUNCH((block_rmsnorm_kernel<BT, PT, GT, OT, 1>), dim3((unsigned)T), dim3(threads), 0, s, a);
    else SSM_LAUNCH((block_rmsnorm_kernel<BT, PT, GT, OT, kPasses>), dim3((unsigned)T), dim3(threads), 0, s, a);
    return hipGetLastError();
}
template <typename BT, typename PT, typename GT> hipError_t block_launch(const BlockNormArgs& a, bool out_bf16, int64_t T, hipStream_t s) {
    return out_bf16 ? block_launch_o<BT, PT, GT, bf16>(a, T, s) : block_launch_o<BT, PT, GT, float>(a, T, s);
}
template <typename BT, typename PT>
hipError_t block_launch_g(const BlockNormArgs& a, bool gate_bf16, bool out_bf16, int64_t T, hipStream_t s) {
    return gate_bf16 ? block_launch<BT, PT, bf16>(a, out_bf16, T, s) : block_launch<BT, PT, float>(a, out_bf16, T, s);
}
template <typename BT>
hipError_t block_launch_p(const BlockNormArgs& a, bool parts_bf16, bool gate_bf16, bool out_bf16, int64_t T, hipStream_t s) {
    return parts_bf16 ? block_launch_g<BT, bf16>(a, gate_bf16, out_bf16, T, s)
                      : block_launch_g<BT, float>(a, gate_bf16, out_bf16, T, s);
}

}  // namespace

int gated_rmsnorm_max_dim() { return 64 * 8 * 4; }

hipError_t launch_gated_rmsnorm(const void* x, int64_t ld_x, bool bf16_act, int64_t T, int heads, int dim,
                                const GatedNormArgs& n, void* out, int64_t ld_out, hipStream_t s) {
    if (T <= 0) return hipSuccess;
    return bf16_act ? gated_launch<bf16>(x, ld_x, T, heads, dim, n, out, ld_out, s)
                    : gated_launch<float>(x, ld_x, T, heads, dim, n, out, ld_out, s);
}

hipError_t launch_block_rmsnorm(const BlockNormArgs& a, bool base_bf16, bool parts_bf16, bool gate_bf16, bool out_bf16,
                                int64_t T, hipStream_t s) {
    if (T <= 0) return hipSuccess;
    return base_bf16 ? block_launch_p<bf16>(a, parts_bf16, gate_bf16, out_bf16, T, s)
                     : block_launch_p<float>(a, parts_bf16, gate_bf16, out_bf16, T, s);
}

}  // namespace ssm
