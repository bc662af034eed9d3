// vbq_norm.cu — the residual addition and the root-mean-square norm before a
// product: r' = type(r + x), out = BF16(r' * rsqrt(mean(r'^2) + eps) * w).
//
// One block per row, the row's values in registers between the two uses, so
// x, r and w are read once and r' and out written once. The sum of squares is
// held in fp32: per thread in element order, then a fixed tree over the lanes
// and the warps, so results do not vary between calls. r' is rounded to the
// residual's type first and the norm is of the rounded values: it is a function
// of the stream as it is stored. BF16 is rounded to once, at the output (the
// products' activation type). One token is bound by its launch and two trips
// to memory (1 x 768: 1.8 us in a graph); 256 x 4096 takes 4.7 us, 2.3 TB/s.
#include <cuda_bf16.h>

#include "vbq_decode.h"
#include "vbq_device.cuh"

namespace vbq {
namespace {

constexpr int NORM_HELD = 16;        // values a thread keeps in registers

__device__ __forceinline__ float bf16_f32(uint32_t bits16) { return __uint_as_float(bits16 << 16); }
__device__ __forceinline__ uint32_t f32_bf16(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }

// VEC values at `at`, in fp32.
template <int VEC>
__device__ __forceinline__ void load_vec(float (&v)[VEC], const void* p, bool f32, int64_t at) {
    if constexpr (VEC == 4) {
        if (f32) {
            const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        } else {
            const uint2 a = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + at);
            v[0] = bf16_f32(a.x & 0xffffu); v[1] = bf16_f32(a.x >> 16);
            v[2] = bf16_f32(a.y & 0xffffu); v[3] = bf16_f32(a.y >> 16);
        }
    } else {
        v[0] = f32 ? static_cast<const float*>(p)[at] : bf16_f32(static_cast<const uint16_t*>(p)[at]);
    }
}
template <int VEC>
__device__ __forceinline__ void store_vec(const float (&v)[VEC], void* p, bool f32, int64_t at) {
    if constexpr (VEC == 4) {
        if (f32)
            *reinterpret_cast<float4*>(static_cast<float*>(p) + at) = make_float4(v[0], v[1], v[2], v[3]);
        else
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + at) =
                make_uint2(f32_bf16(v[0]) | f32_bf16(v[1]) << 16, f32_bf16(v[2]) | f32_bf16(v[3]) << 16);
    } else if (f32) {
        static_cast<float*>(p)[at] = v[0];
    } else {
        static_cast<uint16_t*>(p)[at] = (uint16_t)f32_bf16(v[0]);
    }
}

// r' of VEC values, rounded to the residual's type (x itself without one).
template <int VEC>
__device__ __forceinline__ void summed(float (&v)[VEC], const Norm& n, int64_t at) {
    load_vec<VEC>(v, n.x, n.x_f32, at);
    if (!n.residual) return;
    float r[VEC];
    load_vec<VEC>(r, n.residual, n.residual_f32, at);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        v[i] = __fadd_rn(r[i], v[i]);
        if (!n.residual_f32) v[i] = bf16_f32(f32_bf16(v[i]));
    }
}

template <int VEC>
__global__ void __launch_bounds__(1024) residual_norm_kernel(Norm n) {
    constexpr int HELD = NORM_HELD / VEC;
    __shared__ float part[32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int vecs = n.width / VEC;
    for (int64_t row = blockIdx.x; row < n.rows; row += gridDim.x) {
        const int64_t base = row * n.width;
        float held[HELD][VEC];
        float sum = 0.f;
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int i = threadIdx.x + h * blockDim.x;
            if (i < vecs) summed<VEC>(held[h], n, base + (int64_t)i * VEC);
        }
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int i = threadIdx.x + h * blockDim.x;
            if (i >= vecs) continue;
            if (n.residual) store_vec<VEC>(held[h], n.residual_out, n.residual_f32, base + (int64_t)i * VEC);
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum = fmaf(held[h][e], held[h][e], sum);
        }
        for (int i = threadIdx.x + HELD * blockDim.x; i < vecs; i += blockDim.x) {   // past the registers
            float v[VEC];
            summed<VEC>(v, n, base + (int64_t)i * VEC);
            if (n.residual) store_vec<VEC>(v, n.residual_out, n.residual_f32, base + (int64_t)i * VEC);
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum = fmaf(v[e], v[e], sum);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) part[warp] = sum;
        __syncthreads();
        float all = lane < warps ? part[lane] : 0.f;
#pragma unroll
        for (int o = 16; o; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
        __syncthreads();                                  // part is free for the next row
        const float inv = __fdiv_rn(1.f, __fsqrt_rn(__fadd_rn(__fdiv_rn(all, (float)n.width), n.eps)));
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int i = threadIdx.x + h * blockDim.x;
            if (i >= vecs) continue;
            float w[VEC];
            load_vec<VEC>(w, n.weight, true, (int64_t)i * VEC);
#pragma unroll
            for (int e = 0; e < VEC; ++e) w[e] *= held[h][e] * inv;
            store_vec<VEC>(w, n.out, false, base + (int64_t)i * VEC);
        }
        for (int i = threadIdx.x + HELD * blockDim.x; i < vecs; i += blockDim.x) {
            float v[VEC], w[VEC];
            // r' again: from where this thread stored it (residual_out may be residual itself)
            load_vec<VEC>(v, n.residual ? n.residual_out : n.x, n.residual ? n.residual_f32 : n.x_f32,
                          base + (int64_t)i * VEC);
            load_vec<VEC>(w, n.weight, true, (int64_t)i * VEC);
#pragma unroll
            for (int e = 0; e < VEC; ++e) w[e] *= v[e] * inv;
            store_vec<VEC>(w, n.out, false, base + (int64_t)i * VEC);
        }
    }
}

}  // namespace

cudaError_t launch_residual_norm(const Norm& n, cudaStream_t s) {
    const bool vec = n.width % 4 == 0;                    // rows then start on a vector's boundary
    const int work = vec ? n.width / 4 : n.width;
    int threads = (work + 31) / 32 * 32;
    threads = threads < 64 ? 64 : threads > 1024 ? 1024 : threads;
    const int64_t cap = 1 << 20;
    const int grid = (int)(n.rows < cap ? n.rows : cap);
    return launch_dependent(vec ? residual_norm_kernel<4> : residual_norm_kernel<1>, dim3(grid), threads, 0, s, n);
}

}  // namespace vbq
