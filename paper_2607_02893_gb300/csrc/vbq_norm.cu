// vbq_norm.cu — the residual addition and the root-mean-square norm before a
// product: r' = type(r + x), out = BF16(r' * rsqrt(mean(r'^2) + eps) * w).
//
// One block per row, the row's values in registers between the two uses, so
// x, r and w are read once and r' and out written once. The sum of squares is
// held in fp32: per thread in element order, then a fixed tree over the lanes
// and the warps, so results do not vary between calls. r' is rounded to the
// residual's type first and the norm is of the rounded values: it is a function
// of the stream as it is stored. BF16 is rounded to once, at the output (the
// products' activation type).
//
// One token is bound by its launch, two trips to memory and, between the other
// kernels of a decode step, by fetching its instructions: kernels that know the
// types, and that every row is whole vectors and fits the registers, have few of
// them (1 x 768: 1.2 us in a graph, 2.2 by one kernel for everything; a step of
// 22 layers of width 2048, 45 norms: 712 us against 784). 256 x 4096 takes 2.7
// us, 3.9 TB/s; 200 x 1001, whose rows start anywhere, 2.9 us (13.6 with single
// loads).
#include <cuda_bf16.h>

#include "vbq_decode.h"
#include "vbq_device.cuh"
#include "vbq_kernels.h"

namespace vbq {
namespace {

enum Type { ANY, NONE, F32, BF16 };

__device__ __forceinline__ float bf16_f32(uint32_t bits16) { return __uint_as_float(bits16 << 16); }
__device__ __forceinline__ uint32_t f32_bf16(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }

// A row is cut at the multiples of 4 elements of the whole array, which vector loads need, wherever the row itself
// starts: items 0 .. vecs - 1 are vectors, the items after them the single values before the first and after the last.
// EVEN: the width is a multiple of 4, so every row is vectors only.
template <bool EVEN>
struct Row {
    int64_t base;                    // of the row's first element
    int head, vecs, items;
    __device__ Row(int64_t row, int width) {
        base = row * width;
        head = EVEN ? 0 : min(width, (int)(-base & 3));
        vecs = (width - head) / 4;
        items = EVEN ? vecs : vecs + width - 4 * vecs;
    }
    __device__ __forceinline__ bool wide(int item) const { return EVEN || item < vecs; }
    __device__ __forceinline__ int first(int item) const {               // element of the row
        return EVEN ? 4 * item : item < vecs ? head + 4 * item : item < vecs + head ? item - vecs : item - vecs + 4 * vecs;
    }
};

// An item's values in fp32 (a single one: v[0], zeros beside it); `wide`: it is a vector, on its boundary.
__device__ __forceinline__ float4 load_item(const void* p, bool f32, int64_t at, bool wide) {
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (f32) {
        const float* q = static_cast<const float*>(p) + at;
        if (wide) v = *reinterpret_cast<const float4*>(q); else v.x = *q;
    } else {
        const uint16_t* q = static_cast<const uint16_t*>(p) + at;
        if (wide) {
            const uint2 a = *reinterpret_cast<const uint2*>(q);
            v = make_float4(bf16_f32(a.x & 0xffffu), bf16_f32(a.x >> 16), bf16_f32(a.y & 0xffffu), bf16_f32(a.y >> 16));
        } else {
            v.x = bf16_f32(*q);
        }
    }
    return v;
}
__device__ __forceinline__ void store_item(float4 v, void* p, bool f32, int64_t at, bool wide) {
    if (f32) {
        float* q = static_cast<float*>(p) + at;
        if (wide) *reinterpret_cast<float4*>(q) = v; else *q = v.x;
    } else {
        uint16_t* q = static_cast<uint16_t*>(p) + at;
        if (wide)
            *reinterpret_cast<uint2*>(q) = make_uint2(f32_bf16(v.x) | f32_bf16(v.y) << 16, f32_bf16(v.z) | f32_bf16(v.w) << 16);
        else
            *q = (uint16_t)f32_bf16(v.x);
    }
}
// The weights of an item: their boundary is the row's own.
__device__ __forceinline__ float4 load_weights(const float* w, int j, bool wide) {
    if (wide && (j & 3)) return make_float4(w[j], w[j + 1], w[j + 2], w[j + 3]);
    return load_item(w, true, j, wide);
}

__device__ __forceinline__ float stored(float v, bool f32) { return f32 ? v : bf16_f32(f32_bf16(v)); }

// r' of an item, rounded to the residual's type (x itself without one).
__device__ __forceinline__ float4 summed(const Norm& n, bool adds, int64_t at, bool wide) {
    float4 v = load_item(n.x, n.x_f32, at, wide);
    if (!adds) return v;
    const float4 r = load_item(n.residual, n.residual_f32, at, wide);
    const bool f32 = n.residual_f32;
    return make_float4(stored(__fadd_rn(r.x, v.x), f32), stored(__fadd_rn(r.y, v.y), f32), stored(__fadd_rn(r.z, v.z), f32),
                       stored(__fadd_rn(r.w, v.w), f32));
}
__device__ __forceinline__ float squares(float4 v, float sum) { return fmaf(v.w, v.w, fmaf(v.z, v.z, fmaf(v.y, v.y, fmaf(v.x, v.x, sum)))); }
__device__ __forceinline__ float4 scaled(float4 w, float4 v, float inv) {
    return make_float4(w.x * (v.x * inv), w.y * (v.y * inv), w.z * (v.z * inv), w.w * (v.w * inv));
}

// HELD: the vectors of 4 that a thread keeps in registers. WHOLE: they are the whole row.
// X, R: the types of x and of the residual, if known.
template <bool EVEN, int HELD, bool WHOLE, Type X = ANY, Type R = ANY>
__global__ void __launch_bounds__(1024) residual_norm_kernel(Norm n) {
    if constexpr (X != ANY) n.x_f32 = X == F32;
    if constexpr (R != ANY) n.residual_f32 = R == F32;
    if constexpr (R == NONE) n.residual = nullptr;
    const bool adds = R == ANY ? n.residual != nullptr : R != NONE;
    __shared__ float part[32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    for (int64_t r = blockIdx.x; r < n.rows; r += gridDim.x) {
        const Row<EVEN> row(r, n.width);
        float4 held[HELD], w[HELD];                       // w too: its trip to memory goes beside theirs
        float sum = 0.f;
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int i = threadIdx.x + h * blockDim.x;
            if (i >= row.items) continue;
            const int j = row.first(i);
            const bool wide = row.wide(i);
            held[h] = summed(n, adds, row.base + j, wide);
            w[h] = load_weights(n.weight, j, wide);
        }
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int i = threadIdx.x + h * blockDim.x;
            if (i >= row.items) continue;
            if (adds) store_item(held[h], n.residual_out, n.residual_f32, row.base + row.first(i), row.wide(i));
            sum = squares(held[h], sum);
        }
        for (int i = threadIdx.x + HELD * blockDim.x; !WHOLE && i < row.items; i += blockDim.x) {    // past the registers
            const int64_t at = row.base + row.first(i);
            const float4 v = summed(n, adds, at, row.wide(i));
            if (adds) store_item(v, n.residual_out, n.residual_f32, at, row.wide(i));
            sum = squares(v, sum);
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
            if (i < row.items) store_item(scaled(w[h], held[h], inv), n.out, false, row.base + row.first(i), row.wide(i));
        }
        for (int i = threadIdx.x + HELD * blockDim.x; !WHOLE && i < row.items; i += blockDim.x) {
            const int j = row.first(i);
            const bool wide = row.wide(i);
            // r' again: from where this thread stored it (residual_out may be residual itself)
            const float4 v = adds ? load_item(n.residual_out, n.residual_f32, row.base + j, wide) : load_item(n.x, n.x_f32, row.base + j, wide);
            store_item(scaled(load_weights(n.weight, j, wide), v, inv), n.out, false, row.base + j, wide);
        }
    }
}

template <int HELD, Type X>
cudaError_t launch_known(const Norm& n, dim3 grid, int threads, cudaStream_t s) {
    if (!n.residual) return launch_dependent(residual_norm_kernel<true, HELD, true, X, NONE>, grid, threads, 0, s, n);
    return n.residual_f32 ? launch_dependent(residual_norm_kernel<true, HELD, true, X, F32>, grid, threads, 0, s, n)
                          : launch_dependent(residual_norm_kernel<true, HELD, true, X, BF16>, grid, threads, 0, s, n);
}

}  // namespace

// One vector a thread where every row has an SM, else two (256 x 4096: 2.7 us; one 4.6, four 4.0; more than 512 threads
// leave one block an SM).
cudaError_t launch_residual_norm(const Norm& n, cudaStream_t s) {
    int sms = 0;
    const int err = device_sms(&sms);
    if (err != 0) return (cudaError_t)err;
    const int64_t cap = 1 << 20;
    const dim3 grid((unsigned)(n.rows < cap ? n.rows : cap));
    const bool even = n.width % 4 == 0;
    if (even && n.rows <= sms && n.width <= 4096) {
        const int threads = (n.width / 4 + 31) / 32 * 32;
        return n.x_f32 ? launch_known<1, F32>(n, grid, threads, s) : launch_known<1, BF16>(n, grid, threads, s);
    }
    int threads = (n.width / 8 + 31) / 32 * 32;
    threads = threads < 64 ? 64 : threads > 1024 ? 1024 : threads;
    if (even && n.width <= 8 * threads)
        return n.x_f32 ? launch_known<2, F32>(n, grid, threads, s) : launch_known<2, BF16>(n, grid, threads, s);
    if (even) return launch_dependent(residual_norm_kernel<true, 4, false>, grid, threads, 0, s, n);
    return launch_dependent(residual_norm_kernel<false, 4, false>, grid, threads, 0, s, n);
}

}  // namespace vbq
