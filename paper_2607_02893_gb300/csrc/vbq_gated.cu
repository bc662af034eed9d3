// vbq_gated.cu — the norm per head with its gate, before the output product of
// a linear-attention layer: out = BF16(x rsqrt(mean(x^2) + eps) w silu(z)).
//
// Bytes bound it: a thread holds 8 values of a head (16- or 32-byte loads) and
// the head's threads are neighbours in a warp, so the sum of squares is a few
// shuffles and nothing is read twice. Everything is fp32 but the output. 8191
// rows of 32 heads of 128, BF16 with an fp32 gate: 45.4 us, 5.9 TB/s.
#include "vbq_kernels.h"
#include "vbq_sequences.cuh"

namespace vbq {
namespace {

constexpr int GN_THREADS = 256;

// LANES: threads of a head, a power of two at least width / 8.
template <bool XF32, bool ZF32, int LANES>
__global__ void __launch_bounds__(GN_THREADS) gated_norm_kernel(GatedNorm n) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t total = n.rows * n.heads, step = (int64_t)gridDim.x * (GN_THREADS / LANES);
    const int l = threadIdx.x & (LANES - 1);
    const bool mine = l * 8 < n.width;
    float w[8] = {};
    if (mine) load8<true>(w, n.weight, l * 8);
    for (int64_t i0 = (int64_t)blockIdx.x * (GN_THREADS / LANES); i0 < total; i0 += step) {
        const int64_t i = i0 + threadIdx.x / LANES;
        const bool live = mine && i < total;
        const int64_t row = i / n.heads;
        const int64_t in_row = (i - row * n.heads) * n.width + l * 8;
        float x[8] = {}, z[8] = {};
        if (live) {
            load8<XF32>(x, n.x, row * n.x_stride + in_row);
            if (n.gate) load8<ZF32>(z, n.gate, row * n.gate_stride + in_row);
        }
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
        for (int o = LANES / 2; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const float inv = __fdiv_rn(1.f, __fsqrt_rn(__fadd_rn(__fdiv_rn(sum, (float)n.width), n.eps)));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = w[e] * (x[e] * inv);
            if (n.gate) x[e] *= silu(z[e]);
        }
        if (live) *reinterpret_cast<uint4*>(n.out + row * n.heads * n.width + in_row) = pack_bf16x8(x);
    }
}

template <int LANES>
cudaError_t launch_lanes(const GatedNorm& n, cudaStream_t s) {
    const int64_t want = (n.rows * n.heads * LANES + GN_THREADS - 1) / GN_THREADS, cap = 1 << 24;
    const dim3 grid((unsigned)(want < cap ? want : cap));
    const auto go = [&](auto kernel) { return launch_dependent(kernel, grid, GN_THREADS, 0, s, n); };
    if (n.x_f32) return n.gate_f32 ? go(gated_norm_kernel<true, true, LANES>) : go(gated_norm_kernel<true, false, LANES>);
    return n.gate_f32 ? go(gated_norm_kernel<false, true, LANES>) : go(gated_norm_kernel<false, false, LANES>);
}

}  // namespace

cudaError_t launch_gated_norm(const GatedNorm& n, cudaStream_t s) {
    return n.width <= 64 ? launch_lanes<8>(n, s) : n.width <= 128 ? launch_lanes<16>(n, s) : launch_lanes<32>(n, s);
}

}  // namespace vbq
