// vbq_sequences.cuh — device helpers of the calls on packed sequences
// (vbq_conv.cu, vbq_delta.cu, vbq_delta_chunk.cu): where a sequence's rows and
// state are, and loads of eight neighbouring values.
#pragma once

#include <cuda_bf16.h>

#include "vbq_decode.h"
#include "vbq_device.cuh"

namespace vbq {
namespace {

struct SeqRange {
    int lo, n;                       // first row, rows
    int slot;                        // < 0: unused
    bool fresh;
};

// Whatever `starts` holds, the rows are within 0..tokens. `report`: this thread records a slot outside the pool.
__device__ __forceinline__ SeqRange seq_range(const vbq_sequences& q, int b, int64_t n_slots, bool report, uint32_t* status) {
    SeqRange r;
    const int tokens = (int)q.tokens;
    r.slot = q.slots ? q.slots[b] : b;
    r.fresh = q.fresh && q.fresh[b] != 0;
    if (q.starts) {
        r.lo = min(max(q.starts[b], 0), tokens);
        r.n = max(min(q.starts[b + 1], tokens) - r.lo, 0);
    } else {
        r.lo = b * q.rows;
        r.n = q.rows;
    }
    if (r.slot >= n_slots) {
        if (report) atomicOr(status, VBQ_DEVICE_SLOT);
        r.slot = -1;
    }
    return r;
}

template <bool F32>
__device__ __forceinline__ void load8(float (&x)[8], const void* base, int64_t at) {
    if constexpr (F32) {
        const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at);
        const float4 a = p[0], b = p[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint4 pack_bf16x8(const float (&x)[8]) {
    return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// x / (1 + e^-x), within a few and |x| ulps of fp32 (the exponent's rounding); below -87, where it is smaller than 1e-35, 0
__device__ __forceinline__ float silu(float x) {
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * -1.44269504f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return x * r;
}

// two floats at a time
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 y;
    asm("{.reg .b64 a, b, y; mov.b64 a, {%2, %3}; mov.b64 b, {%4, %5}; mul.rn.f32x2 y, a, b; mov.b64 {%0, %1}, y;}"
        : "=f"(y.x), "=f"(y.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return y;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 y;
    asm("{.reg .b64 a, b, c, y; mov.b64 a, {%2, %3}; mov.b64 b, {%4, %5}; mov.b64 c, {%6, %7}; fma.rn.f32x2 y, a, b, c; mov.b64 {%0, %1}, y;}"
        : "=f"(y.x), "=f"(y.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return y;
}

}  // namespace
}  // namespace vbq
