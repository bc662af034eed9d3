// vbq_delta.cuh — what the two kernels of the gated delta rule share (internal).
#pragma once

#include "vbq_sequences.cuh"

namespace vbq {
namespace {

constexpr float DELTA_UNIT_EPS = 1e-6f;          // of the unit length of q and k
constexpr float DELTA_MOST_DECAY = -100.f;       // log decays below it count as it

// A token's log decay and beta from what the call gives for them. NaN stays NaN.
struct Gate { float g, beta; };
__device__ __forceinline__ float gate_value(const void* p, bool f32, int64_t at) {
    return f32 ? static_cast<const float*>(p)[at] : __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[at] << 16);
}
__device__ __forceinline__ Gate gate_of(float a, float b, bool raw, float rate, float bias) {   // rate: exp(a_log)
    Gate r = {a, b};
    if (raw) {
        const float z = a + bias;
        r.g = -rate * (fmaxf(z, 0.f) + log1pf(expf(-fabsf(z))));
        r.beta = 1.f / (1.f + expf(-b));
        if (z != z) r.g = z;
    }
    r.g = r.g > 0.f ? 0.f : r.g < DELTA_MOST_DECAY ? DELTA_MOST_DECAY : r.g;
    return r;
}

}  // namespace

// Sequences of more than `above` rows, 64 tokens at a time on the tensor cores (vbq_delta_chunk.cu).
cudaError_t launch_delta_chunks(const Delta& d, int above, int sms, cudaStream_t s);

}  // namespace vbq
