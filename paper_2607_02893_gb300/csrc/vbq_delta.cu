// vbq_delta.cu — the gated delta rule, token by token: per head, with the state
// S (head_k x head_v, fp32), S <- e^g S; u = beta (v - S^T k); S <- S + k u^T;
// o = S^T q.
//
// The columns of S do not meet: a warp takes 16 of them and holds all their
// rows in registers, 4 columns a lane and the rows split over 8 groups of
// lanes, so a token needs no exchange but shuffles within the warp. Both
// products are taken of the state before the token, o = e^g S^T q + (q.k) u, so
// their sums go through the shuffles together.
//
// A single token is bound by the state's bytes, 128 KB a head of 128 x 128.
#include "vbq_delta.cuh"
#include "vbq_kernels.h"

namespace vbq {
namespace {

constexpr int DR_WARPS = 2;                      // of a block; 16 columns each
constexpr int DR_COLS = 16 * DR_WARPS;
constexpr int DELTA_ROWS = 16;                  // a sequence of more goes by chunks

template <bool F32, int DK>
__global__ void __launch_bounds__(32 * DR_WARPS) delta_rows_kernel(Delta d, int most) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int PER = DK / 8;                  // rows of the state in a lane
    const int slices = d.head_v / DR_COLS;
    const int unit = (int)(blockIdx.x / slices), slice = (int)(blockIdx.x - unit * slices);
    const int b = unit / d.heads, h = unit - b * d.heads;
    const int lane = threadIdx.x & 31, part = lane >> 2;
    const int col = slice * DR_COLS + (threadIdx.x >> 5) * 16 + (lane & 3) * 4;
    const SeqRange r = seq_range(d.seq, b, d.n_slots, h == 0 && slice == 0 && threadIdx.x == 0);
    if (r.n == 0 || r.n > most) return;
    const int64_t out_row = (int64_t)d.heads * d.head_v;
    uint16_t* out = d.out + r.lo * out_row + h * d.head_v + col;
    if (r.slot < 0) {
        for (int t = part; t < r.n; t += 8) *reinterpret_cast<uint2*>(out + t * out_row) = make_uint2(0, 0);
        return;
    }
    float* state = d.state + ((int64_t)r.slot * d.heads + h) * DK * d.head_v + (int64_t)part * PER * d.head_v + col;
    float4 S[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i)
        S[i] = r.fresh ? make_float4(0.f, 0.f, 0.f, 0.f) : *reinterpret_cast<const float4*>(state + (int64_t)i * d.head_v);
    const int hk = h / (d.heads / d.k_heads);
    const bool raw = d.a_log != nullptr;
    const float rate = raw ? expf(d.a_log[h]) : 0.f, bias = raw ? d.dt_bias[h] : 0.f;
    for (int t = 0; t < r.n; ++t) {
        const int64_t row = (int64_t)r.lo + t;
        float k[PER], q[PER];
#pragma unroll
        for (int i = 0; i < PER; i += 8) {
            float x[8];
            load8<F32>(x, d.k, row * d.k_stride + hk * DK + part * PER + i);
#pragma unroll
            for (int e = 0; e < 8; ++e) k[i + e] = x[e];
            load8<F32>(x, d.q, row * d.q_stride + hk * DK + part * PER + i);
#pragma unroll
            for (int e = 0; e < 8; ++e) q[i + e] = x[e];
        }
        float v[4];
        if constexpr (F32) {
            const float4 x = *reinterpret_cast<const float4*>(static_cast<const float*>(d.v) + row * d.v_stride + h * d.head_v + col);
            v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
        } else {
            const uint2 x = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(d.v) + row * d.v_stride + h * d.head_v + col);
            v[0] = __uint_as_float(x.x << 16); v[1] = __uint_as_float(x.x & 0xffff0000u);
            v[2] = __uint_as_float(x.y << 16); v[3] = __uint_as_float(x.y & 0xffff0000u);
        }
        const Gate g = gate_of(gate_value(d.decay, d.gate_f32, row * d.decay_stride + h),
                               gate_value(d.beta, d.gate_f32, row * d.beta_stride + h), raw, rate, bias);
        // kk, qq, q.k; then k.S and q.S of four columns
        float s[11] = {};
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            s[0] = fmaf(k[i], k[i], s[0]);
            s[1] = fmaf(q[i], q[i], s[1]);
            s[2] = fmaf(q[i], k[i], s[2]);
            s[3] = fmaf(k[i], S[i].x, s[3]);
            s[4] = fmaf(k[i], S[i].y, s[4]);
            s[5] = fmaf(k[i], S[i].z, s[5]);
            s[6] = fmaf(k[i], S[i].w, s[6]);
            s[7] = fmaf(q[i], S[i].x, s[7]);
            s[8] = fmaf(q[i], S[i].y, s[8]);
            s[9] = fmaf(q[i], S[i].z, s[9]);
            s[10] = fmaf(q[i], S[i].w, s[10]);
        }
#pragma unroll
        for (int o = 4; o < 32; o <<= 1)
#pragma unroll
            for (int i = 0; i < 11; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
        const float ck = d.normalize ? 1.f / sqrtf(s[0] + DELTA_UNIT_EPS) : 1.f;
        const float cq = d.scale * (d.normalize ? 1.f / sqrtf(s[1] + DELTA_UNIT_EPS) : 1.f);
        const float keep = expf(g.g), qk = cq * ck * s[2];
        float u[4], o4[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u[j] = g.beta * (v[j] - keep * (ck * s[3 + j]));
            o4[j] = fmaf(qk, u[j], keep * (cq * s[7 + j]));
            u[j] *= ck;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            S[i].x = fmaf(k[i], u[0], keep * S[i].x);
            S[i].y = fmaf(k[i], u[1], keep * S[i].y);
            S[i].z = fmaf(k[i], u[2], keep * S[i].z);
            S[i].w = fmaf(k[i], u[3], keep * S[i].w);
        }
        if (part == 0) *reinterpret_cast<uint2*>(out + t * out_row) = make_uint2(pack_bf16(o4[0], o4[1]), pack_bf16(o4[2], o4[3]));
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) *reinterpret_cast<float4*>(state + (int64_t)i * d.head_v) = S[i];
}

cudaError_t launch_rows(const Delta& d, int most, cudaStream_t s) {
    const dim3 grid((unsigned)((int64_t)d.seq.batch * d.heads * (d.head_v / DR_COLS)));
    const auto go = [&](auto kernel) { return launch_dependent(kernel, grid, 32 * DR_WARPS, 0, s, d, most); };
    if (d.f32) return d.head_k == 64 ? go(delta_rows_kernel<true, 64>) : go(delta_rows_kernel<true, 128>);
    return d.head_k == 64 ? go(delta_rows_kernel<false, 64>) : go(delta_rows_kernel<false, 128>);
}

}  // namespace

// Sequences of up to DELTA_ROWS rows go token by token, longer ones by chunks. Where the call's may be of both kinds, both
// kernels run, each over its own.
cudaError_t launch_delta_rule(const Delta& d, cudaStream_t s) {
    int sms = 0;
    const int err = device_sms(&sms);
    if (err != 0) return (cudaError_t)err;
    if (d.seq.rows <= DELTA_ROWS) return launch_rows(d, INT32_MAX, s);
    if (d.seq.starts && d.seq.batch > 1) {
        const cudaError_t e = launch_rows(d, DELTA_ROWS, s);
        return e != cudaSuccess ? e : launch_delta_chunks(d, DELTA_ROWS, sms, s);
    }
    return launch_delta_chunks(d, 0, sms, s);
}

cudaError_t read_device_status_delta(uint32_t* status) {
    uint32_t chunks = 0;
    cudaError_t e = read_device_status_delta_chunks(&chunks);
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(status, g_device_status, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    const uint32_t mine = *status, zero = 0;
    *status |= chunks;
    return mine == 0 ? cudaSuccess : cudaMemcpyToSymbol(g_device_status, &zero, sizeof(uint32_t));
}

}  // namespace vbq
