// vbq_conv.cu — the short causal convolution of a linear-attention layer:
// y_t = bias + sum_j w_j x_{t - taps + 1 + j} per channel, its silu, BF16 out;
// the last taps - 1 inputs of a sequence are carried between calls.
//
// Two to four multiplications a value: bytes bound it. A thread takes 8
// channels (a 16-byte load of BF16) of a tile of rows and carries the window in
// registers, so a row is read once, but for the taps - 1 before a tile, which
// the tile before has just brought into L2. A sequence's first tile reads its
// carried inputs and also writes the new ones: nobody else touches its slot,
// so no order between blocks is needed, and a tile is never shorter than the
// window (CONV_ROWS >= taps - 1), so no other tile reaches back to them.
#include "vbq_kernels.h"
#include "vbq_sequences.cuh"

namespace vbq {
namespace {

constexpr int CONV_THREADS = 128;
constexpr int CONV_ROWS = 32;        // rows of a tile
constexpr int CONV_AHEAD = 4;        // rows loaded together

// Tile `t` of the call is tile *tile of sequence b. With `starts`, sequence b's tiles are among numbers starts[b] / ROWS + b
// and on: a sequence of n rows spans at most floor(starts[b + 1] / ROWS) - floor(starts[b] / ROWS) + 1 of them, so the
// numbers of two sequences are apart and no prefix sum over the batch is needed. Each round of the search narrows b to a
// 32nd, a lane each.
__device__ __forceinline__ int find_tile(const vbq_sequences& q, int t, int* tile) {
    if (!q.starts) {
        const int per = (q.rows + CONV_ROWS - 1) / CONV_ROWS, b = t / per;
        *tile = t - b * per;
        return b;
    }
    const int lane = threadIdx.x & 31;
    int b = 0, span = q.batch, first = 0;
    while (span > 0) {
        const int step = (span + 31) / 32, i = b + lane * step;
        int f = 0;
        bool before = false;
        if (lane * step < span) {
            f = min(max(q.starts[i], 0), (int)q.tokens) / CONV_ROWS + i;
            before = f <= t;
        }
        const uint32_t m = __ballot_sync(0xffffffffu, before);
        if (m == 0) return -1;
        const int last = 31 - __clz(m);
        first = __shfl_sync(0xffffffffu, f, last);
        b += last * step;
        span = step == 1 ? 0 : min(step, q.batch - b);
    }
    *tile = t - first;
    return b;
}

template <bool F32, int TAPS>
__global__ void __launch_bounds__(CONV_THREADS) causal_conv_kernel(Conv c) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int ch = (int)(blockIdx.y * CONV_THREADS + threadIdx.x) * 8;
    int tile = 0;
    const int b = find_tile(c.seq, (int)blockIdx.x, &tile);
    if (b < 0 || ch >= c.channels) return;
    const SeqRange r = seq_range(c.seq, b, c.n_slots, ch == 0 && tile == 0);
    const int64_t t0 = (int64_t)tile * CONV_ROWS;
    if (t0 >= r.n) return;
    const int rows = min(CONV_ROWS, (int)(r.n - t0));
    const int64_t row0 = r.lo + t0;
    uint16_t* out = c.out + row0 * c.channels + ch;
    if (r.slot < 0) {
        for (int i = 0; i < rows; ++i) *reinterpret_cast<uint4*>(out + (int64_t)i * c.channels) = make_uint4(0, 0, 0, 0);
        return;
    }
    float w[TAPS][8], bias[8] = {}, win[TAPS - 1][8];                // win[j]: the input TAPS - 1 - j rows before
    {
        float wide[TAPS * 8];
        const float4* p = reinterpret_cast<const float4*>(c.weight + (int64_t)ch * TAPS);
#pragma unroll
        for (int i = 0; i < 2 * TAPS; ++i) {
            const float4 v = p[i];
            wide[4 * i] = v.x; wide[4 * i + 1] = v.y; wide[4 * i + 2] = v.z; wide[4 * i + 3] = v.w;
        }
#pragma unroll
        for (int j = 0; j < TAPS; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) w[j][e] = wide[e * TAPS + j];
    }
    if (c.bias) load8<true>(bias, c.bias, ch);
    const int64_t at = row0 * c.x_stride + ch;
    if (tile > 0) {
#pragma unroll
        for (int j = 0; j < TAPS - 1; ++j) load8<F32>(win[j], c.x, at - (int64_t)(TAPS - 1 - j) * c.x_stride);
    } else {
        float* carried = c.state + (int64_t)r.slot * (TAPS - 1) * c.channels + ch;
#pragma unroll
        for (int j = 0; j < TAPS - 1; ++j) {
            if (r.fresh) {
#pragma unroll
                for (int e = 0; e < 8; ++e) win[j][e] = 0.f;
            } else {
                load8<true>(win[j], carried, (int64_t)j * c.channels);
            }
        }
        // the sequence's last TAPS - 1 inputs: of x, or for a shorter one of what was carried
#pragma unroll
        for (int j = 0; j < TAPS - 1; ++j) {
            float last[8];
            if (r.n + j >= TAPS - 1) {
                load8<F32>(last, c.x, at + (int64_t)(r.n + j - (TAPS - 1)) * c.x_stride);
            } else {
#pragma unroll
                for (int m = 0; m < TAPS - 1; ++m)
                    if (m == r.n + j)
#pragma unroll
                        for (int e = 0; e < 8; ++e) last[e] = win[m][e];
            }
            float4* p = reinterpret_cast<float4*>(carried + (int64_t)j * c.channels);
            p[0] = make_float4(last[0], last[1], last[2], last[3]);
            p[1] = make_float4(last[4], last[5], last[6], last[7]);
        }
    }
    for (int i0 = 0; i0 < rows; i0 += CONV_AHEAD) {
        float x[CONV_AHEAD][8];
#pragma unroll
        for (int i = 0; i < CONV_AHEAD; ++i)
            if (i0 + i < rows) load8<F32>(x[i], c.x, at + (int64_t)(i0 + i) * c.x_stride);
#pragma unroll
        for (int i = 0; i < CONV_AHEAD; ++i) {
            if (i0 + i >= rows) break;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float s = bias[e];
#pragma unroll
                for (int j = 0; j < TAPS - 1; ++j) s = fmaf(w[j][e], win[j][e], s);
                s = fmaf(w[TAPS - 1][e], x[i][e], s);
                y[e] = c.silu ? silu(s) : s;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
                for (int j = 0; j + 1 < TAPS - 1; ++j) win[j][e] = win[j + 1][e];
                win[TAPS - 2][e] = x[i][e];
            }
            *reinterpret_cast<uint4*>(out + (int64_t)(i0 + i) * c.channels) = pack_bf16x8(y);
        }
    }
}

}  // namespace

cudaError_t launch_causal_conv(const Conv& c, cudaStream_t s) {
    const vbq_sequences& q = c.seq;
    const int64_t tiles = q.starts ? q.tokens / CONV_ROWS + q.batch : (int64_t)((q.rows + CONV_ROWS - 1) / CONV_ROWS) * q.batch;
    const dim3 grid((unsigned)tiles, (unsigned)((c.channels / 8 + CONV_THREADS - 1) / CONV_THREADS));
    const auto go = [&](auto kernel) { return launch_dependent(kernel, grid, CONV_THREADS, 0, s, c); };
    if (c.f32) return c.taps == 2 ? go(causal_conv_kernel<true, 2>) : c.taps == 3 ? go(causal_conv_kernel<true, 3>) : go(causal_conv_kernel<true, 4>);
    return c.taps == 2 ? go(causal_conv_kernel<false, 2>) : c.taps == 3 ? go(causal_conv_kernel<false, 3>) : go(causal_conv_kernel<false, 4>);
}

cudaError_t read_device_status_conv(uint32_t* status) {
    cudaError_t e = cudaMemcpyFromSymbol(status, g_device_status, sizeof(uint32_t));
    if (e != cudaSuccess || *status == 0) return e;
    const uint32_t zero = 0;
    return cudaMemcpyToSymbol(g_device_status, &zero, sizeof(uint32_t));
}

}  // namespace vbq
