// vbq_conv.cu — the short causal convolution of a linear-attention layer:
// y_t = bias + sum_j w_j x_{t - taps + 1 + j} per channel, its silu, BF16 out;
// the last taps - 1 inputs of a sequence are carried between calls.
//
// Bytes bound it, instructions next (4 multiply-adds and a silu a value). A
// thread takes 4 channels of a tile of rows, two an instruction, loads 8 rows
// ahead and carries the window in registers, so a row is read once, but for the
// taps - 1 before a tile, which the tile before has just brought into L2. 14145
// rows of 8192 channels, BF16, 4 taps: 81 us, 5.75 TB/s; 4 rows ahead 84, tiles
// of 64 rows 80, but half the blocks for a short prompt, blocks of 256 threads
// 90, registers for 6 blocks an SM 113. A sequence's first tile reads its
// carried inputs and also writes the new ones: nobody else touches its slot,
// so no order between blocks is needed, and a tile is never shorter than the
// window (CONV_ROWS >= taps - 1), so no other tile reaches back to them.
#include "vbq_kernels.h"
#include "vbq_sequences.cuh"

namespace vbq {
namespace {

constexpr int CONV_THREADS = 128;
constexpr int CONV_ROWS = 32;        // rows of a tile
constexpr int CONV_AHEAD = 8;        // rows loaded together, ahead of their use

// Up to 2^31 - 1 rows: no sum here passes 32 bits.
__host__ __device__ __forceinline__ int tiles_of(int rows) { return rows / CONV_ROWS + (rows % CONV_ROWS != 0); }

// Tile `t` of the call is tile *tile of sequence b. With `starts`, sequence b's tiles are among numbers starts[b] / ROWS + b
// and on: a sequence of n rows spans at most floor(starts[b + 1] / ROWS) - floor(starts[b] / ROWS) + 1 of them, so the
// numbers of two sequences are apart and no prefix sum over the batch is needed. Each round of the search narrows b to a
// 32nd, a lane each.
__device__ __forceinline__ int find_tile(const vbq_sequences& q, int t, int* tile) {
    if (!q.starts) {
        const int per = tiles_of(q.rows), b = t / per;
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

// Four neighbouring values of a row, as they come and in fp32.
template <bool F32>
struct Four {
    uint4 raw;                       // BF16: the first two words
    __device__ __forceinline__ void load(const void* x, int64_t at) {
        if constexpr (F32) {
            raw = *reinterpret_cast<const uint4*>(static_cast<const float*>(x) + at);
        } else {
            const uint2 a = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(x) + at);
            raw.x = a.x; raw.y = a.y;
        }
    }
    __device__ __forceinline__ void values(float2 (&v)[2]) const {
        if constexpr (F32) {
            v[0] = make_float2(__uint_as_float(raw.x), __uint_as_float(raw.y));
            v[1] = make_float2(__uint_as_float(raw.z), __uint_as_float(raw.w));
        } else {
            v[0] = make_float2(__uint_as_float(raw.x << 16), __uint_as_float(raw.x & 0xffff0000u));
            v[1] = make_float2(__uint_as_float(raw.y << 16), __uint_as_float(raw.y & 0xffff0000u));
        }
    }
};

template <bool F32, int TAPS>
__global__ void __launch_bounds__(CONV_THREADS) causal_conv_kernel(Conv c) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int PAST = TAPS - 1;
    const int ch = (int)(blockIdx.y * CONV_THREADS + threadIdx.x) * 4;
    int tile = 0;
    const int b = find_tile(c.seq, (int)blockIdx.x, &tile);
    if (b < 0 || ch >= c.channels) return;
    const SeqRange r = seq_range(c.seq, b, c.n_slots, ch == 0 && tile == 0, c.status);
    const int64_t t0 = (int64_t)tile * CONV_ROWS;
    if (t0 >= r.n) return;
    const int rows = min(CONV_ROWS, (int)(r.n - t0));
    const int64_t row0 = r.lo + t0;
    uint16_t* out = c.out + row0 * c.channels + ch;
    if (r.slot < 0) {
        for (int i = 0; i < rows; ++i) *reinterpret_cast<uint2*>(out + (int64_t)i * c.channels) = make_uint2(0, 0);
        return;
    }
    const int64_t at = row0 * c.x_stride + ch;
    Four<F32> next[CONV_AHEAD];
#pragma unroll
    for (int i = 0; i < CONV_AHEAD; ++i) next[i].load(c.x, at + min(i, rows - 1) * c.x_stride);
    float2 w[TAPS][2], bias[2] = {}, line[PAST + CONV_AHEAD][2];     // line: the inputs before the rows worked on, and theirs
    {
        float wide[TAPS * 4];
        const float4* p = reinterpret_cast<const float4*>(c.weight + (int64_t)ch * TAPS);
#pragma unroll
        for (int i = 0; i < TAPS; ++i) {
            const float4 v = p[i];
            wide[4 * i] = v.x; wide[4 * i + 1] = v.y; wide[4 * i + 2] = v.z; wide[4 * i + 3] = v.w;
        }
#pragma unroll
        for (int j = 0; j < TAPS; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) w[j][e] = make_float2(wide[2 * e * TAPS + j], wide[(2 * e + 1) * TAPS + j]);
    }
    if (c.bias) {
        const float4 v = *reinterpret_cast<const float4*>(c.bias + ch);
        bias[0] = make_float2(v.x, v.y);
        bias[1] = make_float2(v.z, v.w);
    }
    if (tile > 0) {
#pragma unroll
        for (int j = 0; j < PAST; ++j) {
            Four<F32> x;
            x.load(c.x, at - (int64_t)(PAST - j) * c.x_stride);
            x.values(line[j]);
        }
    } else {
        float* carried = c.state + (int64_t)r.slot * PAST * c.channels + ch;
#pragma unroll
        for (int j = 0; j < PAST; ++j) {
            Four<true> x = {make_uint4(0, 0, 0, 0)};
            if (!r.fresh) x.load(carried, (int64_t)j * c.channels);
            x.values(line[j]);
        }
        // the sequence's last PAST inputs: of x, or for a shorter one of what was carried
#pragma unroll
        for (int j = 0; j < PAST; ++j) {
            float2 last[2];
            if (r.n >= PAST - j) {
                Four<F32> x;
                x.load(c.x, at + (int64_t)(r.n - (PAST - j)) * c.x_stride);
                x.values(last);
            } else {
#pragma unroll
                for (int m = 0; m < PAST; ++m)
                    if (m - j == r.n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) last[e] = line[m][e];
            }
            *reinterpret_cast<float4*>(carried + (int64_t)j * c.channels) = make_float4(last[0].x, last[0].y, last[1].x, last[1].y);
        }
    }
#pragma unroll 1
    for (int i0 = 0; i0 < rows; i0 += CONV_AHEAD) {
#pragma unroll
        for (int i = 0; i < CONV_AHEAD; ++i) next[i].values(line[PAST + i]);
        if (i0 + CONV_AHEAD < rows)
#pragma unroll
            for (int i = 0; i < CONV_AHEAD; ++i) next[i].load(c.x, at + min(i0 + CONV_AHEAD + i, rows - 1) * c.x_stride);
        uint16_t* o = out + (int64_t)i0 * c.channels;
#pragma unroll
        for (int i = 0; i < CONV_AHEAD; ++i) {
            uint32_t y[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float2 s = bias[e];
#pragma unroll
                for (int j = 0; j < TAPS; ++j) s = fma2(w[j][e], line[i + j][e], s);
                y[e] = c.silu ? pack_bf16(silu(s.x), silu(s.y)) : pack_bf16(s.x, s.y);
            }
            if (i0 + i < rows) *reinterpret_cast<uint2*>(o + (int64_t)i * c.channels) = make_uint2(y[0], y[1]);
        }
#pragma unroll
        for (int j = 0; j < PAST; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) line[j][e] = line[CONV_AHEAD + j][e];
    }
}

}  // namespace

cudaError_t launch_causal_conv(const Conv& c, cudaStream_t s) {
    const vbq_sequences& q = c.seq;
    const int64_t tiles = q.starts ? q.tokens / CONV_ROWS + q.batch : (int64_t)tiles_of(q.rows) * q.batch;
    const dim3 grid((unsigned)tiles, (unsigned)((c.channels / 4 + CONV_THREADS - 1) / CONV_THREADS));
    const auto go = [&](auto kernel) { return launch_dependent(kernel, grid, CONV_THREADS, 0, s, c); };
    if (c.f32) return c.taps == 2 ? go(causal_conv_kernel<true, 2>) : c.taps == 3 ? go(causal_conv_kernel<true, 3>) : go(causal_conv_kernel<true, 4>);
    return c.taps == 2 ? go(causal_conv_kernel<false, 2>) : c.taps == 3 ? go(causal_conv_kernel<false, 3>) : go(causal_conv_kernel<false, 4>);
}

}  // namespace vbq
