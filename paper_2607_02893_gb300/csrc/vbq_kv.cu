// vbq_kv.cu — writing the 4-bit key-value cache and reading it back.
//
// Append, per new token and head: the rotary rotation of q and k in fp32 (the
// pairs (i, i + r/2), i < r/2: (a, b) -> (a cos - b sin, b cos + a sin), each
// product and sum rounded once), q to BF16, and k and v quantised in groups of
// 64 as Eq. 1 does at 4 bits: s = FP16(max|x| / 7), code = round-half-even of
// the exact quotient x / s, clipped to +-7. The decisions are exact: an fp32
// estimate of a quotient is compared with thresholds that fp32 holds exactly
// (products of an FP16 number and a small half-integer or of an FP16 midpoint
// and 7), so codes and scales are a pure function of the fp32 values.
//
// A thread owns 8 values (one word of codes) and a group's 8 threads are
// neighbours in a warp: 16- or 32-byte loads, three shuffles for the maximum,
// one 4-byte store. A decoded token is a few blocks of work (48 heads of 128:
// 768 threads) and takes as long as a launch: 4.5 us in a graph with its read;
// a prompt of 256 tokens moves 8 MB, 7.1 us with its read (8.8 with 64-bit
// divisions and the partners of the rotation loaded after the position).
#include <cuda_bf16.h>

#include "vbq_decode.h"
#include "vbq_device.cuh"
#include "vbq_kernels.h"

namespace vbq {
namespace {

constexpr int KA_THREADS = 128;

template <bool F32>
__device__ __forceinline__ void load8(float (&x)[8], const void* base, int64_t at) {
    if (F32) {
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

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// FP16(amax / 7), round to nearest even, saturating at 65504. The fp32 quotient
// rounds to the right FP16 number or to a neighbour of it; the midpoints to
// both neighbours times 7 are exact in fp32 (12 + 3 significant bits) and
// decide.
__device__ __forceinline__ __half scale7(float amax) {
    if (!(amax < 65520.f * 7.f)) return __ushort_as_half(0x7bff);
    uint32_t h = __half_as_ushort(__float2half_rn(__fdiv_rn(amax, 7.f)));
    if (h >= 0x7bffu) return __ushort_as_half(0x7bff);
    const float me = half_bits(h), up = half_bits(h + 1);
    const float hi = __fmul_rn(__fadd_rn(me, up), 3.5f);                   // 7 (me + up) / 2
    if (amax > hi || (amax == hi && (h & 1u))) return __ushort_as_half((uint16_t)(h + 1));
    if (h > 0) {
        const float lo = __fmul_rn(__fadd_rn(half_bits(h - 1), me), 3.5f);
        if (amax < lo || (amax == lo && (h & 1u))) return __ushort_as_half((uint16_t)(h - 1));
    }
    return __ushort_as_half((uint16_t)h);
}

// Offset-binary code of x at scale s > 0 (NaN gives the zero level).
__device__ __forceinline__ uint32_t code4(float x, float s, float inv) {
    const float a = fabsf(x);
    float k = fminf(rintf(__fmul_rn(a, inv)), 7.f);                        // NaN and overflow: 7
    const float up = __fmul_rn(s, k + 0.5f), dn = __fmul_rn(s, k - 0.5f);
    const bool odd = ((int)k) & 1;
    if (k < 7.f && (a > up || (a == up && odd))) k += 1.f;
    else if (k > 0.f && (a < dn || (a == dn && odd))) k -= 1.f;
    if (!(a == a)) k = 0.f;
    return (uint32_t)(8 + (int)copysignf(k, x));
}

// Index: an integer that holds the words of the call (64-bit divisions are long).
template <bool F32, class Index>
__global__ void __launch_bounds__(KA_THREADS) kv_append_kernel(KvView c, KvAppend a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int d = c.head_dim, shift = __ffs(d) - 4, chunks = 1 << shift;   // d / 8, a power of two
    const int heads = a.q ? a.heads : 0;
    const int per_row = (heads + 2 * c.kv_heads) * chunks;                 // a multiple of 8
    const Index total = (Index)((int64_t)a.batch * a.rows * per_row), step = (Index)gridDim.x * KA_THREADS;
    for (Index i0 = (Index)blockIdx.x * KA_THREADS; i0 < total; i0 += step) {
        Index i = i0 + (Index)threadIdx.x;
        const bool live = i < total;                                       // whole groups: total is a multiple of 8
        if (!live) i = total - 1;
        const Index row = i / per_row;
        const int in_row = (int)(i - row * per_row);
        const int vec = in_row >> shift, ch = in_row & (chunks - 1);
        const bool is_q = vec < heads, is_k = !is_q && vec < heads + c.kv_heads;
        const int h = is_q ? vec : is_k ? vec - heads : vec - heads - c.kv_heads;
        const void* src = is_q ? a.q : is_k ? a.k : a.v;
        const int64_t at = (int64_t)row * (is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride) + (int64_t)h * d;
        // The values and their partners in the rotation, then what depends on the position: two trips to memory.
        const int64_t p = a.pos[row];
        const int half = a.rot_dim / 2;                                    // a multiple of 8
        const bool rotated = a.cos && (is_q || is_k) && ch * 8 < a.rot_dim, first = ch * 8 < half;
        const int j = first ? ch * 8 : ch * 8 - half;
        float x[8], y[8];
        load8<F32>(x, src, at + ch * 8);
        if (rotated) load8<F32>(y, src, at + (first ? ch * 8 + half : j));
        bool ok = p >= 0;
        if (ok && ((a.cos && p >= a.rot_rows) || p >= (int64_t)c.table_pages * KV_PAGE)) {
            if (live) atomicOr(&g_device_status, VBQ_DEVICE_RANGE);
            ok = false;
        }
        int64_t page = 0;
        if (ok && !is_q) page = c.table[(int64_t)(row / a.rows) * c.table_stride + p / KV_PAGE];
        if (ok && rotated) {
            float cs[8], sn[8];
            load8<true>(cs, a.cos, p * half + j);
            load8<true>(sn, a.sin, p * half + j);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float m = __fmul_rn(x[e], cs[e]), n = __fmul_rn(y[e], sn[e]);
                x[e] = first ? __fsub_rn(m, n) : __fadd_rn(m, n);
            }
        }
        if (is_q) {
            if (live)
                *reinterpret_cast<uint4*>(a.q_out + ((int64_t)row * a.heads + h) * d + ch * 8) =
                    ok ? make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]),
                                    bf16_pair(x[6], x[7]))
                       : make_uint4(0, 0, 0, 0);
        }
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(x[e]));             // fmaxf drops NaN
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (is_q || !ok || !live) continue;
        if (page < 0 || page >= c.n_pages) {
            atomicOr(&g_device_status, VBQ_DEVICE_RANGE);
            continue;
        }
        const __half sh = scale7(m);
        const float s = __half2float(sh);
        uint32_t w = 0x88888888u;
        if (s > 0.f) {
            const float inv = __fdiv_rn(1.f, s);
            w = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) w |= code4(x[e], s, inv) << (4 * e);
        }
        const int slot = (int)(p % KV_PAGE);
        uint8_t* blob = c.pages + (page * c.kv_heads + h) * kv_blob_bytes(d);
        const int krow = kv_key_row(slot);
        uint8_t* dst = is_k ? blob + krow * (d / 2) + 4 * kv_key_word(ch, d)
                            : blob + kv_values_at(d) + slot * (d / 2) + 4 * kv_value_word(ch, slot, d);
        *reinterpret_cast<uint32_t*>(dst) = kv_turned(w);
        if ((ch & 7) == 0)
            *reinterpret_cast<__half*>(blob + kv_scales_at(d) + krow * (d / 16) + (is_k ? 0 : d / 32) + 2 * (ch >> 3)) = sh;
    }
}

// The inverse: what the cache holds for (sequence, position) rows, in fp32.
// Rows with a negative position, or one outside the cache, give zeros.
template <class Index>
__global__ void __launch_bounds__(KA_THREADS) kv_read_kernel(KvView c, const int32_t* pos, int batch, int rows,
                                                             float* k_out, float* v_out) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int d = c.head_dim, shift = __ffs(d) - 4, chunks = 1 << shift;
    const int per_row = 2 * c.kv_heads * chunks;
    const Index total = (Index)((int64_t)batch * rows * per_row), step = (Index)gridDim.x * KA_THREADS;
    for (Index i = (Index)blockIdx.x * KA_THREADS + (Index)threadIdx.x; i < total; i += step) {
        const Index row = i / per_row;
        const int in_row = (int)(i - row * per_row);
        const int vec = in_row >> shift, ch = in_row & (chunks - 1);
        const bool is_k = vec < c.kv_heads;
        const int h = is_k ? vec : vec - c.kv_heads;
        float* out = is_k ? k_out : v_out;
        if (!out) continue;
        const int64_t p = pos[row];
        float s = 0.f;
        uint32_t w = 0;
        if (p >= 0) {
            int64_t page = -1;
            if (p < (int64_t)c.table_pages * KV_PAGE) page = c.table[(int64_t)(row / rows) * c.table_stride + p / KV_PAGE];
            if (page < 0 || page >= c.n_pages) {
                atomicOr(&g_device_status, VBQ_DEVICE_RANGE);
            } else {
                const int slot = (int)(p % KV_PAGE), krow = kv_key_row(slot);
                const uint8_t* blob = c.pages + (page * c.kv_heads + h) * kv_blob_bytes(d);
                w = kv_unturned(*reinterpret_cast<const uint32_t*>(
                    is_k ? blob + krow * (d / 2) + 4 * kv_key_word(ch, d)
                         : blob + kv_values_at(d) + slot * (d / 2) + 4 * kv_value_word(ch, slot, d)));
                s = __half2float(*reinterpret_cast<const __half*>(blob + kv_scales_at(d) + krow * (d / 16) +
                                                                  (is_k ? 0 : d / 32) + 2 * (ch >> 3)));
            }
        }
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __fmul_rn(s, (float)((int)((w >> (4 * e)) & 15u) - 8));
        if (s == 0.f)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.f;                        // no -0
        float4* o = reinterpret_cast<float4*>(out + ((int64_t)row * c.kv_heads + h) * d + ch * 8);
        o[0] = make_float4(x[0], x[1], x[2], x[3]);
        o[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
}

constexpr int64_t SHORT = 1 << 30;           // below it an int holds a call's words and a step past them

int grid_for(int64_t threads, int sms) {
    const int64_t want = (threads + KA_THREADS - 1) / KA_THREADS, cap = (int64_t)sms * 16;
    return (int)(want < cap ? want : cap);
}

}  // namespace

cudaError_t launch_kv_append(const KvView& c, const KvAppend& a, cudaStream_t s) {
    int sms = 0;
    const int e = device_sms(&sms);
    if (e != 0) return (cudaError_t)e;
    const int64_t total = (int64_t)a.batch * a.rows * ((a.q ? a.heads : 0) + 2 * c.kv_heads) * (c.head_dim / 8);
    const dim3 grid(grid_for(total, sms));
    const auto go = [&](auto kernel) { return launch_dependent(kernel, grid, KA_THREADS, 0, s, c, a); };
    if (total < SHORT) return a.f32 ? go(kv_append_kernel<true, int>) : go(kv_append_kernel<false, int>);
    return a.f32 ? go(kv_append_kernel<true, int64_t>) : go(kv_append_kernel<false, int64_t>);
}

cudaError_t launch_kv_read(const KvView& c, const int32_t* pos, int batch, int rows, float* k_out, float* v_out,
                           cudaStream_t s) {
    int sms = 0;
    const int e = device_sms(&sms);
    if (e != 0) return (cudaError_t)e;
    const int64_t total = (int64_t)batch * rows * 2 * c.kv_heads * (c.head_dim / 8);
    const dim3 grid(grid_for(total, sms));
    const auto go = [&](auto kernel) { return launch_dependent(kernel, grid, KA_THREADS, 0, s, c, pos, batch, rows, k_out, v_out); };
    return total < SHORT ? go(kv_read_kernel<int>) : go(kv_read_kernel<int64_t>);
}

cudaError_t read_device_status_kv(uint32_t* status) {
    cudaError_t e = cudaMemcpyFromSymbol(status, g_device_status, sizeof(uint32_t));
    if (e != cudaSuccess || *status == 0) return e;
    const uint32_t zero = 0;
    return cudaMemcpyToSymbol(g_device_status, &zero, sizeof(uint32_t));
}

}  // namespace vbq
