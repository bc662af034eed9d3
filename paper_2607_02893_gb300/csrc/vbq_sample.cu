// vbq_sample.cu — a token drawn from a row of logits under temperature, top-k,
// top-p and min-p, from a given random number.
//
// e_i = exp((l_i - max) / T) and w_i = e_i rounded to whole multiples of 2^-32:
// sums of whole numbers do not depend on their order, so neither the cuts nor
// the draw do. One block per row. The top-k and top-p cuts are found by radix
// selection on the logits' order-preserving 32-bit keys, 8 bits a pass, with a
// histogram of counts (top-k) or of weights (top-p); a cut that falls among
// equal logits keeps the lowest indices.
#include "vbq_decode.h"
#include "vbq_device.cuh"

namespace vbq {
namespace {

constexpr int SA_THREADS = 1024;
constexpr int SA_WARPS = SA_THREADS / 32;
typedef unsigned long long u64;

__device__ __forceinline__ float logit_at(const Sample& p, int64_t row, int i) {
    const int64_t at = row * p.stride + i;
    const float v = p.f32 ? static_cast<const float*>(p.logits)[at]
                          : __uint_as_float((uint32_t)static_cast<const uint16_t*>(p.logits)[at] << 16);
    return v == v ? v + 0.f : -INFINITY;                  // NaN is never drawn; -0 ties with 0
}
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t u = __float_as_uint(v);
    return u ^ ((int32_t)u < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float chance(float v, float top, float t) {
    return v == top ? 1.f : v == -INFINITY ? 0.f : expf(__fdiv_rn(__fsub_rn(v, top), t));
}
__device__ __forceinline__ u64 weight(float e) { return (u64)rintf(__fmul_rn(e, 0x1p32f)); }

// Sum over the block of each thread's v, and the sum over the threads before.
__device__ u64 block_scan(u64 v, u64* before, u64* part) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    u64 x = v;
    for (int o = 1; o < 32; o <<= 1) {
        const u64 y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) part[warp] = x;
    __syncthreads();
    u64 base = 0, all = 0;
    for (int w = 0; w < SA_WARPS; ++w) {
        if (w < warp) base += part[w];
        all += part[w];
    }
    *before = base + x - v;
    return all;
}

struct Cut { uint32_t key; u64 ties; };                   // keep keys above, and the first `ties` equal ones

__global__ void __launch_bounds__(SA_THREADS) sample_kernel(Sample p) {
    __shared__ u64 hist[256];
    __shared__ u64 part[SA_WARPS];
    __shared__ u64 s_pick[4];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t row = blockIdx.x;
    const int V = p.vocab;
    const float T = p.temperature[row];
    // the maximum and its first index: keys packed above the complement of the index
    u64 best = 0;
    for (int i = threadIdx.x; i < V; i += SA_THREADS) {
        const u64 x = (u64)key_of(logit_at(p, row, i)) << 32 | (uint32_t)~i;
        best = x > best ? x : best;
    }
    for (int o = 16; o; o >>= 1) {
        const u64 y = __shfl_xor_sync(0xffffffffu, best, o);
        best = y > best ? y : best;
    }
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = best;
    __syncthreads();
    for (int w = 0; w < SA_WARPS; ++w) best = part[w] > best ? part[w] : best;
    __syncthreads();
    const int top_i = (int)~(uint32_t)best;
    const float top = logit_at(p, row, top_i);
    if (top == -INFINITY || !(T > 0.f)) {
        if (threadIdx.x == 0) {
            p.tokens[row] = top == -INFINITY ? -1 : top_i;
            if (p.probs) p.probs[row] = top == -INFINITY ? 0.f : 1.f;
            if (p.kept) p.kept[row] = top == -INFINITY ? 0 : 1;
        }
        return;
    }
    Cut cut = {key_of(-INFINITY), 0};                     // every finite logit
    const int k = p.top_k[row];
    const float tp = p.top_p[row];
    for (int which = 0; which < 2; ++which) {             // top-k, then top-p of what it left
        if (which == 0 ? k <= 0 || k >= V : tp >= 1.f) continue;
        u64 mass = 0;                                     // of the kept set (top-p)
        const Cut prev = cut;
        if (which == 1) {
            u64 before, m = 0;
            for (int i = threadIdx.x; i < V; i += SA_THREADS) {
                const float v = logit_at(p, row, i);
                if (key_of(v) > prev.key) m += weight(chance(v, top, T));
            }
            mass = block_scan(m, &before, part);
            const uint32_t u = prev.key;                  // the tied level
            const float tv = __uint_as_float(u ^ ((int32_t)u < 0 ? 0x80000000u : 0xffffffffu));
            if (prev.ties) mass += prev.ties * weight(chance(tv, top, T));
        }
        const double enough = which == 0 ? (double)k : tp > 0.f ? (double)tp * (double)mass : 0.;
        uint32_t prefix = 0, mask = 0;
        u64 above = 0;                                    // count or weight of the keys above the prefix's range
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            if (threadIdx.x < 256) hist[threadIdx.x] = 0;
            __syncthreads();
            for (int i = threadIdx.x; i < V; i += SA_THREADS) {
                const float v = logit_at(p, row, i);
                const uint32_t key = key_of(v);
                if ((key & mask) != prefix) continue;
                if (which == 0) {
                    atomicAdd(&hist[key >> shift & 255u], 1ull);
                } else if (key > prev.key) {
                    atomicAdd(&hist[key >> shift & 255u], weight(chance(v, top, T)));
                }
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                if (which == 1 && prev.ties && (prev.key & mask) == prefix) {
                    const uint32_t u = prev.key;
                    const float tv = __uint_as_float(u ^ ((int32_t)u < 0 ? 0x80000000u : 0xffffffffu));
                    hist[u >> shift & 255u] += prev.ties * weight(chance(tv, top, T));
                }
                u64 a = above;
                int bin = 255;
                for (; bin > 0; --bin) {
                    if ((double)(a + hist[bin]) >= enough && hist[bin]) break;
                    a += hist[bin];
                }
                s_pick[0] = (u64)bin;
                s_pick[1] = a;
                s_pick[2] = hist[bin];
            }
            __syncthreads();
            above = s_pick[1];
            prefix |= (uint32_t)s_pick[0] << shift;
            mask |= 255u << shift;
        }
        const u64 level = s_pick[2];
        __syncthreads();
        const float tv = __uint_as_float(prefix ^ ((int32_t)prefix < 0 ? 0x80000000u : 0xffffffffu));
        const u64 each = which == 0 ? 1 : weight(chance(tv, top, T));
        u64 n = 1;                                        // ties needed
        const u64 most = each ? level / each : 1;
        if (which == 0) {
            n = (u64)k - above;
        } else {
            u64 lo = 1, hi = most > 1 ? most : 1;
            while (lo < hi) {
                const u64 mid = (lo + hi) / 2;
                if ((double)(above + mid * each) >= enough) hi = mid; else lo = mid + 1;
            }
            n = lo;
        }
        cut.key = prefix;
        cut.ties = n;
    }
    const float mp = fminf(p.min_p[row], 1.f);
    // index order: each thread a run of neighbours
    const int run = (V + SA_THREADS - 1) / SA_THREADS, i0 = min(V, (int)threadIdx.x * run), i1 = min(V, i0 + run);
    u64 ties = 0, ties_before;
    for (int i = i0; i < i1; ++i) ties += key_of(logit_at(p, row, i)) == cut.key;
    block_scan(ties, &ties_before, part);
    u64 sum = 0, kept = 0, last = 0;
    for (int pass = 0; pass < 2; ++pass) {
        u64 before = 0, total = 0;
        double target = 0.;
        if (pass == 1) {
            total = block_scan(sum, &before, part);
            u64 kb;
            const u64 kall = block_scan(kept, &kb, part);
            if (threadIdx.x == 0) {
                if (p.kept) p.kept[row] = (int)kall;
                s_pick[3] = 0;
            }
            __syncthreads();
            float u = p.u[row];
            if (!(u > 0.f)) u = 0.f;
            target = (double)u * (double)total;
            if (sum && u >= 1.f) atomicMax(&s_pick[3], last + 1);
            __syncthreads();
            if (u >= 1.f) {
                if (!(sum && s_pick[3] == last + 1)) return;
                target = (double)total;
            } else if (!((double)before <= target && (double)(before + sum) > target)) {
                return;
            }
        }
        u64 t = ties_before, cum = before;
        for (int i = i0; i < i1; ++i) {
            const float v = logit_at(p, row, i);
            const uint32_t key = key_of(v);
            bool in = key > cut.key;
            if (key == cut.key) in = t++ < cut.ties;
            if (!in || v == -INFINITY) continue;
            const float e = chance(v, top, T);
            if (e < mp) continue;
            const u64 w = weight(e);
            if (pass == 0) {
                sum += w;
                ++kept;
                if (w) last = (u64)i;
            } else {
                cum += w;
                if ((double)cum > target || (target == (double)total && (u64)i == last)) {
                    p.tokens[row] = i;
                    if (p.probs) p.probs[row] = __fdiv_rn(e, (float)((double)total * 0x1p-32));
                    return;
                }
            }
        }
    }
}

}  // namespace

cudaError_t launch_sample(const Sample& p, cudaStream_t s) {
    return launch_dependent(sample_kernel, dim3((unsigned)p.batch), SA_THREADS, 0, s, p);
}

}  // namespace vbq
