// vbq_sample.cu — a token drawn from a row of logits under temperature, top-k,
// top-p and min-p, from a given random number.
//
// e_i = exp((l_i - max) / T) and w_i = e_i rounded to whole multiples of 2^-32:
// sums of whole numbers do not depend on their order, so neither the cuts nor
// the draw depend on how the row is split or when an addition arrives.
//
// A cluster of up to 8 blocks holds a row's e in registers (16 or 32 per
// thread), so the logits are read once; everything after that is a few rounds
// of "add up locally, exchange through distributed shared memory, decide", and
// the number of rounds is what bounds it (a row of 128256 is 0.5 MB: 0.08 us of
// HBM bandwidth). A cut (top-k by count, top-p by weight) is found in two rounds
// from one histogram over 2048 bins of e, 64 to an octave: 32 octave sums, then
// the 64 bins of the octave that holds the cut. If no more than LIST tokens lie
// in or above the cut's bin, one block gathers them in index order, sorts them
// by (logit, lowest index first) and finishes alone. Otherwise only the bin's own
// tokens are gathered and sorted, by every block, for the exact cut; a bin that
// holds more (equal logits by the thousand) is narrowed 5 bits of (logit,
// index) a round first. The draw then adds up in index order.
#include <cooperative_groups.h>

#include "vbq_decode.h"
#include "vbq_device.cuh"

namespace vbq {
namespace {

namespace cg = cooperative_groups;
typedef unsigned long long u64;

constexpr uint32_t ALL = 0xffffffffu;
constexpr int SA_THREADS = 1024;
constexpr int SA_WARPS = SA_THREADS / 32;
constexpr int SA_BLOCKS = 8;              // most blocks of a cluster
constexpr int BINS = 2048;
constexpr int LIST = 1024;                // tokens a block sorts, one per thread

struct Sum { u64 w; uint32_t n, pad; };   // weight and count

struct Shared {
    union {
        struct { uint32_t n[BINS], lo[BINS], hi[BINS]; } hist;   // counts; weights' low 16 and high bits
        u64 sorted[LIST];
    };
    u64 list[LIST];                       // gathered tokens, in index order
    Sum coarse[SA_BLOCKS][32];            // written by the blocks of the cluster; the rounds that narrow a
    Sum fine[SA_BLOCKS][64];              // bin take the two in turn, each free since the exchange before
    u64 table[8][SA_WARPS];               // per (quad, warp) sums in index order
    u64 top[SA_BLOCKS];
    Sum total[SA_BLOCKS];
    u64 part[SA_WARPS];
    u64 pick[4];
    int done;
};

__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t u = __float_as_uint(v);
    return u ^ ((int32_t)u < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key ^ ((int32_t)key < 0 ? 0x80000000u : 0xffffffffu));
}
// Order of tokens: the larger logit first, then the lower index.
__device__ __forceinline__ u64 order_of(float v, int i) { return (u64)key_of(v) << 32 | (uint32_t)~i; }
__device__ __forceinline__ float usable(float v) { return v == v ? v + 0.f : -INFINITY; }   // NaN is never drawn; -0 ties with 0

__device__ __forceinline__ float chance(float v, float top, float t) {
    return v == top ? 1.f : v == -INFINITY ? 0.f : expf(__fdiv_rn(__fsub_rn(v, top), t));
}
__device__ __forceinline__ u64 weight(float e) { return (u64)rintf(__fmul_rn(e, 0x1p32f)); }
// Bin of a token: its weight's octave (2^-32 and below: 0) and 6 bits; tokens without weight are bin 0.
__device__ __forceinline__ int bin_of(float e) {
    const int b = (int)(__float_as_uint(e) >> 17) - 95 * 64;
    return e <= 0x1p-33f ? 0 : min(max(b, 1), BINS - 1);
}

__device__ __forceinline__ float logit_at(const Sample& p, const void* row, int i) {
    return usable(p.f32 ? static_cast<const float*>(row)[i]
                        : __uint_as_float((uint32_t)static_cast<const uint16_t*>(row)[i] << 16));
}

__device__ __forceinline__ u64 warp_sum(u64 v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(ALL, v, o);
    return v;
}
__device__ __forceinline__ u64 warp_scan(u64 v) {          // inclusive
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 y = __shfl_up_sync(ALL, v, o);
        if (lane >= o) v += y;
    }
    return v;
}
// Inclusive scan over the block; the block's sum in all.
__device__ __forceinline__ u64 block_scan(u64 v, u64* part, u64* all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const u64 x = warp_scan(v);
    __syncthreads();
    if (lane == 31) part[warp] = x;
    __syncthreads();
    const u64 y = warp_scan(part[lane]);
    *all = __shfl_sync(ALL, y, 31);
    const u64 before = __shfl_sync(ALL, y, max(warp, 1) - 1);
    return x + (warp ? before : 0);
}

template <int C>
__device__ __forceinline__ void cluster_sync() {
    if constexpr (C == 1) {
        __syncthreads();
    } else {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}
// The same shared-memory object in another block of the cluster.
template <int C, class T>
__device__ __forceinline__ T* in_block(T* p, int rank) {
    if constexpr (C == 1) return p;
    return cg::this_cluster().map_shared_rank(p, rank);
}

// The kept set so far: tokens at or above `order` in (logit, index) order; a token's
// bin decides unless it is the cut's own bin.
struct Cut {
    int bin;                              // -1: every token
    u64 order;
};

// Descending bitonic sort of LIST or fewer values, one per thread below size (a
// power of two of at least 32); the others pass through.
__device__ u64 sort_down(u64 v, int size, u64* buf) {
    const int t = threadIdx.x;
    for (int k = 2; k <= size; k <<= 1) {
        for (int j = k >> 1; j; j >>= 1) {
            u64 y;
            if (j >= 32) {
                __syncthreads();
                buf[t] = v;
                __syncthreads();
                y = buf[t ^ j];
            } else {
                y = __shfl_xor_sync(ALL, v, j);
            }
            const bool larger = ((t & j) == 0) == ((t & k) == 0);      // this side keeps the larger
            if (t < size) v = larger ? max(v, y) : min(v, y);
        }
    }
    return v;
}

// C blocks per row, QUADS x 4 tokens per thread: thread t of block r holds tokens
// (r * QUADS + j) * 4096 + 4 t + 0..3.
template <int C, int QUADS>
__global__ void __launch_bounds__(SA_THREADS, 1) sample_kernel(Sample p) {
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = C == 1 ? 0 : (int)(blockIdx.x % C);
    const int64_t row = blockIdx.x / C;
    if constexpr (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // this block has started
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int V = p.vocab;
    const void* logits = static_cast<const uint8_t*>(p.logits) + row * p.stride * (p.f32 ? 4 : 2);
    const int first = rank * QUADS * 4096 + 4 * tid;
    const float T = p.temperature[row];
    const int top_k = p.top_k[row];
    const float top_p = p.top_p[row], mp = p.min_p[row], min_p = mp > 0.f ? fminf(mp, 1.f) : 0.f, u = p.u[row];

    // The logits, and the largest with its first index.
    float e[QUADS * 4];
    const bool vec = (reinterpret_cast<uintptr_t>(logits) & (p.f32 ? 15 : 7)) == 0;
#pragma unroll
    for (int j = 0; j < QUADS; ++j) {
        const int i = first + j * 4096;
        if (vec && i + 3 < V) {
            if (p.f32) {
                const float4 x = *reinterpret_cast<const float4*>(static_cast<const float*>(logits) + i);
                e[4 * j] = x.x; e[4 * j + 1] = x.y; e[4 * j + 2] = x.z; e[4 * j + 3] = x.w;
            } else {
                const uint2 x = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(logits) + i);
                e[4 * j] = __uint_as_float(x.x << 16); e[4 * j + 1] = __uint_as_float(x.x & 0xffff0000u);
                e[4 * j + 2] = __uint_as_float(x.y << 16); e[4 * j + 3] = __uint_as_float(x.y & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                e[4 * j + q] = i + q >= V ? -INFINITY
                               : p.f32   ? static_cast<const float*>(logits)[i + q]
                                         : __uint_as_float((uint32_t)static_cast<const uint16_t*>(logits)[i + q] << 16);
        }
    }
    float mx = -INFINITY;
    int mi = 0;
#pragma unroll
    for (int j = 0; j < QUADS * 4; ++j) {
        e[j] = usable(e[j]);
        if (e[j] > mx) {
            mx = e[j];
            mi = first + (j / 4) * 4096 + j % 4;
        }
    }
    u64 best = mx > -INFINITY ? order_of(mx, mi) : 0;
#pragma unroll
    for (int o = 16; o; o >>= 1) best = max(best, __shfl_xor_sync(ALL, best, o));
    if (lane == 0) sh.part[warp] = best;
    __syncthreads();
    if constexpr (C > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");   // all have: their memory may be written
    if (warp == 0) {
        best = sh.part[lane];
#pragma unroll
        for (int o = 16; o; o >>= 1) best = max(best, __shfl_xor_sync(ALL, best, o));
        if (lane < C) *in_block<C>(&sh.top[rank], lane) = best;
    }
    cluster_sync<C>();
    best = sh.top[0];
#pragma unroll
    for (int r = 1; r < C; ++r) best = max(best, sh.top[r]);
    if (best == 0 || !(T > 0.f)) {                         // nothing to draw from, or greedy
        if (rank == 0 && tid == 0) {
            p.tokens[row] = best == 0 ? -1 : (int)~(uint32_t)best;
            if (p.probs) p.probs[row] = best == 0 ? 0.f : 1.f;
            if (p.kept) p.kept[row] = best == 0 ? 0 : 1;
        }
        return;
    }
    const float top = value_of((uint32_t)(best >> 32));
#pragma unroll
    for (int j = 0; j < QUADS * 4; ++j) e[j] = e[j] == -INFINITY ? -1.f : chance(e[j], top, T);   // -1: not a token

    const auto index_of = [&](int j) { return first + (j / 4) * 4096 + j % 4; };
    Cut cut = {-1, 0};
    const auto is_in = [&](int j) {                        // of the kept set
        if (e[j] < 0.f) return false;
        if (cut.bin < 0) return true;
        const int b = bin_of(e[j]);
        if (b != cut.bin) return b > cut.bin;
        return order_of(logit_at(p, logits, index_of(j)), index_of(j)) >= cut.order;
    };

    for (int which = 0; which < 2; ++which) {              // 0: top-k by count, 1: top-p by weight
        if (which == 0 ? top_k <= 0 || top_k >= V : top_p >= 1.f) continue;
        __syncthreads();
        for (int i = tid; i < BINS; i += SA_THREADS) sh.hist.n[i] = sh.hist.lo[i] = sh.hist.hi[i] = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < QUADS * 4; ++j) {
            if (!is_in(j)) continue;
            const int b = bin_of(e[j]);
            atomicAdd(&sh.hist.n[b], 1u);
            if (which == 1 && b > 0) {
                const u64 w = weight(e[j]);
                atomicAdd(&sh.hist.lo[b], (uint32_t)w & 0xffffu);
                atomicAdd(&sh.hist.hi[b], (uint32_t)(w >> 16));
            }
        }
        __syncthreads();
        {                                                  // octave sums, to every block
            Sum s;
            const int b = 64 * warp + lane;
            s.n = __reduce_add_sync(ALL, sh.hist.n[b] + sh.hist.n[b + 32]);
            s.w = which == 0 ? 0
                             : warp_sum((u64)sh.hist.lo[b] + sh.hist.lo[b + 32] + ((u64)sh.hist.hi[b] + sh.hist.hi[b + 32] << 16));
            s.pad = 0;
            if (lane < C) *in_block<C>(&sh.coarse[rank][warp], lane) = s;
        }
        cluster_sync<C>();
        // The octave that holds the cut (every warp finds it by itself), from the top down: lane i is octave 31 - i.
        Sum s = {0, 0, 0};
#pragma unroll
        for (int r = 0; r < C; ++r) {
            const Sum x = sh.coarse[r][31 - lane];
            s.n += x.n;
            s.w += x.w;
        }
        const u64 mass = which == 0 ? 0 : warp_sum(s.w);
        const double enough = which == 0 ? (double)top_k : top_p > 0.f ? (double)top_p * (double)mass : 0.;
        u64 own = which == 0 ? s.n : s.w, upto = warp_scan(own);
        uint32_t above_n;
        u64 above;
        const uint32_t found = __ballot_sync(ALL, (double)upto >= enough && s.n > 0);
        if (found == 0) continue;                          // fewer tokens than top_k: all are kept
        const int at = __ffs(found) - 1, oct = 31 - at;
        above = __shfl_sync(ALL, upto - own, at);
        {
            const u64 n = warp_scan((u64)s.n);
            above_n = (uint32_t)__shfl_sync(ALL, n - s.n, at);
        }
        if (tid < 64 * C) {                                // the octave's bins, to every block
            const int b = 64 * oct + (tid & 63);
            *in_block<C>(&sh.fine[rank][tid & 63], tid >> 6) =
                Sum{(u64)sh.hist.lo[b] + ((u64)sh.hist.hi[b] << 16), sh.hist.n[b], 0};
        }
        cluster_sync<C>();
        // The bin: lane i holds bins 63 - 2 i and 62 - 2 i.
        Sum a = {0, 0, 0}, z = {0, 0, 0};
#pragma unroll
        for (int r = 0; r < C; ++r) {
            const Sum x = sh.fine[r][63 - 2 * lane], y = sh.fine[r][62 - 2 * lane];
            a.n += x.n; a.w += x.w;
            z.n += y.n; z.w += y.w;
        }
        const u64 ownA = which == 0 ? a.n : a.w, ownZ = which == 0 ? z.n : z.w;
        upto = above + warp_scan(ownA + ownZ);
        const bool hitA = (double)(upto - ownZ) >= enough && a.n > 0, hitZ = (double)upto >= enough && z.n > 0;
        const uint32_t hits = __ballot_sync(ALL, hitA || hitZ);
        const int hl = __ffs(hits) - 1;                    // there is one: the octave holds the cut
        const bool second = !__shfl_sync(ALL, (int)hitA, hl);
        const int bin = 64 * oct + 63 - 2 * hl - second;
        above = __shfl_sync(ALL, second ? upto - ownZ : upto - ownZ - ownA, hl);
        {
            const u64 n = warp_scan((u64)(a.n + z.n));
            above_n += (uint32_t)__shfl_sync(ALL, n - z.n - (second ? 0 : a.n), hl);
        }
        uint32_t in_bin = __shfl_sync(ALL, second ? z.n : a.n, hl);
        const bool finish = above_n + in_bin <= LIST;      // one block takes it from here

        // Narrow a bin that holds too many: digits of (logit, index), 5 bits a round.
        u64 prefix = 0;
        int known = 0;                                     // leading bits of the order that are fixed
        const auto in_range = [&](int j, u64* o) {         // a token of the bin whose order has the prefix
            if (e[j] < 0.f || bin_of(e[j]) != bin || !is_in(j)) return false;
            *o = order_of(logit_at(p, logits, index_of(j)), index_of(j));
            return known == 0 || *o >> (64 - known) == prefix;
        };
        if (!finish) {
            for (int round = 0; in_bin > LIST; ++round) {
                const int bits = min(5, 64 - known);
                __syncthreads();
                if (tid < 32) sh.hist.n[tid] = sh.hist.lo[tid] = sh.hist.hi[tid] = 0;
                __syncthreads();
#pragma unroll
                for (int j = 0; j < QUADS * 4; ++j) {
                    u64 o;
                    if (!in_range(j, &o)) continue;
                    const int d = (int)(o >> (64 - known - bits)) & ((1 << bits) - 1);
                    atomicAdd(&sh.hist.n[d], 1u);
                    const u64 w = weight(e[j]);
                    atomicAdd(&sh.hist.lo[d], (uint32_t)w & 0xffffu);
                    atomicAdd(&sh.hist.hi[d], (uint32_t)(w >> 16));
                }
                __syncthreads();
                Sum* mine = round & 1 ? sh.fine[rank] : sh.coarse[rank];
                if (tid < 32 * C)
                    *in_block<C>(mine + lane, warp) = Sum{(u64)sh.hist.lo[lane] + ((u64)sh.hist.hi[lane] << 16), sh.hist.n[lane], 0};
                cluster_sync<C>();
                Sum x = {0, 0, 0};
#pragma unroll
                for (int r = 0; r < C; ++r) {
                    const Sum y = (round & 1 ? sh.fine[r] : sh.coarse[r])[31 - lane];
                    x.n += y.n; x.w += y.w;
                }
                const u64 o = which == 0 ? x.n : x.w, to = above + warp_scan(o);
                const uint32_t hit = __ballot_sync(ALL, (double)to >= enough && x.n > 0);
                const int l = __ffs(hit) - 1;              // there is one: the bin holds the cut
                above = __shfl_sync(ALL, to - o, l);
                {
                    const u64 n = warp_scan((u64)x.n);
                    above_n += (uint32_t)__shfl_sync(ALL, n - x.n, l);
                }
                in_bin = __shfl_sync(ALL, x.n, l);
                prefix = prefix << bits | (u64)(31 - l);
                known += bits;
            }
        }

        // Gather, in index order: all of the kept set from the bin up (to block 0), or the narrowed bin (to all).
        const auto taken = [&](int j, u64* o) {
            if (!finish) return in_range(j, o);
            if (e[j] < 0.f || bin_of(e[j]) < bin || !is_in(j)) return false;
            *o = order_of(logit_at(p, logits, index_of(j)), index_of(j));
            return true;
        };
        uint32_t flags = 0;
        u64 order[1];
#pragma unroll
        for (int j = 0; j < QUADS * 4; ++j) flags |= (uint32_t)taken(j, order) << j;
#pragma unroll
        for (int j = 0; j < QUADS; ++j) {
            const uint32_t n = __reduce_add_sync(ALL, (uint32_t)__popc(flags >> 4 * j & 15u));
            if (lane == 0) sh.table[j][warp] = n;
        }
        u64 local;
        __syncthreads();
        {
            const u64 n = tid < QUADS * SA_WARPS ? sh.table[tid >> 5][lane] : 0;
            const u64 x = block_scan(n, sh.part, &local);
            if (tid < QUADS * SA_WARPS) sh.table[tid >> 5][lane] = x - n;
        }
        if (tid < C) *in_block<C>(&sh.total[rank], tid) = Sum{0, (uint32_t)local, 0};
        cluster_sync<C>();
        uint32_t base = 0, n_list = 0;
#pragma unroll
        for (int r = 0; r < C; ++r) {
            if (r < rank) base += sh.total[r].n;
            n_list += sh.total[r].n;
        }
#pragma unroll
        for (int j = 0; j < QUADS; ++j) {
            const uint32_t mine = flags >> 4 * j & 15u, c = __popc(mine);
            if (__any_sync(ALL, c != 0)) {
                uint32_t x = c;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const uint32_t y = __shfl_up_sync(ALL, x, o);
                    if (lane >= o) x += y;
                }
                uint32_t to = base + (uint32_t)sh.table[j][warp] + x - c;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (!(mine >> q & 1u)) continue;
                    const int i = first + j * 4096 + q;
                    const u64 o = order_of(logit_at(p, logits, i), i);
                    if (to < LIST) {
                        if (finish) {
                            *in_block<C>(&sh.list[to], 0) = o;
                        } else {
                            for (int r = 0; r < C; ++r) *in_block<C>(&sh.list[to], r) = o;
                        }
                    }
                    ++to;
                }
            }
        }
        cluster_sync<C>();
        if (finish && rank != 0) return;                   // block 0 has all it needs

        // Sorted, a thread's token is the tid-th: the filters are conditions on a prefix.
        int size = 32;
        while (size < (int)n_list) size <<= 1;
        const u64 o = sort_down(tid < (int)n_list ? sh.list[tid] : 0, size, sh.sorted);
        const bool real = tid < (int)n_list;
        const float ce = real ? chance(value_of((uint32_t)(o >> 32)), top, T) : 0.f;
        const u64 cw = real ? weight(ce) : 0;
        u64 all;
        const u64 cum = block_scan(cw, sh.part, &all);
        bool keep;
        if (which == 0) {
            const bool counted = real && (u64)tid < (u64)top_k - (finish ? 0 : above);
            keep = counted;
            if (finish) {
                if (tid == min(top_k, (int)n_list) - 1) sh.pick[0] = cum;
                __syncthreads();
                const double want = top_p > 0.f ? (double)top_p * (double)sh.pick[0] : 0.;
                keep = counted && (top_p >= 1.f || tid == 0 || (double)(cum - cw) < want);
            }
        } else {
            // in the list from the bin up, the weights before a token are all listed
            const u64 before = (finish ? 0 : above) + cum - cw;
            keep = real && ((double)before < enough || (tid == 0 && (finish ? true : above_n == 0)));
        }
        if (finish) keep = keep && !(ce < min_p);
        const int n_keep = __syncthreads_count(keep);      // at least one
        if (tid == n_keep - 1) sh.pick[1] = o;
        __syncthreads();
        const u64 last = sh.pick[1];
        if (!finish) {
            cut.bin = bin;
            cut.order = last;
            continue;
        }
        // The draw, in index order.
        const u64 lo = real ? sh.list[tid] : 0;
        const bool in = real && lo >= last;
        const float le = in ? chance(value_of((uint32_t)(lo >> 32)), top, T) : 0.f;
        const u64 lw = in ? weight(le) : 0;
        const u64 to = block_scan(lw, sh.part, &all);
        const double target = u > 0.f ? (double)u * (double)all : 0.;
        const auto past = [&](u64 x) { return u >= 1.f ? x >= all : (double)x > target; };
        if (lw && past(to) && !past(to - lw)) {
            p.tokens[row] = (int)~(uint32_t)lo;
            if (p.probs) p.probs[row] = __fdiv_rn(le, (float)((double)all * 0x1p-32));
            if (p.kept) p.kept[row] = n_keep;
        }
        return;
    }

    // The draw over the whole row, in index order.
    u64 sum = 0, kept = 0;
    uint32_t flags = 0;
    u64 quad[QUADS];
#pragma unroll
    for (int j = 0; j < QUADS; ++j) {
        quad[j] = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (!is_in(4 * j + q) || e[4 * j + q] < min_p) continue;
            flags |= 1u << (4 * j + q);
            quad[j] += weight(e[4 * j + q]);
        }
        const u64 x = warp_sum(quad[j]);
        if (lane == 0) sh.table[j][warp] = x;
    }
    kept = __popc(flags);
    u64 nk;
    __syncthreads();
    block_scan(kept, sh.part, &nk);
    const u64 mine = tid < QUADS * SA_WARPS ? sh.table[tid >> 5][lane] : 0;
    const u64 upto = block_scan(mine, sh.part, &sum);
    if (tid < QUADS * SA_WARPS) sh.table[tid >> 5][lane] = upto - mine;
    if (tid < C) *in_block<C>(&sh.total[rank], tid) = Sum{sum, (uint32_t)nk, 0};
    cluster_sync<C>();
    u64 before = 0, all = 0;
    uint32_t n_all = 0;
#pragma unroll
    for (int r = 0; r < C; ++r) {
        if (r < rank) before += sh.total[r].w;
        all += sh.total[r].w;
        n_all += sh.total[r].n;
    }
    if (rank == 0 && tid == 0 && p.kept) p.kept[row] = (int)n_all;
    const double target = u > 0.f ? (double)u * (double)all : 0.;
    const auto past = [&](u64 x) { return u >= 1.f ? x >= all : (double)x > target; };
    if (past(before) || !past(before + sum)) return;       // another block's
#pragma unroll
    for (int j = 0; j < QUADS; ++j) {
        const u64 start = before + sh.table[j][warp], x = warp_scan(quad[j]);
        u64 to = start + x - quad[j];
        if (quad[j] == 0 || past(to) || !past(to + quad[j])) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (!(flags >> (4 * j + q) & 1u)) continue;
            const u64 w = weight(e[4 * j + q]);
            if (!past(to) && past(to + w)) {
                p.tokens[row] = first + j * 4096 + q;
                if (p.probs) p.probs[row] = __fdiv_rn(e[4 * j + q], (float)((double)all * 0x1p-32));
            }
            to += w;
        }
    }
}

template <int C, int QUADS>
cudaError_t launch(const Sample& p, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.batch * C);
    cfg.blockDim = dim3(SA_THREADS);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {C, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = C > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, sample_kernel<C, QUADS>, p);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

// As many blocks as 16 tokens a thread need, up to a portable cluster.
cudaError_t launch_sample(const Sample& p, cudaStream_t s) {
    if (p.vocab <= 4096) return launch<1, 1>(p, s);
    if (p.vocab <= 16384) return launch<1, 4>(p, s);
    if (p.vocab <= 32768) return launch<2, 4>(p, s);
    if (p.vocab <= 65536) return launch<4, 4>(p, s);
    if (p.vocab <= 131072) return launch<8, 4>(p, s);
    return launch<8, 8>(p, s);
}

}  // namespace vbq
