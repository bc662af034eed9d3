// vbq_sample.cu — a token drawn from a row of logits under temperature, top-k,
// top-p and min-p, from a given random number.
//
// e_i = exp((l_i - max) / T) and w_i = e_i rounded to whole multiples of 2^-32:
// sums of whole numbers do not depend on their order, so neither the cuts nor
// the draw depend on how the row is split or when an addition arrives.
//
// A cluster of up to 8 blocks holds a row in shared memory, so the logits are
// read once; everything after that is a few rounds of "add up locally,
// exchange through distributed shared memory, decide", and those rounds are
// what bounds it (a row of 128256 is 0.5 MB: 0.08 us of HBM bandwidth). A cut
// (top-k by count, top-p by weight) is found in two rounds from one histogram
// of 4096 bins, 128 to a factor of 2 in weight: 64 sums of 64 bins, then the 64
// bins that hold the cut. For top-k the bins are of the logits themselves and no
// exponential is taken but of the tokens that remain. If no more than LIST
// tokens lie in or above the cut's bin, one block gathers them, ranks each
// against the others by (logit, lowest index first), applies the filters, and
// adds up what is left in index order. Otherwise only the bin's own tokens are
// gathered and ranked, by every block, for the exact cut; a bin that holds more
// than LIST (equal logits by the thousand) is narrowed 5 bits of (logit, index)
// a round first. The draw then adds up in index order over the whole row.
//
// Measured (one GB300, in a graph): 32000 logits under top-k 50 and top-p 0.95:
// 10.5 us; 16 rows of 128256 under top-p 0.9, some 25000 tokens kept: 25.7 us, of
// which the pass that fills the histogram takes 6 and the one that draws 5, both
// bound by instruction issue, and each exchange about 1.
#include <cooperative_groups.h>

#include <atomic>

#include "vbq_decode.h"
#include "vbq_device.cuh"

namespace vbq {
namespace {

namespace cg = cooperative_groups;
typedef unsigned long long u64;

constexpr uint32_t ALL = 0xffffffffu;
constexpr int SA_THREADS = 512;
constexpr int SA_WARPS = SA_THREADS / 32;
constexpr int SA_BLOCKS = 8;              // most blocks of a cluster
constexpr int BINS = 4096;                // 64 groups of 64
constexpr int PER_OCTAVE = 128;           // bins to a factor of 2 in weight
constexpr int LIST = 256;                 // tokens a block ranks

struct Sum { u64 w; uint32_t n, pad; };   // weight and count

struct Found {                            // where a cut lies
    int at;                               // bin, or -1: nothing reaches it
    uint32_t in, above_n;                 // tokens in the bin, and above it
    u64 above;                            // count or weight above it
};

struct Shared {
    union {
        struct { uint32_t n[BINS], hi[BINS]; int lo[BINS]; } hist;   // counts; weights' parts
        uint32_t found[LIST];             // a block's tokens to gather
        Sum beside[SA_THREADS + 16];       // ranking: what a thread has counted, and the whole weight's parts
    };
    u64 list[LIST];                       // gathered tokens
    ulonglong2 ranked[LIST];              // and their weights beside them
    Sum coarse[SA_BLOCKS][64];            // written by the blocks of the cluster; the rounds that narrow a
    Sum fine[SA_BLOCKS][64];              // bin take the two in turn, each free since the exchange before
    u64 top[SA_BLOCKS];
    Sum total[SA_BLOCKS];
    uint32_t count[SA_BLOCKS];            // tokens each block gathers
    u64 part[SA_WARPS], warp_w[SA_WARPS];
    u64 mass, pick[2];
    Found found_cut;
    uint32_t next;
};
constexpr int SHARED_BYTES = (sizeof(Shared) + 15) / 16 * 16;    // the row's slice follows
constexpr size_t SMEM_MOST = 227 * 1024, SMEM_ALONE = 120 * 1024;        // a block's most; more than half an SM's
constexpr int SLICE_MOST = (SMEM_MOST - SHARED_BYTES) / 4;
static_assert(SLICE_MOST >= SAMPLE_MAX_VOCAB / SA_BLOCKS, "the largest slice fits");

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

// e = 2^t for t = (l - max) log2(e) / T: t = n + f with n whole and |f| <= 1/2, then the hardware's 2^f (2 ulps) and n added
// to the exponent. The reduction is Cody and Waite's with a constant of two floats (Software Manual for the Elementary
// Functions, 1980): log2(e) / T = hi + lo, n = round(x hi), f = (x hi - n) + x lo with fused products, so f is off by two
// roundings of a number below 1 and not by those of t. hi is the quotient rounded; its remainder, log2(e) - hi T (log2(e)
// itself as two floats), over T is lo.
struct Scale {
    float top, hi, lo;                                     // the maximum; log2(e) / T
    __device__ Scale(float top_, float T) : top(top_) {
        hi = fminf(__fdiv_rn(1.44269502f, T), 1e30f);
        lo = __fdiv_rn(__fmaf_rn(-hi, T, 1.44269502f) + 1.92596303e-8f, T);
        if (!(hi < 1e30f) || !(fabsf(lo) < 1e20f)) lo = 0.f;             // T below 1.5e-30 or infinite
    }
    __device__ __forceinline__ float chance(float l) const {
        const float x = __fsub_rn(l, top), t = __fmul_rn(x, hi);
        const float r = __fadd_rn(fmaxf(t, -126.f), 0x1.8p23f), n = __fsub_rn(r, 0x1.8p23f);
        const float f = __fmaf_rn(x, lo, __fmaf_rn(x, hi, -n));
        float y;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(f));
        return t < -126.f ? 0.f : __int_as_float(__float_as_int(y) + (__float_as_int(r) << 23));
    }
    // Bin of a logit, from the largest down; 0: 2^-32 and less. Never above a larger logit's bin.
    __device__ __forceinline__ int bin(float l) const {
        const float t = fmaxf(__fmul_rn(__fsub_rn(l, top), hi), -(BINS - 1) / (float)PER_OCTAVE);
        return (int)(__float_as_uint(__fmaf_rn(t, (float)PER_OCTAVE, 0x1.8p23f)) - 0x4b400000u) + BINS - 1;
    }
};
// w = 65536 hi + lo: e in whole multiples of 2^-32, ties to even, lo within +-2^15. Both parts by adding 1.5 2^23, which
// rounds to a whole number there. (Conversions to 64-bit integers and fp64 comparisons are slow on this GPU.)
struct Parts {
    int hi, lo;
    __device__ explicit Parts(float e) {
        const float a = __fmaf_rn(e, 0x1p16f, 0x1.8p23f), h = __fsub_rn(a, 0x1.8p23f);
        const float b = __fadd_rn(__fmaf_rn(h, -0x1p16f, __fmul_rn(e, 0x1p32f)), 0x1.8p23f);
        hi = (int)(__float_as_uint(a) - 0x4b400000u);
        lo = (int)(__float_as_uint(b) - 0x4b400000u);
    }
};
__device__ __forceinline__ u64 whole(long long hi, long long lo) { return (u64)(hi * 65536 + lo); }
__device__ __forceinline__ u64 weight(float e) {
    const Parts w(e);
    return whole(w.hi, w.lo);
}
// The least whole number that is at least (or, `over`, more than) f * m, for 0 < f < 1 and m below 2^51.
__device__ __forceinline__ u64 at_least(float f, u64 m, bool over) {
    const uint32_t bits = __float_as_uint(f), ex = max(bits >> 23, 1u);
    const u64 man = (bits & 0x7fffffu) | (bits >> 23 ? 0x800000u : 0u);
    const int s = 150 - (int)ex;                           // f = man 2^-s, s of 24..149
    const u64 lo = man * m, hi = __umul64hi(man, m);
    u64 whole, rest;
    if (s < 64) {
        whole = hi << (64 - s) | lo >> s;
        rest = lo << (64 - s);
    } else {
        whole = s < 128 ? hi >> (s - 64) : 0;
        rest = s == 64 ? lo : lo | (s < 128 ? hi << (128 - s) : hi);
    }
    return over ? whole + 1 : whole + (rest != 0);
}
__device__ __forceinline__ float logit_at(const Sample& p, const void* row, int i) {
    return usable(p.f32 ? static_cast<const float*>(row)[i]
                        : __uint_as_float((uint32_t)static_cast<const uint16_t*>(row)[i] << 16));
}

// The warp's index, known to the compiler to be one for the whole warp.
__device__ __forceinline__ int uniform_warp() { return __shfl_sync(ALL, (int)threadIdx.x >> 5, 0); }

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
// The weight that a top-p prefix reaches at least.
__device__ __forceinline__ u64 share_of(float top_p, u64 mass) { return top_p > 0.f ? at_least(top_p, mass, false) : 0; }
// The least running weight that is past the random number's share.
__device__ __forceinline__ u64 drawn_at(float u, u64 mass) { return u >= 1.f ? mass : u > 0.f ? at_least(u, mass, true) : 1; }

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

// One warp: the cut's place among PER * 32 bins, from the highest down, whose
// sums are the C blocks' added up; above counts what lies above all of them.
template <int C, int PER>
__device__ __forceinline__ void find_cut(const Sum* tab, int width, bool by_weight, u64 enough, Found* f) {
    const int lane = threadIdx.x & 31, hi = PER * (32 - lane) - 1;       // this lane's bins: hi, hi - 1
    Sum a = {0, 0, 0}, z = {0, 0, 0};
#pragma unroll
    for (int r = 0; r < C; ++r) {
        const Sum x = tab[r * width + hi];
        a.n += x.n; a.w += x.w;
        if (PER == 2) {
            const Sum y = tab[r * width + hi - 1];
            z.n += y.n; z.w += y.w;
        }
    }
    const u64 own_a = by_weight ? a.w : a.n, own_z = by_weight ? z.w : z.n;
    const u64 upto = f->above + warp_scan(own_a + own_z);
    const uint32_t n = f->above_n + (uint32_t)warp_scan((u64)(a.n + z.n));
    const bool hit_a = upto - own_z >= enough && a.n > 0;
    const bool hit_z = PER == 2 && upto >= enough && z.n > 0;
    const uint32_t hits = __ballot_sync(ALL, hit_a || hit_z);
    __syncwarp();                         // every lane has read *f
    if (hits == 0) {
        if (lane == 0) f->at = -1;
    } else if (lane == __ffs(hits) - 1) {
        f->at = hit_a ? hi : hi - 1;
        f->in = hit_a ? a.n : z.n;
        f->above = hit_a ? upto - own_z - own_a : upto - own_z;
        f->above_n = hit_a ? n - z.n - a.n : n - z.n;
    }
}

// Over the list's tokens j that come before this thread's in `first`'s sense: how many and their weight, with the
// list split over the threads that share a token (size: the list's length rounded up to a power of two, 32..LIST).
// Every thread calls it; threads below count get their token's sums, and the whole weight in all.
template <class Before>
__device__ __forceinline__ Sum rank_in(const Shared& sh, Sum* beside, int count, int size, Before before, u64* all) {
    const int tid = threadIdx.x, c = tid & (size - 1), step = SA_THREADS / size;
    Sum s = {0, 0, 0};
    u64 mine = 0;
    if (c < count) {
        const u64 o = sh.list[c];
#pragma unroll 4
        for (int j = tid / size; j < count; j += step) {   // one j for the whole warp
            const ulonglong2 y = sh.ranked[j];
            const bool first = before(y.x, o);
            s.w += first ? y.y : 0;
            s.n += first;
            mine += y.y;
        }
    }
    // Every token's threads have seen the same list: the first token's weights are the whole.
    __syncthreads();
    beside[tid] = s;
    u64* totals = reinterpret_cast<u64*>(beside + SA_THREADS);
    if (c == 0) totals[tid / size] = mine;
    __syncthreads();
    *all = 0;
    s = Sum{0, 0, 0};
    for (int i = 0; i < step; ++i) {
        const Sum x = beside[i * size + c];
        s.w += x.w;
        s.n += x.n;
        *all += totals[i];
    }
    return s;
}

// C blocks per row, each with `slice` neighbouring tokens (a multiple of 4).
template <int C>
__global__ void __launch_bounds__(SA_THREADS) sample_kernel(Sample p, int slice) {
    extern __shared__ __align__(16) uint8_t smem[];
    Shared& sh = *reinterpret_cast<Shared*>(smem);
    float* x = reinterpret_cast<float*>(smem + SHARED_BYTES);
    const int tid = threadIdx.x, lane = tid & 31, warp = uniform_warp();
    const int rank = C == 1 ? 0 : (int)(blockIdx.x % C);
    const int64_t row = blockIdx.x / C;
    if constexpr (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // this block has started
    const auto clear_hist = [&] {
        uint4* h = reinterpret_cast<uint4*>(&sh.hist);
        for (int i = tid; i < (int)(sizeof(sh.hist) / 16); i += SA_THREADS) h[i] = make_uint4(0, 0, 0, 0);
    };
    clear_hist();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int V = p.vocab, first = rank * slice, n = max(0, min(V - first, slice));
    const void* logits = static_cast<const uint8_t*>(p.logits) + row * p.stride * (p.f32 ? 4 : 2);
    const float T = p.temperature[row];
    const int top_k = p.top_k[row];
    const float top_p = fmaxf(p.top_p[row], 0.f), mp = p.min_p[row], min_p = mp > 0.f ? fminf(mp, 1.f) : 0.f, u = p.u[row];

    // The slice, and the largest logit with its first index.
    float mx = -INFINITY;
    int mi = 0;
    const int quads = (reinterpret_cast<uintptr_t>(logits) & (p.f32 ? 15 : 7)) == 0 ? n / 4 : 0;
#pragma unroll 4
    for (int q = tid; q < quads; q += SA_THREADS) {
        float4 v;
        if (p.f32) {
            v = reinterpret_cast<const float4*>(static_cast<const float*>(logits) + first)[q];
        } else {
            const uint2 b = reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(logits) + first)[q];
            v = make_float4(__uint_as_float(b.x << 16), __uint_as_float(b.x & 0xffff0000u), __uint_as_float(b.y << 16),
                            __uint_as_float(b.y & 0xffff0000u));
        }
        v = make_float4(usable(v.x), usable(v.y), usable(v.z), usable(v.w));
        reinterpret_cast<float4*>(x)[q] = v;
        const float m = fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w));
        if (m > mx) {
            mx = m;
            mi = 4 * q + (v.x == m ? 0 : v.y == m ? 1 : v.z == m ? 2 : 3);
        }
    }
    const int quads4 = (n + 3) / 4;                        // the last is filled up with what no row keeps
    float4* x4 = reinterpret_cast<float4*>(x);
    for (int i = 4 * quads + tid; i < 4 * quads4; i += SA_THREADS) {
        const float v = i < n ? logit_at(p, logits, first + i) : -INFINITY;
        x[i] = v;
        if (v > mx) { mx = v; mi = i; }
    }
    u64 best = mx > -INFINITY ? order_of(mx, first + mi) : 0;
#pragma unroll
    for (int o = 16; o; o >>= 1) best = max(best, __shfl_xor_sync(ALL, best, o));
    if (lane == 0) sh.part[warp] = best;
    __syncthreads();
    if constexpr (C > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");   // all have: their memory may be written
    if (warp == 0) {
        best = sh.part[lane & (SA_WARPS - 1)];
#pragma unroll
        for (int o = SA_WARPS / 2; o; o >>= 1) best = max(best, __shfl_xor_sync(ALL, best, o));
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
    float top = value_of((uint32_t)(best >> 32));
    const bool infinite = top == INFINITY;
    if (infinite) {                                        // infinite logits share the draw; the others weigh nothing, at any T
        __syncthreads();
        for (int i = tid; i < 4 * quads4; i += SA_THREADS) x[i] = x[i] == INFINITY ? 0.f : x[i] == -INFINITY ? x[i] : -3e38f;
        __syncthreads();
        top = 0.f;
    }
    const Scale scale(top, infinite ? 1.f : T);

    // What is kept so far: the logits above cut, and those equal to it up to an index.
    float cut = -INFINITY;
    int cut_i = -1;
    bool used = false;                                     // the histogram has been filled
    const auto keeps = [&](float l, int i) { return (l > cut) | ((l == cut) & (first + i <= cut_i)); };

    for (int which = 0; which < 2; ++which) {              // 0: top-k by count, 1: top-p by weight
        if (which == 0 ? top_k <= 0 || top_k >= V : top_p >= 1.f) continue;
        const bool by_weight = which == 1;
        if (by_weight) {
            if (used) {
                __syncthreads();
                clear_hist();
                __syncthreads();
            }
            // Tokens too light to be in the shortest prefix: below (1 - top_p) / V of the largest, all of them together
            // leave top_p of the whole to the others. They count towards the whole weight only. By whole bins (three
            // spare for the rounding), so that a bin's tokens are all in the histogram or all not; and not where the
            // limit is below 64 multiples of 2^-32, of which a weight is a whole number.
            const float light = __fdiv_rn(1.f - top_p, (float)V);
            const int light_bin = light >= 0x1p-26f ? BINS - 4 + (int)floorf((float)PER_OCTAVE * __log2f(light)) : 0;
            int rest_hi = 0;
            int rest_lo = 0;
            for (int q = tid; q < quads4; q += SA_THREADS) {
                const float4 v = x4[q];
                const float* l = &v.x;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool in = keeps(l[j], 4 * q + j);
                    const int b = scale.bin(l[j]);
                    const Parts w(scale.chance(l[j]));
                    if (in & (b >= light_bin)) {
                        atomicAdd(&sh.hist.n[b], 1u);
                        atomicAdd(&sh.hist.lo[b], w.lo);
                        if (w.hi) atomicAdd(&sh.hist.hi[b], (uint32_t)w.hi);
                    }
                    rest_hi += in & (b < light_bin) ? w.hi : 0;
                    rest_lo += in & (b < light_bin) ? w.lo : 0;
                }
            }
            const u64 rest = warp_sum(whole(rest_hi, rest_lo));
            if (lane == 0) sh.warp_w[warp] = rest;
        } else {
            for (int q = tid; q < quads4; q += SA_THREADS) {
                const float4 v = x4[q];
                const float* l = &v.x;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (l[j] > -INFINITY) atomicAdd(&sh.hist.n[scale.bin(l[j])], 1u);
            }
        }
        used = true;
        __syncthreads();
        for (int c = warp; c < 64; c += SA_WARPS) {        // sums of 64 bins, to every block
            const int b = 64 * c + lane;
            Sum s = {0, __reduce_add_sync(ALL, sh.hist.n[b] + sh.hist.n[b + 32]), 0};
            if (by_weight)
                s.w = warp_sum(whole((long long)sh.hist.hi[b] + sh.hist.hi[b + 32], (long long)sh.hist.lo[b] + sh.hist.lo[b + 32]));
            if (by_weight && c == 0) s.w += warp_sum(lane < SA_WARPS ? sh.warp_w[lane] : 0);   // below every possible cut
            if (lane < C) *in_block<C>(&sh.coarse[rank][c], lane) = s;
        }
        cluster_sync<C>();
        if (warp == 0) {
            u64 mass = 0;
            if (by_weight) {
#pragma unroll
                for (int r = 0; r < C; ++r) mass += sh.coarse[r][lane].w + sh.coarse[r][lane + 32].w;
                mass = warp_sum(mass);
            }
            if (lane == 0) {
                sh.mass = mass;
                sh.found_cut = Found{0, 0, 0, 0};
            }
            __syncwarp();
            find_cut<C, 2>(&sh.coarse[0][0], 64, by_weight, !by_weight ? (u64)top_k : share_of(top_p, mass), &sh.found_cut);
        }
        __syncthreads();
        const u64 enough = !by_weight ? (u64)top_k : share_of(top_p, sh.mass);
        const int oct = sh.found_cut.at;
        if (oct < 0) {                                     // fewer tokens than top_k: all are kept
            cluster_sync<C>();                             // every block has read coarse
            continue;
        }
        if (tid < 64 * C) {                                // its bins, to every block
            const int b = 64 * oct + (tid & 63);
            *in_block<C>(&sh.fine[rank][tid & 63], tid >> 6) = Sum{whole(sh.hist.hi[b], sh.hist.lo[b]), sh.hist.n[b], 0};
        }
        cluster_sync<C>();
        if (warp == 0) find_cut<C, 2>(&sh.fine[0][0], 64, by_weight, enough, &sh.found_cut);
        if (tid == 0) sh.next = 0;
        __syncthreads();
        const int in_oct = sh.found_cut.at, bin = 64 * oct + in_oct;
        const bool finish = sh.found_cut.above_n + sh.found_cut.in <= LIST;      // one block takes it from here
        if (warp < C) {                                    // how many tokens block `warp` will gather
            uint32_t c = 0;
            if (finish) {
                c = (lane > oct ? sh.coarse[warp][lane].n : 0) + (lane + 32 > oct ? sh.coarse[warp][lane + 32].n : 0);
                if (lane >= in_oct) c += sh.fine[warp][lane].n;
                if (lane + 32 >= in_oct) c += sh.fine[warp][lane + 32].n;
            } else if (lane == 0) {
                c = sh.fine[warp][in_oct].n;
            }
            c = __reduce_add_sync(ALL, c);
            if (lane == 0) sh.count[warp] = c;
        }
        __syncthreads();

        // A kept token of the bin (or, to finish, from it up), and its order.
        const auto here = [&](float l, int i) {
            const int b = scale.bin(l);
            return (finish ? b >= bin : b == bin) & keeps(l, i);
        };
        const auto order_at = [&](int i) { return order_of(x[i], first + i); };
        // To narrow a bin, orders are taken from the lowest logit that it can hold, so that their leading bits say something.
        const float down = __fdiv_rn(1.f / PER_OCTAVE, scale.hi), dist = (float)(BINS - 1 - bin);
        const bool far = !(down < 1e30f);                  // temperatures past 1e32: any logit may be in any bin
        const uint32_t key_hi = far ? 0xffffffffu : key_of(fmaf(-fmaxf(dist - 0.75f, 0.f), down, top)) + 8;
        const uint32_t key_lo = far || bin == 0 ? 0 : key_of(fmaf(-(dist + 0.75f), down, top)) - 8;
        const auto from_low = [&](int i) {
            return (u64)(min(max(key_of(x[i]), key_lo), key_hi) - key_lo) << 32 | (uint32_t)~(first + i);
        };
        u64 prefix = 0;                                    // of the orders in a narrowed bin
        int known = 0;
        if (!finish && sh.found_cut.in > LIST) known = min(__clz(key_hi - key_lo), 31);
        if (!finish) {
            for (int round = 0; sh.found_cut.in > LIST && known < 64; ++round) {   // 5 bits a round
                const int bits = min(5, 64 - known);
                __syncthreads();
                if (tid < 32) sh.hist.n[tid] = sh.hist.lo[tid] = sh.hist.hi[tid] = 0;
                __syncthreads();
                for (int i = tid; i < n; i += SA_THREADS) {
                    if (!here(x[i], i)) continue;
                    const u64 o = from_low(i);
                    if (known && o >> (64 - known) != prefix) continue;
                    const int d = (int)(o >> (64 - known - bits)) & ((1 << bits) - 1);
                    atomicAdd(&sh.hist.n[d], 1u);
                    if (by_weight) {
                        const Parts w(scale.chance(x[i]));
                        atomicAdd(&sh.hist.lo[d], w.lo);
                        atomicAdd(&sh.hist.hi[d], (uint32_t)w.hi);
                    }
                }
                __syncthreads();
                Sum* tab = round & 1 ? &sh.fine[0][0] : &sh.coarse[0][0];
                const int width = 64;
                for (int r = warp; r < C; r += SA_WARPS)
                    *in_block<C>(tab + rank * width + lane, r) =
                        Sum{whole(sh.hist.hi[lane], sh.hist.lo[lane]), sh.hist.n[lane], 0};
                cluster_sync<C>();
                if (warp == 0) {
                    find_cut<C, 1>(tab, width, by_weight, enough, &sh.found_cut);
                    __syncwarp();
                    if (lane < C) sh.count[lane] = tab[lane * width + sh.found_cut.at].n;
                }
                __syncthreads();
                prefix = prefix << bits | (u64)sh.found_cut.at;
                known += bits;
            }
        }

        // Gather: everything from the bin up (to block 0), or the narrowed bin (to every block).
        uint32_t base = 0, listed = 0;
#pragma unroll
        for (int r = 0; r < C; ++r) {
            if (r < rank) base += sh.count[r];
            listed += sh.count[r];
        }
        const uint32_t mine = sh.count[rank];
        __syncthreads();                                   // the histogram is done with
        for (int q = tid; q < quads4; q += SA_THREADS) {
            const float4 v = x4[q];
            const float* l = &v.x;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (!here(l[j], 4 * q + j)) continue;
                if (known && from_low(4 * q + j) >> (64 - known) != prefix) continue;
                const uint32_t to = atomicAdd(&sh.next, 1u);
                if (to < LIST) sh.found[to] = 4 * q + j;          // in any order
            }
        }
        __syncthreads();
        if (tid < (int)mine) {
            const u64 o = order_at((int)sh.found[tid]);
            if (base + tid < LIST) {
                if (finish) {
                    *in_block<C>(&sh.list[base + tid], 0) = o;
                } else {
#pragma unroll
                    for (int r = 0; r < C; ++r) *in_block<C>(&sh.list[base + tid], r) = o;
                }
            }
        }
        cluster_sync<C>();
        if (finish && rank != 0) return;                   // block 0 has all it needs

        // The filters: a thread's token has `ahead.n` tokens of the list before it, weighing ahead.w.
        const int count = (int)listed;
        int size = 32;
        while (size < count) size <<= 1;
        const bool real = tid < count;
        const u64 o = real ? sh.list[tid] : 0;
        const float ce = real ? scale.chance(value_of((uint32_t)(o >> 32))) : 0.f;
        const u64 cw = real ? weight(ce) : 0;
        if (real) sh.ranked[tid] = make_ulonglong2(o, cw);
        __syncthreads();
        u64 all;
        const Sum ahead = rank_in(sh, sh.beside, count, size, [](u64 j, u64 i) { return j > i; }, &all);
        const u64 above = finish ? 0 : sh.found_cut.above;
        const uint32_t above_n = finish ? 0 : sh.found_cut.above_n;
        bool keep;
        if (!by_weight) {
            keep = real && ahead.n + above < (u64)top_k;
            if (finish) {
                if (real && ahead.n == (uint32_t)top_k - 1) sh.pick[0] = ahead.w + cw;       // the cut lies in the list
                __syncthreads();
                keep = keep && (top_p >= 1.f || ahead.n == 0 || ahead.w < share_of(top_p, sh.pick[0]));
            }
        } else {
            keep = real && (above + ahead.w < enough || ahead.n + above_n == 0);
        }
        if (finish) keep = keep && !(ce < min_p);
        const int n_keep = __syncthreads_count(keep);      // at least one
        if (!finish) {
            if (keep && (int)ahead.n == n_keep - 1) sh.pick[1] = o;      // what is kept comes first
            __syncthreads();
            cut = value_of((uint32_t)(sh.pick[1] >> 32));
            cut_i = (int)~(uint32_t)sh.pick[1];
            continue;
        }
        // The draw, in index order.
        const u64 lw = keep ? cw : 0;
        if (real) sh.ranked[tid].y = lw;
        __syncthreads();
        const u64 to = rank_in(sh, sh.beside, count, size, [](u64 j, u64 i) { return (uint32_t)j > (uint32_t)i; }, &all).w + lw;
        const u64 target = drawn_at(u, all);
        if (real && to >= target && to - lw < target) {
            p.tokens[row] = (int)~(uint32_t)o;
            if (p.probs) p.probs[row] = __fdiv_rn(ce, __ull2float_rn(all) * 0x1p-32f);
            if (p.kept) p.kept[row] = n_keep;
        }
        return;
    }

    // The draw over the whole row, in index order: a warp has neighbouring tokens. x becomes e, 0 where not kept.
    const int run = (quads4 + SA_WARPS - 1) / SA_WARPS, q0 = warp * run, q1 = min(quads4, q0 + run);
    int sum_hi = 0;
    int sum_lo = 0;
    uint32_t kept = 0;
    for (int q = q0 + lane; q < q1; q += 32) {
        float4 v = x4[q];
        float* e = &v.x;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float c = scale.chance(e[j]);
            const bool in = (c >= min_p) & keeps(e[j], 4 * q + j);
            e[j] = in ? c : 0.f;
            kept += in;
            const Parts w(e[j]);
            sum_hi += w.hi;
            sum_lo += w.lo;
        }
        x4[q] = v;
    }
    u64 sum = whole(sum_hi, sum_lo);
    sum = warp_sum(sum);
    kept = __reduce_add_sync(ALL, kept);
    if (lane == 0) {
        sh.warp_w[warp] = sum;
        sh.part[warp] = kept;
    }
    __syncthreads();
    if (warp == 0) {
        const u64 w = warp_sum(lane < SA_WARPS ? sh.warp_w[lane] : 0);
        const uint32_t k = __reduce_add_sync(ALL, lane < SA_WARPS ? (uint32_t)sh.part[lane] : 0);
        if (lane < C) *in_block<C>(&sh.total[rank], lane) = Sum{w, k, 0};
    }
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
    for (int w = 0; w < warp; ++w) before += sh.warp_w[w];
    const u64 target = drawn_at(u, all);
    if (before >= target || before + sum < target) return; // another warp's
    for (int s0 = q0; s0 < q1; s0 += 32) {
        const int q = s0 + lane;
        const float4 v = q < q1 ? x4[q] : make_float4(0.f, 0.f, 0.f, 0.f);
        const float* e = &v.x;
        u64 w[4], own = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = weight(e[j]);
            own += w[j];
        }
        u64 to = before + warp_scan(own);
        before = __shfl_sync(ALL, to, 31);
        if (to >= target && to - own < target) {
            to -= own;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (to < target && to + w[j] >= target) {
                    p.tokens[row] = first + 4 * q + j;
                    if (p.probs) p.probs[row] = __fdiv_rn(e[j], __ull2float_rn(all) * 0x1p-32f);
                }
                to += w[j];
            }
        }
        if (before >= target) return;
    }
}

// A launch of C blocks a row, in clusters if C > 1.
template <int C>
struct Launch {
    static inline LaunchPrep prep;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    Launch(int rows, size_t smem, cudaStream_t s) {
        cfg.gridDim = dim3((unsigned)rows * C);
        cfg.blockDim = dim3(SA_THREADS);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = s;
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim = {C, 1, 1};
        cfg.attrs = attr;
        cfg.numAttrs = C > 1 ? 2 : 1;
    }
};

// least: shared memory to ask for at least.
template <int C>
cudaError_t launch(const Sample& p, size_t least, cudaStream_t s) {
    const int slice = ((p.vocab + C - 1) / C + 3) / 4 * 4;
    const size_t need = SHARED_BYTES + 4 * (size_t)slice;
    int sms = 0;
    cudaError_t e = Launch<C>::prep.get(sample_kernel<C>, SMEM_MOST, &sms);
    if (e != cudaSuccess) return e;
    Launch<C> l(p.batch, need > least ? need : least, s);
    e = cudaLaunchKernelEx(&l.cfg, sample_kernel<C>, p, slice);
    return e != cudaSuccess ? e : cudaGetLastError();
}

// How many rows in clusters of C run at once with an SM to every block (clusters lie within a part of the GPU, so fewer
// than its SMs hold). Asked for once per device.
template <int C>
cudaError_t rows_alone(int* rows) {
    static std::atomic<int> known[LaunchPrep::MAX_DEVICES];              // and 1
    int dev = 0, sms = 0, n = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = Launch<C>::prep.get(sample_kernel<C>, SMEM_MOST, &sms);      // (checks dev)
    if (e != cudaSuccess) return e;
    if ((n = known[dev].load(std::memory_order_relaxed)) == 0) {
        Launch<C> l(1, SMEM_MOST, nullptr);
        if ((e = cudaOccupancyMaxActiveClusters(&n, sample_kernel<C>, &l.cfg)) != cudaSuccess) return e;
        known[dev].store(++n, std::memory_order_relaxed);
    }
    *rows = n - 1;
    return cudaSuccess;
}

}  // namespace

// Blocks per row: few tokens are not worth an exchange. Above that clusters of 8 while every block gets an SM (15 rows on
// the GPU measured), then of 6 while those do (23), then of 8, two to an SM where shared memory allows; beyond, the rows
// queue either way. Under top-p 0.9, us for clusters of 8, of 6 (and of 8 without asking for an SM each):
//   128256 logits   8 rows: 22.2, 25.4 (22.2)   15: 22.4, 25.7 (22.4)   16: 41.2, 25.7 (41.2)   23: 42.4, 25.6 (42.4)   24: 42.5, 46.6 (42.5)
//   32000           8 rows: 13.6, 14.3 (17.6)   15: 14.5, 15.0 (19.1)   16: 25.1, 14.9 (18.9)   23: 26.5, 15.1 (20.4)   24: 26.6, 26.4 (20.3)
// Of 16 x 128256, clusters of 5 take 27.9 and of 4 take 32.1.
cudaError_t launch_sample(const Sample& p, cudaStream_t s) {
    if (p.vocab <= 4096) return launch<1>(p, 0, s);
    if (p.vocab <= 16384) return launch<4>(p, 0, s);
    int rows = 0;
    cudaError_t e = rows_alone<8>(&rows);
    if (e != cudaSuccess) return e;
    if (p.batch <= rows) return launch<8>(p, SMEM_ALONE, s);
    e = rows_alone<6>(&rows);
    if (e != cudaSuccess) return e;
    if (p.batch <= rows && p.vocab <= 6 * (SLICE_MOST - 4)) return launch<6>(p, SMEM_ALONE, s);
    return launch<8>(p, 0, s);
}

}  // namespace vbq
