// vbq_attend.cu — attention over the 4-bit cache, for one to sixteen new rows
// per sequence.
//
// out = sum_j softmax_j(scale q.k_j) v_j over the keys j in (p - window, p] of
// a row at position p, in one pass over the cache with a running maximum and
// sum. The query rows that share a key-value head (its group of heads, times
// the sequence's new rows) go through the cache together, 8 * NT at a time.
//
// Bound: the cache's bytes (136 B per token and head at d = 128) at HBM speed,
// which leaves under three thread instructions per code at full issue: the
// decode has to be nearly free. So the codes go to the tensor cores
// (mma.m16n8k16, f16) as they are: a masked nibble at bits 2..5 of a half is the
// denormal u * 2^-22 exactly, one at bits 6..9 is u * 2^-18, so one mask makes
// two operands, with a byte swap for every second pair (kv_turned). The MMA
// aligns its products by their operands' exponents, and a denormal's is that of
// 2^-14: the fp32 sum resolves 2^-16 of a code's step from bits 2..5 and 2^-20
// from bits 6..9. Keys take both (a score's error is then below 2^-16 of
// sum |q| in units of the key's scale); values are shifted up to bits 6..9
// first, so that a large probability on a zero code leaves nothing behind.
//   - S^T = K Q^T: keys are the MMA's 16 rows, query rows its 8 columns. The
//     middle of the codes (8) enters as the accumulators' start, -8 times the
//     group's sum of q; the key's scale multiplies the group's result in fp32.
//     q enters in f16, scaled per row by a power of two so that its largest
//     value is in [2^12, 2^13): exact for BF16 values down to 2^-25 of it.
//   - O^T = V^T P^T: a value's word holds 8 dimensions of one key, so pairing
//     the words of two keys (a byte permute per 4 operands) gives A fragments
//     whose rows are dimensions. P^T is S^T's accumulators times the key's
//     value scale, rounded to f16 (11 bits) and turned by movmatrix; scales are
//     taken relative to a running power of two, as the maximum is, so that f16
//     never runs out of range. The codes' middle is subtracted at the end: one
//     more MMA with ones sums the rounded P, so what is subtracted is exactly
//     what the rounded probabilities added.
// Weights as the A operand make every decoded nibble pair serve 8 query rows
// and keep the accumulators' columns (rows of q) in the same lanes for S, P and
// O: no shuffles but the maximum's.
//
// A warp takes whole pages (64 keys of one head, one contiguous blob) through
// its own ring of shared-memory stages filled by bulk copies: no barrier in the
// steady state. At 256 dimensions (17 KB a page) the keys' and the values'
// halves of one stage are filled apart, each as soon as it is read, which makes
// room for 8 warps: a page is a chain of 5 us that only more warps hide.
//
// The (sequence, row tile, head) segments are cut into parts of at most `quantum`
// pages, one part per block and one block per SM, if that leaves no block with
// much more than an even share (long segments by whole rounds of a block's warps:
// fewer parts to join); otherwise the pages of all segments form one list that is
// cut evenly, and a block may finish one segment and start another. Parts are
// joined through the workspace by the block that finishes a segment last, in an
// order of their own, so results do not depend on timing.
// With more segments than blocks, teams of a block's warps (1, 2, ... all of
// them) may take whole segments instead, each team by itself: a segment's start
// and join cost a block 5 us, and a list of short ones is a run of those. A
// small cost model picks the team's size or the list, the same in every block.
// Only calls that can have that many segments run the variant with teams: its
// list is 4% slower (32 sequences of 16384: 106 us, 103 without).
//
// A key may be attended to by some rows of a tile only, or by none (before a
// window, between the windows of distant rows, after the last token), and what
// was never written may be any bytes. Scores are masked per row; a key without
// rows also loses its value scale, since 0 times a NaN scale is NaN in the MMA
// for every row. Pages at an edge only; it costs them 0.1 us a call.
//
// Measured (one GB300, in a graph): 8 sequences of 65536 tokens, 32 heads of 128
// over 8: 99 us, 5.75 TB/s of cache. One of 32768: 17 us, of which 7 are the
// pages, 3 the start and 4 the join over 19 blocks. 16 rows each of two
// sequences, 4096 keys a row: 20 us, bound by instruction issue. 100 keys, 12
// heads of 64: 4.9 us, a chain of loads. One sequence of 32768, 16 heads over 2:
// 14.1 us. 64 sequences of up to 100 tokens, 32 heads over 8: 11.7 us (teams of
// 3; 22.7 as a list); of up to 1000: 24.8 (76); 24 of up to 659, 5 rows, 24 heads
// over 12: 17.6 (teams of 4; 41 as a list). 8 of 9000, 8 heads of 256 over 4: 26.
// When the shapes were chosen, each pair in one build of the time: 12 warps took
// 103 us where 8 took 108 and 16 took 118 (8 x 65536, 1022 warp instructions a
// page); parts of 12 pages 13.9 where parts of 7 took 16.7 (32768, 16 heads over
// 2); teams 11 and 25 where single warps took 14 and 48 and whole blocks 27 and
// 35 (64 x up to 100 and 1000); 8 warps of halves at d = 256 26 where 6 warps with
// two whole stages took 30 and 6 with two in halves 31 (8 x 9000).
#include <cuda_bf16.h>

#include <algorithm>

#include "vbq_decode.h"
#include "vbq_device.cuh"
#include "vbq_kernels.h"

namespace vbq {
namespace {

constexpr uint32_t FULL = 0xffffffffu;
constexpr int JOIN = 4;                         // parts whose loads are in flight at once
constexpr int CUT = 6;                           // pages a block takes at least of a segment that is cut
constexpr int STRADDLE = 16;                     // pages whose time a block's second segment costs
constexpr uint32_t LOW = 0x003c003cu, HIGH = 0x03c003c0u;    // codes at bits 2..5 and 6..9 of each half

enum Kind { PLAIN, TEAMS, SHARES };              // when which: at launch

// D: head dimension, NT: 8-row tiles of query rows per pass, W: warps, S: stages per warp,
// HALVES: a page's keys and its values are copied apart, each as soon as its half of the stage is read,
// KIND: what the kernel is made for.
template <int D_, int NT_, int W_, int S_, bool HALVES_, Kind KIND_>
struct Shape {
    static constexpr int D = D_, NT = NT_, W = W_, S = S_;
    static constexpr bool HALVES = HALVES_;
    static constexpr bool MANY = KIND_ == TEAMS, SHARED = KIND_ == SHARES;
    static constexpr int ROWS = 8 * NT;
    static constexpr int GR = D / 64;            // scale groups
    static constexpr int KW = D / 32;            // words of a key per lane
    static constexpr int TILES = D / 16;         // output tiles of 16 dimensions
    static constexpr int BLOB = 68 * D;
    static constexpr int THREADS = 32 * W;
    static constexpr int UNITS = ROWS * D / 4;   // 4 outputs each
    // shared memory
    static constexpr int BARS = W * S * BLOB;                    // full barriers
    static constexpr int VBARS = BARS + (HALVES ? W * S * 8 : 0);   // of the values
    static constexpr int ML = VBARS + W * S * 8;                 // (maximum, sum) per warp and row
    static constexpr int FACTOR = ML + W * ROWS * 8;             // a warp's factor per row, then (maximum, sum) per row
    static constexpr int CUM = FACTOR + W * ROWS * 4 + ROWS * 8; // pages before each sequence
    static_assert(W <= 16 && ROWS * 16 <= THREADS, "the join's first step");
    static constexpr int KEPT = HALVES ? kv_values_at(D) : 0;    // a stage's place for a partial result
    static_assert(KEPT + UNITS * 16 <= BLOB, "a partial result has room in a stage");
    static_assert(KV_MAX_ROWS == 16, "16 lanes to a sequence");
    static constexpr int SPAN = CUM + (KV_MAX_BATCH + 2) * 8;    // first page and last key of each sequence
    static constexpr int FILLED = SPAN + KV_MAX_BATCH * 8;       // sequences with pages before each
    static constexpr int MISC = FILLED + (MANY ? (KV_MAX_BATCH + 4) * 4 : 0);
    static constexpr int SMEM = MISC + 64 + 4 * W;
    static constexpr int PART = ROWS * D + 2 * ROWS;             // floats of a partial result
};

struct Misc {
    int64_t quantum;
    int abort, last;
    int aligned;                                 // a block has one part of one segment
    int team;                                    // warps that take a segment together, 0: none does
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }   // e in -126..127
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t transposed(uint32_t a) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The words at a shared address (16, 8 or 4 bytes at a time).
template <int N>
__device__ __forceinline__ void lds_words(uint32_t (&w)[N], uint32_t at) {
    if constexpr (N == 1) {
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at));
    } else if constexpr (N == 2) {
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3])
                         : "r"(at + 4 * i));
    }
}

// One (sequence, row tile, key-value head): its place in the list of pages.
struct Segment {
    int b, rt, h;
    int64_t start, pages;                        // in the list
    int64_t index;                               // among all segments
};

struct List {
    const int64_t* cum;                          // shared: pages of one head before each sequence
    int batch, kv_heads, per_seq;                // segments per sequence
    __device__ Segment segment(int b, int64_t k) const {
        Segment s;
        s.b = b;
        s.pages = cum[b + 1] - cum[b];
        s.start = cum[b] * per_seq + k * s.pages;
        s.rt = (int)k / kv_heads;
        s.h = (int)k - s.rt * kv_heads;
        s.index = (int64_t)b * per_seq + k;
        return s;
    }
    __device__ __noinline__ Segment at(int64_t p) const {     // of a page of the list
        int b = 0, e = batch;                    // the last b with cum[b] * per_seq <= p (it has pages: p is in the list)
        while (e - b > 1) {
            const int m = (b + e) >> 1;
            if (cum[m] * per_seq <= p) b = m; else e = m;
        }
        const int64_t in = p - cum[b] * per_seq;
        return segment(b, in / (cum[b + 1] - cum[b]));
    }
};

__device__ __forceinline__ int parts_of(int64_t pages, int64_t quantum) {
    return (int)(((uint32_t)pages + (uint32_t)quantum - 1) / (uint32_t)quantum);     // a sequence has below 2^26 pages
}

// A part's pages, up to a whole round of the block's W warps if the join gains by it: a page more costs 0.13 us, a step of
// the join 0.44. (Out of line: few calls come here, and the code in between is time at every start.)
template <int W>
__device__ __noinline__ int whole_rounds(int most, int pages) {
    const int round = (pages + W - 1) / W * W;
    const int steps = (parts_of(most, pages) + JOIN - 1) / JOIN - (parts_of(most, round) + JOIN - 1) / JOIN;
    return 10 * steps > 3 * (round - pages) ? round : pages;
}

// In place of a page that the table has outside the cache: keys and values of scale 0, which change nothing for the rows that
// do not attend to them. Reported if some row (positions pos) does; between the windows of distant rows none need be there.
__device__ uint4 nothing[kv_blob_bytes(256) / 16];
__device__ __noinline__ const uint8_t* no_page(const int32_t* pos, int rows, int window, int64_t page, int64_t table_keys) {
    const int64_t key0 = page * KV_PAGE;
#pragma unroll 1
    for (int t = 0; t < rows; ++t) {
        const int64_t p = pos[t];
        if (p < table_keys && p >= key0 && (window <= 0 || key0 + KV_PAGE - 1 > p - window)) atomicOr(&g_device_status, VBQ_DEVICE_RANGE);
    }
    return reinterpret_cast<const uint8_t*>(nothing);
}

template <class C>
__global__ void __launch_bounds__(C::THREADS, 1) kv_attend_kernel(KvView c, KvAttend a, int row_tiles, uint32_t* counts,
                                                                 float* parts) {
    constexpr int D = C::D, NT = C::NT, W = C::W, S = C::S, GR = C::GR, KW = C::KW;
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t sbase = smem_u32(smem);
    // (the shuffle tells the compiler that its index is one for the whole warp)
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);
    const int g = lane >> 2, t4 = lane & 3;
    // The lane's place in a blob: its key's words, the key's scales, its value words.
    const uint32_t klane = g * (D / 2) + t4 * (D / 8), slane = kv_scales_at(D) + g * (D / 16);
    const uint32_t vlane = kv_values_at(D) + t4 * (D / 2) + (D == 64 ? g : D == 128 ? g ^ ((t4 >> 1) << 2) : g ^ (t4 << 1)) * (D / 16);
    float2* ml = reinterpret_cast<float2*>(smem + C::ML);
    float* factor = reinterpret_cast<float*>(smem + C::FACTOR);
    float2* joined = reinterpret_cast<float2*>(smem + C::FACTOR + W * C::ROWS * 4);
    int64_t* cum = reinterpret_cast<int64_t*>(smem + C::CUM);
    int* filled = reinterpret_cast<int*>(smem + C::FILLED);
    int2* span = reinterpret_cast<int2*>(smem + C::SPAN);
    Misc* misc = reinterpret_cast<Misc*>(smem + C::MISC);
    int* kept_in = reinterpret_cast<int*>(smem + C::MISC + 64);          // where a warp's partial result is
    const uint32_t abort_addr = sbase + C::MISC + 8;
    const int group = a.heads / c.kv_heads, rows_all = group * a.rows, per_seq = row_tiles * c.kv_heads;

    if (tid < W * S) {
        mbar_init(sbase + C::BARS + 8 * tid, C::HALVES ? 2 : 1);         // keys and scales
        if constexpr (C::HALVES) mbar_init(sbase + C::VBARS + 8 * tid, 1);
    }
    if (tid == 0) {
        misc->abort = 0;
        misc->last = 0;
    }
    fence_barrier_init();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // Every sequence's range of pages.
    const int64_t table_keys = (int64_t)c.table_pages * KV_PAGE;
#pragma unroll 1
    for (int b0 = 0; b0 < a.batch; b0 += C::THREADS / KV_MAX_ROWS) {     // a lane per row, 16 to a sequence
        const int b = b0 + tid / KV_MAX_ROWS, t = tid % KV_MAX_ROWS;
        int hi = b < a.batch && t < a.rows ? a.pos[b * a.rows + t] : -1;
        if (hi >= table_keys) {                   // outside the cache: as an unused row
            if (blockIdx.x == 0) atomicOr(&g_device_status, VBQ_DEVICE_RANGE);
            hi = -1;
        }
        int mn = hi >= 0 ? hi : 0x7fffffff;
#pragma unroll
        for (int o = 1; o < KV_MAX_ROWS; o <<= 1) {
            hi = max(hi, __shfl_xor_sync(FULL, hi, o));
            mn = min(mn, __shfl_xor_sync(FULL, mn, o));
        }
        if (t != 0 || b >= a.batch) continue;
        const int lo = hi >= 0 && a.window > 0 && mn >= a.window ? mn - a.window + 1 : 0;
        span[b] = make_int2(lo / KV_PAGE, hi);
        cum[b + 1] = hi < 0 ? 0 : hi / KV_PAGE - lo / KV_PAGE + 1;
    }
    if (tid == 0) {
        cum[0] = 0;
        if constexpr (C::MANY) filled[0] = 0;
    }
    __syncthreads();
    if (warp == 0) {
        int64_t before = 0;
        int most = 0, used = 0;                   // sequences with pages
#pragma unroll 1
        for (int b0 = 0; b0 < a.batch; b0 += 32) {
            const int b = b0 + lane;
            int64_t x = b < a.batch ? cum[b + 1] : 0;
            most = max(most, (int)x);
            const uint32_t has = __ballot_sync(FULL, x > 0);
            if constexpr (C::MANY)
                if (b < a.batch) filled[b + 1] = used + __popc(has << (31 - lane));
            used += __popc(has);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t y = __shfl_up_sync(FULL, x, o);
                if (lane >= o) x += y;
            }
            x += before;
            before = __shfl_sync(FULL, x, 31);
            if (b < a.batch) cum[b + 1] = x;
        }
        most = __reduce_max_sync(FULL, most);
        __syncwarp();
        // An even share of the pages; segments that a block's warps take at once are not cut, and none into parts
        // that cost more to join than to read.
        const int blocks = (int)gridDim.x, least = most <= W ? most : CUT;
        const int64_t total = before * per_seq;
        const int64_t share_up = total < (1 << 30) ? (int64_t)(((uint32_t)total + blocks - 1) / (uint32_t)blocks)
                                                   : (total + blocks - 1) / blocks;
        const int64_t even = max(share_up, (int64_t)max(least, 1));
        // One part per block: parts of at most q pages, the least of a few q that fit.
        const int64_t segments = (int64_t)used * per_seq;
        int aligned = 0;
        int64_t quantum = even;
        if (segments <= blocks && used > 0) {
            const int share = blocks / (int)segments;      // parts each: always fits
            int fit = max((most + share - 1) / share, least), low = (int)even;
#pragma unroll 1
            for (int i = 0; i < 5 && low < fit; ++i) {
                const int q = (low + fit) / 2;
                uint32_t n = 0;
#pragma unroll 1
                for (int b = lane; b < a.batch; b += 32) n += parts_of(cum[b + 1] - cum[b], q);
                n = __reduce_add_sync(FULL, n);
                if ((int64_t)n * per_seq <= blocks) fit = q; else low = q + 1;
            }
            if (fit <= even + STRADDLE) {
                aligned = 1;
                quantum = fit;
                if (most > 2 * JOIN * fit) quantum = whole_rounds<W>(most, fit);
            }
        }
        int team = 0;
        if constexpr (C::MANY) {
            if (segments > blocks) {
                // The cost in pages of a warp (2.8 us, mostly latency): of teams of t warps (lane t - 1) that take their
                // segments one after another, each with its start and join (3.5 us, less for a warp alone); and of the
                // list (lane W), where a block may have a run of the shortest segments (5 us each). Fitted to every team's
                // time over eight sets of sequences; it picks the fastest or one within a tenth of it.
                const uint32_t n = (uint32_t)segments, avg = (uint32_t)((float)total / (float)n + 0.999f), t = lane + 1;
                float cost = INFINITY;
                if (t <= W && W % t == 0) {
                    const uint32_t teams = (uint32_t)blocks * (W / t), rounds = (n + teams - 1) / teams;
                    cost = (float)((most + t - 1) / t) + (float)(rounds - 1) * ((avg + t - 1) / t) +
                           (float)rounds * (t == 1 ? 0.5f : 1.25f + 0.04f * t);
                }
                if (lane == W)
                    cost = (float)even / W + 2.f + 2.f * fminf((float)n / blocks * most / avg, (float)even);
                const uint32_t least_cost = __reduce_min_sync(FULL, __float_as_uint(cost));
                const int pick = __ffs(__ballot_sync(FULL, __float_as_uint(cost) == least_cost));
                team = pick <= W ? pick : 0;
            }
        }
        if (lane == 0) {
            misc->quantum = quantum;
            misc->aligned = aligned;
            misc->team = team;
        }
    }
    __syncthreads();
    const List list{cum, a.batch, c.kv_heads, per_seq};
    const int64_t quantum = misc->quantum;
    const bool aligned = misc->aligned;
    const int team = C::MANY ? misc->team : 0;
    int64_t p0 = 0, p1 = 0;                       // the block's pages of the list
    int first_part = 0, parts_here = 0;           // aligned: the segment's blocks
    Segment s = {};
    if (aligned) {
        int left = blockIdx.x;
#pragma unroll 1
        for (int b = 0; b < a.batch; ++b) {
            const int64_t pages = cum[b + 1] - cum[b];
            const int n = parts_of(pages, quantum);
            if (left < n * per_seq) {
                const int k = left / n, i = left - k * n;
                s = list.segment(b, k);
                const int each = (int)pages / n, more = (int)pages - each * n;
                p0 = s.start + i * each + min(i, more);
                p1 = p0 + each + (i < more);
                first_part = (int)blockIdx.x - i;
                parts_here = n;
                break;
            }
            left -= n * per_seq;
        }
    } else if (!C::MANY || team == 0) {
        const int64_t total = cum[a.batch] * per_seq;
        p0 = min(total, (int64_t)blockIdx.x * quantum);
        p1 = min(total, p0 + quantum);
        if (p0 < p1) s = list.at(p0);
    }

    // Teams: the warp's place in its own, the team's segments (every so many of those with pages).
    int member = 0;
    int next = 0, every = 0, n_segments = 0;     // (below 2^31 segments)
    if constexpr (C::MANY)
        if (team != 0) {
            n_segments = filled[a.batch] * per_seq;
            member = warp % team;
            next = (int)blockIdx.x * (W / team) + warp / team;
            every = (int)gridDim.x * (W / team);
        }
    const auto nth = [&](int r) {
        int b = 0, e = a.batch;                   // the last b with filled[b] * per_seq <= r
#pragma unroll 1
        while (e - b > 1) {
            const int m = (b + e) >> 1;
            if (filled[m] * per_seq <= r) b = m; else e = m;
        }
        return list.segment(b, r - filled[b] * per_seq);
    };

    // Sequences without keys: zeros.
#pragma unroll 1
    for (int b = blockIdx.x; b < a.batch; b += gridDim.x) {
        if (cum[b + 1] != cum[b]) continue;
        uint4* o = reinterpret_cast<uint4*>(a.out + (int64_t)b * a.rows * a.heads * D);
#pragma unroll 1
        for (int64_t i = tid; i < (int64_t)a.rows * a.heads * (D / 8); i += C::THREADS) o[i] = make_uint4(0, 0, 0, 0);
    }

    // The block's pages go round the warps: p0 + warp, + W, ...; the k-th of a warp uses stage k % S.
    const uint32_t n_pages = (uint32_t)(p1 - p0), mine = n_pages / W + ((uint32_t)warp < n_pages % W);
    const uint8_t* src = nullptr;                 // lane i: of the page 32 * n + i
    uint32_t issued = 0, used = 0, landed = 0;    // landed: copies waited for
    uint32_t v_issued = 0, v_landed = 0, last = 0;   // HALVES: the values' (one page behind at most); lane of the last page
    bool ok = true;
    int ahead_next = next;                        // teams: the next segment to copy, and the one being copied
    int ahead = 0, ahead_end = 0;                 // (its next page and its pages)
    const auto page_at = [&](const Segment& t, int64_t in) -> const uint8_t* {       // the blob of a segment's page
        const int64_t page = c.table[t.b * c.table_stride + span[t.b].x + in];
        if (page < 0 || page >= c.n_pages) return no_page(a.pos + t.b * a.rows, a.rows, a.window, span[t.b].x + in, table_keys);
        return c.pages + (page * c.kv_heads + t.h) * C::BLOB;
    };
    auto issue = [&]() {                          // the next page's copy
        if (!ok) return;
        uint32_t from = issued;                   // the lane that knows the page
        bool listed = true;
        if constexpr (C::MANY)
            if (team != 0) {
                while (ahead >= ahead_end) {      // (a short segment has no page for some of the team)
                    if (ahead_next >= n_segments) return;
                    ahead_end = (int)nth(ahead_next).pages;
                    ahead_next += every;
                    ahead = member;
                }
                from = (uint32_t)(ahead / team);
                if ((from & 31) == 0 && ahead + lane * team < ahead_end)
                    src = page_at(nth(ahead_next - every), ahead + lane * team);
                ahead += team;
                listed = false;
            }
        if (listed) {
            if (issued >= mine) return;
            if ((issued & 31) == 0) {
                const uint32_t k = issued + lane;
                if (k < mine) {
                    const int64_t p = p0 + warp + (int64_t)k * W;
                    const Segment t = p < s.start + s.pages ? s : list.at(p);
                    src = page_at(t, p - t.start);
                }
            }
        }
        const int st = (int)(issued % S);
        if constexpr (C::HALVES) {
            const uint32_t stage = sbase + (warp * S + st) * C::BLOB, bar = sbase + C::BARS + 8 * (warp * S + st);
            if (lane == (int)(from & 31)) {
                bulk_load(stage, src, kv_values_at(D), bar);
                bulk_load(stage + kv_scales_at(D), src + kv_scales_at(D), C::BLOB - kv_scales_at(D), bar);
            }
            last = from & 31;
        } else if (lane == (int)(from & 31)) {
            bulk_load(sbase + (warp * S + st) * C::BLOB, src, C::BLOB, sbase + C::BARS + 8 * (warp * S + st));
        }
        ++issued;
    };
    auto issue_values = [&]() {                   // HALVES: of the page whose keys were copied last
        if (!ok || v_issued == issued) return;
        const int st = (int)(v_issued % S);
        if (lane == (int)last)
            bulk_load(sbase + (warp * S + st) * C::BLOB + kv_values_at(D), src + kv_values_at(D),
                      kv_scales_at(D) - kv_values_at(D), sbase + C::VBARS + 8 * (warp * S + st));
        ++v_issued;
    };
    auto refill = [&]() {                         // a stage whose last reads were a partial result's
        if constexpr (C::HALVES) issue_values(); else issue();
    };
    // A segment's queries (16 bytes of each word of the lane's row) and, per accumulator column, its rows' positions.
    uint4 qw[NT][KW];
    int pos[NT][2];
    const auto load_rows = [&] {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = s.rt * C::ROWS + 8 * n + g;
            const bool live = r < rows_all;
            const int t = live ? r / group : 0, hq = live ? s.h * group + r - t * group : 0;
            const uint16_t* q = a.q + (((int64_t)s.b * a.rows + t) * a.heads + hq) * D + 8 * t4;
#pragma unroll
            for (int j = 0; j < KW; ++j)
                qw[n][j] = live ? *reinterpret_cast<const uint4*>(q + 64 * (j / 2) + 32 * (j & 1)) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int rc = s.rt * C::ROWS + 8 * n + 2 * t4 + i;
                pos[n][i] = rc < rows_all ? a.pos[s.b * a.rows + rc / group] : -1;
            }
        }
    };
    if (p0 < p1 && warp == 0) {                   // the first queries, before the copies: behind them they would wait
        const int r = s.rt * C::ROWS + lane % C::ROWS;
        if (r < rows_all) {
            const uint16_t* q = a.q + (((int64_t)s.b * a.rows + r / group) * a.heads + s.h * group + r % group) * D;
            for (int i = lane / C::ROWS; i < D / 64; i += 32 / C::ROWS) asm volatile("prefetch.global.L1 [%0];" :: "l"(q + 64 * i));
        }
    }
#pragma unroll 1
    for (int i = 0; i < S; ++i) {
        issue();
        if constexpr (C::HALVES) issue_values();
    }

    int64_t cur = p0;
#pragma unroll 1
    while (C::MANY && team != 0 ? next < n_segments : cur < p1) {
        if (C::MANY && team != 0) {
            s = nth(next);
            next += every;
        } else if (cur != p0) {
            s = list.at(cur);
        }
        load_rows();
        const int64_t end = C::MANY && team != 0 ? s.start + s.pages : min(p1, s.start + s.pages);
        const int hi_key = span[s.b].y, page0 = span[s.b].x;             // the sequence's last key and first page

        // Query fragments of the tile's rows, and the rows' parameters per accumulator column.
        uint32_t qb[NT][KW][4];
        float corr[NT][GR][2], f[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < KW; ++j) {
                const uint32_t v[4] = {qw[n][j].x, qw[n][j].y, qw[n][j].z, qw[n][j].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) top = max(top, max(v[i] << 16 & 0x7fff0000u, v[i] & 0x7fff0000u));
            }
            top = max(top, __shfl_xor_sync(FULL, top, 1));
            top = max(top, __shfl_xor_sync(FULL, top, 2));
            const int e = max((int)(top >> 23), 13);                     // biased exponent of the row's largest value
            // to [2^12, 2^13), with the scale's sign, so that the scores' factor is positive (scale 0: all scores 0)
            const float up = a.scale > 0.f ? pow2(139 - e) : a.scale < 0.f ? -pow2(139 - e) : 0.f;
            const float fr = fmaxf(fabsf(a.scale) * 1.44269504f * 0x1p22f * pow2(e - 139), 1e-37f);
            float sum[GR];
#pragma unroll
            for (int i = 0; i < GR; ++i) sum[i] = 0.f;
#pragma unroll
            for (int j = 0; j < KW; ++j) {
                const uint32_t v[4] = {qw[n][j].x, qw[n][j].y, qw[n][j].z, qw[n][j].w};
                float x[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[2 * i] = __uint_as_float(v[i] << 16) * up;
                    x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u) * up;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {                            // nibbles i and i + 4; odd ones carry a factor 16
                    const float by = i & 1 ? 0.0625f : 1.f;
                    qb[n][j][i] = half2_bits(x[i] * by, x[i + 4] * by);
                    const __half2 h = *reinterpret_cast<const __half2*>(&qb[n][j][i]);
                    sum[j / 2] += (__low2float(h) + __high2float(h)) * (i & 1 ? 16.f : 1.f);
                }
            }
#pragma unroll
            for (int i = 0; i < GR; ++i) {
                sum[i] += __shfl_xor_sync(FULL, sum[i], 1);
                sum[i] += __shfl_xor_sync(FULL, sum[i], 2);
                corr[n][i][0] = -8.f * 0x1p-22f * __shfl_sync(FULL, sum[i], 8 * t4);
                corr[n][i][1] = -8.f * 0x1p-22f * __shfl_sync(FULL, sum[i], 8 * t4 + 4);
            }
            f[n][0] = __shfl_sync(FULL, fr, 8 * t4);
            f[n][1] = __shfl_sync(FULL, fr, 8 * t4 + 4);
        }
        // Keys that every row of the tile attends to: (open, close].
        int close = 0x7fffffff, open = -1;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (pos[n][i] > hi_key) pos[n][i] = -1;                  // outside the cache: an unused row
                if (s.rt * C::ROWS + 8 * n + 2 * t4 + i < rows_all) close = min(close, pos[n][i]);
                if (a.window > 0 && pos[n][i] >= 0) open = max(open, pos[n][i] - a.window);
            }
        close = min(__reduce_min_sync(FULL, close), hi_key);
        open = __reduce_max_sync(FULL, open);

        float acc[C::TILES][NT][4], ones[GR][NT][4], m[NT][2], l[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int i = 0; i < 2; ++i) { m[n][i] = -INFINITY; l[n][i] = 0.f; }
#pragma unroll
            for (int k = 0; k < C::TILES; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[k][n][i] = 0.f;
#pragma unroll
            for (int k = 0; k < GR; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) ones[k][n][i] = 0.f;
        }
        int vexp = -13;                           // value scales are taken in units of 2^(vexp - 14)
        bool any = false;

        // The warp's pages of the segment, counted from the segment's first.
        const int in_end = (int)(end - s.start), step = C::MANY && team != 0 ? team : W;
#pragma unroll 1
        for (int in = C::MANY && team != 0 ? member : (int)(p0 + warp + (int64_t)used * W - s.start); in < in_end; in += step) {
            any = true;
            const int st = (int)(used % S);
            const uint32_t stage = sbase + (warp * S + st) * C::BLOB;
            if (ok && !warp_wait(sbase + C::BARS + 8 * (warp * S + st), (uint32_t)(used / S) & 1u, abort_addr)) {
                if (lane == 0) raise_abort(&misc->abort);
                ok = false;
            }
            ++used;
            if (!ok) break;
            landed = used;
            const int key0 = (page0 + in) * KV_PAGE;
            float sc[4][NT][4];
            uint32_t vs[4][2][(GR + 1) / 2];      // the value scales of the lane's two keys, in pairs of groups
#pragma unroll
            for (int sub = 0; sub < 4; ++sub) {
                uint32_t k0[KW], k1[KW], sw0[GR], sw1[GR];               // keys g and g + 8 (in row order), their scales
                const uint32_t krow = stage + sub * 8 * D + klane, srow = stage + sub * D + slane;
                lds_words<KW>(k0, krow);
                lds_words<KW>(k1, krow + 4 * D);
                lds_words<GR>(sw0, srow);
                lds_words<GR>(sw1, srow + D / 2);
                const __half* s0 = reinterpret_cast<const __half*>(sw0);
                const __half* s1 = reinterpret_cast<const __half*>(sw1);
#pragma unroll
                for (int q = 0; q < GR; ++q) {
                    float d[NT][4];
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        d[n][0] = d[n][2] = corr[n][q][0];
                        d[n][1] = d[n][3] = corr[n][q][1];
                    }
#pragma unroll
                    for (int j = 2 * q; j < 2 * q + 2; ++j) {
                        const uint32_t x0 = k0[j], x1 = k1[j], y0 = prmt(x0, 0, 0x2301), y1 = prmt(x1, 0, 0x2301);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            mma(d[n], x0 & LOW, x1 & LOW, x0 & HIGH, x1 & HIGH, qb[n][j][0], qb[n][j][1]);
                            mma(d[n], y0 & LOW, y1 & LOW, y0 & HIGH, y1 & HIGH, qb[n][j][2], qb[n][j][3]);
                        }
                    }
                    const float e0 = __half2float(s0[q]), e1 = __half2float(s1[q]);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            sc[sub][n][i] = q == 0 ? d[n][i] * (i < 2 ? e0 : e1) : fmaf(d[n][i], i < 2 ? e0 : e1, sc[sub][n][i]);
                }
                if constexpr (GR == 1) {          // key scale, value scale
                    vs[sub][0][0] = sw0[0] >> 16;
                    vs[sub][1][0] = sw1[0] >> 16;
                } else {
#pragma unroll
                    for (int q = 0; q < GR / 2; ++q) {
                        vs[sub][0][q] = sw0[GR / 2 + q];
                        vs[sub][1][q] = sw1[GR / 2 + q];
                    }
                }
            }
            if constexpr (C::HALVES) {            // the keys' half is read
                __syncwarp();
                issue();
            }
            if (key0 + KV_PAGE - 1 > close || key0 <= open) {            // some row does not attend to all of the page
                uint32_t seen = 0;                // bit 2 sub + x: a row attends to the lane's key
#pragma unroll
                for (int sub = 0; sub < 4; ++sub)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int key = key0 + sub * 16 + (g >> 1) + (g & 1) * 4 + 8 * x;
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                if (key > pos[n][i] || (a.window > 0 && key <= pos[n][i] - a.window))
                                    sc[sub][n][2 * x + i] = -INFINITY;
                                else
                                    seen |= 1u << (2 * sub + x);
                            }
                    }
                // A key that no row attends to (after the last, before a window, between two) may never have been
                // written: a probability of 0 times a scale that is NaN would be NaN, and a large one would raise vexp.
                seen |= __shfl_xor_sync(FULL, seen, 1);
                seen |= __shfl_xor_sync(FULL, seen, 2);
#pragma unroll
                for (int sub = 0; sub < 4; ++sub)
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        if (!(seen >> (2 * sub + x) & 1))
#pragma unroll
                            for (int q = 0; q < (GR + 1) / 2; ++q) vs[sub][x][q] = 0;
            }

            // Running maximum per row, running power of two of the value scales.
            __half2 vtop = *reinterpret_cast<const __half2*>(&vs[0][0][0]);
#pragma unroll
            for (int sub = 0; sub < 4; ++sub)
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int q = 0; q < (GR + 1) / 2; ++q) vtop = __hmax2(vtop, *reinterpret_cast<const __half2*>(&vs[sub][x][q]));
            const uint32_t vb = __reduce_max_sync(
                FULL, max((uint32_t)__half_as_ushort(__low2half(vtop)), (uint32_t)__half_as_ushort(__high2half(vtop))));
            const int vnew = max(vexp, max((int)(vb >> 10), 1) - 14);    // scales below 2^vnew
            bool moved = vnew != vexp;
            float mnew[NT][2], mu[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float x = fmaxf(sc[0][n][i], sc[0][n][i + 2]);
#pragma unroll
                    for (int sub = 1; sub < 4; ++sub) x = fmaxf(x, fmaxf(sc[sub][n][i], sc[sub][n][i + 2]));
                    x = fmaxf(x, __shfl_xor_sync(FULL, x, 4));
                    x = fmaxf(x, __shfl_xor_sync(FULL, x, 8));
                    x = fmaxf(x, __shfl_xor_sync(FULL, x, 16));
                    x = fmaxf(x * f[n][i], m[n][i]);
                    mnew[n][i] = x;
                    mu[n][i] = x == -INFINITY ? 0.f : x;
                    moved |= x != m[n][i];
                }
            if (__any_sync(FULL, moved)) {
                const float shrink = pow2(vexp - vnew);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float fac[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        fac[i] = ex2(m[n][i] - mu[n][i]);
                        l[n][i] *= fac[i];
                        fac[i] *= shrink;
                        m[n][i] = mnew[n][i];
                    }
#pragma unroll
                    for (int k = 0; k < C::TILES; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[k][n][i] *= fac[i & 1];
#pragma unroll
                    for (int k = 0; k < GR; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) ones[k][n][i] *= fac[i & 1];
                }
                vexp = vnew;
            }
            const float vup = pow2(14 - vexp);

            if constexpr (C::HALVES) {
                if (!warp_wait(sbase + C::VBARS + 8 * (warp * S + st), (uint32_t)((used - 1) / S) & 1u, abort_addr)) {
                    if (lane == 0) raise_abort(&misc->abort);
                    ok = false;
                    break;
                }
                v_landed = used;
            }
#pragma unroll
            for (int sub = 0; sub < 4; ++sub) {
                uint32_t vw[4][GR];
                const uint32_t vrow = stage + sub * 8 * D + vlane;
#pragma unroll
                for (int j = 0; j < 4; ++j) lds_words<GR>(vw[j], vrow + j * 2 * D);
                float pr[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) pr[n][i] = ex2(fmaf(sc[sub][n][i], f[n][i & 1], -mu[n][i & 1]));
                    l[n][0] += pr[n][0] + pr[n][2];
                    l[n][1] += pr[n][1] + pr[n][3];
                }
#pragma unroll
                for (int q = 0; q < GR; ++q) {
                    const float e0 = __half2float(reinterpret_cast<const __half*>(vs[sub][0])[q]) * vup,
                                e1 = __half2float(reinterpret_cast<const __half*>(vs[sub][1])[q]) * vup;
                    uint32_t b0[NT], b1[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        b0[n] = transposed(half2_bits(pr[n][0] * e0, pr[n][1] * e0));
                        b1[n] = transposed(half2_bits(pr[n][2] * e1, pr[n][3] * e1));
                    }
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {                     // dimensions 0..3 and 4..7 of the words
                        // codes 0, 1 and (bytes swapped) 2, 3 of the half: two keys' side by side
                        const uint32_t sel = hf ? 0x7632u : 0x5410u, swp = hf ? 0x6723u : 0x4501u;
                        const uint32_t x0 = prmt(vw[0][q], vw[1][q], sel), x2 = prmt(vw[2][q], vw[3][q], sel);
                        const uint32_t y0 = prmt(vw[0][q], vw[1][q], swp), y2 = prmt(vw[2][q], vw[3][q], swp);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            mma(acc[4 * q + 2 * hf][n], x0 << 4 & HIGH, y0 << 4 & HIGH, x2 << 4 & HIGH, y2 << 4 & HIGH,
                                b0[n], b1[n]);
                            mma(acc[4 * q + 2 * hf + 1][n], x0 & HIGH, y0 & HIGH, x2 & HIGH, y2 & HIGH, b0[n], b1[n]);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        mma(ones[q][n], 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, b0[n], b1[n]);
                }
            }
            if (in + step < in_end) {             // refill the stage; the last of the segment is still needed
                __syncwarp();
                refill();
            }
        }

        // The warp's part of the segment, into the stage it has just read.
        if (!any && lane == 0) kept_in[warp] = -1;
        if (any) {
            const int st = (int)((used - 1) % S);
            float4* buf = reinterpret_cast<float4*>(smem + (warp * S + st) * C::BLOB + C::KEPT);
            const float down = pow2(vexp - 14);
            __syncwarp();
#pragma unroll
            for (int k = 0; k < C::TILES; k += 2)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int par = 0; par < 2; ++par) {
                        // dimensions 8 g + 0..3 of a group from tiles 4 q and 4 q + 1, 4..7 from the next two
                        const float z = 8.f * ones[k / 4][n][par];
                        buf[((k / 2 * NT + n) * 2 + par) * 32 + lane] =
                            make_float4((acc[k][n][par] * 0x1p18f - z) * down, (acc[k + 1][n][par] * 0x1p18f - z) * down,
                                        (acc[k][n][2 + par] * 0x1p18f - z) * down, (acc[k + 1][n][2 + par] * 0x1p18f - z) * down);
                    }
            if (lane == 0) kept_in[warp] = (warp * S + st) * C::BLOB + C::KEPT;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float x = l[n][i];
                x += __shfl_xor_sync(FULL, x, 4);
                x += __shfl_xor_sync(FULL, x, 8);
                x += __shfl_xor_sync(FULL, x, 16);
                if (g == 0) ml[warp * C::ROWS + 8 * n + 2 * t4 + i] = make_float2(m[n][i], x);
            }
        const auto store = [&](int r, int dim, float4 v, float sum) {
            const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;        // no keys: zeros; NaN stays
            const __nv_bfloat162 x = __floats2bfloat162_rn(v.x * inv, v.y * inv), y = __floats2bfloat162_rn(v.z * inv, v.w * inv);
            *reinterpret_cast<uint2*>(a.out + (((int64_t)s.b * a.rows + r / group) * a.heads + s.h * group + r % group) * D + dim) =
                make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
        };
        if constexpr (C::MANY)
            if (team != 0) {
                // Join the team: each thread the whole sum of a unit of 4 neighbouring dimensions.
                const auto meet = [&] {
                    if (team == 1) __syncwarp();
                    else asm volatile("bar.sync %0, %1;" :: "r"(1 + warp / team), "r"(32 * team) : "memory");
                };
                meet();
                const int w0 = warp - member;
#pragma unroll 1
                for (int u = 32 * member + lane; u < C::UNITS; u += 32 * team) {
                    const int par = u >> 5 & 1, n = (u >> 6) % NT, qh = (u >> 6) / NT;
                    const int row = 8 * n + 2 * (lane & 3) + par, r = s.rt * C::ROWS + row;
                    if (r >= rows_all) continue;
                    float mx = -INFINITY, sum = 0.f;
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
                    for (int w = w0; w < w0 + team; ++w) mx = fmaxf(mx, ml[w * C::ROWS + row].x);
#pragma unroll 1
                    for (int w = w0; w < w0 + team; ++w) {
                        const float2 x = ml[w * C::ROWS + row];
                        if (x.y == 0.f) continue;                        // no keys: its vector may be anything
                        const float fw = ex2(x.x - mx);
                        const float4 y = reinterpret_cast<const float4*>(smem + kept_in[w])[u];
                        sum = fmaf(x.y, fw, sum);
                        v.x = fmaf(y.x, fw, v.x);
                        v.y = fmaf(y.y, fw, v.y);
                        v.z = fmaf(y.z, fw, v.z);
                        v.w = fmaf(y.w, fw, v.w);
                    }
                    store(r, 64 * (qh >> 1) + 8 * (lane >> 2) + 4 * (qh & 1), v, sum);
                }
                meet();
                if (any) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    refill();
                }
                continue;
            }
        __syncthreads();

        // Join the warps: first each warp's factor per row (16 lanes a row), then the rows, by units of 4 neighbouring
        // dimensions.
        {
            const int row = (tid >> 4) % C::ROWS, w = tid & 15;
            float2 x = ml[min(w, W - 1) * C::ROWS + row];
            if (w >= W) x = make_float2(-INFINITY, 0.f);
            float mx = x.x;
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, o));
            const float fw = x.y == 0.f ? 0.f : ex2(x.x - mx);
            float sum = x.y == 0.f ? 0.f : x.y * fw;
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) sum += __shfl_xor_sync(FULL, sum, o);
            if (tid < 16 * C::ROWS && w < W) factor[w * C::ROWS + row] = fw;
            if (tid < 16 * C::ROWS && w == 0) joined[row] = make_float2(mx, sum);
            // a warp without pages: another's values, times 0
            const int at = w < W ? kept_in[w] : -1, some = __reduce_max_sync(FULL, at);
            __syncthreads();
            if (tid < W && at < 0) kept_in[w] = some;
        }
        __syncthreads();
        const bool whole = s.start >= cur && s.start + s.pages <= end;
        const int64_t slot = aligned ? (int64_t)blockIdx.x : 2 * (int64_t)blockIdx.x + (s.start <= p0 ? 0 : 1);
#pragma unroll 1
        for (int u = tid; u < C::UNITS; u += C::THREADS) {
            const int ln = u & 31, par = u >> 5 & 1, n = (u >> 6) % NT, qh = (u >> 6) / NT;
            const int row = 8 * n + 2 * (ln & 3) + par, dim = 64 * (qh >> 1) + 8 * (ln >> 2) + 4 * (qh & 1);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float fw = factor[w * C::ROWS + row];
                const float4 y = reinterpret_cast<const float4*>(smem + kept_in[w])[u];
                v.x = fmaf(y.x, fw, v.x);
                v.y = fmaf(y.y, fw, v.y);
                v.z = fmaf(y.z, fw, v.z);
                v.w = fmaf(y.w, fw, v.w);
            }
            if (!whole) {
                reinterpret_cast<float4*>(parts + slot * C::PART)[u] = v;
                if (qh == 0 && ln < 4) reinterpret_cast<float2*>(parts + slot * C::PART + C::ROWS * D)[row] = joined[row];
                continue;
            }
            const int r = s.rt * C::ROWS + row;
            if (r < rows_all) store(r, dim, v, joined[row].y);
        }
        if (!whole) {
            // The last of the segment's blocks joins their parts, in order.
            const int64_t b0 = aligned ? first_part : s.start / quantum;
            const int n_parts = aligned ? parts_here : (int)((s.start + s.pages - 1) / quantum - b0) + 1;
            __syncthreads();                      // the part is written: released by the count, acquired by its last adder
            if (tid == 0) misc->last = atom_add_acq_rel_gpu(&counts[s.index], 1u) == (uint32_t)(n_parts - 1);
            __syncthreads();
            if (misc->last) {
                if (tid == 0) counts[s.index] = 0;
                // By units of 4 dimensions. Where the rows that there are leave threads over, and no copy is in flight (a
                // block's one part), several threads to a unit share the parts: the loads are a chain of JOIN at a time.
                const int live = min(C::ROWS, rows_all - s.rt * C::ROWS), units = live * (D / 4);
                int shares = 1, each = n_parts;
                if (C::SHARED && aligned && 2 * units <= C::THREADS && n_parts > JOIN) {
                    shares = min(C::THREADS / units, (n_parts + JOIN - 1) / JOIN);
                    each = (n_parts + shares - 1) / shares;
                }
                float4* ov = reinterpret_cast<float4*>(smem);
                float2* om = reinterpret_cast<float2*>(smem + C::THREADS * 16);
#pragma unroll 1
                for (int i = tid; i < (C::SHARED && shares > 1 ? units * shares : C::UNITS); i += C::THREADS) {
                    int u = i, ka = 0;
                    if (C::SHARED && shares > 1) {
                        const int share = i / units, at = i - share * units, d4 = at / live, row = at - d4 * live;
                        u = (((2 * (d4 >> 4) + (d4 & 1)) * NT + (row >> 3)) * 2 + (row & 1)) * 32 + 4 * (d4 >> 1 & 7) + (row >> 1 & 3);
                        ka = share * each;
                    }
                    const int kb = C::SHARED ? min(ka + each, n_parts) : n_parts;
                    const int ln = u & 31, par = u >> 5 & 1, n = (u >> 6) % NT, qh = (u >> 6) / NT;
                    const int row = 8 * n + 2 * (ln & 3) + par, dim = 64 * (qh >> 1) + 8 * (ln >> 2) + 4 * (qh & 1);
                    const int r = s.rt * C::ROWS + row;
                    if (r >= rows_all) continue;
                    float mx = -INFINITY, sum = 0.f;
                    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
                    for (int k0 = ka; k0 < kb; k0 += JOIN) {             // JOIN parts' loads in flight
                        float2 x[JOIN];
                        float4 y[JOIN];
#pragma unroll
                        for (int j = 0; j < JOIN; ++j) {
                            const int64_t k = b0 + min(k0 + j, kb - 1);
                            const float* part = parts + (aligned ? k : 2 * k + (s.start <= k * quantum ? 0 : 1)) * C::PART;
                            x[j] = __ldcg(reinterpret_cast<const float2*>(part + C::ROWS * D) + row);
                            y[j] = __ldcg(reinterpret_cast<const float4*>(part) + u);
                            if (k0 + j >= kb) x[j] = make_float2(-INFINITY, 0.f);
                        }
                        float mn = mx;
#pragma unroll
                        for (int j = 0; j < JOIN; ++j) {
                            mn = fmaxf(mn, x[j].x);
                        }
                        const float f0 = sum == 0.f ? 0.f : ex2(mx - mn);
                        mx = mn;
                        sum *= f0;
                        o.x *= f0; o.y *= f0; o.z *= f0; o.w *= f0;
#pragma unroll
                        for (int j = 0; j < JOIN; ++j) {
                            if (x[j].y == 0.f) continue;                 // no keys: its vector may be anything
                            const float fj = ex2(x[j].x - mn);
                            sum = fmaf(x[j].y, fj, sum);
                            o.x = fmaf(y[j].x, fj, o.x); o.y = fmaf(y[j].y, fj, o.y);
                            o.z = fmaf(y[j].z, fj, o.z); o.w = fmaf(y[j].w, fj, o.w);
                        }
                    }
                    if (!C::SHARED || shares == 1) {
                        store(r, dim, o, sum);
                    } else {
                        ov[i] = o;
                        om[i] = make_float2(mx, sum);
                    }
                }
                if (C::SHARED && shares > 1) {
                    __syncthreads();
#pragma unroll 1
                    for (int at = tid; at < units; at += C::THREADS) {
                        float mx = -INFINITY, sum = 0.f;
                        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
                        for (int k = 0; k < shares; ++k) mx = fmaxf(mx, om[k * units + at].x);
#pragma unroll 1
                        for (int k = 0; k < shares; ++k) {
                            const float2 x = om[k * units + at];
                            if (x.y == 0.f) continue;
                            const float4 y = ov[k * units + at];
                            const float fk = ex2(x.x - mx);
                            sum = fmaf(x.y, fk, sum);
                            o.x = fmaf(y.x, fk, o.x); o.y = fmaf(y.y, fk, o.y);
                            o.z = fmaf(y.z, fk, o.z); o.w = fmaf(y.w, fk, o.w);
                        }
                        store(s.rt * C::ROWS + at % live, 4 * (at / live), o, sum);
                    }
                }
            }
        }
        __syncthreads();                          // the parts are read: their stages may be filled again
        if (any) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            refill();
        }
        cur = end;
    }
    // A wait that ran out: let every copy land before the block's memory goes.
    if (!ok) {
#pragma unroll 1
        for (; landed < issued; ++landed)
            mbar_wait_bounded(sbase + C::BARS + 8 * (warp * S + (int)(landed % S)), (uint32_t)(landed / S) & 1u);
        if constexpr (C::HALVES)
#pragma unroll 1
            for (; v_landed < v_issued; ++v_landed)
                mbar_wait_bounded(sbase + C::VBARS + 8 * (warp * S + (int)(v_landed % S)), (uint32_t)(v_landed / S) & 1u);
    }
}

template <Kind KIND> using Shape64a = Shape<64, 1, 12, 4, false, KIND>;
template <Kind KIND> using Shape64b = Shape<64, 2, 12, 4, false, KIND>;
template <Kind KIND> using Shape128a = Shape<128, 1, 12, 2, false, KIND>;
template <Kind KIND> using Shape128b = Shape<128, 2, 8, 3, false, KIND>;
template <Kind KIND> using Shape256a = Shape<256, 1, 8, 1, true, KIND>;

// Query rows per pass: 16 where there are more than 8 (the registers for 16
// rows of 256 dimensions are not there). At 128 dimensions 5 passes of 8 cost
// what 3 of 16 do, and start and join sooner: 24 rows in 3 passes of 8 take 52.8
// us where 2 of 16 take 52.5 (8 x 8000 keys, 8 key heads) and 8.6 where they take
// 11.0 (2000 keys, 4 key heads); 40 rows 77.1 and 76.9, 8.8 and 11.2; but 16 rows
// in 2 of 8 take 37.4 where one of 16 takes 30.9. At 64 dimensions a pass of 16
// is always cheaper (24 rows: 35.1 against 37.3).
int tile_rows(int rows, int head_dim) {
    const int by8 = (rows + 7) / 8, by16 = (rows + 15) / 16;
    return by8 == 1 || head_dim > 128 || (head_dim == 128 && 3 * by8 <= 5 * by16) ? 8 : 16;
}

// The same for every shape, so that a workspace's counts do not move between calls.
size_t parts_bytes(int sms) {
    constexpr size_t most = std::max(Shape128b<PLAIN>::PART, Shape256a<PLAIN>::PART);
    return (2 * (size_t)sms * most * sizeof(float) + 255) / 256 * 256;
}

template <class C>
cudaError_t launch_shape(const KvView& c, const KvAttend& a, int row_tiles, cudaStream_t s) {
    static LaunchPrep prep;
    int sms = 0;
    const cudaError_t e = prep.get(kv_attend_kernel<C>, C::SMEM, &sms);
    if (e != cudaSuccess) return e;
    uint32_t* counts = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.workspace) + parts_bytes(sms));
    return launch_dependent(kv_attend_kernel<C>, dim3(sms), C::THREADS, C::SMEM, s, c, a, row_tiles, counts,
                            static_cast<float*>(a.workspace));
}

// TEAMS where there may be more segments than blocks. SHARES where a segment may be cut into more than 2 JOIN parts and
// its rows leave half of the threads over that join them. The code of either costs the others' loop over the pages 2 to 4%
// (registers), and 0.5 us of instructions that come cold between the other kernels of a decode step (12 layers: 387
// against 378 us a step), so each is a kernel of its own. 32768 keys, 4 heads of 128 over 1: 12.2 us (13.4 without SHARES), 1 over
// 1: 11.3 (13.5), 8 of 64 over 1: 9.9 (10.8); 54384 keys of 2 sequences, 6 heads of 256 over 3: 28.4 (32.5). Without TEAMS: above.
template <template <Kind> class C>
cudaError_t launch(const KvView& c, const KvAttend& a, int row_tiles, cudaStream_t s) {
    int sms = 0;
    const int e = device_sms(&sms);
    if (e != 0) return (cudaError_t)e;
    const int64_t segments = (int64_t)a.batch * c.kv_heads * row_tiles;
    const int rows = std::min(a.heads / c.kv_heads * a.rows, +C<PLAIN>::ROWS);
    if (segments > sms) return launch_shape<C<TEAMS>>(c, a, row_tiles, s);
    using P = C<PLAIN>;
    if constexpr (2 * (P::ROWS - 7) * (P::D / 4) <= P::THREADS)          // for the fewest rows that take this shape
        if (segments * 2 * JOIN < sms && c.table_pages > 2 * JOIN * CUT && 2 * rows * (P::D / 4) <= P::THREADS)
            return launch_shape<C<SHARES>>(c, a, row_tiles, s);
    return launch_shape<C<PLAIN>>(c, a, row_tiles, s);
}

}  // namespace

// Two partial results per block (its first and its last segment), then a count
// per segment.
size_t kv_workspace_bytes(int batch, int rows, int heads, int kv_heads, int sms) {
    const int64_t rows_all = (int64_t)(heads / kv_heads) * rows;
    const int64_t tiles = (rows_all + 7) / 8;
    return parts_bytes(sms) + (size_t)batch * (size_t)kv_heads * (size_t)tiles * sizeof(uint32_t) + 256;
}

cudaError_t launch_kv_attend(const KvView& c, const KvAttend& a, cudaStream_t s) {
    const int rows_all = a.heads / c.kv_heads * a.rows, tile = tile_rows(rows_all, c.head_dim);
    const int tiles = (rows_all + tile - 1) / tile;
    if (c.head_dim == 256) return launch<Shape256a>(c, a, tiles, s);
    if (c.head_dim == 128) return tile == 16 ? launch<Shape128b>(c, a, tiles, s) : launch<Shape128a>(c, a, tiles, s);
    return tile == 16 ? launch<Shape64b>(c, a, tiles, s) : launch<Shape64a>(c, a, tiles, s);
}

cudaError_t read_device_status_attend(uint32_t* status) {
    cudaError_t e = cudaMemcpyFromSymbol(status, g_device_status, sizeof(uint32_t));
    if (e != cudaSuccess || *status == 0) return e;
    const uint32_t zero = 0;
    return cudaMemcpyToSymbol(g_device_status, &zero, sizeof(uint32_t));
}

}  // namespace vbq
