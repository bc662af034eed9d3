// vbq_delta_chunk.cu — the gated delta rule over prompts, 64 tokens at a time on
// the tensor cores.
//
// With G_i the sum of a chunk's log decays up to its token i, S the state before
// the chunk and k, q the unit keys and (scaled) queries, the tokens' corrections
// solve a unit lower triangular system, (1 + L) U = R,
//   R_i = beta_i (v_i - e^G_i S^T k_i),   L_ij = beta_i e^(G_i - G_j) k_i.k_j  (j < i),
// and with T = (1 + L)^-1
//   U = T R,   o_i = e^G_i S^T q_i + sum_(j <= i) e^(G_i - G_j) (q_i.k_j) U_j,
//   S <- e^G_last S + sum_j e^(G_last - G_j) k_j U_j^T.
// Only R, U, o and the new state depend on the state; T and the scores do not.
//
// The chunks are a chain, and the columns of S do not meet. So a block takes one
// sequence, one head and 16 columns for each of its chain warps, and a chain warp
// holds S^T for its 16 columns in the accumulators of m16n8k16 (columns x head_k)
// over the whole sequence. Everything is computed transposed: what comes out of one
// product is, in the same registers, the A operand of the next, so the chain has no
// exchange between warps and nothing but key, query, T and score fragments is read
// from shared memory. Where there are two chain warps, two more make the outputs,
// from the parts of S and U that they are handed (when it was added, 2.30 -> 2.16
// ms for 32768 tokens). Eight other warps prepare the next chunk meanwhile, in two
// groups that work side by side. The one for queries takes keys and queries to
// FP16, multiplies queries with keys, makes the scores and goes on to the next
// chunk's rows; the one for keys multiplies keys with keys and makes T: blocks of
// 16 on the diagonal by substitution in fp32, the ones below them by products.
// Named barriers hand the stages over.
//
// What bounds it is neither memory nor the tensor cores (39% busy) but the chain of
// instructions a chunk takes: 15.6 thousand of twelve warps, 0.43 an issue slot,
// each waiting for the one before it or for another group. Two blocks do not
// fit in the registers of an SM. The code of both roles is twice the 32 KB that
// an SM keeps of it, so what a chunk does not need twice is not written out
// twice: loops are rolled wherever registers need no index. One sequence of 32768
// tokens, 32 heads of 128 by 128, blocks of 32 columns: 2.29 ms, 4.5 us a chunk
// (before the outputs took both parts of their operands 4.2, and with three of four
// chunks not prepared 3.4); memory needs 0.12 ms of it.
//
// fp32 through the tensor cores. BF16 keys and queries are taken to FP16 by a power
// of two a token, which they survive unchanged (8 bits of 11) down to 2^-31 of
// their token's largest; S, R, U, T and the scores enter as two FP16 parts, x = hi
// + lo, with a power of two per column of S (the scores: per row), so a product is
// good to 2^-22 (fp32 keys and queries, with a power of two a token, are two parts
// as well). That holds for the outputs too, which are rounded once: with one part
// (2^-11) of S, U, the scores and fp32 queries they were off by many steps of BF16
// where terms cancel (32768 tokens in 2.16 ms against 2.28, five prompts in 515 us
// against 555). A power of two for the rows of a warp together instead of one a
// token cost tokens their digits beside larger ones, and saved 1%. T and L are up
// by 2^10, so that what a strong decay leaves of an earlier token's R keeps its
// digits (parts end at 2^-35, not 2^-25, which had an element of 2e-5 off by 2e-8);
// they overflow from 64 on, and where the rule contracts |T_ij| is at most |beta_i|
// |k_i| |k_j|, 2 for keys of unit length.
//
// NaN and infinities must not reach earlier tokens through the zeros above the
// diagonal: a column whose R is not finite at some token is computed without it
// and gets NaN from that token on.
#include <type_traits>
#include <cuda_fp16.h>

#include "vbq_delta.cuh"
#include "vbq_kernels.h"

namespace vbq {
namespace {

constexpr int CH = 64;                           // tokens of a chunk
constexpr int STAGES = 2;
constexpr float T_UP = 1024.f;                   // T and L in FP16 parts are up by this: see above
constexpr int DP = 20;                           // floats between rows of an fp32 block of 16 x 16

__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" :: "r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int threads) { asm volatile("bar.arrive %0, %1;" :: "r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
// a at p and b eight values on; no branch, which the compiler would follow up with copies of what comes after
__device__ __forceinline__ void store_if(uint16_t* p, uint32_t a, uint32_t b, bool take) {
    asm volatile("{.reg .pred t; setp.ne.u32 t, %3, 0; @t st.global.b32 [%0], %1; @t st.global.b32 [%0 + 16], %2;}" :: "l"(p), "r"(a), "r"(b), "r"((uint32_t)take) : "memory");
}
__device__ __forceinline__ void stmatrix4_trans(uint32_t addr, const uint32_t (&r)[4]) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" :: "r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the first of a sum: c = a b if `first`, else c += a b
__device__ __forceinline__ void mma_from(bool first, float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (!first) return mma(c, a, b0, b1);
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ float exp2_fast(float x) {              // 2 ulps; below 2^-126: 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 16 bytes to shared memory, zeros where `take` is false.
__device__ __forceinline__ void cp_16(uint32_t dst, const void* src, bool take) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(take ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void cp_wait_but_one() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }
__device__ __forceinline__ void cp_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 twice(float x) { return make_float2(x, x); }
// max(m, |x|, |y|); a NaN stays
__device__ __forceinline__ float max_of(float m, float x, float y) {
    asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(fabsf(x)), "f"(fabsf(y)));
    return m;
}
// (x, y) as FP16 parts: hi, and what it leaves (x - hi, an exact difference, by the multiply-add that takes FP16 factors)
__device__ __forceinline__ void split2(float x, float y, uint32_t& hi, uint32_t& lo) {
    hi = pack_f16(x, y);
    asm("{.reg .b16 h, l, m; mov.b32 {l, h}, %2; mov.b16 m, 0xbc00; fma.rn.f32.f16 %0, l, m, %0; fma.rn.f32.f16 %1, h, m, %1;}" : "+f"(x), "+f"(y) : "r"(hi));
    lo = pack_f16(x, y);
}
__device__ __forceinline__ void split2(float2 x, uint32_t& hi, uint32_t& lo) { split2(x.x, x.y, hi, lo); }
// Two neighbouring tiles of 8 columns as A fragments, scaled by row: FP16 parts.
__device__ __forceinline__ void split_a(const float (&x)[4], const float (&y)[4], float s0, float s1, uint32_t (&hi)[4], uint32_t (&lo)[4]) {
    split2(mul2(make_float2(x[0], x[1]), twice(s0)), hi[0], lo[0]);
    split2(mul2(make_float2(x[2], x[3]), twice(s1)), hi[1], lo[1]);
    split2(mul2(make_float2(y[0], y[1]), twice(s0)), hi[2], lo[2]);
    split2(mul2(make_float2(y[2], y[3]), twice(s1)), hi[3], lo[3]);
}
// The power of two that takes a magnitude m to 2^14 .. 2^15 (at most 2^100), and its inverse.
__device__ __forceinline__ float to_f16_range(float m) {
    const uint32_t f = 268u - (__float_as_uint(m) >> 23);
    return __uint_as_float((f > 227u ? 227u : f) << 23);
}
__device__ __forceinline__ float pow2_inverse(float p) { return __uint_as_float((254u << 23) - __float_as_uint(p)); }
__device__ __forceinline__ float quad_max(float m) {              // over the four lanes of a fragment's row
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
    return fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
}

// Byte offset of 16-byte segment `seg` of row `row` in a tile of PITCH-byte rows; eight rows' segments fall in distinct banks.
template <int PITCH>
__device__ __forceinline__ uint32_t tile_at(int row, int seg) {
    return (uint32_t)(row * PITCH + ((seg ^ (row & 7)) << 4));
}

// what the gates of a chunk come to, per token: log2 of the decay from the chunk's start (and what a float of it leaves out),
// the factor of its correction, the decay from it to the end of its 16 tokens
enum { G_HI, G_LO, G_BETA, G_BLOCK };
constexpr int GATES = 4 * CH;

// The same in a tile of two segments a row.
__device__ __forceinline__ uint32_t beside_at(int row, int seg) { return (uint32_t)(32 * row + ((seg ^ ((row >> 2) & 1)) << 4)); }

template <bool F32, int DK, int CW>
struct Shape {
    static constexpr int VC = 16 * CW;                              // columns of a block
    // Bytes of a row of keys in FP16 and of values, 16 more than they hold, so that eight rows' segments fall in distinct
    // banks (fp32 keys: turned by row instead, for want of room).
    static constexpr int KP = 2 * DK + (F32 ? 0 : 16), VP = F32 ? 4 * (VC + 4) : 2 * VC + 16;
    static constexpr int TP = 2 * CH;                               // bytes of a row of T, the scores and L
    static constexpr int CHAIN = 128;                               // a whole warpgroup
    static constexpr int HALF = 128, PREP = 2 * HALF, THREADS = CHAIN + PREP;     // warps for keys, for queries
    // a stage: keys and queries (fp32 ones: the two parts of each, where their raw values land), values, T in two parts (below the
    // diagonal -L, until T takes its place, but for two blocks), scores in two parts, factors
    static constexpr int K = 0, KLO = K + CH * KP, Q = KLO + (F32 ? CH * KP : 0), QLO = Q + CH * KP, V = QLO + (F32 ? CH * KP : 0),
                         THI = (V + CH * VP + 127) / 128 * 128, TLO = THI + CH * TP, P = TLO + CH * TP, PLO = P + CH * TP, FAC = PLO + CH * TP,
                         STAGE = (FAC + (5 * CH + 4) * 4 + 127) / 128 * 128;
    // scratch of the preparing warps: -L's blocks (2, 1) and (3, 1) in FP16 parts, which are still read when T's are written; its
    // blocks on the diagonal in fp32; factors of two chunks; the next chunk's BF16 keys and queries as they come
    static constexpr int BESIDE = 0, PART = 32 * 32, DIAG = BESIDE + 2 * PART, TOKENS = DIAG + 4 * 16 * DP * 4, FACTORS = 2 * CH + GATES, RAW = TOKENS + 2 * FACTORS * 4,
                         SCRATCH = RAW + (F32 ? 0 : 2 * CH * 2 * DK);
    static constexpr int OWN = STAGES * STAGE;
    // Two chain warps leave two of their warpgroup to the outputs (fp32 heads of 128 have no room left to hand things over). What
    // they are handed, each lane by the one at its place: the parts of S and U, their scales, where a column is lost.
    static constexpr bool APART = CW == 2 && !(F32 && DK == 128);
    static constexpr int HANDED = (OWN + SCRATCH + 127) / 128 * 128, HAND_U = DK / 16 * 1024, HAND_SCALES = HAND_U + 4 * 1024, HAND = HAND_SCALES + 3 * 256,
                         BYTES = HANDED + (APART ? CW * HAND : 0);
    static_assert(RAW % 16 == 0);
    // named barriers
    static constexpr int FULL = 1, EMPTY = FULL + STAGES, PREPARING = EMPTY + STAGES, KEYS = PREPARING + 1, S_READY = KEYS + 1, U_READY = S_READY + CW, TAKEN = U_READY + CW;
    static constexpr int CONSUMERS = 32 * CW * (APART ? 2 : 1), FULL_COUNT = CONSUMERS + PREP, EMPTY_COUNT = CONSUMERS + HALF;
    __device__ static __forceinline__ uint32_t key_at(int row, int seg) {
        return F32 ? tile_at<2 * DK>(row, seg) : (uint32_t)(row * KP + seg * 16);
    }
};
// what a stage tells about its tokens
enum { F_BETA, F_STATE, F_END, F_QUERY, F_SCORE };                  // and from F_LAST on: e^G_last
constexpr int F_LAST = 5 * CH;

// ---------------------------------------------------------------------------
// Preparing the chunks: a group of four warps for keys and one for queries. Loops are kept rolled where registers allow: the
// code of both roles has to stay near the instruction cache's size.
// ---------------------------------------------------------------------------

// The power of two for a row of this sum of squares: its largest value comes to at most 2^15, and to 2^10 at least (128
// values); a sum that underflows (values below 2^-60 or so) gives 2^60.
__device__ __forceinline__ float row_scale(float squares) {
    const int e = (int)(__float_as_uint(squares) >> 23) - 127;      // the norm is below 2^((e + 2) >> 1)
    const int up = 15 - ((e + 2) >> 1);
    return __uint_as_float((uint32_t)((up > 60 ? 60 : up) + 127) << 23);
}

// Sums of log2 decays in fixed point, 32 bits of fraction, as magnitudes: a decay of e^-100 among slow ones would cost the
// others their digits in fp32 (and 64-bit floating point runs at a 64th of the rate here).
__device__ __forceinline__ uint64_t to_fixed(float magnitude) {     // 0 .. 2^31
    const float n = floorf(magnitude);
    return ((uint64_t)(uint32_t)n << 32) + __float2uint_rz((magnitude - n) * 4294967296.f);
}
__device__ __forceinline__ float2 from_fixed(uint64_t x) {          // minus x, as a float and the rest
    const float n = (float)(uint32_t)(x >> 32), f = (float)(uint32_t)x * 2.3283064365386963e-10f, hi = n + f;
    return make_float2(-hi, (hi - n) - f);
}

template <bool F32, int DK, int CW>
__device__ __forceinline__ void prepare_chunks(const Delta& d, const SeqRange& r, int h, int col0, char* smem, uint32_t base, int chunks) {
    using Z = Shape<F32, DK, CW>;
    constexpr int PREP = Z::PREP, SEGS = DK / 8, STEP = Z::HALF / SEGS;       // of a warp for queries: 8 values a thread, STEP rows at once
    const int tid = threadIdx.x - Z::CHAIN, warp = tid >> 5 & 3, lane = tid & 31;
    const bool of_q = tid >= Z::HALF;
    const int hk = h / (d.heads / d.k_heads);
    const bool raw = d.a_log != nullptr;
    const float rate = raw ? expf(d.a_log[h]) : 0.f, bias = raw ? d.dt_bias[h] : 0.f;
    char* own = smem + Z::OWN;
    const uint32_t own_b = base + Z::OWN;
    float* diag = reinterpret_cast<float*>(own + Z::DIAG);
    const int seg = tid % SEGS, row_in = tid % Z::HALF / SEGS;
    const int quad = lane & 3, r8 = lane >> 2;
    const int b_row = (lane & 7) + ((lane >> 4) << 3), b_seg = (lane >> 3) & 1;      // B fragments of two tiles; A, transposed
    const int a_row = lane & 15, a_seg = lane >> 4;

    // BF16 keys and queries as they come, each piece to where its thread looks for it; zeros behind the end.
    const auto load_raw = [&](int c) {                              // (the group for queries)
        const int live = min(CH, r.n - c * CH);
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            const int64_t stride = half ? d.q_stride : d.k_stride;
            const uint16_t* p = static_cast<const uint16_t*>(half ? d.q : d.k) + ((int64_t)r.lo + (int64_t)c * CH + row_in) * stride + hk * DK + seg * 8;
            const uint32_t to = own_b + Z::RAW + half * CH * 2 * DK + tid % Z::HALF * 16;
#pragma unroll 2
            for (int i = 0; i < CH / STEP; ++i, p += STEP * stride) cp_16(to + i * Z::HALF * 16, row_in + i * STEP < live ? (const void*)p : d.q, row_in + i * STEP < live);
        }
    };
    // Values, and fp32 keys and queries, 16 bytes at a time straight into the stage.
    const auto load_values = [&](int c, uint32_t to) {
        constexpr int SIZE = F32 ? 4 : 2, PER = Z::VC * SIZE / 16;
        const int live = min(CH, r.n - c * CH);
        const int64_t stride = d.v_stride * SIZE;
        const char* v = static_cast<const char*>(d.v) + ((int64_t)r.lo + (int64_t)c * CH) * stride + (h * d.head_v + col0) * SIZE;
#pragma unroll 1
        for (int i = tid - Z::HALF; i < CH * PER; i += Z::HALF) {
            const int row = i / PER, part = i % PER;
            cp_16(to + row * Z::VP + part * 16, row < live ? v + row * stride + part * 16 : v, row < live);
        }
    };
    const auto load_pieces = [&](const void* from, int64_t stride, int c, uint32_t to, uint32_t more) {
        const int live = min(CH, r.n - c * CH);
        const float* p = static_cast<const float*>(from) + ((int64_t)r.lo + (int64_t)c * CH) * stride + hk * DK + seg * 8;
#pragma unroll 2
        for (int row = row_in; row < CH; row += STEP) {
            const float* q = row < live ? p + row * stride : p;
            cp_16(to + Z::key_at(row, seg), q, row < live);
            cp_16(more + Z::key_at(row, seg), q + 4, row < live);
        }
    };

    // A chunk's gates, two tokens a lane of a warp: as the call gives them, then what they come to.
    float ga[2] = {}, gb[2] = {};
    const auto load_gates = [&](int c) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int t = c * CH + 32 * e + lane;
            if (t < r.n) {
                ga[e] = gate_value(d.decay, d.gate_f32, ((int64_t)r.lo + t) * d.decay_stride + h);
                gb[e] = gate_value(d.beta, d.gate_f32, ((int64_t)r.lo + t) * d.beta_stride + h);
            }
        }
    };
    const auto sum_gates = [&](int c, float* gate) {
        constexpr float LOG2E = 1.44269504f;
        uint64_t before = 0;
        float nan = 0.f;                                            // a NaN decay makes NaNs of the sums that it is in
#pragma unroll 1
        for (int e = 0; e < 2; ++e) {
            const int t = 32 * e + lane;
            Gate x = gate_of(e ? ga[1] : ga[0], e ? gb[1] : gb[0], raw, rate, bias);
            if (t >= r.n - c * CH) x = {0.f, 0.f};
            uint64_t sum = to_fixed(-x.g * LOG2E);
#pragma unroll 1
            for (int o = 1; o < 32; o <<= 1) {
                const uint64_t y = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += y;
            }
            sum += before;
            before = __shfl_sync(0xffffffffu, sum, 31);
            const uint32_t odd = __ballot_sync(0xffffffffu, x.g != x.g);
            const float2 upto = from_fixed(sum);
            gate[G_HI * CH + t] = upto.x + nan + (odd & ((2u << lane) - 1) ? __int_as_float(0x7fffffff) : 0.f);
            gate[G_LO * CH + t] = upto.y;
            gate[G_BETA * CH + t] = x.beta;
            gate[G_BLOCK * CH + t] = exp2_fast(from_fixed(__shfl_sync(0xffffffffu, sum, lane | 15) - sum).x);
            if (odd) nan = __int_as_float(0x7fffffff);
        }
    };

    if (!F32 && of_q) load_raw(0);
    int first = -1;                                                 // a turn for the gates alone
    asm volatile("" : "+r"(first));                                 // unknown to the compiler, which would write that turn out on its own
#pragma unroll 1
    for (int c = first; c < chunks; ++c) {
        const int stage = c & (STAGES - 1), next = c + 1;
        char* st = smem + stage * Z::STAGE;
        const uint32_t sb = base + stage * Z::STAGE;
        float* fac = reinterpret_cast<float*>(st + Z::FAC);
        float *ck = reinterpret_cast<float*>(own + Z::TOKENS) + stage * Z::FACTORS, *cq = ck + CH, *gate = cq + CH;
        const bool gates = !of_q && warp == 3 && next < chunks;
        if (gates) load_gates(next);
        if (c >= 0) {
            if (of_q) {
                bar_sync(Z::EMPTY + stage, Z::EMPTY_COUNT);
                if constexpr (F32) {
                    load_pieces(d.k, d.k_stride, c, sb + Z::K, sb + Z::KLO);
                    load_pieces(d.q, d.q_stride, c, sb + Z::Q, sb + Z::QLO);
                }
                cp_wait_all();
                load_values(c, sb + Z::V);
                cp_commit();
                // keys and queries to FP16 by a power of two a row; what a row's unit length makes of them
                if constexpr (F32) {
#pragma unroll 1
                    for (int half = 0; half < 2; ++half) {          // in place: each piece by the thread that loaded it
                        char* tile = st + (half ? Z::Q : Z::K);
#pragma unroll 1
                        for (int row = row_in; row < CH; row += STEP) {
                            uint4 *at = reinterpret_cast<uint4*>(tile + Z::key_at(row, seg)),
                                  *more = reinterpret_cast<uint4*>(st + (half ? Z::QLO : Z::KLO) + Z::key_at(row, seg));
                            const uint4 x = *at, z = *more;
                            float y[8] = {__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w),
                                          __uint_as_float(z.x), __uint_as_float(z.y), __uint_as_float(z.z), __uint_as_float(z.w)};
                            float sum = 0.f;
#pragma unroll
                            for (int e = 0; e < 8; ++e) sum = fmaf(y[e], y[e], sum);
#pragma unroll
                            for (int o = SEGS / 2; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                            const float up = row_scale(sum);
                            if (seg == 0) (half ? cq : ck)[row] = (d.normalize ? rsqrtf(sum + DELTA_UNIT_EPS) : 1.f) * pow2_inverse(up);
                            uint32_t hi[4], lo[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) split2(y[2 * e] * up, y[2 * e + 1] * up, hi[e], lo[e]);
                            *at = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                            *more = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                        }
                    }
                } else {
                    // a power of two per row, by its largest magnitude: the others have no say in it (two rows' magnitudes in a word)
                    constexpr int ROWS = 4, TURNS = CH / STEP / ROWS;
#pragma unroll 1
                    for (int turn = 0; turn < 2 * TURNS; ++turn) {
                        const bool half = turn >= TURNS;
                        const int row = row_in + (turn - (half ? TURNS : 0)) * ROWS * STEP;
                        const uint4* from = reinterpret_cast<const uint4*>(own + Z::RAW) + turn * ROWS * Z::HALF + tid % Z::HALF;
                        uint4 x[ROWS];
#pragma unroll
                        for (int i = 0; i < ROWS; ++i) x[i] = from[i * Z::HALF];
                        constexpr uint32_t MAGNITUDES = 0x7fff7fffu;
                        uint32_t m[ROWS];
#pragma unroll
                        for (int i = 0; i < ROWS; ++i)
                            m[i] = __vmaxu2(__vmaxu2(x[i].x & MAGNITUDES, x[i].y & MAGNITUDES), __vmaxu2(x[i].z & MAGNITUDES, x[i].w & MAGNITUDES));
#pragma unroll
                        for (int i = 0; i < ROWS; i += 2) {
                            uint32_t both = __vmaxu2(__byte_perm(m[i], m[i + 1], 0x5410), __byte_perm(m[i], m[i + 1], 0x7632));
#pragma unroll
                            for (int o = SEGS / 2; o; o >>= 1) both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, o));
                            m[i] = both << 16;
                            m[i + 1] = both & 0xffff0000u;
                        }
                        char* to = st + (half ? Z::Q : Z::K) + Z::key_at(row, seg);
                        float* down = (half ? cq : ck) + row;
#pragma unroll
                        for (int i = 0; i < ROWS; ++i) {
                            const float up = to_f16_range(__uint_as_float(m[i]));
                            const auto two = [&](uint32_t w) { return pack_f16(__uint_as_float(w << 16) * up, __uint_as_float(w & 0xffff0000u) * up); };
                            *reinterpret_cast<uint4*>(to + i * STEP * Z::KP) = make_uint4(two(x[i].x), two(x[i].y), two(x[i].z), two(x[i].w));
                            if (seg == 0) down[i * STEP] = pow2_inverse(up);
                        }
                    }
                }
            }
            bar_sync(Z::PREPARING, PREP);
            // 16 rows of keys or of queries with the keys up to theirs
            {
                // The four parts of an SM take the warps in turn, so two chain warps leave two parts to the others: those get the
                // rows with most columns (balanced over keys and queries 1% more time for 32768 tokens). Four: balanced.
                const int mt = of_q && CW != 2 ? 3 - warp : warp;
                float acc[8][4];
#pragma unroll
                for (int n = 0; n < 8; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[n][e] = 0.f;
                float squares[2][4] = {};                           // the rows' own block, for its diagonal
                const uint32_t a_at = sb + (of_q ? Z::Q : Z::K), a_in = Z::key_at(16 * mt + a_row, a_seg), own_in = Z::key_at(16 * mt + b_row, b_seg),
                               b_in = Z::key_at(b_row, b_seg);
                if constexpr (F32) {
#pragma unroll 1
                    for (int kk = 0; kk < DK / 16; ++kk) {
                        uint32_t a[4], alo[4], b[4], l[4];
                        ldmatrix4(a, a_at + Z::key_at(16 * mt + a_row, 2 * kk + a_seg));
                        ldmatrix4(alo, sb + (of_q ? Z::QLO : Z::KLO) + Z::key_at(16 * mt + a_row, 2 * kk + a_seg));
#pragma unroll
                        for (int n2 = 0; n2 < 4; ++n2) {
                            if (n2 > mt) break;
                            ldmatrix4(b, sb + Z::K + Z::key_at(16 * n2 + b_row, 2 * kk + b_seg));
                            ldmatrix4(l, sb + Z::KLO + Z::key_at(16 * n2 + b_row, 2 * kk + b_seg));
                            mma(acc[2 * n2], a, b[0], b[1]);
                            mma(acc[2 * n2 + 1], a, b[2], b[3]);
                            mma(acc[2 * n2], alo, b[0], b[1]);
                            mma(acc[2 * n2 + 1], alo, b[2], b[3]);
                            mma(acc[2 * n2], a, l[0], l[1]);
                            mma(acc[2 * n2 + 1], a, l[2], l[3]);
                        }
                    }
                } else {
#pragma unroll 1
                    for (int kk = 0; kk < DK / 16; ++kk) {
                        uint32_t a[4], l[4], b[4][4];
                        ldmatrix4(a, a_at + a_in + 32 * kk);
                        if (of_q) ldmatrix4(l, a_at + own_in + 32 * kk);
#pragma unroll
                        for (int n2 = 0; n2 < 4; ++n2)
                            if (n2 <= mt) ldmatrix4(b[n2], sb + Z::K + b_in + 16 * n2 * Z::KP + 32 * kk);
                        if (of_q) {
                            mma(squares[0], a, l[0], l[1]);
                            mma(squares[1], a, l[2], l[3]);
                        }
#pragma unroll
                        for (int n2 = 0; n2 < 4; ++n2)
                            if (n2 <= mt) {
                                mma(acc[2 * n2], a, b[n2][0], b[n2][1]);
                                mma(acc[2 * n2 + 1], a, b[n2][2], b[n2][3]);
                            }
                    }
                }
                float own_acc[2][4];                                // the block on the diagonal
#pragma unroll
                for (int n2 = 0; n2 < 4; ++n2)
                    if (n2 == mt)
#pragma unroll
                        for (int p = 0; p < 2; ++p)
#pragma unroll
                            for (int e = 0; e < 4; ++e) own_acc[p][e] = acc[2 * n2 + p][e];
                if (!F32 && !of_q)
#pragma unroll
                    for (int p = 0; p < 2; ++p)
#pragma unroll
                        for (int e = 0; e < 4; ++e) squares[p][e] = own_acc[p][e];
                // the rows' factors, their unit lengths among them (BF16: from the diagonals, in the rows' own powers of two)
                if (2 * quad == (r8 & ~1)) {                        // columns 2 quad + e, rows r8 and r8 + 8
                    const bool e = r8 & 1;
                    const float x[2] = {e ? squares[0][1] : squares[0][0], e ? squares[1][3] : squares[1][2]};
                    const int row = 16 * mt + r8;
                    float* unit = (of_q ? cq : ck) + row;
                    float f[2], hi[2], lo[2], start[2];
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        f[p] = unit[8 * p];
                        if (!F32) f[p] *= d.normalize ? rsqrtf(x[p] * f[p] * f[p] + DELTA_UNIT_EPS) : 1.f;
                        hi[p] = gate[G_HI * CH + row + 8 * p];
                        lo[p] = gate[G_LO * CH + row + 8 * p];
                        start[p] = exp2_fast(hi[p] + lo[p]);
                        if (of_q) f[p] *= d.scale;
                        unit[8 * p] = f[p];
                    }
                    if (of_q) {
#pragma unroll
                        for (int p = 0; p < 2; ++p) fac[F_QUERY * CH + row + 8 * p] = start[p] * f[p];
                    } else {
                        const float end_hi = gate[G_HI * CH + CH - 1], end_lo = gate[G_LO * CH + CH - 1];
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            const float g = gate[G_BETA * CH + row + 8 * p];
                            fac[F_BETA * CH + row + 8 * p] = g;
                            fac[F_STATE * CH + row + 8 * p] = g * start[p] * f[p];
                            fac[F_END * CH + row + 8 * p] = exp2_fast((end_hi - hi[p]) + (end_lo - lo[p])) * f[p];
                        }
                        if (row + 8 == CH - 1) fac[F_LAST] = start[1];
                    }
                }
                bar_sync(Z::PREPARING, PREP);
                if (of_q) {
                    if (!F32 && next < chunks) load_raw(next);
                    cp_commit();
                }
                // -L or the scores: products times their tokens' factors and the decay between them. Across blocks of 16 the
                // decay is that from the column's token to its block's end times that from there on, both at most 1.
                const int i0 = 16 * mt + r8, i1 = i0 + 8;
                float m0 = 0.f, m1 = 0.f;
                {
                    const float *upto_hi = gate + G_HI * CH, *upto_lo = gate + G_LO * CH, *beta = gate + G_BETA * CH;
                    const float h0 = upto_hi[i0], h1 = upto_hi[i1], l0 = upto_lo[i0], l1 = upto_lo[i1];
                    const float s0 = of_q ? cq[i0] : -beta[i0] * ck[i0], s1 = of_q ? cq[i1] : -beta[i1] * ck[i1], up = of_q ? 1.f : T_UP;
                    const auto largest = [&](const float (&x)[4]) {
                        m0 = max_of(m0, x[0], x[1]);
                        m1 = max_of(m1, x[2], x[3]);
                    };
#pragma unroll
                    for (int n2 = 0; n2 < 3; ++n2) {
                        if (n2 >= mt) break;
                        const float he = upto_hi[16 * n2 + 15], le = upto_lo[16 * n2 + 15];
                        const float f0 = s0 * up * exp2_fast((h0 - he) + (l0 - le)), f1 = s1 * up * exp2_fast((h1 - he) + (l1 - le));
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            float(&x)[4] = acc[2 * n2 + p];
                            const float2 cj = *reinterpret_cast<const float2*>(ck + 16 * n2 + 8 * p + 2 * quad),
                                         ej = *reinterpret_cast<const float2*>(gate + G_BLOCK * CH + 16 * n2 + 8 * p + 2 * quad);
                            const float c0 = cj.x * ej.x, c1 = cj.y * ej.y;
                            x[0] *= c0 * f0; x[1] *= c1 * f0; x[2] *= c0 * f1; x[3] *= c1 * f1;
                            largest(x);
                        }
                    }
                    const int below = of_q ? 0 : 1;                 // below the diagonal, or up to it
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        float(&x)[4] = own_acc[p];
                        const int j0 = 16 * mt + 8 * p + 2 * quad;
                        const float2 cj = *reinterpret_cast<const float2*>(ck + j0), hj = *reinterpret_cast<const float2*>(upto_hi + j0),
                                     lj = *reinterpret_cast<const float2*>(upto_lo + j0);
                        x[0] = j0 + below <= i0 ? (s0 * cj.x) * exp2_fast((h0 - hj.x) + (l0 - lj.x)) * x[0] : 0.f;
                        x[1] = j0 + 1 + below <= i0 ? (s0 * cj.y) * exp2_fast((h0 - hj.y) + (l0 - lj.y)) * x[1] : 0.f;
                        x[2] = j0 + below <= i1 ? (s1 * cj.x) * exp2_fast((h1 - hj.x) + (l1 - lj.x)) * x[2] : 0.f;
                        x[3] = j0 + 1 + below <= i1 ? (s1 * cj.y) * exp2_fast((h1 - hj.y) + (l1 - lj.y)) * x[3] : 0.f;
                        largest(x);
                    }
                }
                const uint32_t to0 = tile_at<Z::TP>(i0, 0) + 4 * quad, to1 = tile_at<Z::TP>(i1, 0) + 4 * quad;       // segment n: turned by 16 n
                const auto put_parts = [&](const float (&x)[4], float p0, float p1, char* to0, char* to1, int part) {
                    uint32_t hi, lo;
                    split2(x[0] * p0, x[1] * p0, hi, lo);
                    *reinterpret_cast<uint32_t*>(to0) = hi;
                    *reinterpret_cast<uint32_t*>(to0 + part) = lo;
                    split2(x[2] * p1, x[3] * p1, hi, lo);
                    *reinterpret_cast<uint32_t*>(to1) = hi;
                    *reinterpret_cast<uint32_t*>(to1 + part) = lo;
                };
                if (of_q) {
                    const float p0 = to_f16_range(quad_max(m0)), p1 = to_f16_range(quad_max(m1));
                    if (quad == 0) {
                        fac[F_SCORE * CH + i0] = pow2_inverse(p0);
                        fac[F_SCORE * CH + i1] = pow2_inverse(p1);
                    }
                    const auto put_scores = [&](const float (&x)[4], int n) { put_parts(x, p0, p1, st + Z::P + (to0 ^ (n << 4)), st + Z::P + (to1 ^ (n << 4)), Z::PLO - Z::P); };
#pragma unroll
                    for (int n = 0; n < 6; ++n) {
                        if (n >= 2 * mt) break;
                        put_scores(acc[n], n);
                    }
                    put_scores(own_acc[0], 2 * mt);
                    put_scores(own_acc[1], 2 * mt + 1);
                } else {
                    // Rows that are not finite, of keys or gates that are not: T would carry them to earlier tokens through zeros. They
                    // count as 0 there, and their tokens' R as NaN, which the chain deals with.
                    if (__any_sync(0xffffffffu, !(max_of(m0, m1, 0.f) < __int_as_float(0x7f800000)))) {
                        const auto clean = [](float (&x)[4]) {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (!(fabsf(x[e]) < __int_as_float(0x7f800000))) x[e] = 0.f;
                        };
#pragma unroll
                        for (int n = 0; n < 6; ++n) clean(acc[n]);
                        clean(own_acc[0]);
                        clean(own_acc[1]);
                        if (!(m0 < __int_as_float(0x7f800000))) fac[F_STATE * CH + i0] = __int_as_float(0x7fffffff);
                        if (!(m1 < __int_as_float(0x7f800000))) fac[F_STATE * CH + i1] = __int_as_float(0x7fffffff);
                    }
#pragma unroll
                    for (int n = 0; n < 6; ++n) {
                        if (n >= 2 * mt) break;
                        if (n >> 1 == 1 && mt >= 2)
                            put_parts(acc[n], 1.f, 1.f, own + Z::BESIDE + beside_at(i0 - 32, n & 1) + 4 * quad, own + Z::BESIDE + beside_at(i1 - 32, n & 1) + 4 * quad, Z::PART);
                        else
                            put_parts(acc[n], 1.f, 1.f, st + Z::THI + (to0 ^ (n << 4)), st + Z::THI + (to1 ^ (n << 4)), Z::TLO - Z::THI);
                    }
                    // T's block on the diagonal, in fp32: its two blocks of 8 by substitution, a column a lane, then the one below
                    // them, -C^-1 B A^-1 (with B as it stands here, of -L, the sign is gone).
                    float* D = diag + 16 * mt * DP;
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        *reinterpret_cast<float2*>(D + r8 * DP + 8 * p + 2 * quad) = make_float2(own_acc[p][0], own_acc[p][1]);
                        *reinterpret_cast<float2*>(D + (r8 + 8) * DP + 8 * p + 2 * quad) = make_float2(own_acc[p][2], own_acc[p][3]);
                    }
                    __syncwarp();
                    {
                        const int col = lane & 7, at = lane & 8;    // lanes 16 .. 31 do the same again
                        float x[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            float t0 = i == col ? 1.f : 0.f, t1 = 0.f;
#pragma unroll
                            for (int m = 0; m < i; m += 4) {
                                const float4 l = *reinterpret_cast<const float4*>(D + (at + i) * DP + at + m);
                                t0 = fmaf(l.x, x[m], t0);
                                if (m + 1 < i) t1 = fmaf(l.y, x[m + 1], t1);
                                if (m + 2 < i) t0 = fmaf(l.z, x[m + 2], t0);
                                if (m + 3 < i) t1 = fmaf(l.w, x[m + 3], t1);
                            }
                            x[i] = i < col ? 0.f : t0 + t1;
                        }
                        __syncwarp();
                        if (lane < 16)
#pragma unroll
                            for (int i = 0; i < 8; ++i) D[(at + i) * DP + at + col] = x[i];
                        __syncwarp();
                    }
                    const auto times = [&](const float* left, const float* right, float* to) {          // 8 x 8, two columns a lane
                        float2 y = make_float2(0.f, 0.f);
#pragma unroll
                        for (int m = 0; m < 8; ++m) {
                            const float l = left[r8 * DP + m];
                            const float2 a = *reinterpret_cast<const float2*>(right + m * DP + 2 * quad);
                            y.x = fmaf(l, a.x, y.x);
                            y.y = fmaf(l, a.y, y.y);
                        }
                        __syncwarp();
                        *reinterpret_cast<float2*>(to + r8 * DP + 2 * quad) = y;
                        __syncwarp();
                    };
#pragma unroll 1
                    for (int p = 0; p < 2; ++p) times(D + 8 * DP + 8 * p, D + 8 * DP * p, D + 8 * DP);
                    {
                        const int row = lane >> 1, half = lane & 1;
                        const float4 a = *reinterpret_cast<const float4*>(D + row * DP + 8 * half), b = *reinterpret_cast<const float4*>(D + row * DP + 8 * half + 4);
                        const bool above = half && row < 8;         // zeros, whatever stood there
                        uint32_t hi[4], lo[4];
                        const auto two = [&](float x, float y, int i) { split2(above ? 0.f : x * T_UP, above ? 0.f : y * T_UP, hi[i], lo[i]); };
                        two(a.x, a.y, 0);
                        two(a.z, a.w, 1);
                        two(b.x, b.y, 2);
                        two(b.z, b.w, 3);
                        const uint32_t at = tile_at<Z::TP>(16 * mt + row, 2 * mt + half);
                        *reinterpret_cast<uint4*>(st + Z::THI + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                        *reinterpret_cast<uint4*>(st + Z::TLO + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                    }
                }
            }
            if (!of_q) bar_sync(Z::KEYS, Z::HALF);
        }
        // The blocks below the diagonal, N for -L, whose places they take: T_10 and T_32, T_bb N_ba T_aa, a warp each; then, a warp for each of the columns
        // a = 0, 1, X_b = sum_(k <= 1) N_bk T_ka for b = 2, 3, T_2a = T_22 X_2 and T_3a = T_32 X_2 + T_33 X_3. Transposed: T_ka^T,
        // read transposed, is an A fragment, and so is what comes out of the products.
        if (c >= 0 && !of_q) {
            struct Sum { float x[2][4], y[2][4]; };
            const auto times = [&](Sum& s, const uint32_t (&hi)[4], const uint32_t (&lo)[4], int b, int k, bool beside = false) {       // by block (b, k) of N or T
                uint32_t f[4], e[4];
                const uint32_t at = beside ? own_b + Z::BESIDE + beside_at(16 * (b - 2) + b_row, b_seg) : sb + Z::THI + tile_at<Z::TP>(16 * b + b_row, 2 * k + b_seg);
                ldmatrix4(f, at);
                ldmatrix4(e, at + (beside ? Z::PART : Z::TLO - Z::THI));
                mma(s.x[0], hi, f[0], f[1]);
                mma(s.x[1], hi, f[2], f[3]);
                mma(s.y[0], lo, f[0], f[1]);
                mma(s.y[1], lo, f[2], f[3]);
                mma(s.y[0], hi, e[0], e[1]);
                mma(s.y[1], hi, e[2], e[3]);
            };
            const auto get = [&](uint32_t (&hi)[4], uint32_t (&lo)[4], int k, int a) {
                const uint32_t at = tile_at<Z::TP>(16 * k + b_row, 2 * a + b_seg);
                ldmatrix4_trans(hi, sb + Z::THI + at);
                ldmatrix4_trans(lo, sb + Z::TLO + at);
            };
            const auto parts = [&](Sum& s, uint32_t (&hi)[4], uint32_t (&lo)[4]) {
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s.x[p][i] += s.y[p][i];
                split_a(s.x[0], s.x[1], 1.f / T_UP, 1.f / T_UP, hi, lo);        // up by T_UP once, not twice
            };
            const auto put = [&](const uint32_t (&hi)[4], const uint32_t (&lo)[4], int b, int a) {
                const uint32_t at = tile_at<Z::TP>(16 * b + 8 * (lane >> 4) + (lane & 7), 2 * a + ((lane >> 3) & 1));
                stmatrix4_trans(sb + Z::THI + at, hi);
                stmatrix4_trans(sb + Z::TLO + at, lo);
            };
            uint32_t hi[4], lo[4];
            if (warp < 2) {
                const int a = 2 * warp;
                Sum s = {}, t = {};
                get(hi, lo, a, a);
                times(s, hi, lo, a + 1, a);
                parts(s, hi, lo);
                times(t, hi, lo, a + 1, a + 1);
                parts(t, hi, lo);
                put(hi, lo, a + 1, a);
            }
            bar_sync(Z::KEYS, Z::HALF);
            if (warp < 2) {
                Sum s2 = {}, s3 = {}, t2 = {}, t3 = {};
#pragma unroll 1
                for (int k = warp; k < 2; ++k) {
                    get(hi, lo, k, warp);
                    times(s2, hi, lo, 2, k, k == 1);
                    times(s3, hi, lo, 3, k, k == 1);
                }
                uint32_t hi3[4], lo3[4];
                parts(s2, hi, lo);
                parts(s3, hi3, lo3);
                times(t2, hi, lo, 2, 2);
                times(t3, hi, lo, 3, 2);
                times(t3, hi3, lo3, 3, 3);
                parts(t2, hi, lo);
                parts(t3, hi3, lo3);
                put(hi, lo, 2, warp);
                put(hi3, lo3, 3, warp);
            }
        }
        if (c >= 0) {
            cp_wait_but_one();                                      // the values, not what comes for the next chunk
            bar_arrive(Z::FULL + stage, Z::FULL_COUNT);
        }
        if (gates) sum_gates(next, reinterpret_cast<float*>(own + Z::TOKENS) + (next & (STAGES - 1)) * Z::FACTORS + 2 * CH);
    }
}

// ---------------------------------------------------------------------------
// Outputs: e^G S^T q of a chunk's tokens, scaled, and what the scores add. By the chain warps, or by two others.
// ---------------------------------------------------------------------------
__device__ __forceinline__ float2 get2(const float (&x)[4], int i) { return make_float2(x[i], x[i + 1]); }
__device__ __forceinline__ void put2(float (&x)[4], int i, float2 y) { x[i] = y.x; x[i + 1] = y.y; }

// The products with the state by their tokens' factors; NaN from a lost column's token on.
__device__ __forceinline__ void scale_outputs(float (&O)[8][4], const float* fac, float is0, float is1, bool odd, int bad0, int bad1) {
    const int quad = threadIdx.x & 3;
#pragma unroll
    for (int n = 0; n < 8; ++n) {
        const float2 f = *reinterpret_cast<const float2*>(fac + F_QUERY * CH + 8 * n + 2 * quad);
        put2(O[n], 0, mul2(mul2(f, twice(is0)), get2(O[n], 0)));
        put2(O[n], 2, mul2(mul2(f, twice(is1)), get2(O[n], 2)));
    }
    if (odd)
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int t = 8 * n + 2 * quad + e;
                if (t >= bad0) O[n][e] = __int_as_float(0x7fffffff);
                if (t >= bad1) O[n][2 + e] = __int_as_float(0x7fffffff);
            }
}
// O^T + U^T P^T, to where row r8's values of the lane's columns are; `live`: rows from there on.
template <class Z>
__device__ __forceinline__ void put_outputs(const float (&O)[8][4], const uint32_t (&u)[4][4], const uint32_t (&ulo)[4][4], float iu0, float iu1, uint32_t scores, const float* fac,
                                            uint16_t* o, int64_t step, int live) {
    const int lane = threadIdx.x & 31, quad = lane & 3, b_row = (lane & 7) + ((lane >> 4) << 3), b_seg = (lane >> 3) & 1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x[2][4];
#pragma unroll
        for (int j = 0; j <= i; ++j) {
            uint32_t b[4], l[4];
            const uint32_t at = scores + tile_at<Z::TP>(16 * i + b_row, 2 * j + b_seg);
            ldmatrix4(b, at);
            ldmatrix4(l, at + Z::PLO - Z::P);
            mma_from(j == 0, x[0], u[j], b[0], b[1]);
            mma_from(j == 0, x[1], u[j], b[2], b[3]);
            mma(x[0], ulo[j], b[0], b[1]);
            mma(x[1], ulo[j], b[2], b[3]);
            mma(x[0], u[j], l[0], l[1]);
            mma(x[1], u[j], l[2], l[3]);
        }
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int n = 2 * i + p;
            const float2 fp = *reinterpret_cast<const float2*>(fac + F_SCORE * CH + 8 * n + 2 * quad);
            float y[4];
            put2(y, 0, fma2(get2(x[p], 0), mul2(fp, twice(iu0)), get2(O[n], 0)));
            put2(y, 2, fma2(get2(x[p], 2), mul2(fp, twice(iu1)), get2(O[n], 2)));
            const uint32_t a = movmatrix_trans(pack_bf16(y[0], y[1])), b = movmatrix_trans(pack_bf16(y[2], y[3]));
            store_if(o, a, b, 8 * n < live);
            o += step;
        }
    }
}

template <bool F32, int DK, int CW>
__device__ __forceinline__ void run_outputs(const Delta& d, const SeqRange& r, int h, int col0, char* smem, uint32_t base, int chunks) {
    using Z = Shape<F32, DK, CW>;
    const int warp = (threadIdx.x >> 5) - CW, lane = threadIdx.x & 31, r8 = lane >> 2;                 // for chain warp `warp`
    const int64_t step = 8 * (int64_t)d.heads * d.head_v;
    uint16_t* out = d.out + (((int64_t)r.lo + r8) * d.heads + h) * d.head_v + col0 + 16 * warp + 2 * (lane & 3);
    const char* hand = smem + Z::HANDED + warp * Z::HAND;
    const uint4* from = reinterpret_cast<const uint4*>(hand) + lane;
    const int b_row = (lane & 7) + ((lane >> 4) << 3), b_seg = (lane >> 3) & 1;
    for (int i = 0; i < STAGES && i < chunks; ++i) bar_arrive(Z::EMPTY + i, Z::EMPTY_COUNT);
#pragma unroll 1
    for (int c = 0; c < chunks; ++c, out += CH / 8 * step) {
        const int stage = c & (STAGES - 1);
        const uint32_t sb = base + stage * Z::STAGE;
        const float* fac = reinterpret_cast<const float*>(smem + stage * Z::STAGE + Z::FAC);
        float O[8][4];
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) O[n][e] = 0.f;
        bar_sync(Z::FULL + stage, Z::FULL_COUNT);
        bar_sync(Z::S_READY + warp, 64);
#pragma unroll 2
        for (int kk = 0; kk < DK / 16; ++kk) {
            uint32_t f[4][4];
#pragma unroll
            for (int n2 = 0; n2 < 4; ++n2) ldmatrix4(f[n2], sb + Z::Q + Z::key_at(16 * n2 + b_row, 2 * kk + b_seg));
            const uint4 x = from[2 * kk * 32], y = from[(2 * kk + 1) * 32];
            const uint32_t hi[4] = {x.x, x.y, x.z, x.w}, lo[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int n = 0; n < 8; ++n) mma(O[n], hi, f[n >> 1][2 * (n & 1)], f[n >> 1][2 * (n & 1) + 1]);
#pragma unroll
            for (int n = 0; n < 8; ++n) mma(O[n], lo, f[n >> 1][2 * (n & 1)], f[n >> 1][2 * (n & 1) + 1]);
            if constexpr (F32) {
#pragma unroll
                for (int n2 = 0; n2 < 4; ++n2) ldmatrix4(f[n2], sb + Z::QLO + Z::key_at(16 * n2 + b_row, 2 * kk + b_seg));
#pragma unroll
                for (int n = 0; n < 8; ++n) mma(O[n], hi, f[n >> 1][2 * (n & 1)], f[n >> 1][2 * (n & 1) + 1]);
            }
        }
        bar_sync(Z::U_READY + warp, 64);
        uint32_t u[4][4], ulo[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint4 x = from[2 * (DK / 16 + j) * 32], y = from[(2 * (DK / 16 + j) + 1) * 32];
            u[j][0] = x.x; u[j][1] = x.y; u[j][2] = x.z; u[j][3] = x.w;
            ulo[j][0] = y.x; ulo[j][1] = y.y; ulo[j][2] = y.z; ulo[j][3] = y.w;
        }
        const float4 scales = *reinterpret_cast<const float4*>(hand + Z::HAND_SCALES + lane * 16);
        const int2 bad = *reinterpret_cast<const int2*>(hand + Z::HAND_SCALES + 512 + lane * 8);
        if (c + 1 < chunks) bar_arrive(Z::TAKEN + warp, 64);
        scale_outputs(O, fac, scales.x, scales.y, bad.x < CH || bad.y < CH, bad.x, bad.y);
        put_outputs<Z>(O, u, ulo, scales.z, scales.w, sb + Z::P, fac, out, step, r.n - c * CH - r8);
        if (c + STAGES < chunks) bar_arrive(Z::EMPTY + stage, Z::EMPTY_COUNT);
    }
}

// ---------------------------------------------------------------------------
// The chain: a warp, 16 columns.
// ---------------------------------------------------------------------------
template <bool F32, int DK, int CW>
__device__ __forceinline__ void run_chain(const Delta& d, const SeqRange& r, int h, int col0, char* smem, uint32_t base, int chunks) {
    using Z = Shape<F32, DK, CW>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane & 3, r8 = lane >> 2;
    const int vcol = 16 * warp;
    float* state = d.state + ((int64_t)r.slot * d.heads + h) * DK * d.head_v + 2 * quad * d.head_v + col0 + vcol + r8;
    uint16_t* out = d.out + (((int64_t)r.lo + r8) * d.heads + h) * d.head_v + col0 + vcol + 2 * quad;
    char* hand = smem + Z::HANDED + warp * Z::HAND;
    uint4* to = reinterpret_cast<uint4*>(hand) + lane;
    float S[DK / 8][4];                                             // [8 rows of S][columns r8, r8 + 8 x two rows]
    const float* from = state;
#pragma unroll
    for (int j = 0; j < DK / 8; ++j, from += 8 * d.head_v) {
        S[j][0] = r.fresh ? 0.f : from[0]; S[j][2] = r.fresh ? 0.f : from[8];
        S[j][1] = r.fresh ? 0.f : from[d.head_v]; S[j][3] = r.fresh ? 0.f : from[d.head_v + 8];
    }
    for (int i = 0; i < STAGES && i < chunks; ++i) bar_arrive(Z::EMPTY + i, Z::EMPTY_COUNT);
    const int b_row = (lane & 7) + ((lane >> 4) << 3), b_seg = (lane >> 3) & 1;                        // two tiles of tokens
    const int t_row = (lane & 7) + (((lane >> 3) & 1) << 3), t_seg = lane >> 4;                        // transposed: 16 tokens, two tiles of columns
#pragma unroll 1
    for (int c = 0; c < chunks; ++c) {
        const int stage = c & (STAGES - 1);
        const char* st = smem + stage * Z::STAGE;
        const uint32_t sb = base + stage * Z::STAGE;
        const float* fac = reinterpret_cast<const float*>(st + Z::FAC);
        float sc0 = 0.f, sc1 = 0.f;
#pragma unroll
        for (int j = 0; j < DK / 8; ++j) {
            sc0 = max_of(sc0, S[j][0], S[j][1]);
            sc1 = max_of(sc1, S[j][2], S[j][3]);
        }
        sc0 = to_f16_range(quad_max(sc0));
        sc1 = to_f16_range(quad_max(sc1));
        bar_sync(Z::FULL + stage, Z::FULL_COUNT);
        if (Z::APART && c > 0) bar_sync(Z::TAKEN + warp, 64);
        // S^T k and (but for outputs elsewhere) S^T q of every token
        float R[8][4], O[8][4];
        // fragments one step ahead of their products
        uint32_t fk[4][4], fq[4][4];
        const auto load4 = [&](uint32_t (&f)[4][4], int tile, int kk) {
#pragma unroll
            for (int n2 = 0; n2 < 4; ++n2) ldmatrix4(f[n2], sb + tile + Z::key_at(16 * n2 + b_row, 2 * kk + b_seg));
        };
        load4(fk, Z::K, 0);
#pragma unroll
        for (int kk = 0; kk < DK / 16; ++kk) {
            uint32_t hi[4], lo[4];
            split_a(S[2 * kk], S[2 * kk + 1], sc0, sc1, hi, lo);
            if constexpr (Z::APART) {
                to[2 * kk * 32] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                to[(2 * kk + 1) * 32] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            } else {
                load4(fq, Z::Q, kk);
            }
#pragma unroll
            for (int n = 0; n < 8; ++n) mma_from(kk == 0, R[n], hi, fk[n >> 1][2 * (n & 1)], fk[n >> 1][2 * (n & 1) + 1]);
#pragma unroll
            for (int n = 0; n < 8; ++n) mma(R[n], lo, fk[n >> 1][2 * (n & 1)], fk[n >> 1][2 * (n & 1) + 1]);
            if constexpr (F32) {
                load4(fk, Z::KLO, kk);
#pragma unroll
                for (int n = 0; n < 8; ++n) mma(R[n], hi, fk[n >> 1][2 * (n & 1)], fk[n >> 1][2 * (n & 1) + 1]);
            }
            if (kk + 1 < DK / 16) load4(fk, Z::K, kk + 1);
            if constexpr (!Z::APART) {
#pragma unroll
                for (int n = 0; n < 8; ++n) mma_from(kk == 0, O[n], hi, fq[n >> 1][2 * (n & 1)], fq[n >> 1][2 * (n & 1) + 1]);
#pragma unroll
                for (int n = 0; n < 8; ++n) mma(O[n], lo, fq[n >> 1][2 * (n & 1)], fq[n >> 1][2 * (n & 1) + 1]);
                if constexpr (F32) {
                    load4(fq, Z::QLO, kk);
#pragma unroll
                    for (int n = 0; n < 8; ++n) mma(O[n], hi, fq[n >> 1][2 * (n & 1)], fq[n >> 1][2 * (n & 1) + 1]);
                }
            }
        }
        if constexpr (Z::APART) bar_arrive(Z::S_READY + warp, 64);
        // R = beta v - beta e^G (S^T k)
        const float is0 = pow2_inverse(sc0), is1 = pow2_inverse(sc1);
        const float2 down0 = twice(-is0), down1 = twice(-is1);
        float m0 = 0.f, m1 = 0.f;
#pragma unroll
        for (int n2 = 0; n2 < 4; ++n2) {
            uint32_t v[4];
            if constexpr (!F32) ldmatrix4_trans(v, sb + Z::V + (16 * n2 + b_row) * Z::VP + (vcol / 8 + b_seg) * 16);
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int n = 2 * n2 + p, t = 8 * n + 2 * quad;
                float v0[2], v1[2];
                if constexpr (F32) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float* vp = reinterpret_cast<const float*>(st + Z::V + (t + e) * Z::VP) + vcol + r8;
                        v0[e] = vp[0]; v1[e] = vp[8];
                    }
                } else {
                    v0[0] = __uint_as_float(v[2 * p] << 16); v0[1] = __uint_as_float(v[2 * p] & 0xffff0000u);
                    v1[0] = __uint_as_float(v[2 * p + 1] << 16); v1[1] = __uint_as_float(v[2 * p + 1] & 0xffff0000u);
                }
                const float2 fb = *reinterpret_cast<const float2*>(fac + F_BETA * CH + t), fs = *reinterpret_cast<const float2*>(fac + F_STATE * CH + t);
                put2(R[n], 0, fma2(mul2(fs, down0), get2(R[n], 0), mul2(fb, make_float2(v0[0], v0[1]))));
                put2(R[n], 2, fma2(mul2(fs, down1), get2(R[n], 2), mul2(fb, make_float2(v1[0], v1[1]))));
                m0 = max_of(m0, R[n][0], R[n][1]);
                m1 = max_of(m1, R[n][2], R[n][3]);
            }
        }
        const float nan = __int_as_float(0x7fffffff);
        int bad0 = CH, bad1 = CH;                                   // the first tokens whose R is not finite
        const bool odd = __any_sync(0xffffffffu, !(max_of(m0, m1, 0.f) < __int_as_float(0x7f800000)));
        if (odd) {
            m0 = m1 = 0.f;
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int t = 8 * n + 2 * quad + e;
                    if (!(fabsf(R[n][e]) < __int_as_float(0x7f800000))) { bad0 = min(bad0, t); R[n][e] = 0.f; }
                    if (!(fabsf(R[n][2 + e]) < __int_as_float(0x7f800000))) { bad1 = min(bad1, t); R[n][2 + e] = 0.f; }
                    m0 = fmaxf(m0, fabsf(R[n][e]));
                    m1 = fmaxf(m1, fabsf(R[n][2 + e]));
                }
            bad0 = min(bad0, __shfl_xor_sync(0xffffffffu, bad0, 1)); bad0 = min(bad0, __shfl_xor_sync(0xffffffffu, bad0, 2));
            bad1 = min(bad1, __shfl_xor_sync(0xffffffffu, bad1, 1)); bad1 = min(bad1, __shfl_xor_sync(0xffffffffu, bad1, 2));
        }
        if constexpr (!Z::APART) scale_outputs(O, fac, is0, is1, odd, bad0, bad1);
        const float rs0 = to_f16_range(quad_max(m0)), rs1 = to_f16_range(quad_max(m1));
        // U^T = R^T T^T, 16 tokens at a time from the last: a block of U takes the place of the block of R that no other needs
        uint32_t rh[4][4], rl[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) split_a(R[2 * j], R[2 * j + 1], rs0, rs1, rh[j], rl[j]);
        const float ir0 = pow2_inverse(rs0) * (1.f / T_UP), ir1 = pow2_inverse(rs1) * (1.f / T_UP);
        float u0 = 0.f, u1 = 0.f;
#pragma unroll
        for (int i = 3; i >= 0; --i) {
            float x[2][4];
#pragma unroll
            for (int j = 0; j <= i; ++j) {
                const uint32_t at = tile_at<Z::TP>(16 * i + b_row, 2 * j + b_seg);
                uint32_t b[4];
                ldmatrix4(b, sb + Z::THI + at);
                mma_from(j == 0, x[0], rh[j], b[0], b[1]);
                mma_from(j == 0, x[1], rh[j], b[2], b[3]);
                mma(x[0], rl[j], b[0], b[1]);
                mma(x[1], rl[j], b[2], b[3]);
                ldmatrix4(b, sb + Z::TLO + at);
                mma(x[0], rh[j], b[0], b[1]);
                mma(x[1], rh[j], b[2], b[3]);
            }
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                put2(R[2 * i + p], 0, mul2(get2(x[p], 0), twice(ir0)));
                put2(R[2 * i + p], 2, mul2(get2(x[p], 2), twice(ir1)));
            }
        }
        float e0 = 0.f, e1 = 0.f;                                   // of U, and of U as the state takes it
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const float2 fe = *reinterpret_cast<const float2*>(fac + F_END * CH + 8 * n + 2 * quad);
            u0 = max_of(u0, R[n][0], R[n][1]);
            u1 = max_of(u1, R[n][2], R[n][3]);
            const float2 x = mul2(get2(R[n], 0), fe), y = mul2(get2(R[n], 2), fe);
            e0 = max_of(e0, x.x, x.y);
            e1 = max_of(e1, y.x, y.y);
        }
        const float us0 = to_f16_range(quad_max(u0)), us1 = to_f16_range(quad_max(u1));
        const float es0 = to_f16_range(quad_max(e0)), es1 = to_f16_range(quad_max(e1));
        // U as the outputs take it
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 x = mul2(get2(R[2 * j + (e >> 1)], 2 * (e & 1)), twice(e & 1 ? us1 : us0));
                split2(x, rh[j][e], rl[j][e]);
            }
        const float iu0 = pow2_inverse(us0), iu1 = pow2_inverse(us1);
        if constexpr (Z::APART) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                to[2 * (DK / 16 + j) * 32] = make_uint4(rh[j][0], rh[j][1], rh[j][2], rh[j][3]);
                to[(2 * (DK / 16 + j) + 1) * 32] = make_uint4(rl[j][0], rl[j][1], rl[j][2], rl[j][3]);
            }
            *reinterpret_cast<float4*>(hand + Z::HAND_SCALES + lane * 16) = make_float4(is0, is1, iu0, iu1);
            *reinterpret_cast<int2*>(hand + Z::HAND_SCALES + 512 + lane * 8) = make_int2(bad0, bad1);
            bar_arrive(Z::U_READY + warp, 64);
        } else {
            const int64_t step = 8 * (int64_t)d.heads * d.head_v;
            put_outputs<Z>(O, rh, rl, iu0, iu1, sb + Z::P, fac, out + c * (CH / 8) * step, step, r.n - c * CH - r8);
        }
        // S^T <- e^G S^T + U^T k
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int n = 2 * j + (e >> 1);
                const float2 fe = *reinterpret_cast<const float2*>(fac + F_END * CH + 8 * n + 2 * quad);
                split2(mul2(mul2(get2(R[n], 2 * (e & 1)), fe), twice(e & 1 ? es1 : es0)), rh[j][e], rl[j][e]);
            }
        const float ie0 = pow2_inverse(es0), ie1 = pow2_inverse(es1);
        const float last0 = bad0 < CH ? nan : fac[F_LAST], last1 = bad1 < CH ? nan : fac[F_LAST];
        uint32_t fu[2][2][4];
        const auto load2 = [&](uint32_t (&f)[2][4], int tile, int step) {           // 16 tokens by four tiles of S
#pragma unroll
            for (int p = 0; p < 2; ++p)
                ldmatrix4_trans(f[p], sb + tile + Z::key_at(16 * (step & 3) + t_row, 4 * (step >> 2) + 2 * p + t_seg));
        };
        load2(fu[0], Z::K, 0);
#pragma unroll
        for (int j4 = 0; j4 < DK / 32; ++j4) {                       // four tiles of S at a time
            float x[4][4];
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                const int step = 4 * j4 + kk;
                uint32_t (&b)[2][4] = fu[step & 1], (&next)[2][4] = fu[(step + 1) & 1];
                if (F32) load2(next, Z::KLO, step);
                else if (step + 1 < DK / 8) load2(next, Z::K, step + 1);
#pragma unroll
                for (int p = 0; p < 4; ++p) mma_from(kk == 0, x[p], rh[kk], b[p >> 1][2 * (p & 1)], b[p >> 1][2 * (p & 1) + 1]);
#pragma unroll
                for (int p = 0; p < 4; ++p) mma(x[p], rl[kk], b[p >> 1][2 * (p & 1)], b[p >> 1][2 * (p & 1) + 1]);
                if constexpr (F32) {
#pragma unroll
                    for (int p = 0; p < 4; ++p) mma(x[p], rh[kk], next[p >> 1][2 * (p & 1)], next[p >> 1][2 * (p & 1) + 1]);
                    if (step + 1 < DK / 8) load2(next, Z::K, step + 1);
                }
            }
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                float(&s)[4] = S[4 * j4 + p];
                put2(s, 0, fma2(twice(last0), get2(s, 0), mul2(get2(x[p], 0), twice(ie0))));
                put2(s, 2, fma2(twice(last1), get2(s, 2), mul2(get2(x[p], 2), twice(ie1))));
            }
        }
        if (c + STAGES < chunks) bar_arrive(Z::EMPTY + stage, Z::EMPTY_COUNT);
    }
#pragma unroll
    for (int j = 0; j < DK / 8; ++j, state += 8 * d.head_v) {
        state[0] = S[j][0]; state[8] = S[j][2];
        state[d.head_v] = S[j][1]; state[d.head_v + 8] = S[j][3];
    }
}

template <bool F32, int DK, int CW>
__global__ void __launch_bounds__(Shape<F32, DK, CW>::THREADS, 1) delta_chunk_kernel(Delta d, int above) {
    using Z = Shape<F32, DK, CW>;
    extern __shared__ __align__(128) char smem[];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (above > 0) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");     // the kernel of the shorter sequences
    const int slices = d.head_v / Z::VC;
    const int unit = (int)(blockIdx.x / slices), slice = (int)(blockIdx.x - unit * slices);
    const int b = unit / d.heads, h = unit - b * d.heads, col0 = slice * Z::VC;
    const SeqRange r = seq_range(d.seq, b, d.n_slots, h == 0 && slice == 0 && threadIdx.x == 0, d.status);
    if (r.n <= above) return;
    if (r.slot < 0) {
        constexpr int PER = Z::VC / 8;
        for (int64_t i = threadIdx.x; i < (int64_t)r.n * PER; i += Z::THREADS)
            *reinterpret_cast<uint4*>(d.out + ((r.lo + i / PER) * d.heads + h) * d.head_v + col0 + (i % PER) * 8) = make_uint4(0, 0, 0, 0);
        return;
    }
    const uint32_t base = smem_u32(smem);
    const int chunks = (r.n + CH - 1) / CH;
    // Three warpgroups of 168 registers a thread at launch; the chain takes what the preparing warps leave.
    static_assert(Z::THREADS == 384);
    if (threadIdx.x < Z::CHAIN) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        if (threadIdx.x < 32 * CW) run_chain<F32, DK, CW>(d, r, h, col0, smem, base, chunks);
        else if constexpr (Z::APART) run_outputs<F32, DK, CW>(d, r, h, col0, smem, base, chunks);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 136;");
        prepare_chunks<F32, DK, CW>(d, r, h, col0, smem, base, chunks);
    }
}

template <bool F32, int DK, int CW>
cudaError_t launch_shape(const Delta& d, int above, cudaStream_t s) {
    using Z = Shape<F32, DK, CW>;
    static_assert(Z::BYTES <= 227 * 1024, "stages must fit");
    const auto kernel = delta_chunk_kernel<F32, DK, CW>;
    static LaunchPrep prep;
    int sms = 0;
    const cudaError_t e = prep.get(kernel, Z::BYTES, &sms);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)((int64_t)d.seq.batch * d.heads * (d.head_v / Z::VC)));
    return launch_dependent(kernel, grid, Z::THREADS, Z::BYTES, s, d, above);
}

template <bool F32, int DK>
cudaError_t launch_width(const Delta& d, int above, int sms, cudaStream_t s) {
    // Columns of a block. All blocks of a head prepare the same chunks, so fewer and wider ones do less in all, and more and
    // narrower ones fill the GPU. A chunk takes a block of 32 or 64 columns about 4.5 and 5.2 us; the rounds of blocks are
    // counted by the sequences like the longest that the tokens make up. Five sequences of 1774 to 3001 tokens, 32 heads of
    // 128: 859 and 550 us; one of 32768: 2290 and 2650. (128 columns, which leave the preparing warps half the registers,
    // took 11.2 us a chunk.) Measured with BF16 heads of 128 by 128. fp32 values leave no room for the wider one.
    if constexpr (!F32) {
        const int64_t alike = (d.seq.tokens + d.seq.rows / 2) / d.seq.rows, sequences = alike < 1 ? 1 : alike > d.seq.batch ? d.seq.batch : alike;
        const auto cost = [&](int columns, int64_t each) { return (sequences * d.heads * d.head_v / columns + sms - 1) / sms * each; };
        if (cost(64, 52) < cost(32, 45)) return launch_shape<F32, DK, 4>(d, above, s);
    }
    return launch_shape<F32, DK, 2>(d, above, s);
}

}  // namespace

cudaError_t launch_delta_chunks(const Delta& d, int above, int sms, cudaStream_t s) {
    if (d.f32) return d.head_k == 64 ? launch_width<true, 64>(d, above, sms, s) : launch_width<true, 128>(d, above, sms, s);
    return d.head_k == 64 ? launch_width<false, 64>(d, above, sms, s) : launch_width<false, 128>(d, above, sms, s);
}

}  // namespace vbq
