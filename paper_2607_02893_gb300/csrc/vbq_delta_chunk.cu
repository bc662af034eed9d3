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
// sequence, one head and 16 columns for each of its chain warps, and a chain
// warp holds S^T for its 16 columns in the accumulators of m16n8k16 (columns x
// head_k) over the whole sequence. Everything is computed transposed: what comes
// out of one product is, in the same registers, the A operand of the next, so
// the chain has no exchange between warps and nothing but key, query, T and
// score fragments is read from shared memory. Other warps prepare the next
// chunk meanwhile: load, normalise, the two products of keys with keys and
// queries, T by substitution in fp32. Named barriers hand the stages over.
//
// fp32 through the tensor cores. Keys are taken to FP16 by a power of two per
// token, which BF16 values survive unchanged (8 bits of 11, 39 binades down from
// the largest); S, R, U and T enter as two FP16 parts, x = hi + lo, with a power
// of two per column of S, so a product is good to 2^-22 (fp32 keys are two parts
// as well). What reaches the outputs alone, which are rounded to BF16, enters as
// one part (2^-12): queries, scores, and S and U beside them.
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
__device__ __forceinline__ float exp2_fast(float x) {              // 2 ulps; below 2^-126: 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 16 bytes to shared memory, zeros where `take` is false.
__device__ __forceinline__ void cp_16(uint32_t dst, const void* src, bool take) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(take ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// (x, y) as FP16 parts: hi, and what it leaves
__device__ __forceinline__ void split2(float x, float y, uint32_t& hi, uint32_t& lo) {
    hi = pack_f16(x, y);
    const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    lo = pack_f16(x - h.x, y - h.y);
}
// Two neighbouring tiles of 8 columns as A fragments, scaled by row: FP16 parts.
__device__ __forceinline__ void split_a(const float (&x)[4], const float (&y)[4], float s0, float s1, uint32_t (&hi)[4], uint32_t (&lo)[4]) {
    split2(x[0] * s0, x[1] * s0, hi[0], lo[0]);
    split2(x[2] * s1, x[3] * s1, hi[1], lo[1]);
    split2(y[0] * s0, y[1] * s0, hi[2], lo[2]);
    split2(y[2] * s1, y[3] * s1, hi[3], lo[3]);
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
    const int turn = PITCH == 64 ? (row >> 1) & 3 : row & 7;
    return (uint32_t)(row * PITCH + ((seg ^ turn) << 4));
}

// what the gates of a chunk come to, per token, and from G_LAST on for the chunk
enum { G_HI, G_LO, G_BETA, G_START, G_END, G_BLOCK };
constexpr int G_LAST = 6 * CH, GATES = 6 * CH + 4;

template <bool F32, int DK, int CW, int PW>
struct Shape {
    static constexpr int VC = 16 * CW;                              // columns of a block
    // Bytes of a row of keys in FP16 and of values, 16 more than they hold, so that eight rows' segments fall in distinct
    // banks (fp32 keys: turned by row instead, for want of room).
    static constexpr int KP = 2 * DK + (F32 ? 0 : 16), VP = F32 ? 4 * (VC + 4) : 2 * VC + 16;
    static constexpr int TP = 2 * CH;                               // bytes of a row of T, the scores and L
    static constexpr int CHAIN = 32 * (CW < 4 ? 4 : CW);            // whole warpgroups
    static constexpr int PREP = 32 * PW, THREADS = CHAIN + PREP;
    // a stage: keys (fp32 ones: the two parts of them, where their raw values land), queries, values, T, scores, factors
    static constexpr int K = 0, KLO = K + CH * KP, Q = KLO + (F32 ? CH * KP : 0), QLO = Q + CH * KP, V = QLO + (F32 ? CH * KP : 0),
                         THI = (V + CH * VP + 127) / 128 * 128, TLO = THI + CH * TP, P = TLO + CH * TP, FAC = P + CH * TP,
                         STAGE = (FAC + (5 * CH + 4) * 4 + 127) / 128 * 128;
    // scratch of the preparing warps: -L in FP16 parts, its blocks on the diagonal in fp32, factors
    static constexpr int LHI = 0, LLO = LHI + CH * TP, DIAG = LLO + CH * TP, TOKENS = DIAG + 4 * 16 * DP * 4,
                         SCRATCH = TOKENS + (2 * CH + GATES) * 4;
    static constexpr int OWN = STAGES * STAGE, BYTES = OWN + SCRATCH;
    // named barriers
    static constexpr int FULL = 1, EMPTY = FULL + STAGES, PREPARING = EMPTY + STAGES, COUNT = 32 * CW + PREP;
    __device__ static __forceinline__ uint32_t key_at(int row, int seg) {
        return F32 ? tile_at<2 * DK>(row, seg) : (uint32_t)(row * KP + seg * 16);
    }
};
// what a stage tells about its tokens
enum { F_BETA, F_STATE, F_END, F_QUERY, F_SCORE };                  // and from F_LAST on: e^G_last
constexpr int F_LAST = 5 * CH;

// ---------------------------------------------------------------------------
// Preparing the chunks: PW warps (4 or 8), one chunk after the other. Loops are kept rolled where registers allow: the code of both roles
// has to stay in the instruction cache.
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

template <bool F32, int DK, int CW, int PW>
__device__ __forceinline__ void prepare_chunks(const Delta& d, const SeqRange& r, int h, int col0, char* smem, uint32_t base, int chunks) {
    using Z = Shape<F32, DK, CW, PW>;
    constexpr int PREP = Z::PREP, SEGS = DK / 8, STEP = PREP / SEGS, ROWS = CH / STEP;     // 8 values a thread, STEP rows at once
    constexpr bool AHEAD = !F32 && PW == 8;                         // there are registers for the next chunk's keys and queries
    const int tid = threadIdx.x - Z::CHAIN, warp = tid >> 5, lane = tid & 31;
    const int hk = h / (d.heads / d.k_heads);
    const bool raw = d.a_log != nullptr;
    const float rate = raw ? expf(d.a_log[h]) : 0.f, bias = raw ? d.dt_bias[h] : 0.f;
    char* own = smem + Z::OWN;
    const uint32_t own_b = base + Z::OWN;
    float* diag = reinterpret_cast<float*>(own + Z::DIAG);
    float *ck = reinterpret_cast<float*>(own + Z::TOKENS), *cq = ck + CH, *gate = cq + CH;
    const int seg = tid % SEGS, row_in = tid / SEGS;
    const int quad = lane & 3, r8 = lane >> 2;
    const int b_row = (lane & 7) + ((lane >> 4) << 3), b_seg = (lane >> 3) & 1;      // B fragments of two tiles; A, transposed
    const int a_row = lane & 15, a_seg = lane >> 4;
    constexpr int sync = Z::PREPARING;

    // BF16 keys and queries: 8 values of ROWS rows of each in registers (rows past the end: the last one's).
    uint4 keys[ROWS], queries[ROWS];
    const auto load_rows = [&](uint4 (&x)[ROWS], const void* from, int64_t stride, int c) {
        const int last = min(CH, r.n - c * CH) - 1;
        const uint16_t* p = static_cast<const uint16_t*>(from) + ((int64_t)r.lo + (int64_t)c * CH) * stride + hk * DK + seg * 8;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) x[i] = *reinterpret_cast<const uint4*>(p + min(row_in + i * STEP, last) * stride);
    };
    // Values, and fp32 keys and queries, 16 bytes at a time straight into the stage.
    const auto load_values = [&](int c, uint32_t to) {
        constexpr int SIZE = F32 ? 4 : 2, PER = Z::VC * SIZE / 16;
        const int live = min(CH, r.n - c * CH);
        const int64_t stride = d.v_stride * SIZE;
        const char* v = static_cast<const char*>(d.v) + ((int64_t)r.lo + (int64_t)c * CH) * stride + (h * d.head_v + col0) * SIZE;
#pragma unroll 2
        for (int i = tid; i < CH * PER; i += PREP) {
            const int row = i / PER, part = i % PER;
            cp_16(to + row * Z::VP + part * 16, row < live ? v + row * stride + part * 16 : v, row < live);
        }
    };
    const auto load_pieces = [&](const void* from, int64_t stride, int c, uint32_t to) {
        const int live = min(CH, r.n - c * CH);
        const float* p = static_cast<const float*>(from) + ((int64_t)r.lo + (int64_t)c * CH) * stride + hk * DK + seg * 8;
#pragma unroll 2
        for (int row = row_in; row < CH; row += STEP) {
            const float* q = row < live ? p + row * stride : p;
            cp_16(to + Z::key_at(row, seg), q, row < live);
            cp_16(to + CH * Z::KP + Z::key_at(row, seg), q + 4, row < live);
        }
    };

    // A chunk's gates, two neighbouring tokens a lane of the last warp: as the call gives them, then what they come to.
    float ga[2] = {}, gb[2] = {};
    const auto load_gates = [&](int c) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int t = c * CH + 2 * lane + e;
            if (t < r.n) {
                ga[e] = gate_value(d.decay, d.gate_f32, ((int64_t)r.lo + t) * d.decay_stride + h);
                gb[e] = gate_value(d.beta, d.gate_f32, ((int64_t)r.lo + t) * d.beta_stride + h);
            }
        }
    };
    const auto sum_gates = [&](int c) {
        constexpr float LOG2E = 1.44269504f;
        const int t = 2 * lane, live = r.n - c * CH;
        Gate x0 = gate_of(ga[0], gb[0], raw, rate, bias), x1 = gate_of(ga[1], gb[1], raw, rate, bias);
        if (t >= live) x0 = {0.f, 0.f};
        if (t + 1 >= live) x1 = {0.f, 0.f};
        const uint64_t f1 = to_fixed(-x1.g * LOG2E);
        uint64_t sum = to_fixed(-x0.g * LOG2E) + f1;
#pragma unroll 1
        for (int o = 1; o < 32; o <<= 1) {
            const uint64_t x = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += x;
        }
        const uint64_t all = __shfl_sync(0xffffffffu, sum, 31), end = __shfl_sync(0xffffffffu, sum, lane | 7);   // of the chunk; of the token's 16
        // A NaN decay makes NaNs of the sums that it is in.
        const uint32_t odd = __ballot_sync(0xffffffffu, x0.g + x1.g != x0.g + x1.g);
        const float nan0 = (odd & ((2u << lane) - 1)) && (x0.g != x0.g || (odd & ((1u << lane) - 1))) ? __int_as_float(0x7fffffff) : 0.f;
        const float nan1 = odd & ((2u << lane) - 1) ? __int_as_float(0x7fffffff) : 0.f, nan = odd ? __int_as_float(0x7fffffff) : 0.f;
        const float2 u0 = from_fixed(sum - f1), u1 = from_fixed(sum);
        const auto put = [&](int what, float x, float y) { *reinterpret_cast<float2*>(gate + what * CH + t) = make_float2(x, y); };
        put(G_HI, u0.x + nan0, u1.x + nan1);
        put(G_LO, u0.y, u1.y);
        put(G_BETA, x0.beta, x1.beta);
        put(G_START, exp2f(u0.x + nan0), exp2f(u1.x + nan1));
        put(G_END, exp2f(from_fixed(all - sum + f1).x + nan), exp2f(from_fixed(all - sum).x + nan));
        put(G_BLOCK, exp2f(from_fixed(end - sum + f1).x + nan1), exp2f(from_fixed(end - sum).x + nan1));
        if (lane == 0) gate[G_LAST] = exp2f(from_fixed(all).x + nan);
    };

    int first = -1;                                     // a turn that only loads
    asm volatile("" : "+r"(first));                                 // unknown to the compiler, which would write that turn out on its own
#pragma unroll 1
    for (int c = first; c < chunks; ++c) {
        const int stage = c & (STAGES - 1);
        char* st = smem + stage * Z::STAGE;
        const uint32_t sb = base + stage * Z::STAGE;
        float* fac = reinterpret_cast<float*>(st + Z::FAC);
        const int next = c + 1;
        if (warp == PW - 1 && next < chunks) load_gates(next);
        if (c >= 0) {
            if constexpr (!F32 && !AHEAD) load_rows(keys, d.k, d.k_stride, c);
            bar_sync(Z::EMPTY + stage, Z::COUNT);
            load_values(c, sb + Z::V);
            // keys and queries to FP16 by a power of two a row; what a row's unit length makes of them
            if constexpr (F32) {
                load_pieces(d.k, d.k_stride, c, sb + Z::K);
                load_pieces(d.q, d.q_stride, c, sb + Z::Q);
                cp_wait_all();
            }
            if constexpr (F32) {
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {              // in place: each piece by the thread that loaded it
                    char* tile = st + (half ? Z::Q : Z::K);
#pragma unroll 1
                    for (int row = row_in; row < CH; row += STEP) {
                        uint4 *at = reinterpret_cast<uint4*>(tile + Z::key_at(row, seg)), *more = reinterpret_cast<uint4*>(tile + CH * Z::KP + Z::key_at(row, seg));
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
                // one power of two for a thread's rows, by their largest magnitude: what is below 2^-32 of it loses digits
                const auto convert = [&](uint4 (&x)[ROWS], char* tile, float* down) {
                    if (r.n - c * CH < CH)
#pragma unroll
                        for (int i = 0; i < ROWS; ++i)
                            if (row_in + i * STEP >= r.n - c * CH) x[i] = make_uint4(0, 0, 0, 0);
                    constexpr uint32_t MAGNITUDES = 0x7fff7fffu;
                    uint32_t m = 0;
#pragma unroll
                    for (int i = 0; i < ROWS; ++i)
                        m = __vmaxu2(__vmaxu2(m, __vmaxu2(x[i].x & MAGNITUDES, x[i].y & MAGNITUDES)), __vmaxu2(x[i].z & MAGNITUDES, x[i].w & MAGNITUDES));
#pragma unroll
                    for (int o = SEGS / 2; o; o >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
                    const float up = to_f16_range(__uint_as_float(max(m & 0xffffu, m >> 16) << 16)), inverse = pow2_inverse(up);
                    const auto two = [&](uint32_t w) { return pack_f16(__uint_as_float(w << 16) * up, __uint_as_float(w & 0xffff0000u) * up); };
                    char* to = tile + Z::key_at(row_in, seg);
#pragma unroll
                    for (int i = 0; i < ROWS; ++i) {
                        *reinterpret_cast<uint4*>(to + i * STEP * Z::KP) = make_uint4(two(x[i].x), two(x[i].y), two(x[i].z), two(x[i].w));
                        if (seg == 0) down[row_in + i * STEP] = inverse;
                    }
                };
                convert(keys, st + Z::K, ck);
                if constexpr (!AHEAD) load_rows(keys, d.q, d.q_stride, c);
                if constexpr (AHEAD) convert(queries, st + Z::Q, cq);
                else convert(keys, st + Z::Q, cq);
            }
            bar_sync(sync, PREP);
            // 16 rows of keys or of queries with the keys up to theirs. Four warps: of keys, then of queries, those of the warp
            // across, so that each has five blocks of 16 x 16 in all.
#pragma unroll 1
            for (int turn = 0; turn < 8 / PW; ++turn) {
                const bool of_q = PW == 8 ? warp >= 4 : turn;
                const int mt = PW == 8 ? warp & 3 : of_q ? 3 - warp : warp;
                float acc[8][4];
#pragma unroll
                for (int n = 0; n < 8; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[n][e] = 0.f;
                float squares[2][4] = {};                           // the rows' own block, for its diagonal
                const uint32_t a_at = sb + (of_q ? Z::Q : Z::K), a_in = Z::key_at(16 * mt + a_row, a_seg), own_in = Z::key_at(16 * mt + b_row, b_seg),
                               b_in = Z::key_at(b_row, b_seg);
                const auto products = [&](auto blocks) {            // with the keys of blocks 0 .. mt
                    constexpr int N = decltype(blocks)::value;
#pragma unroll(F32 ? 1 : DK / 16)
                    for (int kk = 0; kk < DK / 16; ++kk) {
                        uint32_t a[4], alo[4], b[N][4], l[4];
                        if constexpr (F32) {
                            ldmatrix4(a, a_at + Z::key_at(16 * mt + a_row, 2 * kk + a_seg));
                            ldmatrix4(alo, a_at + CH * Z::KP + Z::key_at(16 * mt + a_row, 2 * kk + a_seg));
                        } else {
                            ldmatrix4(a, a_at + a_in + 32 * kk);
                            if (of_q) ldmatrix4(l, a_at + own_in + 32 * kk);
                        }
#pragma unroll
                        for (int n2 = 0; n2 < N; ++n2)
                            ldmatrix4(b[n2], sb + Z::K + (F32 ? Z::key_at(16 * n2 + b_row, 2 * kk + b_seg) : b_in + 16 * n2 * Z::KP + 32 * kk));
                        if (!F32 && of_q) {
                            mma(squares[0], a, l[0], l[1]);
                            mma(squares[1], a, l[2], l[3]);
                        }
#pragma unroll
                        for (int n2 = 0; n2 < N; ++n2) {
                            mma(acc[2 * n2], a, b[n2][0], b[n2][1]);
                            mma(acc[2 * n2 + 1], a, b[n2][2], b[n2][3]);
                        }
                        if constexpr (F32) {
#pragma unroll
                            for (int n2 = 0; n2 < N; ++n2) {
                                mma(acc[2 * n2], alo, b[n2][0], b[n2][1]);
                                mma(acc[2 * n2 + 1], alo, b[n2][2], b[n2][3]);
                                ldmatrix4(l, sb + Z::KLO + Z::key_at(16 * n2 + b_row, 2 * kk + b_seg));
                                mma(acc[2 * n2], a, l[0], l[1]);
                                mma(acc[2 * n2 + 1], a, l[2], l[3]);
                            }
                        }
                    }
                    if (!F32 && !of_q)
#pragma unroll
                        for (int e = 0; e < 4; ++e) { squares[0][e] = acc[2 * N - 2][e]; squares[1][e] = acc[2 * N - 1][e]; }
                };
                switch (mt) {
                    case 0: products(std::integral_constant<int, 1>()); break;
                    case 1: products(std::integral_constant<int, 2>()); break;
                    case 2: products(std::integral_constant<int, 3>()); break;
                    default: products(std::integral_constant<int, 4>());
                }
                // the rows' factors, their unit lengths among them (BF16: from the diagonals, in the rows' own powers of two)
                const auto put = [&](int row, float x) {
                    float* unit = (of_q ? cq : ck) + row;
                    float f = *unit;
                    if (!F32) f *= d.normalize ? rsqrtf(x * f * f + DELTA_UNIT_EPS) : 1.f;
                    if (of_q) {
                        f *= d.scale;
                        fac[F_QUERY * CH + row] = gate[G_START * CH + row] * f;
                    } else {
                        const float g = gate[G_BETA * CH + row];
                        fac[F_BETA * CH + row] = g;
                        fac[F_STATE * CH + row] = g * gate[G_START * CH + row] * f;
                        fac[F_END * CH + row] = gate[G_END * CH + row] * f;
                    }
                    *unit = f;
                };
                if (2 * quad == (r8 & ~1)) {                        // columns 2 quad + e, rows r8 and r8 + 8
                    put(16 * mt + r8, r8 & 1 ? squares[0][1] : squares[0][0]);
                    put(16 * mt + r8 + 8, r8 & 1 ? squares[1][3] : squares[1][2]);
                }
                if (tid == 0) fac[F_LAST] = gate[G_LAST];
                if (PW == 8 || !of_q) bar_sync(sync, PREP);
                else __syncwarp();
                // -L or the scores: products times their tokens' factors and the decay between them. Across blocks of 16 the
                // decay is that from the column's token to its block's end times that from there on, both at most 1.
                const int i0 = 16 * mt + r8, i1 = i0 + 8;
                float m0 = 0.f, m1 = 0.f;
                {
                    const float *upto_hi = gate + G_HI * CH, *upto_lo = gate + G_LO * CH, *beta = gate + G_BETA * CH;
                    const float h0 = upto_hi[i0], h1 = upto_hi[i1], l0 = upto_lo[i0], l1 = upto_lo[i1];
                    const float s0 = of_q ? cq[i0] : -beta[i0] * ck[i0], s1 = of_q ? cq[i1] : -beta[i1] * ck[i1];
                    const int below = of_q ? 0 : 1;                 // below the diagonal, or up to it
#pragma unroll
                    for (int n2 = 0; n2 < 4; ++n2) {
                        if (n2 > mt) break;
                        const float he = upto_hi[16 * n2 + 15], le = upto_lo[16 * n2 + 15];
                        const float f0 = s0 * exp2_fast((h0 - he) + (l0 - le)), f1 = s1 * exp2_fast((h1 - he) + (l1 - le));
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            float(&x)[4] = acc[2 * n2 + p];
                            const int j0 = 16 * n2 + 8 * p + 2 * quad;
                            const float2 cj = *reinterpret_cast<const float2*>(ck + j0);
                            if (n2 < mt) {
                                const float2 ej = *reinterpret_cast<const float2*>(gate + G_BLOCK * CH + j0);
                                const float c0 = cj.x * ej.x, c1 = cj.y * ej.y;
                                x[0] *= c0 * f0; x[1] *= c1 * f0; x[2] *= c0 * f1; x[3] *= c1 * f1;
                            } else {
                                const float2 hj = *reinterpret_cast<const float2*>(upto_hi + j0), lj = *reinterpret_cast<const float2*>(upto_lo + j0);
                                x[0] = j0 + below <= i0 ? (s0 * cj.x) * exp2_fast((h0 - hj.x) + (l0 - lj.x)) * x[0] : 0.f;
                                x[1] = j0 + 1 + below <= i0 ? (s0 * cj.y) * exp2_fast((h0 - hj.y) + (l0 - lj.y)) * x[1] : 0.f;
                                x[2] = j0 + below <= i1 ? (s1 * cj.x) * exp2_fast((h1 - hj.x) + (l1 - lj.x)) * x[2] : 0.f;
                                x[3] = j0 + 1 + below <= i1 ? (s1 * cj.y) * exp2_fast((h1 - hj.y) + (l1 - lj.y)) * x[3] : 0.f;
                            }
                            m0 = fmaxf(m0, fmaxf(fabsf(x[0]), fabsf(x[1])));
                            m1 = fmaxf(m1, fmaxf(fabsf(x[2]), fabsf(x[3])));
                        }
                    }
                }
                if (of_q) {
                    const float p0 = to_f16_range(quad_max(m0)), p1 = to_f16_range(quad_max(m1));
                    if (quad == 0) {
                        fac[F_SCORE * CH + i0] = pow2_inverse(p0);
                        fac[F_SCORE * CH + i1] = pow2_inverse(p1);
                    }
#pragma unroll
                    for (int n = 0; n < 8; ++n) {
                        if (n > 2 * mt + 1) break;
                        *reinterpret_cast<uint32_t*>(st + Z::P + tile_at<Z::TP>(i0, n) + 4 * quad) = pack_f16(acc[n][0] * p0, acc[n][1] * p0);
                        *reinterpret_cast<uint32_t*>(st + Z::P + tile_at<Z::TP>(i1, n) + 4 * quad) = pack_f16(acc[n][2] * p1, acc[n][3] * p1);
                    }
                } else {
#pragma unroll
                    for (int n = 0; n < 8; ++n) {
                        if (n > 2 * mt + 1) break;
                        if (n < 2 * mt) {
                            uint32_t hi, lo;
                            split2(acc[n][0], acc[n][1], hi, lo);
                            *reinterpret_cast<uint32_t*>(own + Z::LHI + tile_at<Z::TP>(i0, n) + 4 * quad) = hi;
                            *reinterpret_cast<uint32_t*>(own + Z::LLO + tile_at<Z::TP>(i0, n) + 4 * quad) = lo;
                            split2(acc[n][2], acc[n][3], hi, lo);
                            *reinterpret_cast<uint32_t*>(own + Z::LHI + tile_at<Z::TP>(i1, n) + 4 * quad) = hi;
                            *reinterpret_cast<uint32_t*>(own + Z::LLO + tile_at<Z::TP>(i1, n) + 4 * quad) = lo;
                        } else {
                            float* o = diag + i0 * DP + 8 * (n - 2 * mt) + 2 * quad;
                            *reinterpret_cast<float2*>(o) = make_float2(acc[n][0], acc[n][1]);
                            *reinterpret_cast<float2*>(o + 8 * DP) = make_float2(acc[n][2], acc[n][3]);
                        }
                    }
                    // T's block on the diagonal (rows and columns 16 mt ..) by substitution, a column a lane
                    __syncwarp();
                    const float* D = diag + 16 * mt * DP;
                    const int col = lane & 15;
                    float x[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float t0 = i == col ? 1.f : 0.f, t1 = 0.f;
#pragma unroll
                        for (int m = 0; m < i; m += 4) {
                            const float4 l = *reinterpret_cast<const float4*>(D + i * DP + m);
                            t0 = fmaf(l.x, x[m], t0);
                            if (m + 1 < i) t1 = fmaf(l.y, x[m + 1], t1);
                            if (m + 2 < i) t0 = fmaf(l.z, x[m + 2], t0);
                            if (m + 3 < i) t1 = fmaf(l.w, x[m + 3], t1);
                        }
                        x[i] = i < col ? 0.f : t0 + t1;
                    }
                    // the first half of the lanes writes the high parts, the second the low ones
                    char* to = st + (lane < 16 ? Z::THI : Z::TLO) + 2 * (col & 7);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const __half hi = __float2half_rn(x[i]);
                        *reinterpret_cast<__half*>(to + tile_at<Z::TP>(16 * mt + i, 2 * mt + (col >> 3))) =
                            lane < 16 ? hi : __float2half_rn(x[i] - __half2float(hi));
                    }
                }
            }
            bar_sync(sync, PREP);
            if constexpr (AHEAD) {
                if (next < chunks) {
                    load_rows(keys, d.k, d.k_stride, next);
                    load_rows(queries, d.q, d.q_stride, next);
                }
            }
            // The blocks below the diagonal, T_ba = T_bb sum_(a <= c < b) (-L_bc) T_ca, block column a by warp a, transposed: each
            // T_ca^T is an A fragment as it comes out of the products.
            if (warp < 3) {
                uint32_t th[3][4], tl[3][4];
                ldmatrix4_trans(th[0], sb + Z::THI + tile_at<Z::TP>(16 * warp + b_row, 2 * warp + b_seg));
                ldmatrix4_trans(tl[0], sb + Z::TLO + tile_at<Z::TP>(16 * warp + b_row, 2 * warp + b_seg));
#pragma unroll
                for (int bi = 1; bi < 4; ++bi) {
                    const int b = warp + bi;
                    if (b > 3) break;
                    float x[2][4] = {}, y[2][4] = {};
                    uint32_t f[4] = {}, e[4] = {}, hi[4], lo[4];
                    const auto product = [&](const uint32_t (&ah)[4], const uint32_t (&al)[4]) {
                        mma(x[0], ah, f[0], f[1]);
                        mma(x[1], ah, f[2], f[3]);
                        mma(y[0], al, f[0], f[1]);
                        mma(y[1], al, f[2], f[3]);
                        mma(y[0], ah, e[0], e[1]);
                        mma(y[1], ah, e[2], e[3]);
                    };
                    const auto collect = [&] {
#pragma unroll
                        for (int p = 0; p < 2; ++p)
#pragma unroll
                            for (int i = 0; i < 4; ++i) { x[p][i] += y[p][i]; y[p][i] = 0.f; }
                        split_a(x[0], x[1], 1.f, 1.f, hi, lo);
#pragma unroll
                        for (int p = 0; p < 2; ++p)
#pragma unroll
                            for (int i = 0; i < 4; ++i) x[p][i] = 0.f;
                    };
#pragma unroll
                    for (int ci = 0; ci < bi; ++ci) {
                        ldmatrix4(f, own_b + Z::LHI + tile_at<Z::TP>(16 * b + b_row, 2 * (warp + ci) + b_seg));
                        ldmatrix4(e, own_b + Z::LLO + tile_at<Z::TP>(16 * b + b_row, 2 * (warp + ci) + b_seg));
                        product(th[ci], tl[ci]);
                    }
                    ldmatrix4(f, sb + Z::THI + tile_at<Z::TP>(16 * b + b_row, 2 * b + b_seg));
                    ldmatrix4(e, sb + Z::TLO + tile_at<Z::TP>(16 * b + b_row, 2 * b + b_seg));
                    collect();
                    product(hi, lo);
                    collect();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (bi < 3) { th[bi][i] = hi[i]; tl[bi][i] = lo[i]; }
                        const uint32_t at = tile_at<Z::TP>(16 * b + 8 * (i >> 1) + r8, 2 * warp + (i & 1)) + 4 * quad;
                        *reinterpret_cast<uint32_t*>(st + Z::THI + at) = movmatrix_trans(hi[i]);
                        *reinterpret_cast<uint32_t*>(st + Z::TLO + at) = movmatrix_trans(lo[i]);
                    }
                }
            } else if (warp == PW - 1 && next < chunks) {
                sum_gates(next);
            }
            if constexpr (!F32) cp_wait_all();
            bar_arrive(Z::FULL + stage, Z::COUNT);
        } else {
            if constexpr (AHEAD) {
                load_rows(keys, d.k, d.k_stride, next);
                load_rows(queries, d.q, d.q_stride, next);
            }
            if (warp == PW - 1) sum_gates(next);
        }
    }
}

// ---------------------------------------------------------------------------
// The chain: a warp, 16 columns.
// ---------------------------------------------------------------------------
template <bool F32, int DK, int CW, int PW>
__device__ __forceinline__ void run_chain(const Delta& d, const SeqRange& r, int h, int col0, char* smem, uint32_t base, int chunks) {
    using Z = Shape<F32, DK, CW, PW>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane & 3, r8 = lane >> 2;
    const int vcol = 16 * warp;
    float* state = d.state + ((int64_t)r.slot * d.heads + h) * DK * d.head_v + 2 * quad * d.head_v + col0 + vcol + r8;
    float S[DK / 8][4];                                             // [8 rows of S][columns r8, r8 + 8 x two rows]
    const float* from = state;
#pragma unroll
    for (int j = 0; j < DK / 8; ++j, from += 8 * d.head_v) {
        S[j][0] = r.fresh ? 0.f : from[0]; S[j][2] = r.fresh ? 0.f : from[8];
        S[j][1] = r.fresh ? 0.f : from[d.head_v]; S[j][3] = r.fresh ? 0.f : from[d.head_v + 8];
    }
    for (int i = 0; i < STAGES && i < chunks; ++i) bar_arrive(Z::EMPTY + i, Z::COUNT);
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
            sc0 = fmaxf(sc0, fmaxf(fabsf(S[j][0]), fabsf(S[j][1])));
            sc1 = fmaxf(sc1, fmaxf(fabsf(S[j][2]), fabsf(S[j][3])));
        }
        sc0 = to_f16_range(quad_max(sc0));
        sc1 = to_f16_range(quad_max(sc1));
        bar_sync(Z::FULL + stage, Z::COUNT);
        // S^T k and S^T q of every token
        float R[8][4], O[8][4];
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) R[n][e] = O[n][e] = 0.f;
        // fragments one step ahead of their products
        uint32_t fk[2][4][4], fq[4][4];
        const auto load4 = [&](uint32_t (&f)[4][4], int tile, int kk) {
#pragma unroll
            for (int n2 = 0; n2 < 4; ++n2) ldmatrix4(f[n2], sb + tile + Z::key_at(16 * n2 + b_row, 2 * kk + b_seg));
        };
        load4(fk[0], Z::K, 0);
#pragma unroll
        for (int kk = 0; kk < DK / 16; ++kk) {
            uint32_t hi[4], lo[4];
            uint32_t (&b)[4][4] = fk[kk & 1];
            split_a(S[2 * kk], S[2 * kk + 1], sc0, sc1, hi, lo);
            load4(fq, Z::Q, kk);
#pragma unroll
            for (int n = 0; n < 8; ++n) mma(R[n], hi, b[n >> 1][2 * (n & 1)], b[n >> 1][2 * (n & 1) + 1]);
            if (!F32 && kk + 1 < DK / 16) load4(fk[(kk + 1) & 1], Z::K, kk + 1);
            if (F32) load4(fk[(kk + 1) & 1], Z::KLO, kk);
#pragma unroll
            for (int n = 0; n < 8; ++n) mma(R[n], lo, b[n >> 1][2 * (n & 1)], b[n >> 1][2 * (n & 1) + 1]);
            if constexpr (F32) {
                uint32_t (&l)[4][4] = fk[(kk + 1) & 1];
#pragma unroll
                for (int n = 0; n < 8; ++n) mma(R[n], hi, l[n >> 1][2 * (n & 1)], l[n >> 1][2 * (n & 1) + 1]);
                if (kk + 1 < DK / 16) load4(fk[(kk + 1) & 1], Z::K, kk + 1);
            }
#pragma unroll
            for (int n = 0; n < 8; ++n) mma(O[n], hi, fq[n >> 1][2 * (n & 1)], fq[n >> 1][2 * (n & 1) + 1]);
        }
        // R = beta v - beta e^G (S^T k); the queries' part of the outputs
        const float is0 = pow2_inverse(sc0), is1 = pow2_inverse(sc1);
        float m0 = 0.f, m1 = 0.f, odd0 = 0.f, odd1 = 0.f;
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
                const float2 fb = *reinterpret_cast<const float2*>(fac + F_BETA * CH + t), fs = *reinterpret_cast<const float2*>(fac + F_STATE * CH + t),
                             fq = *reinterpret_cast<const float2*>(fac + F_QUERY * CH + t);
                R[n][0] = fb.x * v0[0] - (fs.x * is0) * R[n][0];
                R[n][1] = fb.y * v0[1] - (fs.y * is0) * R[n][1];
                R[n][2] = fb.x * v1[0] - (fs.x * is1) * R[n][2];
                R[n][3] = fb.y * v1[1] - (fs.y * is1) * R[n][3];
                O[n][0] *= fq.x * is0; O[n][1] *= fq.y * is0;
                O[n][2] *= fq.x * is1; O[n][3] *= fq.y * is1;
                m0 = fmaxf(m0, fmaxf(fabsf(R[n][0]), fabsf(R[n][1])));
                m1 = fmaxf(m1, fmaxf(fabsf(R[n][2]), fabsf(R[n][3])));
                odd0 = fmaf(R[n][0], 0.f, fmaf(R[n][1], 0.f, odd0));
                odd1 = fmaf(R[n][2], 0.f, fmaf(R[n][3], 0.f, odd1));
            }
        }
        int bad0 = CH, bad1 = CH;                                   // the first tokens whose R is not finite
        const bool odd = __any_sync(0xffffffffu, !(odd0 == 0.f) || !(odd1 == 0.f));
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
        const float rs0 = to_f16_range(quad_max(m0)), rs1 = to_f16_range(quad_max(m1));
        // U^T = R^T T^T, 16 tokens at a time from the last: a block of U takes the place of the block of R that no other needs
        uint32_t rh[4][4], rl[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) split_a(R[2 * j], R[2 * j + 1], rs0, rs1, rh[j], rl[j]);
        const float ir0 = pow2_inverse(rs0), ir1 = pow2_inverse(rs1);
        float u0 = 0.f, u1 = 0.f;
#pragma unroll
        for (int i = 3; i >= 0; --i) {
            float x[2][4] = {};
#pragma unroll
            for (int j = 0; j <= i; ++j) {
                const uint32_t at = tile_at<Z::TP>(16 * i + b_row, 2 * j + b_seg);
                uint32_t b[4];
                ldmatrix4(b, sb + Z::THI + at);
                mma(x[0], rh[j], b[0], b[1]);
                mma(x[1], rh[j], b[2], b[3]);
                mma(x[0], rl[j], b[0], b[1]);
                mma(x[1], rl[j], b[2], b[3]);
                ldmatrix4(b, sb + Z::TLO + at);
                mma(x[0], rh[j], b[0], b[1]);
                mma(x[1], rh[j], b[2], b[3]);
            }
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                R[2 * i + p][0] = x[p][0] * ir0; R[2 * i + p][1] = x[p][1] * ir0;
                R[2 * i + p][2] = x[p][2] * ir1; R[2 * i + p][3] = x[p][3] * ir1;
            }
        }
        if (odd) {
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int t = 8 * n + 2 * quad + e;
                    if (t >= bad0) R[n][e] = 0.f;
                    if (t >= bad1) R[n][2 + e] = 0.f;
                }
        }
        float e0 = 0.f, e1 = 0.f;                                   // of U, and of U as the state takes it
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const float2 fe = *reinterpret_cast<const float2*>(fac + F_END * CH + 8 * n + 2 * quad);
            u0 = fmaxf(u0, fmaxf(fabsf(R[n][0]), fabsf(R[n][1])));
            u1 = fmaxf(u1, fmaxf(fabsf(R[n][2]), fabsf(R[n][3])));
            e0 = fmaxf(e0, fmaxf(fabsf(R[n][0] * fe.x), fabsf(R[n][1] * fe.y)));
            e1 = fmaxf(e1, fmaxf(fabsf(R[n][2] * fe.x), fabsf(R[n][3] * fe.y)));
        }
        const float us0 = to_f16_range(quad_max(u0)), us1 = to_f16_range(quad_max(u1));
        const float es0 = to_f16_range(quad_max(e0)), es1 = to_f16_range(quad_max(e1));
        // O^T += U^T P^T
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float s = e & 1 ? us1 : us0;
                rh[j][e] = pack_f16(R[2 * j + (e >> 1)][2 * (e & 1)] * s, R[2 * j + (e >> 1)][2 * (e & 1) + 1] * s);
            }
        const float iu0 = pow2_inverse(us0), iu1 = pow2_inverse(us1);
        const int64_t row0 = (int64_t)r.lo + (int64_t)c * CH;
        const int live = min(CH, r.n - c * CH);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[2][4] = {};
#pragma unroll
            for (int j = 0; j <= i; ++j) {
                uint32_t b[4];
                ldmatrix4(b, sb + Z::P + tile_at<Z::TP>(16 * i + b_row, 2 * j + b_seg));
                mma(x[0], rh[j], b[0], b[1]);
                mma(x[1], rh[j], b[2], b[3]);
            }
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int n = 2 * i + p, t = 8 * n + 2 * quad;
                const float2 fp = *reinterpret_cast<const float2*>(fac + F_SCORE * CH + t);
                float y[4] = {fmaf(x[p][0], fp.x * iu0, O[n][0]), fmaf(x[p][1], fp.y * iu0, O[n][1]), fmaf(x[p][2], fp.x * iu1, O[n][2]),
                              fmaf(x[p][3], fp.y * iu1, O[n][3])};
                if (odd) {
                    const float nan = __int_as_float(0x7fffffff);
                    if (t >= bad0) y[0] = nan;
                    if (t + 1 >= bad0) y[1] = nan;
                    if (t >= bad1) y[2] = nan;
                    if (t + 1 >= bad1) y[3] = nan;
                }
                const uint32_t a = movmatrix_trans(pack_bf16(y[0], y[1])), b = movmatrix_trans(pack_bf16(y[2], y[3]));
                const int row = 8 * n + r8;
                if (row < live) {
                    uint16_t* o = d.out + ((row0 + row) * d.heads + h) * d.head_v + col0 + vcol + 2 * quad;
                    *reinterpret_cast<uint32_t*>(o) = a;
                    *reinterpret_cast<uint32_t*>(o + 8) = b;
                }
            }
        }
        // S^T <- e^G S^T + U^T k
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int n = 2 * j + (e >> 1);
                const float2 fe = *reinterpret_cast<const float2*>(fac + F_END * CH + 8 * n + 2 * quad);
                const float s = e & 1 ? es1 : es0;
                split2(R[n][2 * (e & 1)] * fe.x * s, R[n][2 * (e & 1) + 1] * fe.y * s, rh[j][e], rl[j][e]);
            }
        const float ie0 = pow2_inverse(es0), ie1 = pow2_inverse(es1);
        const float last = fac[F_LAST];
        uint32_t fu[2][2][4];
        const auto load2 = [&](uint32_t (&f)[2][4], int tile, int step) {           // 16 tokens by four tiles of S
#pragma unroll
            for (int p = 0; p < 2; ++p)
                ldmatrix4_trans(f[p], sb + tile + Z::key_at(16 * (step & 3) + t_row, 4 * (step >> 2) + 2 * p + t_seg));
        };
        load2(fu[0], Z::K, 0);
#pragma unroll
        for (int j4 = 0; j4 < DK / 32; ++j4) {                       // four tiles of S at a time
            float x[4][4] = {};
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                const int step = 4 * j4 + kk;
                uint32_t (&b)[2][4] = fu[step & 1], (&next)[2][4] = fu[(step + 1) & 1];
                if (F32) load2(next, Z::KLO, step);
                else if (step + 1 < DK / 8) load2(next, Z::K, step + 1);
#pragma unroll
                for (int p = 0; p < 4; ++p) mma(x[p], rh[kk], b[p >> 1][2 * (p & 1)], b[p >> 1][2 * (p & 1) + 1]);
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
                s[0] = fmaf(last, s[0], x[p][0] * ie0); s[1] = fmaf(last, s[1], x[p][1] * ie0);
                s[2] = fmaf(last, s[2], x[p][2] * ie1); s[3] = fmaf(last, s[3], x[p][3] * ie1);
            }
        }
        if (odd) {
            const float nan = __int_as_float(0x7fffffff);
#pragma unroll
            for (int j = 0; j < DK / 8; ++j) {
                if (bad0 < CH) S[j][0] = S[j][1] = nan;
                if (bad1 < CH) S[j][2] = S[j][3] = nan;
            }
        }
        if (c + STAGES < chunks) bar_arrive(Z::EMPTY + stage, Z::COUNT);
    }
#pragma unroll
    for (int j = 0; j < DK / 8; ++j, state += 8 * d.head_v) {
        state[0] = S[j][0]; state[8] = S[j][2];
        state[d.head_v] = S[j][1]; state[d.head_v + 8] = S[j][3];
    }
}

template <bool F32, int DK, int CW, int PW>
__global__ void __launch_bounds__(Shape<F32, DK, CW, PW>::THREADS, 1) delta_chunk_kernel(Delta d, int above) {
    using Z = Shape<F32, DK, CW, PW>;
    extern __shared__ __align__(128) char smem[];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int slices = d.head_v / Z::VC;
    const int unit = (int)(blockIdx.x / slices), slice = (int)(blockIdx.x - unit * slices);
    const int b = unit / d.heads, h = unit - b * d.heads, col0 = slice * Z::VC;
    const SeqRange r = seq_range(d.seq, b, d.n_slots, h == 0 && slice == 0 && threadIdx.x == 0);
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
        if (CW == 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        if (threadIdx.x < 32 * CW) run_chain<F32, DK, CW, PW>(d, r, h, col0, smem, base, chunks);
    } else {
        if (CW == 8) asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 136;");
        prepare_chunks<F32, DK, CW, PW>(d, r, h, col0, smem, base, chunks);
    }
}

template <bool F32, int DK, int CW, int PW>
cudaError_t launch_shape(const Delta& d, int above, cudaStream_t s) {
    using Z = Shape<F32, DK, CW, PW>;
    static_assert(Z::BYTES <= 227 * 1024, "stages must fit");
    const auto kernel = delta_chunk_kernel<F32, DK, CW, PW>;
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
    // narrower ones fill the GPU. A chunk takes a block of 32, 64 or 128 columns about 6.7, 7.1 and 11.5 us; the rounds of
    // blocks are counted by the sequences like the longest that the tokens make up. Five sequences of 1774 to 3001 tokens, 32
    // heads of 128: 1202, 737 and 695 us; one of 32768: 3.5, 3.6 and 6.0 ms.
    if constexpr (!F32) {
        const int64_t alike = (d.seq.tokens + d.seq.rows / 2) / d.seq.rows, sequences = alike < 1 ? 1 : alike > d.seq.batch ? d.seq.batch : alike;
        const auto cost = [&](int columns, int64_t each) { return (sequences * d.heads * d.head_v / columns + sms - 1) / sms * each; };
        const int64_t narrow = cost(32, 67), middle = cost(64, 71), wide = d.head_v % 128 == 0 ? cost(128, 115) : INT64_MAX;
        if (wide < narrow && wide < middle) return launch_shape<F32, DK, 8, 4>(d, above, s);
        if (middle < narrow) return launch_shape<F32, DK, 4, 8>(d, above, s);
    }
    return launch_shape<F32, DK, 2, 8>(d, above, s);
}

}  // namespace

cudaError_t launch_delta_chunks(const Delta& d, int above, int sms, cudaStream_t s) {
    if (d.f32) return d.head_k == 64 ? launch_width<true, 64>(d, above, sms, s) : launch_width<true, 128>(d, above, sms, s);
    return d.head_k == 64 ? launch_width<false, 64>(d, above, sms, s) : launch_width<false, 128>(d, above, sms, s);
}

cudaError_t read_device_status_delta_chunks(uint32_t* status) {
    cudaError_t e = cudaMemcpyFromSymbol(status, g_device_status, sizeof(uint32_t));
    if (e != cudaSuccess || *status == 0) return e;
    const uint32_t zero = 0;
    return cudaMemcpyToSymbol(g_device_status, &zero, sizeof(uint32_t));
}

}  // namespace vbq
