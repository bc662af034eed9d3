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
#include <cuda_fp16.h>

#include "vbq_delta.cuh"
#include "vbq_kernels.h"

namespace vbq {
namespace {

constexpr int CH = 64;                           // tokens of a chunk
constexpr int STAGES = 2;
constexpr int LP = 68;                           // floats between rows of the fp32 scratch matrices

__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" :: "r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int threads) { asm volatile("bar.arrive %0, %1;" :: "r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
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

template <bool F32, int DK, int CW, int GROUPS>
struct Shape {
    static constexpr int VC = 16 * CW;                              // columns of a block
    static constexpr int KP = 2 * DK;                               // bytes of a key row in FP16
    static constexpr int VP = F32 ? 4 * (VC + 4) : 2 * VC;
    static constexpr int THREADS = 32 * (CW + 4 * GROUPS);
    // a stage
    static constexpr int K = 0, KLO = K + CH * KP, Q = KLO + (F32 ? CH * KP : 0), V = Q + CH * KP, THI = V + CH * VP, TLO = THI + CH * 2 * CH,
                         P = TLO + CH * 2 * CH, FAC = P + CH * 2 * CH, STAGE = FAC + (6 * CH + 4) * 4;
    // a group's scratch: L, then the fp32 inverse's blocks
    static constexpr int SCRATCH = STAGES * STAGE, SCRATCH_BYTES = (CH * LP + 32 * LP) * 4 + 5 * CH * 4 + 16;
    static constexpr int BYTES = SCRATCH + GROUPS * SCRATCH_BYTES;
};
// what a stage tells about its tokens
enum { F_BETA, F_STATE, F_END, F_QUERY, F_SCORE };                  // and from F_LAST on: e^G_last
constexpr int F_LAST = 6 * CH;

template <int CW, int GROUPS>
struct Bars {
    static constexpr int COUNT = 32 * CW + 128;
    __device__ static int full(int stage) { return 1 + stage; }
    __device__ static int empty(int stage) { return 1 + STAGES + stage; }
    __device__ static int group(int g) { return 1 + 2 * STAGES + g; }
};

// ---------------------------------------------------------------------------
// Preparing a chunk: 128 threads.
// ---------------------------------------------------------------------------

// 8 values of a row to FP16 by a power of two of the row's largest; returns (scale, sum of squares). LANES neighbours share the row.
template <int LANES>
__device__ __forceinline__ float2 row_stats(const float (&x)[8]) {
    float m = 0.f, s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        m = fmaxf(m, fabsf(x[e]));
        s = fmaf(x[e], x[e], s);
    }
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) {
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        s += __shfl_xor_sync(0xffffffffu, s, o);
    }
    return make_float2(to_f16_range(m), s);
}

template <bool F32, int DK, int CW, int GROUPS>
__device__ __forceinline__ void prepare_chunks(const Delta& d, const SeqRange& r, int h, int col0, char* smem, uint32_t base, int g, int chunks) {
    using Z = Shape<F32, DK, CW, GROUPS>;
    using B = Bars<CW, GROUPS>;
    constexpr int SEGS = DK / 8, ROWS = 128 / SEGS, TURNS = CH / ROWS;
    const int tid = (threadIdx.x - 32 * CW) & 127, warp = tid >> 5, lane = tid & 31;
    const int hk = h / (d.heads / d.k_heads);
    const bool raw = d.a_log != nullptr;
    const float rate = raw ? expf(d.a_log[h]) : 0.f, bias = raw ? d.dt_bias[h] : 0.f;
    float* L = reinterpret_cast<float*>(smem + Z::SCRATCH + g * Z::SCRATCH_BYTES);
    float* Y = L + CH * LP;
    float *upto_hi = Y + 32 * LP, *upto_lo = upto_hi + CH, *beta = upto_lo + CH, *ck = beta + CH, *cq = ck + CH;
    const int seg = tid % SEGS, row_in = tid / SEGS;
    for (int c = g; c < chunks; c += GROUPS) {
        const int stage = c % STAGES;
        const int64_t row0 = (int64_t)r.lo + (int64_t)c * CH;
        const int live = min(CH, r.n - c * CH);
        char* st = smem + stage * Z::STAGE;
        const uint32_t sb = base + stage * Z::STAGE;
        float* fac = reinterpret_cast<float*>(st + Z::FAC);
        // the gates: two neighbouring tokens a lane, their sums in 64 bits (a decay of e^-100 among slow ones would cost the others their digits)
        double g0 = 0, g1 = 0;
        float b0 = 0.f, b1 = 0.f;
        if (warp == 0) {
            const int t = 2 * lane;
            if (t < live) {
                const Gate x = gate_of(gate_value(d.decay, d.gate_f32, (row0 + t) * d.decay_stride + h),
                                       gate_value(d.beta, d.gate_f32, (row0 + t) * d.beta_stride + h), raw, rate, bias);
                g0 = x.g; b0 = x.beta;
            }
            if (t + 1 < live) {
                const Gate x = gate_of(gate_value(d.decay, d.gate_f32, (row0 + t + 1) * d.decay_stride + h),
                                       gate_value(d.beta, d.gate_f32, (row0 + t + 1) * d.beta_stride + h), raw, rate, bias);
                g1 = x.g; b1 = x.beta;
            }
        }
        if (c >= STAGES) bar_sync(B::empty(stage), B::COUNT);
        // keys and queries
        for (int half = 0; half < 2; ++half) {
            const void* src = half ? d.q : d.k;
            const int64_t stride = half ? d.q_stride : d.k_stride;
            float* cs = half ? cq : ck;
            const int at = half ? Z::Q : Z::K;
#pragma unroll
            for (int i = 0; i < TURNS; ++i) {
                const int row = row_in + i * ROWS;
                float x[8] = {};
                if (row < live) load8<F32>(x, src, (row0 + row) * stride + hk * DK + seg * 8);
                const float2 rs = row_stats<SEGS>(x);
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) split2(x[2 * e] * rs.x, x[2 * e + 1] * rs.x, hi[e], lo[e]);
                *reinterpret_cast<uint4*>(st + at + tile_at<Z::KP>(row, seg)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                if (F32 && !half) *reinterpret_cast<uint4*>(st + Z::KLO + tile_at<Z::KP>(row, seg)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                if (seg == 0) {
                    float f = pow2_inverse(rs.x);
                    if (d.normalize) f *= 1.f / sqrtf(rs.y + DELTA_UNIT_EPS);
                    cs[row] = half ? f * d.scale : f;
                }
            }
        }
        // values
        if constexpr (F32) {
            constexpr int PER = Z::VC / 4;
            for (int i = tid; i < CH * PER; i += 128) {
                const int row = i / PER, s = i % PER;
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                if (row < live)
                    x = *reinterpret_cast<const float4*>(static_cast<const float*>(d.v) + (row0 + row) * d.v_stride + h * d.head_v + col0 + s * 4);
                *reinterpret_cast<float4*>(st + Z::V + row * Z::VP + s * 16) = x;
            }
        } else {
            constexpr int PER = Z::VC / 8;
            for (int i = tid; i < CH * PER; i += 128) {
                const int row = i / PER, s = i % PER;
                uint4 x = make_uint4(0, 0, 0, 0);
                if (row < live)
                    x = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(d.v) + (row0 + row) * d.v_stride + h * d.head_v + col0 + s * 8);
                *reinterpret_cast<uint4*>(st + Z::V + tile_at<Z::VP>(row, s)) = x;
            }
        }
        if (warp == 0) {
            constexpr double LOG2E = 1.4426950408889634;
            double sum = g0 + g1;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double x = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += x;
            }
            const double all = __shfl_sync(0xffffffffu, sum, 31) * LOG2E;
            const double u1 = sum * LOG2E, u0 = (sum - g1) * LOG2E;
            const int t = 2 * lane;
            upto_hi[t] = (float)u0; upto_hi[t + 1] = (float)u1;
            upto_lo[t] = (float)(u0 - (float)u0); upto_lo[t + 1] = (float)(u1 - (float)u1);
            beta[t] = b0; beta[t + 1] = b1;
            fac[F_BETA * CH + t] = b0; fac[F_BETA * CH + t + 1] = b1;
            fac[F_STATE * CH + t] = b0 * exp2f((float)u0); fac[F_STATE * CH + t + 1] = b1 * exp2f((float)u1);
            fac[F_QUERY * CH + t] = exp2f((float)u0); fac[F_QUERY * CH + t + 1] = exp2f((float)u1);
            fac[F_END * CH + t] = exp2f((float)(all - u0)); fac[F_END * CH + t + 1] = exp2f((float)(all - u1));
            if (lane == 0) fac[F_LAST] = exp2f((float)all);
        }
        bar_sync(B::group(g), 128);
        // the tokens' other factors
        if (tid < CH) {
            fac[F_STATE * CH + tid] *= ck[tid];
            fac[F_END * CH + tid] *= ck[tid];
        } else {
            fac[F_QUERY * CH + tid - CH] *= cq[tid - CH];
        }
        // keys with keys (16 rows: this warp's) and queries with keys (the rows of the warp across, so that each has ten tiles)
        const int quad = lane & 3, r8 = lane >> 2;
        const uint32_t b_row = (uint32_t)((lane & 7) + ((lane >> 4) << 3)), b_seg = (lane >> 3) & 1;     // B fragments of two tiles
        const uint32_t a_row = (uint32_t)(lane & 15), a_seg = lane >> 4;
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            const int mt = half ? 3 - warp : warp;
            float acc[8][4];
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[n][e] = 0.f;
#pragma unroll
            for (int kk = 0; kk < DK / 16; ++kk) {
                uint32_t a[4], alo[4];
                ldmatrix4(a, sb + (half ? Z::Q : Z::K) + tile_at<Z::KP>(16 * mt + a_row, 2 * kk + a_seg));
                if (F32 && !half) ldmatrix4(alo, sb + Z::KLO + tile_at<Z::KP>(16 * mt + a_row, 2 * kk + a_seg));
#pragma unroll
                for (int n2 = 0; n2 < 4; ++n2) {
                    if (n2 > mt) break;
                    uint32_t b[4];
                    ldmatrix4(b, sb + Z::K + tile_at<Z::KP>(16 * n2 + b_row, 2 * kk + b_seg));
                    mma(acc[2 * n2], a, b[0], b[1]);
                    mma(acc[2 * n2 + 1], a, b[2], b[3]);
                    if (F32 && !half) {
                        mma(acc[2 * n2], alo, b[0], b[1]);
                        mma(acc[2 * n2 + 1], alo, b[2], b[3]);
                        ldmatrix4(b, sb + Z::KLO + tile_at<Z::KP>(16 * n2 + b_row, 2 * kk + b_seg));
                        mma(acc[2 * n2], a, b[0], b[1]);
                        mma(acc[2 * n2 + 1], a, b[2], b[3]);
                    }
                }
            }
            const int i0 = 16 * mt + r8, i1 = i0 + 8;
            const float h0 = upto_hi[i0], h1 = upto_hi[i1], l0 = upto_lo[i0], l1 = upto_lo[i1];
            const float s0 = half ? cq[i0] : beta[i0] * ck[i0], s1 = half ? cq[i1] : beta[i1] * ck[i1];
            float m0 = 0.f, m1 = 0.f;
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                if (n > 2 * mt + 1) break;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int j = 8 * n + 2 * quad + e;
                    const float hj = upto_hi[j], lj = upto_lo[j], cj = ck[j];
                    const bool in0 = half ? j <= i0 : j < i0, in1 = half ? j <= i1 : j < i1;
                    acc[n][e] = in0 ? s0 * cj * exp2f((h0 - hj) + (l0 - lj)) * acc[n][e] : 0.f;
                    acc[n][2 + e] = in1 ? s1 * cj * exp2f((h1 - hj) + (l1 - lj)) * acc[n][2 + e] : 0.f;
                    m0 = fmaxf(m0, fabsf(acc[n][e]));
                    m1 = fmaxf(m1, fabsf(acc[n][2 + e]));
                }
            }
            if (!half) {
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    if (n > 2 * mt + 1) break;
                    *reinterpret_cast<float2*>(L + i0 * LP + 8 * n + 2 * quad) = make_float2(acc[n][0], acc[n][1]);
                    *reinterpret_cast<float2*>(L + i1 * LP + 8 * n + 2 * quad) = make_float2(acc[n][2], acc[n][3]);
                }
            } else {
                const float p0 = to_f16_range(quad_max(m0)), p1 = to_f16_range(quad_max(m1));
                if (quad == 0) {
                    fac[F_SCORE * CH + i0] = pow2_inverse(p0);
                    fac[F_SCORE * CH + i1] = pow2_inverse(p1);
                }
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    if (n > 2 * mt + 1) break;
                    *reinterpret_cast<uint32_t*>(st + Z::P + tile_at<2 * CH>(i0, n) + 4 * quad) = pack_f16(acc[n][0] * p0, acc[n][1] * p0);
                    *reinterpret_cast<uint32_t*>(st + Z::P + tile_at<2 * CH>(i1, n) + 4 * quad) = pack_f16(acc[n][2] * p1, acc[n][3] * p1);
                }
            }
        }
        bar_sync(B::group(g), 128);
        // T = (1 + L)^-1 by 32 x 32 blocks: those on the diagonal by substitution, a column a lane; then -T22 (L21 T11)
        const auto put_t = [&](int i, int j, float x) {
            const __half hi = __float2half_rn(x);
            const uint32_t o = tile_at<2 * CH>(i, j >> 3) + 2 * (j & 7);
            *reinterpret_cast<__half*>(st + Z::THI + o) = hi;
            *reinterpret_cast<__half*>(st + Z::TLO + o) = __float2half_rn(x - __half2float(hi));
        };
        if (warp < 2) {
            const float* D = L + 32 * warp * LP + 32 * warp;
            float x[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                float s0 = i == lane ? 1.f : 0.f, s1 = 0.f;
#pragma unroll
                for (int m = 0; m < i; m += 4) {
                    const float4 l = *reinterpret_cast<const float4*>(D + i * LP + m);
                    s0 = fmaf(-l.x, x[m], s0);
                    if (m + 1 < i) s1 = fmaf(-l.y, x[m + 1], s1);
                    if (m + 2 < i) s0 = fmaf(-l.z, x[m + 2], s0);
                    if (m + 3 < i) s1 = fmaf(-l.w, x[m + 3], s1);
                }
                x[i] = i < lane ? 0.f : s0 + s1;
            }
            __syncwarp();
            // over L's own block, which is not read again
            float* O = L + 32 * warp * LP + 32 * warp + lane;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                O[i * LP] = x[i];
                put_t(32 * warp + i, 32 * warp + lane, x[i]);
            }
        }
        bar_sync(B::group(g), 128);
        {
            const int i = tid >> 2, j = (tid & 3) * 8;
            float y[8] = {};
#pragma unroll 8
            for (int m = 0; m < 32; ++m) {
                const float l = L[(32 + i) * LP + m];
                const float4 a = *reinterpret_cast<const float4*>(L + m * LP + j), b = *reinterpret_cast<const float4*>(L + m * LP + j + 4);
                y[0] = fmaf(l, a.x, y[0]); y[1] = fmaf(l, a.y, y[1]); y[2] = fmaf(l, a.z, y[2]); y[3] = fmaf(l, a.w, y[3]);
                y[4] = fmaf(l, b.x, y[4]); y[5] = fmaf(l, b.y, y[5]); y[6] = fmaf(l, b.z, y[6]); y[7] = fmaf(l, b.w, y[7]);
            }
            *reinterpret_cast<float4*>(Y + i * LP + j) = make_float4(y[0], y[1], y[2], y[3]);
            *reinterpret_cast<float4*>(Y + i * LP + j + 4) = make_float4(y[4], y[5], y[6], y[7]);
            bar_sync(B::group(g), 128);
            float z[8] = {};
#pragma unroll 8
            for (int m = 0; m < 32; ++m) {
                const float l = -L[(32 + i) * LP + 32 + m];
                const float4 a = *reinterpret_cast<const float4*>(Y + m * LP + j), b = *reinterpret_cast<const float4*>(Y + m * LP + j + 4);
                z[0] = fmaf(l, a.x, z[0]); z[1] = fmaf(l, a.y, z[1]); z[2] = fmaf(l, a.z, z[2]); z[3] = fmaf(l, a.w, z[3]);
                z[4] = fmaf(l, b.x, z[4]); z[5] = fmaf(l, b.y, z[5]); z[6] = fmaf(l, b.z, z[6]); z[7] = fmaf(l, b.w, z[7]);
            }
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) split2(z[2 * e], z[2 * e + 1], hi[e], lo[e]);
            const uint32_t o = tile_at<2 * CH>(32 + i, j >> 3);
            *reinterpret_cast<uint4*>(st + Z::THI + o) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            *reinterpret_cast<uint4*>(st + Z::TLO + o) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        bar_arrive(B::full(stage), B::COUNT);
    }
}

// ---------------------------------------------------------------------------
// The chain: a warp, 16 columns.
// ---------------------------------------------------------------------------
template <bool F32, int DK, int CW, int GROUPS>
__device__ __forceinline__ void run_chain(const Delta& d, const SeqRange& r, int h, int col0, char* smem, uint32_t base, int chunks) {
    using Z = Shape<F32, DK, CW, GROUPS>;
    using B = Bars<CW, GROUPS>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane & 3, r8 = lane >> 2;
    const int vcol = 16 * warp;
    float* state = d.state + ((int64_t)r.slot * d.heads + h) * DK * d.head_v + col0 + vcol + r8;
    float S[DK / 8][4];                                             // [8 rows of S][columns r8, r8 + 8 x two rows]
#pragma unroll
    for (int j = 0; j < DK / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            S[j][e] = r.fresh ? 0.f : state[(int64_t)(8 * j + 2 * quad + (e & 1)) * d.head_v + (e >> 1) * 8];
    const uint32_t b_row = (uint32_t)((lane & 7) + ((lane >> 4) << 3)), b_seg = (lane >> 3) & 1;       // two tiles of tokens
    const uint32_t t_row = (uint32_t)((lane & 7) + (((lane >> 3) & 1) << 3)), t_seg = lane >> 4;       // transposed: 16 tokens, two tiles of columns
    for (int c = 0; c < chunks; ++c) {
        const int stage = c % STAGES;
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
        bar_sync(B::full(stage), B::COUNT);
        // S^T k and S^T q of every token
        float R[8][4], O[8][4];
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) R[n][e] = O[n][e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < DK / 16; ++kk) {
            uint32_t hi[4], lo[4];
            split2(S[2 * kk][0] * sc0, S[2 * kk][1] * sc0, hi[0], lo[0]);
            split2(S[2 * kk][2] * sc1, S[2 * kk][3] * sc1, hi[1], lo[1]);
            split2(S[2 * kk + 1][0] * sc0, S[2 * kk + 1][1] * sc0, hi[2], lo[2]);
            split2(S[2 * kk + 1][2] * sc1, S[2 * kk + 1][3] * sc1, hi[3], lo[3]);
#pragma unroll
            for (int n2 = 0; n2 < 4; ++n2) {
                const uint32_t at = tile_at<Z::KP>(16 * n2 + b_row, 2 * kk + b_seg);
                uint32_t b[4];
                ldmatrix4(b, sb + Z::K + at);
                mma(R[2 * n2], hi, b[0], b[1]);
                mma(R[2 * n2 + 1], hi, b[2], b[3]);
                mma(R[2 * n2], lo, b[0], b[1]);
                mma(R[2 * n2 + 1], lo, b[2], b[3]);
                if constexpr (F32) {
                    ldmatrix4(b, sb + Z::KLO + at);
                    mma(R[2 * n2], hi, b[0], b[1]);
                    mma(R[2 * n2 + 1], hi, b[2], b[3]);
                }
                ldmatrix4(b, sb + Z::Q + at);
                mma(O[2 * n2], hi, b[0], b[1]);
                mma(O[2 * n2 + 1], hi, b[2], b[3]);
            }
        }
        // R = beta v - beta e^G (S^T k); the queries' part of the outputs
        const float is0 = pow2_inverse(sc0), is1 = pow2_inverse(sc1);
        float m0 = 0.f, m1 = 0.f, odd0 = 0.f, odd1 = 0.f;
#pragma unroll
        for (int n2 = 0; n2 < 4; ++n2) {
            uint32_t v[4];
            if constexpr (!F32) ldmatrix4_trans(v, sb + Z::V + tile_at<Z::VP>(16 * n2 + b_row, vcol / 8 + b_seg));
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
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float s = e & 1 ? rs1 : rs0;
                split2(R[2 * j + (e >> 1)][2 * (e & 1)] * s, R[2 * j + (e >> 1)][2 * (e & 1) + 1] * s, rh[j][e], rl[j][e]);
            }
        const float ir0 = pow2_inverse(rs0), ir1 = pow2_inverse(rs1);
        float u0 = 0.f, u1 = 0.f;
#pragma unroll
        for (int i = 3; i >= 0; --i) {
            float x[2][4] = {};
#pragma unroll
            for (int j = 0; j <= i; ++j) {
                const uint32_t at = tile_at<2 * CH>(16 * i + b_row, 2 * j + b_seg);
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
                ldmatrix4(b, sb + Z::P + tile_at<2 * CH>(16 * i + b_row, 2 * j + b_seg));
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
#pragma unroll
        for (int j4 = 0; j4 < DK / 32; ++j4) {                       // four tiles of S at a time
            float x[4][4] = {};
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const uint32_t at = tile_at<Z::KP>(16 * kk + t_row, 4 * j4 + 2 * p + t_seg);
                    uint32_t b[4];
                    ldmatrix4_trans(b, sb + Z::K + at);
                    mma(x[2 * p], rh[kk], b[0], b[1]);
                    mma(x[2 * p + 1], rh[kk], b[2], b[3]);
                    mma(x[2 * p], rl[kk], b[0], b[1]);
                    mma(x[2 * p + 1], rl[kk], b[2], b[3]);
                    if constexpr (F32) {
                        ldmatrix4_trans(b, sb + Z::KLO + at);
                        mma(x[2 * p], rh[kk], b[0], b[1]);
                        mma(x[2 * p + 1], rh[kk], b[2], b[3]);
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
        if (c + STAGES < chunks) bar_arrive(B::empty(stage), B::COUNT);
    }
#pragma unroll
    for (int j = 0; j < DK / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) state[(int64_t)(8 * j + 2 * quad + (e & 1)) * d.head_v + (e >> 1) * 8] = S[j][e];
}

template <bool F32, int DK, int CW, int GROUPS>
__global__ void __launch_bounds__(Shape<F32, DK, CW, GROUPS>::THREADS, 1) delta_chunk_kernel(Delta d, int above) {
    using Z = Shape<F32, DK, CW, GROUPS>;
    extern __shared__ __align__(128) char smem[];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
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
    if (threadIdx.x < 32 * CW)
        run_chain<F32, DK, CW, GROUPS>(d, r, h, col0, smem, base, chunks);
    else
        prepare_chunks<F32, DK, CW, GROUPS>(d, r, h, col0, smem, base, (threadIdx.x - 32 * CW) / 128, chunks);
}

template <bool F32, int DK, int CW, int GROUPS>
cudaError_t launch_shape(const Delta& d, int above, cudaStream_t s) {
    using Z = Shape<F32, DK, CW, GROUPS>;
    static_assert(Z::BYTES <= 227 * 1024, "stages must fit");
    const auto kernel = delta_chunk_kernel<F32, DK, CW, GROUPS>;
    static LaunchPrep prep;
    int sms = 0;
    const cudaError_t e = prep.get(kernel, Z::BYTES, &sms);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)((int64_t)d.seq.batch * d.heads * (d.head_v / Z::VC)));
    return launch_dependent(kernel, grid, Z::THREADS, Z::BYTES, s, d, above);
}

template <bool F32, int DK>
cudaError_t launch_width(const Delta& d, int above, int sms, cudaStream_t s) {
    return launch_shape<F32, DK, 2, 2>(d, above, s);
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
