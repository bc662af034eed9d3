// vbq_delta.cu — the gated delta rule, token by token: per head, with the state
// S (head_k x head_v, fp32), S <- e^g S; u = beta (v - S^T k); S <- S + k u^T;
// o = S^T q.
//
// The columns of S do not meet: a warp takes 16 of them and holds all their
// rows in registers, 4 columns a lane and the rows split over 8 groups of
// lanes, so a token needs no exchange but shuffles within the warp. Both
// products are taken of the state before the token, o = e^g S^T q + (q.k) u, so
// their sums go through the shuffles together.
//
// Neither kernel lets the next one start early, nor do the convolution and the
// norm: waiting blocks take places on the SMs where the first ones end, so the
// next call's are spread unevenly (the three of a layer, 32 heads, in a graph:
// 6.3 against 7.3 us a token, 18.6 against 23.3 for 4 x 16 tokens).
//
// A single token is bound by the state's bytes, 128 KB a head of 128 x 128: 64
// sequences of 32 heads, 270 MB, 47.4 us, 5.7 TB/s.
#include <type_traits>

#include "vbq_delta.cuh"
#include "vbq_kernels.h"

namespace vbq {
namespace {

constexpr int DR_WARPS = 2;                      // of a block; 16 columns each
constexpr int DR_COLS = 16 * DR_WARPS;
// A sequence of more rows goes by chunks. Measured with BF16 heads of 128 by 128: token by token 22 and 28 rows take 1 x 32
// heads 8.8 and 10.3 us, 4 x 16 heads 11.1 and 13.1, 16 x 32 heads 54 and 65; one chunk takes them 9.0, 10.6 and 69: the
// first two, whose blocks of 64 columns the GPU holds at once, change over near 22 rows, the third at 30. Others would change
// over elsewhere: fp32 heads of 128 by 128, whose chunks are slower, at more than 64 rows (16 x 32: 132 us against 245 there),
// fp32 heads of 64 by 64 at 34 (3 x 12) or more than 64 (16 x 32), BF16 heads of 64 by 64 at 27 (4 x 16) or 38 (16 x 32).
constexpr int DELTA_ROWS = 22, DELTA_ROWS_FULL = 28;

template <bool F32, int DK>
__global__ void __launch_bounds__(32 * DR_WARPS, 8) delta_token_kernel(Delta d) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int PER = DK / 8;                  // rows of the state in a lane
    const int slices = d.head_v / DR_COLS;
    const int unit = (int)(blockIdx.x / slices), slice = (int)(blockIdx.x - unit * slices);
    const int b = unit / d.heads, h = unit - b * d.heads;
    const int lane = threadIdx.x & 31, part = lane >> 2;
    const int col = slice * DR_COLS + (threadIdx.x >> 5) * 16 + (lane & 3) * 4;
    const SeqRange r = seq_range(d.seq, b, d.n_slots, h == 0 && slice == 0 && threadIdx.x == 0, d.status);
    if (r.n == 0) return;
    const int64_t out_row = (int64_t)d.heads * d.head_v;
    uint16_t* out = d.out + r.lo * out_row + h * d.head_v + col;
    if (r.slot < 0) {
        for (int t = part; t < r.n; t += 8) *reinterpret_cast<uint2*>(out + t * out_row) = make_uint2(0, 0);
        return;
    }
    float* state = d.state + ((int64_t)r.slot * d.heads + h) * DK * d.head_v + (int64_t)part * PER * d.head_v + col;
    float4 S[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i)
        S[i] = r.fresh ? make_float4(0.f, 0.f, 0.f, 0.f) : *reinterpret_cast<const float4*>(state + (int64_t)i * d.head_v);
    const int hk = h / (d.heads / d.k_heads);
    const bool raw = d.a_log != nullptr;
    const float rate = raw ? expf(d.a_log[h]) : 0.f, bias = raw ? d.dt_bias[h] : 0.f;
    // A token's inputs as they come.
    constexpr int WORDS = F32 ? PER / 4 : PER / 8;
    uint4 k_raw[WORDS], q_raw[WORDS], v_raw = make_uint4(0, 0, 0, 0);
    const auto load = [&](int t) {
        const int64_t row = (int64_t)r.lo + t;
        const int64_t ko = row * d.k_stride + hk * DK + part * PER, qo = row * d.q_stride + hk * DK + part * PER, vo = row * d.v_stride + h * d.head_v + col;
        const auto at = [&](const void* p, int64_t o) {
            return F32 ? reinterpret_cast<const uint4*>(static_cast<const float*>(p) + o) : reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + o);
        };
#pragma unroll
        for (int i = 0; i < WORDS; ++i) { k_raw[i] = at(d.k, ko)[i]; q_raw[i] = at(d.q, qo)[i]; }
        if constexpr (F32) {
            v_raw = *at(d.v, vo);
        } else {
            const uint2 x = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(d.v) + vo);
            v_raw.x = x.x; v_raw.y = x.y;
        }
    };
    // Gates of 32 tokens, one a lane.
    float keep_of = 0.f, beta_of = 0.f;
    const auto gates = [&](int t) {
        if (t + lane >= r.n) return;
        const int64_t row = (int64_t)r.lo + t + lane;
        const Gate g = gate_of(gate_value(d.decay, d.gate_f32, row * d.decay_stride + h), gate_value(d.beta, d.gate_f32, row * d.beta_stride + h),
                               raw, rate, bias);
        keep_of = expf(g.g);
        beta_of = g.beta;
    };
    const auto unpack = [&](const uint4 (&w)[WORDS], float (&x)[PER]) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (F32) {
                    x[4 * i + e] = __uint_as_float(u[e]);
                } else {
                    x[8 * i + 2 * e] = __uint_as_float(u[e] << 16);
                    x[8 * i + 2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
                }
            }
        }
    };
#pragma unroll 1
    for (int t = 0; t < r.n; ++t) {
        load(t);
        if ((t & 31) == 0) gates(t);
        float k[PER], q[PER], v[4];
        unpack(k_raw, k);
        unpack(q_raw, q);
        if constexpr (F32) {
            v[0] = __uint_as_float(v_raw.x); v[1] = __uint_as_float(v_raw.y); v[2] = __uint_as_float(v_raw.z); v[3] = __uint_as_float(v_raw.w);
        } else {
            v[0] = __uint_as_float(v_raw.x << 16); v[1] = __uint_as_float(v_raw.x & 0xffff0000u);
            v[2] = __uint_as_float(v_raw.y << 16); v[3] = __uint_as_float(v_raw.y & 0xffff0000u);
        }
        const float keep = __shfl_sync(0xffffffffu, keep_of, t & 31), beta = __shfl_sync(0xffffffffu, beta_of, t & 31);
        // kk, qq, q.k; then k.S and q.S of four columns
        float s[11] = {};
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            s[0] = fmaf(k[i], k[i], s[0]);
            s[1] = fmaf(q[i], q[i], s[1]);
            s[2] = fmaf(q[i], k[i], s[2]);
            s[3] = fmaf(k[i], S[i].x, s[3]);
            s[4] = fmaf(k[i], S[i].y, s[4]);
            s[5] = fmaf(k[i], S[i].z, s[5]);
            s[6] = fmaf(k[i], S[i].w, s[6]);
            s[7] = fmaf(q[i], S[i].x, s[7]);
            s[8] = fmaf(q[i], S[i].y, s[8]);
            s[9] = fmaf(q[i], S[i].z, s[9]);
            s[10] = fmaf(q[i], S[i].w, s[10]);
        }
#pragma unroll
        for (int o = 4; o < 32; o <<= 1)
#pragma unroll
            for (int i = 0; i < 11; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
        const float ck = d.normalize ? rsqrtf(s[0] + DELTA_UNIT_EPS) : 1.f;
        const float cq = d.scale * (d.normalize ? rsqrtf(s[1] + DELTA_UNIT_EPS) : 1.f);
        const float qk = cq * ck * s[2];
        float u[4], o4[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u[j] = beta * (v[j] - keep * (ck * s[3 + j]));
            o4[j] = fmaf(qk, u[j], keep * (cq * s[7 + j]));
            u[j] *= ck;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            S[i].x = fmaf(k[i], u[0], keep * S[i].x);
            S[i].y = fmaf(k[i], u[1], keep * S[i].y);
            S[i].z = fmaf(k[i], u[2], keep * S[i].z);
            S[i].w = fmaf(k[i], u[3], keep * S[i].w);
        }
        if (part == 0) *reinterpret_cast<uint2*>(out + t * out_row) = make_uint2(pack_bf16(o4[0], o4[1]), pack_bf16(o4[2], o4[3]));
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) *reinterpret_cast<float4*>(state + (int64_t)i * d.head_v) = S[i];
}

// A few tokens of a sequence: BATCH at a time through shared memory, copies of the next ones under way. What does not depend
// on the state (unit lengths, q.k, gates) is worked out for all of them first, so a token's chain is its two products with
// the state, a reduction over the 8 groups of lanes and the update.
constexpr int BATCH = 16;
constexpr int RW_WARPS = DR_COLS / 8;            // 8 columns each, 2 a lane

template <bool F32, int DK>
struct Staged {
    using T = typename std::conditional<F32, float, uint16_t>::type;
    T k[BATCH][DK], q[BATCH][DK], v[BATCH][DR_COLS];
};

template <bool F32, int DK>
__global__ void __launch_bounds__(32 * RW_WARPS) delta_rows_kernel(Delta d, int most, bool beside) {
    using In = Staged<F32, DK>;
    __shared__ __align__(16) In in[2];
    __shared__ float4 token[BATCH];              // keep; beta; the unit key's factor; the scaled unit query's
    __shared__ float product[BATCH];             // q.k of these
    // Beside the chunk kernel: that one's blocks let this one start, each after its own griddepcontrol.wait, and no block here
    // starts before the last of them has. So what the kernels before both wrote is complete and in global memory by then: the
    // wait's promise to the chunk kernel, which holds for whatever starts later and has no older copies of a line (the fence
    // drops those that the SM may have). Of the chunk kernel itself nothing is read: each leaves the other's sequences alone.
    // Block 0 waits for it at the end, so that this grid does not count as done before it and what waits for this one has both.
    if (beside) asm volatile("fence.acq_rel.gpu;" ::: "memory");
    else asm volatile("griddepcontrol.wait;" ::: "memory");
    const auto leave = [&] {
        if (beside && blockIdx.x == 0) asm volatile("griddepcontrol.wait;" ::: "memory");
    };
    constexpr int PER = DK / 8;                  // rows of the state in a lane
    const int slices = d.head_v / DR_COLS;
    const int unit = (int)(blockIdx.x / slices), slice = (int)(blockIdx.x - unit * slices);
    const int b = unit / d.heads, h = unit - b * d.heads;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, part = lane >> 2, quad = lane & 3;
    const int col = slice * DR_COLS + warp * 8 + quad * 2;
    const SeqRange r = seq_range(d.seq, b, d.n_slots, h == 0 && slice == 0 && tid == 0, d.status);
    if (r.n == 0 || r.n > most) return leave();
    const int64_t out_row = (int64_t)d.heads * d.head_v;
    uint16_t* out = d.out + r.lo * out_row + h * d.head_v + col;
    if (r.slot < 0) {
        for (int t = part; t < r.n; t += 8) *reinterpret_cast<uint32_t*>(out + t * out_row) = 0;
        return leave();
    }
    const int hk = h / (d.heads / d.k_heads);
    constexpr int SIZE = F32 ? 4 : 2, SEGS = DK * SIZE / 16, VSEGS = DR_COLS * SIZE / 16;
    const auto copy = [&](int t0) {              // tokens t0 .. of the sequence into their half
        In& to = in[(t0 / BATCH) & 1];
        const int n = min(BATCH, r.n - t0);
        const int64_t row0 = (int64_t)r.lo + t0;
        const auto rows = [&](const void* p, int64_t stride, int at, void* dst, int segs) {
            const char* src = static_cast<const char*>(p) + (row0 * stride + at) * SIZE;
            for (int i = tid; i < n * segs; i += 32 * RW_WARPS) {
                const int row = i / segs, seg = i - row * segs;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(smem_u32(dst) + i * 16), "l"(src + row * stride * SIZE + seg * 16) : "memory");
            }
        };
        rows(d.k, d.k_stride, hk * DK, to.k, SEGS);
        rows(d.q, d.q_stride, hk * DK, to.q, SEGS);
        rows(d.v, d.v_stride, h * d.head_v + slice * DR_COLS, to.v, VSEGS);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    copy(0);
    float* state = d.state + ((int64_t)r.slot * d.heads + h) * DK * d.head_v + (int64_t)part * PER * d.head_v + col;
    float2 S[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) S[i] = r.fresh ? make_float2(0.f, 0.f) : *reinterpret_cast<const float2*>(state + i * d.head_v);
    const bool raw = d.a_log != nullptr;
    const float rate = raw ? expf(d.a_log[h]) : 0.f, bias = raw ? d.dt_bias[h] : 0.f;
    const auto two = [&](const typename In::T* p, int i) {           // values 2 i and 2 i + 1
        if constexpr (F32) return *reinterpret_cast<const float2*>(p + 2 * i);
        const uint32_t w = reinterpret_cast<const uint32_t*>(p)[i];
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    };
#pragma unroll 1
    for (int t0 = 0; t0 < r.n; t0 += BATCH) {
        const In& now = in[(t0 / BATCH) & 1];
        const int n = min(BATCH, r.n - t0);
        if (t0 + BATCH < r.n) {
            copy(t0 + BATCH);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        __syncthreads();
        {
            // a token to eight lanes
            const int t = tid >> 3;
            float kk = 0.f, qq = 0.f, qk = 0.f;
            if (t < n)
#pragma unroll 4
                for (int i = tid & 7; i < DK / 2; i += 8) {
                    const float2 k = two(now.k[t], i), q = two(now.q[t], i);
                    kk = fmaf(k.x, k.x, fmaf(k.y, k.y, kk));
                    qq = fmaf(q.x, q.x, fmaf(q.y, q.y, qq));
                    qk = fmaf(q.x, k.x, fmaf(q.y, k.y, qk));
                }
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) {
                kk += __shfl_xor_sync(0xffffffffu, kk, o);
                qq += __shfl_xor_sync(0xffffffffu, qq, o);
                qk += __shfl_xor_sync(0xffffffffu, qk, o);
            }
            if (t < n && (tid & 7) == 0) {
                const int64_t row = (int64_t)r.lo + t0 + t;
                const Gate g = gate_of(gate_value(d.decay, d.gate_f32, row * d.decay_stride + h), gate_value(d.beta, d.gate_f32, row * d.beta_stride + h),
                                       raw, rate, bias);
                const float ck = d.normalize ? rsqrtf(kk + DELTA_UNIT_EPS) : 1.f, cq = d.scale * (d.normalize ? rsqrtf(qq + DELTA_UNIT_EPS) : 1.f);
                token[t] = make_float4(expf(g.g), g.beta, ck, cq);
                product[t] = cq * ck * qk;
            }
        }
        __syncthreads();
#pragma unroll 1
        for (int t = 0; t < n; ++t) {
            const float4 f = token[t];
            float2 ks[2] = {}, qs[2] = {}, kd[PER];             // two sums each, of the even and the odd rows
#pragma unroll
            for (int i = 0; i < PER / 2; ++i) {
                const float2 k = two(now.k[t], part * (PER / 2) + i), q = two(now.q[t], part * (PER / 2) + i);
                kd[2 * i] = make_float2(k.x, k.x);
                kd[2 * i + 1] = make_float2(k.y, k.y);
                ks[0] = fma2(kd[2 * i], S[2 * i], ks[0]);
                qs[0] = fma2(make_float2(q.x, q.x), S[2 * i], qs[0]);
                ks[1] = fma2(kd[2 * i + 1], S[2 * i + 1], ks[1]);
                qs[1] = fma2(make_float2(q.y, q.y), S[2 * i + 1], qs[1]);
            }
            float s[4] = {ks[0].x + ks[1].x, ks[0].y + ks[1].y, qs[0].x + qs[1].x, qs[0].y + qs[1].y};
#pragma unroll
            for (int o = 4; o < 32; o <<= 1)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
            const float2 v = two(now.v[t], warp * 4 + quad), keep = make_float2(f.x, f.x);
            const float fk = -f.x * f.z, fq = f.x * f.w, qk = product[t];
            const float u0 = f.y * fmaf(fk, s[0], v.x), u1 = f.y * fmaf(fk, s[1], v.y);
            const float2 uk = make_float2(u0 * f.z, u1 * f.z);
#pragma unroll
            for (int i = 0; i < PER; ++i) S[i] = fma2(kd[i], uk, mul2(keep, S[i]));
            if (part == 0) *reinterpret_cast<uint32_t*>(out + (t0 + t) * out_row) = pack_bf16(fmaf(qk, u0, fq * s[2]), fmaf(qk, u1, fq * s[3]));
        }
        __syncthreads();                         // the other half is written next
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) *reinterpret_cast<float2*>(state + i * d.head_v) = S[i];
    leave();
}

dim3 grid_of(const Delta& d) { return dim3((unsigned)((int64_t)d.seq.batch * d.heads * (d.head_v / DR_COLS))); }

cudaError_t launch_tokens(const Delta& d, cudaStream_t s) {
    const auto go = [&](auto kernel) { return launch_dependent(kernel, grid_of(d), 32 * DR_WARPS, 0, s, d); };
    if (d.f32) return d.head_k == 64 ? go(delta_token_kernel<true, 64>) : go(delta_token_kernel<true, 128>);
    return d.head_k == 64 ? go(delta_token_kernel<false, 64>) : go(delta_token_kernel<false, 128>);
}
cudaError_t launch_rows(const Delta& d, int most, bool beside, cudaStream_t s) {
    const auto go = [&](auto kernel) { return launch_dependent(kernel, grid_of(d), 32 * RW_WARPS, 0, s, d, most, beside); };
    if (d.f32) return d.head_k == 64 ? go(delta_rows_kernel<true, 64>) : go(delta_rows_kernel<true, 128>);
    return d.head_k == 64 ? go(delta_rows_kernel<false, 64>) : go(delta_rows_kernel<false, 128>);
}

}  // namespace

// Sequences of a few rows go token by token, longer ones by chunks: with `starts` by the rows that they turn out to have, not
// by what the call says of the longest, since up to 22 rows keys may be of any sizes. Where the call's may be of both kinds,
// both kernels run, each over its own and side by side (24 single tokens and a prompt of 2000, 32 heads of 128, when it was
// added: 185 us one after the other, 165 so).
cudaError_t launch_delta_rule(const Delta& d, cudaStream_t s) {
    int sms = 0;
    const int err = device_sms(&sms);
    if (err != 0) return (cudaError_t)err;
    if (d.seq.rows <= 1) return launch_tokens(d, s);
    const int few = (int64_t)d.seq.batch * d.heads * (d.head_v / 64) <= sms ? DELTA_ROWS : DELTA_ROWS_FULL;
    if (d.seq.rows <= few) return launch_rows(d, INT32_MAX, false, s);
    if (d.seq.starts) {
        const cudaError_t e = launch_delta_chunks(d, few, sms, s);
        return e != cudaSuccess ? e : launch_rows(d, few, true, s);
    }
    return launch_delta_chunks(d, 0, sms, s);
}

}  // namespace vbq
