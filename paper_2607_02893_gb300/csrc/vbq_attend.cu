// vbq_attend.cu — attention over the 4-bit cache.
//
// out = sum_j softmax_j(scale q.k_j) v_j over the keys j in (p - window, p] of
// a row at position p. One block per (sequence, row, query head); groups of
// d / 8 lanes take a key each, a lane 8 of its dimensions, with a running
// maximum and sum per group, joined through shared memory at the end.
#include <cuda_bf16.h>

#include "vbq_decode.h"
#include "vbq_device.cuh"

namespace vbq {
namespace {

constexpr int AT_THREADS = 128;

__global__ void __launch_bounds__(AT_THREADS) kv_attend_kernel(KvView c, KvAttend a) {
    extern __shared__ float sh[];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int d = c.head_dim, lanes = d / 8, teams = AT_THREADS / lanes;
    const int team = threadIdx.x / lanes, ch = threadIdx.x % lanes;
    const int64_t row = blockIdx.x / a.heads;
    const int head = (int)(blockIdx.x % a.heads), h = head / (a.heads / c.kv_heads);
    const int64_t b = row / a.rows;
    int64_t p = a.pos[row];
    if (p >= (int64_t)c.table_pages * KV_PAGE) {
        if (threadIdx.x == 0) atomicOr(&g_device_status, VBQ_DEVICE_RANGE);
        p = (int64_t)c.table_pages * KV_PAGE - 1;
    }
    const int64_t lo = a.window && p >= a.window ? p - a.window + 1 : 0;
    float q[8], o[8] = {}, m = -INFINITY, l = 0.f;
    for (int e = 0; e < 8; ++e)
        q[e] = __uint_as_float((uint32_t)a.q[(row * a.heads + head) * d + ch * 8 + e] << 16) * a.scale;
    for (int64_t j0 = lo; j0 <= p; j0 += teams) {
        const int64_t j = j0 + team;
        const bool live = j <= p;
        const int64_t jj = live ? j : p;
        int64_t page = c.table[b * c.table_stride + jj / KV_PAGE];
        if (page < 0 || page >= c.n_pages) {
            atomicOr(&g_device_status, VBQ_DEVICE_RANGE);
            page = 0;
        }
        const int slot = (int)(jj % KV_PAGE), krow = kv_key_row(slot);
        const uint8_t* blob = c.pages + (page * c.kv_heads + h) * kv_blob_bytes(d);
        const uint32_t kw = *reinterpret_cast<const uint32_t*>(blob + krow * (d / 2) + 4 * kv_key_word(ch, d));
        const uint32_t vw = *reinterpret_cast<const uint32_t*>(blob + kv_values_at(d) + slot * (d / 2) +
                                                               4 * kv_value_word(ch, slot, d));
        const __half* sc = reinterpret_cast<const __half*>(blob + kv_scales_at(d) + krow * (d / 16));
        const float ks = __half2float(sc[ch >> 3]), vs = __half2float(sc[d / 64 + (ch >> 3)]);
        float s = 0.f;
        for (int e = 0; e < 8; ++e) s = fmaf(q[e], (float)((int)((kw >> (4 * e)) & 15u) - 8), s);
        s *= ks;
        for (int x = lanes / 2; x; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
        if (!live) continue;
        const float mn = fmaxf(m, s), f = expf(m - mn), w = expf(s - mn);
        l = l * f + w;
        m = mn;
        for (int e = 0; e < 8; ++e) o[e] = o[e] * f + w * vs * (float)((int)((vw >> (4 * e)) & 15u) - 8);
    }
    float* sm = sh + teams * d;
    for (int e = 0; e < 8; ++e) sh[team * d + ch * 8 + e] = o[e];
    if (ch == 0) { sm[2 * team] = m; sm[2 * team + 1] = l; }
    __syncthreads();
    float mx = -INFINITY, ls = 0.f;
    for (int t = 0; t < teams; ++t) mx = fmaxf(mx, sm[2 * t]);
    for (int t = 0; t < teams; ++t) ls += sm[2 * t + 1] > 0.f ? sm[2 * t + 1] * expf(sm[2 * t] - mx) : 0.f;
    for (int i = threadIdx.x; i < d; i += AT_THREADS) {
        float v = 0.f;
        for (int t = 0; t < teams; ++t)
            if (sm[2 * t + 1] > 0.f) v += sh[t * d + i] * expf(sm[2 * t] - mx);
        a.out[(row * a.heads + head) * d + i] = __bfloat16_as_ushort(__float2bfloat16_rn(ls > 0.f ? v / ls : 0.f));
    }
}

}  // namespace

size_t kv_workspace_bytes(int, int, int, int, int, int) { return 256; }

cudaError_t launch_kv_attend(const KvView& c, const KvAttend& a, cudaStream_t s) {
    const size_t smem = (size_t)(AT_THREADS / (c.head_dim / 8)) * (c.head_dim + 2) * sizeof(float);
    return launch_dependent(kv_attend_kernel, dim3((unsigned)(a.batch * a.rows * a.heads)), AT_THREADS, smem, s, c, a);
}

cudaError_t read_device_status_attend(uint32_t* status) {
    cudaError_t e = cudaMemcpyFromSymbol(status, g_device_status, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    const uint32_t zero = 0;
    return cudaMemcpyToSymbol(g_device_status, &zero, sizeof(uint32_t));
}

}  // namespace vbq
