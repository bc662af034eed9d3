// vbq_decode.h — launchers of the kernels a decode step runs around the packed
// products (internal; called by the C ABI in vbq_decode_api.cu): the 4-bit
// key-value cache, the residual norm and the sampler, and those of a
// linear-attention layer. Each returns the cudaError_t of its launch.
#pragma once

#include <cstdarg>
#include <cstddef>
#include <cstdint>
#include <cuda_runtime.h>

#include "../../include/vbq.h"

namespace vbq {

// Records the calling thread's error detail and returns st (vbq_api.cu).
vbq_status_t fail(vbq_status_t st, const char* fmt, ...);
void clear_error();

// ---------------------------------------------------------------------------
// The cache. A page holds KV_PAGE tokens of every key-value head; a (page,
// head) is one contiguous blob, so a kernel copies it in one sweep:
//
//   keys    KV_PAGE rows of d/2 bytes, in the order of kv_key_row
//   values  KV_PAGE rows of d/2 bytes, token order
//   scales  KV_PAGE entries of d/16 bytes, in the order of kv_key_row: the
//           token's d/64 FP16 key scales, then its d/64 FP16 value scales
//
// = 68 d bytes. A row is d/8 words of 8 codes; word c (codes 8c .. 8c + 7, the
// lowest nibble first, offset binary: 8 is zero; then kv_turned) sits at
// kv_key_word / kv_value_word. The orders are those the attention kernel's
// fragments read from shared memory without bank conflicts (vbq_attend.cu).
// ---------------------------------------------------------------------------
constexpr int KV_PAGE = 64;
constexpr int KV_GROUP = 64;                    // codes that share a scale

struct KvView {
    uint8_t* pages;
    const int32_t* table;                       // sequence b's page i at table[b * table_stride + i]
    int64_t table_stride;
    int64_t n_pages;
    int table_pages;
    int kv_heads, head_dim;
};

__host__ __device__ constexpr int64_t kv_blob_bytes(int d) { return 68ll * d; }
__host__ __device__ constexpr int kv_values_at(int d) { return 32 * d; }
__host__ __device__ constexpr int kv_scales_at(int d) { return 64 * d; }

// Each 16-bit half of a word is turned left by 2: codes 0 and 1 of a half are
// then at bits 2..5 and 6..9, the high bits of an f16's fraction, and codes 2
// and 3 are after a swap of the half's bytes.
__host__ __device__ constexpr uint32_t kv_turned(uint32_t w) { return (w << 2 & 0xfffcfffcu) | (w >> 14 & 0x00030003u); }
__host__ __device__ constexpr uint32_t kv_unturned(uint32_t w) { return (w >> 2 & 0x3fff3fffu) | (w << 14 & 0xc000c000u); }

// Row of a token's keys (and scales) within the page: within each 8 tokens the
// first four take the even rows, the last four the odd ones.
__host__ __device__ constexpr int kv_key_row(int slot) {
    const int o = slot & 7;
    return (slot & ~7) | (o < 4 ? 2 * o : 2 * o - 7);
}
// Place of word c in a row of keys: lane c % 4 of a fragment holds its words together.
__host__ __device__ constexpr int kv_key_word(int c, int d) { return (c & 3) * (d / 32) + 2 * (c >> 3) + ((c >> 2) & 1); }
// Place of word c in a token's row of values: word c % 8 of every group
// together, rotated by the token so that four tokens' words fall in distinct
// banks.
__host__ __device__ constexpr int kv_value_word(int c, int slot, int d) {
    const int turn = d == 64 ? 0 : d == 128 ? ((slot >> 1) & 1) << 2 : (slot & 3) << 1;
    return ((c & 7) ^ turn) * (d / 64) + (c >> 3);
}

// Rows of new tokens given to the append kernel: row r of sequence r / rows.
struct KvAppend {
    const int32_t* pos;                         // batch x rows, < 0: an unused row
    int batch, rows;
    const void *q, *k, *v;                      // row r's heads at r * stride values; q may be null
    int64_t q_stride, k_stride, v_stride;
    int heads;                                  // query heads
    int f32;                                    // the three's type: BF16 or float
    const float *cos, *sin;                     // rot_rows x rot_dim / 2, or null
    int rot_dim;
    int64_t rot_rows;
    uint16_t* q_out;                            // BF16, dense
};
cudaError_t launch_kv_append(const KvView& c, const KvAppend& a, cudaStream_t s);
cudaError_t launch_kv_read(const KvView& c, const int32_t* pos, int batch, int rows, float* k_out, float* v_out,
                           cudaStream_t s);

struct KvAttend {
    const int32_t* pos;
    int batch, rows;
    const uint16_t* q;                          // BF16, batch x rows x heads x d
    int heads;
    float scale;
    int window;                                 // 0: none
    uint16_t* out;                              // BF16, as q
    void* workspace;
    size_t workspace_bytes;
};
constexpr int KV_MAX_BATCH = 1024;
constexpr int KV_MAX_ROWS = 16;
size_t kv_workspace_bytes(int batch, int rows, int heads, int kv_heads, int sms);
cudaError_t launch_kv_attend(const KvView& c, const KvAttend& a, cudaStream_t s);

struct Norm {
    const void *x, *residual;                   // residual may be null
    int x_f32, residual_f32;
    const float* weight;
    float eps;
    int64_t rows;
    int width;
    uint16_t* out;                              // BF16
    void* residual_out;
};
cudaError_t launch_residual_norm(const Norm& n, cudaStream_t s);

struct Sample {
    const void* logits;                         // row b at b * stride
    int64_t stride;
    int f32;
    int batch, vocab;
    const float* temperature;
    const int32_t* top_k;
    const float *top_p, *min_p, *u;
    int32_t* tokens;
    float* probs;                               // may be null
    int32_t* kept;                              // may be null
};
constexpr int SAMPLE_MAX_VOCAB = 1 << 18;
cudaError_t launch_sample(const Sample& p, cudaStream_t s);

// ---------------------------------------------------------------------------
// A linear-attention layer (vbq_conv.cu, vbq_delta.cu, vbq_gated.cu).
// ---------------------------------------------------------------------------
struct Conv {
    vbq_sequences seq;
    const void* x;
    int64_t x_stride;
    int f32;
    const float *weight, *bias;                 // bias may be null
    int taps, channels;
    float* state;
    int64_t n_slots;
    int silu;
    uint16_t* out;
    uint32_t* status;                           // sequence_status's word
};
constexpr int CONV_MAX_TAPS = 4;
cudaError_t launch_causal_conv(const Conv& c, cudaStream_t s);

struct Delta {
    vbq_sequences seq;
    float* state;
    int64_t n_slots;
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    int f32;
    int k_heads, head_k, heads, head_v;
    const void *decay, *beta;
    int64_t decay_stride, beta_stride;
    int gate_f32;
    const float *a_log, *dt_bias;               // both or none
    float scale;
    int normalize;
    uint16_t* out;
    uint32_t* status;
};
constexpr int64_t DELTA_MAX_TOKENS = (1ll << 31) - 64;   // row numbers rounded up to a chunk's end are ints
cudaError_t launch_delta_rule(const Delta& d, cudaStream_t s);

struct GatedNorm {
    const void *x, *gate;                       // gate may be null
    int64_t x_stride, gate_stride;
    int x_f32, gate_f32;
    const float* weight;
    float eps;
    int64_t rows;
    int heads, width;
    uint16_t* out;
};
cudaError_t launch_gated_norm(const GatedNorm& n, cudaStream_t s);

// Device status words of the cache kernels (read and cleared). Those on sequences report into the first, whose address on the
// current device they are given: a word of their own would be a copy more, which waits for the device, in every report.
constexpr uint32_t VBQ_DEVICE_RANGE = 2u;       // a position or page outside the cache
constexpr uint32_t VBQ_DEVICE_SLOT = 4u;        // a slot of a call on sequences outside its pool
cudaError_t read_device_status_kv(uint32_t* status);
cudaError_t read_device_status_attend(uint32_t* status);
cudaError_t sequence_status(uint32_t** word);

// Launch with programmatic dependent launch, as the products are: the kernel
// may start before its predecessor on the stream has finished and waits for it
// (griddepcontrol.wait) before it reads anything.
template <class... P, class... A>
cudaError_t launch_dependent(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace vbq
