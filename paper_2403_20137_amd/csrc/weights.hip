// The attention weights that cached tokens collect (kvbfp_accumulate_weights and its paged form):
//     w_out[b][h][t] = decay * w_in[b][h][t] + sum over the rows of kv-head h of exp(score(row, t) - lse(row)),
// scores and rule as in decode_scored.hip, whose lse it takes: a second pass over the keys alone, without any exchange between tokens.
// A wavefront holds the keys of 32 tokens as matrix operands and goes through the rows 16 at a time; a lane sums the weights of its
// row's column in registers, the 16 columns are added at the end: no atomics, the same bits every time.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "kvbfp_internal.h"
#include "scored.h"

namespace {

using namespace kvbfp::scored;

constexpr int kThreads = 256;
constexpr int kWaveTokens = 32;
constexpr int kTileTokens = 128;

// grid = (tiles of 128 tokens, H_kv, B)
template <int P, bool N16, int QL>
__global__ __launch_bounds__(kThreads) void accumulate_weights(Args a) {
    __shared__ __align__(16) float q_s[16 * kQStride];
    __shared__ int perm_s[kD];
    __shared__ int depth_s[64];
    __shared__ RowRule rule_s[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, group = lane >> 4;
    const int b = blockIdx.z, kvh = blockIdx.y;
    const Seq s = sequence(a, b);
    if ((int)blockIdx.x * kTileTokens >= s.len) return;                  // (uniform for the workgroup)
    const int t0 = (int)blockIdx.x * kTileTokens + wave * kWaveTokens;
    const bool some = t0 < s.len;
    const int last16 = (s.len - 1) & ~15;

    Chunk<P, N16> kc[2];
#pragma unroll
    for (int st = 0; st < 2; ++st) {                                     // (a wavefront behind the last token reads the last stage)
        const int from = min(t0 + 16 * st, last16);
        const int off = min(t0 + 16 * st + l16, s.len - 1) - from;
        load_chunk<P, N16>(a, a.k_mant, a.k_exp, stage_row(a, b, kvh, from), off, group, kc[st]);
    }
    // token of this lane in the store, and what it has so far
    const int t_mine = t0 + lane;
    const int64_t unit = (int64_t)b * a.H_kv + kvh;
    const bool mine = lane < kWaveTokens && t_mine < s.len;
    const float before = mine && a.w_in ? a.w_in[unit * a.w_stride + t_mine] : 0.f;
    if (tid < 64) depth_s[tid] = tid < a.n_tok ? node_depth(node_mask(a, b, tid), tid) : 0;
    bf16x8 k[2][4];
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int j = 0; j < 4; ++j) k[st][j] = __builtin_bit_cast(bf16x8, eight<P, N16>(kc[st], j));
    const float mul = a.score_mul * (float)(1 << Decode<P>::kShift);
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int r0 = 0; r0 < a.M; r0 += 16) {
        QueryRows<QL, 16> rows;
        rows.request(a, b, kvh, r0);
        __syncthreads();
        rows.put(a, r0, q_s, perm_s);
        const int r = r0 + l16;
        if (wave == 0 && group == 0) rule_s[l16] = row_rule(a, s, b, kvh, r);
        float lse = -INFINITY;
        if (r < a.M) {
            const int tok = r / a.G;
            lse = a.lse_in[((int64_t)b * a.n_tok + tok) * a.H_q + (int64_t)kvh * a.G + (r - tok * a.G)];
        }
        __syncthreads();
        bf16x8 q[QL][4];
        query_operand<P, QL>(q_s, perm_s, l16, group, q);
        const bool counts = lse > -INFINITY;                             // a row that saw nothing has no weights to give
        const float ref = counts ? lse * 1.4426950408889634f : 0.f;
        float y[8];
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < QL; ++i) sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[st][j], q[i][j], sc, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[4 * st + i] = sc[i];
        }
        const float factor = rule_scores<8, true>(a, s, rule_s + l16, depth_s, false, t0 + 4 * group, mul, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += counts ? exp2_raw(fmaf(y[i], factor, -ref)) : 0.f;
    }
    if (!some) return;
    // acc[4 st + i] of the 16 lanes of a group: token t0 + 16 st + 4 group + i
    float got = 0.f;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        const float sum = row_sum(acc[x]);
        // token 16 (x / 4) + 4 g + x % 4 is stored by the lane of that number
        const float there = __shfl(sum, ((lane >> 2) & 3) * 16);
        if (((lane >> 4) & 1) == (x >> 2) && (lane & 3) == (x & 3)) got = there;
    }
    if (mine) a.w_out[unit * a.w_stride + t_mine] = fmaf(a.decay, before, got);
}

template <int P, bool N16>
void launch(const Args& a, int dt, hipStream_t s) {
    const dim3 grid((unsigned)((a.max_len + kTileTokens - 1) / kTileTokens), (unsigned)a.H_kv, (unsigned)a.batch);
    if (dt == KVBFP_F32) accumulate_weights<P, N16, 3><<<grid, kThreads, 0, s>>>(a);
    else if (dt == KVBFP_F16) accumulate_weights<P, N16, 2><<<grid, kThreads, 0, s>>>(a);
    else accumulate_weights<P, N16, 1><<<grid, kThreads, 0, s>>>(a);
}

}  // namespace

using namespace kvbfp;

static int weights_impl(const char* call, const kvbfp_layout* L, const kvbfp_cache* cache, const Paging* paging, int32_t n_q_heads,
                        int32_t n_q_tokens, const void* q, kvbfp_dtype dtype, const int32_t* seq_len_dev, int64_t max_len,
                        float softmax_scale, const int32_t* perm_k, const kvbfp_score_rule* rule, const float* lse, float decay,
                        const float* weights_in, float* weights_out, int64_t weights_stride, void* hip_stream) {
    clear_error();
    Args a;
    kvbfp_layout logical;
    if (int rc = fill_args(call, L, cache, paging, n_q_heads, n_q_tokens, q, dtype, seq_len_dev, max_len, softmax_scale, rule, false, &a, &logical))
        return rc;
    if (!lse || !weights_out) return fail(KVBFP_ERR_INVALID_ARG, "%s: lse/weights_out is NULL", call);
    if (weights_stride < max_len)
        return fail(KVBFP_ERR_INVALID_ARG, "%s: weights_stride %lld below max_len %lld", call, (long long)weights_stride, (long long)max_len);
    if (!std::isfinite(decay)) return fail(KVBFP_ERR_INVALID_ARG, "%s: decay is not finite", call);
    if (a.H_kv > 65535) return fail(KVBFP_ERR_UNSUPPORTED, "%s: too many heads for the grid", call);
    a.perm_k = perm_k;
    a.lse_in = lse; a.w_in = weights_in; a.w_out = weights_out; a.w_stride = weights_stride; a.decay = decay;
    hipStream_t s = (hipStream_t)hip_stream;
    const bool n16 = logical.block == 16;
    if (logical.mant_bits == 4) {
        if (n16) launch<4, true>(a, (int)dtype, s);
        else launch<4, false>(a, (int)dtype, s);
    } else {
        if (n16) launch<8, true>(a, (int)dtype, s);
        else launch<8, false>(a, (int)dtype, s);
    }
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return fail(KVBFP_ERR_HIP, "%s: %s", call, hipGetErrorString(err));
    return KVBFP_OK;
}

extern "C" {

int kvbfp_accumulate_weights(const kvbfp_layout* L, const kvbfp_cache* cache, int32_t n_q_heads, int32_t n_q_tokens, const void* q,
                             kvbfp_dtype dtype, const int32_t* seq_len_dev, int64_t max_len, float softmax_scale, const int32_t* perm_k,
                             const kvbfp_score_rule* rule, const float* lse, float decay, const float* weights_in, float* weights_out,
                             int64_t weights_stride, void* hip_stream) {
    return weights_impl("accumulate_weights", L, cache, nullptr, n_q_heads, n_q_tokens, q, dtype, seq_len_dev, max_len, softmax_scale, perm_k,
                        rule, lse, decay, weights_in, weights_out, weights_stride, hip_stream);
}

int kvbfp_accumulate_weights_paged(const kvbfp_layout* pool, const kvbfp_cache* cache, const int32_t* block_table, int64_t table_stride,
                                   int32_t batch, int32_t n_q_heads, int32_t n_q_tokens, const void* q, kvbfp_dtype dtype,
                                   const int32_t* seq_len_dev, int64_t max_len, float softmax_scale, const int32_t* perm_k,
                                   const kvbfp_score_rule* rule, const float* lse, float decay, const float* weights_in, float* weights_out,
                                   int64_t weights_stride, void* hip_stream) {
    const Paging pg{block_table, table_stride, batch};
    return weights_impl("accumulate_weights_paged", pool, cache, &pg, n_q_heads, n_q_tokens, q, dtype, seq_len_dev, max_len, softmax_scale,
                        perm_k, rule, lse, decay, weights_in, weights_out, weights_stride, hip_stream);
}

}  // extern "C"
