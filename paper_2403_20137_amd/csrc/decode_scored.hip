// Decode attention with a rule on its scores: a tree of drafted tokens, a tanh cap, a bias by distance, a window, documents, a
// prefix (kvbfp_decode_attention_scored and its paged form).  Every query token brings the G heads of a kv-head's group, M rows in all.
//
// Split pass: both products on the matrix cores, v_mfma_f32_16x16x32_bf16, transposed: S^T = K Q^T and O^T = V^T P^T.  A lane then holds
// scores, maximum, sum and outputs of ONE row; what the rule knows of a row (its nodes, first token, slope) sits in that lane's
// registers, and the registers that hold S^T are, converted, the second operand of the value product: the order of the tokens
// in its reduction is free.  Every wavefront takes 32 tokens for itself: keys go from memory to the operand
// (a lane's 16 bytes are 32 channels of one token, their order follows the query's), values pass through 8 KB of LDS of that
// wavefront, from which ds_read_tr16 returns them by channel.
// The query is not rounded (bf16 one operand, fp16 two, fp32 three); probabilities are two bf16 limbs (16 bits), three with fp32 I/O.
// A tile of 32 tokens whose tokens all precede the drafted ones and are seen by every row takes no mask; tiles that no row
// sees (outside the window, the documents and the prefix) are not read.
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
constexpr int kTileTokens = 128;                 // four wavefronts
constexpr int kOStride = kD + 4;
constexpr int kWaveLds = 16 * kOStride * 4;      // 32 rows of values in bf16 (8192 bytes) or 16 rows of outputs in fp32

// The tiles of a sequence that some row of the workgroup sees: those of the prefix, then those from the first token seen on.
struct Tiles {
    int prefix, from, count;
    __device__ __forceinline__ int at(int v) const { return v < prefix ? v : from + (v - prefix); }
};
__device__ __forceinline__ Tiles tiles_of(const Seq& s, int lo) {
    Tiles t;
    t.prefix = (s.prefix + kTileTokens - 1) / kTileTokens;
    t.from = max(min(max(lo, 0), max(s.base, 0)) / kTileTokens, t.prefix);
    t.count = t.prefix + max((s.len + kTileTokens - 1) / kTileTokens - t.from, 0);
    return t;
}

// The value rows of a wavefront in LDS: 256 bytes a token, the eight 32-byte segments of a row exchanged by its number so that 16 rows of
// one segment lie in different banks.
__device__ __forceinline__ int value_at(int row, int seg) { return row * 256 + ((seg ^ (row & 7)) * 32); }

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
__device__ __forceinline__ s16x4 read_by_channel(const uint8_t* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
}

// o += V^T P^T for 32 tokens: lane (row l % 16): probabilities of tokens 4 (l / 16) .. of either stage.
template <int PL>
__device__ __forceinline__ void add_values(const uint8_t* v_s, int lane, const bf16x8 (&p)[PL], f32x4 (&o)[8]) {
    const int i = lane & 15, row = 4 * (lane >> 4) + (i >> 2), piece = (i & 3) * 8;
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) {
        const s16x4 lo = read_by_channel(v_s + value_at(row, ct) + piece);
        const s16x4 hi = read_by_channel(v_s + value_at(row + 16, ct) + piece);
        const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int l = 0; l < PL; ++l) o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[l], o[ct], 0, 0, 0);
    }
}

// One row of the output, or of lse, from its largest score, sum and sums of values.
template <int QL>
__device__ __forceinline__ void store_out(const Args& a, int64_t at, float v) {
    typedef typename Io<QL>::T T;
    ((T*)a.out)[at] = (T)v;
}
__device__ __forceinline__ float natural_lse(float m, float l) {
    return l > 0.f ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
}
__device__ __forceinline__ int64_t out_row(const Args& a, int b, int kvh, int r) {
    const int tok = r / a.G;
    return ((int64_t)b * a.n_tok + tok) * a.H_q + (int64_t)kvh * a.G + (r - tok * a.G);
}

// grid = (n_splits, H_kv * row_tiles, B); P mantissa bits, N16 blocks of 16, QL limbs of the query, HC times 16 rows.
template <int P, bool N16, int QL, int HC>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(HC == 1 && QL == 1 ? 3 : 2))) void scored_split(Args a) {
    constexpr int PL = QL == 3 ? 3 : 2;
    __shared__ __align__(16) uint8_t smem[4 * kWaveLds];
    __shared__ float ml_s[4][16][2];
    __shared__ int perm_s[kD];
    __shared__ int depth_s[64];
    static_assert(16 * HC * kQStride * 4 <= 4 * kWaveLds, "the query rows fit");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, group = lane >> 4;
    const int b = blockIdx.z, kvh = blockIdx.y / a.row_tiles, r0 = (blockIdx.y % a.row_tiles) * (16 * HC);
    const int split = blockIdx.x;
    const Seq s = sequence(a, b);

    if (tid < 64) depth_s[tid] = tid < a.n_tok ? node_depth(node_mask(a, b, tid), tid) : 0;
    stage_queries<QL, 16 * HC>(a, b, kvh, r0, (float*)smem, perm_s);
    RowRule u[HC];
    int lo_most = INT32_MIN, lo_least = INT32_MAX;
#pragma unroll
    for (int c = 0; c < HC; ++c) {
        u[c] = row_rule(a, s, b, kvh, r0 + 16 * c + l16);
        lo_most = max(lo_most, u[c].lo);
        lo_least = min(lo_least, u[c].lo);
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
        lo_most = max(lo_most, __shfl_xor(lo_most, d));
        lo_least = min(lo_least, __shfl_xor(lo_least, d));
    }
    lo_most = __builtin_amdgcn_readfirstlane(lo_most);
    lo_least = __builtin_amdgcn_readfirstlane(lo_least);
    __syncthreads();
    bf16x8 q[HC][QL][4];
#pragma unroll
    for (int c = 0; c < HC; ++c) query_operand<P, QL>((const float*)smem, perm_s, 16 * c + l16, group, q[c]);
    __syncthreads();                                         // the queries give way to the values

    uint8_t* const v_s = smem + wave * kWaveLds;
    f32x4 o[HC][8];
    float m[HC], l[HC];
#pragma unroll
    for (int c = 0; c < HC; ++c) {
        m[c] = -INFINITY;
        l[c] = 0.f;
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) o[c][ct] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float mul = a.score_mul * (float)(1 << Decode<P>::kShift);
    const Tiles tiles = tiles_of(s, lo_least);
    const int last16 = (s.len - 1) & ~15;
    Chunk<P, N16> k_next[2], v_next[2];
    auto request = [&](int v) {
        const int t0 = tiles.at(v) * kTileTokens + wave * kWaveTokens;
        if (v >= tiles.count || t0 >= s.len) return;         // (uniform for the wavefront)
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const int from = min(t0 + 16 * st, last16);
            const int off = min(t0 + 16 * st + l16, s.len - 1) - from;
            const int64_t row = stage_row(a, b, kvh, from);
            load_chunk<P, N16>(a, a.k_mant, a.k_exp, row, off, group, k_next[st]);
            load_chunk<P, N16>(a, a.v_mant, a.v_exp, row, off, group, v_next[st]);
        }
    };
    request(split);
    for (int v = split; v < tiles.count; v += a.n_splits) {
        const int t0 = tiles.at(v) * kTileTokens + wave * kWaveTokens;
        if (t0 >= s.len) break;                              // the wavefront's part of the last tile is empty
        Chunk<P, N16> kc[2], vc[2];
#pragma unroll
        for (int st = 0; st < 2; ++st) { kc[st] = k_next[st]; vc[st] = v_next[st]; }
        request(v + a.n_splits);
        // scores
        f32x4 sc[HC][2];
#pragma unroll
        for (int st = 0; st < 2; ++st) {
#pragma unroll
            for (int c = 0; c < HC; ++c) sc[c][st] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x8 k = __builtin_bit_cast(bf16x8, eight<P, N16>(kc[st], j));
#pragma unroll
                for (int c = 0; c < HC; ++c)
#pragma unroll
                    for (int i = 0; i < QL; ++i) sc[c][st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[c][i][j], sc[c][st], 0, 0, 0);
            }
        }
        // values to LDS
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *(u32x4*)(v_s + value_at(16 * st + l16, 2 * group + (j >> 1)) + (j & 1) * 16) = eight<P, N16>(vc[st], j);
        wave_fence();
        const bool inner = t0 >= lo_most && t0 + kWaveTokens <= s.base;
#pragma unroll
        for (int c = 0; c < HC; ++c) {
            float y[8], top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = sc[c][i >> 2][i & 3] * mul;
            rule_scores<8>(a, s, u[c], depth_s, inner, t0 + 4 * group, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, y[i]);
            top = rows_max(top);
            if (__builtin_amdgcn_ballot_w64(top > m[c])) {
                const float now = fmaxf(m[c], top);
                const float f = now > -INFINITY ? exp2_raw(m[c] - now) : 1.f;
                m[c] = now;
                l[c] *= f;
#pragma unroll
                for (int ct = 0; ct < 8; ++ct)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[c][ct][i] *= f;
            }
            const float ref = m[c] > -INFINITY ? m[c] : 0.f;
            bf16x8 p[PL];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float w = exp2_raw(y[i] - ref);
                l[c] += w;
                __bf16 lw[PL];
                limbs<PL>(w, lw);
                if (PL == 2) lw[1] = (__bf16)(w - __uint_as_float(__float_as_uint(w) & 0xFFFF0000u));
#pragma unroll
                for (int x = 0; x < PL; ++x) p[x][i] = lw[x];
            }
            add_values<PL>(v_s, lane, p, o[c]);
        }
        wave_fence();
    }

    // the four wavefronts' sums, 16 rows at a time
    const float up = (float)(1 << Decode<P>::kShift);
#pragma unroll
    for (int c = 0; c < HC; ++c) {
        if (r0 + 16 * c >= a.M) break;                       // uniform
        __syncthreads();
        float* const o_s = (float*)v_s;
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) *(f32x4*)(o_s + l16 * kOStride + 16 * ct + 4 * group) = o[c][ct];
        const float sum = rows_sum(l[c]);
        if (group == 0) {
            ml_s[wave][l16][0] = m[c];
            ml_s[wave][l16][1] = sum;
        }
        __syncthreads();
        const int row = tid >> 4, p0 = (tid & 15) * 8, r = r0 + 16 * c + row;
        if (r >= a.M) continue;
        float top = -INFINITY, den = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, ml_s[w][row][0]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (!(ml_s[w][row][0] > -INFINITY)) continue;
            const float f = exp2_raw(ml_s[w][row][0] - top);
            den = fmaf(f, ml_s[w][row][1], den);
            const float* const src = (const float*)(smem + w * kWaveLds) + row * kOStride + p0;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = fmaf(f, src[i], acc[i]);
        }
        if (a.n_splits > 1) {
            const int64_t at = (((int64_t)b * a.H_kv + kvh) * a.M + r) * a.n_splits + split;
            if (p0 == 0) {
                a.part_ml[2 * at] = top;
                a.part_ml[2 * at + 1] = den;
            }
            *(f32x4*)(a.part_o + at * kD + p0) = f32x4{acc[0] * up, acc[1] * up, acc[2] * up, acc[3] * up};
            *(f32x4*)(a.part_o + at * kD + p0 + 4) = f32x4{acc[4] * up, acc[5] * up, acc[6] * up, acc[7] * up};
        } else {
            const int64_t at = out_row(a, b, kvh, r);
            const float by = den > 0.f ? up / den : 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                int ch = position_channel<P>(p0 + i);
                if (a.perm_v) ch = a.perm_v[kvh * kD + ch] & (kD - 1);
                store_out<QL>(a, at * kD + ch, acc[i] * by);
            }
            if (p0 == 0 && a.lse) a.lse[at] = natural_lse(top, den);
        }
    }
}

// Joins the splits: a wavefront per row, two channels a lane.
template <int P, int QL>
__global__ __launch_bounds__(kThreads) void scored_combine(Args a) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);          // (b * H_kv + kvh) * M + r
    if (row >= (int64_t)a.batch * a.H_kv * a.M) return;
    const int unit = (int)(row / a.M), r = (int)(row - (int64_t)unit * a.M), b = unit / a.H_kv, kvh = unit % a.H_kv;
    const int64_t first = row * a.n_splits;
    float top = -INFINITY, den = 0.f;
    float2 acc = {0.f, 0.f};
    for (int i = 0; i < a.n_splits; ++i) top = fmaxf(top, a.part_ml[2 * (first + i)]);
    if (top > -INFINITY) {
        for (int i = 0; i < a.n_splits; ++i) {
            const float f = exp2_raw(a.part_ml[2 * (first + i)] - top);
            if (f == 0.f) continue;                           // a split that saw nothing
            den = fmaf(f, a.part_ml[2 * (first + i) + 1], den);
            const float2 v = *(const float2*)(a.part_o + (first + i) * kD + 2 * lane);
            acc.x = fmaf(f, v.x, acc.x);
            acc.y = fmaf(f, v.y, acc.y);
        }
    }
    const float by = den > 0.f ? 1.f / den : 0.f;
    const int64_t at = out_row(a, b, kvh, r);
    int c0 = position_channel<P>(2 * lane), c1 = position_channel<P>(2 * lane + 1);
    if (a.perm_v) {
        c0 = a.perm_v[kvh * kD + c0] & (kD - 1);
        c1 = a.perm_v[kvh * kD + c1] & (kD - 1);
    }
    store_out<QL>(a, at * kD + c0, acc.x * by);
    store_out<QL>(a, at * kD + c1, acc.y * by);
    if (lane == 0 && a.lse) a.lse[at] = natural_lse(top, den);
}

template <int P, bool N16, int QL, int HC>
void launch_split(const Args& a, hipStream_t s) {
    scored_split<P, N16, QL, HC><<<dim3((unsigned)a.n_splits, (unsigned)(a.H_kv * a.row_tiles), (unsigned)a.batch), kThreads, 0, s>>>(a);
}
template <int P, bool N16>
void launch_split(const Args& a, int dt, int hc, hipStream_t s) {
    if (dt == KVBFP_F32) launch_split<P, N16, 3, 1>(a, s);
    else if (dt == KVBFP_F16 && hc == 1) launch_split<P, N16, 2, 1>(a, s);
    else if (dt == KVBFP_F16) launch_split<P, N16, 2, 2>(a, s);
    else if (hc == 1) launch_split<P, N16, 1, 1>(a, s);
    else launch_split<P, N16, 1, 2>(a, s);
}

template <int P>
void launch_combine(const Args& a, int dt, dim3 grid, hipStream_t s) {
    if (dt == KVBFP_F32) scored_combine<P, 3><<<grid, kThreads, 0, s>>>(a);
    else if (dt == KVBFP_F16) scored_combine<P, 2><<<grid, kThreads, 0, s>>>(a);
    else scored_combine<P, 1><<<grid, kThreads, 0, s>>>(a);
}

// Rows of a workgroup / 16, and the splits: enough workgroups for three per compute unit, and no more splits than tiles.
struct Plan { int32_t hc, row_tiles, n_splits; };
Plan plan(const kvbfp_layout* L, int64_t rows, int64_t max_len) {
    Plan p;
    p.hc = rows > 16 ? 2 : 1;
    p.row_tiles = (int32_t)((rows + 16 * p.hc - 1) / (16 * p.hc));
    const int64_t units = (int64_t)L->batch * L->n_kv_heads * p.row_tiles;
    const int64_t tiles = (max_len + kTileTokens - 1) / kTileTokens;
    p.n_splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(tiles, (768 + units - 1) / units));
    return p;
}
// fp32 I/O takes 16 rows a workgroup: its plan is the one that needs more room.
Plan plan(const kvbfp_layout* L, int64_t rows, int64_t max_len, int dtype) {
    Plan p = plan(L, rows, max_len);
    if (dtype == KVBFP_F32 && p.hc == 2) {
        p.hc = 1;
        p.row_tiles = (int32_t)((rows + 15) / 16);
    }
    return p;
}

size_t partial_bytes(const kvbfp_layout* L, int64_t rows, int32_t n_splits) {
    return n_splits < 2 ? 0 : (size_t)L->batch * (size_t)L->n_kv_heads * (size_t)rows * (size_t)n_splits * (size_t)(kD + 2) * sizeof(float);
}

}  // namespace

namespace kvbfp {
namespace scored {

int fill_args(const char* call, const kvbfp_layout* L, const kvbfp_cache* cache, const Paging* paging, int32_t n_q_heads, int32_t n_q_tokens,
              const void* q, kvbfp_dtype dtype, const int32_t* seq_len_dev, int64_t max_len, float softmax_scale,
              const kvbfp_score_rule* rule, bool need_v, Args* a, kvbfp_layout* logical) {
    if (paging) {
        if (int rc = check_paging(L, *paging, logical)) return rc;
    } else {
        if (int rc = check_device_layout(L)) return rc;
        *logical = *L;
    }
    if (int rc = check_cache(cache, true, need_v)) return rc;
    if (!q) return fail(KVBFP_ERR_INVALID_ARG, "%s: q is NULL", call);
    if (dtype_size(dtype) == 0) return fail(KVBFP_ERR_INVALID_ARG, "%s: unknown dtype %d", call, (int)dtype);
    if ((uintptr_t)q % dtype_size(dtype) != 0) return fail(KVBFP_ERR_INVALID_ARG, "%s: q is not aligned to its elements", call);
    if (n_q_tokens < 1 || n_q_tokens > 64) return fail(KVBFP_ERR_INVALID_ARG, "%s: n_q_tokens = %d (1..64)", call, n_q_tokens);
    if (n_q_heads <= 0 || n_q_heads % logical->n_kv_heads != 0)
        return fail(KVBFP_ERR_INVALID_ARG, "%s: n_q_heads %d not a multiple of n_kv_heads %d", call, n_q_heads, logical->n_kv_heads);
    if (max_len <= 0 || max_len > logical->max_seq)
        return fail(KVBFP_ERR_INVALID_ARG, "%s: max_len %lld outside (0, max_seq=%lld]", call, (long long)max_len, (long long)logical->max_seq);
    if (!std::isfinite(softmax_scale)) return fail(KVBFP_ERR_INVALID_ARG, "%s: softmax_scale is not finite", call);
    if ((int64_t)n_q_heads * n_q_tokens > 65535 || logical->batch > 65535)
        return fail(KVBFP_ERR_UNSUPPORTED, "%s: batch/heads exceed the grid limits", call);
    if (rule) {
        if (rule->struct_bytes != sizeof(kvbfp_score_rule))
            return fail(KVBFP_ERR_INVALID_ARG, "%s: rule.struct_bytes = %u, expected %zu", call, rule->struct_bytes, sizeof(kvbfp_score_rule));
        if (!std::isfinite(rule->cap) || rule->cap < 0.f) return fail(KVBFP_ERR_INVALID_ARG, "%s: rule.cap = %g", call, (double)rule->cap);
        if (rule->window < 0) return fail(KVBFP_ERR_INVALID_ARG, "%s: rule.window = %d", call, rule->window);
        if (rule->tree_mask && rule->tree_stride != 0 && rule->tree_stride < n_q_tokens)
            return fail(KVBFP_ERR_INVALID_ARG, "%s: rule.tree_stride = %d (0, or at least n_q_tokens = %d)", call, rule->tree_stride, n_q_tokens);
    }
    *a = Args{};
    a->k_mant = cache->k_mant; a->k_exp = cache->k_exp; a->v_mant = cache->v_mant; a->v_exp = cache->v_exp;
    a->q = q;
    a->seq_len = seq_len_dev;
    a->max_seq = logical->max_seq; a->max_len = (int32_t)max_len; a->batch = logical->batch;
    a->H_kv = logical->n_kv_heads; a->H_q = n_q_heads; a->G = n_q_heads / logical->n_kv_heads; a->n_tok = n_q_tokens;
    a->M = a->G * n_q_tokens;
    a->n_exps = kD / logical->block;
    while ((1 << a->log2_block) < logical->block) ++a->log2_block;
    constexpr float kLog2e = 1.4426950408889634f;
    a->score_mul = softmax_scale * kLog2e;
    if (paging) {
        a->block_table = paging->block_table; a->table_stride = paging->table_stride; a->n_pages = L->batch;
        while (((int64_t)1 << a->log2_page) < L->max_seq) ++a->log2_page;
    }
    if (rule) {
        if (rule->cap > 0.f) {
            a->cap = rule->cap * kLog2e;
            a->inv_cap = 1.f / a->cap;
            if (!std::isfinite(a->cap) || !std::isfinite(a->inv_cap)) return fail(KVBFP_ERR_INVALID_ARG, "%s: rule.cap = %g", call, (double)rule->cap);
        }
        a->slopes = rule->slopes; a->first = rule->first_dev; a->prefix = rule->prefix_dev;
        a->tree = rule->tree_mask; a->tree_stride = rule->tree_stride;
        a->window = (int64_t)rule->window < max_len + 64 ? rule->window : 0;      // a window beyond every distance is none
    }
    return KVBFP_OK;
}

}  // namespace scored
}  // namespace kvbfp

using namespace kvbfp;

static int scored_impl(const char* call, const kvbfp_layout* L, const kvbfp_cache* cache, const Paging* paging, int32_t n_q_heads,
                       int32_t n_q_tokens, const void* q, kvbfp_dtype dtype, const int32_t* seq_len_dev, int64_t max_len,
                       float softmax_scale, const int32_t* perm_k, const int32_t* perm_v, const kvbfp_score_rule* rule, void* out,
                       float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
    clear_error();
    Args a;
    kvbfp_layout logical;
    if (int rc = fill_args(call, L, cache, paging, n_q_heads, n_q_tokens, q, dtype, seq_len_dev, max_len, softmax_scale, rule, true, &a, &logical))
        return rc;
    if (!out) return fail(KVBFP_ERR_INVALID_ARG, "%s: out is NULL", call);
    if ((uintptr_t)out % dtype_size(dtype) != 0) return fail(KVBFP_ERR_INVALID_ARG, "%s: out is not aligned to its elements", call);
    const Plan p = plan(&logical, a.M, max_len, (int)dtype);
    if ((int64_t)a.H_kv * p.row_tiles > 65535) return fail(KVBFP_ERR_UNSUPPORTED, "%s: too many heads for the grid", call);
    const size_t need = partial_bytes(&logical, a.M, p.n_splits);
    if (need && (!workspace || workspace_bytes < need))
        return fail(KVBFP_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", call, need, workspace ? workspace_bytes : (size_t)0);
    if (need && (uintptr_t)workspace % 256 != 0) return fail(KVBFP_ERR_WORKSPACE, "%s: workspace must be 256-byte aligned", call);
    a.out = out; a.lse = lse; a.perm_k = perm_k; a.perm_v = perm_v;
    a.n_splits = p.n_splits; a.row_tiles = p.row_tiles;
    if (need) {
        a.part_o = (float*)workspace;
        a.part_ml = a.part_o + (size_t)a.batch * a.H_kv * a.M * a.n_splits * kD;
    }
    hipStream_t s = (hipStream_t)hip_stream;
    const bool n16 = logical.block == 16;
    if (logical.mant_bits == 4) {
        if (n16) launch_split<4, true>(a, (int)dtype, p.hc, s);
        else launch_split<4, false>(a, (int)dtype, p.hc, s);
    } else {
        if (n16) launch_split<8, true>(a, (int)dtype, p.hc, s);
        else launch_split<8, false>(a, (int)dtype, p.hc, s);
    }
    hipError_t err = hipGetLastError();
    if (err == hipSuccess && a.n_splits > 1) {
        const int64_t rows = (int64_t)a.batch * a.H_kv * a.M;
        const dim3 grid((unsigned)((rows + 3) / 4));
        if (logical.mant_bits == 4) launch_combine<4>(a, (int)dtype, grid, s);
        else launch_combine<8>(a, (int)dtype, grid, s);
        err = hipGetLastError();
    }
    if (err != hipSuccess) return fail(KVBFP_ERR_HIP, "%s: %s", call, hipGetErrorString(err));
    return KVBFP_OK;
}

extern "C" {

size_t kvbfp_scored_workspace_bytes(const kvbfp_layout* L, int32_t n_q_heads, int32_t n_q_tokens, int64_t max_len) {
    clear_error();
    if (check_device_layout(L) != KVBFP_OK) return 0;
    if (n_q_heads <= 0 || n_q_heads % L->n_kv_heads != 0 || n_q_tokens < 1 || n_q_tokens > 64 || max_len <= 0 || max_len > L->max_seq) {
        fail(KVBFP_ERR_INVALID_ARG, "scored_workspace_bytes: bad n_q_heads/n_q_tokens/max_len");
        return 0;
    }
    const int64_t rows = (int64_t)(n_q_heads / L->n_kv_heads) * n_q_tokens;
    return std::max<size_t>(partial_bytes(L, rows, plan(L, rows, max_len).n_splits), 256);
}

size_t kvbfp_scored_workspace_bytes_paged(const kvbfp_layout* pool, int64_t table_stride, int32_t batch, int32_t n_q_heads,
                                          int32_t n_q_tokens, int64_t max_len) {
    clear_error();
    static const int32_t placeholder = 0;      // only its address is looked at here
    const Paging pg{&placeholder, table_stride, batch};
    kvbfp_layout logical;
    if (check_paging(pool, pg, &logical) != KVBFP_OK) return 0;
    return kvbfp_scored_workspace_bytes(&logical, n_q_heads, n_q_tokens, max_len);
}

int kvbfp_decode_attention_scored(const kvbfp_layout* L, const kvbfp_cache* cache, int32_t n_q_heads, int32_t n_q_tokens, const void* q,
                                  kvbfp_dtype dtype, const int32_t* seq_len_dev, int64_t max_len, float softmax_scale,
                                  const int32_t* perm_k, const int32_t* perm_v, const kvbfp_score_rule* rule, void* out, float* lse,
                                  void* workspace, size_t workspace_bytes, void* hip_stream) {
    return scored_impl("decode_attention_scored", L, cache, nullptr, n_q_heads, n_q_tokens, q, dtype, seq_len_dev, max_len, softmax_scale,
                       perm_k, perm_v, rule, out, lse, workspace, workspace_bytes, hip_stream);
}

int kvbfp_decode_attention_scored_paged(const kvbfp_layout* pool, const kvbfp_cache* cache, const int32_t* block_table, int64_t table_stride,
                                        int32_t batch, int32_t n_q_heads, int32_t n_q_tokens, const void* q, kvbfp_dtype dtype,
                                        const int32_t* seq_len_dev, int64_t max_len, float softmax_scale, const int32_t* perm_k,
                                        const int32_t* perm_v, const kvbfp_score_rule* rule, void* out, float* lse, void* workspace,
                                        size_t workspace_bytes, void* hip_stream) {
    const Paging pg{block_table, table_stride, batch};
    return scored_impl("decode_attention_scored_paged", pool, cache, &pg, n_q_heads, n_q_tokens, q, dtype, seq_len_dev, max_len,
                       softmax_scale, perm_k, perm_v, rule, out, lse, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
