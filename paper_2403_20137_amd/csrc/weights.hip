// The attention weights that cached tokens collect (kvbfp_accumulate_weights and its paged form):
//     w_out[b][h][t] = decay * w_in[b][h][t] + sum over the rows of kv-head h of exp(score(row, t) - lse(row)),
// scores and rule as in decode_scored.hip, whose lse it takes: a second pass over the keys alone, without any exchange between tokens.
// S = Q K^T by v_mfma_f32_16x16x32_bf16: a lane has four rows of one token, so the sum over the rows stays in the lane, and the four 16-lane
// groups are added once at the end: no atomics, the same bits every time.  A wavefront has 32 tokens at a time as operands (the keys go
// from memory to the operand, 32 channels a lane) and goes through up to 128 rows (fp32 I/O 64), which lie in LDS as operands; more rows are
// further passes over the keys, which add to what the pass before has written.
// 8 x 8 heads of 32768 tokens, four rows each: 34.7 us in a graph, 4.6 TB/s (25 for the reading alone, vector instructions 14).  Many rows and few tokens are bound
// by the set-up: 128 rows of 3000 tokens turn into operands in every workgroup for three tiles (vector instructions 39 % of the time, bank conflicts
// of the 2-byte stores 11 %, exponentials 3 %), and by the way of code and first loads: one tile in flight with the loop once took 22.5 us for 4 x 265 rows of 78
// tokens where two with the loop twice took 26.9, and as long for long sequences.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "kvbfp_internal.h"
#include "scored.h"

namespace {

using namespace kvbfp::scored;

constexpr int kThreads = 256;
constexpr int kStages = 2;                       // of 16 tokens, per wavefront
constexpr int kWaveTokens = 16 * kStages;

// ROWS query rows from r0 on (zeros behind the last row of the kv-head) on their way to LDS as matrix operands: QL planes of bf16 numbers, a row
// 256 bytes in the order of eight(), its 16-byte pieces exchanged by the row's number.  Called by the whole workgroup of 256: request(), which
// asks for the first 16 EARLY rows, place(), a barrier, put(), a barrier, staged_operand().  A thread has the same eight channels of every
// sixteenth row, so where they go is worked out once.
template <int P, int QL, int ROWS, int EARLY>
struct StagedRows {
    typedef typename Io<QL>::T T;
    typedef T Tx8 __attribute__((ext_vector_type(8)));
    Tx8 first[EARLY];
    int channel;                         // of the query, that belongs at position tid
    __device__ __forceinline__ Tx8 load(const Args& a, int b, int kvh, int r0) const {
        const int r = min(r0 + (threadIdx.x >> 4), a.M - 1), tok = r / a.G;
        const T* const src = (const T*)a.q + (((int64_t)b * a.n_tok + tok) * a.H_q + (int64_t)kvh * a.G + (r - tok * a.G)) * kD + (threadIdx.x & 15) * 8;
        Tx8 x;
        if (((uintptr_t)a.q & 15u) == 0) {
            x = *(const Tx8*)src;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = src[k];
        }
        return x;
    }
    __device__ __forceinline__ void request(const Args& a, int b, int kvh, int r0) {
        const int cached = position_channel<P>(threadIdx.x & (kD - 1));
        channel = a.perm_k ? a.perm_k[kvh * kD + cached] & (kD - 1) : cached;                     // masked: stays inside the row
#pragma unroll
        for (int p = 0; p < EARLY; ++p) {
            if (p > 0 && r0 + 16 * p >= a.M) break;
            first[p] = load(a, b, kvh, r0 + 16 * p);
        }
    }
    __device__ __forceinline__ void place(int* at_s) const {
        if (threadIdx.x < kD) at_s[channel] = threadIdx.x;
    }
    __device__ __forceinline__ void put(const Args& a, int b, int kvh, int r0, uint8_t* q_s, const int* at_s) const {
        const int row = threadIdx.x >> 4, c = (threadIdx.x & 15) * 8;
        int to[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int at = at_s[c + k] & (kD - 1);           // (masked: what is no permutation leaves entries out)
            to[k] = row * 256 + (((at >> 3) ^ row) * 16) + (at & 7) * 2;
        }
        auto put16 = [&](int p, const Tx8& x) {
            const bool there = r0 + row + 16 * p < a.M;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                __bf16 l[QL];
                limbs<QL>((float)x[k], l);
#pragma unroll
                for (int n = 0; n < QL; ++n) *(uint16_t*)(q_s + n * (ROWS * 256) + p * (16 * 256) + to[k]) = there ? __builtin_bit_cast(unsigned short, l[n]) : 0;
            }
        };
#pragma unroll
        for (int p = 0; p < EARLY; ++p)
            if (p == 0 || r0 + 16 * p < a.M) put16(p, first[p]);
#pragma unroll 1
        for (int p = EARLY; p < ROWS / 16 && r0 + 16 * p < a.M; ++p) put16(p, load(a, b, kvh, r0 + 16 * p));
    }
};
// The operand of 16 rows from r0 on (a multiple of 16): lane (row l % 16, group l / 16), step j: channels 32 group + 8 j .. in the order of eight().
template <int ROWS>
__device__ __forceinline__ bf16x8 staged_operand(const uint8_t* q_s, int n, int r0, int l16, int group, int j) {
    return *(const bf16x8*)(q_s + n * (ROWS * 256) + (r0 + l16) * 256 + (((4 * group + j) ^ l16) * 16));
}

// -lse of a row in base 2; minus infinity: the row has no weights to give.
__device__ __forceinline__ float reference(const Args& a, int b, int kvh, int r) {
    if (r >= a.M) return -INFINITY;
    const int tok = r / a.G;
    const float lse = a.lse_in[((int64_t)b * a.n_tok + tok) * a.H_q + (int64_t)kvh * a.G + (r - tok * a.G)];
    return lse != -INFINITY ? -lse * 1.4426950408889634f : -INFINITY;
}
// v[i] summed over the four groups of 16 lanes, for group i: two exchanges of halves, one of quarters.
__device__ __forceinline__ float groups_sum(const float (&v)[4]) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[0]), __float_as_uint(v[2]), false, false);
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[1]), __float_as_uint(v[3]), false, false);
    const float even = __uint_as_float(x[0]) + __uint_as_float(x[1]), odd = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    const auto z = __builtin_amdgcn_permlane16_swap(__float_as_uint(even), __float_as_uint(odd), false, false);
    return __uint_as_float(z[0]) + __uint_as_float(z[1]);
}

// grid = (n_splits * B, H_kv); QL bf16 numbers of a query.  SHARED: the four wavefronts have the same 32 tokens and every fourth 16 rows, and
// add up in LDS, where there are too few tokens for a resident round of workgroups that have 32 for each wavefront (16 x 128 rows of 3000 tokens:
// 25.4 us by tokens, 20.5 shared).
template <int P, bool N16, int QL, bool SHARED>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(QL == 1 ? 3 : 2))) void accumulate_weights(Args a) {
    constexpr int kChunk = QL == 3 ? 64 : 128;                   // rows in LDS
    constexpr int kTileTokens = SHARED ? kWaveTokens : 4 * kWaveTokens, kStep = SHARED ? 4 : 1;
    __shared__ __align__(16) uint8_t q_s[QL * kChunk * 256];
    __shared__ RowRule rule_s[kChunk];
    __shared__ float ref_s[kChunk];                              // -lse in base 2; minus infinity: the row has no weights to give
    __shared__ int at_s[kD];                                     // position of a channel of the query
    __shared__ int depth_s[64];
    __shared__ float sum_s[2][4][kWaveTokens];                   // SHARED: in turns
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, group = lane >> 4;
    const Place place = place_at(a, blockIdx.x);
    if (place.split < 0) return;
    const int b = place.b, kvh = blockIdx.y;
    const Seq s = sequence(a, b, place.len);
    const int tiles = (s.len + kTileTokens - 1) / kTileTokens, last16 = (s.len - 1) & ~15;
    if (place.split >= tiles) return;                            // (uniform for the workgroup)
    const int64_t unit = (int64_t)b * a.H_kv + kvh;
    const float mul = a.score_mul * (float)(1 << Decode<P>::kShift);
    const ChunkAt whole = chunk_at<P, N16>(a, l16, group);

    if (tid < 64) depth_s[tid] = tid < a.n_tok ? node_depth(node_mask(a, b, tid), tid) : 0;
    for (int r0 = 0; r0 < a.M; r0 += kChunk) {
        StagedRows<P, QL, kChunk, SHARED ? (QL == 3 ? 2 : 4) : 1> queries;
        queries.request(a, b, kvh, r0);
        int lo_least, lo_most;
        row_limits(a, s, b, r0, kChunk, lo_least, lo_most);
        struct Tile {
            Chunk<P, N16> raw[kStages];
            float before;                                        // what the lane's token has so far
        } next;                                                  // one tile in flight
        auto sees = [&](int t0) { return t0 < s.len && (t0 < s.prefix || t0 + kWaveTokens > min(lo_least, max(s.base, 0))); };
        // (without a branch: a load whose result meets another value behind it would be waited for there.  Tiles behind the last one and
        // those that no row sees stand for something that is read anyway.)
        auto request = [&](int v, Tile& to) {
            v = min(v, tiles - 1);
            int t0 = v * kTileTokens + (SHARED ? 0 : wave) * kWaveTokens;
            const int64_t mine = unit * a.w_stride + min(t0 + min(lane, kWaveTokens - 1), s.len - 1);
            to.before = *(r0 > 0 ? a.w_out + mine : a.w_in ? a.w_in + mine : a.lse_in);
            t0 = sees(t0) ? t0 : last16;
#pragma unroll
            for (int st = 0; st < kStages; ++st) {
                const int from = min(t0 + 16 * st, last16);
                ChunkAt at = whole;
                if (t0 + kWaveTokens > s.len) at = chunk_at<P, N16>(a, min(t0 + 16 * st + l16, s.len - 1) - from, group);
                load_chunk<P, N16>(a, a.k_mant, a.k_exp, stage_row(a, b, kvh, from), at, to.raw[st]);
            }
        };
        request(place.split, next);
        queries.place(at_s);
        lds_only_barrier();                                      // at_s is complete; nobody looks at the rows before these any more
        const int rows = min(a.M - r0, kChunk), groups = (rows + 15) / 16;
        queries.put(a, b, kvh, r0, q_s, at_s);
        if (tid < kChunk) {
            rule_s[tid] = row_rule(a, s, b, kvh, r0 + tid);
            ref_s[tid] = reference(a, b, kvh, r0 + tid);
        }
        lds_only_barrier();
        auto step = [&](int v, Tile& from) {
            const int t0 = v * kTileTokens + (SHARED ? 0 : wave) * kWaveTokens;
            if (t0 >= s.len) return;
            float* const w_out = a.w_out + unit * a.w_stride + t0 + lane;
            const bool mine = lane < kWaveTokens && t0 + lane < s.len;
            const float before = from.before;                    // (not multiplied before it is used: that would wait for it)
            float acc[kStages] = {};
            const bool seen = sees(t0), inner = t0 >= lo_most && t0 + kWaveTokens <= s.base;
            bf16x8 k[kStages][4];
            if (seen) {
#pragma unroll
                for (int st = 0; st < kStages; ++st)
#pragma unroll
                    for (int j = 0; j < 4; ++j) k[st][j] = __builtin_bit_cast(bf16x8, eight<P, N16>(from.raw[st], j));
            }
            request(v + place.n, from);
            auto scores = [&](int g, f32x4 (&sc)[kStages]) {
#pragma unroll
                for (int st = 0; st < kStages; ++st) sc[st] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int n = 0; n < QL; ++n) {
                        const bf16x8 q = staged_operand<kChunk>(q_s, n, 16 * g, l16, group, j);
#pragma unroll
                        for (int st = 0; st < kStages; ++st) sc[st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q, k[st][j], sc[st], 0, 0, 0);
                    }
            };
            if (seen && inner && a.cap == 0.f && !a.slopes) {
#pragma unroll 1
                for (int g = SHARED ? wave : 0; g < groups; g += kStep) {
                    f32x4 sc[kStages];
                    scores(g, sc);
                    const f32x4 ref = *(const f32x4*)(ref_s + 16 * g + 4 * group);
#pragma unroll
                    for (int st = 0; st < kStages; ++st)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[st] += exp2_raw(fmaf(sc[st][i], mul, ref[i]));
                }
            } else if (seen) {
#pragma unroll 1
                for (int g = SHARED ? wave : 0; g < groups; g += kStep) {
                    f32x4 sc[kStages];
                    scores(g, sc);
                    const f32x4 ref = *(const f32x4*)(ref_s + 16 * g + 4 * group);
                    float y[4 * kStages];
#pragma unroll
                    for (int i = 0; i < 4 * kStages; ++i) y[i] = sc[i >> 2][i & 3];
                    rule_tokens<kStages>(a, s, rule_s + 16 * g + 4 * group, depth_s, inner, t0 + l16, mul, y);
#pragma unroll
                    for (int i = 0; i < 4 * kStages; ++i) acc[i >> 2] += exp2_raw(y[i] + ref[i & 3]);
                }
            }
            // lane: token 16 group + l16
            float got = 0.f;
#pragma unroll
            for (int st = 0; st < kStages; ++st) {
                const float sum = rows_sum(acc[st]);
                if (group == st) got = sum;
            }
            if (SHARED) {
                float (&sums)[4][kWaveTokens] = sum_s[(v / place.n) & 1];
                if (lane < kWaveTokens) sums[wave][lane] = got;
                lds_only_barrier();                              // (the next tile's sums are the other ones)
                if (wave > 0) return;
                got = lane < kWaveTokens ? (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]) : 0.f;
            }
            if (mine) *w_out = r0 > 0 ? before + got : a.w_in ? fmaf(a.decay, before, got) : got;
        };
        for (int v = place.split; v < tiles; v += place.n) step(v, next);
    }
}

// Up to 16 rows of long sequences: the queries stay in registers, a wavefront has 64 tokens at a time, whose keys are decoded and multiplied
// stage by stage, and in the end a token of its own in each lane: 125 vector instructions for 32 tokens instead of 217, and more wavefronts.  From one
// workgroup a compute unit on: 8 x 8 heads of 32768 tokens 44.8 -> 35 us, ragged 16 x 32 of 1000 20.4 -> 13.9, 2 x 8 of 8000 8.8 -> 7.3;
// below, 1 x 8 of 4000 5.8 -> 6.5.  grid = (n_splits * B, H_kv).
constexpr int kFewStages = 4, kFewTokens = 16 * kFewStages;
template <int P, bool N16, int QL>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(QL == 1 && P == 4 ? 4 : 3))) void accumulate_weights_few(Args a) {
    constexpr int kTileTokens = 4 * kFewTokens;
    __shared__ __align__(16) uint8_t q_s[QL * 16 * 256];
    __shared__ RowRule rule_s[16];
    __shared__ float ref_s[16];
    __shared__ int at_s[kD];
    __shared__ int depth_s[64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, group = lane >> 4;
    const Place place = place_at(a, blockIdx.x);
    if (place.split < 0) return;
    const int b = place.b, kvh = blockIdx.y;
    StagedRows<P, QL, 16, 1> queries;
    queries.request(a, b, kvh, 0);
    const Seq s = sequence(a, b, place.len);
    const int tiles = (s.len + kTileTokens - 1) / kTileTokens, last16 = (s.len - 1) & ~15;
    if (place.split >= tiles) return;                            // (uniform for the workgroup)
    const int64_t unit = (int64_t)b * a.H_kv + kvh;
    const float mul = a.score_mul * (float)(1 << Decode<P>::kShift);
    const ChunkAt whole = chunk_at<P, N16>(a, l16, group);
    int lo_least, lo_most;
    row_limits(a, s, b, 0, 16, lo_least, lo_most);
    auto sees = [&](int t0) { return t0 < s.len && (t0 < s.prefix || t0 + kFewTokens > min(lo_least, max(s.base, 0))); };
    Chunk<P, N16> raw[kFewStages];
    float before;                                                // what the lane's token has so far
    auto request = [&](int v) {                                  // (without a branch, as above)
        int t0 = min(v, tiles - 1) * kTileTokens + wave * kFewTokens;
        const int64_t mine = unit * a.w_stride + min(t0 + lane, s.len - 1);
        before = *(a.w_in ? a.w_in + mine : a.lse_in);
        t0 = sees(t0) ? t0 : last16;
#pragma unroll
        for (int st = 0; st < kFewStages; ++st) {
            const int from = min(t0 + 16 * st, last16);
            ChunkAt at = whole;
            if (t0 + kFewTokens > s.len) at = chunk_at<P, N16>(a, min(t0 + 16 * st + l16, s.len - 1) - from, group);
            load_chunk<P, N16>(a, a.k_mant, a.k_exp, stage_row(a, b, kvh, from), at, raw[st]);
        }
    };
    request(place.split);
    if (tid < 64) depth_s[tid] = tid < a.n_tok ? node_depth(node_mask(a, b, tid), tid) : 0;
    if (tid < 16) {
        rule_s[tid] = row_rule(a, s, b, kvh, tid);
        ref_s[tid] = reference(a, b, kvh, tid);
    }
    queries.place(at_s);
    lds_only_barrier();                                          // (the first cached rows are on their way)
    queries.put(a, b, kvh, 0, q_s, at_s);
    lds_only_barrier();
    bf16x8 q[QL][4];
#pragma unroll
    for (int n = 0; n < QL; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) q[n][j] = staged_operand<16>(q_s, n, 0, l16, group, j);
    const f32x4 ref = *(const f32x4*)(ref_s + 4 * group);
    for (int v = place.split; v < tiles; v += place.n) {
        const int t0 = v * kTileTokens + wave * kFewTokens;
        if (t0 >= s.len) break;                                  // the wavefront's part of the last tile is empty
        const bool seen = sees(t0), inner = t0 >= lo_most && t0 + kFewTokens <= s.base;
        f32x4 sc[kFewStages];
#pragma unroll
        for (int st = 0; st < kFewStages; ++st) sc[st] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (seen) {
#pragma unroll
            for (int st = 0; st < kFewStages; ++st)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bf16x8 k = __builtin_bit_cast(bf16x8, eight<P, N16>(raw[st], j));
#pragma unroll
                    for (int n = 0; n < QL; ++n) sc[st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[n][j], k, sc[st], 0, 0, 0);
                }
        }
        const float was = before;                                // (not multiplied before it is used: that would wait for it)
        request(v + place.n);
        float acc[kFewStages] = {};
        if (seen && inner && a.cap == 0.f && !a.slopes) {
#pragma unroll
            for (int st = 0; st < kFewStages; ++st)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[st] += exp2_raw(fmaf(sc[st][i], mul, ref[i]));
        } else if (seen) {
            float y[4 * kFewStages];
#pragma unroll
            for (int i = 0; i < 4 * kFewStages; ++i) y[i] = sc[i >> 2][i & 3];
            rule_tokens<kFewStages>(a, s, rule_s + 4 * group, depth_s, inner, t0 + l16, mul, y);
#pragma unroll
            for (int i = 0; i < 4 * kFewStages; ++i) acc[i >> 2] += exp2_raw(y[i] + ref[i & 3]);
        }
        const float got = groups_sum(acc);
        if (t0 + lane < s.len) a.w_out[unit * a.w_stride + t0 + lane] = a.w_in ? fmaf(a.decay, was, got) : got;
    }
}

enum Form { kFew, kTokens, kShared };
template <int P, bool N16, int QL>
void launch(const Args& a, Form form, hipStream_t s) {
    const dim3 grid((unsigned)(a.n_splits * a.batch), (unsigned)a.H_kv);
    if (form == kFew) accumulate_weights_few<P, N16, QL><<<grid, kThreads, 0, s>>>(a);
    else if (form == kShared) accumulate_weights<P, N16, QL, true><<<grid, kThreads, 0, s>>>(a);
    else accumulate_weights<P, N16, QL, false><<<grid, kThreads, 0, s>>>(a);
}
template <int P, bool N16>
void launch(const Args& a, int dt, Form form, hipStream_t s) {
    if (dt == KVBFP_F32) launch<P, N16, 3>(a, form, s);
    else if (dt == KVBFP_F16) launch<P, N16, 2>(a, form, s);
    else launch<P, N16, 1>(a, form, s);
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
    const size_t bytes = (size_t)a.batch * (size_t)a.H_kv * (size_t)weights_stride * sizeof(float);
    if (weights_in && weights_in != weights_out && (uintptr_t)weights_in < (uintptr_t)weights_out + bytes &&
        (uintptr_t)weights_out < (uintptr_t)weights_in + bytes)
        return fail(KVBFP_ERR_INVALID_ARG, "%s: weights_out overlaps weights_in without being the same", call);
    if (!std::isfinite(decay)) return fail(KVBFP_ERR_INVALID_ARG, "%s: decay is not finite", call);
    if (a.H_kv > 65535) return fail(KVBFP_ERR_UNSUPPORTED, "%s: too many heads for the grid", call);
    a.perm_k = perm_k;
    a.lse_in = lse; a.w_in = weights_in; a.w_out = weights_out; a.w_stride = weights_stride; a.decay = decay;
    if (int rc = check_arrays(call, L, a, (size_t)dtype_size(dtype), {{"weights_out", weights_out, bytes, sizeof(float)}})) return rc;
    const int64_t units = (int64_t)a.batch * a.H_kv;
    const auto tiles_of = [&](int64_t tokens) { return (max_len + tokens - 1) / tokens; };
    // as many workgroups as the compute units have room for
    const int64_t few = dtype == KVBFP_BF16 && logical.mant_bits == 4 ? 1024 : 768, many = dtype == KVBFP_F16 ? 512 : 768;
    const Form form = a.M <= 16 && tiles_of(4 * kFewTokens) * units >= 256 ? kFew
                    : a.M > 16 && tiles_of(4 * kWaveTokens) * units < many    ? kShared
                                                                               : kTokens;
    const int64_t tiles = tiles_of(form == kFew ? 4 * kFewTokens : form == kShared ? kWaveTokens : 4 * kWaveTokens);
    const int64_t round = form == kFew ? few : many;
    const bool shares = seq_len_dev && a.batch > 1 && a.batch <= 64;
    a.n_splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(tiles, round_of(round, units, shares)));
    a.share = shares && a.n_splits > 1;
    hipStream_t s = (hipStream_t)hip_stream;
    const bool n16 = logical.block == 16;
    if (logical.mant_bits == 4) {
        if (n16) launch<4, true>(a, (int)dtype, form, s);
        else launch<4, false>(a, (int)dtype, form, s);
    } else {
        if (n16) launch<8, true>(a, (int)dtype, form, s);
        else launch<8, false>(a, (int)dtype, form, s);
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
