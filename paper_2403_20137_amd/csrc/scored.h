// Attention with a rule on its scores, and the weights it gives to cached tokens: argument block, the rule itself and the reading of
// packed rows, shared by decode_scored.hip and weights.hip (internal, not part of the C ABI).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "decode_dev.h"
#include "kvbfp_internal.h"

namespace kvbfp {
namespace scored {

using namespace kvbfp::dev;

struct Args {
    const uint8_t* k_mant;
    const uint8_t* k_exp;
    const uint8_t* v_mant;
    const uint8_t* v_exp;
    const void* q;             // [B][n_tok][H_q][D]
    void* out;                 // the same
    float* lse;                // [B][n_tok][H_q] or nullptr
    const int32_t* seq_len;    // [B] or nullptr
    const int32_t* perm_k;     // [H_kv][D] or nullptr
    const int32_t* perm_v;
    float* part_o;             // [H_kv][M][n_splits * B][D], in the order of the positions in LDS (see position_channel)
    float* part_ml;            // [H_kv][M][n_splits * B][2]: reference (base 2), sum of the weights relative to it
    const int32_t* block_table;
    int64_t table_stride, max_seq;
    int32_t log2_page, n_pages;
    int32_t max_len, batch, H_kv, H_q, G, n_tok;
    int32_t M;                 // rows of a kv-head: query token * G + member of its group
    int32_t n_splits, row_tiles;
    int32_t share;             // the n_splits * B places of a kv-head are shared out by the lengths
    int32_t n_exps, log2_block;
    float score_mul;           // softmax_scale * log2(e): scores are kept in base 2
    float cap, inv_cap;        // base 2; cap = 0: none
    const float* slopes;       // [H_q] or nullptr
    const int32_t* first;      // [B][n_tok] or nullptr
    const int32_t* prefix;     // [B] or nullptr
    const uint64_t* tree;      // [B][n_tok] (tree_stride 0: [n_tok], one for all) or nullptr: each token sees those up to itself
    int32_t tree_stride;
    int32_t window;            // 0: none
    // kvbfp_accumulate_weights
    const float* lse_in;       // [B][n_tok][H_q]
    const float* w_in;         // [B][H_kv][w_stride] or nullptr
    float* w_out;
    int64_t w_stride;
    float decay;
};

// What a kernel knows of its sequence.
struct Seq {
    int32_t len, base, prefix;           // tokens [base, len) are the last n_tok; base may be negative
};
__device__ __forceinline__ Seq sequence(const Args& a, int b, int len) {
    Seq s;
    s.len = len;
    s.base = s.len - a.n_tok;
    s.prefix = a.prefix ? min(max(a.prefix[b], 0), s.len) : 0;
    return s;
}

// Which part of which sequence a place takes: part `split` of `n`, the places of the sequence begin at `first`.  Equal parts
// (n_splits each), or shared out by what the sequences have to read (up to 64 of them, a lane each): one each, the others in
// proportion, rounded down, what is left by the largest remainders.
struct Place { int b, split, n, first, len; };
// Splits of each sequence and head that fill one resident round of workgroups; two where they are shared out by lengths and more than one
// fits: with one split the longest sequence is one workgroup's.
inline int64_t round_of(int64_t round, int64_t units, bool shares) { return round / units == 1 && shares && round > units ? 2 : round / units; }
__device__ __forceinline__ int length_of(const Args& a, int b) { return a.seq_len ? min(max(a.seq_len[b], 0), a.max_len) : a.max_len; }
// Lane b: the places of sequence b, the first of them, its length.
__device__ __forceinline__ void share_places(const Args& a, int lane, int& n, int& first, int& len) {
    len = length_of(a, min(lane, a.batch - 1));
    int read = len;                      // about what there is to read: documents are not looked at
    if (a.window) read = tokens_read(len, a.window, a.n_tok, a.prefix ? min(max(a.prefix[min(lane, a.batch - 1)], 0), len) : 0);
    const float mine = lane < a.batch ? (float)(read + 1) : 0.f;
    const float all = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(wave_scan(mine)), 63));
    const float extra = (float)((a.n_splits - 1) * a.batch);
    const float share = extra * (mine / all) * (1.f + 0x1p-20f);         // (a whole number stays one)
    n = lane < a.batch ? 1 + (int)share : 0;
    // the sum of rounded-down shares is at most what there is to share
    const int left = a.n_splits * a.batch - __builtin_amdgcn_readlane(wave_scan(n), 63);
    const float rest = share - floorf(share);
    int before = 0;
    for (int j = 0; j < a.batch; ++j) {
        const float other = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(rest), j));
        before += other > rest || (other == rest && j < lane);
    }
    if (lane < a.batch && before < left) ++n;
    first = wave_scan(n) - n;
}
// The place `at`; split = -1: nobody's.
__device__ __forceinline__ Place place_at(const Args& a, int at) {
    Place p;
    if (!a.share) {
        p.b = at / a.n_splits;
        p.split = at - p.b * a.n_splits;
        p.n = a.n_splits;
        p.first = at - p.split;
        p.len = length_of(a, p.b);
        return p;
    }
    int n, first, len;
    share_places(a, threadIdx.x & 63, n, first, len);
    const uint64_t found = __ballot(at >= first && at < first + n);
    const int who = found ? __ffsll((unsigned long long)found) - 1 : 0;
    p.b = __builtin_amdgcn_readfirstlane(who);
    p.n = __builtin_amdgcn_readlane(n, p.b);
    p.first = __builtin_amdgcn_readlane(first, p.b);
    p.len = __builtin_amdgcn_readlane(len, p.b);
    p.split = found ? at - p.first : -1;
    return p;
}
// The places of sequence b.
__device__ __forceinline__ Place places_of(const Args& a, int b) {
    Place p = {b, 0, a.n_splits, b * a.n_splits, 0};
    if (a.share) {
        int n, first, len;
        share_places(a, threadIdx.x & 63, n, first, len);
        p.n = __builtin_amdgcn_readlane(n, b);
        p.first = __builtin_amdgcn_readlane(first, b);
    }
    return p;
}

// Nodes that node i of sequence b sees (bits behind the last node mean nothing).
__device__ __forceinline__ uint64_t node_mask(const Args& a, int b, int i) {
    if (a.tree) return a.tree[(int64_t)b * a.tree_stride + i] & (~0ull >> (64 - a.n_tok));
    return i >= 63 ? ~0ull : (2ull << i) - 1;
}
// Its position behind the tokens before the nodes: how many others it sees.
__device__ __forceinline__ int node_depth(uint64_t mask, int i) { return __popcll(mask & ~(1ull << i)); }

// The rule for one row (query token, head).
struct RowRule {
    uint64_t nodes;
    int32_t lo;                // tokens before the nodes are seen from here on
    int32_t first, pos;        // nodes: from `first` on, nearer than the window
    float slope;               // base 2
};
// The tokens before the nodes that rows r0 .. r0 + count see (count <= 128): none before `least`, all of them from `most` on.  By
// every wavefront for itself.
__device__ __forceinline__ void row_limits(const Args& a, const Seq& s, int b, int r0, int count, int& least, int& most) {
    least = most = 0;
    if (!a.first && !a.window) return;
    least = INT32_MAX;
    most = INT32_MIN;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = min(r0 + min((int)(threadIdx.x & 63) + 64 * h, count - 1), a.M - 1) / a.G;
        const int first = a.first ? a.first[(int64_t)b * a.n_tok + i] : 0;
        const int lo = a.window ? max(first, s.base + node_depth(node_mask(a, b, i), i) - a.window + 1) : first;
        least = min(least, lo);
        most = max(most, lo);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        least = min(least, __shfl_xor(least, d));
        most = max(most, __shfl_xor(most, d));
    }
    least = __builtin_amdgcn_readfirstlane(least);
    most = __builtin_amdgcn_readfirstlane(most);
}
__device__ __forceinline__ RowRule row_rule(const Args& a, const Seq& s, int b, int kvh, int r) {
    r = min(r, a.M - 1);
    const int i = r / a.G, head = kvh * a.G + r - i * a.G;
    RowRule u;
    u.nodes = node_mask(a, b, i);
    u.pos = s.base + node_depth(u.nodes, i);
    u.first = a.first ? a.first[(int64_t)b * a.n_tok + i] : 0;
    u.lo = a.window ? max(u.first, u.pos - a.window + 1) : u.first;
    u.slope = a.slopes ? a.slopes[head] * 1.4426950408889634f : 0.f;
    return u;
}

// y = cap * tanh(y / cap), x = y / cap.  Up to |x| = 0.9 as y + y x^2 q(x^2), q of degree 5 with the least largest error (1.6e-8 relative; with its roundings
// 1.7 times 2^-24); beyond, where the difference cancels no more, as cap - 2 cap / (1 + e^(2 x)), within 6 times 2^-24 of the result.  That form alone for every
// score is off by 4 times 2^-24 of the cap, twelve times as much as tanh in fp32 where scores are a fifteenth of it, and lse is an fp32 output.
// One branch asks on behalf of all N scores whether any is beyond.
template <int N>
__device__ __forceinline__ void cap_scores(float (&y)[N], float mul, float cap, float inv_cap) {
    float most = 0.f, v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        y[i] *= mul;
        const float x = y[i] * inv_cap, z = x * x;
        float q = fmaf(z, 0.00130395917f, -0.00686005456f);
        q = fmaf(z, q, 0.0209041256f);
        q = fmaf(z, q, -0.0537214912f);
        q = fmaf(z, q, 0.133303598f);
        q = fmaf(z, q, -0.333332121f);
        v[i] = fmaf(y[i] * z, q, y[i]);
        most = fmaxf(most, fabsf(x));
    }
    constexpr float kSeries = 0.9f;
    if (__builtin_amdgcn_ballot_w64(most > kSeries)) {
        const float turn = inv_cap * 2.8853900817779268f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float e = fmaf(-2.f * cap, __builtin_amdgcn_rcpf(1.f + exp2_raw(y[i] * turn)), cap);
            v[i] = fabsf(y[i] * inv_cap) > kSeries ? e : v[i];
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = v[i];
}

// Scores (base 2) of one row for the tokens t0 + 16 (i / 4) + i % 4, i < N, from the products of query and keys, which times `mul` are the
// plain scores; -inf where a token is not seen.  `inner`: all of them are seen, and are no nodes.  Returns what they are still to
// be multiplied with: 1, or a positive `mul` that nothing has to come before, which costs nothing in the exponent's multiply-add.  The rule
// lies in LDS: few tiles ask for it.
template <int N>
__device__ __forceinline__ float rule_scores(const Args& a, const Seq& s, const RowRule* rule_s, const int* depth_s, bool inner, int t0, float mul,
                                             float (&y)[N]) {
    float factor = 1.f;
    if (a.cap != 0.f) {
        cap_scores<N>(y, mul, a.cap, a.inv_cap);
    } else if (a.slopes || !(mul > 0.f)) {
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] *= mul;
    } else {
        factor = mul;
    }
    if (inner) {
        if (a.slopes) {
            const float far = (float)(rule_s->pos - t0), slope = rule_s->slope;
#pragma unroll
            for (int i = 0; i < N; ++i) y[i] = fmaf(-slope, far - (float)(16 * (i >> 2) + (i & 3)), y[i]);
        }
        return factor;
    }
    const RowRule u = *rule_s;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int t = t0 + 16 * (i >> 2) + (i & 3), node = t - s.base;
        bool seen = t >= u.lo;
        int far = u.pos - t;
        if (node >= 0) {
            far = u.pos - s.base - depth_s[node & 63];
            seen = ((u.nodes >> (node & 63)) & 1) && t >= u.first && (a.window == 0 || far < a.window);
        }
        seen = (seen || t < s.prefix) && t < s.len;
        if (a.slopes) y[i] = fmaf(-u.slope, fabsf((float)far), y[i]);
        y[i] = seen ? y[i] : -INFINITY;
    }
    return factor;
}

// The same for four rows (rule_s[0] ..) of the ST tokens t0 + 16 st, y[4 st + row]; everything multiplied.
template <int ST>
__device__ __forceinline__ void rule_tokens(const Args& a, const Seq& s, const RowRule* rule_s, const int* depth_s, bool inner, int t0, float mul,
                                            float (&y)[4 * ST]) {
    if (a.cap != 0.f) {
#pragma unroll
        for (int st = 0; st < ST; ++st) {
            float v[4] = {y[4 * st], y[4 * st + 1], y[4 * st + 2], y[4 * st + 3]};
            cap_scores<4>(v, mul, a.cap, a.inv_cap);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[4 * st + i] = v[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4 * ST; ++i) y[i] *= mul;
    }
    if (inner) {
        if (a.slopes) {
#pragma unroll
            for (int i = 0; i < 4 * ST; ++i) y[i] = fmaf(-rule_s[i & 3].slope, (float)(rule_s[i & 3].pos - (t0 + 16 * (i >> 2))), y[i]);
        }
        return;
    }
    int depth[ST];
#pragma unroll
    for (int st = 0; st < ST; ++st) depth[st] = depth_s[(t0 + 16 * st - s.base) & 63];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const RowRule u = rule_s[i];
#pragma unroll
        for (int st = 0; st < ST; ++st) {                    // (both answers, one taken: a branch would wait for each read by itself)
            const int t = t0 + 16 * st, node = t - s.base;
            const bool drafted = node >= 0;
            const int far = u.pos - (drafted ? s.base + depth[st] : t);
            const bool near = (((u.nodes >> (node & 63)) & 1) != 0) & (t >= u.first) & ((a.window == 0) | (far < a.window));
            const bool seen = ((drafted ? near : t >= u.lo) | (t < s.prefix)) & (t < s.len);
            float v = y[4 * st + i];
            if (a.slopes) v = fmaf(-u.slope, fabsf((float)far), v);
            y[4 * st + i] = seen ? v : -INFINITY;
        }
    }
}

// 32 channels of one cached row, as loaded: lane (row l % 16 of a stage of 16 tokens, chunk l / 16).  N16: blocks of 16, two in a chunk.
template <int P, bool N16>
struct Chunk {
    u32x4 m[P / 4];
    uint32_t e[N16 ? 2 : 1];
};
// Where in a stage's rows a lane's chunk lies: bytes of the mantissa and of the exponent plane.  The same for every stage but the last.
struct ChunkAt { uint32_t m, e; };
template <int P, bool N16>
__device__ __forceinline__ ChunkAt chunk_at(const Args& a, int row, int chunk) {
    return ChunkAt{(uint32_t)(row * (16 * P) + chunk * (4 * P)), (uint32_t)(row * a.n_exps + (N16 ? 2 * chunk : (chunk * 32) >> a.log2_block))};
}
template <int P, bool N16>
__device__ __forceinline__ void load_chunk(const Args& a, const uint8_t* mant, const uint8_t* exps, int64_t row0, ChunkAt at, Chunk<P, N16>& c) {
    const uint8_t* const m = mant + row0 * (16 * P);
    const uint8_t* const e = exps + row0 * a.n_exps;
#pragma unroll
    for (int i = 0; i < P / 4; ++i) c.m[i] = __builtin_nontemporal_load((const u32x4*)(m + at.m) + i);
#pragma unroll
    for (int i = 0; i < (N16 ? 2 : 1); ++i) c.e[i] = e[at.e + i];
}

// Row of the planes that a stage of 16 tokens (t a multiple of 16, t < len) begins at.  Page numbers come from device memory that the
// host cannot check: they are clamped to the pool.
__device__ __forceinline__ int64_t stage_row(const Args& a, int b, int kvh, int t) {
    if (!a.block_table) return ((int64_t)b * a.H_kv + kvh) * a.max_seq + t;
    int page = a.block_table[(int64_t)b * a.table_stride + (t >> a.log2_page)];
    page = min(max(page, 0), a.n_pages - 1);
    return (((int64_t)page * a.H_kv + kvh) << a.log2_page) + (t & ((1 << a.log2_page) - 1));
}

// Codes are decoded to bf16 as value * 2^-kShift, exactly for exponent bytes 3 to the largest that fits the conversion's operand; bytes
// above it are taken as that one, so that a row that is not seen cannot bring an infinity into a product with 0.
template <int P>
struct Decode {
    static constexpr int kShift = P == 4 ? 7 : 3;
    static constexpr uint32_t kTop = P == 4 ? 254u : 251u;
};
template <int P>
__device__ __forceinline__ uint32_t exp_field(uint32_t e) { return min(e, Decode<P>::kTop) << 23; }

__device__ __forceinline__ uint32_t pack_top(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }

// Channels [8 j, 8 j + 8) of a chunk as eight bf16, in the order of the conversions (4 bits: even channels, then odd ones).
template <int P, bool N16>
__device__ __forceinline__ u32x4 eight(const Chunk<P, N16>& c, int j) {
    const uint32_t field = exp_field<P>(c.e[N16 ? j >> 1 : 0]);
    u32x4 r;
    if constexpr (P == 4) {
        const Unpacked4 u = unpack8_p4(c.m[0][j], __uint_as_float(field));
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, u.p[i]);
    } else {
        // a byte s mmmm lll is the sum of the FP8 numbers s000mmmm (eight times the scale) and s0000lll; seven significant bits
        const float s_lo = __uint_as_float(field), s_hi = __uint_as_float(field + (3u << 23));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t hi, lo;
            spread8(c.m[j >> 1][(2 * j + h) & 3], hi, lo);
            const auto h01 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, s_hi, false), h23 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, s_hi, true);
            const auto l01 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(lo, s_lo, false), l23 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(lo, s_lo, true);
            r[2 * h] = pack_top(__float_as_uint(h01[0] + l01[0]), __float_as_uint(h01[1] + l01[1]));
            r[2 * h + 1] = pack_top(__float_as_uint(h23[0] + l23[0]), __float_as_uint(h23[1] + l23[1]));
        }
    }
    return r;
}
// Cache channel of position p of a row decoded that way.
template <int P>
__host__ __device__ __forceinline__ int position_channel(int p) {
    if (P == 8) return p;
    const int x = p & 7;
    return (p & ~7) | ((x < 4) ? 2 * x : 2 * (x - 4) + 1);
}

// All-reduce over the four 16-lane rows of a wavefront.
__device__ __forceinline__ float rows_max(float v) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
    const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float rows_sum(float v) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(y[0]) + __uint_as_float(y[1]);
}

__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The element type goes with the number of bf16 numbers that hold one of its values: bf16 one, fp16 two, fp32 three.
template <int QL>
struct Io { typedef __bf16 T; };
template <>
struct Io<2> { typedef _Float16 T; };
template <>
struct Io<3> { typedef float T; };

// ROWS query rows from r0 on (zeros behind the last row of the kv-head) on their way to q_s[ROWS][kQStride] as fp32, in the query's own channel
// order, and the permutation to perm_s[kD].  Called by the whole workgroup of 256; the caller puts a barrier behind put().
constexpr int kQStride = kD + 4;
template <int QL, int ROWS>
struct QueryRows {
    typedef typename Io<QL>::T T;
    typedef T Tx8 __attribute__((ext_vector_type(8)));
    Tx8 x[ROWS / 16];
    int perm;
    __device__ __forceinline__ void request(const Args& a, int b, int kvh, int r0) {
        const int tid = threadIdx.x;
        perm = a.perm_k ? a.perm_k[kvh * kD + (tid & (kD - 1))] & (kD - 1) : tid & (kD - 1);      // masked: stays inside the row
        const bool vec = ((uintptr_t)a.q & 15u) == 0;
#pragma unroll
        for (int p = 0; p < ROWS / 16; ++p) {
            const int c = (tid & 15) * 8, r = r0 + (tid >> 4) + 16 * p, rc = min(r, a.M - 1), tok = rc / a.G;
            const T* const src = (const T*)a.q + (((int64_t)b * a.n_tok + tok) * a.H_q + (int64_t)kvh * a.G + (rc - tok * a.G)) * kD + c;
            if (vec) {
                x[p] = *(const Tx8*)src;
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) x[p][k] = src[k];
            }
        }
    }
    __device__ __forceinline__ void put(const Args& a, int r0, float* q_s, int* perm_s) const {
        const int tid = threadIdx.x;
        if (tid < kD) perm_s[tid] = perm;
#pragma unroll
        for (int p = 0; p < ROWS / 16; ++p) {
            const int row = (tid >> 4) + 16 * p;
            float* const to = q_s + row * kQStride + (tid & 15) * 8;
            const float there = r0 + row < a.M ? 1.f : 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4 v;
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = there != 0.f ? (float)x[p][4 * h + k] : 0.f;
                *(f32x4*)(to + 4 * h) = v;
            }
        }
    }
};

// x as QL bf16 numbers whose sum it is: bf16 has one, fp16 8 + 3 bits, fp32 three times 8.
template <int QL>
__device__ __forceinline__ void limbs(float x, __bf16 (&l)[QL]) {
#pragma unroll
    for (int i = 0; i < QL; ++i) {
        const uint32_t top = __float_as_uint(x) & 0xFFFF0000u;
        l[i] = __builtin_bit_cast(__bf16, (unsigned short)(top >> 16));
        x -= __uint_as_float(top);
    }
}

// The query operand of 16 rows: lane (row l % 16, group l / 16), step j: channels 32 group + 8 j .. in the order of eight().
template <int P, int QL>
__device__ __forceinline__ void query_operand(const float* q_s, const int* perm_s, int row, int group, bf16x8 (&op)[QL][4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            __bf16 l[QL];
            limbs<QL>(q_s[row * kQStride + perm_s[position_channel<P>(32 * group + 8 * j + x)]], l);
#pragma unroll
            for (int i = 0; i < QL; ++i) op[i][j][x] = l[i];
        }
    }
}

// Checks of the arguments that both calls have, and what the kernels need of them (score rule included).
// `L`: the pool where paging is given.  On success *logical is the layout that the sequences appear to have.
int fill_args(const char* call, const kvbfp_layout* L, const kvbfp_cache* cache, const Paging* paging, int32_t n_q_heads, int32_t n_q_tokens,
              const void* q, kvbfp_dtype dtype, const int32_t* seq_len_dev, int64_t max_len, float softmax_scale,
              const kvbfp_score_rule* rule, bool need_v, Args* a, kvbfp_layout* logical);
// What the call reads, as `a` has it by now, against what it writes.
int check_arrays(const char* call, const kvbfp_layout* L, const Args& a, size_t element, std::initializer_list<Span> written);

}  // namespace scored
}  // namespace kvbfp
