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
//
// What bounds it (times in a graph over three caches).  Few rows and long sequences: 8 x 8 heads of 32768 tokens, four rows each, capped scores, 61 us (4.7 TB/s; the
// same without the cap 58; 45 at the rate of a reading kernel): decoding to bf16 and the softmax issue vector instructions in 69 % of the cycles,
// and three workgroups a compute unit overlap them and the reading only in part.  Many rows: matrix and vector instructions, which hardly overlap within
// a compute unit, as the wavefronts of a workgroup go in step: 8 sequences of up to 8192 tokens with trees of 64 (256 rows a kv-head, capped) 152 us,
// 294 TFLOP/s of the two products, vector instructions in 72 % of the cycles, matrix instructions in 24 %; the second limb of the
// probabilities is a third of the matrix work and stays, as one bf16 is off by 2^-9 of every weight.  A short sequence: the way of
// the first loads and of the code itself, 7 to 9 us; loops that run once are not unrolled where that only makes them longer.
// Measured and not kept: products of the next tile ahead of the values of this one, two tiles in flight, four workgroups a compute unit, 32 rows a
// wavefront for 33 to 64 rows, rows of the output stored by channels.
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
constexpr int kTileTokens = 128;                 // scored_split: four wavefronts
constexpr int kWideTokens = 64;                  // scored_split_wide: a tile in LDS
constexpr int kOStride = kD + 4;
constexpr int kWaveLds = 16 * kOStride * 4;      // 32 rows of values in bf16 (8192 bytes) or 16 rows of outputs in fp32

// The tiles of a sequence that some row of the workgroup sees: those of the prefix, then those from the first token seen on.
template <int TT>
struct Tiles {
    int prefix, from, count;
    __device__ __forceinline__ int at(int v) const { return v < prefix ? v : from + (v - prefix); }
};
template <int TT>
__device__ __forceinline__ Tiles<TT> tiles_of(const Seq& s, int lo) {
    Tiles<TT> t;
    t.prefix = (s.prefix + TT - 1) / TT;
    t.from = max(min(max(lo, 0), max(s.base, 0)) / TT, t.prefix);
    t.count = t.prefix + max((s.len + TT - 1) / TT - t.from, 0);
    return t;
}

// Byte of a value row's 16-byte piece in LDS: 256 bytes a token; the eight 32-byte segments of a row are exchanged by its number, so that
// 8 rows of one segment lie in different banks, and the halves of a segment by the number's next bit, so that 16 rows written at once
// use all banks.
__device__ __forceinline__ int value_at(int row, int seg, int half) {
    return row * 256 + ((seg ^ (row & 7)) * 32) + ((half ^ ((row >> 3) & 1)) * 16);
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
__device__ __forceinline__ s16x4 read_by_channel(const uint8_t* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
}

// Values of 32 tokens by channel: the first operand of the value product for 16 channels each.
struct Values { bf16x8 v[8]; };
__device__ __forceinline__ bf16x8 values_of(const uint8_t* v_s, int lane, int ct) {
    const int i = lane & 15, row = 4 * (lane >> 4) + (i >> 2), half = (i >> 1) & 1, word = (i & 1) * 8;
    const s16x4 lo = read_by_channel(v_s + value_at(row, ct, half) + word);
    const s16x4 hi = read_by_channel(v_s + value_at(row + 16, ct, half) + word);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
// o += V^T P^T for 32 tokens and HC times 16 rows: lane (row l % 16): probabilities of tokens 4 (l / 16) .. of either stage.
template <int PL, int HC, class ByChannel>
__device__ __forceinline__ void add_values(ByChannel&& values, const bf16x8 (&p)[HC][PL], f32x4 (&o)[HC][8]) {
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) {
        const bf16x8 v = values(ct);
#pragma unroll
        for (int c = 0; c < HC; ++c)
#pragma unroll
            for (int l = 0; l < PL; ++l) o[c][ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[c][l], o[c][ct], 0, 0, 0);
    }
}

// Running maximum of one row.  The sums are relative to a reference that scores may exceed by 2^kSlack before they are rescaled: 16 rows
// have a new maximum nearly every tile otherwise, and 32 products each time.  Sums of values with exponent bytes up to kOrdinary have
// room for that (below 2^74, times 2^kSlack, times 2^30 tokens); from the first larger byte on no score may exceed the reference, and it rises above
// the maximum with the sum of the weights: the largest values, as decoded, are below 2^122, so that weights of 2^6 in all fit.
constexpr float kSlack = 8.f;
constexpr uint32_t kOrdinary = 200;
struct Running {
    float ref = -INFINITY, most = -INFINITY, sum = 0.f;       // (sum: of this lane's tokens, a quarter)
    // After a tile with large values (weights of 32 at most): sums beyond 16 go down by 2^4, the reference up.
    __device__ __forceinline__ void keep_room(f32x4 (&o)[8]) {
        const bool full = rows_max(sum) > 4.f;
        const float f = full ? 0x1p-4f : 1.f;
        ref += full ? 4.f : 0.f;
        sum *= f;
#pragma unroll
        for (int ct = 0; ct < 8; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[ct][i] *= f;
    }
};
// Takes N scores (y times factor, up to eight a lane) into account; returns what they are taken relative to.  `large`: there are such values.
template <int N>
__device__ __forceinline__ float follow(const float (&y)[N], float factor, bool large, Running& x, f32x4 (&o)[8]) {
    float top = y[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, y[i]);
    x.most = fmaxf(x.most, rows_max(top * factor));
    if (__builtin_amdgcn_ballot_w64(x.most > x.ref + (large ? 0.f : kSlack))) {        // (the reference begins at minus infinity)
        const float to = fmaxf(x.ref, x.most), f = to > -INFINITY ? exp2_raw(x.ref - to) : 1.f;
        x.ref = to;
        x.sum *= f;
#pragma unroll
        for (int ct = 0; ct < 8; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[ct][i] *= f;
    }
    return x.ref > -INFINITY ? x.ref : 0.f;
}
// N scores of a row -> its probabilities as bf16 pairs, PL of them for each, and their sum.
template <int PL, int N>
__device__ __forceinline__ void probabilities(const float (&y)[N], float factor, float base, float& sum, uint32_t (&p)[PL][N / 2]) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        __bf16 l[2][PL];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float w = exp2_raw(fmaf(y[2 * i + h], factor, -base));
            sum += w;
            limbs<PL>(w, l[h]);
            if (PL == 2) l[h][1] = (__bf16)(w - __uint_as_float(__float_as_uint(w) & 0xFFFF0000u));     // rounded, not cut
        }
#pragma unroll
        for (int x = 0; x < PL; ++x) p[x][i] = __builtin_bit_cast(uint32_t, bf16x2{l[0][x], l[1][x]});
    }
}
template <int P, bool N16>
__device__ __forceinline__ bool has_large(const Chunk<P, N16>& c) { return max(c.e[0], c.e[N16 ? 1 : 0]) > kOrdinary; }

// Scores of 32 tokens for HC times 16 rows: products of the keys of two stages of 16 tokens, key(stage, step) an operand, with the queries.
template <int QL, int HC, class Key>
__device__ __forceinline__ void products(Key&& key, const bf16x8 (&q)[HC][QL][4], float (&y)[HC][8]) {
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        f32x4 sc[HC];
#pragma unroll
        for (int c = 0; c < HC; ++c) sc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bf16x8 k = key(st, j);
#pragma unroll
            for (int c = 0; c < HC; ++c)
#pragma unroll
                for (int i = 0; i < QL; ++i) sc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[c][i][j], sc[c], 0, 0, 0);
        }
#pragma unroll
        for (int c = 0; c < HC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[c][4 * st + i] = sc[c][i];
    }
}

// One row of the output, or of lse, from its largest score, sum and sums of values.
template <int QL>
__device__ __forceinline__ void store_out(const Args& a, int64_t at, float v) {
    typedef typename Io<QL>::T T;
    ((T*)a.out)[at] = (T)v;
}
template <int QL>
__device__ __forceinline__ void store_eight(const Args& a, int64_t at, const float (&v)[8]) {
    typedef typename Io<QL>::T T;
    typedef T Tx8 __attribute__((ext_vector_type(8)));
    Tx8 x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (T)v[i];
    if (((uintptr_t)a.out & 15u) == 0) {
        *(Tx8*)((T*)a.out + at) = x;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) ((T*)a.out)[at + i] = x[i];
    }
}
__device__ __forceinline__ float natural_lse(float m, float l) {
    return l > 0.f ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
}
__device__ __forceinline__ int64_t out_row(const Args& a, int b, int kvh, int r) {
    const int tok = r / a.G;
    return ((int64_t)b * a.n_tok + tok) * a.H_q + (int64_t)kvh * a.G + (r - tok * a.G);
}

// Up to 8 times 768 parts are joined: sums with large values, whose weights are 2^5.6 at most in all, are joined 2^-16 times, and handed on so with a
// reference 16 higher.
constexpr float kDown = 0x1p-16f, kUp = 0x1p16f;

// Partial results of a wavefront's own 16 rows from r0 on.
__device__ __forceinline__ void store_partial(const Args& a, int kvh, int r0, int place, int lane, const f32x4 (&o)[8], const Running& x, bool large) {
    const int l16 = lane & 15, group = lane >> 4, r = r0 + l16;
    const float sum = rows_sum(x.sum), by = large ? kDown : 1.f;
    if (r >= a.M) return;
    const int64_t at = ((int64_t)kvh * a.M + r) * a.n_splits * a.batch + place;
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) *(f32x4*)(a.part_o + at * kD + 16 * ct + 4 * group) = o[ct] * by;
    if (group == 0) *(float2*)(a.part_ml + 2 * at) = make_float2(large ? x.ref + 16.f : x.ref, sum * by);
}
// The sums of a workgroup's wavefronts for RP * RW rows from r0 on, joined over the 4 / RW that hold the same rows (wavefront w: rows
// 16 (w % RW) .., or twice the same 8 rows, RP = 8, RW = 1) and written as this split's partial result, or as the output
// where there is one split.  smem: four times kWaveLds, free when this is called.
template <int P, int QL, int RW, int RP>
__device__ __forceinline__ void finish(const Args& a, int b, int kvh, int r0, int place, uint8_t* smem, float (*ml_s)[16][2], int wave, int lane,
                                       const f32x4 (&o)[8], const Running& x, bool large) {
    const int tid = threadIdx.x, l16 = lane & 15, group = lane >> 4;
    constexpr float up = (float)(1 << Decode<P>::kShift);       // (partial results keep the scale of the decoded values)
    float* const o_s = (float*)(smem + wave * kWaveLds);
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) *(f32x4*)(o_s + l16 * kOStride + 16 * ct + 4 * group) = o[ct];
    const float sum = rows_sum(x.sum);
    if (group == 0) {
        ml_s[wave][l16][0] = x.ref;
        ml_s[wave][l16][1] = large ? -sum : sum;             // (the sign says so)
    }
    const int row = tid >> 4, p0 = (tid & 15) * 8;
    int channel[8];
    if (a.n_splits == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            channel[i] = position_channel<P>(p0 + i);
            if (a.perm_v) channel[i] = a.perm_v[kvh * kD + channel[i]] & (kD - 1);
        }
    }
    __syncthreads();
#pragma unroll 1
    for (int rw = 0; rw < RW; ++rw) {
        const int r = r0 + 16 * rw + row;
        if (row >= RP || r >= a.M) continue;
        float top = -INFINITY, least = 0.f, den = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = rw; w < 4; w += RW)
#pragma unroll
            for (int h = 0; h < 16; h += RP) {
                top = fmaxf(top, ml_s[w][(row + h) & 15][0]);
                least = fminf(least, ml_s[w][(row + h) & 15][1]);
            }
        const bool any_large = least < 0.f;
        const float down = any_large ? kDown : 1.f;
#pragma unroll
        for (int w = rw; w < 4; w += RW) {
#pragma unroll
            for (int h = 0; h < 16; h += RP) {
                const int at = (row + h) & 15;
                if (!(ml_s[w][at][0] > -INFINITY)) continue;
                const float f = exp2_raw(ml_s[w][at][0] - top);
                den = fmaf(f, fabsf(ml_s[w][at][1]), den);
                const float* const src = (const float*)(smem + w * kWaveLds) + at * kOStride + p0;
                const float f_o = f * down;
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] = fmaf(f_o, src[i], acc[i]);
            }
        }
        if (a.n_splits > 1) {
            const int64_t at = ((int64_t)kvh * a.M + r) * a.n_splits * a.batch + place;
            if (p0 == 0) *(float2*)(a.part_ml + 2 * at) = make_float2(any_large ? top + 16.f : top, den * down);
            *(f32x4*)(a.part_o + at * kD + p0) = f32x4{acc[0], acc[1], acc[2], acc[3]};
            *(f32x4*)(a.part_o + at * kD + p0 + 4) = f32x4{acc[4], acc[5], acc[6], acc[7]};
        } else {
            // into the order of the output in LDS, where the row came from (nobody but these 16 lanes looks at it): stores of single
            // channels took longer than everything before them with 108 rows of two tokens, 23 us against 18.7
            const int64_t at = out_row(a, b, kvh, r);
            const float by = den > 0.f ? up / den * (any_large ? kUp : 1.f) : 0.f;
            float* const row_s = (float*)(smem + rw * kWaveLds) + row * kOStride;
            wave_fence();
#pragma unroll
            for (int i = 0; i < 8; ++i) row_s[channel[i]] = acc[i] * by;
            wave_fence();
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = row_s[p0 + i];
            store_eight<QL>(a, at * kD + p0, acc);
            if (p0 == 0 && a.lse) a.lse[at] = natural_lse(top, den);
        }
    }
}

// Up to 16 rows: every wavefront has all of them and takes 32 tokens of a tile of 128 for itself.  With up to 8 rows (RP = 8) the 16
// columns are these rows twice, once for either stage of 16 tokens: each lane then has four scores instead of eight, half of which would
// be nobody's; the columns are joined in the end like another wavefront's (8 x 32768 tokens 68 us with them once, 64.5 twice).
// grid = (n_splits * B, H_kv); P mantissa bits, N16 blocks of 16, QL bf16 numbers of a query.  <8, true, 1, 16> and <8, true, 1, 8> spill 3 registers and 1
// under three wavefronts a SIMD, which a workgroup needs 168 registers for; no other form does.
template <int P, bool N16, int QL, int RP>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(QL == 1 ? 3 : 2))) void scored_split(Args a) {
    constexpr int PL = QL == 3 ? 3 : 2;
    __shared__ __align__(16) uint8_t smem[4 * kWaveLds];
    __shared__ float ml_s[4][16][2];
    __shared__ int perm_s[kD];
    __shared__ int depth_s[64];
    __shared__ RowRule rule_s[16];
    static_assert(16 * kQStride * 4 <= 4 * kWaveLds, "the query rows fit");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, group = lane >> 4;
    const Place place = place_at(a, blockIdx.x);
    if (place.split < 0) return;
    const int b = place.b, kvh = blockIdx.y, n_splits = place.n;
    QueryRows<QL, 16> rows;
    rows.request(a, b, kvh, 0);
    const Seq s = sequence(a, b, place.len);
    int lo_least, lo_most;
    row_limits(a, s, b, 0, 16, lo_least, lo_most);
    const auto tiles = tiles_of<kTileTokens>(s, lo_least);
    const int last16 = (s.len - 1) & ~15;
    Chunk<P, N16> k_next[2], v_next[2];
    // (without a branch: a load whose result meets another value behind it would be waited for there.  Tokens behind the last one and
    // tiles behind the last one stand for something that is read anyway.)
    const ChunkAt whole = chunk_at<P, N16>(a, l16, group);
    auto request = [&](int v) {
        const int t0 = tiles.at(v) * kTileTokens + wave * kWaveTokens;
        ChunkAt at[2] = {whole, whole};
        if (t0 + kWaveTokens > s.len) {
#pragma unroll
            for (int st = 0; st < 2; ++st) at[st] = chunk_at<P, N16>(a, min(t0 + 16 * st + l16, s.len - 1) - min(t0 + 16 * st, last16), group);
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const int64_t row = stage_row(a, b, kvh, min(t0 + 16 * st, last16));
            load_chunk<P, N16>(a, a.k_mant, a.k_exp, row, at[st], k_next[st]);
            load_chunk<P, N16>(a, a.v_mant, a.v_exp, row, at[st], v_next[st]);
        }
    };
    const bool some = place.split < tiles.count;             // (else there may be no token at all)
    if (some) request(place.split);
    if (tid < 64) depth_s[tid] = tid < a.n_tok ? node_depth(node_mask(a, b, tid), tid) : 0;
    rows.put(a, 0, (float*)smem, perm_s);
    if (tid < RP) rule_s[tid] = row_rule(a, s, b, kvh, tid);
    const int row = l16 & (RP - 1), mine = RP == 8 ? 16 * (l16 >> 3) : 0;      // its row; where its tokens begin
    const uint32_t second = l16 & 8 ? ~0u : 0u;
    lds_only_barrier();                                      // (the first rows are on their way)
    bf16x8 q[1][QL][4];
    query_operand<P, QL>((const float*)smem, perm_s, row, group, q[0]);
    lds_only_barrier();                                      // the queries give way to the values

    uint8_t* const v_s = smem + wave * kWaveLds;
    f32x4 o[1][8];
    Running x[1];
    bool large = false;
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) o[0][ct] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float mul = a.score_mul * (float)(1 << Decode<P>::kShift);
    for (int v = place.split; v < tiles.count; v += n_splits) {
        const int t0 = tiles.at(v) * kTileTokens + wave * kWaveTokens;
        if (t0 >= s.len) break;                              // the wavefront's part of the last tile is empty
        Chunk<P, N16> kc[2], vc[2];
#pragma unroll
        for (int st = 0; st < 2; ++st) { kc[st] = k_next[st]; vc[st] = v_next[st]; }
        request(v + n_splits < tiles.count ? v + n_splits : v);
        float y[1][8];
        products<QL, 1>([&](int st, int j) { return __builtin_bit_cast(bf16x8, eight<P, N16>(kc[st], j)); }, q, y);
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *(u32x4*)(v_s + value_at(16 * st + l16, 2 * group + (j >> 1), j & 1)) = eight<P, N16>(vc[st], j);
        if (__builtin_amdgcn_ballot_w64(has_large(vc[0]) || has_large(vc[1]))) large = true;
        wave_fence();
        constexpr int N = RP / 2;
        float z[N];
#pragma unroll
        for (int i = 0; i < N; ++i)                          // (by bits: a choice between elements of an array would go through memory)
            z[i] = RP == 16 ? y[0][i] : __uint_as_float((__float_as_uint(y[0][i & 3]) & ~second) | (__float_as_uint(y[0][4 + (i & 3)]) & second));
        const float factor = rule_scores<N>(a, s, rule_s + row, depth_s, t0 >= lo_most && t0 + kWaveTokens <= s.base,
                                                     t0 + mine + 4 * group, mul, z);
        const float base = follow<N>(z, factor, large, x[0], o[0]);
        uint32_t w[PL][N / 2];
        probabilities<PL, N>(z, factor, base, x[0].sum, w);
        bf16x8 p[1][PL];
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            u32x4 v;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = RP == 16 || ((l16 & 8) != 0) == (k >= 2) ? w[i][k & (N / 2 - 1)] : 0u;
            p[0][i] = __builtin_bit_cast(bf16x8, v);
        }
        add_values<PL, 1>([&](int ct) { return values_of(v_s, lane, ct); }, p, o);
        if (large) x[0].keep_room(o[0]);
        wave_fence();
    }
    __syncthreads();
    finish<P, QL, 1, RP>(a, b, kvh, 0, blockIdx.x, smem, ml_s, wave, lane, o[0], x[0], large);
}

// More rows: a workgroup decodes 64 tokens at a time to bf16 in LDS, once for all its rows.  RW wavefronts have HC times 16 rows each
// (the rows of a workgroup: 16 * RW * HC) and the 4 / RW that have the same ones share the tokens of a tile out.  While one half of
// the LDS is multiplied with, the next tile is decoded into the other and the one after it is requested: one barrier a tile.
// grid = (n_splits * B, H_kv * row_tiles).
template <int P, bool N16, int QL, int HC, int RW>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void scored_split_wide(Args a) {
    constexpr int PL = QL == 3 ? 3 : 2;
    constexpr int KS = RW / 2;                               // steps of 32 tokens per wavefront and tile
    constexpr int kPlane = kWideTokens * 256, kTile = 2 * kPlane;      // keys, values
    __shared__ __align__(16) uint8_t smem[2 * kTile];
    __shared__ float ml_s[4][16][2];
    __shared__ int perm_s[kD];
    __shared__ int depth_s[64];
    __shared__ RowRule rule_s[16 * RW * HC];
    __shared__ int large_s[2];                               // a value byte above kOrdinary was decoded into this half
    static_assert(16 * RW * kQStride * 4 <= 2 * kTile && 4 * kWaveLds <= 2 * kTile, "the query rows and the sums fit");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, group = lane >> 4;
    const Place place = place_at(a, blockIdx.x);
    if (place.split < 0) return;
    const int b = place.b, n_splits = place.n;
    const int kvh = blockIdx.y / a.row_tiles, r0 = (blockIdx.y % a.row_tiles) * (16 * HC * RW);
    const int rw = wave % RW, part = wave / RW;              // its rows; its part of a tile's tokens
    QueryRows<QL, 16 * RW> rows[HC];
#pragma unroll
    for (int c = 0; c < HC; ++c) rows[c].request(a, b, kvh, r0 + 16 * RW * c);
    const Seq s = sequence(a, b, place.len);
    int lo_least, lo_most;
    row_limits(a, s, b, r0, 16 * RW * HC, lo_least, lo_most);
    const auto tiles = tiles_of<kWideTokens>(s, lo_least);
    const int last16 = (s.len - 1) & ~15;
    // a thread decodes 32 channels of one token, keys and values: wavefront w tokens 16 w ..
    const ChunkAt whole = chunk_at<P, N16>(a, l16, group);
    Chunk<P, N16> k_raw, v_raw;
    auto request = [&](int v) {                              // (without a branch, as in scored_split)
        const int t0 = tiles.at(v) * kWideTokens + 16 * wave, from = min(t0, last16);
        ChunkAt at = whole;
        if (t0 + 16 > s.len) at = chunk_at<P, N16>(a, min(t0 + l16, s.len - 1) - from, group);
        const int64_t row = stage_row(a, b, kvh, from);
        load_chunk<P, N16>(a, a.k_mant, a.k_exp, row, at, k_raw);
        load_chunk<P, N16>(a, a.v_mant, a.v_exp, row, at, v_raw);
    };
    if (place.split < tiles.count) request(place.split);
    if (tid < 64) depth_s[tid] = tid < a.n_tok ? node_depth(node_mask(a, b, tid), tid) : 0;
    if (tid < 2) large_s[tid] = 0;
    for (int i = tid; i < 16 * RW * HC; i += kThreads) rule_s[i] = row_rule(a, s, b, kvh, r0 + i);
    bf16x8 q[HC][QL][4];
#pragma unroll 1
    for (int c = 0;; ++c) {
        rows[0].put(a, r0 + 16 * RW * c, (float*)smem, perm_s);
        lds_only_barrier();                                  // (the first rows are on their way)
        query_operand<P, QL>((const float*)smem, perm_s, 16 * rw + l16, group, q[HC - 1]);
        if (c == HC - 1) break;
#pragma unroll
        for (int i = 0; i < QL; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) q[0][i][j] = q[HC - 1][i][j];
        rows[0] = rows[HC - 1];
        lds_only_barrier();
    }
    lds_only_barrier();                                      // the queries give way to keys and values

    f32x4 o[HC][8];
    Running x[HC];
#pragma unroll
    for (int c = 0; c < HC; ++c)
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) o[c][ct] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float mul = a.score_mul * (float)(1 << Decode<P>::kShift);
    auto key_at = [](int row, int piece) { return row * 256 + ((piece ^ (row & 15)) * 16); };
    auto decode = [&](int half) {
        uint8_t* const tile = smem + half * kTile;
        const int row = 16 * wave + l16;
#pragma unroll
        for (int j = 0; j < 4; ++j) *(u32x4*)(tile + key_at(row, 4 * group + j)) = eight<P, N16>(k_raw, j);
#pragma unroll
        for (int j = 0; j < 4; ++j) *(u32x4*)(tile + kPlane + value_at(row, 2 * group + (j >> 1), j & 1)) = eight<P, N16>(v_raw, j);
        if (__builtin_amdgcn_ballot_w64(has_large(v_raw)) && lane == 0) large_s[half] = 1;
    };
    const auto after = [&](int v) { return v + n_splits < tiles.count ? v + n_splits : v; };
    if (place.split < tiles.count) {
        decode(0);
        request(after(place.split));
    }
    int half = 0;
    bool large = false;
    for (int v = place.split; v < tiles.count; v += n_splits, half ^= 1) {
        lds_only_barrier();                                  // this tile is complete; the one before it is not looked at any more
        const uint8_t* const tile = smem + half * kTile;
        if (v + n_splits < tiles.count) decode(half ^ 1);
        request(after(after(v)));
        if (__builtin_amdgcn_readfirstlane(large_s[half])) large = true;
        // 32 tokens at a time, not unrolled: the registers of two steps together do not fit.  With 16 rows a wavefront the values and the
        // next keys are read ahead of the softmax, whose instructions then fill the time of the reads.
        bf16x8 k[2][4];
        auto read_keys = [&](int row) {
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int j = 0; j < 4; ++j) k[st][j] = *(const bf16x8*)(tile + key_at(row + 16 * st + l16, 4 * group + j));
        };
        if (HC == 1) read_keys(32 * KS * part);
#pragma unroll 1
        for (int ks = 0; ks < KS; ++ks) {
            const int row = 32 * (KS * part + ks), t0 = tiles.at(v) * kWideTokens + row;
            const uint8_t* const v_s = tile + kPlane + row * 256;
            float y[HC][8];
            Values by_channel;
            if (HC == 1) {
                products<QL, HC>([&](int st, int j) { return k[st][j]; }, q, y);
#pragma unroll
                for (int ct = 0; ct < 8; ++ct) by_channel.v[ct] = values_of(v_s, lane, ct);
                if (ks + 1 < KS) read_keys(row + 32);
                __builtin_amdgcn_sched_barrier(0);
            } else {
                products<QL, HC>([&](int st, int j) { return *(const bf16x8*)(tile + key_at(row + 16 * st + l16, 4 * group + j)); }, q, y);
            }
            __builtin_amdgcn_s_setprio(0);
            const bool inner = t0 >= lo_most && t0 + 32 <= s.base;
            bf16x8 p[HC][PL];
#pragma unroll
            for (int c = 0; c < HC; ++c) {
                uint32_t w[PL][4];
                const float factor = rule_scores<8>(a, s, rule_s + 16 * (RW * c + rw) + l16, depth_s, inner, t0 + 4 * group, mul, y[c]);
                const float base = follow<8>(y[c], factor, large, x[c], o[c]);
                probabilities<PL, 8>(y[c], factor, base, x[c].sum, w);
#pragma unroll
                for (int i = 0; i < PL; ++i) p[c][i] = __builtin_bit_cast(bf16x8, u32x4{w[i][0], w[i][1], w[i][2], w[i][3]});
            }
            __builtin_amdgcn_s_setprio(1);
            if (HC == 1) add_values<PL, HC>([&](int ct) { return by_channel.v[ct]; }, p, o);
            else add_values<PL, HC>([&](int ct) { return values_of(v_s, lane, ct); }, p, o);
            if (large) {
#pragma unroll
                for (int c = 0; c < HC; ++c) x[c].keep_room(o[c]);
            }
        }
    }
#pragma unroll 1
    for (int c = 0;; ++c) {                                  // (a loop: code that runs once is as long as its way from memory)
        const int rc = r0 + 16 * RW * c;
        if (RW == 4 && a.n_splits > 1) {                     // nothing to join
            store_partial(a, kvh, rc + 16 * wave, blockIdx.x, lane, o[0], x[0], large);
        } else {
            __syncthreads();
            finish<P, QL, RW, 16>(a, b, kvh, rc, blockIdx.x, smem, ml_s, wave, lane, o[0], x[0], large);
        }
        if (c == HC - 1 || rc + 16 * RW >= a.M) break;
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) o[0][ct] = o[HC - 1][ct];
        x[0] = x[HC - 1];
    }
}

// Joins the splits, two channels a lane, sixteen partial results in flight: four wavefronts for a row, which take every fourth split (FOUR),
// or one for four rows of a kv-head, four splits of each at a time.
template <int P, int QL, bool FOUR>
__global__ __launch_bounds__(kThreads) void scored_combine(Args a) {
    __shared__ float join_s[4][64][4];
    constexpr int kRows = FOUR ? 1 : 4, kFly = 16 / kRows, kStep = FOUR ? 4 : 1;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles = (a.M + kRows - 1) / kRows;               // of rows, per kv-head
    const int64_t tile = FOUR ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
    if (tile >= (int64_t)a.batch * a.H_kv * tiles) return;     // (uniform for the workgroup where it has a barrier)
    const int unit = (int)(tile / tiles), r0 = (int)(tile - (int64_t)unit * tiles) * kRows, b = unit / a.H_kv, kvh = unit - b * a.H_kv;
    const Place place = places_of(a, b);
    int c0 = position_channel<P>(2 * lane), c1 = position_channel<P>(2 * lane + 1);
    if (a.perm_v) {
        c0 = a.perm_v[kvh * kD + c0] & (kD - 1);
        c1 = a.perm_v[kvh * kD + c1] & (kD - 1);
    }
    float top[kRows], den[kRows];
    float2 acc[kRows];
    int64_t first[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        top[k] = -INFINITY;
        den[k] = acc[k].x = acc[k].y = 0.f;
        first[k] = ((int64_t)kvh * a.M + min(r0 + k, a.M - 1)) * a.n_splits * a.batch + place.first;
    }
    const int part = FOUR ? wave : 0;
    for (int i0 = part; i0 < place.n; i0 += kFly * kStep) {
        float2 v[kRows][kFly], ml[kRows];
        const int mine = i0 + (lane & (kFly - 1)) * kStep;
#pragma unroll
        for (int k = 0; k < kRows; ++k) ml[k] = *(const float2*)(a.part_ml + 2 * (first[k] + min(mine, place.n - 1)));
#pragma unroll
        for (int k = 0; k < kRows; ++k)
#pragma unroll
            for (int i = 0; i < kFly; ++i)
                if (i == 0 || i0 + i * kStep < place.n) v[k][i] = *(const float2*)(a.part_o + (first[k] + i0 + i * kStep) * kD + 2 * lane);
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            if (mine >= place.n) ml[k].x = -INFINITY;
            const float now = fmaxf(top[k], row_max(ml[k].x));
            const float ref = now > -INFINITY ? now : 0.f;
            const float w = exp2_raw(ml[k].x - ref), was = exp2_raw(top[k] - ref);       // 0 for a split that saw nothing
            top[k] = now;
            acc[k].x *= was;
            acc[k].y *= was;
            den[k] *= was;
#pragma unroll
            for (int i = 0; i < kFly; ++i) {
                if (i > 0 && i0 + i * kStep >= place.n) break;                           // (not by a weight of 0)
                const float wi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), i));
                acc[k].x = fmaf(wi, v[k][i].x, acc[k].x);
                acc[k].y = fmaf(wi, v[k][i].y, acc[k].y);
                den[k] = fmaf(wi, __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ml[k].y), i)), den[k]);
            }
        }
    }
    if (FOUR) {
        *(f32x4*)join_s[wave][lane] = f32x4{top[0], den[0], acc[0].x, acc[0].y};
        __syncthreads();
        if (part) return;
        float all = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) all = fmaxf(all, join_s[w][lane][0]);
        const float ref = all > -INFINITY ? all : 0.f;
        top[0] = all;
        den[0] = acc[0].x = acc[0].y = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const f32x4 x = *(const f32x4*)join_s[w][lane];
            const float f = exp2_raw(x[0] - ref);
            den[0] = fmaf(f, x[1], den[0]);
            acc[0].x = fmaf(f, x[2], acc[0].x);
            acc[0].y = fmaf(f, x[3], acc[0].y);
        }
    }
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        if (r0 + k >= a.M) break;
        const float by = den[k] > 0.f ? (float)(1 << Decode<P>::kShift) / den[k] : 0.f;
        const int64_t at = out_row(a, b, kvh, r0 + k);
        store_out<QL>(a, at * kD + c0, acc[k].x * by);
        store_out<QL>(a, at * kD + c1, acc[k].y * by);
        if (lane == 0 && a.lse) a.lse[at] = natural_lse(top[k], den[k]);
    }
}

// Rows of a workgroup: 16 in scored_split (rw = 1), 16 * rw * hc in scored_split_wide.  More of them decode a tile for more rows, fewer take less
// time for a tile: 64 rows instead of 32 from kFourFrom tiles on (8 x 64 rows of 300 and 1000 tokens 11.8 and 12.1 us with 64 rows, 10.4 and 11.3
// with 32; 48 x 60 rows of 3000 30.2 and 31.6), 128 (with bf16 I/O, which has the registers for it) from kTwoFrom on (32 x 256 rows of 3000
// and 24000 tokens 52.7 and 212 us with 128 rows, 44.4 and 219 with 64).
// Splits: as many as make one resident round of workgroups (three a compute unit in scored_split, two in scored_split_wide) and no more
// than there are tiles; none where the partial results and the second kernel would take longer than a few more tiles (32 x 256
// rows of 200 and 400 tokens 19.3 and 21.9 us in two splits, 13.0 and 16.7 in one; 8 x 4 rows of 400 8.6 in four, 10.6 in one).
constexpr int64_t kFourFrom = 1024, kTwoFrom = 8192;
struct Plan { int32_t hc, rw, row_tiles, n_splits; };

template <int P, bool N16, int QL>
void launch_split(const Args& a, const Plan& p, hipStream_t s) {
    const dim3 grid((unsigned)(a.n_splits * a.batch), (unsigned)(a.H_kv * a.row_tiles));
    constexpr int kTwo = QL == 1 ? 2 : 1;                    // fp16 and fp32 have no registers for two, and are not planned with them
    if (a.M <= 8) scored_split<P, N16, QL, 8><<<grid, kThreads, 0, s>>>(a);
    else if (p.rw == 1) scored_split<P, N16, QL, 16><<<grid, kThreads, 0, s>>>(a);
    else if (p.rw == 2) scored_split_wide<P, N16, QL, 1, 2><<<grid, kThreads, 0, s>>>(a);
    else if (p.hc == 1) scored_split_wide<P, N16, QL, 1, 4><<<grid, kThreads, 0, s>>>(a);
    else scored_split_wide<P, N16, QL, kTwo, 4><<<grid, kThreads, 0, s>>>(a);
}
template <int P>
void launch_split(const Args& a, int dt, const Plan& p, hipStream_t s) {
    const bool n16 = a.log2_block == 4;
    if (dt == KVBFP_F32 && n16) launch_split<P, true, 3>(a, p, s);
    else if (dt == KVBFP_F32) launch_split<P, false, 3>(a, p, s);
    else if (dt == KVBFP_F16 && n16) launch_split<P, true, 2>(a, p, s);
    else if (dt == KVBFP_F16) launch_split<P, false, 2>(a, p, s);
    else if (n16) launch_split<P, true, 1>(a, p, s);
    else launch_split<P, false, 1>(a, p, s);
}

// Few rows: four wavefronts for each, which share its splits (32 rows in 6 splits and an fp32 tree of 22 rows a kv-head: 8.7 and 11.6 us, with one
// for four rows 10.9 and 19.9); many: one for four rows, the same work with fewer wavefronts (16384 rows in four splits 150.3 us in all, with
// four for each 152).
template <int P, int QL>
void launch_combine(const Args& a, hipStream_t s) {
    const int64_t rows = (int64_t)a.batch * a.H_kv * a.M;
    const int64_t tiles = (int64_t)a.batch * a.H_kv * ((a.M + 3) / 4);
    if (rows <= 2048) scored_combine<P, QL, true><<<dim3((unsigned)rows), kThreads, 0, s>>>(a);
    else scored_combine<P, QL, false><<<dim3((unsigned)((tiles + 3) / 4)), kThreads, 0, s>>>(a);
}
template <int P>
void launch_combine(const Args& a, int dt, hipStream_t s) {
    if (dt == KVBFP_F32) launch_combine<P, 3>(a, s);
    else if (dt == KVBFP_F16) launch_combine<P, 2>(a, s);
    else launch_combine<P, 1>(a, s);
}

Plan plan(const kvbfp_layout* L, int64_t rows, int64_t max_len, int dtype, bool shares) {
    const int64_t units = (int64_t)L->batch * L->n_kv_heads, tiles = (max_len + kWideTokens - 1) / kWideTokens;
    const auto parts = [&](int64_t of_wg) { return units * ((rows + of_wg - 1) / of_wg); };
    Plan p;
    p.rw = rows <= 16 ? 1 : rows <= 32 || parts(64) * tiles < kFourFrom ? 2 : 4;
    p.hc = rows > 64 && dtype == KVBFP_BF16 && parts(128) * tiles >= kTwoFrom ? 2 : 1;
    const int64_t of_wg = 16 * p.hc * p.rw, steps = p.rw == 1 ? (max_len + kTileTokens - 1) / kTileTokens : tiles;
    p.row_tiles = (int32_t)((rows + of_wg - 1) / of_wg);
    const bool one = steps <= 2 + std::min<int64_t>(units * rows / 1024, 8);
    p.n_splits = one ? 1 : (int32_t)std::max<int64_t>(1, std::min<int64_t>(steps, round_of(p.rw == 1 ? 768 : 512, parts(of_wg), shares)));
    return p;
}
// The most splits that a call takes, whatever its type and lengths: the workspace has room for them.
int32_t splits_of(const kvbfp_layout* L, int64_t rows, int64_t max_len) {
    int32_t most = 1;
    for (int dtype : {KVBFP_BF16, KVBFP_F16})
        for (bool shares : {false, true}) most = std::max(most, plan(L, rows, max_len, dtype, shares).n_splits);
    return most;
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
    if (!std::isfinite(a->score_mul * 128.f))                // (times the scale of the decoded codes)
        return fail(KVBFP_ERR_INVALID_ARG, "%s: softmax_scale = %g", call, (double)softmax_scale);
    if (paging) {
        a->block_table = paging->block_table; a->table_stride = paging->table_stride; a->n_pages = L->batch;
        while (((int64_t)1 << a->log2_page) < L->max_seq) ++a->log2_page;
    }
    if (rule) {
        if (rule->cap > 0.f) {
            a->cap = rule->cap * kLog2e;
            a->inv_cap = 1.f / a->cap;
            // (what scores are multiplied with on their way into the exponential, with the scale of the decoded codes)
            const float turn = a->inv_cap * 2.8853900817779268f * std::max(1.f, std::fabs(a->score_mul) * 128.f);
            if (!std::isfinite(a->cap) || !std::isfinite(turn)) return fail(KVBFP_ERR_INVALID_ARG, "%s: rule.cap = %g", call, (double)rule->cap);
        }
        a->slopes = rule->slopes; a->first = rule->first_dev; a->prefix = rule->prefix_dev;
        a->tree = rule->tree_mask; a->tree_stride = rule->tree_stride;
        a->window = (int64_t)rule->window < max_len + 64 ? rule->window : 0;      // a window beyond every distance is none
    }
    return KVBFP_OK;
}

int check_arrays(const char* call, const kvbfp_layout* L, const Args& a, size_t element, std::initializer_list<Span> written) {
    size_t m, e;
    if (int rc = kvbfp_cache_bytes(L, &m, &e)) return rc;
    const size_t batch = (size_t)a.batch, rows = batch * (size_t)a.n_tok * (size_t)a.H_q, perm = (size_t)a.H_kv * kD * sizeof(int32_t);
    return check_spans(call, written,
                       {{"k_mant", a.k_mant, m}, {"k_exp", a.k_exp, e}, {"v_mant", a.v_mant, m}, {"v_exp", a.v_exp, e},
                        {"q", a.q == a.out ? nullptr : a.q, rows * kD * element, element},
                        {"lse", a.lse_in, rows * sizeof(float), sizeof(float)},
                        {"weights_in", a.w_in == a.w_out ? nullptr : a.w_in, batch * (size_t)a.H_kv * (size_t)a.w_stride * sizeof(float), sizeof(float)},
                        {"seq_len_dev", a.seq_len, batch * sizeof(int32_t), sizeof(int32_t)},
                        {"perm_k", a.perm_k, perm, sizeof(int32_t)}, {"perm_v", a.perm_v, perm, sizeof(int32_t)},
                        {"block_table", a.block_table, batch * (size_t)a.table_stride * sizeof(int32_t), sizeof(int32_t)},
                        {"rule.slopes", a.slopes, (size_t)a.H_q * sizeof(float), sizeof(float)},
                        {"rule.first_dev", a.first, batch * (size_t)a.n_tok * sizeof(int32_t), sizeof(int32_t)},
                        {"rule.prefix_dev", a.prefix, batch * sizeof(int32_t), sizeof(int32_t)},
                        {"rule.tree_mask", a.tree, ((batch - 1) * (size_t)a.tree_stride + (size_t)a.n_tok) * sizeof(uint64_t), sizeof(uint64_t)}});
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
    const bool shares = seq_len_dev && a.batch > 1 && a.batch <= 64;
    const Plan p = plan(&logical, a.M, max_len, (int)dtype, shares);
    if ((int64_t)a.H_kv * p.row_tiles > 65535) return fail(KVBFP_ERR_UNSUPPORTED, "%s: too many heads for the grid", call);
    const size_t need = partial_bytes(&logical, a.M, p.n_splits);
    if (need && (!workspace || workspace_bytes < need))
        return fail(KVBFP_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", call, need, workspace ? workspace_bytes : (size_t)0);
    if (need && (uintptr_t)workspace % 256 != 0) return fail(KVBFP_ERR_WORKSPACE, "%s: workspace must be 256-byte aligned", call);
    a.out = out; a.lse = lse; a.perm_k = perm_k; a.perm_v = perm_v;
    a.n_splits = p.n_splits; a.row_tiles = p.row_tiles;
    a.share = shares && p.n_splits > 1;
    if (need) {
        a.part_o = (float*)workspace;
        a.part_ml = a.part_o + (size_t)a.batch * a.H_kv * a.M * a.n_splits * kD;
    }
    const size_t rows = (size_t)a.batch * (size_t)a.n_tok * (size_t)a.H_q, element = (size_t)dtype_size(dtype);
    if (int rc = check_arrays(call, L, a, element, {{"out", out, rows * kD * element, element}, {"lse", lse, rows * sizeof(float), sizeof(float)},
                                                    {"workspace", need ? workspace : nullptr, need}}))
        return rc;
    hipStream_t s = (hipStream_t)hip_stream;
    if (logical.mant_bits == 4) launch_split<4>(a, (int)dtype, p, s);
    else launch_split<8>(a, (int)dtype, p, s);
    hipError_t err = hipGetLastError();
    if (err == hipSuccess && a.n_splits > 1) {
        if (logical.mant_bits == 4) launch_combine<4>(a, (int)dtype, s);
        else launch_combine<8>(a, (int)dtype, s);
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
    return std::max<size_t>(partial_bytes(L, rows, splits_of(L, rows, max_len)), 256);
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
