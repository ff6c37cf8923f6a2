// Eviction of cached tokens by the weight they have collected (kvbfp_evict and its paged form): per sequence and kv-head the first n_first
// tokens, the last n_recent and those with the largest weights between them stay, n_keep in all, and go in their order to another cache.
//
// Selection (evict_select), a workgroup of 16 wavefronts per sequence and kv-head, each with a stretch of the tokens, up to 2048 of
// it in LDS: the weight of the last one that stays is found by its bits, eleven at a time from the top (a histogram in LDS of
// those that agree in the bits so far; the search ends as soon as all that agree stay), ties go to the lowest index, and what stays is
// written in order by counts of the wavefronts' ballots.  64 x 32768 weights take 21 us: 48 vector instructions a weight over the passes,
// 11 us on the 64 compute units that have a workgroup, the rest their barriers.  (Thirty-two loads a lane in flight instead of
// sixteen change nothing.)
// Rows (evict_rows): 16 bytes a thread and plane, four rows in flight, stores past the cache.  Bound by memory: 64 x 8192 of 32768 rows of 64
// bytes in 42 us; of the 128-byte lines that are fetched every second half is a row that goes (137 MB for 71), and with the 72 MB that are
// written this is the rate of a plain copy, 5.0 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "decode_dev.h"
#include "kvbfp_internal.h"

namespace {

using kvbfp::dev::kD;
using kvbfp::dev::wave_scan;

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;

struct EvictArgs {
    const uint8_t* src[4];               // k_mant, k_exp, v_mant, v_exp
    uint8_t* dst[4];
    const int32_t* src_table;
    const int32_t* dst_table;
    int64_t src_stride, dst_stride, src_seq, dst_seq;      // tables; tokens of a region
    int32_t src_log2_page, dst_log2_page, src_pages, dst_pages;
    const float* weights;                // [B][H][w_stride]
    int64_t w_stride;
    const int32_t* seq_len;
    int32_t max_len, H, batch, n_keep, n_first, n_recent;
    int32_t* kept;                       // [B][H][n_keep]
    int32_t* new_len;                    // [B]
    float* w_out;                        // [B][H][n_keep] or nullptr
    int32_t n_exps;                      // of a row
    int32_t held;                        // keys of a lane that have room in LDS
};

__device__ __forceinline__ int length_of(const EvictArgs& a, int b) {
    return a.seq_len ? min(max(a.seq_len[b], 0), a.max_len) : a.max_len;
}

// Weights in the order of unsigned integers: NaN lowest, both zeros alike; tokens that stay anyway above all others, and what lies behind
// the last token like NaN (its index is larger than theirs, and there are enough others).
__device__ __forceinline__ uint32_t key_of(float w, int t, int lo, int hi, int len) {
    const uint32_t u = __float_as_uint(w + 0.f);
    const uint32_t k = w != w ? 0u : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return (uint32_t)(t - lo) < (uint32_t)(hi - lo) ? k : t < len ? ~0u : 0u;
}
// COUNT weights 64 apart, from w[t] on; those behind the last token are the last one's.
template <int COUNT>
__device__ __forceinline__ void load_weights(const float* w, int t0, int lane, int len, float (&x)[COUNT]) {
    if (t0 + 64 * COUNT <= len) {                          // (uniform: the addresses then differ by constants)
        const float* const at = w + t0 + lane;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) x[i] = at[64 * i];
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) x[i] = w[min(t0 + 64 * i + lane, len - 1)];
    }
}
__device__ __forceinline__ int bits_below(uint64_t m, int base) {          // base + bits of m below this lane's
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, (uint32_t)base));
}

constexpr int kHeld = 32;                                  // keys of a lane in LDS
constexpr int kBins = 2048;

// f(i, key) for the tokens from + 64 i + lane of a wavefront's stretch, i < n (a multiple of 8), in order: the first keys are in LDS (held:
// this wavefront's, 64 times kHeld at most), others are read again, eight in flight.
template <class F>
__device__ __forceinline__ void each_key(const uint32_t* held, int n, const float* w, int from, int lo, int hi, int len, F&& f) {
    const int lane = threadIdx.x & 63;
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += 8) {
        uint32_t k[8];
        if (i0 < kHeld) {
#pragma unroll
            for (int i = 0; i < 8; ++i) k[i] = held[64 * (i0 + i) + lane];
        } else {
            float x[8];
            load_weights<8>(w, from + 64 * i0, lane, len, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) k[i] = key_of(x[i], from + 64 * (i0 + i) + lane, lo, hi, len);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) f(i0 + i, k[i]);
    }
}

// grid = (H, B)
__global__ __launch_bounds__(kThreads) void evict_select(EvictArgs a) {
    extern __shared__ uint32_t held_s[];                   // [wavefronts][a.held][64]
    __shared__ int hist_s[2 * kBins];                      // even and odd lanes: fewer of them meet in one bin
    __shared__ int wave_s[kWaves][2];
    __shared__ int found_s[3];                             // digit, how many are above it, how many it has
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = blockIdx.x, b = blockIdx.y;
    const int len = length_of(a, b), unit = b * a.H + h;
    const int count = min(len, a.n_keep);
    int32_t* const kept = a.kept + (int64_t)unit * a.n_keep;
    if (h == 0 && tid == 0) a.new_len[b] = count;
    for (int i = count + tid; i < a.n_keep; i += kThreads) kept[i] = -1;
    if (len <= a.n_keep) {
        for (int i = tid; i < len; i += kThreads) kept[i] = i;
        return;
    }
    const float* const w = a.weights + (int64_t)unit * a.w_stride;
    const int lo = a.n_first, hi = len - a.n_recent;       // the others stay anyway
    int need = a.n_keep;                                   // of those that agree with `bits` where it is known
    uint32_t bits = 0, known = 0;                          // of the smallest key that stays
    const int stretch = ((len + kWaves - 1) / kWaves + 511) & ~511;        // (whole groups of eight keys a lane)
    const int from = min(wave * stretch, len), to = min(from + stretch, len), n = ((to - from + 511) & ~511) / 64;
    uint32_t* const held = held_s + wave * (64 * a.held);
    int* const hist = hist_s + (lane & 1) * kBins;
    for (int shift = 21; shift >= 0; shift = shift == 10 ? 0 : shift - 11) {         // 11, 11 and 10 bits
        const uint32_t digits = shift == 0 ? 1023u : 2047u;
        for (int i = tid; i < 2 * kBins; i += kThreads) hist_s[i] = 0;
        __syncthreads();
        if (shift == 21) {                                 // the first time: from memory, and all agree
            float x[8], next[8];
            load_weights<8>(w, from, lane, len, x);
#pragma unroll 1
            for (int i0 = 0; i0 < n; i0 += 8) {
                load_weights<8>(w, from + 64 * min(i0 + 8, n - 8), lane, len, next);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t k = key_of(x[i], from + 64 * (i0 + i) + lane, lo, hi, len);
                    if (i0 < kHeld) held[64 * (i0 + i) + lane] = k;
                    atomicAdd(&hist[k >> 21], 1);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = next[i];
            }
        } else {
            each_key(held, n, w, from, lo, hi, len, [&](int, uint32_t k) {
                if ((k & known) == bits) atomicAdd(&hist[(k >> shift) & digits], 1);
            });
        }
        __syncthreads();
        // the digit in which the need-th largest lies: thread i has the bins 2047 - 2 i and 2046 - 2 i, sums from the top
        int2 mine = *(const int2*)(hist_s + kBins - 2 - 2 * tid);
        const int2 odd = *(const int2*)(hist_s + 2 * kBins - 2 - 2 * tid);
        mine.x += odd.x;
        mine.y += odd.y;
        const int total = mine.x + mine.y;
        int before = wave_scan(total);
        if (lane == 63) wave_s[wave][0] = before;
        __syncthreads();
        before -= total;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) before += i < wave ? wave_s[i][0] : 0;
        if (before < need && need <= before + mine.y) {
            found_s[0] = kBins - 1 - 2 * tid;
            found_s[1] = before;
            found_s[2] = mine.y;
        } else if (before + mine.y < need && need <= before + total) {
            found_s[0] = kBins - 2 - 2 * tid;
            found_s[1] = before + mine.y;
            found_s[2] = mine.x;
        }
        __syncthreads();
        bits |= (uint32_t)found_s[0] << shift;
        known |= digits << shift;
        need -= found_s[1];
        if (need == found_s[2] || shift == 0) break;   // all that agree stay, or there is nothing left to tell them apart
    }
    // in order: what every wavefront keeps and how many ties it has, then where they go
    int n_more = 0, n_tie = 0;
    each_key(held, n, w, from, lo, hi, len, [&](int, uint32_t k) {
        n_more += __popcll(__ballot((k & known) > bits));
        n_tie += __popcll(__ballot((k & known) == bits));
    });
    __syncthreads();                                       // (nobody looks at the sums of the last digit any more)
    if (lane == 0) {
        wave_s[wave][0] = n_more;
        wave_s[wave][1] = n_tie;
    }
    __syncthreads();
    int at = 0, ties = 0;                                  // places taken, ties seen before this stretch
    for (int i = 0; i < wave; ++i) {
        at += wave_s[i][0];
        ties += wave_s[i][1];
    }
    at += min(ties, need);
    each_key(held, n, w, from, lo, hi, len, [&](int i, uint32_t k) {
        bool stays = (k & known) > bits;
        const uint64_t all_ties = __ballot((k & known) == bits);
        if (all_ties) {                                    // (uniform, and rare)
            stays = stays || (((all_ties >> lane) & 1) && bits_below(all_ties, ties) < need);
            ties += __popcll(all_ties);
        }
        const uint64_t all = __ballot(stays);
        const int place = bits_below(all, at);
        if (stays && place < a.n_keep) kept[place] = from + 64 * i + lane;
        at += __popcll(all);
    });
}

__device__ __forceinline__ int64_t row_of(const int32_t* table, int64_t stride, int log2_page, int pages, int64_t seq, int H, int b, int h, int t) {
    if (!table) return ((int64_t)b * H + h) * seq + t;
    const int page = min(max(table[(int64_t)b * stride + (t >> log2_page)], 0), pages - 1);
    return (((int64_t)page * H + h) << log2_page) + (t & ((1 << log2_page) - 1));
}

// PER threads have 16 bytes each of the key and of the value row of four kept tokens.  grid = (rows / (1024 / PER), H, B)
template <int PER>
__global__ __launch_bounds__(256) void evict_rows(EvictArgs a) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    constexpr int kRows = 4, kGroup = 256 / PER;
    const int part = threadIdx.x % PER, i0 = blockIdx.x * (kRows * kGroup) + threadIdx.x / PER;
    const int h = blockIdx.y, b = blockIdx.z;
    const int count = min(length_of(a, b), a.n_keep);
    const int64_t unit = (int64_t)b * a.H + h;
    int t[kRows];
    int64_t from[kRows], to[kRows];
    u32x4 k[kRows], v[kRows];
    uint8_t ke[kRows], ve[kRows];
    float w[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) t[r] = a.kept[unit * a.n_keep + min(i0 + r * kGroup, max(count - 1, 0))];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int i = i0 + r * kGroup;
        if (i >= count) continue;                          // (what lies behind the last kept token stays as it was)
        t[r] = min(max(t[r], 0), a.max_len - 1);
        from[r] = row_of(a.src_table, a.src_stride, a.src_log2_page, a.src_pages, a.src_seq, a.H, b, h, t[r]);
        to[r] = row_of(a.dst_table, a.dst_stride, a.dst_log2_page, a.dst_pages, a.dst_seq, a.H, b, h, i);
        k[r] = *(const u32x4*)(a.src[0] + from[r] * (PER * 16) + part * 16);
        v[r] = *(const u32x4*)(a.src[2] + from[r] * (PER * 16) + part * 16);
        if (part < a.n_exps) {                             // (n_exps <= 8; with PER = 4 the other half below)
            ke[r] = a.src[1][from[r] * a.n_exps + part];
            ve[r] = a.src[3][from[r] * a.n_exps + part];
        }
        if (a.w_out && part == 0) w[r] = a.weights[unit * a.w_stride + t[r]];
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int i = i0 + r * kGroup;
        if (i >= count) continue;
        __builtin_nontemporal_store(k[r], (u32x4*)(a.dst[0] + to[r] * (PER * 16) + part * 16));
        __builtin_nontemporal_store(v[r], (u32x4*)(a.dst[2] + to[r] * (PER * 16) + part * 16));
        if (part < a.n_exps) {
            a.dst[1][to[r] * a.n_exps + part] = ke[r];
            a.dst[3][to[r] * a.n_exps + part] = ve[r];
        }
        if (PER < 8 && part + PER < a.n_exps) {            // blocks of 16, 4-bit mantissas
            a.dst[1][to[r] * a.n_exps + part + PER] = a.src[1][from[r] * a.n_exps + part + PER];
            a.dst[3][to[r] * a.n_exps + part + PER] = a.src[3][from[r] * a.n_exps + part + PER];
        }
        if (a.w_out && part == 0) a.w_out[unit * a.n_keep + i] = w[r];
    }
}

}  // namespace

using namespace kvbfp;

static int evict_impl(const char* call, const kvbfp_layout* L, const kvbfp_cache* cache, const Paging* paging, const kvbfp_layout* dst_L,
                      const kvbfp_cache* dst, const Paging* dst_paging, const float* weights, int64_t weights_stride,
                      const int32_t* seq_len_dev, int64_t max_len, int32_t n_keep, int32_t n_first, int32_t n_recent, int32_t* kept,
                      int32_t* new_len, float* weights_out, void* hip_stream) {
    clear_error();
    kvbfp_layout from, to;
    if (paging) {
        if (int rc = check_paging(L, *paging, &from)) return rc;
        if (int rc = check_paging(dst_L, *dst_paging, &to)) return rc;
    } else {
        if (int rc = check_device_layout(L)) return rc;
        if (int rc = check_device_layout(dst_L)) return rc;
        from = *L;
        to = *dst_L;
    }
    if (int rc = check_cache(cache, true, true)) return rc;
    if (int rc = check_cache(dst, true, true)) return rc;
    if (from.block != to.block || from.mant_bits != to.mant_bits || from.n_kv_heads != to.n_kv_heads || from.batch != to.batch)
        return fail(KVBFP_ERR_INVALID_ARG, "%s: the two caches differ in block, mant_bits, heads or batch", call);
    if (!weights || !kept || !new_len) return fail(KVBFP_ERR_INVALID_ARG, "%s: weights/kept/new_len is NULL", call);
    if (max_len <= 0 || max_len > from.max_seq)
        return fail(KVBFP_ERR_INVALID_ARG, "%s: max_len %lld outside (0, max_seq=%lld]", call, (long long)max_len, (long long)from.max_seq);
    if (weights_stride < max_len)
        return fail(KVBFP_ERR_INVALID_ARG, "%s: weights_stride %lld below max_len %lld", call, (long long)weights_stride, (long long)max_len);
    if (n_keep <= 0 || n_keep > to.max_seq)
        return fail(KVBFP_ERR_INVALID_ARG, "%s: n_keep %d outside (0, max_seq=%lld] of the cache that it goes to", call, n_keep, (long long)to.max_seq);
    if (n_first < 0 || n_recent < 0 || (int64_t)n_first + n_recent > n_keep)
        return fail(KVBFP_ERR_INVALID_ARG, "%s: n_first %d and n_recent %d (together at most n_keep = %d)", call, n_first, n_recent, n_keep);
    if (from.batch > 65535 || from.n_kv_heads > 65535) return fail(KVBFP_ERR_UNSUPPORTED, "%s: batch/heads exceed the grid limits", call);
    const void* const p[4] = {cache->k_mant, cache->k_exp, cache->v_mant, cache->v_exp};
    const void* const q[4] = {dst->k_mant, dst->k_exp, dst->v_mant, dst->v_exp};
    const bool one_pool = paging && std::equal(p, p + 4, q);                 // other pages of it
    if (one_pool && (L->max_seq != dst_L->max_seq || L->batch != dst_L->batch))
        return fail(KVBFP_ERR_INVALID_ARG, "%s: one pool with two layouts", call);
    // what is read and what is written, at the same time
    size_t m[2], e[2];
    if (int rc = kvbfp_cache_bytes(L, &m[0], &e[0])) return rc;
    if (int rc = kvbfp_cache_bytes(dst_L, &m[1], &e[1])) return rc;
    const size_t units = (size_t)from.batch * (size_t)from.n_kv_heads, kept_bytes = units * (size_t)n_keep * sizeof(int32_t),
                 lens = (size_t)from.batch * sizeof(int32_t);
    const auto source = [&](int i) { return Span{"the first cache", one_pool ? nullptr : p[i], i & 1 ? e[0] : m[0]}; };
    const auto table = [&](const char* what, const Paging* pg) {
        return Span{what, pg ? pg->block_table : nullptr, pg ? lens * (size_t)pg->table_stride : 0, sizeof(int32_t)};
    };
    if (int rc = check_spans(call,
                             {{"kept", kept, kept_bytes, sizeof(int32_t)}, {"new_len", new_len, lens, sizeof(int32_t)},
                              {"weights_out", weights_out, kept_bytes, sizeof(float)},
                              {"the second cache", q[0], m[1]}, {"the second cache", q[1], e[1]},
                              {"the second cache", q[2], m[1]}, {"the second cache", q[3], e[1]}},
                             {{"weights", weights, units * (size_t)weights_stride * sizeof(float), sizeof(float)},
                              {"seq_len_dev", seq_len_dev, lens, sizeof(int32_t)}, table("block_table", paging), table("dst_table", dst_paging),
                              source(0), source(1), source(2), source(3)}))
        return rc;
    EvictArgs a{};
    a.src[0] = cache->k_mant; a.src[1] = cache->k_exp; a.src[2] = cache->v_mant; a.src[3] = cache->v_exp;
    a.dst[0] = dst->k_mant; a.dst[1] = dst->k_exp; a.dst[2] = dst->v_mant; a.dst[3] = dst->v_exp;
    a.src_seq = from.max_seq; a.dst_seq = to.max_seq;
    if (paging) {
        a.src_table = paging->block_table; a.src_stride = paging->table_stride; a.src_pages = L->batch;
        a.dst_table = dst_paging->block_table; a.dst_stride = dst_paging->table_stride; a.dst_pages = dst_L->batch;
        while (((int64_t)1 << a.src_log2_page) < L->max_seq) ++a.src_log2_page;
        while (((int64_t)1 << a.dst_log2_page) < dst_L->max_seq) ++a.dst_log2_page;
    }
    a.weights = weights; a.w_stride = weights_stride; a.seq_len = seq_len_dev;
    a.max_len = (int32_t)max_len; a.H = from.n_kv_heads; a.batch = from.batch;
    a.n_keep = n_keep; a.n_first = n_first; a.n_recent = n_recent;
    a.kept = kept; a.new_len = new_len; a.w_out = weights_out;
    a.n_exps = kD / from.block;
    hipStream_t s = (hipStream_t)hip_stream;
    a.held = (int32_t)std::min<int64_t>(kHeld, ((max_len + kThreads - 1) / kThreads + 7) / 8 * 8);
    evict_select<<<dim3((unsigned)a.H, (unsigned)a.batch), kThreads, (size_t)a.held * kThreads * sizeof(uint32_t), s>>>(a);
    hipError_t err = hipGetLastError();
    if (err == hipSuccess) {
        const int per = from.mant_bits, rows = 1024 / per;                     // 64 or 128 bytes a row
        const int64_t most = std::min<int64_t>(n_keep, max_len);
        const dim3 grid((unsigned)((most + rows - 1) / rows), (unsigned)a.H, (unsigned)a.batch);
        if (per == 4) evict_rows<4><<<grid, 256, 0, s>>>(a);
        else evict_rows<8><<<grid, 256, 0, s>>>(a);
        err = hipGetLastError();
    }
    if (err != hipSuccess) return fail(KVBFP_ERR_HIP, "%s: %s", call, hipGetErrorString(err));
    return KVBFP_OK;
}

extern "C" {

int kvbfp_evict(const kvbfp_layout* L, const kvbfp_cache* cache, const kvbfp_layout* dst_L, const kvbfp_cache* dst, const float* weights,
                int64_t weights_stride, const int32_t* seq_len_dev, int64_t max_len, int32_t n_keep, int32_t n_first, int32_t n_recent,
                int32_t* kept, int32_t* new_len, float* weights_out, void* hip_stream) {
    return evict_impl("evict", L, cache, nullptr, dst_L, dst, nullptr, weights, weights_stride, seq_len_dev, max_len, n_keep, n_first,
                      n_recent, kept, new_len, weights_out, hip_stream);
}

int kvbfp_evict_paged(const kvbfp_layout* pool, const kvbfp_cache* cache, const int32_t* block_table, int64_t table_stride, int32_t batch,
                      const kvbfp_layout* dst_pool, const kvbfp_cache* dst, const int32_t* dst_table, int64_t dst_stride,
                      const float* weights, int64_t weights_stride, const int32_t* seq_len_dev, int64_t max_len, int32_t n_keep,
                      int32_t n_first, int32_t n_recent, int32_t* kept, int32_t* new_len, float* weights_out, void* hip_stream) {
    const Paging pg{block_table, table_stride, batch}, dst_pg{dst_table, dst_stride, batch};
    return evict_impl("evict_paged", pool, cache, &pg, dst_pool, dst, &dst_pg, weights, weights_stride, seq_len_dev, max_len, n_keep,
                      n_first, n_recent, kept, new_len, weights_out, hip_stream);
}

}  // extern "C"
