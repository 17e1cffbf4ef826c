// Sampling options of a row: temperature, top-k, top-p and min-p.
//
// A row of logits z, its temperature T and the largest eligible logit m give
// weights w_k = exp((z_k - m) / T).  In the order of z descending, index
// ascending, the kept tokens are a prefix: each filter stops at a rank (top-k
// at rank k, top-p where the weights before reach top_p of all, min-p where w
// falls below min_p), and the earliest stop counts.  The prefix ends at a pair
// (key, index): a token is kept iff its logit is larger, or equal with an index
// no larger.  So nothing is sorted: the end is found by histograms of counts
// and weights, digit by digit of an order-preserving integer key of the logit.
//
// Weights are 64-bit fixed-point numbers (rounded once from a double), so sums
// of them are exact and the same in every order, LDS atomics included.
#include <algorithm>

#include "../../include/sd_verify.h"
#include "sdv_device.h"
#include "sdv_internal.h"

namespace sdv {
namespace {

typedef unsigned long long u64;

struct FilterP {
    const void* z;       // [n][stride] fp32 or bf16
    int64_t stride;
    int V;
    int scale_bits;      // weights are multiples of 2^-scale_bits; sums of V stay below 2^63
    const float* temp;   // each [n] or null
    const int32_t* topk;
    const float* topp;
    const float* minp;
    const float* u;      // [n] (draw)
    int32_t* token;
    float* prob;
    int32_t* kept;
    float* out;          // [n][ostride] (filtered rows)
    int64_t ostride;
};

// NaN becomes -inf (never kept), -0 becomes +0 (equal logits have equal keys)
__device__ __forceinline__ float clean(float z) { return z == z ? z + 0.0f : -INFINITY; }
template <typename T> __device__ __forceinline__ float row_at(const T* z, int i) { return clean(ld<T>(z, i)); }
// larger logit, larger key; -inf has the smallest key that occurs
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// What a row's filters are, with every value defined.
struct RowOpts {
    double c;      // log2(e) / T; greedy: unused
    double lmin;   // log2 of min_p, or -inf
    double p;      // top_p; off: +inf
    int k;         // top_k; off: INT_MAX
    bool greedy;
};
__device__ __forceinline__ RowOpts row_opts(const FilterP& p, int row) {
    RowOpts o;
    const float t = p.temp ? p.temp[row] : 1.f;
    o.greedy = !(t > 0.f);
    o.c = o.greedy ? 0.0 : 1.4426950408889634 / (double)t;
    const int k = p.topk ? p.topk[row] : 0;
    o.k = k > 0 ? k : 0x7fffffff;
    const float tp = p.topp ? p.topp[row] : 1.f;
    o.p = tp < 1.f ? (double)tp : INFINITY;
    const float mp = p.minp ? p.minp[row] : 0.f;
    o.lmin = mp > 0.f ? log2((double)mp) : -INFINITY;
    return o;
}
// log2 of the weight of logit z in a row with maximum m
__device__ __forceinline__ double log2_weight(float z, float m, double c) {
    return z == m ? 0.0 : ((double)z - (double)m) * c;
}
__device__ __forceinline__ u64 fixed_weight(double y, int bits) { return (u64)rint(ldexp(exp2(y), bits)); }

constexpr int kBins = 1024;

struct Shared {
    u64 sum[kBins];
    uint32_t cnt[kBins];
    u64 wsum[16], wpre[17];
    uint32_t wcnt[16];
    uint32_t lo, hi;
    uint32_t above_c;
    u64 above_s;
    float fmax[16];
    int found;
};

__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// One workgroup a row.  Passes over the row: maximum; weights' total; one a
// digit of the prefix's last key (10 bits each); the last key's ties if not all
// of them are kept; the kept weights by wave segments; the segment drawn from,
// or the rows written.
template <typename T, bool DRAW>
__global__ __launch_bounds__(1024) void k_filter_row(FilterP p) {
    __shared__ Shared s;
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const T* z = (const T*)p.z + (size_t)row * p.stride;
    const int V = p.V;
    const RowOpts o = row_opts(p, row);
    float m = -INFINITY;
    for (int i = tid; i < V; i += 1024) m = fmaxf(m, row_at(z, i));
    m = wave_max(m);
    if (lane == 0) s.fmax[w] = m;
    __syncthreads();
    for (int i = 0; i < 16; ++i) m = fmaxf(m, s.fmax[i]);
    if (m == -INFINITY) {
        // nothing is eligible
        if (tid == 0) {
            if (DRAW) {
                p.token[row] = -1;
                if (p.prob) p.prob[row] = 0.f;
            }
            if (p.kept) p.kept[row] = 0;
        }
        if (!DRAW)
            for (int i = tid; i < V; i += 1024) p.out[(size_t)row * p.ostride + i] = -INFINITY;
        return;
    }
    // the smallest logit that counts as eligible (an infinite maximum takes all the weight)
    const bool alone = o.greedy || m == INFINITY;
    auto eligible = [&](float v) { return alone ? v == m : v > -INFINITY; };
    // total weight
    u64 S = 0;
    for (int i = tid; i < V; i += 1024) {
        const float v = row_at(z, i);
        if (eligible(v)) S += fixed_weight(log2_weight(v, m, o.c), p.scale_bits);
    }
    S = wave_sum_u64(S);
    if (lane == 0) s.wsum[w] = S;
    __syncthreads();
    S = 0;
    for (int i = 0; i < 16; ++i) S += s.wsum[i];
    // the prefix's last key
    const int k = o.greedy ? 1 : o.k;
    const double P = o.p * (double)S;  // +inf when off
    uint32_t lo = key_of(-INFINITY) + 1, hi = key_of(m), above_c = 0;
    if (alone) lo = hi;
    u64 above_s = 0;
    bool all = false;  // nothing stops the prefix but eligibility and min-p
    // (rank 0 is kept whatever the filters say: a min_p above 1 counts as 1)
    auto passes = [&](float v) { return eligible(v) && log2_weight(v, m, o.c) >= fmin(o.lmin, 0.0); };
    for (;;) {
        const int span = 32 - __clz(hi - lo);  // bits of hi - lo
        const int sh = hi == lo ? 0 : max(0, span - 10);
        s.sum[tid] = 0;
        s.cnt[tid] = 0;
        __syncthreads();
        for (int i = tid; i < V; i += 1024) {
            const float v = row_at(z, i);
            const uint32_t key = key_of(v);
            if (key < lo || key > hi || !passes(v)) continue;
            atomicAdd(&s.cnt[(key - lo) >> sh], 1u);
            atomicAdd(&s.sum[(key - lo) >> sh], fixed_weight(log2_weight(v, m, o.c), p.scale_bits));
        }
        __syncthreads();
        // from the top bin down, the first where a filter stops
        const int b = kBins - 1 - tid;
        const uint32_t c = s.cnt[b];
        const u64 ws = s.sum[b];
        uint32_t ic = c;
        u64 is = ws;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t c2 = __shfl_up(ic, d, 64);
            const u64 s2 = __shfl_up(is, d, 64);
            if (lane >= d) { ic += c2; is += s2; }
        }
        if (lane == 63) { s.wcnt[w] = ic; s.wsum[w] = is; }
        if (tid == 0) s.found = kBins;
        __syncthreads();
        ic += above_c;
        is += above_s;
        for (int i = 0; i < w; ++i) { ic += s.wcnt[i]; is += s.wsum[i]; }
        const bool stops = c > 0 && (ic >= (uint32_t)k || (double)is >= P);
        if (stops) atomicMin(&s.found, tid);
        __syncthreads();
        if (s.found == kBins) { all = true; break; }  // (first digit only)
        if (tid == s.found) {
            s.above_c = ic - c;
            s.above_s = is - ws;
            s.lo = lo + ((uint32_t)b << sh);
            s.hi = min(hi, s.lo + ((1u << sh) - 1));
        }
        __syncthreads();
        lo = s.lo; hi = s.hi; above_c = s.above_c; above_s = s.above_s;
        if (sh == 0) break;
        __syncthreads();
    }
    // ties of the last key: the first `take` of them in index order
    uint32_t take = 0xffffffffu;
    int last = V;  // largest index kept among the ties
    uint32_t cut = all ? 0 : lo;
    if (!all) {
        const double wt = ldexp(exp2(log2_weight(key_value(lo), m, o.c)), p.scale_bits);
        double jp = (double)0xffffffffu;
        if (P < INFINITY) {
            const double left = P - (double)above_s;
            jp = left <= 0.0 ? 0.0 : (wt > 0.0 ? fmin(ceil(left / wt), jp) : jp);
        }
        take = (uint32_t)jp;
        take = min(take, (uint32_t)k - above_c);
        if (above_c == 0) take = max(take, 1u);  // rank 0
        // ties in each wave's segment of the row
        const int seg = (V + 15) / 16, i0 = w * seg, i1 = min(V, i0 + seg);
        uint32_t n = 0;
        for (int i = i0 + lane; i < i1; i += 64) n += key_of(row_at(z, i)) == lo;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) n += __shfl_xor(n, d, 64);
        __syncthreads();
        if (lane == 0) s.wcnt[w] = n;
        if (tid == 0) s.found = V;
        __syncthreads();
        uint32_t before = 0, ties = 0;
        for (int i = 0; i < 16; ++i) {
            if (i < w) before += s.wcnt[i];
            ties += s.wcnt[i];
        }
        take = min(take, ties);
        if (take < ties && before < take && before + n >= take) {
            uint32_t need = take - before;
            for (int i = i0; i < i1; i += 64) {
                const u64 hit = __ballot(i + lane < i1 && key_of(row_at(z, i + lane)) == lo);
                const uint32_t c = __popcll(hit);
                if (c >= need) {
                    if ((hit >> lane & 1) && __popcll(hit & ((2ull << lane) - 1)) == need) s.found = i + lane;
                    break;
                }
                need -= c;
            }
        }
        __syncthreads();
        last = s.found;
    }
    auto keeps = [&](float v, int i) {
        const uint32_t key = key_of(v);
        return passes(v) && (key > cut || (key == cut && i <= last));
    };
    // kept weights and number, by wave segments
    const int seg = (V + 15) / 16, i0 = w * seg, i1 = min(V, i0 + seg);
    u64 ks = 0;
    uint32_t kc = 0;
    for (int i = i0 + lane; i < i1; i += 64) {
        const float v = row_at(z, i);
        const bool on = keeps(v, i);
        if (!DRAW) p.out[(size_t)row * p.ostride + i] = on ? (o.greedy ? 0.f : (float)(log2_weight(v, m, o.c) * 0.6931471805599453)) : -INFINITY;
        if (!on) continue;
        ++kc;
        if (DRAW) ks += fixed_weight(log2_weight(v, m, o.c), p.scale_bits);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) kc += __shfl_xor(kc, d, 64);
    ks = wave_sum_u64(ks);
    __syncthreads();
    if (lane == 0) { s.wcnt[w] = kc; s.wsum[w] = ks; }
    __syncthreads();
    if (tid == 0) {
        u64 t = 0;
        uint32_t c = 0;
        for (int i = 0; i < 16; ++i) { s.wpre[i] = t; t += s.wsum[i]; c += s.wcnt[i]; }
        s.wpre[16] = t;
        if (p.kept) p.kept[row] = (int)c;
    }
    if (!DRAW) return;
    __syncthreads();
    const u64 K = s.wpre[16];
    float u = p.u[row];
    u = u > 0.f ? fminf(u, 1.f - 0x1p-24f) : 0.f;
    const u64 target = min((u64)((double)u * (double)K), K - 1);
    if (!(s.wpre[w] <= target && target < s.wpre[w + 1])) return;
    u64 base = s.wpre[w];
    for (int i = i0; i < i1; i += 64) {
        const float v = i + lane < i1 ? row_at(z, i + lane) : -INFINITY;
        const bool on = i + lane < i1 && keeps(v, i + lane);
        const u64 wt = on ? fixed_weight(log2_weight(v, m, o.c), p.scale_bits) : 0;
        u64 inc = wt;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const u64 x = __shfl_up(inc, d, 64);
            if (lane >= d) inc += x;
        }
        const u64 hit = __ballot(base + inc > target);
        if (hit) {
            if (lane == __ffsll(hit) - 1) {
                p.token[row] = i + lane;
                if (p.prob) p.prob[row] = (float)(ldexp(exp2(log2_weight(v, m, o.c)), p.scale_bits) / (double)K);
            }
            return;
        }
        base += __shfl(inc, 63, 64);
    }
}

}  // namespace

size_t filter_workspace(int n_rows, int V) {
    (void)n_rows; (void)V;
    return 256;
}

template <typename T>
static void launch_typed(const FilterCall& c, const FilterP& p, hipStream_t s) {
    if (c.out)
        hipLaunchKernelGGL((k_filter_row<T, false>), dim3(c.n_rows), dim3(1024), 0, s, p);
    else
        hipLaunchKernelGGL((k_filter_row<T, true>), dim3(c.n_rows), dim3(1024), 0, s, p);
}

void launch_filter(const FilterCall& c, hipStream_t s) {
    FilterP p{};
    p.z = c.logits; p.stride = c.stride; p.V = c.V;
    p.scale_bits = 62;
    while ((1ll << (62 - p.scale_bits)) < c.V) --p.scale_bits;
    p.temp = c.temp; p.topk = c.topk; p.topp = c.topp; p.minp = c.minp;
    p.u = c.u; p.token = c.token; p.prob = c.prob; p.kept = c.kept;
    p.out = c.out; p.ostride = c.ostride;
    if (c.bf16) launch_typed<bf16_t>(c, p, s);
    else launch_typed<float>(c, p, s);
}

}  // namespace sdv

extern "C" {

sd_status sd_filter_query_size(int32_t n_rows, int32_t vocab, uint64_t* workspace_bytes) {
    if (!workspace_bytes || n_rows < 1 || vocab < 1) return SD_EINVAL;
    if (n_rows > SD_FILTER_MAX_ROWS || vocab > SD_FILTER_MAX_VOCAB) return SD_ELIMIT;
    *workspace_bytes = sdv::filter_workspace(n_rows, vocab);
    return SD_OK;
}

// What both calls require; fills the part of c that they share.
static sd_status filter_call(int32_t n_rows, int32_t vocab, const void* logits, int32_t dtype, int64_t row_stride,
                             const sd_filter* f, void* workspace, uint64_t workspace_bytes, sdv::FilterCall* c) {
    uint64_t need = 0;
    const sd_status r = sd_filter_query_size(n_rows, vocab, &need);
    if (r != SD_OK) return r;
    if (!logits || !workspace || (dtype != SD_F32 && dtype != SD_BF16) || row_stride < vocab) return SD_EINVAL;
    if ((uintptr_t)logits % (dtype == SD_BF16 ? 2 : 4) || (uintptr_t)workspace % 256) return SD_EINVAL;
    if (workspace_bytes < need) return SD_ENOMEM;
    c->n_rows = n_rows;
    c->V = vocab;
    c->bf16 = dtype == SD_BF16;
    c->logits = logits;
    c->stride = row_stride;
    if (f) {
        c->temp = f->temperature;
        c->topk = f->top_k;
        c->topp = f->top_p;
        c->minp = f->min_p;
        if (((uintptr_t)c->temp | (uintptr_t)c->topk | (uintptr_t)c->topp | (uintptr_t)c->minp) % 4) return SD_EINVAL;
    }
    c->ws = workspace;
    return SD_OK;
}

sd_status sd_sample_filtered(int32_t n_rows, int32_t vocab, const void* logits, int32_t dtype, int64_t row_stride,
                             const sd_filter* filter, const float* u, int32_t* token, float* prob, int32_t* kept,
                             void* workspace, uint64_t workspace_bytes, sd_stream stream) {
    sdv::FilterCall c{};
    const sd_status r = filter_call(n_rows, vocab, logits, dtype, row_stride, filter, workspace, workspace_bytes, &c);
    if (r != SD_OK) return r;
    if (!u || !token || ((uintptr_t)u | (uintptr_t)token | (uintptr_t)prob | (uintptr_t)kept) % 4) return SD_EINVAL;
    c.u = u;
    c.token = token;
    c.prob = prob;
    c.kept = kept;
    sdv::launch_filter(c, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? SD_OK : SD_EHIP;
}

sd_status sd_filter_logits(int32_t n_rows, int32_t vocab, const void* logits, int32_t dtype, int64_t row_stride,
                           const sd_filter* filter, float* out, int64_t out_stride, int32_t* kept, void* workspace,
                           uint64_t workspace_bytes, sd_stream stream) {
    sdv::FilterCall c{};
    const sd_status r = filter_call(n_rows, vocab, logits, dtype, row_stride, filter, workspace, workspace_bytes, &c);
    if (r != SD_OK) return r;
    if (!out || out_stride < vocab || ((uintptr_t)out | (uintptr_t)kept) % 4) return SD_EINVAL;
    // the rows may be rewritten in place, and may not overlap otherwise
    const uintptr_t i0 = (uintptr_t)logits, o0 = (uintptr_t)out;
    const uintptr_t i1 = i0 + ((uint64_t)(n_rows - 1) * row_stride + vocab) * (dtype == SD_BF16 ? 2 : 4);
    const uintptr_t o1 = o0 + ((uint64_t)(n_rows - 1) * out_stride + vocab) * 4;
    const bool same = i0 == o0 && dtype == SD_F32 && (n_rows == 1 || row_stride == out_stride);
    if (!same && i0 < o1 && o0 < i1) return SD_EINVAL;
    c.out = out;
    c.ostride = out_stride;
    c.kept = kept;
    sdv::launch_filter(c, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? SD_OK : SD_EHIP;
}

}  // extern "C"
