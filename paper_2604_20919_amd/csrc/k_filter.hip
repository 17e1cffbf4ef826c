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
// Weights are rounded to 64-bit fixed-point numbers, so sums of them within a
// workgroup are exact and the same in every order, LDS atomics included; the sums
// of a row's chunks are merged in 64-bit floating point, in a fixed order.
#include <algorithm>

#include "../../include/sd_verify.h"
#include "sdv_device.h"
#include "sdv_internal.h"

// z c and what is subtracted from it are rounded apart everywhere: the largest
// logit's logarithm has to cancel exactly, however large
#pragma clang fp contract(off)

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
    const int32_t* only; // [n]: rows where it is 0 are left as they are (kernels with ONLY)
};
template <bool ONLY> __device__ __forceinline__ bool left_alone(const FilterP& p, int row) {
    return ONLY && p.only[row] == 0;
}

// NaN becomes -inf (never kept)
__device__ __forceinline__ float clean(float z) { return z > -INFINITY ? z : -INFINITY; }
template <typename T> __device__ __forceinline__ float row_at(const T* z, int i) { return clean(ld<T>(z, i)); }
// the larger of numbers that are no NaN (fmaxf would first quiet each)
__device__ __forceinline__ float max_clean(float a, float b) {
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ float max_clean(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// larger logit, larger key, and both zeros the same; -inf has the smallest key
// that occurs
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

constexpr int kMaxShift = 12;  // (2^17 octaves in all, which the logarithms' grid still holds)
// What a row's filters are, with every value defined.
struct RowOpts {
    double c, rc;  // log2(e) / T and its inverse; greedy: 0
    double lmin;   // log2 of min_p, or -inf
    double p;      // top_p; off: +inf
    int k;         // top_k; off: INT_MAX
    int sh;        // buckets are 2^sh eighths of an octave wide
    bool greedy;
    bool filters;  // any of top-k, top-p, min-p
};
__device__ __forceinline__ RowOpts row_opts(const FilterP& p, int row) {
    RowOpts o;
    const float t = p.temp ? p.temp[row] : 1.f;
    o.greedy = !(t > 0.f);
    o.c = o.greedy ? 0.0 : 1.4426950408889634 / (double)t;
    o.rc = o.greedy ? 0.0 : (double)t * 0.6931471805599453;
    // (the lower the temperature, the more octaves a logit makes: the buckets of a row
    // together are 13 to 27 wide in logits from T = 0.6 down to 1.5e-4, where
    // kMaxShift ends it (0.9 at 1e-5), and 22 T above.  With eighths
    // at every temperature the prefix of the 50 largest at T = 0.1 ended below them,
    // and the whole-row path took 600 us for one row of 151936 and 1220 for 416, against 26
    // and 104; the shift costs the first read 65 -> 68 us for 416 rows.)
    o.sh = o.greedy ? 0 : min(max(-ilogbf(t * (1.f / 0.6f)), 0), kMaxShift);
    const int k = p.topk ? p.topk[row] : 0;
    o.k = k > 0 ? k : 0x7fffffff;
    const float tp = p.topp ? p.topp[row] : 1.f;
    o.p = tp < 1.f ? (double)tp : INFINITY;
    const float mp = p.minp ? p.minp[row] : 0.f;
    o.lmin = mp > 0.f ? log2((double)mp) : -INFINITY;
    o.filters = k > 0 || tp < 1.f || mp > 0.f;
    return o;
}
// log2 of the weight of logit z in a row with maximum m
__device__ __forceinline__ double log2_weight(float z, float m, double c) {
    return z == m ? 0.0 : ((double)z - (double)m) * c;
}
__device__ __forceinline__ u64 fixed_weight(double y, int bits) { return (u64)rint(ldexp(exp2(y), bits)); }

constexpr int kRowThreads = 512;  // of the kernels that take a row by one workgroup
constexpr int kRowWaves = kRowThreads / 64;
constexpr int kBins = kRowThreads;  // a digit of 9 bits

struct RowShared {
    u64 sum[kBins];
    uint32_t cnt[kBins];
    u64 wsum[kRowWaves], wpre[kRowWaves + 1];
    uint32_t wcnt[kRowWaves];
    uint32_t lo, hi;
    uint32_t above_c;
    u64 above_s;
    float fmax[kRowWaves];
    uint32_t ties;
    int found;
};

// Scans over the lanes of a wave by moves within the vector registers (a
// shuffle through LDS takes about ten times as long): shifts by 1, 2, 4 and 8
// within rows of 16, then the last lane of rows 0 and 2, and of 1, to the rest.
template <int CTRL, int ROWS, typename T> __device__ __forceinline__ T lane_move(T v, T other) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, other),
                                                                 __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
    } else {
        const u64 a = __builtin_bit_cast(u64, v), b = __builtin_bit_cast(u64, other);
        const uint32_t lo = __builtin_amdgcn_update_dpp((int)(uint32_t)b, (int)(uint32_t)a, CTRL, ROWS, 0xf, false);
        const uint32_t hi = __builtin_amdgcn_update_dpp((int)(b >> 32), (int)(a >> 32), CTRL, ROWS, 0xf, false);
        return __builtin_bit_cast(T, (u64)hi << 32 | lo);
    }
}
// inclusive scan; `none` leaves a value as it is
template <typename T, typename Op> __device__ __forceinline__ T wave_scan(T v, T none, Op op) {
    v = op(v, lane_move<0x111, 0xf>(v, none));
    v = op(v, lane_move<0x112, 0xf>(v, none));
    v = op(v, lane_move<0x114, 0xf>(v, none));
    v = op(v, lane_move<0x118, 0xf>(v, none));
    v = op(v, lane_move<0x142, 0xa>(v, none));
    v = op(v, lane_move<0x143, 0xc>(v, none));
    return v;
}
template <typename T> __device__ __forceinline__ T last_lane(T v) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
    } else {
        const u64 a = __builtin_bit_cast(u64, v);
        const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)a, 63);
        const uint32_t hi = __builtin_amdgcn_readlane((int)(a >> 32), 63);
        return __builtin_bit_cast(T, (u64)hi << 32 | lo);
    }
}
template <typename T> __device__ __forceinline__ T scan_add(T v) {
    return wave_scan(v, (T)0, [](T a, T b) { return a + b; });
}
template <typename T> __device__ __forceinline__ T wave_add(T v) { return last_lane(scan_add(v)); }
__device__ __forceinline__ float wave_top(float v) {
    return last_lane(wave_scan(v, -INFINITY, [](float a, float b) { return max_clean(a, b); }));
}
__device__ __forceinline__ uint32_t wave_least(uint32_t v) {
    return last_lane(wave_scan(v, 0xffffffffu, [](uint32_t a, uint32_t b) { return min(a, b); }));
}

// A whole row by one workgroup, whatever its values: the rows
// that the chunked kernels below leave (see kModeRow).  Bound by its passes' latencies: 0.22 to
// 1.2 ms for one row of 151936, 0.6 to 2.6 ms for 416 (many equal logits, which meet
// in one bin, the longest) against 0.03 and 0.11 ms for rows in chunks; such rows are
// rare, but at 2^20 tokens ordinary ones are among them: more than kList of 2^20 N(0, 1.43) logits
// share the bucket in which top-p 0.95 ends, 4.6 ms a row.  Passes over the row:
// maximum; weights' total; one a digit of the prefix's last key (9 bits
// each); the last key's ties if not all of them are kept; the kept weights by
// wave segments; the segment drawn from, or the rows written.
template <typename T, bool DRAW>
__device__ void filter_row(const FilterP& p, int row, RowShared& s) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const T* z = (const T*)p.z + (size_t)row * p.stride;
    const int V = p.V;
    const RowOpts o = row_opts(p, row);
    float m = -INFINITY;
    for (int i = tid; i < V; i += kRowThreads) m = fmaxf(m, row_at(z, i));
    m = wave_top(m);
    if (lane == 0) s.fmax[w] = m;
    __syncthreads();
    for (int i = 0; i < kRowWaves; ++i) m = fmaxf(m, s.fmax[i]);
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
            for (int i = tid; i < V; i += kRowThreads) p.out[(size_t)row * p.ostride + i] = -INFINITY;
        return;
    }
    // the smallest logit that counts as eligible (an infinite maximum takes all the weight)
    const bool alone = o.greedy || m == INFINITY;
    auto eligible = [&](float v) { return alone ? v == m : v > -INFINITY; };
    // total weight
    u64 S = 0;
    for (int i = tid; i < V; i += kRowThreads) {
        const float v = row_at(z, i);
        if (eligible(v)) S += fixed_weight(log2_weight(v, m, o.c), p.scale_bits);
    }
    S = wave_add(S);
    if (lane == 0) s.wsum[w] = S;
    __syncthreads();
    S = 0;
    for (int i = 0; i < kRowWaves; ++i) S += s.wsum[i];
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
        const int sh = hi == lo ? 0 : max(0, span - 9);
        s.sum[tid] = 0;
        s.cnt[tid] = 0;
        __syncthreads();
        for (int i = tid; i < V; i += kRowThreads) {
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
        uint32_t ic = scan_add(c);
        u64 is = scan_add(ws);
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
        const int seg = (V + kRowWaves - 1) / kRowWaves, i0 = w * seg, i1 = min(V, i0 + seg);
        uint32_t n = 0;
        for (int i = i0 + lane; i < i1; i += 64) n += key_of(row_at(z, i)) == lo;
        n = wave_add(n);
        __syncthreads();
        if (lane == 0) s.wcnt[w] = n;
        if (tid == 0) s.found = V;
        __syncthreads();
        uint32_t before = 0, ties = 0;
        for (int i = 0; i < kRowWaves; ++i) {
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
    const int seg = (V + kRowWaves - 1) / kRowWaves, i0 = w * seg, i1 = min(V, i0 + seg);
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
    kc = wave_add(kc);
    ks = wave_add(ks);
    __syncthreads();
    if (lane == 0) { s.wcnt[w] = kc; s.wsum[w] = ks; }
    __syncthreads();
    if (tid == 0) {
        u64 t = 0;
        uint32_t c = 0;
        for (int i = 0; i < kRowWaves; ++i) { s.wpre[i] = t; t += s.wsum[i]; c += s.wcnt[i]; }
        s.wpre[kRowWaves] = t;
        if (p.kept) p.kept[row] = (int)c;
    }
    if (!DRAW) return;
    __syncthreads();
    const u64 K = s.wpre[kRowWaves];
    float u = p.u[row];
    u = u > 0.f ? fminf(u, 1.f - 0x1p-24f) : 0.f;
    const u64 target = min((u64)((double)u * (double)K), K - 1);
    if (!(s.wpre[w] <= target && target < s.wpre[w + 1])) return;
    u64 base = s.wpre[w];
    for (int i = i0; i < i1; i += 64) {
        const float v = i + lane < i1 ? row_at(z, i + lane) : -INFINITY;
        const bool on = i + lane < i1 && keeps(v, i + lane);
        const u64 wt = on ? fixed_weight(log2_weight(v, m, o.c), p.scale_bits) : 0;
        const u64 inc = scan_add(wt);
        const u64 hit = __ballot(base + inc > target);
        if (hit) {
            if (lane == __ffsll(hit) - 1) {
                p.token[row] = i + lane;
                if (p.prob) p.prob[row] = (float)(ldexp(exp2(log2_weight(v, m, o.c)), p.scale_bits) / (double)K);
            }
            return;
        }
        base += last_lane(inc);
    }
}


// ---------------------------------------------------------------------------
// Rows in chunks of kChunk elements, a workgroup each.
//
// k_filter_scan reads the row once: a chunk's maximum, its weights' sum and, for
// rows with a filter, counts and weights by buckets an eighth of an octave wide
// (in the logarithm of the weight; at low temperatures, where a step of the logit
// is many octaves, 2, 4, 8 .. eighths).  Weights are taken relative to 2^G, G the
// chunk's own largest logarithm rounded up, so that chunks need not know the
// row's maximum, and buckets lie on one grid for all of them: what another
// chunk counts moves by whole buckets, its sums by powers of two.
// k_filter_find merges the chunks of a row and finds the bucket the prefix
// ends in; k_filter_collect writes that bucket's members out in index order;
// k_filter_resolve finds the end among them and draws; k_filter_write writes
// the filtered rows.  The row itself is read by the first and, where a chunk has
// members of the last bucket, the third kernel, and by the writing one.
// ---------------------------------------------------------------------------
// (Chunks of 8192 make half the records, but a chunk with a member of the last
// bucket is read again whole: 416 rows of 151936, 146 against 130 us in all.)
constexpr int kChunk = 4096;
constexpr int kChunkThreads = 256, kChunkWaves = kChunkThreads / 64;
constexpr int kPer = kChunk / kChunkThreads;  // elements a thread
static_assert(kPer <= 32, "k_filter_collect marks them in 32 bits");
constexpr int kBuckets = 256;                 // 32 octaves times 2^sh; what lies below is not counted
constexpr int kList = 16384;                  // most members of the last bucket
constexpr int kFix = 50;                      // chunk sums: multiples of 2^(G - 50), below 2^63
// A bucket of a chunk is one number: the count from bit kCountBit up, and below it
// the weights in units of 2^(G - kHistFix), which stay under it.
constexpr int kCountBit = 50, kHistFix = 37;
// (the count's one rides through the same shift)
__device__ __forceinline__ u64 hist_entry(u64 w) {
    static_assert(kCountBit + kFix - kHistFix == 63, "the count's one is the top bit before the shift");
    return (w + (1ull << 63) + (1ull << (kFix - kHistFix - 1))) >> (kFix - kHistFix);
}
__device__ __forceinline__ u64 hist_weight(u64 w) { return (w + (1ull << (kFix - kHistFix - 1))) >> (kFix - kHistFix); }
constexpr int kMaxChunks = SD_FILTER_MAX_VOCAB / kChunk;
constexpr int kLaneChunks = kMaxChunks / 64;  // of a row, a lane
static_assert(kMaxChunks % 64 == 0 && kMaxChunks <= 4 * kBuckets, "chunks over the lanes and over k_filter_find's threads");

// What a row still needs after k_filter_find.
enum { kModeDone = 0, kModeAll = 1, kModeBorder = 2, kModeRow = 3, kModeEmpty = 4 };

struct ChunkRec {
    double G;       // an integer above the largest log2 weight (z c)
    u64 S;          // sum of weights, units of 2^(G - kFix)
    float m;        // largest logit
    int first;      // its lowest index
    uint32_t n;     // eligible elements
    int bucket;     // the chunk's number of the row's last bucket; -1: above all of its own
    uint32_t off;   // members of the last bucket in the chunks before
    uint32_t have;  // its own
    u64 above;      // kept weights outside the last bucket, units of 2^(G - kHistFix)
};
struct RowRec {
    double G, above, P;  // weights above the last bucket and the filter's bound, units of 2^G
    double c, rc, lmin;  // the row's options (RowOpts)
    int k, sh;
    int mode;
    float m;
    uint32_t n_list, above_c;
    uint32_t klo, khi;   // keys of the last bucket's members
    uint32_t kmin;       // smallest key that min-p lets pass
    uint32_t cut;        // the prefix's last key and last index among its ties
    int last;
};

// Workspace: row records, chunk records, histograms, lists
struct Work {
    RowRec* rows;
    ChunkRec* recs;   // [n][chunks]
    u64* hist;        // [n][chunks][kBuckets]
    uint2* list;      // [n][list_n] (key, index)
    int list_n;       // kList, or the row where that is shorter
};
int chunks_of(int V) { return (V + kChunk - 1) / kChunk; }
size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
size_t layout(int n, int V, void* base, Work* w) {
    const size_t nc = (size_t)n * chunks_of(V);
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += up256(bytes); return (char*)base + at; };
    char* a = take(n * sizeof(RowRec));
    char* b = take(nc * sizeof(ChunkRec));
    char* c = take(nc * kBuckets * 8);
    const int list_n = std::min(kList, V);
    char* d = take((size_t)n * list_n * 8);
    if (w) *w = Work{(RowRec*)a, (ChunkRec*)b, (u64*)c, (uint2*)d, list_n};
    return o;
}

// Element e (0 .. kPer-1) of a thread: 16-byte pieces, threads next to each other
template <typename T> __device__ __forceinline__ int elem_at(int tid, int e) {
    constexpr int W = 16 / sizeof(T);
    return (e / W) * (kChunkThreads * W) + tid * W + e % W;
}
// The thread's elements of the chunk [k0, V) of a row; -inf past the end
template <typename T> __device__ __forceinline__ void load_chunk(const T* z, int k0, int V, float (&v)[kPer]) {
    constexpr int W = 16 / sizeof(T);
    T raw[kPer];
    // (any alignment: the hardware takes 16-byte loads at every address)
    if (k0 + kChunk <= V) {
#pragma unroll
        for (int g = 0; g < kPer / W; ++g)
            __builtin_memcpy(&raw[g * W], z + k0 + elem_at<T>(threadIdx.x, g * W), 16);
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[e] = clean(ld<T>(raw, e));
        return;
    }
#pragma unroll
    for (int g = 0; g < kPer / W; ++g) {
        const int i = k0 + elem_at<T>(threadIdx.x, g * W);
        if (i + W <= V) {
            __builtin_memcpy(&raw[g * W], z + i, 16);
        } else {
#pragma unroll
            for (int e = 0; e < W; ++e) {
                raw[g * W + e] = 0;
                if (i + e < V) raw[g * W + e] = z[i + e];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        v[e] = k0 + elem_at<T>(threadIdx.x, e) < V ? clean(ld<T>(raw, e)) : -INFINITY;
}

// Logarithms on a grid of 2^-32: y = z c - G, -64 <= y < 0, is rounded once, by
// adding 1.5 2^20 in the same operation; the low word is then the fraction,
// the high word kGridHi + floor(y).  The grid is the same for every integer G.
// (Half a table step is added as well: a weight's table entry is the nearest.)
constexpr int kGridHi = 0x41380000;  // high word of 1.5 2^20
constexpr double kGridAdd = 0x1.8p20 + 0x1p-9;
struct Grid {
    double c, add;  // add = kGridAdd - G
    float zmin;     // smaller logits (-inf among them) weigh less than 2^-63: nothing
};
// (rows outside of these bounds, which need |z / T| > 2^39 or T > 10^36, take the whole-row path)
__device__ __forceinline__ bool grid_holds(float m, double c) {
    return c >= 4e-37 && fabs((double)m * c) < 0x1p40;
}
// (zmin's rounding may only make it smaller: far from zero its steps are many
// octaves, up to 2^18 of them, which the grid still holds)
__device__ __forceinline__ Grid grid_of(double G, double c, double rc, int sh = 0) {
    const double z = (G - (double)(32 + (32 << sh))) * rc;
    return Grid{c, kGridAdd - G, (float)(z - fabs(z) * 0x1p-23)};
}
__device__ __forceinline__ double on_grid(const Grid& g, float z) { return fma((double)max_clean(z, g.zmin), g.c, g.add); }
// an integer above m's logarithm on the grid
__device__ __forceinline__ double grid_top(float m, double c, double rc) {
    const double G = floor((double)m * c) + 1.0;
    return on_grid(grid_of(G, c, rc), m) >= kGridAdd ? G + 1.0 : G;
}
// Buckets, 0 the heaviest, are 2^sh eighths of an octave wide and begin at
// multiples of that, whatever G is: `rest` eighths of G are over.
__device__ __forceinline__ int grid_eighths(double y) {
    return (int)(__builtin_amdgcn_alignbit((uint32_t)__double2hiint(y), (uint32_t)__double2loint(y), 29) -
                 ((uint32_t)kGridHi << 3));
}
__device__ __forceinline__ int grid_rest(double G, int sh) { return (int)((long long)(8.0 * G) & ((1ll << sh) - 1)); }
__device__ __forceinline__ int grid_bucket(double y, int rest, int sh) { return -((grid_eighths(y) + rest) >> sh); }

// 2^y in units of 2^-kFix, to about 2^-30 of it: 2^(j/256) from a table in LDS
// (2^30 of it, less the bits of kMagic, and the same as a float) times a second-order series in the rest of
// the fraction, 1/512 at most, as a 31-bit integer; then a shift.  64-bit
// floating point takes twice the time of 32-bit here: the power series up to f^8 in
// it took 43 us of vector work for 256 rows of 151936, this about half.
constexpr int kTab = 256;
constexpr float kMagic = 12582912.f;  // 1.5 2^23: the sum's low bits are the rounded number
constexpr uint32_t kMagicBits = 0x4b400000u;
constexpr double const_exp2(double x) {
    double t = 1.0, r = 1.0;
    for (int k = 1; k < 24; ++k) { t *= x * 0.6931471805599453 / k; r += t; }
    return r;
}
struct Exp2Table {
    uint2 e[kTab];
};
constexpr Exp2Table make_table() {
    Exp2Table t{};
    for (int j = 0; j < kTab; ++j) {
        const double v = const_exp2((double)j / kTab) * 1073741824.0;
        t.e[j].x = (uint32_t)(v + 0.5) - kMagicBits;
        t.e[j].y = __builtin_bit_cast(uint32_t, (float)v);
    }
    return t;
}
__device__ const Exp2Table g_exp2 = make_table();
__device__ __forceinline__ u64 grid_weight(const uint2* tab, double y) {
    const uint32_t lo = (uint32_t)__double2loint(y);
    const uint2 t = tab[lo >> 24];
    // ln2 2^-32 (u - 2^23) + (ln2 2^-32 (u - 2^23))^2 / 2, expanded in u
    constexpr double k1 = 0.6931471805599453 * 0x1p-32, k2 = k1 * k1 / 2, h = 8388608.0;
    const float u = (float)(lo & 0xffffffu);
    const float p = fmaf(fmaf((float)k2, u, (float)(k1 - 2 * k2 * h)), u, (float)(k2 * h * h - k1 * h));
    const uint32_t w = t.x + __float_as_uint(fmaf(__uint_as_float(t.y), p, kMagic));
    const uint32_t s = min((uint32_t)(kGridHi + 62 - kFix) - (uint32_t)__double2hiint(y), 63u);
    return ((u64)w << 32) >> s;
}
__device__ __forceinline__ double pow2(double d) { return d < -1000.0 ? 0.0 : ldexp(1.0, (int)d); }
// buckets between a chunk's numbering and the row's
__device__ __forceinline__ int bucket_shift(double G, double Gc, int sh) {
    const double e = ldexp(8.0, -sh);
    return (int)fmin(floor(e * G) - floor(e * Gc), (double)kBuckets);
}

// Bound by vector instructions, about 30 an element: 416 rows of 151936 fp32 take
// 68 us (3.7 TB/s; reading alone takes 40), rows without filters 35 us for 256 (4.4 TB/s).
// One LDS atomic an element carries count and weight; copies of the histogram
// against bank conflicts changed nothing (2 or 4 of them: -1 or +3 us).
template <typename T, bool ONLY>
__global__ __launch_bounds__(kChunkThreads) void k_filter_scan(FilterP p, Work wk) {
    __shared__ u64 hs[kBuckets];  // (the lightest first: one instruction less an element)
    __shared__ float sm[kChunkWaves];
    __shared__ int si[kChunkWaves];
    __shared__ u64 ss[kChunkWaves];
    __shared__ uint32_t sn[kChunkWaves];
    __shared__ uint2 tab[kTab];
    __shared__ RowOpts opts;
    const int c = blockIdx.x, row = blockIdx.y, nch = gridDim.x;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    if (left_alone<ONLY>(p, row)) return;
    float v[kPer];
    load_chunk<T>((const T*)p.z + (size_t)row * p.stride, c * kChunk, p.V, v);
    if (w == 0) {  // (divisions in 64 bits: for all waves they were an eighth of the work)
        const RowOpts o = row_opts(p, row);
        if (lane == 0) {
            opts.c = o.c;
            opts.rc = o.rc;
            opts.sh = o.sh;
            opts.greedy = o.greedy;
            opts.filters = o.filters;
        }
    }
    for (int i = tid; i < kBuckets; i += kChunkThreads) hs[i] = 0;
    for (int i = tid; i < kTab; i += kChunkThreads) tab[i] = g_exp2.e[i];
    float M = v[0];
#pragma unroll
    for (int e = 1; e < kPer; e += 2) M = max_clean(M, v[e], v[min(e + 1, kPer - 1)]);
    M = wave_top(M);
    if (lane == 0) sm[w] = M;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kChunkWaves; ++i) M = fmaxf(M, sm[i]);
    const double oc = opts.c, orc = opts.rc;
    const bool greedy = opts.greedy, hist = !greedy && opts.filters;
    u64 S = 0;
    uint32_t n = 0;  // of the wave
#pragma unroll
    for (int e = 0; e < kPer; ++e) n += __popcll(__ballot(v[e] > -INFINITY));
    int first = 0x7fffffff;
    double G = floor((double)M * oc) + 1.0;
    if (greedy) {
#pragma unroll
        for (int e = kPer - 1; e >= 0; --e)
            if (v[e] == M) first = c * kChunk + elem_at<T>(tid, e);
        first = (int)wave_least((uint32_t)first);
    } else if (M > -INFINITY && grid_holds(M, oc)) {
        G = grid_top(M, oc, orc);
        const int sh = __builtin_amdgcn_readfirstlane(opts.sh), rest = grid_rest(G, sh);
        const Grid g = grid_of(G, oc, orc, sh);
        // (four elements at a time in flight: more take registers from other waves)
        if (hist) {
#pragma unroll
            for (int e0 = 0; e0 < kPer; e0 += 4) {
                u64 x[4];
                int b[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const double y = on_grid(g, v[e0 + e]);
                    x[e] = grid_weight(tab, y);
                    b[e] = (grid_eighths(y) + rest) >> sh;
                    S += x[e];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (b[e] > -kBuckets) atomicAdd(&hs[b[e] + (kBuckets - 1)], hist_entry(x[e]));
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                S += grid_weight(tab, on_grid(g, v[e]));
                if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    S = wave_add(S);
    if (lane == 0) { si[w] = first; ss[w] = S; sn[w] = n; }
    __syncthreads();
    const size_t at = (size_t)row * nch + c;
    if (hist)
        for (int i = tid; i < kBuckets; i += kChunkThreads) wk.hist[at * kBuckets + i] = hs[kBuckets - 1 - i];
    if (tid == 0) {
        for (int i = 1; i < kChunkWaves; ++i) { first = min(first, si[i]); S += ss[i]; n += sn[i]; }
        ChunkRec r{};
        r.G = G; r.S = S; r.m = M; r.first = first; r.n = n;
        wk.recs[at] = r;
    }
}

// Smallest key for which `in`, monotone in the key, holds; it does for `top`.
// One wave narrows a bracket of keys, 64 at once, from the keys around the logit
// `edge` that the border should have.
template <typename F>
__device__ __forceinline__ uint32_t first_key(F in, double edge, double off, uint32_t top, int lane) {
    const uint32_t least = key_of(-INFINITY);
    uint32_t lo = key_of((float)(edge - off)), hi = key_of((float)(edge + off));
    if (!(lo >= least && lo < hi && !in(lo))) lo = least;
    if (!(hi > lo && hi <= top && in(hi))) hi = top;
    while (hi - lo > 1) {  // lo is out (or -inf), hi is in
        const uint32_t step = (hi - lo + 63) / 64;
        const int i = __ffsll(__ballot(in(min(lo + step * (lane + 1), hi)))) - 1;  // (the last lane's key is hi)
        lo += step * i;
        hi = min(lo + step, hi);
    }
    return hi;
}

// One workgroup a row; four threads hold each bucket of the row and take a
// quarter of its chunks.  Bound by its chain of loads and barriers: 9 us for 1 to
// 130 rows of 151936, 14 us for 416.
constexpr int kFindThreads = 4 * kBuckets;
template <bool DRAW, bool ONLY>
__global__ __launch_bounds__(kFindThreads) void k_filter_find(FilterP p, Work wk, int nch) {
    __shared__ double cG[kMaxChunks], cS[kMaxChunks], unit[kMaxChunks], bsum[4][kBuckets], sd[16];
    __shared__ uint32_t bcnt[4][kBuckets], cn[kMaxChunks], cfirst[kMaxChunks], su[16];
    __shared__ float cm[kMaxChunks];
    __shared__ int shift[kMaxChunks];  // from a chunk's buckets to the row's; kBuckets: none is shared
    __shared__ int sfound;
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int bk = tid % kBuckets, part = tid / kBuckets;
    if (left_alone<ONLY>(p, row)) return;
    ChunkRec* recs = wk.recs + (size_t)row * nch;
    const RowOpts o = row_opts(p, row);
    if (tid < nch) {
        const ChunkRec r = recs[tid];
        cG[tid] = r.G; cS[tid] = (double)r.S; cm[tid] = r.m; cn[tid] = r.n; cfirst[tid] = r.first;
    }
    if (tid == 0) sfound = kBuckets;
    __syncthreads();
    // the row's maximum, its lowest index and 2^G that its sums refer to (each wave by itself)
    float m = -INFINITY;
    for (int c = lane; c < nch; c += 64) m = fmaxf(m, cm[c]);
    m = wave_top(m);
    const double G = grid_top(m, o.c, o.rc);  // that of the chunk with the maximum
    RowRec r{};
    r.G = G;
    r.m = m;
    r.c = o.c;
    r.rc = o.rc;
    r.lmin = fmin(o.lmin, 0.0);
    r.k = o.k;
    r.sh = o.sh;
    r.last = p.V;
    r.cut = key_of(-INFINITY) + 1;
    if (m == -INFINITY || o.greedy || !grid_holds(m, o.c)) {
        if (w) return;
        int first = 0x7fffffff;
        for (int c = lane; c < nch; c += 64)
            if (cm[c] == m) first = min(first, (int)cfirst[c]);
        first = (int)wave_least((uint32_t)first);
        if (lane == 0) {
            r.mode = m == -INFINITY ? kModeEmpty : o.greedy ? kModeDone : kModeRow;
            r.cut = key_of(m);
            r.last = first;
            wk.rows[row] = r;
            if (r.mode != kModeRow) {
                const bool one = r.mode == kModeDone;
                if (p.kept) p.kept[row] = one;
                if (DRAW) {
                    p.token[row] = one ? first : -1;
                    if (p.prob) p.prob[row] = one ? 1.f : 0.f;
                }
            }
        }
        return;
    }
    // the chunks' places and units in the row's histogram, once for all threads
    if (tid < nch) {
        shift[tid] = cm[tid] > -INFINITY ? bucket_shift(G, cG[tid], o.sh) : kBuckets;
        unit[tid] = cm[tid] > -INFINITY ? pow2(cG[tid] - G - kHistFix) : 0.0;
    }
    // total weight and number
    double S = 0.0;
    uint32_t n = 0;
    for (int c = lane; c < nch; c += 64) {
        if (cm[c] == -INFINITY) continue;
        S += cS[c] * pow2(cG[c] - G - kFix);
        n += cn[c];
    }
    S = wave_add(S);
    n = wave_add(n);
    r.P = o.p * S;
    r.mode = kModeAll;
    if (!o.filters) {
        if (tid == 0) {
            wk.rows[row] = r;
            if (p.kept) p.kept[row] = (int)n;
        }
        return;
    }
    __syncthreads();
    {
        uint32_t cnt = 0;
        double sum = 0.0;
        const size_t at0 = (size_t)row * nch * kBuckets;
        constexpr int kAhead = 12;  // loads at once
        for (int c0 = part; c0 < nch; c0 += 4 * kAhead) {
            u64 x[kAhead];
            int b[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int c = c0 + 4 * j;
                b[j] = c < nch ? bk - shift[c] : -1;
                x[j] = wk.hist[at0 + (size_t)min(c, nch - 1) * kBuckets + max(b[j], 0)];
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (b[j] < 0) continue;
                cnt += (uint32_t)(x[j] >> kCountBit);
                sum += (double)(x[j] & ((1ull << kCountBit) - 1)) * unit[c0 + 4 * j];
            }
        }
        bcnt[part][bk] = cnt;
        bsum[part][bk] = sum;
    }
    __syncthreads();
    uint32_t cnt = 0, ic = 0;
    double sum = 0.0, is = 0.0;
    if (tid < kBuckets) {
        ic = cnt = bcnt[0][tid] + bcnt[1][tid] + bcnt[2][tid] + bcnt[3][tid];
        is = sum = (bsum[0][tid] + bsum[1][tid]) + (bsum[2][tid] + bsum[3][tid]);
        ic = scan_add(ic);
        is = scan_add(is);
        if (lane == 63) { su[w] = ic; sd[w] = is; }
    }
    __syncthreads();
    // from the heaviest bucket down, the first where a filter stops
    const int rest = grid_rest(G, o.sh);
    const Grid g = grid_of(G, o.c, o.rc, o.sh);
    if (tid < kBuckets) {
        for (int i = 0; i < w; ++i) { ic += su[i]; is += sd[i]; }
        const double y = on_grid(g, m);
        const int bmin = o.lmin > -INFINITY
            ? (int)fmin(-floor(ldexp(floor(8.0 * (y - 0x1.8p20 + r.lmin)) + rest, -o.sh)), (double)kBuckets) : kBuckets;
        if (cnt > 0 && (ic >= (uint32_t)o.k || is >= r.P || tid >= bmin)) atomicMin(&sfound, tid);
    }
    __syncthreads();
    const int border = sfound;
    if (border == kBuckets) {
        // all counted ones are kept; if there are more, the whole row decides
        const uint32_t counted = su[0] + su[1] + su[2] + su[3];
        if (counted < n) r.mode = kModeRow;
        if (tid == 0) {
            wk.rows[row] = r;
            if (p.kept && r.mode == kModeAll) p.kept[row] = (int)n;
        }
        return;
    }
    if (tid == border) {
        su[8] = cnt;
        su[9] = ic - cnt;
        sd[8] = is - sum;
    }
    __syncthreads();
    if (w == 0) {
        // members of each chunk before the next
        uint32_t run = 0;
        for (int c0 = 0; c0 < nch; c0 += 64) {
            const int c = c0 + lane;
            int b = -1;
            uint32_t k = 0;
            if (c < nch) {
                b = border - shift[c];
                if (b >= 0) k = (uint32_t)(wk.hist[((size_t)row * nch + c) * kBuckets + b] >> kCountBit);
            }
            const uint32_t inc = scan_add(k);
            if (c < nch) {
                recs[c].bucket = max(b, -1);
                recs[c].off = run + inc - k;
                recs[c].have = k;
            }
            run += last_lane(inc);
        }
    } else if (w < 4) {
        // waves 1 and 2: the border bucket's keys; wave 3: min-p's
        const uint32_t top = key_of(m);
        uint32_t k = 0;
        if (w < 3) {
            const int b = border + 1 - w;
            k = top + 1;  // (no bucket above the maximum's)
            if (grid_bucket(on_grid(g, m), rest, o.sh) <= b)
                k = first_key([&](uint32_t x) { return grid_bucket(on_grid(g, key_value(x)), rest, o.sh) <= b; },
                              (G - 0.125 * (ldexp((double)b, o.sh) + rest) - 0x1p-9) * o.rc,
                              0x1p-31 * o.rc + fabs(G * o.rc) * 0x1p-22, top, lane);
        } else if (o.lmin > -INFINITY) {
            k = first_key([&](uint32_t x) {
                const float z = key_value(x);
                return z == m || ((double)z - (double)m) * o.c >= r.lmin;
            }, (double)m + r.lmin / o.c, (fabs((double)m) + fabs(r.lmin / o.c)) * 0x1p-22, top, lane);
        }
        if (lane == 0) su[9 + w] = k;
    }
    __syncthreads();
    if (tid == 0) {
        r.n_list = su[8];
        r.above_c = su[9];
        r.above = sd[8];
        r.klo = su[10];
        r.khi = su[11] - 1;
        r.kmin = su[12];
        r.mode = r.n_list > (uint32_t)wk.list_n ? kModeRow : kModeBorder;
        wk.rows[row] = r;
    }
}

// The members of the last bucket, in index order, and (DRAW) each chunk's
// weights above it.  Chunks without members are not read: 4.5 us for one row of
// 151936, 27 us for 416, whose chunks all have some (9.4 TB/s, most of it from the
// caches).
template <typename T, bool DRAW, bool ONLY>
__global__ __launch_bounds__(kChunkThreads) void k_filter_collect(FilterP p, Work wk) {
    constexpr int W = 16 / sizeof(T), NG = kPer / W;
    __shared__ uint32_t sc[NG][kChunkWaves];
    const int c = blockIdx.x, row = blockIdx.y, nch = gridDim.x;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    if (left_alone<ONLY>(p, row)) return;
    const RowRec& rr = wk.rows[row];
    const int mode = rr.mode;
    if (mode != kModeBorder) return;
    ChunkRec* rec = wk.recs + (size_t)row * nch + c;
    const int bucket = rec->bucket;
    if (DRAW && w == kChunkWaves - 1) {
        const u64* h = wk.hist + ((size_t)row * nch + c) * kBuckets;
        u64 a = 0;
#pragma unroll
        for (int e = 0; e < kBuckets / 64; ++e)
            if (lane + 64 * e < bucket) a += h[lane + 64 * e] & ((1ull << kCountBit) - 1);
        a = wave_add(a);
        if (lane == 0) rec->above = a;
    }
    if (rec->have == 0) return;
    const uint32_t klo = rr.klo, khi = rr.khi, off = rec->off;
    float v[kPer];
    load_chunk<T>((const T*)p.z + (size_t)row * p.stride, c * kChunk, p.V, v);
    uint32_t mine = 0;  // bit e: element e is a member
    uint32_t before[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        uint32_t b = 0, tot = 0;
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const uint32_t key = key_of(v[g * W + e]);
            const bool in = key >= klo && key <= khi;
            const u64 mask = __ballot(in);
            mine |= in ? 1u << (g * W + e) : 0u;
            b += __popcll(mask & ((1ull << lane) - 1));
            tot += __popcll(mask);
        }
        before[g] = b;
        if (lane == 0) sc[g][w] = tot;
    }
    __syncthreads();
    const uint32_t room = (uint32_t)wk.list_n - off;
    uint2* list = wk.list + (size_t)row * wk.list_n + off;
    uint32_t base = 0;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        uint32_t at = base + before[g];
        for (int i = 0; i < kChunkWaves; ++i) {
            if (i < w) at += sc[g][i];
            base += sc[g][i];
        }
#pragma unroll
        for (int e = 0; e < W; ++e)
            // (there is room for every member; the bound holds if someone writes the logits meanwhile)
            if ((mine >> (g * W + e) & 1) && at < room)
                list[at++] = uint2{key_of(v[g * W + e]), (uint32_t)(c * kChunk + elem_at<T>(tid, g * W + e))};
    }
}

struct ResolveShared {
    u64 sum[4][kBins];      // a digit's weights and counts
    uint32_t cnt[4][kBins];
    u64 wsum[kRowWaves];
    uint32_t wcnt[kRowWaves];
    uint32_t ties_of[64];
    uint32_t lo, hi, above_c, ties, kept, key;
    u64 above_s, goal;
    int found, last, chunk;
    double K;
    u64 cadd[kMaxChunks];  // chunks' kept weights from the last bucket, units of 2^(G_chunk - kHistFix)
    double cG[kMaxChunks];
    RowRec r;
};
constexpr int kHeld = 8;                        // members of the last bucket that a thread holds
constexpr int kHeldAll = kHeld * kRowThreads;   // at once; longer lists are read again for each pass

// One workgroup a row: the end of the prefix among the last bucket's members,
// then the chunk and the element drawn.  Bound by its chain of passes over the
// members: 11 us for one row of 151936, 26 us for 416.  PLAIN: no row has a
// filter, and the chunks are merged here: 6.5 us for 256 rows, against 15.5 us
// of this kernel and the two before it.
template <typename T, bool DRAW, bool PLAIN, bool ONLY>
__global__ __launch_bounds__(kRowThreads, 4) void k_filter_resolve(FilterP p, Work wk, int nch) {
    __shared__ union { RowShared row; ResolveShared s; } sh;
    __shared__ uint2 tab[kTab];
    ResolveShared& s = sh.s;
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    if (left_alone<ONLY>(p, row)) return;
    const ChunkRec* recs = wk.recs + (size_t)row * nch;
    // (wave 0 holds the chunks' weights from here to the draw)
    u64 cabove[kLaneChunks];
    double cG[kLaneChunks];
#pragma unroll
    for (int e = 0; e < kLaneChunks; ++e) {
        cabove[e] = 0;
        cG[e] = 0.0;
    }
    float u = 0.f;
    RowRec r;
    if (PLAIN) {
        if (w == 0) {
            const RowOpts o = row_opts(p, row);
            u = p.u[row];
            float cm[kLaneChunks], top = -INFINITY;
            uint32_t n = 0, first = 0xffffffffu, cf[kLaneChunks];
#pragma unroll
            for (int e = 0; e < kLaneChunks; ++e) {
                const int c = lane + 64 * e;
                cm[e] = -INFINITY;
                cf[e] = 0;
                if (c < nch) {
                    cm[e] = recs[c].m;
                    cf[e] = (uint32_t)recs[c].first;
                    n += recs[c].n;
                    if (cm[e] > -INFINITY) {
                        cG[e] = recs[c].G;
                        cabove[e] = recs[c].S;
                    }
                }
                top = max_clean(top, cm[e]);
                s.cG[c] = cG[e];
                s.cadd[c] = 0;
            }
            r = RowRec{};
            r.m = wave_top(top);
            r.c = o.c;
            r.rc = o.rc;
            r.sh = o.sh;
            r.cut = key_of(-INFINITY) + 1;
            r.last = p.V;
            r.mode = r.m == -INFINITY ? kModeEmpty : o.greedy ? kModeDone : grid_holds(r.m, o.c) ? kModeAll : kModeRow;
            if (r.mode == kModeAll) r.G = grid_top(r.m, o.c, o.rc);
            n = wave_add(n);
#pragma unroll
            for (int e = 0; e < kLaneChunks; ++e)
                if (cm[e] == r.m) first = min(first, cf[e]);
            first = wave_least(first);
            if (lane == 0) {
                s.r = r;
                if (r.mode != kModeRow) {
                    if (p.kept) p.kept[row] = r.mode == kModeAll ? (int)n : r.mode == kModeDone;
                    if (r.mode != kModeAll) {
                        p.token[row] = r.mode == kModeDone ? (int)first : -1;
                        if (p.prob) p.prob[row] = r.mode == kModeDone ? 1.f : 0.f;
                    }
                }
            }
        }
        __syncthreads();
        r = s.r;
        __syncthreads();  // (the whole-row path takes the same memory)
    } else {
        r = wk.rows[row];
    }
    if (r.mode == kModeDone || r.mode == kModeEmpty) return;
    if (r.mode == kModeRow) {
        filter_row<T, DRAW>(p, row, sh.row);
        return;
    }
    if (!DRAW && r.mode == kModeAll) return;
    const bool border = !PLAIN && r.mode == kModeBorder;
    if (tid < kTab) tab[tid] = g_exp2.e[tid];
    if (!PLAIN && DRAW && w == 0) {
        u = p.u[row];
#pragma unroll
        for (int e = 0; e < kLaneChunks; ++e) {
            const int c = lane + 64 * e;
            if (c < nch && recs[c].m > -INFINITY) {
                cG[e] = recs[c].G;
                cabove[e] = border ? recs[c].above : recs[c].S;
            }
            s.cG[c] = cG[e];
            s.cadd[c] = 0;
        }
    }
    if (border) {
        const uint2* list = wk.list + (size_t)row * wk.list_n;
        const int n = (int)r.n_list, w0 = __builtin_amdgcn_readfirstlane(tid & ~63);
        uint2 held[kHeld];
        auto hold = [&](int i0) {
#pragma unroll
            for (int j = 0; j < kHeld; ++j) {
                const int i = i0 + j * kRowThreads + tid;
                held[j] = list[min(i, n - 1)];
                if (i >= n) held[j].x = 0;  // (no member has key 0)
            }
        };
        hold(0);
#pragma unroll
        for (int i = 0; i < 4; ++i) { s.sum[i][tid] = 0; s.cnt[i][tid] = 0; }
        if (tid == 0) { s.found = 0; s.kept = 0; }
        __syncthreads();
        uint32_t lo = max(r.klo, r.kmin), hi = r.khi, cut = hi, ties = 0, take = 0;
        int last = -1;  // (min-p leaves none of them)
        if (lo <= hi) {
            // weights in units of 2^(Gb - kFix), Gb above the bucket's logarithms by one at
            // least: sums of kList stay below 2^63
            const double Gb = floor((double)key_value(hi) * r.c) + 2.0;
            const Grid g = grid_of(Gb, r.c, r.rc, r.sh);
            // (a bound of nothing stops at the first: rank 0 is kept)
            const double need = fmax((r.P - r.above) * ldexp(1.0, (int)fmin(fmax(r.G - Gb, -100.0), 100.0) + kFix), 0.5);
            uint32_t above_c = r.above_c;
            u64 above_s = 0;
            for (int it = 0; it < 4; ++it) {
                const int sf = hi == lo ? 0 : max(0, 32 - __clz(hi - lo) - 9);
                for (int i0 = 0; i0 < n; i0 += kHeldAll) {
                    if (n > kHeldAll) hold(i0);
#pragma unroll
                    for (int j = 0; j < kHeld; ++j) {
                        if (i0 + j * kRowThreads + w0 >= n) break;
                        const uint32_t key = held[j].x;
                        if (key < lo || key > hi) continue;
                        atomicAdd(&s.cnt[it][(key - lo) >> sf], 1u);
                        atomicAdd(&s.sum[it][(key - lo) >> sf], grid_weight(tab, on_grid(g, key_value(key))));
                    }
                }
                __syncthreads();
                const int b = kBins - 1 - tid;
                const uint32_t c = s.cnt[it][b];
                const u64 ws = s.sum[it][b];
                uint32_t ic = scan_add(c);
                u64 is = scan_add(ws);
                if (lane == 63) { s.wcnt[w] = ic; s.wsum[w] = is; }
                __syncthreads();
                ic += above_c;
                is += above_s;
#pragma unroll
                for (int i = 0; i < kRowWaves - 1; ++i)
                    if (i < w) { ic += s.wcnt[i]; is += s.wsum[i]; }
                // the bin in which a filter stops: the sums grow, so there is one
                if (c > 0 && (ic >= (uint32_t)r.k || (double)is >= need) &&
                    !(ic - c >= (uint32_t)r.k || (double)(is - ws) >= need)) {
                    s.above_c = ic - c;
                    s.above_s = is - ws;
                    s.lo = lo + ((uint32_t)b << sf);
                    s.hi = min(hi, lo + ((uint32_t)b << sf) + ((1u << sf) - 1));
                    s.ties = c;
                    s.found = it + 1;
                }
                __syncthreads();
                if (s.found != it + 1) {  // min-p alone ends the prefix
                    cut = lo;
                    last = p.V;
                    break;
                }
                lo = s.lo; hi = s.hi; above_c = s.above_c; above_s = s.above_s;
                ties = s.ties;
                if (sf && ties == 1 && n <= kHeldAll) {
                    // one member: its key is the last, and it is kept (a filter stops at it, not before)
#pragma unroll
                    for (int j = 0; j < kHeld; ++j)
                        if (held[j].x >= lo && held[j].x <= hi) s.key = held[j].x;
                    __syncthreads();
                    cut = s.key;
                    take = ties;
                    last = p.V;
                    break;
                }
                if (sf) continue;
                cut = lo;
                double jp = 4e9;
                if (need < INFINITY) {
                    const double wt = (double)grid_weight(tab, on_grid(g, key_value(lo)));
                    const double left = need - (double)above_s;
                    jp = left <= 0.0 ? 0.0 : wt > 0.0 ? fmin(ceil(left / wt), jp) : jp;
                }
                take = min((uint32_t)jp, (uint32_t)r.k - above_c);
                if (above_c == 0) take = max(take, 1u);
                last = p.V;
                break;
            }
            if (take < ties) {
                // the index of the last tie kept: ties by wave and piece of the list
                uint32_t left = take;
                for (int i0 = 0; i0 < n; i0 += kHeldAll) {
                    if (n > kHeldAll) hold(i0);
#pragma unroll
                    for (int j = 0; j < kHeld; ++j) {
                        const u64 hit = __ballot(held[j].x == cut);
                        if (lane == 0) s.ties_of[j * kRowWaves + w] = __popcll(hit);
                    }
                    __syncthreads();
                    const uint32_t c = s.ties_of[lane], inc = scan_add(c);
                    const u64 past = __ballot(inc >= left);
                    if (past) {
                        const int at = __ffsll(past) - 1;
                        const uint32_t nth = left - (__shfl(inc, at, 64) - __shfl(c, at, 64));
#pragma unroll
                        for (int j = 0; j < kHeld; ++j) {
                            if (at != j * kRowWaves + w) continue;
                            const u64 hit = __ballot(held[j].x == cut);
                            if ((hit >> lane & 1) && __popcll(hit & ((2ull << lane) - 1)) == nth) s.last = (int)held[j].y;
                        }
                        __syncthreads();
                        break;
                    }
                    left -= last_lane(inc);
                    __syncthreads();
                }
                last = s.last;
            }
        }
        // number kept, and the members' weights by chunk (those of a wave mostly lie in one)
        for (int i0 = 0; i0 < n; i0 += kHeldAll) {
            if (n > kHeldAll) hold(i0);
#pragma unroll
            for (int j = 0; j < kHeld; ++j) {
                if (i0 + j * kRowThreads + w0 >= n) break;
                const uint2 x = held[j];
                const bool on = x.x > cut || (x.x == cut && (int)x.y <= last);
                const u64 who = __ballot(on);
                if (!who) continue;
                if (lane == 0) atomicAdd(&s.kept, (uint32_t)__popcll(who));
                if (DRAW) {
                    const int c = (int)x.y / kChunk, c0 = __builtin_amdgcn_readlane(c, __ffsll(who) - 1);
                    const u64 wt = on ? hist_weight(grid_weight(tab, on_grid(grid_of(s.cG[c], r.c, r.rc, r.sh), key_value(x.x)))) : 0;
                    if (__ballot(on && c != c0)) {
                        if (on) atomicAdd(&s.cadd[c], wt);
                    } else {
                        const u64 sum = wave_add(wt);
                        if (lane == 0) atomicAdd(&s.cadd[c0], sum);
                    }
                }
            }
        }
        __syncthreads();
        if (tid == 0) {
            if (p.kept) p.kept[row] = (int)(r.above_c + s.kept);
            if (!DRAW) {
                wk.rows[row].cut = cut;
                wk.rows[row].last = last;
            }
        }
        r.cut = cut;
        r.last = last;
    }
    if (!DRAW) return;
    // the chunk in which the running sum passes the target (the last with weight
    // if rounding lets none): wave 0, kLaneChunks a lane
    const int unit = border ? kHistFix : kFix;
    if (w == 0) {
        double x[kLaneChunks], inc[kLaneChunks], K = 0.0;
#pragma unroll
        for (int e = 0; e < kLaneChunks; ++e) {
            inc[e] = x[e] = 0.0;
            if (64 * e >= nch) continue;
            cabove[e] += s.cadd[lane + 64 * e];
            x[e] = cabove[e] ? (double)cabove[e] * pow2(cG[e] - r.G - unit) : 0.0;
            inc[e] = K + scan_add(x[e]);
            K = last_lane(inc[e]);
        }
        u = u > 0.f ? fminf(u, 1.f - 0x1p-24f) : 0.f;
        const double target = (double)u * K;
        int ch = -1, last = 0;
#pragma unroll
        for (int e = 0; e < kLaneChunks; ++e) {
            const u64 past = __ballot(x[e] > 0.0 && inc[e] > target), some = __ballot(x[e] > 0.0);
            if (ch < 0 && past) ch = 64 * e + __ffsll(past) - 1;
            if (some) last = 64 * e + 63 - __clzll(some);
        }
        if (ch < 0) ch = last;
#pragma unroll
        for (int e = 0; e < kLaneChunks; ++e)
            if (lane + 64 * e == ch) {
                const double local = fmin(fmax((target - (inc[e] - x[e])) * pow2(r.G - cG[e] + unit), 0.0), 0x1p63);
                s.chunk = ch;
                s.K = K;
                s.goal = min((u64)local, cabove[e] - 1);
            }
    }
    __syncthreads();
    const int ch = s.chunk;
    const u64 goal = s.goal;
    // its elements in index order: the first whose running sum exceeds the goal
    constexpr int E = kChunk / kRowThreads, W = 16 / sizeof(T);
    const Grid g = grid_of(s.cG[ch], r.c, r.rc, r.sh);
    const T* z = (const T*)p.z + (size_t)row * p.stride;
    const int i0 = ch * kChunk + tid * E;
    T raw[E];
    if ((ch + 1) * kChunk <= p.V) {
#pragma unroll
        for (int q = 0; q < E; q += W) __builtin_memcpy(&raw[q], z + i0 + q, 16);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) raw[e] = z[min(i0 + e, p.V - 1)];
    }
    u64 x[E], mysum = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float v = i0 + e < p.V ? clean(ld<T>(raw, e)) : -INFINITY;
        const uint32_t key = key_of(v);
        const bool on = key > r.cut || (key == r.cut && i0 + e <= r.last);
        const u64 t = grid_weight(tab, on_grid(g, v));
        x[e] = on ? (border ? hist_weight(t) : t) : 0;
        mysum += x[e];
    }
    const u64 inc = scan_add(mysum);
    if (lane == 63) s.wsum[w] = inc;
    __syncthreads();
    u64 at = inc - mysum;
#pragma unroll
    for (int i = 0; i < kRowWaves - 1; ++i)
        if (i < w) at += s.wsum[i];
    if (at <= goal && goal < at + mysum) {
        int hit = 0;
        float v = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (at <= goal && goal < at + x[e]) {
                hit = e;
                v = ld<T>(raw, e);
            }
            at += x[e];
        }
        p.token[row] = i0 + hit;
        if (p.prob) p.prob[row] = (float)(exp2(fma((double)v, r.c, -r.G)) / s.K);  // (as the weights: one rounding)
    }
}

// The filtered rows from each row's cut.  Chunks of which nothing is kept are not
// read again, and what is written goes past the caches, which hold the rows of
// the first read: 229 rows of 151936, 44 -> 38 us, and 44 -> 39 us for the first
// read of the next rows, which then finds no lines to be written back.
template <typename T, bool ONLY>
__global__ __launch_bounds__(kChunkThreads) void k_filter_write(FilterP p, Work wk) {
    constexpr int W = 16 / sizeof(T);
    const int c = blockIdx.x, row = blockIdx.y;
    if (left_alone<ONLY>(p, row)) return;
    const RowRec& rr = wk.rows[row];
    const int mode = rr.mode;
    if (mode == kModeRow) return;  // written by k_filter_resolve
    const uint32_t cut = rr.cut;
    float v[kPer];
    if (mode != kModeEmpty && key_of(wk.recs[(size_t)row * gridDim.x + c].m) >= cut) {
        load_chunk<T>((const T*)p.z + (size_t)row * p.stride, c * kChunk, p.V, v);
    } else {
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[e] = -INFINITY;
    }
    const float m = rr.m;
    const int last = rr.last;
    const float t = p.temp ? p.temp[row] : 1.f;
    const double it = t > 0.f ? 1.0 / (double)t : 0.0;
    float* out = p.out + (size_t)row * p.ostride;
#pragma unroll
    for (int g = 0; g < kPer / W; ++g) {
        const int i = c * kChunk + elem_at<T>(threadIdx.x, g * W);
        float f[W];
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const float x = v[g * W + e];
            const uint32_t key = key_of(x);
            const bool on = mode != kModeEmpty && (key > cut || (key == cut && i + e <= last));
            f[e] = on ? (x == m ? 0.f : (float)(((double)x - (double)m) * it)) : -INFINITY;
        }
        if (i + W <= p.V) {
#pragma unroll
            for (int e = 0; e < W; e += 4) {
                typedef float Any __attribute__((ext_vector_type(4), aligned(4)));
                Any q;
                __builtin_memcpy(&q, f + e, 16);
                __builtin_nontemporal_store(q, (Any*)(out + i + e));
            }
        } else {
#pragma unroll
            for (int e = 0; e < W; ++e)
                if (i + e < p.V) out[i + e] = f[e];
        }
    }
}

// Rows as sd_filter_logits writes them without options, z - max; rows of `own`
// (filtered already: their largest is 0) as they are.  Not-a-numbers stay.  A
// diagnostic's copy, one workgroup a row.
__global__ __launch_bounds__(1024) void k_shown_rows(const float* z, const int32_t* own, int V, float* out) {
    __shared__ float sm[16];
    const size_t at = (size_t)blockIdx.x * V;
    float m = -INFINITY;
    if (own[blockIdx.x]) {
        m = 0.f;
    } else {
        for (int i = threadIdx.x; i < V; i += 1024) m = fmaxf(m, clean(z[at + i]));
        m = wave_top(m);
        if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = m;
        __syncthreads();
        for (int i = 0; i < 16; ++i) m = fmaxf(m, sm[i]);
    }
    for (int i = threadIdx.x; i < V; i += 1024) {
        const float x = z[at + i];
        out[at + i] = x == -INFINITY ? x : x == m ? 0.f : (float)((double)x - (double)m);
    }
}

}  // namespace

void launch_shown_rows(int T, int V, const float* logits, const int32_t* own, float* out, hipStream_t s) {
    hipLaunchKernelGGL(k_shown_rows, dim3(T), dim3(1024), 0, s, logits, own, V, out);
}

size_t filter_workspace(int n_rows, int V) { return layout(n_rows, V, nullptr, nullptr); }
int filter_rows(size_t bytes, int V, int most) {
    if (filter_workspace(most, V) <= bytes) return most;
    // (each of the four sections is rounded up once)
    const size_t row = filter_workspace(256, V) / 256;
    int n = (int)std::min<size_t>(bytes / row + 1, most);
    while (n > 0 && filter_workspace(n, V) > bytes) --n;
    return n;
}

// ONLY: rows may be left alone (fp32 rows that are rewritten)
template <typename T, bool ONLY>
static void launch_typed(const FilterCall& c, const FilterP& p, hipStream_t s) {
    Work wk;
    layout(c.n_rows, c.V, c.ws, &wk);
    const int nch = chunks_of(c.V);
    const dim3 g(nch, c.n_rows), rows(c.n_rows), of_row(kRowThreads);
    hipLaunchKernelGGL((k_filter_scan<T, ONLY>), g, dim3(kChunkThreads), 0, s, p, wk);
    if (ONLY || c.out) {
        hipLaunchKernelGGL((k_filter_find<false, ONLY>), rows, dim3(kFindThreads), 0, s, p, wk, nch);
        hipLaunchKernelGGL((k_filter_collect<T, false, ONLY>), g, dim3(kChunkThreads), 0, s, p, wk);
        hipLaunchKernelGGL((k_filter_resolve<T, false, false, ONLY>), rows, of_row, 0, s, p, wk, nch);
        hipLaunchKernelGGL((k_filter_write<T, ONLY>), g, dim3(kChunkThreads), 0, s, p, wk);
        return;
    }
    if constexpr (!ONLY) {
        if (!c.topk && !c.topp && !c.minp) {
            hipLaunchKernelGGL((k_filter_resolve<T, true, true, false>), rows, of_row, 0, s, p, wk, nch);
        } else {
            hipLaunchKernelGGL((k_filter_find<true, false>), rows, dim3(kFindThreads), 0, s, p, wk, nch);
            hipLaunchKernelGGL((k_filter_collect<T, true, false>), g, dim3(kChunkThreads), 0, s, p, wk);
            hipLaunchKernelGGL((k_filter_resolve<T, true, false, false>), rows, of_row, 0, s, p, wk, nch);
        }
    }
}

void launch_filter(const FilterCall& c, hipStream_t s) {
    FilterP p{};
    p.z = c.logits; p.stride = c.stride; p.V = c.V;
    p.scale_bits = 62;
    while ((1ll << (62 - p.scale_bits)) < c.V) --p.scale_bits;
    p.temp = c.temp; p.topk = c.topk; p.topp = c.topp; p.minp = c.minp;
    p.u = c.u; p.token = c.token; p.prob = c.prob; p.kept = c.kept;
    p.out = c.out; p.ostride = c.ostride;
    p.only = c.only;
    if (c.only) launch_typed<float, true>(c, p, s);
    else if (c.bf16) launch_typed<bf16_t, false>(c, p, s);
    else launch_typed<float, false>(c, p, s);
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
