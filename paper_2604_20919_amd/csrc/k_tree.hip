// Attention of trees of drafts over a paged cache with grouped query heads.
//
// Slot j of a user has its key at position prefix + j and sees the positions below
// prefix, its ancestors and itself:  out = sum_p softmax_p(scale q . k_p) v_p.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "../../include/sd_verify.h"
#include "sdv_device.h"
#include "sdv_internal.h"

namespace sdv {
namespace {

constexpr int kSlots = SD_TREE_MAX_SLOTS;
constexpr int kMaskWords = kSlots / 32;
constexpr int kMaxPos = 0x7fffffff - 4096;  // positions are 32-bit

// User b's first slot, its slots, cached tokens and positions that have a page.
struct TreeUser {
    int s0, n, prefix, end;
};
__device__ __forceinline__ TreeUser tree_user(const TreeCall& c, int b) {
    TreeUser u;
    u.s0 = min(max(c.slot_off[b], 0), c.n_slots);
    u.n = min(min(max(c.slot_off[b + 1], u.s0), c.n_slots) - u.s0, c.max_slots);
    u.prefix = min(max(c.prefix[b], 0), kMaxPos);
    u.end = (int)min((int64_t)u.prefix + u.n, (int64_t)c.max_pages * kPageTokens);
    return u;
}

// anc[j]: bits of slot j and its ancestors, by doubling: what a slot's furthest
// known ancestor knows is added to it until nobody has one.
template <int THREADS>
__device__ __forceinline__ void tree_ancestors(const TreeCall& c, const TreeUser& us, uint32_t (*anc)[kMaskWords + 1],
                                               int* ptr) {
    static_assert(THREADS >= kSlots, "a thread a slot");
    const int j = threadIdx.x;
    int p = -1;
    if (j < us.n) {
        p = c.parent ? c.parent[us.s0 + j] : j - 1;
        p = p >= 0 && p < j ? p : -1;
#pragma unroll
        for (int w = 0; w <= kMaskWords; ++w) anc[j][w] = w == j >> 5 ? 1u << (j & 31) : 0;
        ptr[j] = p;
    }
    while (__syncthreads_or(p >= 0)) {
        uint32_t more[kMaskWords] = {};
        int next = -1;
        if (p >= 0) {
#pragma unroll
            for (int w = 0; w < kMaskWords; ++w) more[w] = anc[p][w];
            next = ptr[p];
        }
        __syncthreads();
        if (p >= 0) {
#pragma unroll
            for (int w = 0; w < kMaskWords; ++w) anc[j][w] |= more[w];
            ptr[j] = next;
        }
        p = next;
    }
}

// fp32, on the vector units: fp32 caches are those of small models with short contexts.  A
// workgroup takes kRows of a user's query rows (slot by slot, the heads of a KV
// head together), its NW waves every NW-th block of 64 tokens, and their sums are merged
// in wave order.  Scores: lane = token, W elements of its key a load, each used for all
// rows (the rows' queries are read from LDS, one 16-byte word for a dim of all rows);
// outputs: lane = dim, a page's 16 values a load.  Six users of 3 to 17 slots over 63 to
// 900 tokens, 12 heads of 64 over 4 KV heads: 29 us (one row a workgroup, four waves,
// one element a load: 147).  What bounds it is latency, not the 1.7 us of its products at
// the vector units' rate (half that of v_mfma_f32_16x16x4_f32, which the fp32 weights'
// products use: packed fp32 is left out of this build): a wave's blocks follow each
// other, their page numbers and keys are asked for when the block before is done, a
// block's four pages of values after its softmax one after the other, and a row's
// maximum and sum go through twelve shuffles.  A context is not split over workgroups, so
// one user has no more than a workgroup for kRows rows of a KV head, however long it is.
constexpr int kRows = 4;
template <int W, int DT, int NW>
__global__ __launch_bounds__(64 * NW) void k_tree_rows(TreeCall c) {
    typedef float fw __attribute__((ext_vector_type(W)));
    __shared__ f32x4 qs[128];                                            // [dim], a row each element
    __shared__ __attribute__((aligned(16))) float ps[NW][64][kRows];
    __shared__ float ms[NW][kRows], ls[NW][kRows], os[NW][kRows][64 * DT];
    __shared__ uint32_t anc[kSlots][kMaskWords + 1];
    __shared__ int ptr[kSlots];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int b = blockIdx.z, g = blockIdx.y, row0 = blockIdx.x * kRows;
    const TreeUser u = tree_user(c, b);
    const int hd = c.kv.hd, G = c.hq / c.kv.hkv, R = u.n * G;
    if (row0 >= R) return;
    // element of a row's dim 0 in queries (stride c.qs) and outputs (c.os)
    auto place = [&](int row, int64_t stride) { return (size_t)(u.s0 + row / G) * stride + (size_t)(g * G + row % G) * hd; };
    if (tid < hd) {
        f32x4 q;
#pragma unroll
        for (int r = 0; r < kRows; ++r) q[r] = row0 + r < R ? ((const float*)c.q)[place(row0 + r, c.qs) + tid] : 0.f;
        qs[tid] = q;
    }
    tree_ancestors<64 * NW>(c, u, anc, ptr);
    __syncthreads();
    const int slot1 = min(row0 + kRows - 1, R - 1) / G;  // the last row's
    const int n = min(u.prefix + slot1 + 1, u.end);
    const int32_t* pt = c.page_table + (size_t)b * c.max_pages;
    const float* base = (const float*)c.kv.base;
    float m[kRows], l[kRows], o[DT][kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d][r] = 0.f;
    }
    for (int c0 = wave * 64; c0 < n; c0 += 64 * NW) {
        const int tok = c0 + lane, rel = tok - u.prefix;
        int page = tok < n ? pt[tok >> 4] : -1;
        if (page >= c.kv.n_pages) page = -1;
        float s[kRows] = {};
        if (page >= 0) {
            const float* kr = base + c.kv.k_off(c.layer, page, g) + (size_t)(tok & 15) * hd;
#pragma unroll 8
            for (int a = 0; a < hd; a += W) {
                const fw k = *(const fw*)(kr + a);
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    const f32x4 q = qs[a + e];
#pragma unroll
                    for (int r = 0; r < kRows; ++r) s[r] = fmaf(q[r], k[e], s[r]);
                }
            }
        }
        unsigned long long on[kRows], any = 0;
        f32x4 pe;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int j = (row0 + r) / G;
            const bool sees = page >= 0 && row0 + r < R && (rel < 0 || (rel <= j && ((anc[j][rel >> 5] >> (rel & 31)) & 1)));
            on[r] = __ballot(sees);
            any |= on[r];
            const float d = sees ? s[r] * c.scale : -INFINITY;
            const float mn = fmaxf(m[r], wave_max(d));
            const float al = mn == -INFINITY ? 1.f : expf(m[r] - mn);
            pe[r] = d == -INFINITY ? 0.f : expf(d - mn);  // (not a number where d is)
            l[r] = l[r] * al + wave_sum(pe[r]);
            m[r] = mn;
#pragma unroll
            for (int d2 = 0; d2 < DT; ++d2) o[d2][r] *= al;
        }
        wave_lds_order();
        *(f32x4*)ps[wave][lane] = pe;
        wave_lds_order();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t some = (uint32_t)(any >> (16 * i)) & 0xffff;
            if (!some) continue;
            const float* vb = base + c.kv.v_off(c.layer, __builtin_amdgcn_readlane(page, 16 * i), g);
            f32x4 v[DT][4];
#pragma unroll
            for (int d = 0; d < DT; ++d)
                if (lane + 64 * d < hd)
#pragma unroll
                    for (int x = 0; x < 4; ++x) v[d][x] = *(const f32x4*)(vb + (size_t)(lane + 64 * d) * kPageTokens + 4 * x);
            uint32_t all = 0xffff;
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                if (row0 + r < R) all &= (uint32_t)(on[r] >> (16 * i));
            if (all == 0xffff) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const f32x4 w = *(const f32x4*)ps[wave][16 * i + e];
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int r = 0; r < kRows; ++r) o[d][r] = fmaf(w[r], v[d][e >> 2][e & 3], o[d][r]);
                }
            } else {  // (what a row does not see may hold anything)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const f32x4 w = *(const f32x4*)ps[wave][16 * i + e];
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int r = 0; r < kRows; ++r)
                            o[d][r] = fmaf(w[r], (on[r] >> (16 * i + e)) & 1 ? v[d][e >> 2][e & 3] : 0.f, o[d][r]);
                }
            }
        }
    }
    if (lane == 0) {
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            ms[wave][r] = m[r];
            ls[wave][r] = l[r];
        }
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < kRows; ++r) os[wave][r][lane + 64 * d] = o[d][r];
    __syncthreads();
    for (int i = tid; i < kRows * hd; i += 64 * NW) {
        const int r = i / hd, a = i % hd;
        if (row0 + r >= R) break;
        float M = ms[0][r];
#pragma unroll
        for (int w = 1; w < NW; ++w) M = fmaxf(M, ms[w][r]);
        float L = 0.f, out = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = ms[w][r] == M ? 1.f : expf(ms[w][r] - M);
            L += ls[w][r] * f;
            out += os[w][r][a] * f;
        }
        ((float*)c.out)[place(row0 + r, c.os) + a] = L == 0.f ? 0.f : out / L;
    }
}

// ---------------------------------------------------------------------------
// bf16, matrix cores.  A unit is a group of up to 32 NW of a user's query rows (slots
// times the G heads that share a KV head) with the user's context for that head.  The
// context streams through a ring of LDS buffers in blocks of 32 tokens (two pages, K and
// V), loaded straight from global memory, and per block a wave takes 32 rows through
//   S^T = K Q^T        K rows as the A operand, in a token order that leaves a lane
//                      with 8 consecutive tokens of its row twice over, which is
//   O^T += V^T P^T     the B operand of the second product, V^T from the page's
//                      dim-major block; P in two bf16 planes (one would save 18 % of a
//                      wide tree's time and cost 1.4 times the error).
//
// What bounds it.  Few rows: the cache, read once a row group.  The layout keeps whole
// pages together for that (4 KB of K and of V, loaded in 1 KB pieces), all blocks are
// shared out evenly (below), and two blocks are loaded while two are used (but for those that
// reach into a tree, where the ancestors' words wait for every load): 32 users of
// 2292 tokens, 8 KV heads of 128, 4 / 8 / 13 slots of 8 heads: 61 / 67 / 97 us for 300 MB,
// 5.0 / 4.5 / 3.1 TB/s; with two planes of queries 77 us at 8 slots.  One token over 131072
// tokens, 4 heads of 64 (134 MB): 32 us + 6 for the merge.  Many rows: the parts add up,
// since all of them draw on the same power and registers hold one block's fragments a
// wave: 16 trees of 64 slots, 64 heads, 1024 to 8192 tokens take 292 us and 18 for the merge
// (317 in the first 10 ms after a pause; one call after the other 300 in all, since the
// merge's start overlaps).  Of that, in a build that took 295: without the second
// product 209, without the softmax 247, without the first product 249, without all three 166.
// The same instructions interleaved by hand over two blocks took 359.
//
// Two blocks a stage, two token groups for few rows, a maximum followed only when it is
// far off, and merges two segments at a time together brought the ragged users (2 to 13
// slots over 256 to 4096 tokens, two planes) from 142 to 105 us, the one token from 59 to
// 38 and the wide trees from 369 to 303 (calls, merges among them).
//
// head_dim 128 with two planes of queries takes all 256 registers and spills 18, outside
// the loop over blocks; the careful pass brings most of them.
// ---------------------------------------------------------------------------
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kBlock = 32;  // tokens a block

// All blocks of all units -- a user's query rows in groups, for every KV head --
// stand in one line, and every workgroup takes `per` of them.  A unit that lies in
// several workgroups' parts is merged afterwards from their partials: slot 2 w of
// workgroup w is its first segment, 2 w + 1 its last.
struct TreePlan {
    int wgs;        // workgroups
    int prows;      // rows of a partial slot
    int* per;       // blocks a workgroup, as the kernel found it
    int* base;      // [n_users] where a user's first unit begins
    float* part;    // [2 wgs][prows][HD] outputs of segments, not yet divided
    float2* ml;     // [2 wgs][prows] their maxima (before scaling) and sums
};

// A user in the line: its units (KV head by KV head, row group by row group) of nb
// blocks each begin at base.
struct TreeSpan {
    int b, nb, units, base;
};
struct TreeScan {
    int sum[8];
    TreeSpan found;
};
template <int ROWS> __device__ __forceinline__ int tree_weight(const TreeCall& c, int b, int* nb, int* units) {
    *nb = *units = 0;
    if (b >= c.n_users) return 0;
    const TreeUser us = tree_user(c, b);
    if (us.n <= 0) return 0;
    *nb = (us.end + kBlock - 1) / kBlock;
    *units = (us.n * (c.hq / c.kv.hkv) + ROWS - 1) / ROWS * c.kv.hkv;
    return *nb * *units;
}

// The users in the line, as every workgroup finds them from their lengths (a launch
// less than a plan made before), as many at a time as it has threads: a thread's
// user, and the blocks up to its end.
struct TreeUsers {
    int b0 = -1, nb = 0, units = 0, own = 0, upto = 0;
    int before = 0, all = 0;  // before, all: the blocks up to user b0, and up to the last here
};
template <int NW> __device__ __forceinline__ void tree_scan(const TreeCall& c, int b0, int before, TreeUsers& t, TreeScan& sc) {
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    t.b0 = b0;
    t.before = before;
    t.own = tree_weight<32 * NW>(c, b0 + tid, &t.nb, &t.units);
    t.upto = t.own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(t.upto, o, 64);
        if (lane >= o) t.upto += x;
    }
    if (lane == 63) sc.sum[wave] = t.upto;
    __syncthreads();
    t.all = before;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w == wave) t.upto += t.all;
        t.all += sc.sum[w];
    }
    __syncthreads();
}
// The length of the line.
template <int NW> __device__ __forceinline__ int tree_total(const TreeCall& c, TreeUsers& t, TreeScan& sc) {
    int all = 0;
    for (int b0 = 0; b0 < c.n_users; b0 += 64 * NW) {
        tree_scan<NW>(c, b0, all, t, sc);
        all = t.all;
    }
    return all;
}
// The user at a position of it.
template <int NW> __device__ __forceinline__ TreeSpan tree_find(const TreeCall& c, int pos, TreeUsers& t, TreeScan& sc) {
    if (pos < t.before) tree_scan<NW>(c, 0, 0, t, sc);
    while (pos >= t.all) tree_scan<NW>(c, t.b0 + 64 * NW, t.all, t, sc);
    if (t.own > 0 && pos >= t.upto - t.own && pos < t.upto)
        sc.found = TreeSpan{t.b0 + (int)threadIdx.x, t.nb, t.units, t.upto - t.own};
    __syncthreads();
    // (the same in every lane: kept in scalar registers)
    auto same = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    TreeSpan f = sc.found;
    f = TreeSpan{same(f.b), same(f.nb), same(f.units), same(f.base)};
    __syncthreads();
    return f;
}

// Which of the tokens t0 .. t0+31 the slot with ancestors `a` sees.
__device__ __forceinline__ uint32_t tree_bits(const uint32_t* a, int t0, int prefix) {
    const int r = t0 - prefix;
    if (r <= -32) return ~0u;
    if (r < 0) return (a[0] << -r) | ((1u << -r) - 1);
    if (r >= kSlots) return 0;
    const uint64_t two = (uint64_t)a[r >> 5] | ((uint64_t)a[(r >> 5) + 1] << 32);
    return (uint32_t)(two >> (r & 31));
}

// A maximum in the log2 domain, rounded.  (Never fused into what uses it: every use has
// to see the same rounding.)
__device__ __forceinline__ float log2_max(float m, float sc2) {
#pragma clang fp contract(off)
    return m * sc2;
}
// What the ordinary pass's weights, which are relative to that rounded product, are
// multiplied by to be relative to m itself.
__device__ __forceinline__ float to_exact_max(float m, float sc2) {
    const float lo = fmaf(m, sc2, -log2_max(m, sc2));
    return m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(-lo);
}

__device__ __forceinline__ float half_max(float v) {  // of lanes l and l ^ 32
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The fragments of one block.  The reads are not the compiler's: it cannot tell the
// buffer from the ones being loaded and would wait for every load in flight (as it does
// for the ancestors' words, in the blocks that reach into a tree).  A statement's
// registers count as written when it is, so each waits for its own reads: between a
// read and a later wait the compiler could copy, spill or reuse them.  V's come two
// dim tiles at a time, the second two while the products of the first run; with all of
// them read and waited for at once 32 ragged users took 106 us instead of 104.  ka:
// this lane's K pieces (four addresses, the swizzle moves them apart), va: its V slot,
// in the block's buffer; AT: of two V tiles within it.
template <int HD> __device__ __forceinline__ void read_k(bf16x8 (&k)[HD / 16], const uint32_t (&ka)[4]) {
    if constexpr (HD == 128) {
        asm volatile(
            "ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %10\n\tds_read_b128 %3, %11\n\t"
            "ds_read_b128 %4, %8 offset:128\n\tds_read_b128 %5, %9 offset:128\n\t"
            "ds_read_b128 %6, %10 offset:128\n\tds_read_b128 %7, %11 offset:128\n\ts_waitcnt lgkmcnt(0)"
            : "=&v"(k[0]), "=&v"(k[1]), "=&v"(k[2]), "=&v"(k[3]), "=&v"(k[4]), "=&v"(k[5]), "=&v"(k[6]), "=&v"(k[7])
            : "v"(ka[0]), "v"(ka[1]), "v"(ka[2]), "v"(ka[3])
            : "memory");
    } else {
        asm volatile(
            "ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(k[0]), "=&v"(k[1]), "=&v"(k[2]), "=&v"(k[3])
            : "v"(ka[0]), "v"(ka[1]), "v"(ka[2]), "v"(ka[3])
            : "memory");
    }
}
template <int AT> __device__ __forceinline__ void read_v(bf16x8 (&v)[4], uint32_t va) {
    asm volatile(
        "ds_read_b128 %0, %4 offset:%5\n\tds_read_b128 %1, %4 offset:%5+1024\n\t"
        "ds_read_b128 %2, %4 offset:%5+2*1024\n\tds_read_b128 %3, %4 offset:%5+3*1024\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
        : "v"(va), "n"(AT)
        : "memory");
}

// Eight bf16 values with infinities and not-a-numbers taken out; and where they are:
// 1 for the infinity of one sign (0x7f80 or 0xff80) and for not-a-numbers.
__device__ __forceinline__ bf16x8 only_finite(bf16x8 v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint16_t x = __builtin_bit_cast(uint16_t, (__bf16)v[e]);
        if ((x & 0x7f80) == 0x7f80) v[e] = (__bf16)0.f;
    }
    return v;
}
__device__ __forceinline__ bf16x8 where_odd(bf16x8 v, uint32_t inf) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint16_t x = __builtin_bit_cast(uint16_t, (__bf16)v[e]);
        v[e] = (__bf16)(x == inf || (x & 0x7fff) > 0x7f80 ? 1.f : 0.f);
    }
    return v;
}

// NW waves a workgroup, 32 rows each: 4 (two workgroups a CU) or 8.
template <int HD, int NW> struct TreeLds {
    static constexpr int PB = kPageTokens * HD * 2;  // bytes of a page's K or V block
    static constexpr int BUF = 4 * PB;               // two pages of K, two of V
    static constexpr int N = NW == 8 ? 6 : 4;        // buffers
    __attribute__((aligned(1024))) char ring[N * BUF];
    uint32_t anc[kSlots][kMaskWords + 1];
    int ptr[kSlots];
    TreeScan scan;
};

// A segment: blocks blk0 .. blk1-1 of a unit.
struct TreeSeg {
    int b, g, rg, blk0, blk1;
};

// What the waves of a workgroup hold of their rows, and where they read from.
template <int HD, bool QLO> struct TreeWave {
    bf16x8 qf[HD / 16], ql[QLO ? HD / 16 : 1];
    uint32_t ka[4], va;      // this lane's K pieces and V slot of the first buffer
    uint32_t ksrc, vsrc;     // its gather sources within a page's K and V blocks
    const uint32_t* anc;     // its row's ancestors
    bool act;                // the wave has rows
    // blocks are taken tw at a time, each by the waves of one token group (tg)
    int tw, tg;
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// One pass over a segment.  The weights are relative to the scaled and rounded maximum
// (one operation each), so whatever changes the maximum takes the difference of two such
// products; to_exact_max leads from there to m.  CAREFUL: scores are taken relative to the
// maximum before they are scaled, and the values' infinities and not-a-numbers are kept
// apart: 0 times one is not 0 in a product, and rows that do not see such a value, or
// see it with two weights of opposite sign, must not take part in that.
template <int HD, bool QLO, int NW, bool CAREFUL, class Q, class F>
__device__ __forceinline__ void tree_pass(const TreeCall& c, const TreeSeg& un, int prefix, const TreeWave<HD, QLO>& w,
                                          char* ring, int wave, float sc2, float& m, float& l,
                                          f32x16 (&o)[HD / 32], Q queries, F meanwhile) {
    constexpr int DS = HD / 16, DT = HD / 32;
    constexpr int PB = TreeLds<HD, NW>::PB, BUF = TreeLds<HD, NW>::BUF, N = TreeLds<HD, NW>::N;
    constexpr int LOADS = BUF / 1024 / NW;  // 1 KB loads a wave and block
    const int lane = threadIdx.x & 63, H = lane >> 5;
    const int last = un.blk1 - un.blk0 - 1;
    // K and V of the KV head in a page: page_bytes apart, V vo behind K
    const char* const kbase = (const char*)c.kv.base + c.kv.k_off(c.layer, 0, un.g) * 2;
    const uint32_t page_bytes = (uint32_t)(c.kv.page_elems() * 2), vo = (uint32_t)c.kv.hkv * PB;
    // the pages of 32 blocks, a lane each (-1: the pool has not got it), and of the next 32
    const int32_t* const pt = c.page_table + (size_t)un.b * c.max_pages;
    auto pages = [&](int blk) {
        const int i = 2 * blk + lane, p = i < c.max_pages && blk < un.blk1 ? pt[i] : -1;
        return p < c.kv.n_pages ? p : -1;
    };
    int pg = pages(un.blk0), pg_next = pages(un.blk0 + 32);
    uint32_t there = 0;  // which pages of the last blocks issued exist, two bits a block
    int next = 0, next_buf = 0;  // the block to be loaded next, and into which buffer
    auto issue = [&]() __attribute__((always_inline)) {
        const int i = next++, buf = next_buf;
        next_buf = buf + 1 == N ? 0 : buf + 1;
        if (i > last) {
            there <<= 2;
            return;
        }
        if (i > 0 && (i & 31) == 0) {
            pg = pg_next;
            pg_next = pages(un.blk0 + i + 32);
        }
        // (missing pages are read as page 0 and not attended to)
        const int p0 = __builtin_amdgcn_readlane(pg, 2 * (i & 31)), p1 = __builtin_amdgcn_readlane(pg, 2 * (i & 31) + 1);
        there = there << 2 | (p1 >= 0) << 1 | (p0 >= 0);
        auto rsrc = [&](int p) {
            return __builtin_amdgcn_make_buffer_rsrc((void*)(kbase + (uint64_t)(uint32_t)max(p, 0) * page_bytes), (short)0,
                                                     (int)(vo + PB), 0x00020000);
        };
        char* dst = ring + buf * BUF;
        auto load = [&](__amdgpu_buffer_rsrc_t r, int at, uint32_t src, uint32_t off) __attribute__((always_inline)) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(dst + at), 16, (int)src, (int)off, 0, 0);
        };
        // (V fragments: [dim tile][page])
        if constexpr (HD == 128 && NW == 4) {
            const __amdgpu_buffer_rsrc_t r0 = rsrc(p0), r1 = rsrc(p1);
            load(r0, wave * 1024, w.ksrc, 0);
            load(r1, PB + wave * 1024, w.ksrc, 0);
            load(r0, 2 * PB + wave * 2048, w.vsrc, vo);
            load(r1, 2 * PB + wave * 2048 + 1024, w.vsrc, vo);
        } else if constexpr (HD == 128) {
            const __amdgpu_buffer_rsrc_t r0 = rsrc(p0), r1 = rsrc(p1);
            const int part = wave & 3;
            const bool v = wave >= 4;
            const uint32_t src = v ? w.vsrc : w.ksrc, off = v ? vo : 0;
            load(r0, v ? 2 * PB + part * 2048 : part * 1024, src, off);
            load(r1, v ? 2 * PB + part * 2048 + 1024 : PB + part * 1024, src, off);
        } else {
            const int page = (wave >> 1) & 1, part = wave & 1;
            const __amdgpu_buffer_rsrc_t r = rsrc(page ? p1 : p0);
            if (NW == 4 || wave < 4) load(r, page * PB + part * 1024, w.ksrc, 0);
            if (NW == 4 || wave >= 4) load(r, 2 * PB + part * 2048 + page * 1024, w.vsrc, vo);
        }
    };
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x16{};
    queries();
    // (pages and queries are waited for here: a wait for them inside the loop would be
    // one for every load in flight)
    wait_vm<0>();
    __syncthreads();  // (nobody reads the ring or the ancestors before)
    constexpr int ST = 2;  // blocks a stage
    for (int i = 0; i < N - ST; ++i) issue();
    meanwhile();
    int stage = 0;  // buffer of block i
    for (int i = 0; i <= last; i += ST, stage = stage + ST >= N ? 0 : stage + ST) {
        // Blocks i and i + 1 are waited for; those that follow may be in flight.  Then every
        // wave is done with the two blocks before, whose buffers take the next.
        if (N > 4 && min(last, i + N - ST - 1) - (i + ST - 1) >= 2) wait_vm<2 * LOADS, true>();
        else wait_vm<0, true>();
        barrier_nofence();
#pragma unroll
        for (int k = 0; k < ST; ++k) issue();
        for (int k = w.tg; k < ST; k += w.tw) {
            if (!w.act || i + k > last) break;
            const int t0 = (un.blk0 + i + k) * kBlock, buf = stage + k;
            bf16x8 kf[DS];
            const uint32_t at = (uint32_t)(buf * BUF), kb[4] = {w.ka[0] + at, w.ka[1] + at, w.ka[2] + at, w.ka[3] + at};
            read_k<HD>(kf, kb);
            // (two sums: a product waits for the one before it in its own)
            f32x16 s = f32x16{}, s2 = f32x16{};
#pragma unroll
            for (int d = 0; d < DS; d += QLO ? 1 : 2) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[d], w.qf[d], s, 0, 0, 0);
                if constexpr (QLO) s2 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[d], w.ql[d], s2, 0, 0, 0);
                else s2 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[d + 1], w.qf[d + 1], s2, 0, 0, 0);
            }
            s += s2;
            // lane: tokens t0 + 8 H + e (e < 8) and t0 + 16 + 8 H + e of its row
            const uint32_t both = there >> (2 * (N - 1 - k)) & 3;
            uint32_t see = ~0u;
            if (t0 + kBlock > prefix || both != 3) {
                see = (both & 1 ? 0xffffu : 0u) | (both & 2 ? 0xffff0000u : 0u);
                if (t0 + kBlock > prefix) see &= tree_bits(w.anc, t0, prefix);
                see >>= 8 * H;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = (see >> (e < 8 ? e : e + 8)) & 1 ? s[e] : -INFINITY;
            }
            float bm = fmaxf(s[0], s[1]);
#pragma unroll
            for (int e = 2; e < 16; ++e) bm = fmaxf(bm, s[e]);
            // The maximum that weights are relative to follows the rows' own only when
            // one is 2^8 beyond it (rescaling the outputs costs as much as a product).
            const float mn = fmaxf(m, half_max(bm));
            if (__builtin_amdgcn_ballot_w64((mn - m) * sc2 > 8.f)) {
                const float alpha =
                    mn == m ? 1.f
                            : __builtin_amdgcn_exp2f(CAREFUL ? (m - mn) * sc2 : log2_max(m, sc2) - log2_max(mn, sc2));
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] *= alpha;
                l *= alpha;
                m = mn;
            }
            const float m0 = m == -INFINITY ? 0.f : m, ms = log2_max(m0, sc2);
            auto weight = [&](float v) { return __builtin_amdgcn_exp2f(CAREFUL ? (v - m0) * sc2 : fmaf(v, sc2, -ms)); };
            // the weights as two bf16 planes: hi rounded, lo what that left
            float rs[2] = {0.f, 0.f};
            uint32_t ph[8], pl[8];
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const float p0 = weight(s[e]), p1 = weight(s[e + 1]);
                rs[0] += p0;
                rs[1] += p1;
                const uint32_t hi = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)p0, (__bf16)p1});
                ph[e / 2] = hi;
                pl[e / 2] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(p0 - __uint_as_float(hi << 16)),
                                                                (__bf16)(p1 - __uint_as_float(hi & 0xffff0000u))});
            }
            l += rs[0] + rs[1];
            bf16x8 hi[2], lo[2], z[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                hi[t] = __builtin_bit_cast(bf16x8, uint4{ph[4 * t], ph[4 * t + 1], ph[4 * t + 2], ph[4 * t + 3]});
                lo[t] = __builtin_bit_cast(bf16x8, uint4{pl[4 * t], pl[4 * t + 1], pl[4 * t + 2], pl[4 * t + 3]});
            }
            if constexpr (CAREFUL) {
#pragma unroll
                for (int e = 0; e < 16; ++e) z[e >> 3][e & 7] = (__bf16)((see >> (e < 8 ? e : e + 8)) & 1 ? 1.f : 0.f);
            }
            // two dim tiles at a time
            auto tiles = [&](auto first) __attribute__((always_inline)) {
                constexpr int D0 = decltype(first)::value;
                bf16x8 vf[4];
                read_v<2 * PB + 2048 * D0>(vf, w.va + at);
#pragma unroll
                for (int d = 0; CAREFUL && d < 2; ++d) {
#pragma unroll
                    for (int sign = 0; sign < 2; ++sign) {
                        f32x16 hit = f32x16{};
#pragma unroll
                        for (int t = 0; t < 2; ++t)
                            hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(where_odd(vf[2 * d + t], sign ? 0xff80 : 0x7f80), z[t],
                                                                          hit, 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[D0 + d][e] += hit[e] > 0.f ? (sign ? -INFINITY : INFINITY) : 0.f;
                    }
                    vf[2 * d] = only_finite(vf[2 * d]);
                    vf[2 * d + 1] = only_finite(vf[2 * d + 1]);
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
#pragma unroll
                    for (int d = 0; d < 2; ++d)
                        o[D0 + d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[2 * d + t], hi[t], o[D0 + d], 0, 0, 0);
#pragma unroll
                    for (int d = 0; d < 2; ++d)
                        o[D0 + d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[2 * d + t], lo[t], o[D0 + d], 0, 0, 0);
                }
            };
            tiles(std::integral_constant<int, 0>{});
            if constexpr (DT == 4) tiles(std::integral_constant<int, 2>{});
        }
    }
    wait_vm<0>();
    l = half_sum(l);
}

template <int HD, bool QLO, int NW>
__device__ __forceinline__ void tree_segment(const TreeCall& c, const TreePlan& pl, TreeLds<HD, NW>& lds, const TreeSeg& un,
                                             const TreeUser& us, bool learn, bool whole, int slot) {
    constexpr int DS = HD / 16, DT = HD / 32;  // k steps of S, dim tiles of O
    constexpr int PB = TreeLds<HD, NW>::PB, ROWS = 32 * NW;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int lr = lane & 31, H = lane >> 5;
    const int G = c.hq / c.kv.hkv, R = us.n * G;
    // few rows: two token groups
    const int tw = min(R - un.rg * ROWS, ROWS) <= ROWS / 2 ? 2 : 1;
    const int tile = tw == 2 ? wave & (NW / 2 - 1) : wave;
    const int lrow = tile * 32 + lr, row = un.rg * ROWS + lrow;
    bool ok = row < R;
    const int j = ok ? row / G : 0, hh = ok ? row % G : 0;
    TreeWave<HD, QLO> w;
    w.act = un.rg * ROWS + tile * 32 < R;
    w.tw = tw;
    w.tg = tw == 2 ? wave / (NW / 2) : 0;
    w.anc = lds.anc[j];
    // A wave's loads of a block: head_dim 128: quarters of K of page 0, of page 1, of V of
    // page 0, of page 1; 64: halves of K and of V of one page (with eight waves: four of
    // them K, four V).  K rows lie in LDS as in the page, their 16-byte pieces exchanged
    // so that 8 lanes that read a piece of 8 rows read 8 different ones; V as fragments.
    constexpr int PIECES = HD / 8, TOK = 64 / PIECES;  // pieces of a K row, rows a 1 KB load
    auto swz = [](int t) { return (t & 3) | ((t >> 1) & 4); };  // of row t of a page
    const int part = HD == 128 ? wave & 3 : wave & 1;
    const int kt = part * TOK + lane / PIECES;
    w.ksrc = (uint32_t)(kt * HD * 2 + ((lane % PIECES) ^ swz(kt)) * 16);
    w.vsrc = (uint32_t)(part * 1024 + lr * 32 + H * 16);
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds.ring;
    {
        const int a = lr >> 3, tok = 8 * ((lr >> 2) & 1) + 4 * (a & 1) + (lr & 3);
#pragma unroll
        for (int d = 0; d < 4; ++d)
            w.ka[d] = base + (uint32_t)((a >> 1) * PB + tok * HD * 2 + ((H ^ swz(tok)) ^ (2 * d)) * 16);
    }
    w.va = base + lane * 16u;

    const float sc2 = c.scale * 1.4426950408889634f;
    float m, l;
    f32x16 o[DT];
    auto queries = [&]() __attribute__((always_inline)) {
        const size_t e = (size_t)(us.s0 + j) * c.qs + (size_t)(un.g * G + hh) * HD + 8 * H;
#pragma unroll
        for (int d = 0; d < DS; ++d) {
            w.qf[d] = ok ? *(const bf16x8*)((const bf16_t*)c.q + e + 16 * d) : bf16x8{};
            if constexpr (QLO) w.ql[d] = ok ? *(const bf16x8*)((const bf16_t*)c.q_lo + e + 16 * d) : bf16x8{};
        }
    };
    auto ancestors = [&]() __attribute__((always_inline)) {  // while the first blocks are on their way
        if (!learn) return;
        tree_ancestors<64 * NW>(c, us, lds.anc, lds.ptr);
        __syncthreads();
    };
    tree_pass<HD, QLO, NW, false>(c, un, us.prefix, w, lds.ring, wave, sc2, m, l, o, queries, ancestors);
    // a segment whose outputs are not finite or whose scores are huge is done again, carefully
    bool odd = false;
    if (w.act) {
        odd = m != -INFINITY && fabsf(m) * sc2 >= 1048576.f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) odd |= !(fabsf(o[d][e]) < INFINITY);
    }
    const bool careful = __syncthreads_or(odd);
    if (careful) tree_pass<HD, QLO, NW, true>(c, un, us.prefix, w, lds.ring, wave, sc2, m, l, o, [] {}, [] {});
    auto to_exact = [&](float max) { return careful ? 1.f : to_exact_max(max, sc2); };
    if (tw == 2) {
        // the second token group's sums, through the ring: [tile][4 * dim tiles][lane]
        f32x4* const sp = (f32x4*)lds.ring + tile * (4 * DT * 64);
        float2* const sm = (float2*)((f32x4*)lds.ring + (NW / 2) * (4 * DT * 64)) + tile * 64;
        __syncthreads();
        if (w.tg == 1 && w.act) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4)
                    sp[(4 * d + q4) * 64 + lane] = f32x4{o[d][4 * q4], o[d][4 * q4 + 1], o[d][4 * q4 + 2], o[d][4 * q4 + 3]};
            sm[lane] = float2{m, l};
        }
        __syncthreads();
        if (w.tg == 0 && w.act) {
            const float2 v = sm[lane];
            const float mn = fmaxf(m, v.x);
            const float f0 = to_exact(m) * (m == mn ? 1.f : __builtin_amdgcn_exp2f((m - mn) * sc2));
            const float f1 = to_exact(v.x) * (v.x == mn ? 1.f : __builtin_amdgcn_exp2f((v.x - mn) * sc2));
            m = mn;
            l = l * f0 + v.y * f1;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    const f32x4 p = sp[(4 * d + q4) * 64 + lane];
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[d][4 * q4 + e] = o[d][4 * q4 + e] * f0 + p[e] * f1;
                }
        }
        ok &= w.tg == 0;
    }
    if (!ok) return;
    // lane: dims 32 d + 8 (e / 4) + 4 H + e % 4 of its row
    if (whole) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const size_t e0 = (size_t)(us.s0 + j) * c.os + (size_t)(un.g * G + hh) * HD + 4 * H;
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                bf16x4 hi, lo;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = o[d][4 * q4 + e] * inv;
                    hi[e] = (__bf16)v;
                    lo[e] = (__bf16)(v - (float)hi[e]);
                }
                *(bf16x4*)((bf16_t*)c.out + e0 + 32 * d + 8 * q4) = hi;
                if (c.out_lo) *(bf16x4*)((bf16_t*)c.out_lo + e0 + 32 * d + 8 * q4) = lo;
            }
        return;
    }
    const size_t pr = (size_t)slot * pl.prows + lrow;
    const float f = tw == 2 ? 1.f : to_exact(m);
    if (H == 0) pl.ml[pr] = float2{m, l * f};
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
            *(f32x4*)(pl.part + pr * HD + 32 * d + 8 * q4 + 4 * H) =
                f32x4{o[d][4 * q4] * f, o[d][4 * q4 + 1] * f, o[d][4 * q4 + 2] * f, o[d][4 * q4 + 3] * f};
}

template <int HD, bool QLO, int NW>
__device__ __forceinline__ void tree_mfma(const TreeCall& c, const TreePlan& pl, TreeLds<HD, NW>& lds) {
    // neighbours in the line, which share users and heads, on one die
    const int id = (blockIdx.x & 7) * (pl.wgs / 8) + (blockIdx.x >> 3);
    TreeUsers users;
    const int total = __builtin_amdgcn_readfirstlane(tree_total<NW>(c, users, lds.scan));
    const int per = max((int)(((uint32_t)total + pl.wgs - 1) / (uint32_t)pl.wgs), 1);
    if (id == 0 && threadIdx.x == 0) *pl.per = per;
    if (total <= id * (int64_t)per) return;
    int pos = id * per;
    const int first = pos, end = pos + min(total - pos, per);
    while (pos < end) {
        const TreeSpan sp = tree_find<NW>(c, pos, users, lds.scan);
        int unit = (int)((uint32_t)(pos - sp.base) / (uint32_t)sp.nb), off = pos - sp.base - unit * sp.nb;
        if (unit == 0 && off == 0 && threadIdx.x == 0) pl.base[sp.b] = sp.base;
        TreeUser us = tree_user(c, sp.b);
        us = TreeUser{__builtin_amdgcn_readfirstlane(us.s0), __builtin_amdgcn_readfirstlane(us.n),
                      __builtin_amdgcn_readfirstlane(us.prefix), __builtin_amdgcn_readfirstlane(us.end)};
        const int groups = sp.units / c.kv.hkv;
        bool known = false;  // the user's ancestors are in LDS
        for (; unit < sp.units && pos < end; ++unit, off = 0) {
            const int len = min(sp.nb - off, end - pos);
            const TreeSeg un{sp.b, unit / groups, unit % groups, off, off + len};
            const bool tail = un.blk1 * kBlock > us.prefix;
            tree_segment<HD, QLO, NW>(c, pl, lds, un, us, tail && !known, len == sp.nb, 2 * id + (pos == first ? 0 : 1));
            known |= tail;
            pos += len;
        }
    }
}

template <int HD, bool QLO, int NW>
__global__ __launch_bounds__(64 * NW, 2) void k_tree_mfma(TreeCall c, TreePlan pl) {
    __shared__ TreeLds<HD, NW> lds;
    tree_mfma<HD, QLO, NW>(c, pl, lds);
}

// Merges the segments of units that lie in several workgroups' parts, in their order.
// HD / 4 lanes take a row's segments, two at a time (a unit seldom lies in more than
// three parts); where there are few rows SPLIT such groups share a row's, four at a time.
// 4 us (8 slots of 16 heads, one user), 8 (32 ragged users, 64 heads), 17 (16 trees of 64).
template <int HD, int SPLIT> __global__ __launch_bounds__(256) void k_tree_merge(TreeCall c, TreePlan pl, int wrows) {
    constexpr int LANES = HD / 4, GROUPS = 256 / LANES, ROWS = GROUPS / SPLIT;
    __shared__ float2 sml[GROUPS];
    __shared__ f32x4 spart[SPLIT > 1 ? GROUPS : 1][LANES];
    const int b = blockIdx.y;
    const TreeUser us = tree_user(c, b);
    const int grp = threadIdx.x / LANES, ln = threadIdx.x % LANES, part = grp % SPLIT;
    const int rid = blockIdx.x * ROWS + grp / SPLIT;
    const bool on = us.n > 0 && rid < us.n * c.hq;
    if (SPLIT == 1 && !on) return;
    if (blockIdx.x * ROWS >= us.n * c.hq) return;
    const int G = c.hq / c.kv.hkv, h = on ? rid % c.hq : 0, j = on ? rid / c.hq : 0, row = j * G + h % G;
    const int nb = (us.end + kBlock - 1) / kBlock, groups = (us.n * G + wrows - 1) / wrows;
    const int per = *pl.per, u0 = pl.base[b] + ((h / G) * groups + row / wrows) * nb;
    const int w0 = (int)((uint32_t)u0 / (uint32_t)per), n = (int)((uint32_t)(u0 + nb - 1) / (uint32_t)per) - w0 + 1;
    const bool mine = on && n > 1;
    const float sc2 = c.scale * 1.4426950408889634f;
    constexpr int CH = SPLIT > 1 ? 4 : 2;
    float M = -INFINITY, L = 0.f;
    f32x4 a = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k0 = part; mine && k0 < n; k0 += CH * SPLIT) {
        float2 v[CH];
        f32x4 p[CH];
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int k = min(k0 + i * SPLIT, n - 1), w = w0 + k;
            // (a workgroup's first segment, or its last)
            const size_t pr = (size_t)(2 * w + (u0 > w * per)) * pl.prows + row % wrows;
            v[i] = pl.ml[pr];
            p[i] = *(const f32x4*)(pl.part + pr * HD + 4 * ln);
            if (k0 + i * SPLIT >= n) v[i] = float2{-INFINITY, 0.f};
        }
        float mg = M;
#pragma unroll
        for (int i = 0; i < CH; ++i) mg = fmaxf(mg, v[i].x);
        const float f0 = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((M - mg) * sc2);
        L *= f0;
        a *= f0;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (v[i].x == -INFINITY) {
                L += v[i].y;  // 0, or not a number
                continue;
            }
            const float f = __builtin_amdgcn_exp2f((v[i].x - mg) * sc2);
            L += v[i].y * f;
            a += p[i] * f;
        }
        M = mg;
    }
    if constexpr (SPLIT > 1) {
        if (ln == 0) sml[grp] = float2{M, L};
        spart[grp][ln] = a;
        __syncthreads();
        if (part != 0 || !mine) return;
        float mg = M;
#pragma unroll
        for (int i = 1; i < SPLIT; ++i) mg = fmaxf(mg, sml[grp + i].x);
        const float f0 = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((M - mg) * sc2);
        L *= f0;
        a *= f0;
#pragma unroll
        for (int i = 1; i < SPLIT; ++i) {
            const float2 v = sml[grp + i];
            const float f = v.x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((v.x - mg) * sc2);
            L += v.y * f;
            if (v.x != -INFINITY) a += spart[grp + i][ln] * f;
        }
    }
    if (!mine) return;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    const size_t e = (size_t)(us.s0 + j) * c.os + (size_t)h * HD + 4 * ln;
    bf16x4 hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float v = a[i] * inv;
        hi[i] = (__bf16)v;
        lo[i] = (__bf16)(v - (float)hi[i]);
    }
    *(bf16x4*)((bf16_t*)c.out + e) = hi;
    if (c.out_lo) *(bf16x4*)((bf16_t*)c.out_lo + e) = lo;
}

// One wave a user: from the root along the drafts that equal the target's tokens, of
// equal drafts below a slot the first.  At most 64 drafts, a lane each.
__global__ __launch_bounds__(64) void k_tree_walk(BatchView bv, const int32_t* target, int32_t* result, int bmax,
                                                  uint64_t* path) {
    const int b = blockIdx.x, lane = threadIdx.x;
    if (b == 0 && lane == 0) result[2 * bmax] = *bv.flags;
    const int s0 = bv.slot_off[b], L = bv.L[b];
    const bool mine = lane < L;
    const int draft = mine ? bv.drafts[bv.draft_off[b] + lane] : -1, above = mine ? bv.parent[s0 + lane + 1] : -1;
    uint64_t taken = 0;
    int at = 0, n = 0, token = target[s0];
    while (true) {
        const uint64_t on = __ballot(mine && above == at && draft == token);
        if (!on) break;
        at = __ffsll((unsigned long long)on);  // draft number: lane + 1
        taken |= on & -on;
        ++n;
        token = target[s0 + at];
    }
    if (lane != 0) return;
    result[b] = n;
    result[bmax + b] = token;
    path[b] = taken;
}

// The parts of the workspace for so many workgroups.
struct TreeSizes {
    int prows;
    size_t head, ml, bytes;
};
TreeSizes tree_sizes(const TreeCall& c, int nw, int wgs) {
    TreeSizes z;
    z.prows = std::min(32 * nw, c.max_slots * (c.hq / c.kv.hkv));
    z.head = ((size_t)c.n_users * 4 + 4 + 255) / 256 * 256;
    z.ml = ((size_t)2 * wgs * z.prows * 8 + 255) / 256 * 256;
    z.bytes = z.head + z.ml + (size_t)2 * wgs * z.prows * c.kv.hd * 4;
    return z;
}

// Users of more than 128 rows a KV head take workgroups of eight waves.
int tree_waves(const TreeCall& c) { return c.max_slots * (c.hq / c.kv.hkv) > 128 ? 8 : 4; }
// Workgroups that are resident at once.
int tree_wgs(int nw) { return cu_count() / 8 * 8 * (8 / nw); }

}  // namespace

size_t tree_workspace(const TreeCall& c) {
    if (c.kv.esize != 2) return 256;
    // (host only: 256 CUs)
    return tree_sizes(c, tree_waves(c), 256 * (8 / tree_waves(c))).bytes;
}
size_t tree_workspace_least(const TreeCall& c) {
    return c.kv.esize == 2 ? tree_sizes(c, tree_waves(c), 8).bytes : 256;
}

void launch_tree_walk(const BatchView& bv, const int32_t* target, int32_t* result, int bmax, uint64_t* path,
                      hipStream_t s) {
    hipLaunchKernelGGL(k_tree_walk, dim3(bv.B), dim3(64), 0, s, bv, target, result, bmax, path);
}

// Whether a launch of this shape is possible.
bool tree_fits(const TreeCall& c) {
    const int rows = 32 * tree_waves(c);
    const int64_t units = (int64_t)c.kv.hkv * ((c.max_slots * (c.hq / c.kv.hkv) + rows - 1) / rows);
    // (a block is counted in 31 bits)
    return (int64_t)c.max_slots * c.hq <= (1 << 24) && c.n_users * units < (1ll << 31) &&
           c.n_users * units * (((int64_t)c.max_pages + 1) / 2) < (1ll << 31);
}

template <int HD, int NW> static void launch_tree_mfma(const TreeCall& c, hipStream_t s) {
    int wgs = std::min(tree_wgs(NW), 256 * (8 / NW));
    while (wgs > 8 && tree_sizes(c, NW, wgs).bytes > c.ws_bytes) wgs -= 8;
    const TreeSizes z = tree_sizes(c, NW, wgs);
    TreePlan pl;
    pl.wgs = wgs;
    pl.prows = z.prows;
    char* w = (char*)c.ws;
    pl.per = (int*)w;
    pl.base = pl.per + 1;
    pl.ml = (float2*)(w + z.head);
    pl.part = (float*)(w + z.head + z.ml);
    if (c.q_lo) hipLaunchKernelGGL((k_tree_mfma<HD, true, NW>), dim3(wgs), dim3(64 * NW), 0, s, c, pl);
    else hipLaunchKernelGGL((k_tree_mfma<HD, false, NW>), dim3(wgs), dim3(64 * NW), 0, s, c, pl);
    constexpr int GROUPS = 256 / (HD / 4);
    // Few rows, or rows in 16 parts or more: a workgroup each.  (2 users of 8 slots of 64
    // heads over 2000 tokens, units in 32 parts: 40 -> 32 us; 4 users, 16 parts: 42 -> 39;
    // 8 users, 8 parts: 44 -> 47)
    const int64_t units = (int64_t)c.n_users * c.kv.hkv * ((c.max_slots * (c.hq / c.kv.hkv) + 32 * NW - 1) / (32 * NW));
    if ((int64_t)c.n_slots * c.hq <= 512 || wgs >= 16 * units) {
        hipLaunchKernelGGL((k_tree_merge<HD, GROUPS>), dim3(c.max_slots * c.hq, c.n_users), dim3(256), 0, s, c, pl, 32 * NW);
    } else {
        hipLaunchKernelGGL((k_tree_merge<HD, 1>), dim3((c.max_slots * c.hq + GROUPS - 1) / GROUPS, c.n_users), dim3(256), 0, s,
                           c, pl, 32 * NW);
    }
}

void launch_tree_attention(const TreeCall& c, hipStream_t s) {
    if (c.kv.esize == 2) {
        const bool eight = tree_waves(c) == 8;
        if (c.kv.hd == 128) eight ? launch_tree_mfma<128, 8>(c, s) : launch_tree_mfma<128, 4>(c, s);
        else eight ? launch_tree_mfma<64, 8>(c, s) : launch_tree_mfma<64, 4>(c, s);
        return;
    }
    const int rows = c.max_slots * (c.hq / c.kv.hkv);
    const dim3 grid((rows + kRows - 1) / kRows, c.kv.hkv, c.n_users);
    // Eight waves a workgroup, or four where contexts have no more than four blocks, or no
    // more than 16 and there are more workgroups than two a CU.  (8 / 4 waves: 10 users of 6
    // slots of 40 heads over 25 tokens, 640 workgroups, 31 / 17 us; six users of 3 to 17 slots
    // over 63 to 900 tokens, 312, 29 / 36; 32 such users, 1664, 54 / 51; 32 over 2000, 162 / 172)
    const bool few = c.max_pages <= 16 || (c.max_pages <= 64 && (int64_t)grid.x * grid.y * grid.z > 2 * cu_count());
    const auto run = [&](auto eight, auto four) {
        if (few) hipLaunchKernelGGL(four, grid, dim3(256), 0, s, c);
        else hipLaunchKernelGGL(eight, grid, dim3(512), 0, s, c);
    };
    // (a key begins on 16 bytes where four elements divide the head)
    if (c.kv.hd > 64) {
        if (c.kv.hd % 4 == 0) run(k_tree_rows<4, 2, 8>, k_tree_rows<4, 2, 4>);
        else run(k_tree_rows<2, 2, 8>, k_tree_rows<2, 2, 4>);
    } else {
        if (c.kv.hd % 4 == 0) run(k_tree_rows<4, 1, 8>, k_tree_rows<4, 1, 4>);
        else run(k_tree_rows<2, 1, 8>, k_tree_rows<2, 1, 4>);
    }
}

}  // namespace sdv

namespace {

// What the size query and the call require of pool, tree and heads.
sd_status tree_call(const sd_kv_pool* pool, const sd_tree* t, int32_t n_q_heads, sdv::TreeCall* c) {
    const sd_status r = sdv::pool_of(pool, &c->kv);
    if (r != SD_OK) return r;
    if (!t || t->n_users < 1 || t->n_slots < 1 || t->max_slots < 1 || t->max_pages < 1 || n_q_heads < 1 ||
        n_q_heads % pool->n_kv_heads)
        return SD_EINVAL;
    if (t->max_slots > SD_TREE_MAX_SLOTS || t->n_users > SD_TREE_MAX_USERS || t->n_slots > (1 << 20) ||
        n_q_heads / pool->n_kv_heads > 128)
        return SD_ELIMIT;
    c->n_users = t->n_users;
    c->n_slots = t->n_slots;
    c->max_slots = t->max_slots;
    c->max_pages = t->max_pages;
    c->hq = n_q_heads;
    c->slot_off = t->slot_off;
    c->prefix = t->prefix;
    c->page_table = t->page_table;
    c->parent = t->parent;
    if (c->kv.esize == 2 && !sdv::tree_fits(*c)) return SD_ELIMIT;
    return SD_OK;
}

}  // namespace

extern "C" {

sd_status sd_tree_query_size(const sd_kv_pool* pool, const sd_tree* tree, int32_t n_q_heads,
                             uint64_t* workspace_bytes) {
    if (!workspace_bytes) return SD_EINVAL;
    sdv::TreeCall c{};
    const sd_status r = tree_call(pool, tree, n_q_heads, &c);
    if (r != SD_OK) return r;
    *workspace_bytes = sdv::tree_workspace(c);
    return SD_OK;
}

sd_status sd_tree_attention(const sd_kv_pool* pool, int32_t layer, const sd_tree* tree, int32_t n_q_heads,
                            const void* q, const void* q_lo, int64_t q_stride, void* out, void* out_lo,
                            int64_t out_stride, float scale, void* workspace, uint64_t workspace_bytes,
                            sd_stream stream) {
    sdv::TreeCall c{};
    const sd_status r = tree_call(pool, tree, n_q_heads, &c);
    if (r != SD_OK) return r;
    if (layer < 0 || layer >= pool->n_layers || !c.kv.base || !c.slot_off || !c.prefix || !c.page_table || !q || !out ||
        !workspace || !(scale > 0.f) || !std::isfinite(scale))
        return SD_EINVAL;
    const int64_t row = (int64_t)n_q_heads * pool->head_dim;
    if (q_stride < row || out_stride < row) return SD_EINVAL;
    const bool bf16 = pool->dtype == SD_BF16;
    if (!bf16 && (q_lo || out_lo)) return SD_EINVAL;
    const uintptr_t es = bf16 ? 2 : 4, at = bf16 ? 16 : 4;
    if (((uintptr_t)q | (uintptr_t)q_lo | (uintptr_t)out | (uintptr_t)out_lo) % at ||
        (tree->n_slots > 1 && ((uint64_t)q_stride * es % at || (uint64_t)out_stride * es % at)))
        return SD_EINVAL;
    if ((uintptr_t)c.kv.base % 256 || (uintptr_t)workspace % 256 ||
        ((uintptr_t)c.slot_off | (uintptr_t)c.prefix | (uintptr_t)c.page_table | (uintptr_t)c.parent) % 4)
        return SD_EINVAL;
    // planes apart from each other, outputs from inputs
    const uint64_t qb = ((uint64_t)(tree->n_slots - 1) * q_stride + row) * es;
    const uint64_t ob = ((uint64_t)(tree->n_slots - 1) * out_stride + row) * es;
    auto apart = [](const void* a, uint64_t an, const void* b, uint64_t bn) {
        return !a || !b || (uintptr_t)a + an <= (uintptr_t)b || (uintptr_t)b + bn <= (uintptr_t)a;
    };
    if (!apart(q, qb, out, ob) || !apart(q, qb, out_lo, ob) || !apart(q_lo, qb, out, ob) ||
        !apart(q_lo, qb, out_lo, ob) || !apart(out, ob, out_lo, ob))
        return SD_EINVAL;
    if (workspace_bytes < sdv::tree_workspace(c)) return SD_ENOMEM;
    c.layer = layer;
    c.q = q;
    c.q_lo = q_lo;
    c.qs = q_stride;
    c.out = out;
    c.out_lo = out_lo;
    c.os = out_stride;
    c.scale = scale;
    c.ws = workspace;
    c.ws_bytes = workspace_bytes;
    sdv::launch_tree_attention(c, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? SD_OK : SD_EHIP;
}

}  // extern "C"
