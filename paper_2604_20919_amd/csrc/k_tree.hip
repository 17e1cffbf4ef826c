// Attention of trees of drafts over a paged cache with grouped query heads.
//
// Slot j of a user has its key at position prefix + j and sees the positions below
// prefix, its ancestors and itself:  out = sum_p softmax_p(scale q . k_p) v_p.
#include <algorithm>
#include <cmath>

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

// One workgroup per (user, slot, query head); its waves take every fourth block of 64
// tokens and are merged in wave order.  Scores: lane = token; outputs: lane = dim.
template <typename T>
__global__ __launch_bounds__(256) void k_tree_rows(TreeCall c) {
    __shared__ float qs[128];
    __shared__ int par[kSlots];
    __shared__ uint32_t anc[kMaskWords];
    __shared__ float ps[4][64];
    __shared__ float ms[4], ls[4], os[4][128];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int h = blockIdx.x, j = blockIdx.y, b = blockIdx.z;
    const TreeUser u = tree_user(c, b);
    if (j >= u.n) return;
    const int hd = c.kv.hd, g = h / (c.hq / c.kv.hkv);
    const size_t t = u.s0 + j;
    if (tid < kMaskWords) anc[tid] = 0;
    if (tid <= j) {
        const int p = c.parent ? c.parent[u.s0 + tid] : tid - 1;
        par[tid] = p < tid ? p : -1;
    }
    if (tid < hd) {
        const size_t e = t * c.qs + (size_t)h * hd + tid;
        qs[tid] = ld<T>((const T*)c.q, e) + (c.q_lo ? ld<T>((const T*)c.q_lo, e) : 0.f);
    }
    __syncthreads();
    if (tid == 0)
        for (int a = j; a >= 0; a = par[a]) anc[a >> 5] |= 1u << (a & 31);
    __syncthreads();
    const int n = min(u.prefix + j + 1, u.end);
    const int32_t* pt = c.page_table + (size_t)b * c.max_pages;
    const T* base = (const T*)c.kv.base;
    float m = -INFINITY, l = 0.f, a0 = 0.f, a1 = 0.f;
    for (int c0 = wave * 64; c0 < n; c0 += 256) {
        const int tok = c0 + lane, r = tok - u.prefix;
        float d = -INFINITY;
        const int page = tok < n ? pt[tok >> 4] : -1;
        const bool sees = page >= 0 && page < c.kv.n_pages && (r < 0 || ((anc[r >> 5] >> (r & 31)) & 1));
        if (sees) {
            const T* kr = base + c.kv.k_off(c.layer, page, g) + (size_t)(tok & 15) * hd;
            float s = 0.f;
            for (int a = 0; a < hd; ++a) s = fmaf(qs[a], ld<T>(kr, a), s);
            d = s * c.scale;
        }
        const float mn = fmaxf(m, wave_max(d));
        const float al = mn == -INFINITY ? 1.f : expf(m - mn), pe = sees ? expf(d - mn) : 0.f;
        l = l * al + wave_sum(pe);
        m = mn;
        a0 *= al;
        a1 *= al;
        const unsigned long long on = __ballot(sees);
        wave_lds_order();
        ps[wave][lane] = pe;
        wave_lds_order();
        for (int p = 0; p < 64; ++p) {
            if (!((on >> p) & 1)) continue;  // (what a row does not see may hold anything)
            const T* vb = base + c.kv.v_off(c.layer, pt[(c0 + p) >> 4], g) + (p & 15);
            const float w = ps[wave][p];
            if (lane < hd) a0 = fmaf(w, ld<T>(vb, (size_t)lane * kPageTokens), a0);
            if (lane + 64 < hd) a1 = fmaf(w, ld<T>(vb, (size_t)(lane + 64) * kPageTokens), a1);
        }
    }
    if (lane == 0) {
        ms[wave] = m;
        ls[wave] = l;
    }
    os[wave][lane] = a0;
    os[wave][lane + 64] = a1;
    __syncthreads();
    if (tid >= hd) return;
    const float M = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3]));
    float L = 0.f, o = 0.f;
    for (int w = 0; w < 4; ++w) {
        if (ms[w] == -INFINITY) continue;
        const float f = expf(ms[w] - M);
        L += ls[w] * f;
        o += os[w][tid] * f;
    }
    const size_t e = t * c.os + (size_t)h * hd + tid;
    const float v = M == -INFINITY ? 0.f : o / L;
    if constexpr (sizeof(T) == 2) {
        const __bf16 hi = (__bf16)v;
        ((__bf16*)c.out)[e] = hi;
        if (c.out_lo) ((__bf16*)c.out_lo)[e] = (__bf16)(v - (float)hi);
    } else {
        ((float*)c.out)[e] = v;
    }
}


// ---------------------------------------------------------------------------
// bf16, matrix cores.  A workgroup takes one unit -- a chunk of one user's context
// for one KV head -- and up to 128 of the user's query rows (slots times the G
// heads that share the KV head), a wave 32 of them.  The chunk streams through a
// ring of LDS buffers in blocks of 32 tokens (two pages, K and V), loaded straight
// from global memory, and per block
//   S^T = K Q^T        K rows as the A operand, in a token order that leaves a lane
//                      with 8 consecutive tokens of its row twice over, which is
//   O^T += V^T P^T     the B operand of the second product, V^T from the page's
//                      dim-major block; P in two bf16 planes.
// ---------------------------------------------------------------------------
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(4))) const int32_t cint32_t;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kRows = 128;   // query rows a workgroup
constexpr int kBlock = 32;   // tokens a block
constexpr int kBuffers = 3;  // LDS ring
constexpr int kResident = 2; // workgroups a CU

struct TreePlan {
    int cap;       // units times row groups aimed at
    int groups;    // row groups of the widest user
    int units;     // most units
    float* part;   // [rows][HD] outputs of chunks, not yet divided
    float2* ml;    // [rows] their maxima (log2 domain) and sums
    int2* table;   // [n_users] chunks, first row of the partials
};

// What one workgroup does: user, head, its chunk of blocks, its partials' first row.
struct TreeUnit {
    int b, g, chunk, chunks, blk0, blk1, row0;
};

// The unit of number u: users in order, a user's chunks in order, heads.  Every
// workgroup works this out for itself from the users' lengths (a launch less than a
// plan made before).  A chunk has as many blocks as leave all units times row
// groups within `cap`, evened out within a user.
__device__ __forceinline__ bool tree_unit(const TreeCall& c, const TreePlan& pl, int u, TreeUnit* out) {
    __shared__ int64_t wsum[4];
    __shared__ int wu[4], wr[4];
    __shared__ TreeUnit found;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, G = c.hq / c.kv.hkv;
    auto blocks_of = [&](int b, int* rows) {
        const TreeUser us = tree_user(c, b);
        *rows = us.n * G;
        return us.n > 0 ? (us.end + kBlock - 1) / kBlock : 0;
    };
    int64_t total = 0;
    int rows = 0;
    for (int b = tid; b < c.n_users; b += 256) {
        const int nb = blocks_of(b, &rows);
        total += (int64_t)nb * ((rows + kRows - 1) / kRows);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o, 64);
    if (lane == 0) wsum[wave] = total;
    if (tid == 0) found.b = -1;
    __syncthreads();
    total = (wsum[0] + wsum[1] + wsum[2] + wsum[3]) * c.kv.hkv;
    const int len = (int)min(max((total + pl.cap - 1) / pl.cap, (int64_t)1), (int64_t)1 << 30);
    int u0 = 0, r0 = 0;  // units and partial rows of the users before
    for (int b0 = 0; b0 < c.n_users; b0 += 256) {
        const int b = b0 + tid;
        const int nb = b < c.n_users ? blocks_of(b, &rows) : 0;
        const int nc = (nb + len - 1) / len;
        int su = nc, sr = nc > 1 ? nc * rows : 0;  // inclusive sums over the users
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(su, o, 64), y = __shfl_up(sr, o, 64);
            if (lane >= o) { su += x; sr += y; }
        }
        if (lane == 63) { wu[wave] = su; wr[wave] = sr; }
        __syncthreads();
        for (int w = 0; w < 4; ++w) {
            if (w < wave) { su += wu[w]; sr += wr[w]; }
        }
        const int first = (u0 + su - nc) * c.kv.hkv;
        if (nc > 0 && u >= first && u < first + nc * c.kv.hkv) {
            const int k = (u - first) / c.kv.hkv, each = (nb + nc - 1) / nc;
            found.b = b;
            found.g = (u - first) % c.kv.hkv;
            found.chunk = k;
            found.chunks = nc;
            found.blk0 = min(nb, k * each);
            found.blk1 = min(nb, (k + 1) * each);
            found.row0 = (r0 + sr - (nc > 1 ? nc * rows : 0)) * c.kv.hkv;
        }
        u0 += wu[0] + wu[1] + wu[2] + wu[3];
        r0 += wr[0] + wr[1] + wr[2] + wr[3];
        __syncthreads();
        if (found.b >= 0) break;
    }
    // (the same in every lane: kept in scalar registers)
    auto same = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    *out = TreeUnit{same(found.b), same(found.g), same(found.chunk), same(found.chunks),
                    same(found.blk0), same(found.blk1), same(found.row0)};
    return out->b >= 0;
}

// anc[j]: bits of slot j and its ancestors, by doubling: what a slot's furthest
// known ancestor knows is added to it until nobody has one.
__device__ __forceinline__ void tree_ancestors(const TreeCall& c, const TreeUser& us, uint32_t (*anc)[kMaskWords + 1],
                                               int* ptr) {
    const int j = threadIdx.x;
    int p = -1;
    if (j < us.n) {
        p = c.parent ? c.parent[us.s0 + j] : j - 1;
        p = p >= 0 && p < j ? p : -1;
#pragma unroll
        for (int w = 0; w <= kMaskWords; ++w) anc[j][w] = w == j >> 5 ? 1u << (j & 31) : 0;
    }
    ptr[j] = p;
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
        }
        p = next;
        ptr[j] = p;
    }
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

__device__ __forceinline__ float half_max(float v) {  // of lanes l and l ^ 32
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The fragments of one block, K's waited for and V's on their way.  The reads are
// not the compiler's: it cannot tell the buffer from the ones being loaded and
// would wait for every load in flight.  ka: this lane's K pieces (four addresses, the
// swizzle moves them apart), va: its V slot, in the block's buffer.
template <int HD>
__device__ __forceinline__ void read_block(bf16x8 (&k)[HD / 16], bf16x8 (&v)[HD / 16], const uint32_t (&ka)[4], uint32_t va) {
    if constexpr (HD == 128) {
        asm volatile(
            "ds_read_b128 %0, %16 offset:%21\n\tds_read_b128 %1, %17 offset:%21\n\t"
            "ds_read_b128 %2, %18 offset:%21\n\tds_read_b128 %3, %19 offset:%21\n\t"
            "ds_read_b128 %4, %16 offset:%22\n\tds_read_b128 %5, %17 offset:%22\n\t"
            "ds_read_b128 %6, %18 offset:%22\n\tds_read_b128 %7, %19 offset:%22\n\t"
            "ds_read_b128 %8, %20 offset:%23\n\tds_read_b128 %9, %20 offset:%24\n\t"
            "ds_read_b128 %10, %20 offset:%25\n\tds_read_b128 %11, %20 offset:%26\n\t"
            "ds_read_b128 %12, %20 offset:%27\n\tds_read_b128 %13, %20 offset:%28\n\t"
            "ds_read_b128 %14, %20 offset:%29\n\tds_read_b128 %15, %20 offset:%30\n\t"
            "s_waitcnt lgkmcnt(8)"
            : "=&v"(k[0]), "=&v"(k[1]), "=&v"(k[2]), "=&v"(k[3]), "=&v"(k[4]), "=&v"(k[5]), "=&v"(k[6]), "=&v"(k[7]),
              "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
            : "v"(ka[0]), "v"(ka[1]), "v"(ka[2]), "v"(ka[3]), "v"(va), "n"(0), "n"(128), "n"(8192),
              "n"(9216), "n"(10240), "n"(11264), "n"(12288), "n"(13312), "n"(14336),
              "n"(15360)
            : "memory");
    } else {
        asm volatile(
            "ds_read_b128 %0, %8 offset:%13\n\tds_read_b128 %1, %9 offset:%13\n\t"
            "ds_read_b128 %2, %10 offset:%13\n\tds_read_b128 %3, %11 offset:%13\n\t"
            "ds_read_b128 %4, %12 offset:%14\n\tds_read_b128 %5, %12 offset:%15\n\t"
            "ds_read_b128 %6, %12 offset:%16\n\tds_read_b128 %7, %12 offset:%17\n\t"
            "s_waitcnt lgkmcnt(4)"
            : "=&v"(k[0]), "=&v"(k[1]), "=&v"(k[2]), "=&v"(k[3]), "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
            : "v"(ka[0]), "v"(ka[1]), "v"(ka[2]), "v"(ka[3]), "v"(va), "n"(0), "n"(4096), "n"(5120),
              "n"(6144), "n"(7168)
            : "memory");
    }
}
template <int N> __device__ __forceinline__ void wait_v(bf16x8 (&v)[N]) {
    if constexpr (N == 8)
        asm volatile("s_waitcnt lgkmcnt(0)"
                     : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]), "+v"(v[4]), "+v"(v[5]), "+v"(v[6]), "+v"(v[7]));
    else
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]));
}

// Eight bf16 values: infinities and not-a-numbers taken out (fin), and where they
// were: 1 in up for +inf and not-a-numbers, in down for -inf and not-a-numbers.
__device__ __forceinline__ void split_odd(const bf16x8& v, bf16x8& fin, bf16x8& up, bf16x8& down) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint16_t x = __builtin_bit_cast(uint16_t, (__bf16)v[e]);
        const bool odd = (x & 0x7f80) == 0x7f80, nan = odd && (x & 0x7f);
        fin[e] = odd ? (__bf16)0.f : v[e];
        up[e] = (__bf16)(nan || (odd && !(x >> 15)) ? 1.f : 0.f);
        down[e] = (__bf16)(nan || (odd && (x >> 15)) ? 1.f : 0.f);
    }
}

template <int HD> struct TreeLds {
    static constexpr int PB = kPageTokens * HD * 2;  // bytes of a page's K or V block
    static constexpr int BUF = 4 * PB;               // two pages of K, two of V
    __attribute__((aligned(1024))) char ring[kBuffers * BUF];
    uint32_t anc[kSlots][kMaskWords + 1];
    int ptr[kSlots];
};

template <int HD, bool QLO>
__device__ __forceinline__ void tree_mfma(const TreeCall& c, const TreePlan& pl, TreeLds<HD>& lds) {
    constexpr int DS = HD / 16, DT = HD / 32;  // k steps of S, dim tiles of O
    constexpr int PB = TreeLds<HD>::PB, BUF = TreeLds<HD>::BUF;
    constexpr int LOADS = BUF / 4096;          // 1 KB loads a wave and block
    char* const ring = lds.ring;
    auto& anc = lds.anc;
    auto& ptr = lds.ptr;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int lr = lane & 31, H = lane >> 5;
    // workgroups that share a chunk (row groups) on one die, one after the other
    const int x = blockIdx.x & 7, k = blockIdx.x >> 3, rg = k % pl.groups, u = (k / pl.groups) * 8 + x;
    TreeUnit un;
    if (!tree_unit(c, pl, u, &un)) return;
    TreeUser us = tree_user(c, un.b);
    us = TreeUser{__builtin_amdgcn_readfirstlane(us.s0), __builtin_amdgcn_readfirstlane(us.n),
                  __builtin_amdgcn_readfirstlane(us.prefix), __builtin_amdgcn_readfirstlane(us.end)};
    const int G = c.hq / c.kv.hkv, R = us.n * G;
    if (rg * kRows >= R) return;
    if (un.g == 0 && un.chunk == 0 && rg == 0 && tid == 0) pl.table[un.b] = int2{un.chunks, un.row0};
    if (un.blk1 * kBlock > us.prefix) tree_ancestors(c, us, anc, ptr);
    const cint32_t* pt = (const cint32_t*)(c.page_table + (size_t)un.b * c.max_pages);
    const int row = rg * kRows + wave * 32 + lr;
    const bool act = rg * kRows + wave * 32 < R, ok = row < R;
    const int j = ok ? row / G : 0, hh = ok ? row % G : 0;
    bf16x8 qf[DS], ql[QLO ? DS : 1];
    {
        const size_t e = (size_t)(us.s0 + j) * c.qs + (size_t)(un.g * G + hh) * HD + 8 * H;
#pragma unroll
        for (int d = 0; d < DS; ++d) {
            qf[d] = ok ? *(const bf16x8*)((const bf16_t*)c.q + e + 16 * d) : bf16x8{};
            if constexpr (QLO) ql[d] = ok ? *(const bf16x8*)((const bf16_t*)c.q_lo + e + 16 * d) : bf16x8{};
        }
    }
    // this lane's gather sources within a page's K and V blocks, and what it reads of a buffer
    constexpr int PIECES = HD / 8, TOK = 64 / PIECES;  // 16-byte pieces of a K row, rows a 1 KB load
    auto swz = [](int t) { return (t & 3) | ((t >> 1) & 4); };  // of token t of a page
    // load i of a wave (hd 128: K page 0, K page 1, V page 0, V page 1, a quarter each; hd 64:
    // K, V, half a page each)
    const int part = HD == 128 ? wave : wave & 1;
    const int kt = part * TOK + lane / PIECES;
    const uint32_t ksrc = (uint32_t)(kt * HD * 2 + ((lane % PIECES) ^ swz(kt)) * 16);
    const uint32_t vsrc = (uint32_t)(part * 1024 + lr * 32 + H * 16);
    uint32_t ka[4];
    {
        const int a = lr >> 3, tok = 8 * ((lr >> 2) & 1) + 4 * (a & 1) + (lr & 3);
        const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)ring;
#pragma unroll
        for (int d = 0; d < 4; ++d)
            ka[d] = base + (uint32_t)((a >> 1) * PB + tok * HD * 2 + ((H ^ swz(tok)) ^ (2 * d)) * 16);
    }
    const uint32_t va = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)ring + lane * 16u;

    auto page_at = [&](int i) { return i < c.max_pages ? pt[i] : -1; };
    auto in_pool = [&](int p) { return p >= 0 && p < c.kv.n_pages; };
    auto issue = [&](int p0, int p1, int buf) __attribute__((always_inline)) {
        // (pages that the pool has not got are read as page 0 and not attended to)
        p0 = in_pool(p0) ? p0 : 0;
        p1 = in_pool(p1) ? p1 : 0;
        const char* base = (const char*)c.kv.base;
        auto rsrc = [&](size_t elems) {
            return __builtin_amdgcn_make_buffer_rsrc((void*)(base + elems * 2), (short)0, PB, 0x00020000);
        };
        char* dst = ring + buf * BUF;
        if constexpr (HD == 128) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(c.kv.k_off(c.layer, p0, un.g)), (lds_void*)(dst + wave * 1024), 16, (int)ksrc, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(c.kv.k_off(c.layer, p1, un.g)), (lds_void*)(dst + PB + wave * 1024), 16, (int)ksrc, 0, 0, 0);
            // V fragments [dim tile][page]
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(c.kv.v_off(c.layer, p0, un.g)), (lds_void*)(dst + 2 * PB + wave * 2048), 16, (int)vsrc, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(c.kv.v_off(c.layer, p1, un.g)), (lds_void*)(dst + 2 * PB + wave * 2048 + 1024), 16, (int)vsrc, 0, 0, 0);
        } else {
            const int pg = wave >> 1, p = pg ? p1 : p0;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(c.kv.k_off(c.layer, p, un.g)), (lds_void*)(dst + pg * PB + part * 1024), 16, (int)ksrc, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(c.kv.v_off(c.layer, p, un.g)), (lds_void*)(dst + 2 * PB + part * 2048 + pg * 1024), 16, (int)vsrc, 0, 0, 0);
        }
    };

    const float sc2 = c.scale * 1.4426950408889634f;
    float m, l;
    f32x16 o[DT];
    // A chunk whose outputs are not finite is done again with the values' infinities
    // and not-a-numbers apart: 0 times one is not 0 in a product, and rows that do
    // not see such a value, or see it with two weights of opposite sign, must not
    // take part in that.
    for (int careful = 0; careful < 2; ++careful) {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = f32x16{};
        const int nblk = un.blk1 - un.blk0, last = nblk - 1;
        constexpr int PD = kBuffers - 1;
        __syncthreads();  // (the ring is free, the ancestors are there)
        wait_vm<0>();
        int np0 = 0, np1 = 0;  // pages of the block to be loaded next
#pragma unroll
        for (int i = 0; i < PD; ++i) {
            const int blk = un.blk0 + min(i, last);
            issue(page_at(2 * blk), page_at(2 * blk + 1), i);
        }
        np0 = page_at(2 * (un.blk0 + min(PD, last)));
        np1 = page_at(2 * (un.blk0 + min(PD, last)) + 1);
        auto block = [&](int BI, int i) __attribute__((always_inline)) {
            const int blk = un.blk0 + i, t0 = blk * kBlock;
            if (i + PD <= last) {
                wait_vm<LOADS * (PD - 1), true>();
                barrier_nofence();
                issue(np0, np1, (BI + PD) % kBuffers);
                const int nx = un.blk0 + min(i + PD + 1, last);
                np0 = page_at(2 * nx);
                np1 = page_at(2 * nx + 1);
            } else {
                if (last - i >= 1) wait_vm<LOADS, true>();
                else wait_vm<0, true>();
                barrier_nofence();
            }
            if (!act) return;
            bf16x8 kf[DS], vf[DS];
            const uint32_t at = (uint32_t)(BI * BUF), kb[4] = {ka[0] + at, ka[1] + at, ka[2] + at, ka[3] + at};
            read_block<HD>(kf, vf, kb, va + at);
            f32x16 s = f32x16{};
#pragma unroll
            for (int d = 0; d < DS; ++d) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[d], qf[d], s, 0, 0, 0);
                if constexpr (QLO) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[d], ql[d], s, 0, 0, 0);
            }
            // lane: tokens t0 + 8 H + e (e < 8) and t0 + 16 + 8 H + e of its row
            uint32_t see = ~0u;
            const bool all = t0 + kBlock <= us.prefix && in_pool(page_at(2 * blk)) && in_pool(page_at(2 * blk + 1));
            if (!all) {
                see = (in_pool(page_at(2 * blk)) ? 0xffffu : 0u) | (in_pool(page_at(2 * blk + 1)) ? 0xffff0000u : 0u);
                if (t0 + kBlock > us.prefix) see &= tree_bits(anc[j], t0, us.prefix);
                see >>= 8 * H;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = (see >> (e < 8 ? e : e + 8)) & 1 ? s[e] : -INFINITY;
            }
            float bm = fmaxf(s[0], s[1]);
#pragma unroll
            for (int e = 2; e < 16; ++e) bm = fmaxf(bm, s[e]);
            const float mn = fmaxf(m, half_max(bm));
            const bool live = mn != -INFINITY;
            const float ms = live ? mn * sc2 : 0.f;
            const float alpha = live ? __builtin_amdgcn_exp2f((m - mn) * sc2) : 1.f;
            float rs = 0.f;
            bf16x8 ph[2], plo[2];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float pe = __builtin_amdgcn_exp2f(fmaf(s[e], sc2, -ms));
                rs += pe;
                ph[e >> 3][e & 7] = (__bf16)pe;
                plo[e >> 3][e & 7] = (__bf16)(pe - (float)ph[e >> 3][e & 7]);
            }
            l = fmaf(l, alpha, rs);
            m = mn;
            if (__builtin_amdgcn_ballot_w64(alpha != 1.f)) {
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] *= alpha;
            }
            wait_v(vf);
            if (careful) {
                bf16x8 z[2];
#pragma unroll
                for (int e = 0; e < 16; ++e) z[e >> 3][e & 7] = (__bf16)((see >> (e < 8 ? e : e + 8)) & 1 ? 1.f : 0.f);
                if (all) z[0] = z[1] = bf16x8{1, 1, 1, 1, 1, 1, 1, 1};
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    f32x16 up = f32x16{}, down = f32x16{};
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        bf16x8 fin, fu, fd;
                        split_odd(vf[2 * d + t], fin, fu, fd);
                        vf[2 * d + t] = fin;
                        up = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fu, z[t], up, 0, 0, 0);
                        down = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fd, z[t], down, 0, 0, 0);
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        o[d][e] += (up[e] > 0.f ? INFINITY : 0.f) + (down[e] > 0.f ? -INFINITY : 0.f);
                }
            }
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[2 * d + t], ph[t], o[d], 0, 0, 0);
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[2 * d + t], plo[t], o[d], 0, 0, 0);
                }
        };
        for (int i0 = 0; i0 < nblk; i0 += kBuffers) {
            block(0, i0);
            if (i0 + 1 < nblk) block(1, i0 + 1);
            if (i0 + 2 < nblk) block(2, i0 + 2);
        }
        wait_vm<0>();
        l = half_sum(l);
        if (careful) break;
        bool odd = false;
        if (act) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) odd |= !(fabsf(o[d][e]) < INFINITY);
        }
        if (!__syncthreads_or(odd)) break;
    }
    if (!ok) return;
    // lane: dims 32 d + 8 (e / 4) + 4 H + e % 4 of its row
    if (un.chunks == 1) {
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
    const size_t pr = un.row0 + ((size_t)un.chunk * c.kv.hkv + un.g) * R + row;
    if (H == 0) pl.ml[pr] = float2{m == -INFINITY ? -INFINITY : m * sc2, l};
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
            *(f32x4*)(pl.part + pr * HD + 32 * d + 8 * q4 + 4 * H) =
                f32x4{o[d][4 * q4], o[d][4 * q4 + 1], o[d][4 * q4 + 2], o[d][4 * q4 + 3]};
}

template <int HD, bool QLO>
__global__ __launch_bounds__(256, kResident) void k_tree_mfma(TreeCall c, TreePlan pl) {
    __shared__ TreeLds<HD> lds;
    tree_mfma<HD, QLO>(c, pl, lds);
}

// Merges the chunks of a user's rows in chunk order; HD / 4 lanes a row.
template <int HD> __global__ __launch_bounds__(256) void k_tree_merge(TreeCall c, TreePlan pl) {
    constexpr int LANES = HD / 4, ROWS = 256 / LANES;
    const int b = blockIdx.y;
    const TreeUser us = tree_user(c, b);
    const int rid = blockIdx.x * ROWS + threadIdx.x / LANES, ln = threadIdx.x % LANES;
    if (us.n == 0 || rid >= us.n * c.hq) return;
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    const size_t e = (size_t)(us.s0 + rid / c.hq) * c.os + (size_t)(rid % c.hq) * HD + 4 * ln;
    if (us.end == 0) {  // no position has a page: no unit either
        *(bf16x4*)((bf16_t*)c.out + e) = bf16x4{};
        if (c.out_lo) *(bf16x4*)((bf16_t*)c.out_lo + e) = bf16x4{};
        return;
    }
    const int2 tb = pl.table[b];
    if (tb.x <= 1) return;
    const int G = c.hq / c.kv.hkv, R = us.n * G, h = rid % c.hq, row = rid / c.hq * G + h % G;
    float M = -INFINITY, L = 0.f;
    f32x4 a = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < tb.x; k0 += 8) {
        float2 v[8];
        f32x4 p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const size_t pr = tb.y + ((size_t)min(k0 + i, tb.x - 1) * c.kv.hkv + h / G) * R + row;
            v[i] = pl.ml[pr];
            p[i] = *(const f32x4*)(pl.part + pr * HD + 4 * ln);
            if (k0 + i >= tb.x) v[i].x = -INFINITY;
        }
        float mg = M;
#pragma unroll
        for (int i = 0; i < 8; ++i) mg = fmaxf(mg, v[i].x);
        if (mg == -INFINITY) {
            // nothing seen so far -- or scores that are not numbers, which show in the sums
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k0 + i < tb.x) L += v[i].y;
            continue;
        }
        const float f0 = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M - mg);
        L *= f0;
        a *= f0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (k0 + i >= tb.x) continue;
            if (v[i].x == -INFINITY) {
                L += v[i].y;
                continue;
            }
            const float f = __builtin_amdgcn_exp2f(v[i].x - mg);
            L += v[i].y * f;
            a += p[i] * f;
        }
        M = mg;
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
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

// The plan's sizes: units times row groups aimed at, and the workspace it takes.
struct TreeSizes {
    int cap, groups, units, rows;  // rows: partial rows
    size_t bytes;
};
TreeSizes tree_sizes(const TreeCall& c, int cap) {
    TreeSizes z;
    const int G = c.hq / c.kv.hkv;
    z.cap = cap;
    z.groups = (c.max_slots * G + kRows - 1) / kRows;
    const int64_t least = (int64_t)c.n_users * c.kv.hkv;  // one unit a user and head
    z.units = (int)std::min<int64_t>(cap + least, INT32_MAX);
    // a unit has one row group's rows for each of its row groups, at most
    const int64_t rows = (cap + least * z.groups) * std::min(kRows, c.max_slots * G);
    z.rows = (int)std::min<int64_t>(rows, INT32_MAX);
    z.bytes = ((size_t)c.n_users * 8 + 255) / 256 * 256 + ((size_t)rows * 8 + 255) / 256 * 256 + (size_t)rows * c.kv.hd * 4;
    return z;
}

}  // namespace

// Workgroups that are resident at once; fewer where the workspace is smaller.
constexpr int kTreeCap = 256 * kResident;

size_t tree_workspace(const TreeCall& c) {
    if (c.kv.esize != 2) return 256;
    return tree_sizes(c, kTreeCap).bytes;
}

size_t tree_workspace_least(const TreeCall& c) { return c.kv.esize == 2 ? tree_sizes(c, 1).bytes : 256; }

void launch_tree_walk(const BatchView& bv, const int32_t* target, int32_t* result, int bmax, uint64_t* path,
                      hipStream_t s) {
    hipLaunchKernelGGL(k_tree_walk, dim3(bv.B), dim3(64), 0, s, bv, target, result, bmax, path);
}

// Whether a launch of this shape is possible.
bool tree_fits(const TreeCall& c) {
    const TreeSizes z = tree_sizes(c, kTreeCap);
    return (int64_t)z.units * z.groups <= (1 << 23) && z.rows < INT32_MAX && (int64_t)c.max_slots * c.hq <= (1 << 24);
}

template <int HD> static void launch_tree_mfma(const TreeCall& c, hipStream_t s) {
    int cap = kTreeCap;
    while (cap > 1 && tree_sizes(c, cap).bytes > c.ws_bytes) cap /= 2;
    const TreeSizes z = tree_sizes(c, cap);
    TreePlan pl;
    pl.cap = cap;
    pl.groups = z.groups;
    pl.units = z.units;
    char* w = (char*)c.ws;
    pl.table = (int2*)w;
    w += ((size_t)c.n_users * 8 + 255) / 256 * 256;
    pl.ml = (float2*)w;
    w += ((size_t)z.rows * 8 + 255) / 256 * 256;
    pl.part = (float*)w;
    const dim3 grid((z.units + 7) / 8 * 8 * z.groups);
    if (c.q_lo) hipLaunchKernelGGL((k_tree_mfma<HD, true>), grid, dim3(256), 0, s, c, pl);
    else hipLaunchKernelGGL((k_tree_mfma<HD, false>), grid, dim3(256), 0, s, c, pl);
    constexpr int ROWS = 256 / (HD / 4);
    hipLaunchKernelGGL(k_tree_merge<HD>, dim3((c.max_slots * c.hq + ROWS - 1) / ROWS, c.n_users), dim3(256), 0, s, c, pl);
}

void launch_tree_attention(const TreeCall& c, hipStream_t s) {
    if (c.kv.esize == 2) {
        if (c.kv.hd == 128) launch_tree_mfma<128>(c, s);
        else launch_tree_mfma<64>(c, s);
        return;
    }
    hipLaunchKernelGGL(k_tree_rows<float>, dim3(c.hq, c.max_slots, c.n_users), dim3(256), 0, s, c);
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
