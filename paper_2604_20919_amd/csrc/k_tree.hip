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

}  // namespace

size_t tree_workspace(const TreeCall&) { return 256; }

void launch_tree_attention(const TreeCall& c, hipStream_t s) {
    const dim3 grid(c.hq, c.max_slots, c.n_users);
    if (c.kv.esize == 2) hipLaunchKernelGGL(k_tree_rows<bf16_t>, grid, dim3(256), 0, s, c);
    else hipLaunchKernelGGL(k_tree_rows<float>, grid, dim3(256), 0, s, c);
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
