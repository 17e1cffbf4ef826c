// Pages of a paged cache: copied in every layer (a user forked), and rows moved
// together inside a user's pages (the accepted path of a tree of drafts).
#include <algorithm>

#include "../../include/sd_verify.h"
#include "sdv_device.h"
#include "sdv_internal.h"

namespace sdv {
namespace {

// A copy is bound by memory: every page read once and written once.  A workgroup copies
// 4 KB of one page of one layer, 16 bytes a thread, and the stores go past the cache (a
// user's copy is not read by what follows it at once).  80 pages of 64 KB in 64 layers
// (2 x 335 MB) take 110 us, 6.1 TB/s; with cached stores 114, with 8 or 16 KB a workgroup
// 123 to 135, and three pages in 28 layers 17 us instead of 6.6.
constexpr int kCopyPiece = 4096;

template <class Ids>
__global__ __launch_bounds__(256) void k_copy_pages(char* base, int n_pages, uint32_t page_bytes, int pieces, Ids ids) {
    const uint32_t i = blockIdx.x / (uint32_t)pieces, piece = blockIdx.x % (uint32_t)pieces, layer = blockIdx.y;
    const int src = ids.src[i], dst = ids.dst[i];
    if (src < 0 || src >= n_pages || dst < 0 || dst >= n_pages) return;
    const char* from = base + ((size_t)layer * n_pages + src) * page_bytes;
    char* to = base + ((size_t)layer * n_pages + dst) * page_bytes;
    const uint32_t o = piece * kCopyPiece + threadIdx.x * 16;
    if (o < page_bytes) __builtin_nontemporal_store(*(const f32x4*)(from + o), (f32x4*)(to + o));
}

struct DeviceIds {
    const int32_t *src, *dst;
};

template <class Ids> void copy_pages(const KVPool& kv, int layers, int n, const Ids& ids, hipStream_t s) {
    const uint32_t bytes = (uint32_t)(kv.page_elems() * kv.esize);
    const int pieces = (int)((bytes + kCopyPiece - 1) / kCopyPiece);
    hipLaunchKernelGGL(k_copy_pages<Ids>, dim3((uint32_t)n * pieces, layers), dim3(256), 0, s, (char*)kv.base, kv.n_pages,
                       bytes, pieces, ids);
}

// One workgroup moves the rows of one user, layer, KV head and slice of dims: all
// into LDS, then all out, so the order and overlap of the rows do not matter.  Bound by
// V: a row is a column of its block and each element lies in a 32-byte sector of its
// own, so a row's V costs a whole 4 KB block at the source and one at the target, sixteen
// times its size.  32 users' paths of up to 8 rows in 64 layers of 8 heads of 128: 69 us,
// where the sectors alone take about 57 at a copy's rate; one user's three rows in 28
// layers 7.3 us, a launch and two dependent round trips.
template <typename T>
__global__ __launch_bounds__(256) void k_compact(CompactCall c, int dw, int slices) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ int src[SD_KV_COMPACT_MAX], dst[SD_KV_COMPACT_MAX];
    const int sl = blockIdx.x % slices, g = blockIdx.x / slices, layer = blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x;
    const int n = c.path ? __popcll(c.path[b]) + 1 : min(max(c.n_keep[b], 0), c.max_keep);
    const int64_t p0 = max(c.prefix[b], 0);
    const int32_t* pt = c.page_table + (size_t)b * c.max_pages;
    bool mine = false;
    if (tid < n) {
        int k = tid;
        if (c.path) {
            if (tid > 0) {
                uint64_t m = c.path[b];
                for (int i = 1; i < tid; ++i) m &= m - 1;
                k = __ffsll((unsigned long long)m);
            }
        } else {
            k = c.keep[(size_t)b * c.max_keep + tid];
        }
        auto place = [&](int64_t p) -> int {
            if (p >= (int64_t)c.max_pages * kPageTokens) return -1;
            const int page = pt[p / kPageTokens];
            return page < 0 || page >= c.kv.n_pages ? -1 : page * kPageTokens + (int)(p % kPageTokens);
        };
        const int from = k < 0 || k == tid ? -1 : place(p0 + k), to = place(p0 + tid);
        mine = from >= 0 && to >= 0;
        src[tid] = mine ? from : -1;
        dst[tid] = to;
    }
    if (!__syncthreads_or(mine)) return;
    const int hd = c.kv.hd, d0 = sl * dw, w = min(dw, hd - d0);
    T* const ks = (T*)lds;
    T* const vs = ks + (size_t)n * dw;
    T* const base = (T*)c.kv.base;
    for (int e = tid; e < n * w; e += 256) {
        const int i = e / w, d = e % w, s = src[i];
        if (s < 0) continue;
        ks[i * dw + d] = base[c.kv.k_off(layer, s / kPageTokens, g) + (size_t)(s % kPageTokens) * hd + d0 + d];
        vs[i * dw + d] = base[c.kv.v_off(layer, s / kPageTokens, g) + (size_t)(d0 + d) * kPageTokens + s % kPageTokens];
    }
    __syncthreads();
    for (int e = tid; e < n * w; e += 256) {
        const int i = e / w, d = e % w, t = dst[i];
        if (src[i] < 0) continue;
        base[c.kv.k_off(layer, t / kPageTokens, g) + (size_t)(t % kPageTokens) * hd + d0 + d] = ks[i * dw + d];
        base[c.kv.v_off(layer, t / kPageTokens, g) + (size_t)(d0 + d) * kPageTokens + t % kPageTokens] = vs[i * dw + d];
    }
}

}  // namespace

void launch_copy_pages(const KVPool& kv, int layers, int n, const int32_t* src, const int32_t* dst, hipStream_t s) {
    copy_pages(kv, layers, n, DeviceIds{src, dst}, s);
}
void launch_copy_pages(const KVPool& kv, int layers, int n, const CopyPages& pages, hipStream_t s) {
    copy_pages(kv, layers, n, pages, s);
}

void launch_compact(const CompactCall& c, hipStream_t s) {
    // slices of dims that leave a workgroup's rows within 32 KB of LDS
    int dw = c.kv.hd;
    while ((size_t)2 * c.max_keep * dw * c.kv.esize > 32768) dw = (dw + 1) / 2;
    const int slices = (c.kv.hd + dw - 1) / dw;
    const size_t lds = (size_t)2 * c.max_keep * dw * c.kv.esize;
    const dim3 grid(c.kv.hkv * slices, c.layers, c.n_users);
    if (c.kv.esize == 2) hipLaunchKernelGGL(k_compact<bf16_t>, grid, dim3(256), lds, s, c, dw, slices);
    else hipLaunchKernelGGL(k_compact<float>, grid, dim3(256), lds, s, c, dw, slices);
}

int32_t pool_of(const sd_kv_pool* p, KVPool* kv) {
    if (!p || p->n_layers < 1 || p->n_pages < 1 || p->n_kv_heads < 1 || p->head_dim < 1) return SD_EINVAL;
    if (p->dtype != SD_F32 && p->dtype != SD_BF16) return SD_EINVAL;
    if (p->dtype == SD_BF16 ? p->head_dim != 64 && p->head_dim != 128 : p->head_dim % 2 || p->head_dim > 128)
        return SD_ENOTIMPL;
    // (a page of a layer is counted in 31 bits, a row of the layer's pages in 32)
    if (p->n_pages > (1 << 27) || p->n_kv_heads > (1 << 13) || p->n_layers > (1 << 12)) return SD_ELIMIT;
    kv->base = p->base;
    kv->n_pages = p->n_pages;
    kv->hkv = p->n_kv_heads;
    kv->hd = p->head_dim;
    kv->esize = p->dtype == SD_BF16 ? 2 : 4;
    return SD_OK;
}

}  // namespace sdv

extern "C" {

sd_status sd_kv_copy_pages(const sd_kv_pool* pool, int32_t n, const int32_t* src, const int32_t* dst,
                           sd_stream stream) {
    sdv::KVPool kv;
    const sd_status r = sdv::pool_of(pool, &kv);
    if (r != SD_OK) return r;
    if (n < 1 || !kv.base || !src || !dst || (uintptr_t)kv.base % 256 || ((uintptr_t)src | (uintptr_t)dst) % 4)
        return SD_EINVAL;
    const uint64_t bytes = kv.page_elems() * kv.esize;
    if ((bytes + sdv::kCopyPiece - 1) / sdv::kCopyPiece * (uint64_t)n >= (1u << 24)) return SD_ELIMIT;
    sdv::launch_copy_pages(kv, pool->n_layers, n, src, dst, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? SD_OK : SD_EHIP;
}

sd_status sd_kv_compact(const sd_kv_pool* pool, int32_t n_users, const int32_t* prefix, const int32_t* page_table,
                        int32_t max_pages, const int32_t* keep, int32_t max_keep, const int32_t* n_keep,
                        sd_stream stream) {
    sdv::CompactCall c{};
    const sd_status r = sdv::pool_of(pool, &c.kv);
    if (r != SD_OK) return r;
    if (n_users < 1 || max_keep < 1 || max_pages < 1 || !c.kv.base || !prefix || !page_table || !keep || !n_keep)
        return SD_EINVAL;
    if ((uintptr_t)c.kv.base % 256 ||
        ((uintptr_t)prefix | (uintptr_t)page_table | (uintptr_t)keep | (uintptr_t)n_keep) % 4)
        return SD_EINVAL;
    if (max_keep > SD_KV_COMPACT_MAX || n_users > SD_TREE_MAX_USERS) return SD_ELIMIT;
    c.layers = pool->n_layers;
    c.n_users = n_users;
    c.max_pages = max_pages;
    c.max_keep = max_keep;
    c.prefix = prefix;
    c.page_table = page_table;
    c.keep = keep;
    c.n_keep = n_keep;
    sdv::launch_compact(c, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? SD_OK : SD_EHIP;
}

}  // extern "C"
