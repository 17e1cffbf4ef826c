// Rules on rows of logits: penalties for repeated tokens, biases, grammar masks.
//
// Per row and token k, with c the times that k is in the output and s whether it is
// in prompt or output:  s: z / r or z * r by z's sign;  c: z - (f c + p);  listed:
// z + bias;  not allowed: -inf.
//
// What bounds it: the row read once and written once in 32 bits (6 bytes a token for
// bfloat16 rows); history, biases and masks are a few percent of that, but every
// workgroup of a row looks through the whole of its history and biases.  So a workgroup
// takes kChunk tokens of up to kRowsMax rows: it counts the chunk's tokens of a history
// in LDS (integers: the order does not matter), keeps the words while the next row has
// the same history and biases, as the slots of a user do, and adds the row's own drafts
// for that row alone.  The row's elements are loaded one row ahead, before the lists are
// looked through.  Between short chunks (more workgroups a CU to hide the lists' loads)
// and long ones (fewer looks through the lists), and between few and many rows, 416 bf16
// rows of 155136 with histories, biases and masks (389 MB) took
//     kChunk 2048, rows 2 / 4 / 8:  168 / 144 / 141 us;  229 such rows  73 / 69 / 70
//     kChunk 4096, rows 2 / 4 / 8:  166 / 162 / 168 us   (an earlier form of the lists)
// so 2048 and 4: 2.7 TB/s.  Of the 144 us the rows alone are 80 (4.8 TB/s, a copy's rate),
// histories 17 to 22, masks 12 to 17, biases 22 to 31.  In place the rows are read and
// written only where something changes them, but looked through the same: 229 fp32 rows
// with histories and biases 51 us instead of 65 of their own, 416 with masks 126 of 146.
// A row's drafts are found by one thread, parent after parent: 256 rows of 151936 tokens
// take 56 us as 256 roots, 95 as one path of 256.
#include <algorithm>

#include "../../include/sd_verify.h"
#include "sdv_device.h"
#include "sdv_internal.h"

namespace sdv {
namespace {

constexpr int kChunk = 2048;         // tokens a workgroup
constexpr int kRowsMax = 4;          // rows a workgroup
constexpr int kBack = SD_TREE_MAX_SLOTS;  // rows below a row that its drafts may be in
constexpr int kHeld = 2;             // biases a thread keeps in registers, the rest are read again
// a token's word: in the prompt, with a bias, how often in the output
constexpr uint32_t kPrompt = 0x80000000u, kBias = 0x40000000u, kCount = 0x3fffffffu;

__device__ __forceinline__ float fin(const float* p, int t, float off) {
    const float v = p ? p[t] : off;
    return isfinite(v) ? v : off;
}

// A list's entries by the whole workgroup, kAhead loads in flight a thread.
constexpr int kAhead = 8;
template <class F> __device__ __forceinline__ void for_list(const int32_t* list, int begin, int end, F f) {
    for (int i0 = begin + (int)threadIdx.x; i0 < end; i0 += 256 * kAhead) {
        int k[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) k[u] = i0 + 256 * u < end ? list[i0 + 256 * u] : -1;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) f(i0 + 256 * u, k[u]);
    }
}

// Four elements of a row as they lie in memory, where a row may begin at any element:
// the hardware takes a wide access at any address (229 rows of 155133 fp32 logits take
// 71 us where those of 155136 take 69; one element a load took 127).
typedef float f32x4e __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2e __attribute__((ext_vector_type(2), aligned(2)));
template <typename T> struct Four;
template <> struct Four<float> {
    f32x4e v;
    __device__ __forceinline__ void load(const float* z) { v = *(const f32x4e*)z; }
    __device__ __forceinline__ void some(const float* z, int n) {  // the first n < 4
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) v[e] = z[e];
    }
    __device__ __forceinline__ void get(float (&o)[4]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = v[e];
    }
};
template <> struct Four<bf16_t> {
    u32x2e v;
    __device__ __forceinline__ void load(const bf16_t* z) { v = *(const u32x2e*)z; }
    __device__ __forceinline__ void some(const bf16_t* z, int n) {
        const uint16_t* h = (const uint16_t*)z;
        v[0] = h[0] | (n > 1 ? (uint32_t)h[1] << 16 : 0u);
        v[1] = n > 2 ? h[2] : 0u;
    }
    __device__ __forceinline__ void get(float (&o)[4]) const {
        o[0] = __uint_as_float(v.x << 16);
        o[1] = __uint_as_float(v.x & 0xffff0000u);
        o[2] = __uint_as_float(v.y << 16);
        o[3] = __uint_as_float(v.y & 0xffff0000u);
    }
};

// What rules a row has.
struct RowRules {
    int nb, nf, ne, ob, oe;  // its history's begin, first output and end, its biases
    float rep, pres, freq;
    const uint32_t* mask;
};
__device__ __forceinline__ RowRules row_rules(const RulesCall& c, int t, int words) {
    RowRules r{};
    if (c.hist) {
        r.nb = min(max(c.hist[3 * (size_t)t], 0), c.n_tokens);
        r.nf = min(max(c.hist[3 * (size_t)t + 1], r.nb), c.n_tokens);
        r.ne = min(max(c.hist[3 * (size_t)t + 2], r.nf), c.n_tokens);
    }
    if (c.bias) {
        r.ob = min(max(c.bias[2 * (size_t)t], 0), c.n_bias);
        r.oe = min(max(c.bias[2 * (size_t)t + 1], r.ob), c.n_bias);
    }
    r.rep = c.rep ? c.rep[t] : 1.f;
    if (!(r.rep > 0.f && isfinite(r.rep))) r.rep = 1.f;
    r.pres = fin(c.pres, t, 0.f);
    r.freq = fin(c.freq, t, 0.f);
    const int m = c.mask ? c.mask_row[t] : -1;
    r.mask = m >= 0 && m < c.n_masks ? c.mask + (size_t)m * words : nullptr;
    return r;
}

// Rows of `out` apart from the logits: the next row's loads are in flight while one is
// written.  PLACE: in place, where only what changes is read and written.
template <typename T, bool PLACE>
__global__ __launch_bounds__(256) void k_rules(RulesCall c, int rows, int words) {
    extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
    __shared__ int par[kBack + kRowsMax], tokw[kBack + kRowsMax];
    __shared__ uint16_t own[kRowsMax][kBack + 1];  // a row's drafts in this chunk
    __shared__ int n_own[kRowsMax];
    __shared__ RowRules rules[kRowsMax];
    uint32_t* const cnt = lds;            // [kChunk]
    // where a token's word says kBias: [kChunk] the bias's entry, [kChunk] its value
    uint32_t* const bix = lds + kChunk;
    float* const bval = (float*)(lds + 2 * kChunk);
    const int tid = threadIdx.x;
    const int k0 = blockIdx.x * kChunk, kn = min(kChunk, c.V - k0);
    const int r0 = blockIdx.y * rows, r1 = min(c.n_rows, r0 + rows);
    constexpr int Q = kChunk / 1024;
    Four<T> now[Q], next[Q];
    uint32_t m[Q], mnext[Q];  // the mask's bits of the thread's elements
    auto load = [&](int t, Four<T> (&q)[Q]) __attribute__((always_inline)) {
        const T* z = (const T*)c.logits + (size_t)t * c.stride + k0;
#pragma unroll
        for (int u = 0; u < Q; ++u) {
            const int k = 4 * tid + 1024 * u;
            if (k + 4 <= kn) q[u].load(z + k);
            else if (k < kn) q[u].some(z + k, kn - k);
        }
    };
    auto load_mask = [&](const uint32_t* mask, uint32_t (&q)[Q]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < Q; ++u) {
            const int k = 4 * tid + 1024 * u;
            q[u] = mask && k < kn ? mask[(k0 + k) >> 5] >> ((k0 + k) & 31) : 0xfu;
        }
    };
    if constexpr (!PLACE) load(r0, now);
    if (tid < r1 - r0) rules[tid] = row_rules(c, r0 + tid, words);
    if (c.row_token) {
        const int w0 = r0 - kBack;
        for (int i = tid; i < kBack + r1 - r0; i += 256) {
            const int t = w0 + i;
            int p = -1;
            if (t >= 0) {
                const int j = c.slot_j ? c.slot_j[t] : 0;
                p = !c.row_parent ? (j > 0 ? t - 1 : -1) : c.row_parent[t];
                // (user-local parents: the user's first slot is row t - j)
                if (c.row_parent && c.slot_j) p = p < 0 || p >= j ? -1 : t - j + p;
            }
            par[i] = p >= 0 && p < t ? p : -1;
            tokw[i] = t >= 0 ? c.row_token[t] : -1;
        }
        __syncthreads();
        if (tid < r1 - r0) {
            const int t = r0 + tid, low = max(0, t - kBack);
            int n = 0;
            for (int a = t; a >= low; a = par[a - w0]) {
                const int k = tokw[a - w0] - k0;
                if (k >= 0 && k < kn) own[tid][n++] = (uint16_t)k;
            }
            n_own[tid] = n;
        }
    } else if (tid < rows) {
        n_own[tid] = 0;
    }
    __syncthreads();
    load_mask(rules[0].mask, m);
    // every entry of the row's biases whose token is in the chunk: those held, those beyond
    auto for_biases = [&](int oe, int more, const int (&bk)[kHeld], const float (&bv)[kHeld], auto chunk_of, auto f) {
#pragma unroll
        for (int u = 0; u < kHeld; ++u)
            if (bk[u] >= 0) f(more - 256 * (kHeld - u) + tid, bk[u], bv[u]);
        for (int i = more + tid; i < oe; i += 256) {
            const int k = chunk_of(c.bias_token[i]);
            if (k >= 0) f(i, k, c.bias_value[i]);
        }
    };
    int hb = -1, hf = -1, he = -1, bb = -1, be = -1;
    for (int t = r0; t < r1; ++t) {
        if (t + 1 < r1) {
            if constexpr (!PLACE) load(t + 1, next);
            load_mask(rules[t + 1 - r0].mask, mnext);
        }
        const RowRules r = rules[t - r0];
        // the words: anew where history or biases are others, else as they are
        if (r.nb != hb || r.nf != hf || r.ne != he || r.ob != bb || r.oe != be) {
            // (the first biases in registers from here on)
            int bk[kHeld];
            float bv[kHeld];
#pragma unroll
            for (int u = 0; u < kHeld; ++u) {
                const int i = r.ob + tid + 256 * u;
                bk[u] = i < r.oe ? c.bias_token[i] - k0 : -1;
                bv[u] = i < r.oe ? c.bias_value[i] : 0.f;
                if (bk[u] >= kn) bk[u] = -1;
            }
            const int more = r.ob + 256 * kHeld;
            __syncthreads();  // the previous row has been read
            for (int i = 4 * tid; i < kChunk; i += 1024) *(uint4*)(cnt + i) = uint4{0, 0, 0, 0};
            auto chunk_of = [&](int k) { return k >= k0 && k < k0 + kn ? k - k0 : -1; };
            for_biases(r.oe, more, bk, bv, chunk_of, [&](int, int k, float) { bix[k] = 0; });
            __syncthreads();
            for_list(c.tokens, r.nb, r.ne, [&](int i, int k) {
                k -= k0;
                if (k < 0 || k >= kn) return;
                if (i < r.nf) atomicOr(&cnt[k], kPrompt);
                else atomicAdd(&cnt[k], 1u);
            });
            for_biases(r.oe, more, bk, bv, chunk_of, [&](int i, int k, float) {
                atomicOr(&cnt[k], kBias);
                atomicMax(&bix[k], (uint32_t)(i - r.ob));  // the last entry of a token
            });
            if (r.oe > r.ob) {
                __syncthreads();
                for_biases(r.oe, more, bk, bv, chunk_of, [&](int i, int k, float v) {
                    if (bix[k] == (uint32_t)(i - r.ob)) bval[k] = v;
                });
            }
            hb = r.nb; hf = r.nf; he = r.ne;
            bb = r.ob; be = r.oe;
            __syncthreads();
        }
        const int mine = n_own[t - r0];
        if (mine) {
            __syncthreads();
            for (int i = tid; i < mine; i += 256) atomicAdd(&cnt[own[t - r0][i]], 1u);
            __syncthreads();
        }
        const T* z = (const T*)c.logits + (size_t)t * c.stride;
        float* o = c.out + (size_t)t * c.ostride;
        auto rule = [&](float v, uint32_t w, int k) {
            const uint32_t times = w & kCount;
            if (w & (kPrompt | kCount)) v = v > 0.f ? v / r.rep : v * r.rep;
            if (times) v -= r.freq * (float)times + r.pres;
            if (w & kBias) v += bval[k];
            return v;
        };
#pragma unroll
        for (int u = 0; u < Q; ++u) {
            const int k = 4 * tid + 1024 * u;
            if (k >= kn) break;
            const uint4 w = *(const uint4*)(cnt + k);
            if constexpr (PLACE) {
                if (!(w.x | w.y | w.z | w.w) && !(~m[u] & 0xf)) continue;
                if (k + 4 <= kn) now[u].load(z + k0 + k);
                else now[u].some(z + k0 + k, kn - k);
            }
            float v[4];
            now[u].get(v);
            if (w.x | w.y | w.z | w.w) {
                v[0] = rule(v[0], w.x, k);
                v[1] = rule(v[1], w.y, k + 1);
                v[2] = rule(v[2], w.z, k + 2);
                v[3] = rule(v[3], w.w, k + 3);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = m[u] >> e & 1 ? v[e] : -INFINITY;
            if (k + 4 <= kn) {
                *(f32x4e*)(o + k0 + k) = f32x4e{v[0], v[1], v[2], v[3]};
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (k + e < kn) o[k0 + k + e] = v[e];
            }
        }
#pragma unroll
        for (int u = 0; u < Q; ++u) {
            if constexpr (!PLACE) now[u] = next[u];
            m[u] = mnext[u];
        }
        if (mine && t + 1 < r1) {
            __syncthreads();
            for (int i = tid; i < mine; i += 256) atomicSub(&cnt[own[t - r0][i]], 1u);
            __syncthreads();
        }
    }
}

}  // namespace

void launch_rules(const RulesCall& c, hipStream_t s) {
    const int chunks = (c.V + kChunk - 1) / kChunk;
    // rows that share their histories' counts, while there are workgroups for every CU
    int rows = kRowsMax;
    while (rows > 1 && (int64_t)((c.n_rows + rows - 1) / rows) * chunks < 4 * cu_count()) rows /= 2;
    const size_t lds = (size_t)kChunk * 4 * (c.bias ? 3 : 1);
    const int words = (c.V + 31) / 32;
    const dim3 grid(chunks, (c.n_rows + rows - 1) / rows);
    const bool place = c.logits == (const void*)c.out;  // (fp32)
    const auto run = [&](auto fn) { hipLaunchKernelGGL(fn, grid, dim3(256), lds, s, c, rows, words); };
    if (c.bf16) run(k_rules<bf16_t, false>);
    else place ? run(k_rules<float, true>) : run(k_rules<float, false>);
}

// The rules' arrays; out is left to the caller.
int32_t rules_of(const sd_logit_rules* r, RulesCall* c) {
    if (!r) return SD_EINVAL;
    if (r->n_tokens < 0 || r->n_bias < 0 || r->n_masks < 0) return SD_EINVAL;
    // histories, biases and masks come with their index tables (and a table of empty
    // ranges with nothing)
    auto fit = [](const void* list, int64_t n, const void* table) {
        return table ? list || n == 0 : list == nullptr;
    };
    if (!fit(r->tokens, r->n_tokens, r->hist) || !fit(r->bias_token, r->n_bias, r->bias) ||
        !fit(r->bias_value, r->n_bias, r->bias) || !fit(r->mask, r->n_masks, r->mask_row) ||
        (r->row_token != nullptr) != (r->row_parent != nullptr))
        return SD_EINVAL;
    if (((uintptr_t)r->tokens | (uintptr_t)r->hist | (uintptr_t)r->row_token | (uintptr_t)r->row_parent |
         (uintptr_t)r->repetition | (uintptr_t)r->presence | (uintptr_t)r->frequency | (uintptr_t)r->bias_token |
         (uintptr_t)r->bias_value | (uintptr_t)r->bias | (uintptr_t)r->mask | (uintptr_t)r->mask_row) % 4)
        return SD_EINVAL;
    // (a token's word counts to 2^30, and a list's index runs past its end by a step)
    if (r->n_tokens > (1 << 30) - 4096 || r->n_bias > (1 << 30) - 4096) return SD_ELIMIT;
    c->tokens = r->tokens;
    c->n_tokens = (int)r->n_tokens;
    c->hist = r->hist;
    c->row_token = r->row_token;
    c->row_parent = r->row_parent;
    c->slot_j = nullptr;
    c->rep = r->repetition;
    c->pres = r->presence;
    c->freq = r->frequency;
    c->bias_token = r->bias_token;
    c->bias_value = r->bias_value;
    c->n_bias = (int)r->n_bias;
    c->bias = r->bias;
    c->mask = r->mask;
    c->n_masks = r->n_masks;
    c->mask_row = r->mask_row;
    return SD_OK;
}

}  // namespace sdv

extern "C" {

sd_status sd_adjust_logits(int32_t n_rows, int32_t vocab, const void* logits, int32_t dtype, int64_t row_stride,
                           const sd_logit_rules* rules, float* out, int64_t out_stride, sd_stream stream) {
    if (n_rows < 1 || vocab < 1 || !logits || !out || (dtype != SD_F32 && dtype != SD_BF16) || row_stride < vocab ||
        out_stride < vocab)
        return SD_EINVAL;
    if (n_rows > SD_FILTER_MAX_ROWS || vocab > SD_FILTER_MAX_VOCAB) return SD_ELIMIT;
    const uintptr_t es = dtype == SD_BF16 ? 2 : 4;
    if ((uintptr_t)logits % es || (uintptr_t)out % 4) return SD_EINVAL;
    // the rows may be rewritten in place, and may not overlap otherwise
    const uintptr_t i0 = (uintptr_t)logits, o0 = (uintptr_t)out;
    const uintptr_t i1 = i0 + ((uint64_t)(n_rows - 1) * row_stride + vocab) * es;
    const uintptr_t o1 = o0 + ((uint64_t)(n_rows - 1) * out_stride + vocab) * 4;
    const bool same = dtype == SD_F32 && i0 == o0 && (n_rows == 1 || row_stride == out_stride);
    if (!same && i0 < o1 && o0 < i1) return SD_EINVAL;
    sdv::RulesCall c{};
    const sd_status r = sdv::rules_of(rules, &c);
    if (r != SD_OK) return r;
    c.n_rows = n_rows;
    c.V = vocab;
    c.bf16 = dtype == SD_BF16;
    c.logits = logits;
    c.stride = row_stride;
    c.out = out;
    c.ostride = out_stride;
    sdv::launch_rules(c, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? SD_OK : SD_EHIP;
}

}  // extern "C"
