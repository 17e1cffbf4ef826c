// Rules on rows of logits: penalties for repeated tokens, biases, grammar masks.
//
// Per row and token k, with c the times that k is in the output and s whether it is
// in prompt or output:  s: z / r or z * r by z's sign;  c: z - (f c + p);  listed:
// z + bias;  not allowed: -inf.
//
// A workgroup takes a chunk of the vocabulary and a few rows.  It counts the
// chunk's tokens of a row's history in LDS (integers: the order does not matter),
// keeps the counts while the next row has the same history, as the slots of a user
// do, and adds the row's own drafts for that row alone.
#include <algorithm>

#include "../../include/sd_verify.h"
#include "sdv_device.h"
#include "sdv_internal.h"

namespace sdv {
namespace {

constexpr int kChunk = 4096;         // tokens a workgroup
constexpr int kRowsMax = 8;          // rows a workgroup
constexpr int kBack = SD_TREE_MAX_SLOTS;  // rows below a row that its drafts may be in
constexpr uint32_t kPrompt = 0x80000000u;  // count word: the token is in the prompt

__device__ __forceinline__ float fin(const float* p, int t, float off) {
    const float v = p ? p[t] : off;
    return isfinite(v) ? v : off;
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_rules(RulesCall c, int rows, int words) {
    extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
    __shared__ int par[kBack + kRowsMax], tokw[kBack + kRowsMax];
    __shared__ uint16_t own[kRowsMax][kBack + 1];  // a row's drafts in this chunk
    __shared__ int n_own[kRowsMax];
    uint32_t* const cnt = lds;            // [kChunk]
    uint32_t* const bix = lds + kChunk;   // [kChunk] entry + 1 of the token's bias (with biases only)
    const int tid = threadIdx.x;
    const int k0 = blockIdx.x * kChunk, kn = min(kChunk, c.V - k0);
    const int r0 = blockIdx.y * rows, r1 = min(c.n_rows, r0 + rows);
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
    int hb = -1, hf = -1, he = -1, bb = -1, be = -1;
    for (int t = r0; t < r1; ++t) {
        int nb = 0, nf = 0, ne = 0, ob = 0, oe = 0;
        if (c.hist) {
            nb = min(max(c.hist[3 * (size_t)t], 0), c.n_tokens);
            nf = min(max(c.hist[3 * (size_t)t + 1], nb), c.n_tokens);
            ne = min(max(c.hist[3 * (size_t)t + 2], nf), c.n_tokens);
        }
        if (c.bias) {
            ob = min(max(c.bias[2 * (size_t)t], 0), c.n_bias);
            oe = min(max(c.bias[2 * (size_t)t + 1], ob), c.n_bias);
        }
        __syncthreads();  // the previous row has been read
        if (nb != hb || nf != hf || ne != he) {
            for (int i = tid; i < kChunk; i += 256) cnt[i] = 0;
            __syncthreads();
            for (int i = nb + tid; i < ne; i += 256) {
                const int k = c.tokens[i] - k0;
                if (k < 0 || k >= kn) continue;
                if (i < nf) atomicOr(&cnt[k], kPrompt);
                else atomicAdd(&cnt[k], 1u);
            }
            hb = nb; hf = nf; he = ne;
        }
        if (c.bias && (ob != bb || oe != be)) {
            for (int i = tid; i < kChunk; i += 256) bix[i] = 0;
            __syncthreads();
            for (int i = ob + tid; i < oe; i += 256) {
                const int k = c.bias_token[i] - k0;
                if (k >= 0 && k < kn) atomicMax(&bix[k], (uint32_t)i + 1);  // the last entry of a token
            }
            bb = ob; be = oe;
        }
        for (int i = tid; i < n_own[t - r0]; i += 256) atomicAdd(&cnt[own[t - r0][i]], 1u);
        float rep = c.rep ? c.rep[t] : 1.f;
        if (!(rep > 0.f && isfinite(rep))) rep = 1.f;
        const float pres = fin(c.pres, t, 0.f), freq = fin(c.freq, t, 0.f);
        const int mr = c.mask ? c.mask_row[t] : -1;
        const uint32_t* mask = mr >= 0 && mr < c.n_masks ? c.mask + (size_t)mr * words : nullptr;
        const T* z = (const T*)c.logits + (size_t)t * c.stride;
        float* o = c.out + (size_t)t * c.ostride;
        const bool in_place = (const void*)z == (const void*)o;
        __syncthreads();
        auto rule = [&](int k, float v, uint32_t w, uint32_t bx, bool allowed) {
            const uint32_t times = w & ~kPrompt;
            if (w) v = v > 0.f ? v / rep : v * rep;
            if (times) v -= freq * (float)times + pres;
            if (bx) v += c.bias_value[bx - 1];
            return allowed ? v : -INFINITY;
        };
        if (VEC) {
            for (int k = 4 * tid; k < kn; k += 1024) {
                float v[4];
                const uint4 w = *(const uint4*)(cnt + k);
                uint4 bx = uint4{0, 0, 0, 0};
                if (c.bias) bx = *(const uint4*)(bix + k);
                const uint32_t m = mask ? mask[(k0 + k) >> 5] >> ((k0 + k) & 31) : 0xfu;
                const bool touch = (w.x | w.y | w.z | w.w | bx.x | bx.y | bx.z | bx.w) || (~m & 0xf);
                if (in_place && !touch) continue;
                if constexpr (sizeof(T) == 2) {
                    const uint2 u = *(const uint2*)(z + k0 + k);
                    v[0] = bf16_to_f32(u.x & 0xffff); v[1] = bf16_to_f32(u.x >> 16);
                    v[2] = bf16_to_f32(u.y & 0xffff); v[3] = bf16_to_f32(u.y >> 16);
                } else {
                    const float4 u = *(const float4*)(z + k0 + k);
                    v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
                }
                if (touch) {
                    v[0] = rule(k, v[0], w.x, bx.x, m & 1);
                    v[1] = rule(k + 1, v[1], w.y, bx.y, m & 2);
                    v[2] = rule(k + 2, v[2], w.z, bx.z, m & 4);
                    v[3] = rule(k + 3, v[3], w.w, bx.w, m & 8);
                }
                *(float4*)(o + k0 + k) = float4{v[0], v[1], v[2], v[3]};
            }
        } else {
            for (int k = tid; k < kn; k += 256) {
                const uint32_t w = cnt[k], bx = c.bias ? bix[k] : 0;
                const bool ok = !mask || ((mask[(k0 + k) >> 5] >> ((k0 + k) & 31)) & 1);
                if (in_place && !w && !bx && ok) continue;
                o[k0 + k] = rule(k, ld<T>(z, k0 + k), w, bx, ok);
            }
        }
        if (n_own[t - r0]) {
            __syncthreads();
            for (int i = tid; i < n_own[t - r0]; i += 256) atomicSub(&cnt[own[t - r0][i]], 1u);
        }
    }
}

}  // namespace

void launch_rules(const RulesCall& c, hipStream_t s) {
    const int chunks = (c.V + kChunk - 1) / kChunk;
    // rows that share their histories' counts, while there are workgroups for every CU
    int rows = kRowsMax;
    while (rows > 1 && (int64_t)((c.n_rows + rows - 1) / rows) * chunks < 4 * cu_count()) rows /= 2;
    const size_t lds = (size_t)kChunk * 4 * (c.bias ? 2 : 1);
    const int words = (c.V + 31) / 32;
    const dim3 grid(chunks, (c.n_rows + rows - 1) / rows);
    // four elements a load where every row starts on that
    const uintptr_t es = c.bf16 ? 2 : 4;
    const bool vec = c.V % 4 == 0 && c.stride % 4 == 0 && c.ostride % 4 == 0 && (uintptr_t)c.logits % (4 * es) == 0 &&
                     (uintptr_t)c.out % 16 == 0;
    if (c.bf16) {
        if (vec) hipLaunchKernelGGL((k_rules<bf16_t, true>), grid, dim3(256), lds, s, c, rows, words);
        else hipLaunchKernelGGL((k_rules<bf16_t, false>), grid, dim3(256), lds, s, c, rows, words);
    } else {
        if (vec) hipLaunchKernelGGL((k_rules<float, true>), grid, dim3(256), lds, s, c, rows, words);
        else hipLaunchKernelGGL((k_rules<float, false>), grid, dim3(256), lds, s, c, rows, words);
    }
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
    if (r->n_tokens > 0x7fffffff || r->n_bias > 0x7fffffff) return SD_ELIMIT;
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
