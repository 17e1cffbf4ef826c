// Low-rank adapters of many requests beside a shared projection:
// y[t] += scale[a] * B_a (A_a x[t]), a the adapter of row t.
#include <algorithm>

#include "../../include/sd_verify.h"
#include "sdv_device.h"
#include "sdv_internal.h"

namespace sdv {
namespace {

// one rounding to the output's type (NaN stays NaN)
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t* p, float v) { *p = __builtin_bit_cast(bf16_t, (__bf16)v); }

// h[t][r] = A_a[r] . x[t], a wave each
template <typename T>
__global__ __launch_bounds__(256) void k_lora_down(LoraCall c, float* h) {
    const int R = c.n_seg * c.rank;
    const int r = blockIdx.y * 4 + (threadIdx.x >> 6), t = blockIdx.x, lane = threadIdx.x & 63;
    const int a = c.ids[t];
    if (r >= R || a < 0 || a >= c.n_adapters) return;
    const T* A = (const T*)c.a + ((size_t)a * R + r) * c.d_in;
    const T* x = (const T*)c.x + (size_t)t * c.xs;
    const T* xl = c.x_lo ? (const T*)c.x_lo + (size_t)t * c.xs : nullptr;
    float s = 0.f;
    for (int i = lane; i < c.d_in; i += 64) s += ld<T>(A, i) * (ld<T>(x, i) + (xl ? ld<T>(xl, i) : 0.f));
    s = wave_sum(s);
    if (lane == 0) h[(size_t)t * R + r] = s;
}

template <typename T, typename Y>
__global__ __launch_bounds__(256) void k_lora_up(LoraCall c, const float* h) {
    const int col = blockIdx.y * 256 + threadIdx.x, t = blockIdx.x;
    if (col >= c.d_out) return;
    const int a = c.ids[t];
    const Y* yi = (const Y*)c.y_in + (size_t)t * c.ys;
    Y* yo = (Y*)c.y_out + (size_t)t * c.yos;
    if (a < 0 || a >= c.n_adapters) {
        if (yi != yo) yo[col] = yi[col];
        return;
    }
    int seg = 0;
    while (col >= c.seg[seg + 1]) ++seg;
    const float* hr = h + ((size_t)t * c.n_seg + seg) * c.rank;
    const T* B = (const T*)c.b + ((size_t)a * c.d_out + col) * c.rank;
    float s = 0.f;
    for (int r = 0; r < c.rank; ++r) s += ld<T>(B, r) * hr[r];
    put(yo + col, ld<Y>(yi, col) + (c.scale ? c.scale[a] : 1.f) * s);
}

}  // namespace

size_t lora_workspace(int T, int rank, int n_seg) { return ((size_t)T * rank * n_seg * 4 + 255) & ~(size_t)255; }

void launch_lora(const LoraCall& c, hipStream_t s) {
    float* h = (float*)c.ws;
    const dim3 gd(c.T, (c.n_seg * c.rank + 3) / 4), gu(c.T, (c.d_out + 255) / 256);
    if (c.bf16) {
        hipLaunchKernelGGL(k_lora_down<bf16_t>, gd, dim3(256), 0, s, c, h);
        if (c.y_bf16) hipLaunchKernelGGL((k_lora_up<bf16_t, bf16_t>), gu, dim3(256), 0, s, c, h);
        else hipLaunchKernelGGL((k_lora_up<bf16_t, float>), gu, dim3(256), 0, s, c, h);
    } else {
        hipLaunchKernelGGL(k_lora_down<float>, gd, dim3(256), 0, s, c, h);
        if (c.y_bf16) hipLaunchKernelGGL((k_lora_up<float, bf16_t>), gu, dim3(256), 0, s, c, h);
        else hipLaunchKernelGGL((k_lora_up<float, float>), gu, dim3(256), 0, s, c, h);
    }
}

}  // namespace sdv

extern "C" {

sd_status sd_lora_query_size(const sd_lora* w, int32_t n_rows, uint64_t* workspace_bytes) {
    if (!w || !workspace_bytes || n_rows < 1 || w->n_adapters < 1 || w->rank < 1 || w->d_in < 1 || w->d_out < 1 ||
        w->n_seg < 1)
        return SD_EINVAL;
    if (w->dtype != SD_F32 && w->dtype != SD_BF16) return SD_EINVAL;
    if (w->rank > SD_LORA_MAX_RANK || w->n_seg > SD_LORA_MAX_SEGS || n_rows > (1 << 20) || w->d_in > (1 << 20) ||
        w->d_out > (1 << 20))
        return SD_ELIMIT;
    if (w->seg_off[0] != 0 || w->seg_off[w->n_seg] != w->d_out) return SD_EINVAL;
    for (int i = 0; i < w->n_seg; ++i)
        if (w->seg_off[i] >= w->seg_off[i + 1]) return SD_EINVAL;
    *workspace_bytes = sdv::lora_workspace(n_rows, w->rank, w->n_seg);
    return SD_OK;
}

sd_status sd_lora_apply(const sd_lora* w, int32_t n_rows, const int32_t* adapter, const void* x, const void* x_lo,
                        int64_t x_stride, const void* y_in, int64_t y_in_stride, void* y_out, int64_t y_out_stride,
                        int32_t y_dtype, void* workspace, uint64_t workspace_bytes, sd_stream stream) {
    uint64_t need = 0;
    const sd_status r = sd_lora_query_size(w, n_rows, &need);
    if (r != SD_OK) return r;
    if (!w->a || !w->b || !adapter || !x || !y_in || !y_out || !workspace) return SD_EINVAL;
    if ((y_dtype != SD_F32 && y_dtype != SD_BF16) || (x_lo && w->dtype != SD_BF16)) return SD_EINVAL;
    if (x_stride < w->d_in || y_in_stride < w->d_out || y_out_stride < w->d_out) return SD_EINVAL;
    const uintptr_t es = w->dtype == SD_BF16 ? 2 : 4, ey = y_dtype == SD_BF16 ? 2 : 4;
    if (((uintptr_t)w->a | (uintptr_t)w->b | (uintptr_t)x | (uintptr_t)x_lo) % es ||
        ((uintptr_t)y_in | (uintptr_t)y_out) % ey || ((uintptr_t)adapter | (uintptr_t)w->scale) % 4 ||
        (uintptr_t)workspace % 256)
        return SD_EINVAL;
    // in place, or apart
    const uintptr_t i0 = (uintptr_t)y_in, o0 = (uintptr_t)y_out;
    const uintptr_t i1 = i0 + ((uint64_t)(n_rows - 1) * y_in_stride + w->d_out) * ey;
    const uintptr_t o1 = o0 + ((uint64_t)(n_rows - 1) * y_out_stride + w->d_out) * ey;
    if (!(i0 == o0 && (n_rows == 1 || y_in_stride == y_out_stride)) && i0 < o1 && o0 < i1) return SD_EINVAL;
    if (workspace_bytes < need) return SD_ENOMEM;
    sdv::LoraCall c{};
    c.T = n_rows;
    c.d_in = w->d_in;
    c.d_out = w->d_out;
    c.rank = w->rank;
    c.n_seg = w->n_seg;
    c.n_adapters = w->n_adapters;
    for (int i = 0; i <= sdv::kLoraSegs; ++i) c.seg[i] = w->seg_off[std::min(i, w->n_seg)];
    c.bf16 = w->dtype == SD_BF16;
    c.y_bf16 = y_dtype == SD_BF16;
    c.a = w->a;
    c.b = w->b;
    c.scale = w->scale;
    c.ids = adapter;
    c.x = x;
    c.x_lo = x_lo;
    c.xs = x_stride;
    c.y_in = y_in;
    c.y_out = y_out;
    c.ys = y_in_stride;
    c.yos = y_out_stride;
    c.ws = workspace;
    sdv::launch_lora(c, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? SD_OK : SD_EHIP;
}

}  // extern "C"
