// Low-rank adapters of many requests beside a shared projection:
// y[t] += scale[a] * B_a (A_a x[t]), a the adapter of row t.  Two products with
// the rank between them, both bound by what they read and write: A and B of the
// adapters in use for few rows, x and y for many.
#include <algorithm>

#include "../../include/sd_verify.h"
#include "sdv_device.h"
#include "sdv_internal.h"

namespace sdv {
namespace {

// Both products run on 16x16 matrix instructions with rows of the batch as the
// right operand's columns: D[m][n] = sum_k L[m][k] x[n][k], L the rows of A (or
// of B).  Rows of a tile that have different adapters are computed for each
// of them, and each row keeps its own: no row is moved, and an adapter's
// matrices are read once a tile.
//
// A lane (row l % 16, group l / 16) loads 16 bytes of a row at a time, kE
// elements; a step of the product is the four groups' pieces.  Two steps are
// interleaved so that the groups' pieces make 128 contiguous bytes of a row.
template <typename T> struct Mma;
template <> struct Mma<bf16_t> {
    static constexpr int kE = 8;
    typedef bf16x8 Frag;
    static __device__ __forceinline__ f32x4 run(Frag a, Frag b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Mma<float> {
    static constexpr int kE = 4;
    typedef f32x4 Frag;
    static __device__ __forceinline__ f32x4 run(Frag a, Frag b, f32x4 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};

// 16 bytes of a row from element k on, zeros from n on (any alignment: the
// hardware takes 16-byte loads at every address)
template <typename T> __device__ __forceinline__ typename Mma<T>::Frag piece(const T* row, int k, int n) {
    constexpr int E = Mma<T>::kE;
    typename Mma<T>::Frag f;
    if (k + E <= n) {
        __builtin_memcpy(&f, row + k, 16);
    } else {
        T v[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            v[i] = 0;
            if (k + i < n) v[i] = row[k + i];
        }
        __builtin_memcpy(&f, v, 16);
    }
    return f;
}
template <typename T> __device__ __forceinline__ typename Mma<T>::Frag piece(const T* row, int k) {
    typename Mma<T>::Frag f;
    __builtin_memcpy(&f, row + k, 16);
    return f;
}

// one rounding to the output's type (NaN stays NaN)
__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(bf16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t* p, float v) { *p = __builtin_bit_cast(bf16_t, (__bf16)v); }

// The adapters of a tile's rows, one a lane (lane n: row n); -1: none
__device__ __forceinline__ int tile_id(const LoraCall& c, int t0, int rows, int lane) {
    const int t = t0 + lane;
    const int a = lane < rows && t < c.T ? c.ids[t] : -1;
    return a >= 0 && a < c.n_adapters ? a : -1;
}

// h = A x: one workgroup a tile of 16 NT rows, a range of k and every gridDim.z-th
// of the tile's adapters, its waves taking 128-byte pieces of the rows in turn,
// their sums added in LDS and left as plane blockIdx.y of h ([planes][T][R]) that
// the second product adds up.
template <typename T, int NT, int NW, bool LO>
__global__ __launch_bounds__(64 * NW) void k_lora_down(LoraCall c, float* h) {
    typedef typename Mma<T>::Frag Frag;
    constexpr int E = Mma<T>::kE, KB = 8 * E, MT = 4;
    __shared__ f32x4 part[NW][MT * NT][64];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, n = lane & 15, g = lane >> 4;
    const int t0 = blockIdx.x * 16 * NT, R = c.n_seg * c.rank;
    const int nkb = (c.d_in + KB - 1) / KB, full = c.d_in / KB;
    const int kb0 = (int)((int64_t)nkb * blockIdx.y / gridDim.y), kb1 = (int)((int64_t)nkb * (blockIdx.y + 1) / gridDim.y);
    const T *x[NT], *xl[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const size_t at = (size_t)min(t0 + 16 * j + n, c.T - 1) * c.xs;
        x[j] = (const T*)c.x + at;
        xl[j] = LO ? (const T*)c.x_lo + at : nullptr;
    }
    const int id = tile_id(c, t0, 16 * NT, lane);
    unsigned long long left = __ballot(id >= 0);
    for (int ord = 0; left; ++ord) {
        const int a = __builtin_amdgcn_readlane(id, __ffsll(left) - 1);
        left &= ~__ballot(id == a);
        if (ord % gridDim.z != blockIdx.z) continue;
        for (int r0 = 0; r0 < R; r0 += 16 * MT) {
            const int mt = min(MT, (R - r0 + 15) / 16);
            const T* A[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) A[m] = (const T*)c.a + ((size_t)a * R + min(r0 + 16 * m + n, R - 1)) * c.d_in;
            f32x4 acc[MT][NT];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            auto step = [&](int k, auto load) {
                Frag xf[NT][2], xlf[NT][2];
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        xf[j][e] = load(x[j], k + e * E);
                        if (LO) xlf[j][e] = load(xl[j], k + e * E);
                    }
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    if (m >= mt) break;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const Frag af = load(A[m], k + e * E);
#pragma unroll
                        for (int j = 0; j < NT; ++j) {
                            acc[m][j] = Mma<T>::run(af, xf[j][e], acc[m][j]);
                            if (LO) acc[m][j] = Mma<T>::run(af, xlf[j][e], acc[m][j]);
                        }
                    }
                }
            };
            const int end = min(kb1, full);
            int kb = kb0 + w;
#pragma unroll 2
            for (; kb < end; kb += NW) step(kb * KB + 2 * E * g, [](const T* p, int k) { return piece(p, k); });
            if (kb < kb1)  // the row's last, incomplete piece
                step(kb * KB + 2 * E * g, [&](const T* p, int k) { return piece(p, k, c.d_in); });
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    if (m < mt) part[w][m * NT + j][lane] = acc[m][j];
            __syncthreads();
            // (m, j) tiles over the waves
            for (int q = w; q < mt * NT; q += NW) {
                const int m = q / NT, j = q % NT;
                f32x4 s = part[0][q][lane];
#pragma unroll
                for (int i = 1; i < NW; ++i) s += part[i][q][lane];
                const int t = t0 + 16 * j + n, r = r0 + 16 * m + 4 * g;
                if (__shfl(id, 16 * j + n, 64) == a) {
                    float* o = h + ((size_t)blockIdx.y * c.T + t) * R + r;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (r + i < R) o[i] = s[i];
                }
            }
            __syncthreads();
        }
    }
}

// y_out = y_in + scale B h: a wave takes 16 NT rows, `per` blocks of 16 CT columns
// and every gridDim.z-th of the rows' adapters.  h is the sum of its planes, in
// bf16 as two planes of its own (hi + lo, about 16 bits, two products), kept
// in registers over the wave's columns.  RB: steps of the product that hold the rank.
template <typename T, typename Y, int NT, int RB>
__global__ __launch_bounds__(256) void k_lora_up(LoraCall c, const float* h, int planes, int per) {
    typedef typename Mma<T>::Frag Frag;
    constexpr int E = Mma<T>::kE, CT = 4;
    constexpr int W = 16 / sizeof(Y), JW = W / 4;  // columns of a lane next to each other: from JW tiles
    constexpr bool LO = sizeof(T) == 2;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, n = lane & 15, g = lane >> 4;
    const int t0 = blockIdx.x * 16 * NT, R = c.n_seg * c.rank;
    // the wave's first block of columns: segments are cut apart
    int blk = (blockIdx.y * 4 + w) * per, seg0 = 0;
    auto blocks = [&](int s) { return (c.seg[s + 1] - c.seg[s] + 16 * CT - 1) / (16 * CT); };
    while (seg0 < c.n_seg && blk >= blocks(seg0)) blk -= blocks(seg0++);
    if (seg0 == c.n_seg) return;
    const int id = tile_id(c, t0, 16 * NT, lane);
    unsigned long long left = __ballot(id >= 0);
    int mine[NT];  // the adapter of the lane's row
#pragma unroll
    for (int j = 0; j < NT; ++j) mine[j] = __shfl(id, 16 * j + n, 64);
    // tile q's row 4 g + i is this lane's column col(q) + i; left operand's row n is column lcol(q)
    auto col = [&](int q) { return (q / JW) * 16 * JW + W * g + 4 * (q % JW); };
    auto lcol = [&](int q) { return (q / JW) * 16 * JW + W * (n / 4) + 4 * (q % JW) + n % 4; };
    // blocks of columns from the wave's first on
    auto each_block = [&](auto f) {
        int s = seg0, b = blk;
        for (int i = 0; i < per; ++i) {
            f(s, c.seg[s] + b * 16 * CT, c.seg[s + 1]);
            if (++b == blocks(s)) {
                b = 0;
                if (++s == c.n_seg) break;
            }
        }
    };
    for (int ord = 0; left; ++ord) {
        const int a = __builtin_amdgcn_readlane(id, __ffsll(left) - 1);
        left &= ~__ballot(id == a);
        if (ord % gridDim.z != blockIdx.z) continue;
        const float sc = c.scale ? c.scale[a] : 1.f;
        Frag hf[NT][RB], lf[NT][RB];
        int have = -1;  // the segment whose h they hold
        each_block([&](int seg, int c0, int c1) {
            Frag bf[RB][CT];
#pragma unroll
            for (int q = 0; q < CT; ++q) {
                const T* B = (const T*)c.b + ((size_t)a * c.d_out + min(c0 + lcol(q), c1 - 1)) * c.rank;
#pragma unroll
                for (int r = 0; r < RB; ++r) bf[r][q] = piece(B, (4 * r + g) * E, c.rank);
            }
            Y y[NT][CT / JW][W];
#pragma unroll
            for (int j = 0; j < NT; ++j)
                if (mine[j] == a) {
                    const Y* yi = (const Y*)c.y_in + (size_t)(t0 + 16 * j + n) * c.ys;
#pragma unroll
                    for (int q = 0; q < CT / JW; ++q) {
                        const int k = c0 + col(q * JW);
                        if (k + W <= c1) {
                            __builtin_memcpy(y[j][q], yi + k, 16);
                        } else {
#pragma unroll
                            for (int i = 0; i < W; ++i)
                                if (k + i < c1) y[j][q][i] = yi[k + i];
                        }
                    }
                }
            if (have != seg) {
                have = seg;
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    // (rows of other adapters may hold anything: their columns are not used)
                    const float* hr = h + (size_t)min(t0 + 16 * j + n, c.T - 1) * R + seg * c.rank;
#pragma unroll
                    for (int r = 0; r < RB; ++r) {
                        const int k = (4 * r + g) * E;
                        float v[E];
#pragma unroll
                        for (int i = 0; i < E; ++i) v[i] = 0.f;
                        if (k + E <= c.rank) {
#pragma unroll 4
                            for (int p = 0; p < planes; ++p) {
                                float u[E];
                                __builtin_memcpy(u, hr + (size_t)p * c.T * R + k, sizeof(u));
#pragma unroll
                                for (int i = 0; i < E; ++i) v[i] += u[i];
                            }
                        } else {
                            for (int p = 0; p < planes; ++p)
#pragma unroll
                                for (int i = 0; i < E; ++i)
                                    if (k + i < c.rank) v[i] += hr[(size_t)p * c.T * R + k + i];
                        }
                        if constexpr (LO) {
#pragma unroll
                            for (int i = 0; i < E; ++i) {
                                hf[j][r][i] = (__bf16)v[i];
                                lf[j][r][i] = (__bf16)(v[i] - (float)hf[j][r][i]);
                            }
                        } else {
                            __builtin_memcpy(&hf[j][r], v, 16);
                        }
                    }
                }
            }
            f32x4 acc[CT][NT];
#pragma unroll
            for (int q = 0; q < CT; ++q)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    acc[q][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int r = 0; r < RB; ++r) {
                        acc[q][j] = Mma<T>::run(bf[r][q], hf[j][r], acc[q][j]);
                        if constexpr (LO) acc[q][j] = Mma<T>::run(bf[r][q], lf[j][r], acc[q][j]);
                    }
                }
#pragma unroll
            for (int j = 0; j < NT; ++j)
                if (mine[j] == a) {
                    Y* yo = (Y*)c.y_out + (size_t)(t0 + 16 * j + n) * c.yos;
#pragma unroll
                    for (int q = 0; q < CT / JW; ++q) {
                        const int k = c0 + col(q * JW);
#pragma unroll
                        for (int i = 0; i < W; ++i)
                            put(&y[j][q][i], as_float(y[j][q][i]) + sc * acc[q * JW + i / 4][j][i % 4]);
                        if (k + W <= c1) {
                            __builtin_memcpy(yo + k, y[j][q], 16);
                        } else {
#pragma unroll
                            for (int i = 0; i < W; ++i)
                                if (k + i < c1) yo[k + i] = y[j][q][i];
                        }
                    }
                }
        });
    }
    // rows without an adapter
    if (c.y_in == c.y_out || blockIdx.z) return;
    each_block([&](int, int c0, int c1) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int t = t0 + 16 * j + n;
            if (t >= c.T || mine[j] >= 0) continue;
            const Y* yi = (const Y*)c.y_in + (size_t)t * c.ys;
            Y* yo = (Y*)c.y_out + (size_t)t * c.yos;
#pragma unroll
            for (int q = 0; q < CT / JW; ++q) {
                const int k = c0 + col(q * JW);
                if (k + W <= c1) {
                    __builtin_memcpy(yo + k, yi + k, 16);
                } else {
#pragma unroll
                    for (int i = 0; i < W; ++i)
                        if (k + i < c1) yo[k + i] = yi[k + i];
                }
            }
        }
    });
}

// Launch shapes.  Few rows: tiles of 16, up to kShare workgroups sharing out a
// tile's adapters; many: tiles of 32.  Ranges of k: about kDownGroups workgroups
// in all, a 128-byte piece a wave at least.
constexpr int kWideRows = 2048;
constexpr int kDownGroups = 512, kMaxPlanes = 16, kShare = 8;
struct Shape {
    int rows, waves, tiles, share, planes;
};
Shape shape_of(int T, int d_in, int es, int n_adapters) {
    Shape s;
    const bool wide = T >= kWideRows;
    s.rows = wide ? 32 : 16;
    s.waves = 8;
    s.tiles = (T + s.rows - 1) / s.rows;
    s.share = wide ? 1 : std::min(std::min(kShare, n_adapters), T);
    const int pieces = (d_in * es + 127) / 128, groups = s.tiles * std::min(s.share, 4);
    s.planes = std::max(1, std::min(std::min((kDownGroups + groups - 1) / groups, pieces / s.waves), kMaxPlanes));
    return s;
}

template <typename T, int NT>
void launch_down(const LoraCall& c, const Shape& sh, float* h, hipStream_t s) {
    const dim3 g(sh.tiles, sh.planes, sh.share);
    if constexpr (sizeof(T) == 2) {
        if (c.x_lo) {
            hipLaunchKernelGGL((k_lora_down<T, NT, 8, true>), g, dim3(512), 0, s, c, h);
            return;
        }
    }
    hipLaunchKernelGGL((k_lora_down<T, NT, 8, false>), g, dim3(512), 0, s, c, h);
}
template <typename T, int NT, int RB>
void launch_up(const LoraCall& c, const Shape& sh, const float* h, hipStream_t s) {
    int blocks = 0;
    for (int i = 0; i < c.n_seg; ++i) blocks += (c.seg[i + 1] - c.seg[i] + 63) / 64;
    // as many blocks a wave as leave about 16 waves a CU
    const int per = std::max(1, (int)std::min<int64_t>((int64_t)blocks * sh.tiles / (16 * cu_count()), 16));
    const int waves = (blocks + per - 1) / per;
    const dim3 g(sh.tiles, (waves + 3) / 4, sh.share);
    if (c.y_bf16) hipLaunchKernelGGL((k_lora_up<T, bf16_t, NT, RB>), g, dim3(256), 0, s, c, h, sh.planes, per);
    else hipLaunchKernelGGL((k_lora_up<T, float, NT, RB>), g, dim3(256), 0, s, c, h, sh.planes, per);
}
template <typename T, int NT>
void launch_both(const LoraCall& c, const Shape& sh, hipStream_t s) {
    float* h = (float*)c.ws;
    launch_down<T, NT>(c, sh, h, s);
    constexpr int K = 4 * Mma<T>::kE;  // a step of the product
    if (c.rank <= 32) launch_up<T, NT, 32 / K>(c, sh, h, s);
    else if (c.rank <= 64) launch_up<T, NT, 64 / K>(c, sh, h, s);
    else launch_up<T, NT, 128 / K>(c, sh, h, s);
}
template <typename T>
void launch_typed(const LoraCall& c, hipStream_t s) {
    const Shape sh = shape_of(c.T, c.d_in, sizeof(T), c.n_adapters);
    if (sh.rows == 16) launch_both<T, 1>(c, sh, s);
    else launch_both<T, 2>(c, sh, s);
}

}  // namespace

// (enough for every smaller T too: planes times rows, the rows rounded up to tiles)
size_t lora_workspace(int T, int rank, int n_seg) {
    const size_t rows = std::min((size_t)kMaxPlanes * T, (size_t)32 * (kDownGroups + (T + 15) / 16));
    return (rows * rank * n_seg * 4 + 255) & ~(size_t)255;
}

void launch_lora(const LoraCall& c, hipStream_t s) {
    if (c.bf16) launch_typed<bf16_t>(c, s);
    else launch_typed<float>(c, s);
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
