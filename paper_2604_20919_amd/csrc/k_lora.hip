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

// 16 bytes of a row of n elements from element k on, with what lies past its end
// to be dropped by `inside`, where they are used, so that nothing waits before:
// a branch for the lanes past the end would wait for the loads of the others, one
// piece after the other.  (Any alignment: the hardware takes 16-byte loads at
// every address.)  Lanes past the end read the row's start.  WHOLE: rows are whole
// pieces (229 rows, rank 16: 11.9 us, 12.5 without the difference); else a piece may
// reach into what follows the row, up to `end` (rank 12: 17 us, element by element 109).
template <bool WHOLE, typename T>
__device__ __forceinline__ typename Mma<T>::Frag piece(const T* row, int k, int n, const T* end) {
    constexpr int E = Mma<T>::kE;
    typename Mma<T>::Frag f;
    const T* from = row + (k < n ? k : 0);
    if (WHOLE || __all(from + E <= end)) {
        __builtin_memcpy(&f, from, 16);
    } else {
        T v[E];
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = row[k + i < n ? k + i : 0];
        __builtin_memcpy(&f, v, 16);
    }
    return f;
}
template <bool WHOLE, typename F> __device__ __forceinline__ F inside(F f, int k, int n) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(F) / sizeof(f[0])); ++i) f[i] = k + (WHOLE ? 0 : i) < n ? f[i] : 0;
    return f;
}
template <typename T> __device__ __forceinline__ typename Mma<T>::Frag piece(const T* row, int k) {
    typename Mma<T>::Frag f;
    __builtin_memcpy(&f, row + k, 16);
    return f;
}
// 16 bytes that no one else reads, past what the caches keep for others
template <typename T> __device__ __forceinline__ void load_once(T* to, const T* from) {
    typedef f32x4 Any __attribute__((aligned(2)));  // (at any address, as above)
    const f32x4 v = __builtin_nontemporal_load((const Any*)from);
    __builtin_memcpy(to, &v, 16);
}
// one by one, zeros past the end: the incomplete last piece of a row
template <typename T> __device__ __forceinline__ typename Mma<T>::Frag last_piece(const T* row, int k, int n) {
    constexpr int E = Mma<T>::kE;
    typename Mma<T>::Frag f;
    T v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const T x = row[k + i < n ? k + i : 0];
        v[i] = k + i < n ? x : (T)0;
    }
    __builtin_memcpy(&f, v, 16);
    return f;
}

// one rounding to the output's type (NaN stays NaN)
__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(bf16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t* p, float v) { *p = __builtin_bit_cast(bf16_t, (__bf16)v); }

// The adapters of a tile's 16 rows, one a lane (lane n: row n); -1: none
__device__ __forceinline__ int tile_id(const LoraCall& c, int t0, int lane) {
    const int t = t0 + lane;
    const int a = lane < 16 && t < c.T ? c.ids[t] : -1;
    return a >= 0 && a < c.n_adapters ? a : -1;
}

// h = A x: one workgroup a tile of 16 rows, a range of k, 64 of A's rows and every
// share-th of the tile's adapters (both in blockIdx.z), its waves taking 128-byte pieces
// of the rows in turn, their sums added in LDS and left as plane blockIdx.y of h
// ([planes][T][R]) that the second product adds up.  Bound by what it reads: 80 rows of
// 25600 in two planes with 16 adapters of rank 32, 34 MB, 16 us (one workgroup taking
// all of a tile's adapters: 52 us), 229 rows of 5120, 11 us (19); a plain read of 34 MB, one
// after the other, takes 7.5 us on the card.  Deeper unrolling, other orders of the
// pieces, twice the ranges of k or half the waves left both where they are.
template <typename T, int NW, bool LO>
__global__ __launch_bounds__(64 * NW) void k_lora_down(LoraCall c, float* h, int share) {
    typedef typename Mma<T>::Frag Frag;
    constexpr int E = Mma<T>::kE, KB = 8 * E, MT = 4;
    __shared__ f32x4 part[NW][MT][64];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const int t0 = blockIdx.x * 16, R = c.n_seg * c.rank;
    const int nkb = (c.d_in + KB - 1) / KB, full = c.d_in / KB;
    const int kb0 = (int)((int64_t)nkb * blockIdx.y / gridDim.y), kb1 = (int)((int64_t)nkb * (blockIdx.y + 1) / gridDim.y);
    const size_t xrow = (size_t)min(t0 + n, c.T - 1) * c.xs;
    const T* x = (const T*)c.x + xrow;
    const T* xl = LO ? (const T*)c.x_lo + xrow : nullptr;
    const int id = tile_id(c, t0, lane), mine = __shfl(id, n, 64);
    unsigned long long left = __ballot(id >= 0);
    for (int ord = 0; left; ++ord) {
        const int a = __builtin_amdgcn_readlane(id, __ffsll(left) - 1);
        left &= ~__ballot(id == a);
        if (ord % share != (int)blockIdx.z % share) continue;
        const int r0 = (int)blockIdx.z / share * 16 * MT, mt = min(MT, (R - r0 + 15) / 16);
        const T* A[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) A[m] = (const T*)c.a + ((size_t)a * R + min(r0 + 16 * m + n, R - 1)) * c.d_in;
        f32x4 acc[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto step = [&](int k, auto load) {
            Frag xf[2], xlf[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                xf[e] = load(x, k + e * E);
                if (LO) xlf[e] = load(xl, k + e * E);
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if (m >= mt) break;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const Frag af = load(A[m], k + e * E);
                    acc[m] = Mma<T>::run(af, xf[e], acc[m]);
                    if (LO) acc[m] = Mma<T>::run(af, xlf[e], acc[m]);
                }
            }
        };
        const int end = min(kb1, full);
        int kb = kb0 + w;
#pragma unroll 2
        for (; kb < end; kb += NW) step(kb * KB + 2 * E * g, [](const T* p, int k) { return piece(p, k); });
        if (kb < kb1)  // the row's last, incomplete piece
            step(kb * KB + 2 * E * g, [&](const T* p, int k) { return last_piece(p, k, c.d_in); });
#pragma unroll
        for (int m = 0; m < MT; ++m)
            if (m < mt) part[w][m][lane] = acc[m];
        __syncthreads();
        if (w < mt) {  // the tiles over the waves
            f32x4 s = part[0][w][lane];
#pragma unroll
            for (int i = 1; i < NW; ++i) s += part[i][w][lane];
            const int r = r0 + 16 * w + 4 * g;
            if (mine == a) {
                float* o = h + ((size_t)blockIdx.y * c.T + t0 + n) * R + r;
                if (r + 4 <= R) {
                    __builtin_memcpy(o, &s, 16);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (r + i < R) o[i] = s[i];
                }
            }
        }
        __syncthreads();
    }
}

// h of a row's segment as right operand: the sum of its planes, in bf16 carried
// on in three planes of its own that hold all of its 24 bits (three products; two
// planes, 16 bits, take as long at up to rank 64 with whole pieces: 21.3 against
// 21.4 us for 229 rows, 99.7 against 99.9 for 8192; dearer for many rows of other
// ranks, whose registers it is that bound them: 2000 rows of rank 12 25.5 against 26.2,
// of rank 50 25.5 against 28.3, 1024 of rank 128 50 against 52, with y in bf16 43 against 49)
template <typename T> constexpr int kInner = sizeof(T) == 2 ? 3 : 1;
template <typename T> struct Inner {
    typename Mma<T>::Frag p[kInner<T>];
};
// Each plane takes the eight highest bits that are left: nothing is rounded, and
// numbers next to the largest do not become infinite.  (An infinity or a
// not-a-number is in the first plane alone; inf - inf would make one of the other.)
__device__ __forceinline__ Inner<bf16_t> inner_planes(const float (&v)[8]) {
    Inner<bf16_t> r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(v[i]);
        float left = v[i] - __uint_as_float(a & 0xffff0000u);
        left = (a & 0x7f800000u) != 0x7f800000u ? left : 0.f;
        const uint32_t b = __float_as_uint(left);
        const uint32_t c = __float_as_uint(left - __uint_as_float(b & 0xffff0000u));
        r.p[0][i] = __builtin_bit_cast(__bf16, (uint16_t)(a >> 16));
        r.p[1][i] = __builtin_bit_cast(__bf16, (uint16_t)(b >> 16));
        r.p[2][i] = __builtin_bit_cast(__bf16, (uint16_t)(c >> 16));
    }
    return r;
}
__device__ __forceinline__ Inner<float> inner_planes(const float (&v)[4]) {
    Inner<float> r;
    __builtin_memcpy(&r.p[0], v, 16);
    return r;
}
// (pieces may reach past the row, the last one past the planes: the workspace does too)
template <typename T>
__device__ __forceinline__ Inner<T> inner_piece(const float* hr, int k, int rank, size_t stride, int planes) {
    constexpr int E = Mma<T>::kE;
    float v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = 0.f;
    const float* from = hr + (k < rank ? k : 0);
#pragma unroll 8
    for (int p = 0; p < planes; ++p) {
        float u[E];
        __builtin_memcpy(u, from + p * stride, sizeof(u));
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] += u[i];
    }
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = k + i < rank ? v[i] : 0.f;
    return inner_planes(v);
}

// y_out = y_in + scale B h: a wave takes 16 rows, `per` blocks of 16 CT columns
// and every gridDim.z-th of the rows' adapters.  A row's h, y and scale do not
// wait for the adapters: they are requested first, and each adapter's B while the
// one before is multiplied.  RB: steps of the product that hold the rank.  Bound by y
// and B: 229 rows of 10240 columns, 27 MB, 12 us; 80 rows of 5120, 8 us.
template <typename T, typename Y, int RB, bool WHOLE>
__global__ __launch_bounds__(256) void k_lora_up(LoraCall c, const float* h, int planes, int per) {
    typedef typename Mma<T>::Frag Frag;
    constexpr int E = Mma<T>::kE, CT = 4;
    constexpr int W = 16 / sizeof(Y), JW = W / 4;  // columns of a lane next to each other: from JW tiles
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const int t0 = blockIdx.x * 16, t = t0 + n, R = c.n_seg * c.rank;
    // the wave's first block of columns: segments are cut apart
    int b = (blockIdx.y * 4 + w) * per, s = 0;
    auto blocks = [&](int i) { return (c.seg[i + 1] - c.seg[i] + 16 * CT - 1) / (16 * CT); };
    while (s < c.n_seg && b >= blocks(s)) b -= blocks(s++);
    if (s == c.n_seg) return;
    const int id = tile_id(c, t0, lane);
    const size_t row = (size_t)min(t, c.T - 1);
    const Y* yi = (const Y*)c.y_in + row * c.ys;
    Y* yo = (Y*)c.y_out + row * c.yos;
    // tile q's row 4 g + i is this lane's column col(q) + i; left operand's row n is column lcol(q)
    auto col = [&](int q) { return (q / JW) * 16 * JW + W * g + 4 * (q % JW); };
    auto lcol = [&](int q) { return (q / JW) * 16 * JW + W * (n / 4) + 4 * (q % JW) + n % 4; };
    const T* b_end = (const T*)c.b + (size_t)c.n_adapters * c.d_out * c.rank;
    Inner<T> hv[RB];
    Y y[CT / JW][W];
    int have = -1;  // the segment of hv
    unsigned long long todo = 0;  // first rows of the adapters that are this workgroup's
    int mine = -1;
    bool write = false;
    float sc = 1.f;
    for (int i = 0; i < per; ++i) {
        const int c0 = c.seg[s] + b * 16 * CT, c1 = c.seg[s + 1];
        if (have != s) {
            have = s;
#pragma unroll
            for (int r = 0; r < RB; ++r)
                hv[r] = inner_piece<T>(h + row * R + s * c.rank, (4 * r + g) * E, c.rank, (size_t)c.T * R, planes);
        }
#pragma unroll
        for (int q = 0; q < CT / JW; ++q) {
            const int k = c0 + col(q * JW);
            if (k + W <= c1) {
                __builtin_memcpy(y[q], yi + k, 16);
            } else {
#pragma unroll
                for (int e = 0; e < W; ++e) y[q][e] = k + e < c1 ? yi[k + e] : (Y)0;
            }
        }
        if (i == 0) {
            mine = __shfl(id, n, 64);
            write = mine < 0 && t < c.T && blockIdx.z == 0 && c.y_in != c.y_out;
            unsigned long long left = __ballot(id >= 0);
            for (int ord = 0; left; ++ord) {
                const int f = __ffsll(left) - 1, a = __builtin_amdgcn_readlane(id, f);
                left &= ~__ballot(id == a);
                if (ord % gridDim.z != blockIdx.z) continue;
                todo |= 1ull << f;
                write |= mine == a;
            }
            if (!__ballot(write)) return;
            if (c.scale && mine >= 0) sc = c.scale[mine];
        }
        f32x4 out[CT];
#pragma unroll
        for (int q = 0; q < CT; ++q) out[q] = f32x4{0.f, 0.f, 0.f, 0.f};
        Frag bf[RB][CT];
        auto fetch = [&](int a) {
#pragma unroll
            for (int q = 0; q < CT; ++q) {
                const T* B = (const T*)c.b + ((size_t)a * c.d_out + min(c0 + lcol(q), c1 - 1)) * c.rank;
#pragma unroll
                for (int r = 0; r < RB; ++r) bf[r][q] = piece<WHOLE>(B, (4 * r + g) * E, c.rank, b_end);
            }
        };
        unsigned long long left = todo;
        int a = left ? __builtin_amdgcn_readlane(id, __ffsll(left) - 1) : -1;
        if (a >= 0) fetch(a);
        while (a >= 0) {
            left &= left - 1;
            const int next = left ? __builtin_amdgcn_readlane(id, __ffsll(left) - 1) : -1;
            f32x4 acc[CT];
#pragma unroll
            for (int q = 0; q < CT; ++q) {
                acc[q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    const Frag f = inside<WHOLE>(bf[r][q], (4 * r + g) * E, c.rank);
#pragma unroll
                    for (int i = 0; i < kInner<T>; ++i) acc[q] = Mma<T>::run(f, hv[r].p[i], acc[q]);
                }
            }
            if (next >= 0) fetch(next);
#pragma unroll
            for (int q = 0; q < CT; ++q)
#pragma unroll
                for (int e = 0; e < 4; ++e) out[q][e] = mine == a ? acc[q][e] : out[q][e];
            a = next;
        }
        if (write) {
#pragma unroll
            for (int q = 0; q < CT / JW; ++q) {
                const int k = c0 + col(q * JW);
                if (mine >= 0)
#pragma unroll
                    for (int e = 0; e < W; ++e) put(&y[q][e], as_float(y[q][e]) + sc * out[q * JW + e / 4][e % 4]);
                if (k + W <= c1) {
                    __builtin_memcpy(yo + k, y[q], 16);
                } else {
#pragma unroll
                    for (int e = 0; e < W; ++e)
                        if (k + e < c1) yo[k + e] = y[q][e];
                }
            }
        }
        if (++b == blocks(s)) {
            b = 0;
            if (++s == c.n_seg) return;
        }
    }
}

// Many rows: a workgroup takes kWideTile of them, a wave 16, and 16 MT of the adapter's
// rows go through LDS once for all waves (each wave loading them by itself took
// as long as x: 8192 rows of 8192, rank 64, 92 us against 46 without).
// Row tiles of the workgroup that have no row of the adapter skip the products.
constexpr int kWideWaves = 8, kWideTile = 16 * kWideWaves;

// The adapters of the workgroup's rows, one at a time: the lowest that is above
// `after`; -1: no more.  `ids`: the rows' adapters in LDS.
__device__ __forceinline__ int next_id(const int* ids, int after, int lane) {
    int best = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < kWideTile / 64; ++i) {
        const int v = ids[64 * i + lane];
        if (v > after) best = min(best, v);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) best = min(best, __shfl_xor(best, d, 64));
    return best == 0x7fffffff ? -1 : best;
}

// Workgroups next to each other in launch order take the same rows' next ranges
// of k; up to eight of them, one on each of the chip's dies, so that a die's L2
// holds its range of A (46 -> 42 us).
template <typename T, bool LO, int MT, int ST>
__global__ __launch_bounds__(64 * kWideWaves) void k_lora_down_wide(LoraCall c, float* h) {
    typedef typename Mma<T>::Frag Frag;
    constexpr int E = Mma<T>::kE, KC = 4 * E * ST;  // ST steps of the product a chunk
    constexpr int P = KC + E;  // elements between the rows in LDS: 16 rows' pieces in different banks
    __shared__ __align__(16) T as[2][16 * MT * P];
    __shared__ int ids[kWideTile];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const int t0 = blockIdx.y * kWideTile, R = c.n_seg * c.rank;
    const int nch = (c.d_in + KC - 1) / KC;
    const int ch0 = (int)((int64_t)nch * blockIdx.x / gridDim.x), ch1 = (int)((int64_t)nch * (blockIdx.x + 1) / gridDim.x);
    for (int i = tid; i < kWideTile; i += 64 * kWideWaves) {
        const int t = t0 + i, a = t < c.T ? c.ids[t] : -1;
        ids[i] = a >= 0 && a < c.n_adapters ? a : -1;
    }
    __syncthreads();
    const int t = t0 + 16 * w + n, mine = ids[16 * w + n];
    const T* x = (const T*)c.x + (size_t)min(t, c.T - 1) * c.xs;
    const T* xl = LO ? (const T*)c.x_lo + (size_t)min(t, c.T - 1) * c.xs : nullptr;
    for (int a = -1; (a = next_id(ids, a, lane)) >= 0;) {
        const bool part = __ballot(mine == a) != 0;
        for (int r0 = 0; r0 < R; r0 += 16 * MT) {
            const int rows = min(16 * MT, R - r0), mt = (rows + 15) / 16;
            const T* A = (const T*)c.a + ((size_t)a * R + r0) * c.d_in;
            // a chunk of A: 16 MT rows of ST * 4 pieces, two a thread
            constexpr int PP = 16 * MT * ST * 4 / (64 * kWideWaves);
            Frag st[PP];
            Frag xf[ST], xlf[ST];
            auto load = [&](int ch, auto get) {
#pragma unroll
                for (int i = 0; i < PP; ++i) {
                    const int q = tid + 64 * kWideWaves * i, r = q / (ST * 4);
                    st[i] = get(A + (size_t)min(r, rows - 1) * c.d_in, ch * KC + (q % (ST * 4)) * E);
                }
                if (!part) return;
#pragma unroll
                for (int e = 0; e < ST; ++e) {
                    xf[e] = get(x, ch * KC + (ST * g + e) * E);
                    if (LO) xlf[e] = get(xl, ch * KC + (ST * g + e) * E);
                }
            };
            auto fetch = [&](int ch) {
                if ((ch + 1) * KC <= c.d_in) load(ch, [](const T* p, int k) { return piece(p, k); });
                else load(ch, [&](const T* p, int k) { return last_piece(p, k, c.d_in); });
            };
            auto store = [&](int b) {
#pragma unroll
                for (int i = 0; i < PP; ++i) {
                    const int q = tid + 64 * kWideWaves * i;
                    *(Frag*)&as[b][(q / (ST * 4)) * P + (q % (ST * 4)) * E] = st[i];
                }
            };
            f32x4 acc[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
            // (tiles begin at different chunks: rows are often a power of two apart, and
            // everyone reading the same columns at once meets in few memory channels,
            // 62 against 50 us for 8192 rows of 8192)
            const int cn = ch1 - ch0, turn = cn > 0 ? (int)(blockIdx.y % cn) : 0;
            auto at = [&](int ch) { return ch + turn < ch1 ? ch + turn : ch + turn - cn; };
            if (ch0 < ch1) {
                fetch(at(ch0));
                store(0);
            }
            __syncthreads();
            for (int ch = ch0; ch < ch1; ++ch) {
                const int b = (ch - ch0) & 1;
                Frag xc[ST], xlc[ST];
#pragma unroll
                for (int e = 0; e < ST; ++e) {
                    xc[e] = xf[e];
                    if (LO) xlc[e] = xlf[e];
                }
                if (ch + 1 < ch1) fetch(at(ch + 1));
                if (part) {
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        if (m >= mt) break;
#pragma unroll
                        for (int e = 0; e < ST; ++e) {
                            const Frag af = *(const Frag*)&as[b][(16 * m + n) * P + (ST * g + e) * E];
                            acc[m] = Mma<T>::run(af, xc[e], acc[m]);
                            if (LO) acc[m] = Mma<T>::run(af, xlc[e], acc[m]);
                        }
                    }
                }
                if (ch + 1 < ch1) store(b ^ 1);
                __syncthreads();
            }
            if (mine == a) {
                float* o = h + ((size_t)blockIdx.x * c.T + t) * R + r0;
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const int r = 16 * m + 4 * g;
                    if (r + 4 <= rows) {
                        __builtin_memcpy(o + r, &acc[m], 16);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (r + i < rows) o[r + i] = acc[m][i];
                    }
                }
            }
        }
    }
}

// The planes of h added up, into the first.
__global__ __launch_bounds__(256) void k_lora_join(float* h, size_t n, int planes) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    float v = 0.f;
#pragma unroll 8
    for (int p = 0; p < planes; ++p) v += h[p * n + i];
    h[i] = v;
}

// Workgroups next to each other in launch order take the same rows' next columns:
// those that run together then have whole rows between them, not one piece of
// each row (8192 rows of 5120 columns, rank 64: 66 -> 60 us), and y passes by what
// the caches keep of B and h (60 -> 56 us).  Up to rank 64 two workgroups are on a
// CU (2000 rows of rank 12 26.2 us, 28.5 with one).
template <typename T, typename Y, int RB, bool WHOLE>
__global__ __launch_bounds__(64 * kWideWaves, RB * Mma<T>::kE <= 16 ? 4 : 2) void k_lora_up_wide(LoraCall c, const float* h, int per) {
    typedef typename Mma<T>::Frag Frag;
    constexpr int E = Mma<T>::kE, CT = 4;
    constexpr int W = 16 / sizeof(Y), JW = W / 4;
    constexpr int P = 4 * RB * E + E;  // elements between the columns' rows of B in LDS
    __shared__ __align__(16) T bs[2][16 * CT * P];
    __shared__ int ids[kWideTile];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const int t0 = blockIdx.y * kWideTile, R = c.n_seg * c.rank;
    int blk = blockIdx.x * per, seg0 = 0;
    auto blocks = [&](int s) { return (c.seg[s + 1] - c.seg[s] + 16 * CT - 1) / (16 * CT); };
    while (seg0 < c.n_seg && blk >= blocks(seg0)) blk -= blocks(seg0++);
    if (seg0 == c.n_seg) return;
    for (int i = tid; i < kWideTile; i += 64 * kWideWaves) {
        const int t = t0 + i, a = t < c.T ? c.ids[t] : -1;
        ids[i] = a >= 0 && a < c.n_adapters ? a : -1;
    }
    __syncthreads();
    const int t = t0 + 16 * w + n, mine = ids[16 * w + n];
    const Y* yi = (const Y*)c.y_in + (size_t)min(t, c.T - 1) * c.ys;
    Y* yo = (Y*)c.y_out + (size_t)min(t, c.T - 1) * c.yos;
    auto col = [&](int q) { return (q / JW) * 16 * JW + W * g + 4 * (q % JW); };
    auto lcol = [&](int q) { return (q / JW) * 16 * JW + W * (n / 4) + 4 * (q % JW) + n % 4; };
    const T* b_end = (const T*)c.b + (size_t)c.n_adapters * c.d_out * c.rank;
    // the next block of columns in place of (s, b); false: the wave's last, or the projection's
    int left = per;
    auto next_block = [&](int& s, int& b) {
        if (--left <= 0) return false;
        if (++b == blocks(s)) {
            b = 0;
            ++s;
        }
        return s < c.n_seg;
    };
    for (int a = -1; (a = next_id(ids, a, lane)) >= 0;) {
        const bool part = __ballot(mine == a) != 0;
        const float sc = c.scale ? c.scale[a] : 1.f;
        Inner<T> hv[RB];
        // B of a block of columns: 16 CT rows of 4 RB pieces
        constexpr int N = 16 * CT * 4 * RB, PP = (N + 64 * kWideWaves - 1) / (64 * kWideWaves);
        Frag st[PP];
        auto fetch = [&](int s, int b) {
            const int c0 = c.seg[s] + b * 16 * CT, c1 = c.seg[s + 1];
#pragma unroll
            for (int i = 0; i < PP; ++i) {
                const int q = tid + 64 * kWideWaves * i;
                if (N % (64 * kWideWaves) && q >= N) break;
                const T* row = (const T*)c.b + ((size_t)a * c.d_out + min(c0 + q / (4 * RB), c1 - 1)) * c.rank;
                st[i] = piece<WHOLE>(row, (q % (4 * RB)) * E, c.rank, b_end);
            }
        };
        auto store = [&](int buf) {
#pragma unroll
            for (int i = 0; i < PP; ++i) {
                const int q = tid + 64 * kWideWaves * i;
                if (N % (64 * kWideWaves) && q >= N) break;
                *(Frag*)&bs[buf][(q / (4 * RB)) * P + (q % (4 * RB)) * E] =
                    inside<WHOLE>(st[i], (q % (4 * RB)) * E, c.rank);
            }
        };
        Y y[CT / JW][W];
        auto fetch_y = [&](int s, int b) {
            if (mine != a) return;
            const int c0 = c.seg[s] + b * 16 * CT, c1 = c.seg[s + 1];
#pragma unroll
            for (int q = 0; q < CT / JW; ++q) {
                const int k = c0 + col(q * JW);
                if (k + W <= c1) {
                    load_once(y[q], yi + k);
                } else {
#pragma unroll
                    for (int i = 0; i < W; ++i)
                        if (k + i < c1) y[q][i] = yi[k + i];
                }
            }
        };
        int s = seg0, b = blk, have = -1;
        left = per;
        fetch(s, b);
        fetch_y(s, b);
        store(0);
        __syncthreads();
        for (int buf = 0;; buf ^= 1) {
            const int c0 = c.seg[s] + b * 16 * CT, c1 = c.seg[s + 1];
            if (have != s && part) {
                have = s;
                const float* hr = h + (size_t)min(t, c.T - 1) * R + s * c.rank;
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    const int k = (4 * r + g) * E;
                    float v[E];
                    __builtin_memcpy(v, hr + (k < c.rank ? k : 0), sizeof(v));
#pragma unroll
                    for (int i = 0; i < E; ++i) v[i] = k + i < c.rank ? v[i] : 0.f;
                    hv[r] = inner_planes(v);
                }
            }
            Y yc[CT / JW][W];
            __builtin_memcpy(yc, y, sizeof(y));
            const bool more = next_block(s, b);
            if (more) {
                fetch(s, b);
                fetch_y(s, b);
            }
            if (part) {
                f32x4 acc[CT];
#pragma unroll
                for (int q = 0; q < CT; ++q) {
                    acc[q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int r = 0; r < RB; ++r) {
                        const Frag bf = *(const Frag*)&bs[buf][lcol(q) * P + (4 * r + g) * E];
#pragma unroll
                        for (int i = 0; i < kInner<T>; ++i) acc[q] = Mma<T>::run(bf, hv[r].p[i], acc[q]);
                    }
                }
                if (mine == a) {
#pragma unroll
                    for (int q = 0; q < CT / JW; ++q) {
                        const int k = c0 + col(q * JW);
#pragma unroll
                        for (int i = 0; i < W; ++i)
                            put(&yc[q][i], as_float(yc[q][i]) + sc * acc[q * JW + i / 4][i % 4]);
                        if (k + W <= c1) {
                            __builtin_memcpy(yo + k, yc[q], 16);
                        } else {
#pragma unroll
                            for (int i = 0; i < W; ++i)
                                if (k + i < c1) yo[k + i] = yc[q][i];
                        }
                    }
                }
            }
            if (more) store(buf ^ 1);
            __syncthreads();
            if (!more) break;
        }
    }
    // rows without an adapter
    if (c.y_in == c.y_out || t >= c.T || mine >= 0) return;
    int s = seg0, b = blk;
    left = per;
    do {
        const int c0 = c.seg[s] + b * 16 * CT, c1 = c.seg[s + 1];
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
    } while (next_block(s, b));
}

// Launch shapes.  Tiles of 16 rows with up to kShare workgroups sharing out a
// tile's adapters, or (wide) of kWideTile rows, whose workgroup takes its adapters one after
// the other.  Wide is the faster the more rows, the more inner results a row and
// the longer the runs of one adapter, of which the host only knows the number of
// adapters there are; from kWideWork rows x inner results an adapter on (16 adapters
// at most) it mostly is.  us a call, tiles of 16 against wide, d_in 5120 / d_out
// 10240 in three segments or 8192 / 5120 in one:
//   one or two adapters, 24 inner results: 640 rows 24 / 28, 2047 rows 70 / 62
//   one or two adapters, 64: 400 rows 21 / 18, 1024 rows 42 / 26, 4096 rows 120 / 68
//   8 adapters in runs of 30, 16: 2047 rows 37 / 46; 64: 640 rows 40 / 35, 4096 rows 135 / 98
//   32 adapters in runs of 7, 16: 4096 rows 101 / 174; 64: 2047 rows 122 / 149, 4096 rows 239 / 233
// Ranges of k: about kGroups (kWideGroups) workgroups in all, a 128-byte piece a wave (a
// chunk of 256 bytes) at least.  More ranges make the first product shorter and the
// second longer, which adds them up (229 rows qkv 32B, 512 / 1024 groups: 13.3 +
// 10.9 / 10.7 + 11.7 us; wide, 8192 rows of 64, 512 / 1024 groups: 104 / 114 us; 32 ranges
// at most against 16: 640 rows of 64 23.5 / 26 us, but 2047 rows of 192 105 / 95).
constexpr int kWideRows = 384, kWideWork = 8192, kWideFew = 2, kWideMany = 16, kWideInner = 16;
constexpr int kGroups = 1024, kWideGroups = 512, kMaxPlanes = 8, kWidePlanes = 32, kShare = 8;
struct Shape {
    bool wide;
    int tiles, share, blocks, planes;  // blocks: of 64 of A's rows, apart
};
Shape shape_of(int T, int d_in, int es, int n_adapters, int R) {
    Shape s;
    s.wide = T >= kWideRows && (int64_t)T * std::max(R, kWideInner) >=
                                   (int64_t)kWideWork * std::max(kWideFew, std::min(n_adapters, kWideMany));
    const int rows = s.wide ? kWideTile : 16;
    s.tiles = (T + rows - 1) / rows;
    s.share = s.wide ? 1 : std::min(std::min(kShare, n_adapters), T);
    const int pieces = s.wide ? (d_in * es + 255) / 256 : (d_in * es + 127) / 128 / 8;
    s.blocks = s.wide ? 1 : (R + 63) / 64;
    const int groups = s.tiles * s.share * s.blocks, want = s.wide ? kWideGroups : kGroups;
    const int most = !s.wide ? kMaxPlanes : R <= 64 ? kWidePlanes : kWidePlanes / 2;
    s.planes = std::max(1, std::min(std::min((want + groups - 1) / groups, pieces), most));
    return s;
}

template <typename T, bool LO>
void launch_down(const LoraCall& c, const Shape& sh, float* h, hipStream_t s) {
    const dim3 g(sh.tiles, sh.planes, sh.share * sh.blocks), wide(64 * kWideWaves);
    if (sh.wide) {
        const dim3 gw(sh.planes, sh.tiles);
        if constexpr (LO) {
            // x is read once for each block of A's rows: 128 of them, in chunks half as
            // long (the registers), where there are more than 64 (8192 rows of 5120, two
            // planes: 96 of A's rows 281 -> 253 us with the second product, 192 rows 328 -> 314;
            // 63 rows, one block either way, 239 us with chunks half as long against 244, but
            // 2805 rows 98 against 94; x in one plane, 192 rows: 283 against 260)
            if (c.n_seg * c.rank > 64) {
                hipLaunchKernelGGL((k_lora_down_wide<T, true, 8, 2>), gw, wide, 0, s, c, h);
                return;
            }
        }
        hipLaunchKernelGGL((k_lora_down_wide<T, LO, 4, 4>), gw, wide, 0, s, c, h);
        return;
    }
    hipLaunchKernelGGL((k_lora_down<T, 8, LO>), g, dim3(512), 0, s, c, h, sh.share);
}
template <typename T, typename Y, int RB, bool WHOLE>
void launch_up(const LoraCall& c, const Shape& sh, float* h, hipStream_t s) {
    int blocks = 0;
    for (int i = 0; i < c.n_seg; ++i) blocks += (c.seg[i + 1] - c.seg[i] + 63) / 64;
    const int64_t units = (int64_t)blocks * sh.tiles;
    if (sh.wide) {
        const size_t n = (size_t)c.T * c.n_seg * c.rank;
        hipLaunchKernelGGL(k_lora_join, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, h, n, sh.planes);
        // as many blocks a workgroup as leave about four workgroups a CU
        const int per = std::max(1, (int)std::min<int64_t>(units / (4 * cu_count()), 16));
        const dim3 g((blocks + per - 1) / per, sh.tiles);
        hipLaunchKernelGGL((k_lora_up_wide<T, Y, RB, WHOLE>), g, dim3(64 * kWideWaves), 0, s, c, h, per);
        return;
    }
    // as many blocks a wave as leave about 16 waves a CU; with fewer than 8 a CU the
    // adapters of a tile are shared out as well
    const int per = std::max(1, (int)std::min<int64_t>(units / (16 * cu_count()), 16));
    const int share = std::max(1, std::min(sh.share, (int)(8 * cu_count() / units)));
    const int waves = (blocks + per - 1) / per;
    const dim3 g(sh.tiles, (waves + 3) / 4, share);
    hipLaunchKernelGGL((k_lora_up<T, Y, RB, WHOLE>), g, dim3(256), 0, s, c, h, sh.planes, per);
}
template <typename T, typename Y, bool WHOLE>
void launch_up_rank(const LoraCall& c, const Shape& sh, float* h, hipStream_t s) {
    constexpr int K = 4 * Mma<T>::kE;  // a step of the product
    if (c.rank <= 32) launch_up<T, Y, 32 / K, WHOLE>(c, sh, h, s);
    else if (c.rank <= 64) launch_up<T, Y, 64 / K, WHOLE>(c, sh, h, s);
    else launch_up<T, Y, 128 / K, WHOLE>(c, sh, h, s);
}
template <typename T>
void launch_typed(const LoraCall& c, hipStream_t s) {
    const Shape sh = shape_of(c.T, c.d_in, sizeof(T), c.n_adapters, c.n_seg * c.rank);
    float* h = (float*)c.ws;
    if constexpr (sizeof(T) == 2) {
        if (c.x_lo) launch_down<T, true>(c, sh, h, s);
        else launch_down<T, false>(c, sh, h, s);
    } else {
        launch_down<T, false>(c, sh, h, s);
    }
    if (c.rank % Mma<T>::kE == 0) {
        if (c.y_bf16) launch_up_rank<T, bf16_t, true>(c, sh, h, s);
        else launch_up_rank<T, float, true>(c, sh, h, s);
    } else {
        if (c.y_bf16) launch_up_rank<T, bf16_t, false>(c, sh, h, s);
        else launch_up_rank<T, float, false>(c, sh, h, s);
    }
}

}  // namespace

// (enough for every smaller T, rank and n_seg too: planes times rows, the rows rounded up to tiles)
size_t lora_workspace(int T, int rank, int n_seg, int d_in, int bf16) {
    const int planes = std::min(kWidePlanes, (d_in * (bf16 ? 2 : 4) + 255) / 256);
    const size_t rows = std::min((size_t)planes * T, (size_t)kWideTile * (kGroups + (T + 15) / 16));
    // (and a piece of 32 bytes past the end)
    return (rows * rank * n_seg * 4 + 32 + 255) & ~(size_t)255;
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
    *workspace_bytes = sdv::lora_workspace(n_rows, w->rank, w->n_seg, w->d_in, w->dtype == SD_BF16);
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
