// Gated feed-forward block and dropout, forward and backward, for AMD gfx950 (wave64): kernels and C ABI
// (include/zvc_ffn.h has the formulas).

#include "zvc_ffn.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

namespace {

using bf16 = __bf16;
using fp16 = _Float16;

inline size_t div_up(size_t a, size_t b) { return (a + b - 1) / b; }
inline size_t round_up(size_t a, size_t b) { return div_up(a, b) * b; }

// ------------------------------------------------------------------ dropout
// What a kernel needs to drop: the 32-bit fraction in its upper and lower half, the factor of what stays.
struct Drop {
    unsigned high, low;                // high: up to 65536, at which everything goes
    float scale;
    uint64_t seed, offset;
    const uint64_t* d_offset;
    bool active;
};

struct Words {
    unsigned w[4];
};

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011): a block cipher's rounds of two 32 x 32 bit products each.
__device__ __forceinline__ Words philox(uint64_t index, uint64_t offset, uint64_t seed) {
    unsigned c0 = static_cast<unsigned>(index), c1 = static_cast<unsigned>(index >> 32);
    unsigned c2 = static_cast<unsigned>(offset), c3 = static_cast<unsigned>(offset >> 32);
    unsigned k0 = static_cast<unsigned>(seed), k1 = static_cast<unsigned>(seed >> 32);
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t a = static_cast<uint64_t>(0xD2511F53u) * c0, b = static_cast<uint64_t>(0xCD9E8D57u) * c2;
        c0 = static_cast<unsigned>(b >> 32) ^ c1 ^ k0;
        c1 = static_cast<unsigned>(b);
        c2 = static_cast<unsigned>(a >> 32) ^ c3 ^ k1;
        c3 = static_cast<unsigned>(a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// Bit j: element 8 * group + j stays.  16 bits decide, but for one in 65536 elements, where 16 more do.
__device__ __forceinline__ unsigned keep_group(const Drop& d, uint64_t offset, uint64_t group) {
    const Words r = philox(group, offset, d.seed);
    unsigned keep = 0, tie = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const unsigned half = (r.w[j / 2] >> (16 * (j % 2))) & 0xFFFFu;
        keep |= static_cast<unsigned>(half >= d.high) << j;
        tie |= static_cast<unsigned>(half == d.high) << j;
    }
    if (d.low != 0 && tie != 0) {
        const Words more = philox(group | (uint64_t{1} << 63), offset, d.seed);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned half = (more.w[j / 2] >> (16 * (j % 2))) & 0xFFFFu;
            if ((tie >> j & 1u) != 0 && half < d.low) keep &= ~(1u << j);
        }
    }
    return keep;
}

// Bits for elements first .. first + 7, wherever they begin.
__device__ __forceinline__ unsigned keep_span(const Drop& d, uint64_t offset, uint64_t first) {
    const unsigned shift = static_cast<unsigned>(first & 7);
    unsigned keep = keep_group(d, offset, first >> 3);
    if (shift != 0) keep |= keep_group(d, offset, (first >> 3) + 1) << 8;
    return (keep >> shift) & 0xFFu;
}

__device__ __forceinline__ uint64_t effective_offset(const Drop& d) {
    return d.offset + (d.d_offset != nullptr ? *d.d_offset : 0);
}

// Eight consecutive elements, held in 32 bits.
struct Eight {
    float v[8];
};

template <typename T>
struct alignas(16) Pack {
    T v[16 / sizeof(T)];
};

template <typename T>
__device__ __forceinline__ Eight load8(const T* at) {          // 16-byte aligned
    Eight out;
    constexpr int kPer = 16 / sizeof(T);
#pragma unroll
    for (int h = 0; h < 8 / kPer; ++h) {
        const Pack<T> p = reinterpret_cast<const Pack<T>*>(at)[h];
#pragma unroll
        for (int j = 0; j < kPer; ++j) out.v[h * kPer + j] = static_cast<float>(p.v[j]);
    }
    return out;
}

template <typename T>
__device__ __forceinline__ void store8(T* at, const Eight& e) {   // 16-byte aligned
    constexpr int kPer = 16 / sizeof(T);
#pragma unroll
    for (int h = 0; h < 8 / kPer; ++h) {
        Pack<T> p;
#pragma unroll
        for (int j = 0; j < kPer; ++j) p.v[j] = static_cast<T>(e.v[h * kPer + j]);
        reinterpret_cast<Pack<T>*>(at)[h] = p;
    }
}

constexpr int kDropThreads = 256;

// y = drop(x) [+ residual].  A lane owns eight consecutive elements, one counter of the generator.  VECTOR: every
// row's groups of eight lie at multiples of 16 bytes, and no group straddles two rows.
template <typename T, bool VECTOR>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(const T* x, size_t ldx, const T* residual, size_t ldr,
                                                               T* y, size_t ldy, size_t cols, uint64_t total, Drop d) {
    const uint64_t group = static_cast<uint64_t>(blockIdx.x) * kDropThreads + threadIdx.x;
    const uint64_t first = group * 8;
    if (first >= total) return;
    const unsigned keep = d.active ? keep_group(d, effective_offset(d), group) : 0xFFu;
    uint64_t row = first / cols, col = first - row * cols;
    if constexpr (VECTOR) {
        Eight e = load8(x + row * ldx + col);
#pragma unroll
        for (int j = 0; j < 8; ++j) e.v[j] = (keep >> j & 1u) ? e.v[j] * d.scale : 0.f;
        if (residual != nullptr) {
            const Eight r = load8(residual + row * ldr + col);
#pragma unroll
            for (int j = 0; j < 8; ++j) e.v[j] += r.v[j];
        }
        store8(y + row * ldy + col, e);
    } else {
        for (int j = 0; j < 8 && first + j < total; ++j) {
            float v = (keep >> j & 1u) ? static_cast<float>(x[row * ldx + col]) * d.scale : 0.f;
            if (residual != nullptr) v += static_cast<float>(residual[row * ldr + col]);
            y[row * ldy + col] = static_cast<T>(v);
            if (++col == cols) col = 0, ++row;
        }
    }
}

// ------------------------------------------------------------------ the activation
struct ActValue {
    float value, slope;
};

__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + __expf(-x)); }

// act(g) and its derivative.  relu: a NaN is not <= 0 and stays.
__device__ __forceinline__ ActValue activate(int act, float g) {
    if (act == ZVC_RELU) return {g <= 0.f ? 0.f : g, g <= 0.f ? 0.f : 1.f};
    if (act == ZVC_SILU) {
        const float s = sigmoid(g);
        return {g * s, s + g * s * (1.f - s)};
    }
    if (act == ZVC_GELU) {
        const float cdf = 0.5f * erfcf(-0.70710678f * g);
        return {g * cdf, cdf + g * 0.39894228f * __expf(-0.5f * g * g)};
    }
    // (1 + tanh(z)) / 2 = sigmoid(2 z)
    const float s = sigmoid(1.5957691f * (g + 0.044715f * g * g * g));
    return {g * s, s + g * s * (1.f - s) * 1.5957691f * (1.f + 0.134145f * g * g)};
}

// ------------------------------------------------------------------ the block
constexpr int kTile = 64, kStep = 16, kTileThreads = 256;

// An operand of a product: element (index, reduction) at at[index * by_index + reduction * by_step].
template <typename T>
struct Operand {
    const T* at;
    size_t by_index, by_step;
};

// acc[i][j] += sum over the reduction of rows (4 ty + i) x columns (4 tx + j) of a 64 x 64 tile.
template <typename T>
__device__ void tile_product(float (&acc)[4][4], Operand<T> rows, size_t row0, size_t m, Operand<T> cols, size_t col0,
                             size_t n, size_t steps) {
    __shared__ float a[kStep][kTile + 1], b[kStep][kTile + 1];
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (size_t s0 = 0; s0 < steps; s0 += kStep) {
        for (int i = threadIdx.x; i < kTile * kStep; i += kTileThreads) {
            const int t = rows.by_step == 1 ? i % kStep : i / kTile, r = rows.by_step == 1 ? i / kStep : i % kTile;
            a[t][r] = row0 + r < m && s0 + t < steps
                          ? static_cast<float>(rows.at[(row0 + r) * rows.by_index + (s0 + t) * rows.by_step]) : 0.f;
        }
        for (int i = threadIdx.x; i < kTile * kStep; i += kTileThreads) {
            const int t = cols.by_step == 1 ? i % kStep : i / kTile, c = cols.by_step == 1 ? i / kStep : i % kTile;
            b[t][c] = col0 + c < n && s0 + t < steps
                          ? static_cast<float>(cols.at[(col0 + c) * cols.by_index + (s0 + t) * cols.by_step]) : 0.f;
        }
        __syncthreads();
        for (int t = 0; t < kStep; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] += a[t][4 * ty + i] * b[t][4 * tx + j];
        __syncthreads();
    }
}

template <typename T>
struct GluArgs {
    const T *x, *wg, *wu, *dh;
    const T *gate_in, *up_in;
    T *h, *gate, *up, *dg, *du;
    size_t ldx, ldw, lddh, ldh, ldp, ldd, m, n, k;
    int act;
    Drop d;
};

// Forward (dh null): h, and gate and up where wanted.  Backward (dh not null): dg and du.
template <typename T>
__device__ void finish_element(const GluArgs<T>& p, uint64_t offset, size_t row, size_t col, float g, float u) {
    const uint64_t i = static_cast<uint64_t>(row) * p.n + col;
    const bool keep = !p.d.active || (keep_group(p.d, offset, i >> 3) >> (i & 7) & 1u);
    const ActValue a = activate(p.act, g);
    if (p.dh != nullptr) {
        const float dh = keep ? static_cast<float>(p.dh[row * p.lddh + col]) * p.d.scale : 0.f;
        p.dg[row * p.ldd + col] = static_cast<T>(p.act == ZVC_RELU ? (g <= 0.f ? 0.f : dh * u) : dh * u * a.slope);
        p.du[row * p.ldd + col] = static_cast<T>(dh * a.value);
        return;
    }
    p.h[row * p.ldh + col] = static_cast<T>(keep ? a.value * u * p.d.scale : 0.f);
    if (p.gate != nullptr) {
        const bool relu = p.act == ZVC_RELU;
        p.gate[row * p.ldp + col] = static_cast<T>(!keep ? 0.f : relu ? a.value : g);
        p.up[row * p.ldp + col] = static_cast<T>(!keep || (relu && g <= 0.f) ? 0.f : u);
    }
}

template <typename T>
__global__ __launch_bounds__(kTileThreads) void glu_project_kernel(GluArgs<T> p) {
    const size_t row0 = static_cast<size_t>(blockIdx.y) * kTile, col0 = static_cast<size_t>(blockIdx.x) * kTile;
    float g[4][4] = {}, u[4][4] = {};
    tile_product<T>(g, {p.x, p.ldx, 1}, row0, p.m, {p.wg, p.ldw, 1}, col0, p.n, p.k);
    tile_product<T>(u, {p.x, p.ldx, 1}, row0, p.m, {p.wu, p.ldw, 1}, col0, p.n, p.k);
    const uint64_t offset = effective_offset(p.d);
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const size_t row = row0 + 4 * (threadIdx.x / 16) + i, col = col0 + 4 * (threadIdx.x % 16) + j;
            if (row < p.m && col < p.n) finish_element(p, offset, row, col, g[i][j], u[i][j]);
        }
}

// dg and du from kept projections.
template <typename T>
__global__ __launch_bounds__(256) void glu_slope_kernel(GluArgs<T> p) {
    const uint64_t offset = effective_offset(p.d);
    const uint64_t step = static_cast<uint64_t>(gridDim.x) * 256;
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; i < static_cast<uint64_t>(p.m) * p.n; i += step) {
        const size_t row = i / p.n, col = i - row * p.n;
        finish_element(p, offset, row, col, static_cast<float>(p.gate_in[row * p.ldp + col]),
                       static_cast<float>(p.up_in[row * p.ldp + col]));
    }
}

// out (rows x cols, stride ld) = a1 b1 + a2 b2, the second where a2.at is not null.
template <typename T>
__global__ __launch_bounds__(kTileThreads) void product_kernel(Operand<T> a1, Operand<T> b1, Operand<T> a2, Operand<T> b2,
                                                               T* out, size_t ld, size_t rows, size_t cols, size_t steps) {
    const size_t row0 = static_cast<size_t>(blockIdx.y) * kTile, col0 = static_cast<size_t>(blockIdx.x) * kTile;
    float acc[4][4] = {};
    tile_product<T>(acc, a1, row0, rows, b1, col0, cols, steps);
    if (a2.at != nullptr) tile_product<T>(acc, a2, row0, rows, b2, col0, cols, steps);
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const size_t row = row0 + 4 * (threadIdx.x / 16) + i, col = col0 + 4 * (threadIdx.x % 16) + j;
            if (row < rows && col < cols) out[row * ld + col] = static_cast<T>(acc[i][j]);
        }
}

// ------------------------------------------------------------------ host side
template <typename K, typename... A>
zvc_status launch(K kernel, dim3 grid, unsigned threads, hipStream_t stream, A... args) {
    (void)hipGetLastError();
    hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, args...);
    return hipGetLastError() == hipSuccess ? ZVC_OK : ZVC_E_HIP;
}

inline size_t type_bytes(int type) { return type == ZVC_FP32 ? 4 : type == ZVC_FP16 || type == ZVC_BF16 ? 2 : 0; }
inline bool aligned_to(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// A rows x cols matrix with a row stride, all in bytes but rows.
struct Region {
    const void* at;
    size_t ld, rows, cols;
    size_t bytes() const { return rows == 0 || cols == 0 ? 0 : (rows - 1) * ld + cols; }
};

// Whether two share a byte; rows that interleave at the same stride do not.
bool overlap(const Region& a, const Region& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
    if (a.at == nullptr || b.at == nullptr || a.bytes() == 0 || b.bytes() == 0) return false;
    if (x + a.bytes() <= y || y + b.bytes() <= x) return false;
    if (a.ld != b.ld || a.rows <= 1 || b.rows <= 1) return true;
    const size_t gap = y >= x ? (y - x) % a.ld : (a.ld - (x - y) % a.ld) % a.ld;
    return !(gap >= a.cols && gap + b.cols <= a.ld);
}

zvc_status make_drop(uint64_t drop, uint64_t seed, uint64_t offset, const uint64_t* d_offset, Drop* out) {
    if (drop > (uint64_t{1} << 32)) return ZVC_E_ARG;
    if (!aligned_to(d_offset, 8)) return ZVC_E_ALIGN;
    const double stays = 1.0 - static_cast<double>(drop) / 4294967296.0;
    *out = {static_cast<unsigned>(drop >> 16), static_cast<unsigned>(drop & 0xFFFF),
            stays > 0 ? static_cast<float>(1.0 / stays) : 0.f, seed, offset, d_offset, drop != 0};
    return ZVC_OK;
}

template <typename T>
zvc_status dropout_as(const void* x, size_t ldx, const void* residual, size_t ldr, void* y, size_t ldy, size_t rows,
                      size_t cols, const Drop& d, hipStream_t stream) {
    if (ldx == cols && ldy == cols && (residual == nullptr || ldr == cols)) cols *= rows, rows = 1, ldx = ldy = ldr = cols;
    const uint64_t total = static_cast<uint64_t>(rows) * cols;
    const bool vector = cols % 8 == 0 && aligned_to(x, 16) && aligned_to(y, 16) && aligned_to(residual, 16) &&
                        (rows == 1 || (ldx * sizeof(T) % 16 == 0 && ldy * sizeof(T) % 16 == 0 &&
                                       (residual == nullptr || ldr * sizeof(T) % 16 == 0)));
    const size_t blocks = div_up(div_up(total, 8), kDropThreads);
    if (blocks > 0x7FFFFFFF) return ZVC_E_ARG;
    return launch(vector ? dropout_kernel<T, true> : dropout_kernel<T, false>, dim3(blocks), kDropThreads, stream,
                  static_cast<const T*>(x), ldx, static_cast<const T*>(residual), ldr, static_cast<T*>(y), ldy, cols, total, d);
}

// Where the parts of a workspace begin.
struct Layout {
    size_t dg, du, bytes;
};

Layout layout_of(size_t m, size_t n, size_t k, size_t w, bool backward) {
    (void)k;
    const size_t part = backward ? round_up(m * n * w, 256) : 0;
    return {0, part, 2 * part};
}

bool sizes_ok(size_t m, size_t n, size_t k) {
    return m <= ZVC_FFN_MAX_ROWS && n <= ZVC_FFN_MAX_COLUMNS && k <= ZVC_FFN_MAX_COLUMNS;
}

bool stride_ok(size_t ld, size_t cols) { return ld >= cols && ld <= ZVC_FFN_MAX_COLUMNS; }

template <typename T>
zvc_status product(Operand<T> a1, Operand<T> b1, Operand<T> a2, Operand<T> b2, void* out, size_t ld, size_t rows,
                   size_t cols, size_t steps, hipStream_t stream) {
    return launch(product_kernel<T>, dim3(div_up(cols, kTile), div_up(rows, kTile)), kTileThreads, stream, a1, b1, a2, b2,
                  static_cast<T*>(out), ld, rows, cols, steps);
}

template <typename T>
zvc_status project(const GluArgs<T>& p, hipStream_t stream) {
    return launch(glu_project_kernel<T>, dim3(div_up(p.n, kTile), div_up(p.m, kTile)), kTileThreads, stream, p);
}

template <typename T>
zvc_status backward_as(GluArgs<T> p, void* dx, size_t lddx, void* dwg, void* dwu, size_t lddw, hipStream_t stream) {
    if (p.m != 0 && p.n != 0) {
        zvc_status st;
        if (p.gate_in == nullptr) {
            st = project(p, stream);
        } else {
            const size_t blocks = div_up(p.m * p.n, 256);
            st = launch(glu_slope_kernel<T>, dim3(blocks < 65536 ? blocks : 65536), 256, stream, p);
        }
        if (st != ZVC_OK) return st;
    }
    const Operand<T> none = {nullptr, 0, 0};
    if (dx != nullptr && p.m != 0 && p.k != 0)
        if (zvc_status st = product<T>({p.dg, p.ldd, 1}, {p.wg, 1, p.ldw}, {p.du, p.ldd, 1}, {p.wu, 1, p.ldw}, dx, lddx, p.m,
                                       p.k, p.n, stream)) return st;
    if (dwg == nullptr || p.n == 0 || p.k == 0) return ZVC_OK;
    if (zvc_status st = product<T>({p.dg, 1, p.ldd}, {p.x, 1, p.ldx}, none, none, dwg, lddw, p.n, p.k, p.m, stream)) return st;
    return product<T>({p.du, 1, p.ldd}, {p.x, 1, p.ldx}, none, none, dwu, lddw, p.n, p.k, p.m, stream);
}

}  // namespace

// ------------------------------------------------------------------ C ABI
extern "C" {

uint64_t zvc_dropout_fraction(double p) {
    return p >= 0.0 && p <= 1.0 ? static_cast<uint64_t>(std::nearbyint(p * 4294967296.0)) : ~uint64_t{0};
}

zvc_status zvc_dropout(const void* d_x, size_t ldx, const void* d_residual, size_t ldr, void* d_y, size_t ldy,
                       size_t rows, size_t cols, int type, uint64_t drop, uint64_t seed, uint64_t offset,
                       const uint64_t* d_offset, hipStream_t stream) {
    const size_t w = type_bytes(type);
    if (w == 0) return ZVC_E_ARG;
    Drop d;
    if (zvc_status st = make_drop(drop, seed, offset, d_offset, &d)) return st;
    if (ldx < cols || ldy < cols || (d_residual != nullptr && ldr < cols)) return ZVC_E_ARG;
    constexpr size_t kMost = size_t{1} << 40;               // elements that a row stride may span in all
    const size_t widest = ldx > ldy ? (ldx > ldr ? ldx : ldr) : ldy > ldr ? ldy : ldr;
    if (widest > kMost || (rows != 0 && widest > kMost / rows)) return ZVC_E_ARG;
    if (rows == 0 || cols == 0) return ZVC_OK;
    if (d_x == nullptr || d_y == nullptr) return ZVC_E_ARG;
    if (!aligned_to(d_x, w) || !aligned_to(d_y, w) || !aligned_to(d_residual, w)) return ZVC_E_ALIGN;
    const Region out{d_y, ldy * w, rows, cols * w};
    if (!(d_y == d_x && (ldy == ldx || rows == 1)) && overlap(out, {d_x, ldx * w, rows, cols * w})) return ZVC_E_ARG;
    if (!(d_y == d_residual && (ldy == ldr || rows == 1)) && overlap(out, {d_residual, ldr * w, rows, cols * w}))
        return ZVC_E_ARG;
    switch (type) {
        case ZVC_FP32: return dropout_as<float>(d_x, ldx, d_residual, ldr, d_y, ldy, rows, cols, d, stream);
        case ZVC_FP16: return dropout_as<fp16>(d_x, ldx, d_residual, ldr, d_y, ldy, rows, cols, d, stream);
        default: return dropout_as<bf16>(d_x, ldx, d_residual, ldr, d_y, ldy, rows, cols, d, stream);
    }
}

size_t zvc_glu_workspace_bytes(size_t m, size_t n, size_t k, int type, int backward, int loose) {
    const size_t w = type_bytes(type);
    (void)loose;
    return w == 0 || !sizes_ok(m, n, k) ? 0 : layout_of(m, n, k, w, backward != 0).bytes + 256;
}

zvc_status zvc_glu_forward(const void* d_x, size_t ldx, const void* d_wg, const void* d_wu, size_t ldw, void* d_h,
                           size_t ldh, void* d_gate, void* d_up, size_t ldp, size_t m, size_t n, size_t k, int type,
                           int activation, uint64_t drop, uint64_t seed, uint64_t offset, const uint64_t* d_offset,
                           void* d_ws, size_t ws, hipStream_t stream) {
    const size_t w = type_bytes(type);
    if (w == 0 || activation < ZVC_RELU || activation > ZVC_GELU_TANH || !sizes_ok(m, n, k)) return ZVC_E_ARG;
    Drop d;
    if (zvc_status st = make_drop(drop, seed, offset, d_offset, &d)) return st;
    if (!stride_ok(ldx, k) || !stride_ok(ldw, k) || !stride_ok(ldh, n) || (d_gate != nullptr) != (d_up != nullptr) ||
        (d_gate != nullptr && !stride_ok(ldp, n)))
        return ZVC_E_ARG;
    if (m == 0 || n == 0) return ZVC_OK;
    if (d_h == nullptr || (k != 0 && (d_x == nullptr || d_wg == nullptr || d_wu == nullptr)) || d_ws == nullptr) return ZVC_E_ARG;
    const void* all[] = {d_x, d_wg, d_wu, d_h, d_gate, d_up};
    for (const void* p : all)
        if (!aligned_to(p, w)) return ZVC_E_ALIGN;
    if (!aligned_to(d_ws, 256)) return ZVC_E_ALIGN;
    const bool loose = !aligned_to(d_x, 16) || !aligned_to(d_wg, 16) || !aligned_to(d_wu, 16) || ldx * w % 16 != 0 || ldw * w % 16 != 0;
    if (ws < zvc_glu_workspace_bytes(m, n, k, type, 0, loose)) return ZVC_E_WORKSPACE;
    const Region in[] = {{d_x, ldx * w, m, k * w}, {d_wg, ldw * w, n, k * w}, {d_wu, ldw * w, n, k * w}};
    const Region out[] = {{d_h, ldh * w, m, n * w}, {d_gate, ldp * w, m, n * w}, {d_up, ldp * w, m, n * w}, {d_ws, ws, 1, ws}};
    for (int i = 0; i < 4; ++i) {
        for (const Region& r : in)
            if (overlap(out[i], r)) return ZVC_E_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return ZVC_E_ARG;
    }
    const auto as = [&](auto zero) {
        using T = decltype(zero);
        return project(GluArgs<T>{static_cast<const T*>(d_x), static_cast<const T*>(d_wg), static_cast<const T*>(d_wu), nullptr,
                                  nullptr, nullptr, static_cast<T*>(d_h), static_cast<T*>(d_gate), static_cast<T*>(d_up), nullptr,
                                  nullptr, ldx, ldw, 0, ldh, ldp, 0, m, n, k, activation, d}, stream);
    };
    return type == ZVC_FP32 ? as(0.f) : type == ZVC_FP16 ? as(fp16{}) : as(bf16{});
}

zvc_status zvc_glu_backward(const void* d_dh, size_t lddh, const void* d_x, size_t ldx, const void* d_wg,
                            const void* d_wu, size_t ldw, const void* d_gate, const void* d_up, size_t ldp, void* d_dx,
                            size_t lddx, void* d_dwg, void* d_dwu, size_t lddw, size_t m, size_t n, size_t k, int type,
                            int activation, uint64_t drop, uint64_t seed, uint64_t offset, const uint64_t* d_offset,
                            void* d_ws, size_t ws, hipStream_t stream) {
    const size_t w = type_bytes(type);
    if (w == 0 || activation < ZVC_RELU || activation > ZVC_GELU_TANH || !sizes_ok(m, n, k)) return ZVC_E_ARG;
    Drop d;
    if (zvc_status st = make_drop(drop, seed, offset, d_offset, &d)) return st;
    if (!stride_ok(lddh, n) || !stride_ok(ldx, k) || !stride_ok(ldw, k) || (d_gate != nullptr) != (d_up != nullptr) ||
        (d_gate != nullptr && !stride_ok(ldp, n)) || (d_dx != nullptr && !stride_ok(lddx, k)) ||
        (d_dwg != nullptr) != (d_dwu != nullptr) || (d_dwg != nullptr && !stride_ok(lddw, k)))
        return ZVC_E_ARG;
    const bool sums = m != 0 && n != 0;                          // else every output is 0
    if (k == 0 || (m == 0 && n == 0) || (d_dx == nullptr && d_dwg == nullptr)) return ZVC_OK;
    if ((sums && (d_dh == nullptr || d_x == nullptr || d_wg == nullptr || d_wu == nullptr)) || d_ws == nullptr) return ZVC_E_ARG;
    const void* all[] = {d_dh, d_x, d_wg, d_wu, d_gate, d_up, d_dx, d_dwg, d_dwu};
    for (const void* p : all)
        if (!aligned_to(p, w)) return ZVC_E_ALIGN;
    if (!aligned_to(d_ws, 256)) return ZVC_E_ALIGN;
    const bool loose = !aligned_to(d_x, 16) || !aligned_to(d_wg, 16) || !aligned_to(d_wu, 16) || ldx * w % 16 != 0 || ldw * w % 16 != 0;
    if (ws < zvc_glu_workspace_bytes(m, n, k, type, 1, loose)) return ZVC_E_WORKSPACE;
    const Region in[] = {{d_dh, lddh * w, m, n * w}, {d_x, ldx * w, m, k * w}, {d_wg, ldw * w, n, k * w},
                         {d_wu, ldw * w, n, k * w}, {d_gate, ldp * w, m, n * w}, {d_up, ldp * w, m, n * w}};
    const Region out[] = {{d_dx, lddx * w, m, k * w}, {d_dwg, lddw * w, n, k * w}, {d_dwu, lddw * w, n, k * w}, {d_ws, ws, 1, ws}};
    for (int i = 0; i < 4; ++i) {
        for (const Region& r : in)
            if (overlap(out[i], r)) return ZVC_E_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return ZVC_E_ARG;
    }
    const Layout at = layout_of(m, n, k, w, true);
    const auto as = [&](auto zero) {
        using T = decltype(zero);
        unsigned char* base = static_cast<unsigned char*>(d_ws);
        GluArgs<T> p{static_cast<const T*>(d_x), static_cast<const T*>(d_wg), static_cast<const T*>(d_wu),
                     static_cast<const T*>(d_dh), static_cast<const T*>(d_gate), static_cast<const T*>(d_up), nullptr, nullptr,
                     nullptr, reinterpret_cast<T*>(base + at.dg), reinterpret_cast<T*>(base + at.du), ldx, ldw, lddh, 0, ldp, n,
                     m, n, k, activation, d};
        return backward_as(p, d_dx, lddx, d_dwg, d_dwu, lddw, stream);
    };
    return type == ZVC_FP32 ? as(0.f) : type == ZVC_FP16 ? as(fp16{}) : as(bf16{});
}

}  // extern "C"
