// Gated feed-forward block and dropout, forward and backward, for AMD gfx950 (wave64): kernels and C ABI
// (include/zvc_ffn.h has the formulas).
//
//   * dropout_kernel: one pass over the data, the mask made on the way by the counter-based generator.
//   * product_kernel, gradients_kernel: the large products (both projections with what becomes of them; dx with dWg and dWu),
//     tiles on the matrix cores, staged from memory straight to LDS, with the activation, dropout and the kept projections, or
//     their gradients, in the tile's epilogue.  Sums too long for the few tiles there are are cut into parts that a join adds.
//   * token_kernel: the projections of up to 128 tokens, bound by reading the weights once.
//   * slope_kernel: dg and du from kept projections; align_kernel: copies of inputs that do not take 16-byte accesses.
//
// Times in the comments are us on one MI355X, where a large copy moves 4.8 to 5.0 TB/s and a large bf16 product of the vendor's library
// reaches 1230 to 1460 TFLOP/s (fp32 155): calls one behind the other over several sets of tensors.  Cards differ by 6 % in long
// products, and the first milliseconds on a card that was idle run up to a third longer; both sides of a comparison ran in turn.

#include "tiles.h"

#include <cmath>

namespace {

// ------------------------------------------------------------------ dropout
// What a kernel needs to drop: the 32-bit fraction in its upper and lower half, the factor of what stays.
struct Drop {
    unsigned high, low;                // high: up to 65536, at which everything goes
    float scale;
    uint64_t seed, offset;
    const uint64_t* d_offset;
    bool active;
};

// Whether 16 bits are enough for all eight: none of them equals the fraction's upper half (or that has no lower one).
__device__ __forceinline__ bool decided(const Drop& d, const Words& r) {
    if (d.low == 0) return true;
    unsigned equal = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned x = r.w[i] ^ (d.high * 0x10001u);             // a half of zeros where equal
        equal |= (x - 0x10001u) & ~x & 0x80008000u;
    }
    return equal == 0;
}

// Bit j: element 8 * group + j stays.  `r`: the group's words.
__device__ __forceinline__ unsigned keep_bits(const Drop& d, uint64_t offset, uint64_t group, const Words& r) {
    unsigned keep = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) keep |= static_cast<unsigned>(half_of(r, j) >= d.high) << j;
    if (!decided(d, r)) {                                            // one element in 65536: 16 bits more
        const Words more = philox(group | (uint64_t{1} << 63), offset, d.seed);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (half_of(r, j) == d.high && half_of(more, j) < d.low) keep &= ~(1u << j);
    }
    return keep;
}

__device__ __forceinline__ unsigned keep_group(const Drop& d, uint64_t offset, uint64_t group) {
    return keep_bits(d, offset, group, philox(group, offset, d.seed));
}

// Bits for elements first .. first + 7, wherever they begin.
__device__ __forceinline__ unsigned keep_span(const Drop& d, uint64_t offset, uint64_t first) {
    const unsigned shift = static_cast<unsigned>(first & 7), groups = shift != 0 ? 2 : 1;
    unsigned keep = 0;
#pragma unroll 1                       // (one copy of the generator: the products' code has to stay small)
    for (unsigned i = 0; i < groups; ++i) keep |= keep_group(d, offset, (first >> 3) + i) << (8 * i);
    return (keep >> shift) & 0xFFu;
}

__device__ __forceinline__ uint64_t effective_offset(const Drop& d) {
    return d.offset + (d.d_offset != nullptr ? *d.d_offset : 0);
}

constexpr int kDropThreads = 256;
constexpr unsigned kDropRow = 1u << 20;            // workgroups in a row of the grid: a dimension holds fewer than 2^32 lanes

// Zeros in the place of a group's dropped elements.  Where 16 bits decide all of them each is compared where it lies: the
// generator and these comparisons are what a 16-bit tensor's call spends beside its traffic.
__device__ __forceinline__ void drop_group(const Drop& d, uint64_t offset, uint64_t group, const Words& words, Eight& e) {
    if (!decided(d, words)) {
        drop8(keep_bits(d, offset, group, words), e);
    } else if (d.high != 0) {
        const unsigned below = (d.high << 16) - 1;                   // (p = 1: nothing is above)
#pragma unroll
        for (int j = 0; j < 8; ++j) e.v[j] = (j % 2 ? words.w[j / 2] : words.w[j / 2] << 16) > below ? e.v[j] : 0.f;
    }
}

// y = drop(x) [+ residual].  A lane owns GROUPS times eight consecutive elements, each one counter of the generator.  Memory bounds
// it, and with 16-bit elements nearly the generator too (20 multiplications for 16 bytes).  33.5 M elements, us and TB/s: bf16
// 27.3, 4.9 (25.4 without the generator); fp32 49, 5.5; bf16 with a residual at 67 M elements 74.4, 5.4.  GROUPS = 1 | 2 | 4:
// bf16 28.8 | 27.3 | 30.4, fp32 with a residual 68.3 | 71.1 | 71.9.
//
// Its stores leave y in the caches for what reads it next.  Past them the call alone takes less, and the codec or a product that reads y
// more than that; us, as it is | past: bf16 of 96 MB 38.5 | 36, with the codec 73 | 78.3, with a product 116 | 118; 128 MB and a residual
// 72.8 | 63.2, with a product 161 | 165; 192 MB with the codec 131 | 141.  (An addition behind it: 96 MB 72 | 72, 64 MB and a
// residual 63 | 55.6, 192 MB and a residual 176.6 | 183.6.)
template <typename T, int GROUPS>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(const T* x, size_t ldx, const T* residual, size_t ldr,
                                                               T* y, size_t ldy, size_t cols, uint64_t total, Drop d) {
    const uint64_t offset = d.active ? effective_offset(d) : 0;
    const uint64_t group0 = (static_cast<uint64_t>(blockIdx.y) * kDropRow + blockIdx.x) * (kDropThreads * GROUPS) + threadIdx.x;
    Eight e[GROUPS], r[GROUPS];
    uint64_t row[GROUPS], col[GROUPS];
    bool inside[GROUPS];                                           // eight elements of one row
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const uint64_t first = (group0 + g * kDropThreads) * 8;
        row[g] = cols >= total ? 0 : first / cols;
        col[g] = first - row[g] * cols;
        inside[g] = first + 8 <= total && col[g] + 8 <= cols;
        if (!inside[g]) continue;
        e[g] = load8(x + row[g] * ldx + col[g]);
        if (residual != nullptr) r[g] = load8(residual + row[g] * ldr + col[g]);
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const uint64_t group = group0 + g * kDropThreads, first = group * 8;
        if (first >= total) continue;
        const Words words = d.active ? philox(group, offset, d.seed) : Words{};
        if (inside[g]) {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[g].v[j] *= d.scale;
            if (d.active) drop_group(d, offset, group, words, e[g]);
            if (residual != nullptr) {
#pragma unroll
                for (int j = 0; j < 8; ++j) e[g].v[j] += r[g].v[j];
            }
            store8(y + row[g] * ldy + col[g], e[g]);
        } else {
            const unsigned keep = d.active ? keep_bits(d, offset, group, words) : 0xFFu;
            uint64_t line = row[g], at = col[g];
            for (int j = 0; j < 8 && first + j < total; ++j) {
                float v = (keep >> j & 1u) != 0 ? static_cast<float>(x[line * ldx + at]) * d.scale : 0.f;
                if (residual != nullptr) v += static_cast<float>(residual[line * ldr + at]);
                y[line * ldy + at] = static_cast<T>(v);
                if (++at == cols) at = 0, ++line;
            }
        }
    }
}

// ------------------------------------------------------------------ the activation
struct ActValue {
    float value, slope;
};

// 1 / (1 + exp(-x)).  In fp32 to a few units in the last place, by exp of what is below 0, also where it is no normal number.  For
// 16-bit types by the shortest way: exp's argument is rounded as a multiple of ln 2, which leaves |x| x 2^-24 of the result,
// 5e-6 at -80, and below -87 the result is 0.
template <typename T>
__device__ __forceinline__ float sigmoid(float x) {
    if constexpr (sizeof(T) == 4) {
        const float e = expf(-fabsf(x));
        return (x < 0.f ? e : 1.f) * __builtin_amdgcn_rcpf(1.f + e);
    } else {
        return __builtin_amdgcn_rcpf(1.f + __expf(-x));
    }
}

// act(g) and its derivative.  relu: a NaN is not <= 0 and stays.
template <int ACT, typename T>
__device__ __forceinline__ ActValue activate(float g) {
    if constexpr (ACT == ZVC_RELU) {
        return {g <= 0.f ? 0.f : g, g <= 0.f ? 0.f : 1.f};
    } else if constexpr (ACT == ZVC_SILU) {
        const float s = sigmoid<T>(g), a = g * s;
        return {a, s + a * (1.f - s)};
    } else if constexpr (ACT == ZVC_GELU) {
        const float density = __expf(-0.5f * g * g);
        float cdf;
        if constexpr (sizeof(T) == 4) {
            cdf = 0.5f * erfcf(-0.70710678f * g);
        } else {
            // The distribution function below 0 over the density's exp, by t = 1 / (1 + c |g|): a rational function there, fitted
            // as a polynomial of degree seven without a constant term, so that it falls off like 1 / |g|.  The fit minimises the
            // larger of the error relative to the value, 1.2e-5, and 64 times the absolute one, 1.9e-7: far below 0 the result is
            // this value itself, and a 16-bit type rounds it by 2^-9 or 2^-12 of itself.  (Two more terms than the absolute
            // error alone would need; erfcf, 64 times per lane and tile, takes many times that.)
            const float t = __builtin_amdgcn_rcpf(1.f + 0.37056866f * fabsf(g));
            const float tail = density * t * (0.14783728f + t * (0.14762331f + t * (0.13156720f + t * (0.058789373f + t * (0.12566245f + t * (-0.15569937f + t * 0.044219945f))))));
            cdf = g <= 0.f ? tail : 1.f - tail;
        }
        return {g * cdf, cdf + g * 0.39894228f * density};
    } else {
        // (1 + tanh(z)) / 2 = sigmoid(2 z)
        const float s = sigmoid<T>(1.5957691f * (g + 0.044715f * g * g * g)), a = g * s;
        // (beyond 16 either s or 1 - s is 0: g^2 is held there, or it becomes an infinity and the product a NaN)
        return {a, s + a * (1.f - s) * 1.5957691f * (1.f + 0.134145f * fminf(g * g, 256.f))};
    }
}

// f(constant) for the activation.
template <typename F>
__device__ __forceinline__ void with_activation(int act, F f) {
    switch (act) {
        case ZVC_RELU: f(std::integral_constant<int, ZVC_RELU>{}); break;
        case ZVC_SILU: f(std::integral_constant<int, ZVC_SILU>{}); break;
        case ZVC_GELU: f(std::integral_constant<int, ZVC_GELU>{}); break;
        default: f(std::integral_constant<int, ZVC_GELU_TANH>{});
    }
}

enum class Does { kForward, kSlope, kDx, kDw };

template <typename T>
struct GluArgs {
    const T *x, *wg, *wu, *dh;
    const T *gate_in, *up_in;
    T *h, *gate, *up, *dg, *du;
    T *dx, *dwg, *dwu;
    unsigned ldx, ldw, lddh, ldh, ldp, ldd, lddx, lddw, m, n, k;   // (32 bits hold them: scalar registers are short)
    int act;
    Drop d;
};

// Eight neighbouring columns' projections g and u, col a multiple of eight: dg and du in their place, before what is dropped is ...
template <int ACT, typename T>
__device__ __forceinline__ void slope8(const GluArgs<T>& p, const Eight& dh, Eight& g, Eight& u) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const ActValue a = activate<ACT, T>(g.v[j]);
        const float d = dh.v[j] * p.d.scale;
        g.v[j] = ACT == ZVC_RELU ? (g.v[j] <= 0.f ? 0.f : d * u.v[j]) : d * u.v[j] * a.slope;
        u.v[j] = d * a.value;
    }
}
// ... or h.
template <int ACT, typename T>
__device__ __forceinline__ Eight forward8(const GluArgs<T>& p, const Eight& g, const Eight& u) {
    Eight h;
#pragma unroll
    for (int j = 0; j < 8; ++j) h.v[j] = activate<ACT, T>(g.v[j]).value * u.v[j] * p.d.scale;
    return h;
}

// What is kept of them, in their place.
template <typename T>
__device__ __forceinline__ void kept8(const GluArgs<T>& p, unsigned keep, Eight& g, Eight& u) {
    if (p.act == ZVC_RELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) u.v[j] = g.v[j] <= 0.f ? 0.f : u.v[j], g.v[j] = g.v[j] <= 0.f ? 0.f : g.v[j];
    }
    if (p.d.active) drop8(keep, g), drop8(keep, u);
}

// What becomes of them in their row: `there` of them (none: dg's and du's filling) are columns.  dh: for the slope.
template <typename T, Does DOES>
__device__ __forceinline__ void finish8(const GluArgs<T>& p, unsigned keep, unsigned row, unsigned col, int there, bool full, const Eight& dh, Eight& g, Eight& u) {
    if constexpr (DOES == Does::kSlope) {
        with_activation(p.act, [&](auto act) { slope8<decltype(act)::value>(p, dh, g, u); });
        drop8(keep & ((1u << there) - 1u), g), drop8(keep & ((1u << there) - 1u), u);
        store8(cell(p.dg, row, p.ldd, col), g);
        store8(cell(p.du, row, p.ldd, col), u);
    } else {
        Eight h;
        with_activation(p.act, [&](auto act) { h = forward8<decltype(act)::value>(p, g, u); });
        drop8(keep, h);
        store_some(cell(p.h, row, p.ldh, col), h, there, full);
        if (p.gate != nullptr) {
            kept8(p, keep, g, u);
            store_some(cell(p.gate, row, p.ldp, col), g, there, full);
            store_some(cell(p.up, row, p.ldp, col), u, there, full);
        }
    }
}

// What becomes of a lane's strip of a tile, eight columns of QB rows 16 apart: straight code, row after row (the fences keep the
// compiler from working on all rows at once, out of registers), and what is rare in another place (a tile's code that the
// instruction cache has to fetch anew costs 3 us).
template <typename T, Does DOES, class S>
__device__ __forceinline__ void finish_tile(const GluArgs<T>& p, unsigned row, unsigned col, bool full, bool past, float4v (&acc)[S::PB][S::QB]) {
    static_assert(S::QB <= 8, "a bit for each of a lane's elements");
    if constexpr (S::QT < 256) past = false;                     // (code that these tiles do not need)
    if (col >= (DOES == Does::kSlope ? p.ldd : p.n)) return;     // (dg and du are written up to their rows' ends)
    const int there = columns_left(p.n, col);
    uint64_t keep = ~uint64_t{0};
    if (p.d.active) {
        const uint64_t offset = effective_offset(p.d);
        keep = 0;
#pragma unroll 1
        for (int j = 0; j < S::QB; ++j)
            keep |= static_cast<uint64_t>(keep_span(p.d, offset, static_cast<uint64_t>(row + j * 16) * p.n + col)) << (8 * j);
    }
    const auto take = [&](int j, Eight& g, Eight& u) {
#pragma unroll
        for (int e = 0; e < 8; ++e) g.v[e] = acc[e / 4][j][e % 4], u.v[e] = acc[2 + e / 4][j][e % 4];
    };
    const auto keeps = [&](int j) { return static_cast<unsigned>(keep >> (8 * j)) & 0xFFu; };
    if (!full) {                                    // (only where the columns end inside a strip)
#pragma unroll
        for (int j = 0; j < S::QB; ++j) {
            if (row + j * 16 < p.m) {
                Eight g, u;
                take(j, g, u);
                const Eight dh = DOES == Does::kSlope ? load_some(cell(p.dh, row + j * 16, p.lddh, col), there, false) : Eight{};
                finish8<T, DOES>(p, keeps(j), row + j * 16, col, there, false, dh, g, u);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        return;
    }
    if constexpr (DOES == Does::kSlope) {
        const auto load = [&](int j) { return j < S::QB && row + j * 16 < p.m ? load8(cell(p.dh, row + j * 16, p.lddh, col)) : Eight{}; };
        with_activation(p.act, [&](auto act) {
            Eight dh = load(0);
#pragma unroll
            for (int j = 0; j < S::QB; ++j) {
                const Eight next = load(j + 1);
                Eight g, u;
                take(j, g, u);
                slope8<decltype(act)::value>(p, dh, g, u);
                if (p.d.active) drop8(keeps(j), g), drop8(keeps(j), u);
                if (row + j * 16 < p.m) {
                    store8(cell(p.dg, row + j * 16, p.ldd, col), g);
                    store8(cell(p.du, row + j * 16, p.ldd, col), u);
                }
                dh = next;
                __builtin_amdgcn_sched_barrier(0);
            }
        });
    } else {
        if (p.gate != nullptr) {
#pragma unroll
            for (int j = 0; j < S::QB; ++j) {
                Eight g, u;
                take(j, g, u);
                kept8(p, keeps(j), g, u);
                if (row + j * 16 < p.m) {
                    store8(cell(p.gate, row + j * 16, p.ldp, col), g, past);
                    store8(cell(p.up, row + j * 16, p.ldp, col), u, past);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        with_activation(p.act, [&](auto act) {
#pragma unroll
            for (int j = 0; j < S::QB; ++j) {
                Eight g, u;
                take(j, g, u);
                Eight h = forward8<decltype(act)::value>(p, g, u);
                if (p.d.active) drop8(keeps(j), h);
                if (row + j * 16 < p.m) store8(cell(p.h, row + j * 16, p.ldh, col), h, past);
                __builtin_amdgcn_sched_barrier(0);
            }
        });
    }
}

// How one product is cut into work items: tp x tq tiles, of which the first `whole` are summed in one go and the others in `parts`
// parts of the reduction each, whose sums lie part by part, tile by tile as they lie in it, and are joined.  past: the outputs of the
// large tiles go past the caches.
struct Plan {
    float* sums;
    unsigned tp, tq, whole, parts;
    bool past;
    __host__ __device__ unsigned items() const { return whole + (tp * tq - whole) * parts; }
};

// One workgroup's view of a tile: where its operands and its part of the reduction lie.
template <typename T, Does DOES, class S>
struct Tile {
    static constexpr bool kFold = DOES == Does::kForward || DOES == Does::kSlope;
    static constexpr Lies kP = kFold ? Lies::kAlong : Lies::kAcross, kQ = DOES == Does::kDw ? Lies::kAcross : Lies::kAlong;
    static constexpr int W = sizeof(T), kSteps = kStageBytes / W;
    static constexpr int kCols = kFold ? S::PT / 2 : S::PT;
    using InP = Operand<T, kP, S::PT, S::kWavesAll, kFold>;
    using InQ = Operand<T, kQ, S::QT, S::kWavesAll, false>;
    static_assert(!kFold || 32 % (InP::kLoads * InP::kRowsPerLoad) == 0 || InP::kLoads * InP::kRowsPerLoad == 64, "a wave fetches one weight's rows, or a run of each");
    static_assert(!kFold || S::PB == 4, "a wave's strip is 32 rows of each weight");

    unsigned col0, row0;
    bool second, split;                             // dW: of dWu; summed in parts
    unsigned number, part;                          // of the split tiles; of its reduction
    unsigned begin, end, once;                      // stages; dx: the first `once` are Wg's
    InP in_p;
    InQ in_q;
    uint64_t p0, p1, q0, q1;

    // Where tile `at` lies.  Tiles are walked in bands of some rows: what 32 workgroups of an XCD read at a time then fits its L2.
    // (4 | 8 | 16 rows: long prompt 2235 | 2205 | 2288 us, largest backward 3478 | 3515 | 3598.)
    __device__ __forceinline__ void locate(unsigned at, unsigned tp, unsigned tq) {
        constexpr unsigned kBand = kFold ? 8 : 4;
        const unsigned band = at / (kBand * tp), in_band = at % (kBand * tp), height = tq - band * kBand < kBand ? tq - band * kBand : kBand;
        const unsigned tile_q = band * kBand + in_band % height, halves = tq / 2;
        col0 = in_band / height * kCols;
        second = DOES == Does::kDw && tile_q >= halves;
        row0 = (second ? tile_q - halves : tile_q) * S::QT;
    }
    __device__ __forceinline__ void init(const GluArgs<T>& p, const Plan& plan, unsigned item, int wave, int lane) {
        const unsigned rest = plan.tp * plan.tq - plan.whole;
        split = item >= plan.whole;
        part = 0;
        if (split) {
            const unsigned at = place_of(item - plan.whole, rest * plan.parts);
            part = at / rest;
            number = at - part * rest;
            locate(plan.whole + number, plan.tp, plan.tq);
        } else {
            locate(place_of(item, plan.whole), plan.tp, plan.tq);
        }
        const unsigned parts = split ? plan.parts : 1;
        const unsigned rows = DOES == Does::kDw ? p.n : p.m, cols = kFold ? p.n : p.k;
        once = (length(p) + kSteps - 1) / kSteps;
        // (parts differ by a stage at most)
        const unsigned stages = DOES == Does::kDx ? 2 * once : once, each = split ? stages / plan.parts : stages, longer = stages - each * parts;
        begin = part * each + (part < longer ? part : longer);
        end = begin + each + (part < longer ? 1 : 0);
        in_p.init(wave, lane, kFold || DOES == Does::kDx ? p.ldw : p.ldx, cols - col0 < S::PT ? cols - col0 : S::PT);
        in_q.init(wave, lane, kFold ? p.ldx : p.ldd, rows - row0 < S::QT ? rows - row0 : S::QT);
        p0 = reinterpret_cast<uint64_t>(kFold ? cell(p.wg, col0, p.ldw, 0) : DOES == Does::kDx ? p.wg + col0 : p.x + col0);
        p1 = reinterpret_cast<uint64_t>(kFold ? cell(p.wu, col0, p.ldw, 0) : p.wu + col0);
        q0 = reinterpret_cast<uint64_t>(kFold ? cell(p.x, row0, p.ldx, 0) : DOES == Does::kDx ? cell(p.dg, row0, p.ldd, 0) : (second ? p.du : p.dg) + row0);
        q1 = reinterpret_cast<uint64_t>(cell(p.du, row0, p.ldd, 0));
    }
    static __device__ __forceinline__ unsigned length(const GluArgs<T>& p) { return kFold ? p.k : DOES == Does::kDx ? p.n : p.m; }

    __device__ __forceinline__ void fetch(const GluArgs<T>& p, unsigned s, unsigned lds) const {
        const unsigned step_p = kFold ? kStageBytes : kSteps * W * (DOES == Does::kDx ? p.ldw : p.ldx);
        const unsigned step_q = DOES == Does::kDw ? kSteps * W * p.ldd : kStageBytes;
        const bool late = DOES == Does::kDx && s >= once;
        const unsigned t = late ? s - once : s;
        const int left = static_cast<int>(length(p) - t * kSteps);
        in_p.fetch((late ? p1 : p0) + static_cast<uint64_t>(t) * step_p, p1 + static_cast<uint64_t>(t) * step_p, left, lds);
        // (dx: the columns of dg and du behind the last are zeros, up to a whole stage)
        in_q.fetch((late ? q1 : q0) + static_cast<uint64_t>(t) * step_q, 0, DOES == Does::kDx ? kSteps : left, lds + S::PT * kStageBytes);
    }
};

// Workgroups take tiles until there are none left; the next tile's first stages are on their way while a tile is finished.
//
// What bounds it, with the large tile: the card's power.  16384 x 11264 x 4096 (forward, bf16) takes 2170 to 2300 on different cards, 1310
// to 1390 TFLOP/s.  Where it took 2220 to 2260: 0.485 for each step of k, at which the matrix cores are busy for 87 % of the cycles of a
// clock that is held near 1.7 GHz, and the rest to begin and finish 22 tiles.  LDS is next: a half stage's reads take 768 of its 1024 cycles.  Four waves
// of 128 x 128 with sums in accumulation registers read a third less, 0.472 a step, and finish tiles so much slower that it
// is 2700 in all; instructions of 32 x 32 2430; a ring of five half stages 2660; one wave at a raised priority 2360; without the
// reads between the products 2540; with tiles that are not persistent and epilogues with a branch per element 2440.  Small tiles
// are bound by LDS: 64 x 64 a wave, 0.85 a stage for the two of a compute unit.
//
// `base`: the ring in LDS.  `next`: gives this workgroup's items, and kNone behind the last.
template <typename T, Does DOES, class S, typename Next>
__device__ __forceinline__ void work(const GluArgs<T>& p, const Plan& plan, unsigned base, int lane, Next next) {
    using Where = Tile<T, DOES, S>;
    constexpr bool kFold = Where::kFold;
    constexpr int kRing = S::kRing;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wp = wave % S::WP, wq = wave / S::WP, r = lane & 15, quarter = lane >> 4;

    using ReadP = Reader<T, Where::kP, S::PT, S::PB, kFold>;
    using ReadQ = Reader<T, Where::kQ, S::QT, S::QB, false>;
    ReadP out_p;
    ReadQ out_q;
    out_p.init(base, wp, lane);
    out_q.init(base + S::PT * kStageBytes, wq, lane);
    using Frag = typename Fragment<T>::type;
    Frag a[2][S::PB], b[2][S::QB];
    float4v acc[S::PB][S::QB];
    const auto read = [&](auto half, unsigned stage) {
        constexpr int kHalf = decltype(half)::value;
#pragma unroll
        for (int i = 0; i < S::PB; ++i) a[kHalf][i] = out_p.read(i, kHalf, stage);
#pragma unroll
        for (int j = 0; j < S::QB; ++j) b[kHalf][j] = out_q.read(j, kHalf, stage);
    };
    const auto product = [&](auto half) {
        constexpr int kHalf = decltype(half)::value;
#pragma unroll
        for (int j = 0; j < S::QB; ++j)
#pragma unroll
            for (int i = 0; i < S::PB; ++i) acc[i][j] = multiply(a[kHalf][i], b[kHalf][j], acc[i][j]);
        interleave<ReadP::kReads + ReadQ::kReads, S::PB * S::QB * (sizeof(T) == 4 ? 4 : 1)>();
    };
    constexpr std::integral_constant<int, 0> kFirst{};
    constexpr std::integral_constant<int, 1> kSecond{};

    Where tile;
    const auto begin = [&](unsigned item) {
        tile.init(p, plan, item, wave, lane);
#pragma unroll
        for (int i = 0; i < kRing; ++i)
            if (tile.begin + i < tile.end) tile.fetch(p, tile.begin + i, base + i * S::kStage);
    };
    // Waits until the loads of `stages` stages at most are on their way, if as many as the ring holds were asked for.
    constexpr int kLoads = Where::InP::kLoads + Where::InQ::kLoads;
    const auto wait_stages = [&](auto stages, bool full) {
        constexpr int kLeft = decltype(stages)::value * kLoads;
        if (kLeft != 0 && full) wait_loads<kLeft>();
        else wait_loads<0>();
    };
    const auto place = [&](unsigned s) { return ((s - tile.begin) & (kRing - 1)) * S::kStage; };
    static_assert((kRing & (kRing - 1)) == 0, "stages take places in turn");
    unsigned item = next();
    if (item == kNone) return;
    begin(item);
    while (item != kNone) {
#pragma unroll
        for (int i = 0; i < S::PB; ++i)
#pragma unroll
            for (int j = 0; j < S::QB; ++j) acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};
        // A stage is multiplied in two halves.  While a half's products run, the next half is read from LDS; between
        // the halves everyone has read the stage, and its place takes the one after the ring's last.
        wait_stages(std::integral_constant<int, kRing - 1>{}, tile.begin + kRing <= tile.end);
        group_barrier();
        read(kFirst, 0);
        for (unsigned s = tile.begin; s < tile.end; ++s) {
            read(kSecond, place(s));
            product(kFirst);
            wait_stages(std::integral_constant<int, kRing - 2>{}, s + kRing <= tile.end);
            group_barrier();                     // stage s + 1 is there, and everyone has read stage s
            if (s + kRing < tile.end) tile.fetch(p, s + kRing, base + place(s));
            read(kFirst, place(s + 1));          // (behind the last stage: what the place held, for nothing)
            product(kSecond);
        }
        const unsigned col0 = tile.col0, row0 = tile.row0;
        const bool second = tile.second, split = tile.split;
        float* const sums = plan.sums + (static_cast<size_t>(tile.part) * (plan.tp * plan.tq - plan.whole) + tile.number) * (S::PT * S::QT);
        item = next();
        group_barrier();                         // (the reads for nothing are done)
        if (item != kNone) begin(item);

        const int row_in = wq * S::QB * 16 + r;
        const unsigned row_first = row0 + row_in;
        if (split) {                             // the sums as they lie in the tile: QT rows of the reduction's PT indexes
#pragma unroll
            for (int j = 0; j < S::QB; ++j)
#pragma unroll
                for (int i = 0; i < S::PB; ++i) {
                    // (folded: the strip's eight columns of g, then of u)
                    const int at = kFold ? i / 2 * (S::PT / 2) + wp * 32 + quarter * 8 + i % 2 * 4 : (wp * S::PB + i) * 16 + quarter * 4;
                    *reinterpret_cast<float4v*>(sums + (row_in + j * 16) * S::PT + at) = acc[i][j];
                }
        } else if constexpr (kFold) {
            finish_tile<T, DOES, S>(p, row_first, col0 + wp * 32 + quarter * 8, col0 + wp * 32 + 32 <= p.n, plan.past, acc);
        } else {
            const unsigned rows = DOES == Does::kDw ? p.n : p.m;
            T* const out = DOES == Does::kDx ? p.dx : second ? p.dwu : p.dwg;
            const unsigned ldo = DOES == Does::kDx ? p.lddx : p.lddw;
            const bool full = col0 + (wp + 1) * S::PB * 16 <= p.k;
            const unsigned col = col0 + wp * S::PB * 16 + quarter * 4;
            struct Four { T v[4]; };
            const auto four = [&](int i, int j) {
                Four f;
#pragma unroll
                for (int e = 0; e < 4; ++e) f.v[e] = static_cast<T>(acc[i][j][e]);
                return f;
            };
            if (full) {
#pragma unroll
                for (int j = 0; j < S::QB; ++j) {
                    T* const at = cell(out, row_first + j * 16, ldo, col);
                    if (row_first + j * 16 < rows) {
#pragma unroll
                        for (int i = 0; i < S::PB; ++i) {
                            const Four f = four(i, j);
                            __builtin_memcpy(at + i * 16, &f, sizeof f);
                        }
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < S::QB; ++j) {
                    T* const at = cell(out, row_first + j * 16, ldo, col);
                    if (row_first + j * 16 >= rows) continue;
#pragma unroll
                    for (int i = 0; i < S::PB; ++i) {
                        const Four f = four(i, j);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (col + i * 16 + e < p.k) at[i * 16 + e] = f.v[e];
                    }
                }
            }
        }
    }
}

template <typename T, Does DOES, class S>
__global__ __launch_bounds__(S::kThreads, S::kPerUnit) void product_kernel(GluArgs<T> p, Plan plan) {
    work<T, DOES, S>(p, plan, ring<S>(), threadIdx.x & 63, Turns{blockIdx.x, plan.items()});
}

// dx, and behind it dWg and dWu, in one go: either alone leaves compute units idle in its last round.  The workgroups without a
// dx item in its last round take `ahead` items of dW before the others take their first.
template <typename T, class S>
__global__ __launch_bounds__(S::kThreads, S::kPerUnit) void gradients_kernel(GluArgs<T> p, Plan dx, Plan dw, unsigned ahead) {
    // (a lane's number that is had again at any time: no register holds the thread's through both)
    const int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0));
    const unsigned base = ring<S>(), first = dx.items() % gridDim.x, idle = gridDim.x - first;
    work<T, Does::kDx, S>(p, dx, base, lane, Turns{blockIdx.x, dx.items()});
    const unsigned items = dw.items(), mine = blockIdx.x >= first ? blockIdx.x - first : blockIdx.x + idle;
    unsigned turn = mine < idle ? 0 : ahead;
    work<T, Does::kDw, S>(p, dw, base, lane, [&]() {
        const unsigned item = turn < ahead ? mine + turn * idle : ahead * idle + mine + (turn - ahead) * gridDim.x;
        ++turn;
        return item < items ? item : kNone;
    });
}

// The same for one group of eight columns, outside a tile.
template <typename T, Does DOES>
__device__ __forceinline__ void finish_group(const GluArgs<T>& p, unsigned row, unsigned col, Eight& g, Eight& u) {
    const int there = columns_left(p.n, col);
    const unsigned keep = p.d.active && there > 0 ? keep_span(p.d, effective_offset(p.d), static_cast<uint64_t>(row) * p.n + col) : 0xFFu;
    const bool full = __all(there == 8);
    const Eight dh = DOES == Does::kSlope ? load_some(cell(p.dh, row, p.lddh, col), there, full) : Eight{};
    finish8<T, DOES>(p, keep, row, col, there, full, dh, g, u);
}

// ------------------------------------------------------------------ few tokens
constexpr int kTokenCols = 16;                  // columns of both weights that a workgroup takes

// The waves' sums of a workgroup's 16 columns of both projections, joined in `sums` in the order of the waves, and what becomes of them.
template <typename T, Does DOES, int TB, int WAVES>
__device__ __forceinline__ void finish_tokens(const GluArgs<T>& p, unsigned col0, int lane, int wave, float4v (*sums)[2][TB * 16][4], const float4v (&acc)[2][TB]) {
    const int r = lane & 15, quarter = lane >> 4;
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int c = 0; c < 2; ++c) sums[wave][c][t * 16 + r][quarter] = acc[c][t];
    __syncthreads();
    float4v* const flat = &sums[0][0][0][0];
    constexpr int kFlat = 2 * TB * 16 * kTokenCols / 4;
    for (int i = threadIdx.x; i < kFlat; i += 64 * WAVES) {
        float4v sum = flat[i];
#pragma unroll
        for (int other = 1; other < WAVES; ++other) sum += flat[other * kFlat + i];
        flat[i] = sum;
    }
    __syncthreads();
    constexpr int kGroups = kTokenCols / 8;
    static_assert(TB * 16 * kGroups <= 64 * WAVES, "a lane for each group of eight columns");
    const unsigned token = threadIdx.x / kGroups, group = threadIdx.x % kGroups, col = col0 + group * 8;
    if (token >= p.m || token >= TB * 16 || col >= (DOES == Does::kSlope ? p.ldd : p.n)) return;
    Eight g, u;
#pragma unroll
    for (int e = 0; e < 8; ++e) g.v[e] = sums[0][0][token][group * 2 + e / 4][e % 4], u.v[e] = sums[0][1][token][group * 2 + e / 4][e % 4];
    finish_group<T, DOES>(p, token, col, g, u);
}

// The projections of up to 16 TB tokens.  Every weight is read once and used for all of them, so this is a matter of reading the
// weights.  A workgroup takes 16 columns of both; its WAVES waves take turns along the reduction, 128 bytes of it at a time, and
// their sums meet in LDS.  Each wave stages its own turns' rows, RING of them on their way at a time, and reads them back as the
// matrix instructions want them: no wave waits for another.  (Read straight into registers, neighbouring lanes want rows that
// lie apart, and a compute unit gets 14 bytes a cycle: 64 tokens, n = k = 4096, 25.6 | 19.2 so; 11264 x 4096 68 | 48.)  Workgroups
// begin at different places along the reduction: rows lie a power of two apart, and the same place in all of them is in few of
// the memory's channels.  Weights from memory, bf16: 11264 x 4096 one token 31.5 (5.9 TB/s), 16 tokens 33.4, 32 tokens 38.2.
// Every workgroup reads all of x, from the caches: with 64 tokens twice what it reads of the weights.
template <typename T, Does DOES, int TB, int WAVES, int RING>
__global__ __launch_bounds__(64 * WAVES) void token_kernel(GluArgs<T> p) {
    constexpr int W = sizeof(T), kSpan = kStageBytes / W, kStage = (2 * 16 + TB * 16) * kStageBytes;
    using InW = Operand<T, Lies::kAlong, 16, 1, false>;
    using InX = Operand<T, Lies::kAlong, TB * 16, 1, false>;
    using ReadW = Reader<T, Lies::kAlong, 32, 2, false>;
    using ReadX = Reader<T, Lies::kAlong, TB * 16, TB, false>;
    constexpr int kLoads = 2 * InW::kLoads + InX::kLoads;
    __shared__ alignas(1024) unsigned char lds[WAVES * RING * kStage];
    static_assert(sizeof lds >= sizeof(float4v[WAVES][2][TB * 16][4]), "the sums take the stages' place");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned col0 = blockIdx.x * kTokenCols;
    const unsigned base = static_cast<unsigned>(reinterpret_cast<uintptr_t>((LdsByte*)lds)) + wave * (RING * kStage);
    InW in_w;
    InX in_x;
    in_w.init(0, lane, p.ldw, col0 < p.n ? p.n - col0 : 0);
    in_x.init(0, lane, p.ldx, p.m);
    ReadW read_w;
    ReadX read_x;
    read_w.init(base, 0, lane);
    read_x.init(base + 32 * kStageBytes, 0, lane);
    const unsigned spans = static_cast<unsigned>(div_up(p.k, kSpan)), start = blockIdx.x * 29 % spans;
    const unsigned mine = static_cast<unsigned>(wave) < spans ? (spans - 1 - wave) / WAVES + 1 : 0;
    const uint64_t wg = reinterpret_cast<uint64_t>(cell(p.wg, col0, p.ldw, 0)), wu = reinterpret_cast<uint64_t>(cell(p.wu, col0, p.ldw, 0));
    const auto fetch = [&](unsigned i) {
        const unsigned turn = wave + i * WAVES + start, t = (turn < spans ? turn : turn - spans) * kSpan, to = base + i % RING * kStage;
        const int left = p.k - t;
        in_w.fetch(wg + t * W, 0, left, to);
        in_w.fetch(wu + t * W, 0, left, to + 16 * kStageBytes);
        in_x.fetch(reinterpret_cast<uint64_t>(p.x) + t * W, 0, left, to + 32 * kStageBytes);
    };
    float4v acc[2][TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) acc[0][t] = acc[1][t] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (unsigned i = 0; i < RING; ++i)
        if (i < mine) fetch(i);
    for (unsigned i = 0; i < mine; ++i) {
        if (i + RING <= mine) wait_loads<(RING - 1) * kLoads>();
        else wait_loads<0>();
        const unsigned stage = i % RING * kStage;
        typename Fragment<T>::type f[2][2 + TB];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            f[half][0] = read_w.read(0, half, stage), f[half][1] = read_w.read(1, half, stage);
#pragma unroll
            for (int t = 0; t < TB; ++t) f[half][2 + t] = read_x.read(t, half, stage);
        }
        wait_reads();                                                    // before their place is written again
        if (i + RING < mine) fetch(i + RING);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int t = 0; t < TB; ++t)
#pragma unroll
                for (int c = 0; c < 2; ++c) acc[c][t] = multiply(f[half][c], f[half][2 + t], acc[c][t]);
    }
    __syncthreads();
    finish_tokens<T, DOES, TB, WAVES>(p, col0, lane, wave, reinterpret_cast<float4v(*)[2][TB * 16][4]>(lds), acc);
}

// The parts' sums of the tiles that are summed in parts, joined in the order of the parts.  A lane takes eight neighbouring columns.
// (Sums joined by atomics would depend on who comes first.)  67 MB of sums: 15.
template <typename T, Does DOES, class S>
__device__ __forceinline__ void join(const GluArgs<T>& p, const Plan& plan, unsigned i) {
    using Where = Tile<T, DOES, S>;
    constexpr int kGroups = Where::kCols / 8, kPerTile = S::QT * kGroups;
    const unsigned rest = plan.tp * plan.tq - plan.whole, number = i / kPerTile;
    if (number >= rest) return;
    const int row_in = i % kPerTile / kGroups, col_in = i % kGroups * 8;
    Where tile;
    tile.locate(plan.whole + number, plan.tp, plan.tq);
    const unsigned rows = DOES == Does::kDw ? p.n : p.m, cols = Where::kFold ? p.n : p.k;
    const unsigned row = tile.row0 + row_in, col = tile.col0 + col_in;
    if (row >= rows || col >= (DOES == Does::kSlope ? p.ldd : cols)) return;
    const auto sum = [&](int from) {
        Eight e = {};
        const float* at = plan.sums + static_cast<size_t>(number) * (S::PT * S::QT) + row_in * S::PT + from + col_in;
        const size_t step = static_cast<size_t>(rest) * (S::PT * S::QT);
#pragma unroll 4
        for (unsigned part = 0; part < plan.parts; ++part, at += step) {
            const Eight x = load8(at);
#pragma unroll
            for (int j = 0; j < 8; ++j) e.v[j] += x.v[j];
        }
        return e;
    };
    if constexpr (Where::kFold) {
        Eight g = sum(0), u = sum(S::PT / 2);
        finish_group<T, DOES>(p, row, col, g, u);
    } else {
        const int there = columns_left(cols, col);
        T* const out = DOES == Does::kDx ? p.dx : tile.second ? p.dwu : p.dwg;
        store_some(cell(out, row, DOES == Does::kDx ? p.lddx : p.lddw, col), sum(0), there, __all(there == 8));
    }
}

template <typename T, Does DOES, class S>
__global__ __launch_bounds__(256) void join_kernel(GluArgs<T> p, Plan plan) {
    join<T, DOES, S>(p, plan, blockIdx.x * 256 + threadIdx.x);
}

// The first `blocks` workgroups: dx; the others: dWg and dWu.
template <typename T, class S>
__global__ __launch_bounds__(256) void join_gradients_kernel(GluArgs<T> p, Plan dx, Plan dw, unsigned blocks) {
    if (blockIdx.x < blocks) join<T, Does::kDx, S>(p, dx, blockIdx.x * 256 + threadIdx.x);
    else join<T, Does::kDw, S>(p, dw, (blockIdx.x - blocks) * 256 + threadIdx.x);
}

// dg and du from kept projections; their rows are filled with zeros up to ldd.  Memory bounds it: 4096 x 5632 bf16 42, 5.5 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void slope_kernel(GluArgs<T> p) {
    const unsigned groups = p.ldd / 8;
    const uint64_t total = static_cast<uint64_t>(groups) * p.m, step = static_cast<uint64_t>(gridDim.x) * 256;
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += step) {
        const unsigned row = static_cast<unsigned>(i / groups), col = static_cast<unsigned>(i - static_cast<uint64_t>(row) * groups) * 8;
        const int there = columns_left(p.n, col);
        const bool full = __all(there == 8);
        Eight g = load_some(cell(p.gate_in, row, p.ldp, col), there, full), u = load_some(cell(p.up_in, row, p.ldp, col), there, full);
        finish_group<T, Does::kSlope>(p, row, col, g, u);
    }
}

// A copy of a rows x cols matrix whose rows are filled with zeros up to a multiple of 16 bytes.
template <typename T>
__global__ __launch_bounds__(256) void align_kernel(const T* from, size_t ld, T* to, size_t ld_to, size_t rows, size_t cols) {
    constexpr int kPer = 16 / sizeof(T);
    const uint64_t groups = ld_to / kPer, total = groups * rows, step = static_cast<uint64_t>(gridDim.x) * 256;
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += step) {
        const size_t row = i / groups, col = (i - row * groups) * kPer;
        Pack<T> p;
#pragma unroll
        for (int j = 0; j < kPer; ++j) p.v[j] = col + j < cols ? from[row * ld + col + j] : static_cast<T>(0.f);
        *reinterpret_cast<Pack<T>*>(to + row * ld_to + col) = p;
    }
}

// ------------------------------------------------------------------ host side

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
    constexpr int kGroups = sizeof(T) == 2 ? 2 : 1;
    const size_t blocks = div_up(div_up(total, 8), static_cast<size_t>(kDropThreads) * kGroups);
    const dim3 grid(blocks < kDropRow ? blocks : kDropRow, div_up(blocks, kDropRow));
    return launch(dropout_kernel<T, kGroups>, grid, kDropThreads, stream, static_cast<const T*>(x), ldx, static_cast<const T*>(residual), ldr,
                  static_cast<T*>(y), ldy, cols, total, d);
}

bool sizes_ok(size_t m, size_t n, size_t k) {
    return m <= ZVC_FFN_MAX_ROWS && n <= ZVC_FFN_MAX_COLUMNS && k <= ZVC_FFN_MAX_COLUMNS && m * n <= ZVC_FFN_MAX_ELEMENTS &&
           m * k <= ZVC_FFN_MAX_ELEMENTS;
}

template <typename T>
void set_sizes(GluArgs<T>* p, size_t ldx, size_t ldw, size_t ldp, size_t m, size_t n, size_t k, int activation, const Drop& d) {
    p->ldx = static_cast<unsigned>(ldx), p->ldw = static_cast<unsigned>(ldw), p->ldp = static_cast<unsigned>(ldp);
    p->m = static_cast<unsigned>(m), p->n = static_cast<unsigned>(n), p->k = static_cast<unsigned>(k);
    p->act = activation, p->d = d;
}

bool stride_ok(size_t ld, size_t cols) { return ld >= cols && ld <= ZVC_FFN_MAX_COLUMNS; }

using Large = Shape<4, 2, 4, 8, 2>;             // 256 x 256, eight waves
using Small = Shape<2, 2, 4, 4, 2>;             // 128 x 128, four waves
// The same for projections, of eight waves, among which an epilogue's long functions hide better: 777 x 2730 x 1000 fp16 with gelu
// 23.2 -> 21.8, computed again for its gradients 66.0 -> 63.4; with short functions, larger or in fp32 the same within 1 %.
using Eights = Shape<2, 4, 4, 2, 2>;
using Thin = Shape<4, 1, 4, 2, 2>;              // 256 x 32, four waves: few tokens
using Lone = Shape<2, 4, 4, 2, 4>;              // 128 x 128, eight waves, alone on a compute unit: a deeper ring
using Half = Shape<2, 2, 4, 2, 4>;              // 128 x 64, four waves, the same

constexpr double kAlone = 0.6;                  // a stage's time where one workgroup has a compute unit that takes two
constexpr double kJoinUs = 3, kSumsPerUs = 3e6;

// Tiles of a product of this shape, by columns and rows.
template <Does DOES, class S>
void tiles_of(size_t m, size_t n, size_t k, size_t* cols, size_t* rows) {
    constexpr bool kFold = DOES == Does::kForward || DOES == Does::kSlope;
    *cols = kFold ? div_up(n, S::PT / 2) : div_up(k, S::PT);
    *rows = DOES == Does::kDw ? 2 * div_up(n, S::QT) : div_up(m, S::QT);
}

enum class Size { kLarge, kSmall, kThin, kLone, kHalf, kTokens };

// How a product is cut: the tiles' shape, how many tiles are summed whole, and in how many parts of the reduction the others are,
// to be joined by a second kernel.  kTokens: no tiles, but the kernel for few tokens.
struct Cut {
    Size size;
    unsigned whole, parts;
    size_t sums;                                // bytes of the parts' sums
    double cost;
};

// The cut that takes the least time by this account, in us: workgroups take items in rounds; an item costs its stages and
// something to begin and finish; joining costs a launch and the sums' way to memory and back.  The stages' times are fitted to
// calls with every cut forced in turn (L, S: large and small tiles, S of four waves): 4096 x 5632 x 2048 L 175, S 171, but with outputs kept and
// other work around them 210 and 250; 2048 x 5632 x 2048 L 101, L in 2 parts behind the first round 98, S 93.  The account's choice
// is within 15 % of the best of them.  Where the tiles are one round or less, a workgroup alone on a compute unit hides memory's
// latency by a deeper ring: 512 x 4096 x 4096 128 x 128 tiles 42.6 (small 60), 128 x 64 68; 256 x 4096 x 4096 35.3 (43), 128 x 64 33.3;
// 256 x 2816 x 1024 11.8 (14.3), 128 x 64 11.0; 128 x 11264 x 4096 50.3 (66); but 1024 x 4096 x 4096 78 (73) and 777 x 2730 x 1000 26 (23).
template <class S>
void try_cut(Size size, double stage_us, double item_us, size_t m, size_t n, size_t k, size_t w, Cut* best) {
    size_t cols, rows;
    tiles_of<Does::kForward, S>(m, n, k, &cols, &rows);
    const size_t tiles = cols * rows, slots = kUnits * S::kPerUnit;
    const size_t stages = div_up(k, kStageBytes / w);
    const auto rounds = [&](size_t items, size_t stages_each) {
        const size_t last = items % slots;             // alone on its compute unit, an item of two takes less time
        const double alone = last != 0 && last <= kUnits && slots > kUnits ? kAlone : 1;
        return items / slots * (stages_each * stage_us + item_us) + (last != 0 ? stages_each * stage_us * alone + item_us : 0);
    };
    const auto consider = [&](size_t whole, size_t parts) {
        const size_t rest = tiles - whole;
        const double sums = parts > 1 ? 4.0 * S::PT * S::QT * rest * parts : 0;
        const double cost = rounds(whole, stages) + rounds(rest * parts, div_up(stages, parts)) + (parts > 1 ? kJoinUs + sums / kSumsPerUs : 0);
        if (cost < best->cost) *best = {size, static_cast<unsigned>(whole), static_cast<unsigned>(parts), static_cast<size_t>(sums), cost};
    };
    consider(tiles, 1);
    const size_t full = tiles / slots * slots;
    for (size_t parts = 2; parts <= 32 && parts * 2 <= stages; ++parts)
        if (full != tiles) consider(full, parts);
}

// Whether m tokens take the kernel for few of them.  us (weights from memory), tiles | that kernel: bf16 n = k = 4096, 1 token
// 22.6 | 13.2, 32 23.1 | 14.7, 64 22.7 | 19.6, 96 28.1 | 22.9, 128 28.6 | 26.6; 11264 x 4096, 1 token 45.6 | 31.5, 48 42.7 | 42.5,
// 64 42.8 | 48.5, 96 46.8 | 60.6; 5632 x 2048, 64 19.5 | 18.6, 96 19.3 | 23.9; 2816 x 1024, 96 10.6 | 7.8, 128 10.6 | 9.4.  fp32, where
// the products come in sooner: n = k = 4096, 32 tokens 38.9 | 29, 48 48.7 | 39; 11264 x 4096, 48 122 | 109, 64 126 | 134; 2816 x 1024,
// 64 18.3 | 14.5.  So more than 48 only where every workgroup has a compute unit of its own.
bool few_tokens(size_t m, size_t n, size_t w) { return m <= 48 || (m <= (w == 4 ? 64 : 128) && n <= kUnits * kTokenCols); }

// The projections' cut.
Cut cut_of(size_t m, size_t n, size_t k, size_t w) {
    if (k != 0 && few_tokens(m, n, w)) return {Size::kTokens, 0, 1, 0, 0};
    Cut best{Size::kSmall, 0, 1, 0, 1e300};
    if (w == 4) {                                // the products bound it, whatever the tile; a stage is 32 steps
        try_cut<Eights>(Size::kSmall, 3.8, 5, m, n, k, w, &best);
        try_cut<Thin>(Size::kThin, 1.95, 4, m, n, k, w, &best);
        return best;
    }
    try_cut<Large>(Size::kLarge, 1.45, 8, m, n, k, w, &best);
    try_cut<Eights>(Size::kSmall, 0.85, 5, m, n, k, w, &best);
    try_cut<Thin>(Size::kThin, 0.9, 4, m, n, k, w, &best);
    try_cut<Lone>(Size::kLone, 0.45, 5, m, n, k, w, &best);
    try_cut<Half>(Size::kHalf, 0.32, 4, m, n, k, w, &best);
    return best;
}

// How dx's and dW's products are cut, of one tile shape, and how many items of dW go ahead where dx leaves compute units idle.
struct Pair {
    Cut dx, dw;
    unsigned ahead;
    double cost;
};

// The pair that takes the least time by the same account: the most loaded workgroup's items, and the joining.  With every pair
// forced in turn (tiles, parts of dx, parts of dW, ahead), the gradients and dg, du: 4096 x 5632 x 2048 bf16 L 1 1 3 347, L 2 1 0 374,
// S 1 2 0 422; 2048 x 2816 x 1024 L 3 1 1 78, S 3 1 0 79, thin 101; 512 x 4096 x 4096 S 2 1 5 115, L 3 1 4 117; 1024 x 5632 x 2048 L 4 1 2 123,
// L 3 1 3 (taken) 131; 64 x 4096 x 4096 S 8 1 4 57, S 6 1 5 (taken) 55, L 63, thin 62; 777 x 2730 x 1000 S 3 1 2 49, L 6 1 0 (taken) 50.
// The account's choice is within 7 % of the best.  Either product in a launch of its own, each cut for itself: 389, 100, 117, 143.
template <class S>
void try_pair(Size size, double dx_us, double dw_us, double item_us, size_t m, size_t n, size_t k, size_t w, Pair* best) {
    static constexpr unsigned kParts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
    struct Side {                                // one of the two products, with the parts that are tried
        size_t tiles, stages;
        double stage_us;
        unsigned whole, parts, items;
        double each, longest, sums;
    };
    size_t cols, rows;
    tiles_of<Does::kDx, S>(m, n, k, &cols, &rows);
    Side x{cols * rows, 2 * div_up(n, kStageBytes / w), dx_us, 0, 0, 0, 0, 0, 0};
    tiles_of<Does::kDw, S>(m, n, k, &cols, &rows);
    Side y{cols * rows, div_up(m, kStageBytes / w), dw_us, 0, 0, 0, 0, 0, 0};
    const unsigned slots = kUnits * S::kPerUnit;
    const auto set = [&](Side* side, unsigned parts, double alone) {
        const unsigned full = static_cast<unsigned>(side->tiles / slots * slots);
        if (parts > 1 && (full == side->tiles || parts * 2 > side->stages)) return false;
        side->parts = parts;
        side->whole = parts == 1 ? static_cast<unsigned>(side->tiles) : full;
        const unsigned rest = static_cast<unsigned>(side->tiles) - side->whole;
        side->items = side->whole + rest * parts;
        side->longest = side->stages * side->stage_us * alone + item_us;
        const double short_one = div_up(side->stages, parts) * side->stage_us * alone + item_us;
        side->each = side->items == 0 ? 0 : (side->whole * side->longest + rest * parts * short_one) / side->items;
        side->sums = parts > 1 ? 4.0 * S::PT * S::QT * rest * parts : 0;
        return true;
    };
    for (const unsigned parts_x : kParts)
        for (const unsigned parts_y : kParts) {
            if (!set(&x, parts_x, 1) || !set(&y, parts_y, 1)) continue;
            if (slots > kUnits && x.items + y.items <= kUnits) set(&x, parts_x, kAlone), set(&y, parts_y, kAlone);
            const unsigned first = x.items % slots, idle = slots - first;
            const double turns = x.items / slots * x.each;
            const double joining = x.sums + y.sums > 0 ? kJoinUs + (x.sums + y.sums) / kSumsPerUs : 0;
            const unsigned most = first == 0 || y.each == 0 ? 0 : static_cast<unsigned>(x.each / y.each + 0.5);
            for (const unsigned ahead : {0u, most}) {
                const unsigned behind = y.items > ahead * idle ? y.items - ahead * idle : 0, round = behind / slots, last = behind % slots;
                const unsigned early = behind > 0 ? ahead : static_cast<unsigned>(div_up(y.items, idle));
                const double of_idle = (early + round + (last > 0 ? 1 : 0)) * y.each;
                const double of_others = first == 0 ? 0 : x.each + (round + (last > idle ? 1 : 0)) * y.each;
                const double cost = turns + (of_idle > of_others ? of_idle : of_others) + joining;
                if (cost < best->cost)
                    *best = {{size, x.whole, x.parts, static_cast<size_t>(x.sums), 0}, {size, y.whole, y.parts, static_cast<size_t>(y.sums), 0}, ahead, cost};
            }
        }
}

Pair pair_of(size_t m, size_t n, size_t k, size_t w) {
    const Cut none{Size::kSmall, 0, 1, 0, 0};
    Pair best{none, none, 0, 1e300};
    if (w == 4) {
        try_pair<Small>(Size::kSmall, 3.8, 3.8, 5, m, n, k, w, &best);
        try_pair<Thin>(Size::kThin, 1.95, 1.95, 4, m, n, k, w, &best);
        return best;
    }
    try_pair<Large>(Size::kLarge, 1.55, 1.6, 8, m, n, k, w, &best);
    try_pair<Small>(Size::kSmall, 1.1, 1.1, 5, m, n, k, w, &best);
    try_pair<Thin>(Size::kThin, 0.9, 0.9, 4, m, n, k, w, &best);
    return best;
}

template <Does DOES, class S>
Plan plan_of(const Cut& cut, size_t m, size_t n, size_t k, float* sums) {
    size_t cols, rows;
    tiles_of<DOES, S>(m, n, k, &cols, &rows);
    return {sums, static_cast<unsigned>(cols), static_cast<unsigned>(rows), cut.whole, cut.parts, false};
}

// The blocks of a join, 0 where there is none.
template <typename T, Does DOES, class S>
unsigned join_blocks(const Plan& plan) {
    if (plan.parts == 1) return 0;
    return static_cast<unsigned>(div_up(size_t{plan.tp * plan.tq - plan.whole} * (S::QT * Tile<T, DOES, S>::kCols / 8), 256));
}

constexpr size_t kCacheBytes = size_t{256} << 20, kL2Bytes = size_t{32} << 20;      // in front of the memory; of the XCDs' L2 together
constexpr unsigned kLongSum = 2048;              // k from which on the products take longer than the outputs' way to memory

// Whether a forward call's outputs go past the caches and leave the operands there: as much as the caches hold or more, or an h
// larger than L2 behind long sums; in rows that are whole halves of the memory's 128 bytes (others are written in pieces that nothing
// puts together any more).  us, past | not, relu and dropout, alone, with a product that reads h, with the codec that reads the kept
// projections or else h: 8192 x 5632 x 2048 kept (264 MB in all) 340 | 370, 474 | 495, 399 | 403; 16384 x 8192 x 512 (256) 309 | 333, 473 | 507,
// 395 | 401; 16384 x 11264 x 1024 (352) 680 | 740, 942 | 988, 790 | 838.  Short sums and less: 8192 x 4096 x 1024 kept (192) 164 | 151, 222 | 208,
// 212 | 190; 1024 x 8192 x 128 kept (48) 25 | 20.6, 41 | 35, 43 | 39.  Long sums and less, three sets of inputs in turn: 4096 x 5632 x 2048 (44) 159 | 169,
// kept (132) 178 | 189; 8192 x 4096 x 2048 kept (192) 245 | 274; in a chain of eight blocks, each with its product and dropout, the first
// 269 | 271, 291 | 291, with the codec 331 | 324.  Rows of 11280 bytes: 8192 x 5640 x 2048 kept 434 | 389, 589 | 543, 492 | 417; of 11328 343 | 374, 486 | 518, 400 | 408.
template <typename T>
bool past_caches(const GluArgs<T>& p) {
    const auto whole = [&](const T* at, unsigned ld) { return at == nullptr || (aligned_to(at, 64) && size_t{ld} * sizeof(T) % 64 == 0); };
    const size_t bytes = size_t{p.m} * p.n * sizeof(T), all = p.gate != nullptr ? 3 * bytes : bytes;
    return (all >= kCacheBytes || (p.k >= kLongSum && bytes > kL2Bytes)) && whole(p.h, p.ldh) && whole(p.gate, p.ldp) && whole(p.up, p.ldp);
}

template <typename T, Does DOES, class S>
zvc_status product_of(const GluArgs<T>& p, const Cut& cut, float* sums, hipStream_t stream) {
    Plan plan = plan_of<DOES, S>(cut, p.m, p.n, p.k, sums);
    plan.past = DOES == Does::kForward && S::QT >= 256 && past_caches(p);
    const unsigned items = plan.items(), room = kUnits * S::kPerUnit;
    const zvc_status st = launch(product_kernel<T, DOES, S>, dim3(items < room ? items : room), S::kThreads, stream, p, plan);
    const unsigned blocks = join_blocks<T, DOES, S>(plan);
    return st != ZVC_OK || blocks == 0 ? st : launch(join_kernel<T, DOES, S>, dim3(blocks), 256, stream, p, plan);
}

// dx and dW, or what of them is wanted: cut the same way in any case.
template <typename T, class S>
zvc_status gradients_of(const GluArgs<T>& p, const Pair& pair, float* sums, hipStream_t stream) {
    Plan dx = plan_of<Does::kDx, S>(pair.dx, p.m, p.n, p.k, sums), dw = plan_of<Does::kDw, S>(pair.dw, p.m, p.n, p.k, sums + pair.dx.sums / 4);
    const Plan nothing{nullptr, 0, 0, 0, 1, false};
    if (p.dx == nullptr) dx = nothing;
    if (p.dwg == nullptr) dw = nothing;
    const unsigned items = dx.items() + dw.items(), room = kUnits * S::kPerUnit;
    if (items == 0) return ZVC_OK;
    // (fewer workgroups than a round holds take one item each)
    const zvc_status st = launch(gradients_kernel<T, S>, dim3(items < room ? items : room), S::kThreads, stream, p, dx, dw, items < room ? 0u : pair.ahead);
    const unsigned blocks = join_blocks<T, Does::kDx, S>(dx), more = join_blocks<T, Does::kDw, S>(dw);
    return st != ZVC_OK || blocks + more == 0 ? st : launch(join_gradients_kernel<T, S>, dim3(blocks + more), 256, stream, p, dx, dw, blocks);
}

template <typename T, Does DOES, int TB, int WAVES, int RING>
zvc_status tokens_of(const GluArgs<T>& p, hipStream_t stream) {
    const size_t cols = DOES == Does::kSlope ? p.ldd : p.n;
    return launch(token_kernel<T, DOES, TB, WAVES, RING>, dim3(div_up(cols, kTokenCols)), 64 * WAVES, stream, p);
}

template <typename T, Does DOES>
zvc_status project(const GluArgs<T>& p, const Cut& cut, float* sums, hipStream_t stream) {
    if (cut.size == Size::kTokens) {
        // (waves and ring: most of LDS, as one workgroup or as two of which one reads while the other finishes.  11264 x 4096 bf16, 16 tokens
        // 4 x 3 33.4, 8 x 3 36.6, 4 x 6 36.9; 32: 4 x 2 38.2, 4 x 3 40.6, 8 x 2 40.7, 2 x 4 44.2; 64: 3 x 2 48.4, 4 x 3 50, 6 x 2 51.7, 2 x 3 56)
        if (p.m <= 16) return tokens_of<T, DOES, 1, 4, 3>(p, stream);
        if (p.m <= 32) return tokens_of<T, DOES, 2, 4, 2>(p, stream);
        if (p.m <= 48) return tokens_of<T, DOES, 3, 4, 2>(p, stream);
        if constexpr (sizeof(T) == 2) {
            if (p.m <= 64) return tokens_of<T, DOES, 4, 3, 2>(p, stream);
            return p.m <= 96 ? tokens_of<T, DOES, 6, 4, 2>(p, stream) : tokens_of<T, DOES, 8, 4, 2>(p, stream);
        } else {
            return tokens_of<T, DOES, 4, 4, 3>(p, stream);
        }
    }
    if constexpr (sizeof(T) == 2) {
        if (cut.size == Size::kLarge) return product_of<T, DOES, Large>(p, cut, sums, stream);
        if (cut.size == Size::kLone) return product_of<T, DOES, Lone>(p, cut, sums, stream);
        if (cut.size == Size::kHalf) return product_of<T, DOES, Half>(p, cut, sums, stream);
    }
    return cut.size == Size::kSmall ? product_of<T, DOES, Eights>(p, cut, sums, stream) : product_of<T, DOES, Thin>(p, cut, sums, stream);
}

template <typename T>
zvc_status gradients(const GluArgs<T>& p, const Pair& pair, float* sums, hipStream_t stream) {
    if constexpr (sizeof(T) == 2)
        if (pair.dx.size == Size::kLarge) return gradients_of<T, Large>(p, pair, sums, stream);
    return pair.dx.size == Size::kSmall ? gradients_of<T, Small>(p, pair, sums, stream) : gradients_of<T, Thin>(p, pair, sums, stream);
}

constexpr size_t kColumnsUp = 64;               // dg's and du's rows are filled up to a multiple of this

// Where the parts of a workspace begin.
struct Layout {
    size_t dg, du, x, wg, wu, sums, bytes;
    size_t ldd, aligned_k;              // row strides of dg and du, and of the copies of x, Wg and Wu
    Cut cut;                            // of the projections
    Pair pair;                          // of the gradients
};

// `copies`: x, Wg and Wu do not all take 16-byte accesses.
Layout layout_of(size_t m, size_t n, size_t k, size_t w, bool backward, bool copies) {
    Layout at{};
    at.ldd = round_up(n, kColumnsUp);
    at.aligned_k = round_up(k, 16 / w);
    const auto part = [&](size_t bytes) {
        const size_t begin = at.bytes;
        at.bytes += round_up(bytes, 256);
        return begin;
    };
    if (backward) at.dg = part(m * at.ldd * w), at.du = part(m * at.ldd * w);
    if (copies) at.x = part(m * at.aligned_k * w), at.wg = part(n * at.aligned_k * w), at.wu = part(n * at.aligned_k * w);
    at.cut = cut_of(m, n, k, w);
    size_t sums = at.cut.sums;
    if (backward) {
        at.pair = pair_of(m, n, k, w);
        if (at.pair.dx.sums + at.pair.dw.sums > sums) sums = at.pair.dx.sums + at.pair.dw.sums;
    }
    at.sums = part(sums);
    at.bytes += 256;
    return at;
}

// Copies of x and the weights where they do not take 16-byte accesses as they lie.
template <typename T>
zvc_status align_inputs(GluArgs<T>* p, const Layout& at, unsigned char* base, hipStream_t stream) {
    const auto copy = [&](const T** from, unsigned* ld, size_t rows, size_t to) {
        if (rows == 0 || p->k == 0) return ZVC_OK;
        T* const out = reinterpret_cast<T*>(base + to);
        const size_t blocks = div_up(rows * at.aligned_k * sizeof(T) / 16, 256);
        const zvc_status st = launch(align_kernel<T>, dim3(blocks < 65536 ? blocks : 65536), 256, stream, *from, size_t{*ld}, out,
                                     at.aligned_k, rows, size_t{p->k});
        *from = out;
        *ld = static_cast<unsigned>(at.aligned_k);
        return st;
    };
    const bool odd = p->k * sizeof(T) % 16 != 0;
    if (odd || !aligned_to(p->x, 16) || p->ldx * sizeof(T) % 16 != 0)
        if (zvc_status st = copy(&p->x, &p->ldx, p->m, at.x)) return st;
    if (odd || !aligned_to(p->wg, 16) || !aligned_to(p->wu, 16) || p->ldw * sizeof(T) % 16 != 0) {
        unsigned ld = p->ldw;
        if (zvc_status st = copy(&p->wg, &ld, p->n, at.wg)) return st;
        return copy(&p->wu, &p->ldw, p->n, at.wu);
    }
    return ZVC_OK;
}

template <typename T>
zvc_status forward_as(GluArgs<T> p, const Layout& at, unsigned char* base, hipStream_t stream) {
    if (zvc_status st = align_inputs(&p, at, base, stream)) return st;
    return project<T, Does::kForward>(p, at.cut, reinterpret_cast<float*>(base + at.sums), stream);
}

template <typename T>
zvc_status backward_as(GluArgs<T> p, T* dx, size_t lddx, T* dwg, T* dwu, size_t lddw, const Layout& at, unsigned char* base,
                       hipStream_t stream) {
    if (zvc_status st = align_inputs(&p, at, base, stream)) return st;
    float* const sums = reinterpret_cast<float*>(base + at.sums);
    if (p.m != 0 && p.n != 0) {
        zvc_status st;
        if (p.gate_in == nullptr) {
            st = project<T, Does::kSlope>(p, at.cut, sums, stream);
        } else {
            const size_t blocks = div_up(size_t{p.m} * (p.ldd / 8), 256);
            st = launch(slope_kernel<T>, dim3(blocks < 65536 ? blocks : 65536), 256, stream, p);
        }
        if (st != ZVC_OK) return st;
    }
    p.dx = p.m != 0 ? dx : nullptr, p.lddx = static_cast<unsigned>(lddx);
    p.dwg = p.n != 0 ? dwg : nullptr, p.dwu = dwu, p.lddw = static_cast<unsigned>(lddw);
    return gradients(p, at.pair, sums, stream);
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
    return w == 0 || !sizes_ok(m, n, k) ? 0 : layout_of(m, n, k, w, backward != 0, loose != 0 || k * w % 16 != 0).bytes;
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
    const Layout at = layout_of(m, n, k, w, false, loose || k * w % 16 != 0);
    if (ws < at.bytes) return ZVC_E_WORKSPACE;
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
        GluArgs<T> p{};
        p.x = static_cast<const T*>(d_x), p.wg = static_cast<const T*>(d_wg), p.wu = static_cast<const T*>(d_wu);
        p.h = static_cast<T*>(d_h), p.gate = static_cast<T*>(d_gate), p.up = static_cast<T*>(d_up);
        set_sizes(&p, ldx, ldw, ldp, m, n, k, activation, d);
        p.ldh = static_cast<unsigned>(ldh);
        return forward_as(p, at, static_cast<unsigned char*>(d_ws), stream);
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
    const Layout at = layout_of(m, n, k, w, true, loose || k * w % 16 != 0);
    if (ws < at.bytes) return ZVC_E_WORKSPACE;
    const Region in[] = {{d_dh, lddh * w, m, n * w}, {d_x, ldx * w, m, k * w}, {d_wg, ldw * w, n, k * w},
                         {d_wu, ldw * w, n, k * w}, {d_gate, ldp * w, m, n * w}, {d_up, ldp * w, m, n * w}};
    const Region out[] = {{d_dx, lddx * w, m, k * w}, {d_dwg, lddw * w, n, k * w}, {d_dwu, lddw * w, n, k * w}, {d_ws, ws, 1, ws}};
    for (int i = 0; i < 4; ++i) {
        for (const Region& r : in)
            if (overlap(out[i], r)) return ZVC_E_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return ZVC_E_ARG;
    }
    const auto as = [&](auto zero) {
        using T = decltype(zero);
        unsigned char* const base = static_cast<unsigned char*>(d_ws);
        GluArgs<T> p{};
        p.x = static_cast<const T*>(d_x), p.wg = static_cast<const T*>(d_wg), p.wu = static_cast<const T*>(d_wu);
        p.dh = static_cast<const T*>(d_dh), p.gate_in = static_cast<const T*>(d_gate), p.up_in = static_cast<const T*>(d_up);
        p.dg = reinterpret_cast<T*>(base + at.dg), p.du = reinterpret_cast<T*>(base + at.du);
        set_sizes(&p, ldx, ldw, ldp, m, n, k, activation, d);
        p.lddh = static_cast<unsigned>(lddh), p.ldd = static_cast<unsigned>(at.ldd);
        return backward_as(p, static_cast<T*>(d_dx), lddx, static_cast<T*>(d_dwg), static_cast<T*>(d_dwu), lddw, at, base, stream);
    };
    return type == ZVC_FP32 ? as(0.f) : type == ZVC_FP16 ? as(fp16{}) : as(bf16{});
}

}  // extern "C"
