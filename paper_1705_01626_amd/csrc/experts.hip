// Router and matrix products for mixtures of experts, forward and backward, for AMD gfx950 (wave64): kernels and C ABI
// (include/zvc_experts.h has the formulas).

#include "tiles.h"
#include "zvc_experts.h"

#include <cmath>

namespace {

// ------------------------------------------------------------------ the router
constexpr int kRowLanes = 16;                   // lanes that share a token
constexpr int kRouteThreads = 512;
constexpr unsigned kRouteTokens = kRouteThreads / kRowLanes;        // of a workgroup: a bit for each in a word
constexpr float kOut = -INFINITY;               // an expert that is out, or taken

// x of the lane that is N further on within 16 lanes, around.
template <int N>
__device__ __forceinline__ int turned(int x) { return __builtin_amdgcn_update_dpp(0, x, 0x120 + N, 0xF, 0xF, false); }
template <int N>
__device__ __forceinline__ float turned(float x) { return __builtin_bit_cast(float, turned<N>(__builtin_bit_cast(int, x))); }

// Over 16 lanes, in all of them.
template <typename X, typename F>
__device__ __forceinline__ X over_row(X x, F f) {
    x = f(x, turned<8>(x));
    x = f(x, turned<4>(x));
    x = f(x, turned<2>(x));
    return f(x, turned<1>(x));
}
__device__ __forceinline__ float row_max(float x) { return over_row(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ int row_min(int x) { return over_row(x, [](int a, int b) { return min(a, b); }); }
__device__ __forceinline__ float row_sum(float x) { return over_row(x, [](float a, float b) { return a + b; }); }

// A token's logits over its 16 lanes: CHUNKS times 16 bytes each, side by side.
template <typename T, int CHUNKS>
struct Logits {
    static constexpr int kPer = 16 / sizeof(T), kAll = CHUNKS * kPer;
    float v[kAll];

    static __device__ __forceinline__ int column(int i, int lane) { return (i / kPer * kRowLanes + lane) * kPer + i % kPer; }

    // kOut for what is out and behind the last expert.
    __device__ __forceinline__ void load(const T* row, int experts, int lane) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = column(c * kPer, lane);
            Pack<T> p;
            if (at + kPer <= experts) {
                __builtin_memcpy(&p, row + at, 16);
            } else {
#pragma unroll
                for (int j = 0; j < kPer; ++j) p.v[j] = at + j < experts ? row[at + j] : static_cast<T>(kOut);
            }
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const float x = static_cast<float>(p.v[j]);
                v[c * kPer + j] = x > kOut ? x : kOut;
            }
        }
    }
    __device__ __forceinline__ float most() const {
        float m = v[0];
#pragma unroll
        for (int i = 1; i < kAll; ++i) m = fmaxf(m, v[i]);
        return m;
    }
};

struct RouteArgs {
    const void* logits;
    size_t ldl;
    int32_t* chosen;
    float* weights;
    int64_t *offsets, *order, *place;
    unsigned* counts;            // experts x blocks, then each expert's total
    unsigned m, experts, top, blocks;
    bool normalize;
};

__device__ __forceinline__ float weight_of(float logit, float most) { return logit > kOut ? expf(logit - most) : 0.f; }

// Chooses a token's experts: lane s of the 16 gets choice s (-1: none) and its weight.
template <typename T, int CHUNKS>
__device__ __forceinline__ void choose(const RouteArgs& p, unsigned token, int lane, int* expert, float* weight) {
    Logits<T, CHUNKS> l;
    l.load(static_cast<const T*>(p.logits) + static_cast<size_t>(token) * p.ldl, p.experts, lane);
    float logit = kOut, sum = 0.f;
    const float most = row_max(l.most());
    if (!p.normalize) {
#pragma unroll
        for (int i = 0; i < l.kAll; ++i) sum += weight_of(l.v[i], most);
        sum = row_sum(sum);
    }
    *expert = -1;
    for (unsigned s = 0; s < p.top; ++s) {
        const float best = s == 0 ? most : row_max(l.most());
        int at = 1 << 30;
#pragma unroll
        for (int i = l.kAll - 1; i >= 0; --i) at = l.v[i] == best ? l.column(i, lane) : at;
        at = row_min(at);
        if (static_cast<unsigned>(lane) == s && best > kOut) *expert = at, logit = best;
#pragma unroll
        for (int i = 0; i < l.kAll; ++i) l.v[i] = l.column(i, lane) == at ? kOut : l.v[i];
    }
    const float e = weight_of(logit, most);
    if (p.normalize) sum = row_sum(e);
    *weight = *expert >= 0 ? e / sum : 0.f;
}

// Inclusive sums over a workgroup's threads in their order.  `room`: a word for each wave.
template <int THREADS>
__device__ __forceinline__ unsigned running_sum(unsigned x, unsigned* room) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const unsigned before = __shfl_up(x, d);
        x += lane >= d ? before : 0;
    }
    if (lane == 63) room[wave] = x;
    __syncthreads();
    for (int w = 0; w < wave; ++w) x += room[w];
    __syncthreads();
    return x;
}

// Where each expert's rows begin, and the end of the last's, from `count(e)`, in `starts`.
template <typename F>
__device__ __forceinline__ void starts_of(unsigned experts, unsigned* starts, unsigned* room, F count) {
    constexpr unsigned kEach = ZVC_EXPERTS_MAX / kRouteThreads;
    unsigned own[kEach], sum = 0;
#pragma unroll
    for (unsigned j = 0; j < kEach; ++j) {
        const unsigned e = threadIdx.x * kEach + j;
        own[j] = e < experts ? count(e) : 0;
        sum += own[j];
    }
    unsigned at = running_sum<kRouteThreads>(sum, room) - sum;
#pragma unroll
    for (unsigned j = 0; j < kEach; ++j) {
        const unsigned e = threadIdx.x * kEach + j;
        if (e <= experts) starts[e] = at;
        at += own[j];
    }
    if (experts == ZVC_EXPERTS_MAX && threadIdx.x == kRouteThreads - 1) starts[experts] = at;
    __syncthreads();
}

// The workgroup's 32 tokens: their choices and weights, and for each expert a word of the tokens that have it.  An entry's rank among
// the workgroup's of its expert is the number of earlier tokens in that word.  ALONE: there is no other workgroup, and the places are final.
template <typename T, int CHUNKS, bool ALONE>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(RouteArgs p) {
    __shared__ unsigned having[ZVC_EXPERTS_MAX], starts[ALONE ? ZVC_EXPERTS_MAX + 1 : 1], room[kRouteThreads / 64];
    const int lane = threadIdx.x % kRowLanes, slot = threadIdx.x / kRowLanes;
    const unsigned token = blockIdx.x * kRouteTokens + slot;
    for (unsigned e = threadIdx.x; e < p.experts; e += kRouteThreads) having[e] = 0;
    __syncthreads();
    int expert = -1;
    float weight = 0.f;
    const bool there = token < p.m && static_cast<unsigned>(lane) < p.top;
    const size_t entry = static_cast<size_t>(token) * p.top + lane;
    if (token < p.m) choose<T, CHUNKS>(p, token, lane, &expert, &weight);
    if (there) {
        p.chosen[entry] = expert, p.weights[entry] = weight;
        if (expert >= 0) atomicOr(&having[expert], 1u << slot);
    }
    __syncthreads();
    const unsigned rank = expert >= 0 ? __popc(having[expert] & ((1u << slot) - 1u)) : 0;
    if constexpr (ALONE) {
        starts_of(p.experts, starts, room, [&](unsigned e) { return static_cast<unsigned>(__popc(having[e])); });
        for (unsigned e = threadIdx.x; e <= p.experts; e += kRouteThreads) p.offsets[e] = starts[e];
        if (there) {
            const int64_t row = expert >= 0 ? static_cast<int64_t>(starts[expert]) + rank : -1;
            p.place[entry] = row;
            if (row >= 0) p.order[row] = static_cast<int64_t>(entry);
            if (entry >= starts[p.experts]) p.order[entry] = -1;
        }
    } else {
        if (there) p.place[entry] = rank;
        for (unsigned e = threadIdx.x; e < p.experts; e += kRouteThreads)
            p.counts[static_cast<size_t>(e) * p.blocks + blockIdx.x] = __popc(having[e]);
    }
}

// A wave an expert: its counts by workgroup become sums of those before, and their total is written behind all counts.
__global__ __launch_bounds__(64) void route_sums_kernel(RouteArgs p) {
    unsigned* const counts = p.counts + static_cast<size_t>(blockIdx.x) * p.blocks;
    unsigned before = 0;
    for (unsigned at = 0; at < p.blocks; at += 64) {
        const unsigned b = at + threadIdx.x, own = b < p.blocks ? counts[b] : 0;
        unsigned x = own;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const unsigned other = __shfl_up(x, d);
            x += static_cast<int>(threadIdx.x) >= d ? other : 0;
        }
        if (b < p.blocks) counts[b] = before + x - own;
        before += __shfl(x, 63);
    }
    if (threadIdx.x == 0) p.counts[static_cast<size_t>(p.experts) * p.blocks + blockIdx.x] = before;
}

// Ranks become rows.
__global__ __launch_bounds__(kRouteThreads) void route_places_kernel(RouteArgs p) {
    __shared__ unsigned starts[ZVC_EXPERTS_MAX + 1], room[kRouteThreads / 64];
    const unsigned* const totals = p.counts + static_cast<size_t>(p.experts) * p.blocks;
    starts_of(p.experts, starts, room, [&](unsigned e) { return totals[e]; });
    if (blockIdx.x == 0)
        for (unsigned e = threadIdx.x; e <= p.experts; e += kRouteThreads) p.offsets[e] = starts[e];
    const unsigned per = kRouteTokens * p.top, entries = p.m * p.top, first = blockIdx.x * per;
    const unsigned end = entries - first < per ? entries : first + per;
    for (unsigned i = first + threadIdx.x; i < end; i += kRouteThreads) {
        const int expert = p.chosen[i];
        int64_t row = -1;
        if (expert >= 0) {
            row = static_cast<int64_t>(starts[expert]) + p.counts[static_cast<size_t>(expert) * p.blocks + blockIdx.x] + p.place[i];
            p.order[row] = i;
        }
        p.place[i] = row;
        if (i >= starts[p.experts]) p.order[i] = -1;
    }
}

struct RouteBackArgs {
    const float* dweights;
    const void* logits;
    size_t ldl, ldd;
    const int32_t* chosen;
    void* dlogits;
    unsigned m, experts, top;
    bool normalize;
};

// Lane s of a token's 16 has its choice s; every lane has some columns and looks all choices over for each.
template <typename T, int CHUNKS>
__global__ __launch_bounds__(256) void route_backward_kernel(RouteBackArgs p) {
    const int lane = threadIdx.x % kRowLanes;
    const unsigned token = blockIdx.x * (256 / kRowLanes) + threadIdx.x / kRowLanes;
    if (token >= p.m) return;
    const T* const row = static_cast<const T*>(p.logits) + static_cast<size_t>(token) * p.ldl;
    T* const out = static_cast<T*>(p.dlogits) + static_cast<size_t>(token) * p.ldd;
    const bool mine = static_cast<unsigned>(lane) < p.top;
    const size_t entry = static_cast<size_t>(token) * p.top + lane;
    int expert = mine ? p.chosen[entry] : -1;
    if (expert < 0 || static_cast<unsigned>(expert) >= p.experts) expert = -1;
    const float logit = expert >= 0 ? static_cast<float>(row[expert]) : kOut;
    const float dw = expert >= 0 ? p.dweights[entry] : 0.f;
    using L = Logits<T, CHUNKS>;
    L l;
    float share;                             // of this lane's choice
    float most, sum;
    if (p.normalize) {
        const float live = logit > kOut ? logit : kOut;
        most = row_max(live);
        share = weight_of(live, most);
        sum = row_sum(share);
    } else {
        l.load(row, p.experts, lane);
        most = row_max(l.most());
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < L::kAll; ++i) sum += l.v[i] = weight_of(l.v[i], most);
        sum = row_sum(sum);
        share = logit > kOut ? weight_of(logit, most) : 0.f;
    }
    const float over = sum != 0.f ? 1.f / sum : 0.f;
    share *= over;
    const float mean = row_sum(share != 0.f ? share * dw : 0.f);
    float grad[L::kAll];
#pragma unroll
    for (int i = 0; i < L::kAll; ++i) grad[i] = p.normalize ? 0.f : l.v[i] * over * -mean;
    const float own = p.normalize ? share * (dw - mean) : share * dw;
    const int first = (threadIdx.x & 63) - lane;
    for (unsigned s = 0; s < p.top; ++s) {
        const int of = __shfl(expert, first + s);
        const float g = __shfl(own, first + s);
#pragma unroll
        for (int i = 0; i < L::kAll; ++i) grad[i] += L::column(i, lane) == of ? g : 0.f;
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = L::column(c * L::kPer, lane);
        Pack<T> q;
#pragma unroll
        for (int j = 0; j < L::kPer; ++j) q.v[j] = static_cast<T>(grad[c * L::kPer + j]);
        if (at + L::kPer <= static_cast<int>(p.experts)) {
            __builtin_memcpy(out + at, &q, 16);
        } else {
#pragma unroll
            for (int j = 0; j < L::kPer; ++j)
                if (at + j < static_cast<int>(p.experts)) out[at + j] = q.v[j];
        }
    }
}

// ------------------------------------------------------------------ the experts' products
template <typename T>
struct ExpertArgs {
    const T *x, *w, *dy;
    T *y, *dx, *dw;
    size_t ldx, ldw, sw, ldy, lddx, lddw, sdw;
    const int64_t* offsets;
    unsigned m, experts, n, k;
};

__device__ __forceinline__ unsigned start_of(const int64_t* offsets, unsigned e, unsigned m) {
    int64_t most = 0;
    for (unsigned i = 0; i <= e; ++i) most = max(most, offsets[i]);
    return static_cast<unsigned>(min(most, static_cast<int64_t>(m)));
}

enum class Does { kForward, kDx, kDw };

// A thread for each element of an output, one expert after the other.
template <typename T, Does DOES>
__global__ __launch_bounds__(256) void plain_kernel(ExpertArgs<T> p) {
    const unsigned e = blockIdx.z, begin = start_of(p.offsets, e, p.m), end = start_of(p.offsets, e + 1, p.m);
    const unsigned cols = DOES == Does::kForward ? p.n : p.k, col = blockIdx.x * 64 + threadIdx.x % 64;
    const unsigned rows = DOES == Does::kDw ? p.n : end - begin;
    if (col >= cols) return;
    for (unsigned row = blockIdx.y * 4 + threadIdx.x / 64; row < rows; row += gridDim.y * 4) {
        float sum = 0.f;
        if constexpr (DOES == Does::kForward) {
            for (unsigned t = 0; t < p.k; ++t)
                sum += static_cast<float>(p.x[(begin + row) * p.ldx + t]) * static_cast<float>(p.w[e * p.sw + col * p.ldw + t]);
            p.y[(begin + row) * p.ldy + col] = static_cast<T>(sum);
        } else if constexpr (DOES == Does::kDx) {
            for (unsigned t = 0; t < p.n; ++t)
                sum += static_cast<float>(p.dy[(begin + row) * p.ldy + t]) * static_cast<float>(p.w[e * p.sw + t * p.ldw + col]);
            p.dx[(begin + row) * p.lddx + col] = static_cast<T>(sum);
        } else {
            for (unsigned t = begin; t < end; ++t)
                sum += static_cast<float>(p.dy[t * p.ldy + row]) * static_cast<float>(p.x[t * p.ldx + col]);
            p.dw[e * p.sdw + row * p.lddw + col] = static_cast<T>(sum);
        }
    }
}

// ------------------------------------------------------------------ host side
// f(chunks) for the 16-byte pieces that a lane has of a token's logits.
template <typename T, typename F>
zvc_status with_chunks(size_t experts, F f) {
    const size_t chunks = div_up(experts, kRowLanes * 16 / sizeof(T));
    if (chunks <= 1) return f(std::integral_constant<int, 1>{});
    if (chunks <= 2) return f(std::integral_constant<int, 2>{});
    if (chunks <= 4) return f(std::integral_constant<int, 4>{});
    if constexpr (sizeof(T) == 2) {
        return f(std::integral_constant<int, 8>{});
    } else {
        return chunks <= 8 ? f(std::integral_constant<int, 8>{}) : f(std::integral_constant<int, 16>{});
    }
}

bool route_sizes_ok(size_t m, size_t experts, size_t top) {
    return experts >= 1 && experts <= ZVC_EXPERTS_MAX && top >= 1 && top <= ZVC_EXPERTS_MAX_TOP && top <= experts &&
           m <= ZVC_EXPERTS_MAX_ENTRIES / top;
}

template <typename T>
zvc_status route_as(const RouteArgs& p, hipStream_t stream) {
    return with_chunks<T>(p.experts, [&](auto chunks) {
        constexpr int kChunks = decltype(chunks)::value;
        if (p.blocks <= 1) return launch(route_kernel<T, kChunks, true>, dim3(1), kRouteThreads, stream, p);
        if (zvc_status st = launch(route_kernel<T, kChunks, false>, dim3(p.blocks), kRouteThreads, stream, p)) return st;
        if (zvc_status st = launch(route_sums_kernel, dim3(p.experts), 64, stream, p)) return st;
        return launch(route_places_kernel, dim3(p.blocks), kRouteThreads, stream, p);
    });
}

template <typename T>
zvc_status route_backward_as(const RouteBackArgs& p, hipStream_t stream) {
    return with_chunks<T>(p.experts, [&](auto chunks) {
        return launch(route_backward_kernel<T, decltype(chunks)::value>, dim3(div_up(p.m, 256 / kRowLanes)), 256, stream, p);
    });
}

bool expert_sizes_ok(size_t m, size_t experts, size_t n, size_t k) {
    return experts >= 1 && experts <= ZVC_EXPERTS_MAX && m <= ZVC_FFN_MAX_ROWS && n <= ZVC_FFN_MAX_COLUMNS && k <= ZVC_FFN_MAX_COLUMNS &&
           m * n <= ZVC_FFN_MAX_ELEMENTS && m * k <= ZVC_FFN_MAX_ELEMENTS && experts * n * k <= ZVC_FFN_MAX_ELEMENTS;
}
bool stride_ok(size_t ld, size_t cols) { return ld >= cols && ld <= ZVC_FFN_MAX_COLUMNS; }
// A stack of n x k matrices.
bool stack_ok(size_t ld, size_t stride, size_t experts, size_t n, size_t k) {
    if (!stride_ok(ld, k)) return false;
    if (experts <= 1 || n == 0 || k == 0) return true;
    return stride >= (n - 1) * ld + k && stride <= ZVC_FFN_MAX_ELEMENTS / experts;
}
// As one region: what lies between the experts belongs to it.
Region stack_region(const void* at, size_t ld, size_t stride, size_t experts, size_t n, size_t k, size_t w) {
    if (n == 0 || k == 0) return {at, 0, 0, 0};
    const size_t bytes = ((experts - 1) * stride + (n - 1) * ld + k) * w;
    return {at, bytes, 1, bytes};
}

}  // namespace

// ------------------------------------------------------------------ C ABI
extern "C" {

size_t zvc_route_workspace_bytes(size_t m, size_t experts, size_t top) {
    if (!route_sizes_ok(m, experts, top)) return 0;
    const size_t blocks = div_up(m, kRouteTokens);
    return 256 + (blocks > 1 ? round_up(experts * (blocks + 1) * sizeof(unsigned), 256) : 0);
}

zvc_status zvc_route(const void* d_logits, size_t ldl, int32_t* d_chosen, float* d_weights, int64_t* d_offsets, int64_t* d_order,
                     int64_t* d_place, size_t m, size_t experts, size_t top, int type, int normalize, void* d_ws, size_t ws,
                     hipStream_t stream) {
    const size_t w = type_bytes(type);
    if (w == 0 || !route_sizes_ok(m, experts, top) || !stride_ok(ldl, experts)) return ZVC_E_ARG;
    if (d_offsets == nullptr || d_ws == nullptr) return ZVC_E_ARG;
    if (m != 0 && (d_logits == nullptr || d_chosen == nullptr || d_weights == nullptr || d_order == nullptr || d_place == nullptr)) return ZVC_E_ARG;
    if (!aligned_to(d_logits, w) || !aligned_to(d_chosen, 4) || !aligned_to(d_weights, 4) || !aligned_to(d_offsets, 8) || !aligned_to(d_order, 8) ||
        !aligned_to(d_place, 8) || !aligned_to(d_ws, 256))
        return ZVC_E_ALIGN;
    if (ws < zvc_route_workspace_bytes(m, experts, top)) return ZVC_E_WORKSPACE;
    const size_t entries = m * top, blocks = div_up(m, kRouteTokens);
    const auto flat = [](const void* at, size_t bytes) { return Region{at, bytes, 1, bytes}; };
    const Region all[] = {flat(d_chosen, entries * 4), flat(d_weights, entries * 4), flat(d_offsets, (experts + 1) * 8), flat(d_order, entries * 8),
                          flat(d_place, entries * 8), flat(d_ws, ws), {d_logits, ldl * w, m, experts * w}};
    for (int i = 0; i < 7; ++i)
        for (int j = 0; j < i; ++j)
            if (overlap(all[i], all[j])) return ZVC_E_ARG;
    const RouteArgs p = {d_logits, ldl, d_chosen, d_weights, d_offsets, d_order, d_place, static_cast<unsigned*>(d_ws), static_cast<unsigned>(m),
                         static_cast<unsigned>(experts), static_cast<unsigned>(top), static_cast<unsigned>(blocks), normalize != 0};
    switch (type) {
        case ZVC_FP32: return route_as<float>(p, stream);
        case ZVC_FP16: return route_as<fp16>(p, stream);
        default: return route_as<bf16>(p, stream);
    }
}

zvc_status zvc_route_backward(const float* d_dweights, const void* d_logits, size_t ldl, const int32_t* d_chosen, void* d_dlogits, size_t ldd,
                              size_t m, size_t experts, size_t top, int type, int normalize, hipStream_t stream) {
    const size_t w = type_bytes(type);
    if (w == 0 || !route_sizes_ok(m, experts, top) || !stride_ok(ldl, experts) || !stride_ok(ldd, experts)) return ZVC_E_ARG;
    if (m == 0) return ZVC_OK;
    if (d_dweights == nullptr || d_logits == nullptr || d_chosen == nullptr || d_dlogits == nullptr) return ZVC_E_ARG;
    if (!aligned_to(d_dweights, 4) || !aligned_to(d_logits, w) || !aligned_to(d_chosen, 4) || !aligned_to(d_dlogits, w)) return ZVC_E_ALIGN;
    const Region out{d_dlogits, ldd * w, m, experts * w}, in[] = {{d_dweights, m * top * 4, 1, m * top * 4}, {d_chosen, m * top * 4, 1, m * top * 4},
                                                                  {d_logits, ldl * w, m, experts * w}};
    for (const Region& r : in)
        if (overlap(out, r)) return ZVC_E_ARG;
    const RouteBackArgs p = {d_dweights, d_logits, ldl, ldd, d_chosen, d_dlogits, static_cast<unsigned>(m), static_cast<unsigned>(experts),
                             static_cast<unsigned>(top), normalize != 0};
    switch (type) {
        case ZVC_FP32: return route_backward_as<float>(p, stream);
        case ZVC_FP16: return route_backward_as<fp16>(p, stream);
        default: return route_backward_as<bf16>(p, stream);
    }
}

size_t zvc_expert_workspace_bytes(size_t m, size_t experts, size_t n, size_t k, int type, int backward) {
    return type_bytes(type) == 0 || !expert_sizes_ok(m, experts, n, k) ? 0 : 256;
}

zvc_status zvc_expert_product(const void* d_x, size_t ldx, const void* d_w, size_t ldw, size_t sw, const int64_t* d_offsets, void* d_y,
                              size_t ldy, size_t m, size_t experts, size_t n, size_t k, int type, void* d_ws, size_t ws, hipStream_t stream) {
    const size_t w = type_bytes(type);
    if (w == 0 || !expert_sizes_ok(m, experts, n, k)) return ZVC_E_ARG;
    if (!stride_ok(ldx, k) || !stack_ok(ldw, sw, experts, n, k) || !stride_ok(ldy, n)) return ZVC_E_ARG;
    if (m == 0 || n == 0) return ZVC_OK;
    if (d_offsets == nullptr || d_y == nullptr || (k != 0 && (d_x == nullptr || d_w == nullptr)) || d_ws == nullptr) return ZVC_E_ARG;
    const void* all[] = {d_x, d_w, d_y};
    for (const void* p : all)
        if (!aligned_to(p, w)) return ZVC_E_ALIGN;
    if (!aligned_to(d_offsets, 8) || !aligned_to(d_ws, 256)) return ZVC_E_ALIGN;
    if (ws < zvc_expert_workspace_bytes(m, experts, n, k, type, 0)) return ZVC_E_WORKSPACE;
    const size_t last = (experts + 1) * sizeof(int64_t);
    const Region in[] = {{d_x, ldx * w, m, k * w}, stack_region(d_w, ldw, sw, experts, n, k, w), {d_offsets, last, 1, last}};
    const Region out[] = {{d_y, ldy * w, m, n * w}, {d_ws, ws, 1, ws}};
    if (overlap(out[0], out[1])) return ZVC_E_ARG;
    for (const Region& r : in)
        if (overlap(out[0], r) || overlap(out[1], r)) return ZVC_E_ARG;
    const auto as = [&](auto zero) {
        using T = decltype(zero);
        ExpertArgs<T> p{};
        p.x = static_cast<const T*>(d_x), p.w = static_cast<const T*>(d_w), p.y = static_cast<T*>(d_y);
        p.ldx = ldx, p.ldw = ldw, p.sw = sw, p.ldy = ldy, p.offsets = d_offsets;
        p.m = static_cast<unsigned>(m), p.experts = static_cast<unsigned>(experts), p.n = static_cast<unsigned>(n), p.k = static_cast<unsigned>(k);
        return launch(plain_kernel<T, Does::kForward>, dim3(div_up(n, 64), m < 256 ? div_up(m, 4) : 64, experts), 256, stream, p);
    };
    return type == ZVC_FP32 ? as(0.f) : type == ZVC_FP16 ? as(fp16{}) : as(bf16{});
}

zvc_status zvc_expert_gradients(const void* d_dy, size_t lddy, const void* d_x, size_t ldx, const void* d_w, size_t ldw, size_t sw,
                                const int64_t* d_offsets, void* d_dx, size_t lddx, void* d_dw, size_t lddw, size_t sdw, size_t m,
                                size_t experts, size_t n, size_t k, int type, void* d_ws, size_t ws, hipStream_t stream) {
    const size_t w = type_bytes(type);
    if (w == 0 || !expert_sizes_ok(m, experts, n, k)) return ZVC_E_ARG;
    if (!stride_ok(lddy, n) || !stride_ok(ldx, k) || !stack_ok(ldw, sw, experts, n, k) || (d_dx != nullptr && !stride_ok(lddx, k)) ||
        (d_dw != nullptr && !stack_ok(lddw, sdw, experts, n, k)))
        return ZVC_E_ARG;
    const bool want_dx = d_dx != nullptr && m != 0 && k != 0, want_dw = d_dw != nullptr && n != 0 && k != 0;
    if (!want_dx && !want_dw) return ZVC_OK;
    const bool rows = m != 0 && n != 0;
    if (d_offsets == nullptr || d_ws == nullptr || (rows && d_dy == nullptr) || (rows && want_dw && d_x == nullptr) || (rows && want_dx && d_w == nullptr))
        return ZVC_E_ARG;
    const void* all[] = {d_dy, d_x, d_w, d_dx, d_dw};
    for (const void* p : all)
        if (!aligned_to(p, w)) return ZVC_E_ALIGN;
    if (!aligned_to(d_offsets, 8) || !aligned_to(d_ws, 256)) return ZVC_E_ALIGN;
    if (ws < zvc_expert_workspace_bytes(m, experts, n, k, type, 1)) return ZVC_E_WORKSPACE;
    const size_t last = (experts + 1) * sizeof(int64_t);
    const Region in[] = {{d_dy, lddy * w, m, n * w}, {d_x, ldx * w, m, k * w}, stack_region(d_w, ldw, sw, experts, n, k, w), {d_offsets, last, 1, last}};
    const Region out[] = {{d_dx, lddx * w, m, k * w}, stack_region(d_dw, lddw, sdw, experts, n, k, w), {d_ws, ws, 1, ws}};
    for (int i = 0; i < 3; ++i) {
        for (const Region& r : in)
            if (overlap(out[i], r)) return ZVC_E_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return ZVC_E_ARG;
    }
    const auto as = [&](auto zero) {
        using T = decltype(zero);
        ExpertArgs<T> p{};
        p.x = static_cast<const T*>(d_x), p.w = static_cast<const T*>(d_w), p.dy = static_cast<const T*>(d_dy);
        p.dx = static_cast<T*>(d_dx), p.dw = static_cast<T*>(d_dw);
        p.ldx = ldx, p.ldw = ldw, p.sw = sw, p.ldy = lddy, p.lddx = lddx, p.lddw = lddw, p.sdw = sdw, p.offsets = d_offsets;
        p.m = static_cast<unsigned>(m), p.experts = static_cast<unsigned>(experts), p.n = static_cast<unsigned>(n), p.k = static_cast<unsigned>(k);
        if (want_dx)
            if (zvc_status st = launch(plain_kernel<T, Does::kDx>, dim3(div_up(k, 64), m < 256 ? div_up(m, 4) : 64, experts), 256, stream, p)) return st;
        if (want_dw) return launch(plain_kernel<T, Does::kDw>, dim3(div_up(k, 64), n < 256 ? div_up(n, 4) : 64, experts), 256, stream, p);
        return ZVC_OK;
    };
    return type == ZVC_FP32 ? as(0.f) : type == ZVC_FP16 ? as(fp16{}) : as(bf16{});
}

}  // extern "C"
