// Router and matrix products for mixtures of experts, forward and backward, for AMD gfx950 (wave64): kernels and C ABI
// (include/zvc_experts.h has the formulas).
//
//   * route_kernel, route_sums_kernel, route_places_kernel: the choice; counts of each expert's entries by workgroup, their sums, and with these each
//     entry's row.  Up to 32 tokens are one workgroup's, which does all three.  route_backward_kernel: the logits' gradient.
//   * expert_product_kernel, expert_gradients_kernel: persistent workgroups over all experts' tiles, on the matrix cores, staged straight to LDS.
//     Every workgroup makes a table of the experts' rows and tiles from the offsets first, so that the host has to know neither.
//   * loose_kernel: the same tiles where operands do not take 16-byte accesses, staged by way of registers.
//   * solo_kernel, solo_join_kernel: few rows, few tiles or short sums; workgroups whose waves take turns along the sum.
//
// Times in the comments are us on one MI355X, where a large copy moves 5.0 TB/s and a large bf16 product of the vendor's library
// reaches 1180 to 1460 TFLOP/s (fp32 155): calls one behind the other over several sets of tensors, both sides of a comparison in turn.

#include "tiles.h"
#include "zvc_experts.h"

#include <cmath>

namespace {

// ------------------------------------------------------------------ the router
// A token's logits lie over 16 lanes, a row of the cross-lane instructions, so that a maximum over all experts is a few instructions for each
// of a lane's logits and four for the rest, without LDS.  16384 tokens of 256 experts, fp32, 8 choices: 19.4; the profiler, which adds some to
// each of three kernels, has 13.0 for the choice, 3.8 for the sums and 5.0 for the rows.  Reading the logits is 3.4 of them, and the rest of the choice is its 8 rounds of maximum, search and removal over a lane's 16 logits, one behind
// the other.  8 tokens of 64 experts: 4.1, a launch and one chain from the load to the rows.
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

// 16-bit gradients take the shorter exp, which loses |logit - most| x 2^-24 of the result.
template <typename T = float>
__device__ __forceinline__ float weight_of(float logit, float most) { return logit > kOut ? (sizeof(T) == 4 ? expf(logit - most) : __expf(logit - most)) : 0.f; }

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
        // (columns counted from the lane's first: constants)
        constexpr int kNone = 1 << 20;
        int first = kNone;
#pragma unroll
        for (int i = l.kAll - 1; i >= 0; --i) first = l.v[i] == best ? l.column(i, 0) : first;
        const int at = row_min(first + l.column(0, lane)), taken = at - l.column(0, lane);
        if (static_cast<unsigned>(lane) == s && best > kOut) *expert = at, logit = best;
#pragma unroll
        for (int i = 0; i < l.kAll; ++i) l.v[i] = l.column(i, 0) == taken ? kOut : l.v[i];
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

// A workgroup an expert: its counts by workgroup become sums of those before, and their total is written behind all counts.  Counts lie expert by expert,
// since these sums run along them (512 counts of each of 256 experts: 3.8, latency of one load and two barriers).
constexpr int kSumThreads = 256;
__global__ __launch_bounds__(kSumThreads) void route_sums_kernel(RouteArgs p) {
    constexpr unsigned kEach = 4;
    __shared__ unsigned room[kSumThreads / 64], total;
    unsigned* const counts = p.counts + static_cast<size_t>(blockIdx.x) * p.blocks;
    unsigned before = 0;
    for (unsigned at = 0; at < p.blocks; at += kSumThreads * kEach) {
        unsigned own[kEach], sum = 0;
#pragma unroll
        for (unsigned j = 0; j < kEach; ++j) {
            const unsigned b = at + threadIdx.x * kEach + j;
            own[j] = b < p.blocks ? counts[b] : 0;
        }
#pragma unroll
        for (unsigned j = 0; j < kEach; ++j) sum += own[j];
        const unsigned through = running_sum<kSumThreads>(sum, room);
        unsigned x = before + through - sum;
#pragma unroll
        for (unsigned j = 0; j < kEach; ++j) {
            const unsigned b = at + threadIdx.x * kEach + j;
            if (b < p.blocks) counts[b] = x;
            x += own[j];
        }
        if (threadIdx.x == kSumThreads - 1) total = x;
        __syncthreads();
        before = total;
        __syncthreads();
    }
    if (threadIdx.x == 0) p.counts[static_cast<size_t>(p.experts) * p.blocks + blockIdx.x] = before;
}

// Ranks become rows, by the workgroups that made them (16384 x 8 entries: 5.0; each workgroup sums the experts' totals again, which spares a launch).
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

// The gradient of a softmax over the chosen, or over all with only the chosen ones' gradients: dl_j = p_j ([j chosen] dw_j - sum p_i dw_i).  Bound by the
// launch and one pass over the row: 16384 x 256, bf16, 6.4 on the GPU, 8.2 MB in and out each.
// Lane s of a token's 16 has its choice s.  The row is written as if nothing had been chosen, and then the chosen experts' elements over it, once the
// row is there.  (Every lane looking all choices over for its columns instead: 16384 x 256 bf16, 8 choices, 8.9.)
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
    const float given = expert >= 0 ? static_cast<float>(row[expert]) : kOut;
    const float logit = given > kOut ? given : kOut;
    const float dw = expert >= 0 ? p.dweights[entry] : 0.f;
    using L = Logits<T, CHUNKS>;
    L l;
    float most, sum = 0.f;
    if (p.normalize) {
        most = row_max(logit);
    } else {
        l.load(row, p.experts, lane);
        most = row_max(l.most());
#pragma unroll
        for (int i = 0; i < L::kAll; ++i) sum += l.v[i] = weight_of<T>(l.v[i], most);
    }
    float share = weight_of<T>(logit, most);                         // of this lane's choice
    sum = row_sum(p.normalize ? share : sum);
    const float over = sum != 0.f ? 1.f / sum : 0.f;
    share *= over;
    const float mean = row_sum(share != 0.f ? share * dw : 0.f);
    const float own = p.normalize ? share * (dw - mean) : share * dw;
    float grad = p.normalize ? 0.f : -share * mean;                  // with what other choices of the same expert add
    const int first = (threadIdx.x & 63) - lane;
    for (unsigned s = 0; s < p.top; ++s) {
        const int of = __shfl(expert, first + s);
        const float g = __shfl(own, first + s);
        grad += of == expert ? g : 0.f;
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = L::column(c * L::kPer, lane);
        Pack<T> q = {};
        if (!p.normalize) {
#pragma unroll
            for (int j = 0; j < L::kPer; ++j) q.v[j] = static_cast<T>(l.v[c * L::kPer + j] * over * -mean);
        }
        if (at + L::kPer <= static_cast<int>(p.experts)) {
            __builtin_memcpy(out + at, &q, 16);
        } else {
#pragma unroll
            for (int j = 0; j < L::kPer; ++j)
                if (at + j < static_cast<int>(p.experts)) out[at + j] = q.v[j];
        }
    }
    wait_loads<0>();                                                 // (and stores)
    if (expert >= 0) out[expert] = static_cast<T>(logit > kOut ? grad : 0.f);
    // Who is out has weight 0, but 0 times an infinity or a NaN is none: those are written again.  (Looked for in every element instead: 65536 x 256, bf16, 20.3
    // instead of 19.7.)
    if (!p.normalize && !(fabsf(over * mean) < INFINITY))
        for (unsigned e = lane; e < p.experts; e += kRowLanes)
            if (!(static_cast<float>(row[e]) > kOut)) out[e] = static_cast<T>(0.f);
}

// ------------------------------------------------------------------ the experts' products
//
// Every product is  out[row][col] = sum over t of Q(row, t) P(col, t)  within one expert, in the terms of tiles.h:  forward  P = W, Q = x;
// dx  P = W by columns, Q = dy;  dW  P = x by columns, Q = dy by columns, the sum over the expert's rows.
enum class Does { kForward, kDx, kDw };

template <typename T>
struct ExpertArgs {
    const T *p, *q;
    T* out;
    size_t sp, so;                       // from an expert's P, or its output, to the next one's
    const int64_t* offsets;
    unsigned ldp, ldq, ldo, m, experts, cols, rows, length;   // rows: of dW; length: of the sum (dW: unused)
};

// Where each expert's rows begin and which tile is its first, in LDS.  (As many words as there can be experts, no more: with the
// smaller tiles' rings two workgroups fill a compute unit's LDS.)
struct Groups {
    unsigned *starts, *firsts;
    unsigned experts, end, items;

    __device__ __forceinline__ unsigned start(unsigned e) const { return e < experts ? starts[e] : end; }
    __device__ __forceinline__ unsigned rows(unsigned e) const { return start(e + 1) - start(e); }
    // The expert of a tile: the last one whose first tile is not behind it.
    __device__ __forceinline__ unsigned expert_of(unsigned item, int lane) const {
        unsigned low = 0, left = experts;
        while (left > 1) {
            const unsigned stride = (left + 63) / 64, at = lane * stride;
            const bool before = at < left && firsts[low + at] <= item;
            const unsigned last = static_cast<unsigned>(__popcll(__ballot(before))) - 1;
            low += last * stride;
            left = min(stride, left - last * stride);
        }
        return __builtin_amdgcn_readfirstlane(low);
    }
};

// f over a workgroup's threads in their order, inclusive; the last one's in `all`.  `room`: a word for each wave.
template <int THREADS, typename F>
__device__ __forceinline__ unsigned running(unsigned x, unsigned* room, unsigned* all, F f) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const unsigned before = __shfl_up(x, d);
        x = lane >= d ? f(x, before) : x;
    }
    if (lane == 63) room[wave] = x;
    __syncthreads();
    unsigned sum = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w == wave && w != 0) x = f(x, sum);
        sum = w == 0 ? room[0] : f(sum, room[w]);
    }
    *all = sum;
    __syncthreads();
    return x;
}

// Offsets that go down count as the one before, and none lies outside the rows: no table holds what would lead out of them.
template <int THREADS>
__device__ __forceinline__ Groups groups_of(const int64_t* offsets, unsigned experts, unsigned m, unsigned across, unsigned tile_rows, unsigned* table, unsigned* room) {
    constexpr unsigned kEach = ZVC_EXPERTS_MAX / THREADS;
    Groups g{table, table + ZVC_EXPERTS_MAX, experts, 0, 0};
    unsigned at[kEach + 1], most = 0;
#pragma unroll
    for (unsigned j = 0; j < kEach; ++j) {
        const unsigned e = threadIdx.x * kEach + j;
        const int64_t offset = e <= experts ? offsets[e] : 0;
        most = max(most, static_cast<unsigned>(min(max(offset, int64_t{0}), static_cast<int64_t>(m))));
        at[j] = most;
    }
    const int64_t last = experts == ZVC_EXPERTS_MAX ? offsets[experts] : 0;
    unsigned all;
    const unsigned through = running<THREADS>(most, room, &all, [](unsigned a, unsigned b) { return max(a, b); });
    const unsigned before = __shfl_up(through, 1);
    if ((threadIdx.x & 63) == 63) room[threadIdx.x >> 6] = through;
    __syncthreads();
    const unsigned carried = (threadIdx.x & 63) != 0 ? before : threadIdx.x != 0 ? room[(threadIdx.x >> 6) - 1] : 0;
    __syncthreads();
#pragma unroll
    for (unsigned j = 0; j < kEach; ++j) at[j] = max(at[j], carried);
    g.end = max(all, static_cast<unsigned>(min(max(last, int64_t{0}), static_cast<int64_t>(m))));
#pragma unroll
    for (unsigned j = 0; j < kEach; ++j)
        if (threadIdx.x * kEach + j < experts) g.starts[threadIdx.x * kEach + j] = at[j];
    __syncthreads();
    unsigned own[kEach], sum = 0;
#pragma unroll
    for (unsigned j = 0; j < kEach; ++j) {
        const unsigned e = threadIdx.x * kEach + j;
        own[j] = e < experts ? across * ((g.rows(e) + tile_rows - 1) / tile_rows) : 0;
        sum += own[j];
    }
    unsigned first = running<THREADS>(sum, room, &g.items, [](unsigned a, unsigned b) { return a + b; }) - sum;
#pragma unroll
    for (unsigned j = 0; j < kEach; ++j) {
        const unsigned e = threadIdx.x * kEach + j;
        if (e < experts) g.firsts[e] = first;
        first += own[j];
    }
    __syncthreads();
    return g;
}

__host__ __device__ inline unsigned parts_of(unsigned tiles) { return (tiles + 7) / 8; }

// dW's tiles: workgroups go to the eight XCDs in turn, and each XCD takes a part of every expert's, since experts differ in what a tile costs.
// Parts are rounded up; what they have too much is no tile.  Of the `width` workgroups of an XCD the first `idle` have nothing else to do at the beginning and take `ahead`
// tiles each before the others take their first.
struct Parts {
    unsigned xcd, width, mine, idle, ahead, each, tiles, count, turn;     // each: of an expert; count: of all experts
    __device__ __forceinline__ Parts(unsigned of_expert, unsigned experts, unsigned busy, unsigned ahead_)
        : xcd(blockIdx.x % 8), width(gridDim.x / 8), ahead(ahead_), each(parts_of(of_expert)), tiles(of_expert), count(each * experts) {
        const unsigned at = blockIdx.x / 8, first = busy % width;         // (busy: items that the XCD's workgroups have before)
        idle = width - first;
        mine = at >= first ? at - first : at + idle;
        turn = mine < idle ? 0 : ahead;
    }
    __device__ __forceinline__ unsigned operator()() {
        while (true) {
            const unsigned at = turn < ahead ? mine + turn * idle : ahead * idle + mine + (turn - ahead) * width;
            ++turn;
            if (at >= count) return kNone;
            if (xcd * each + at % each < tiles) return at * 8 + xcd;
        }
    }
};

// One workgroup's view of a tile.  OF: tiles of which this is a quarter, or S.
template <typename T, Does DOES, class S, class OF = S>
struct Tile {
    static constexpr Lies kP = DOES == Does::kForward ? Lies::kAlong : Lies::kAcross, kQ = DOES == Does::kDw ? Lies::kAcross : Lies::kAlong;
    static constexpr int W = sizeof(T), kSteps = kStageBytes / W;
    using InP = Operand<T, kP, S::PT, S::kWavesAll, false>;
    using InQ = Operand<T, kQ, S::QT, S::kWavesAll, false>;

    static constexpr bool kQuarter = !std::is_same_v<S, OF>;
    static_assert(!kQuarter || (OF::PT == 2 * S::PT && OF::QT == 2 * S::QT), "quarters");

    unsigned col0, row0, end;            // of the output; the first row that is not the tile's expert's
    unsigned length, stages;
    T* out;
    const T *p, *q;
    InP in_p;
    InQ in_q;

    // Tiles of an expert are walked in bands of some rows: what the workgroups of an XCD read at a time then fits its L2.
    __device__ __forceinline__ void locate(unsigned at, unsigned tp, unsigned tq) {
        constexpr unsigned kBand = DOES == Does::kForward ? 8 : 4;
        const unsigned band = at / (kBand * tp), in_band = at % (kBand * tp), height = tq - band * kBand < kBand ? tq - band * kBand : kBand;
        col0 = in_band / height * OF::PT;
        row0 = (band * kBand + in_band % height) * OF::QT;
    }
    // from: the tile that the first four quarters are of.
    __device__ __forceinline__ void init(const ExpertArgs<T>& a, const Groups& g, unsigned items, unsigned from, unsigned item, int wave, int lane) {
        const unsigned tp = (a.cols + OF::PT - 1) / OF::PT;
        unsigned e;
        if constexpr (DOES == Does::kDw) {
            const unsigned tq = (a.rows + S::QT - 1) / S::QT, each = parts_of(tp * tq);
            e = item / 8 / each;
            locate(item % 8 * each + (item / 8 - e * each), tp, tq);
            const unsigned begin = __builtin_amdgcn_readfirstlane(g.start(e));
            end = a.rows;
            length = __builtin_amdgcn_readfirstlane(g.start(e + 1)) - begin;
            p = cell(a.p, begin, a.ldp, col0);
            q = cell(a.q, begin, a.ldq, row0);
            out = a.out + e * a.so;
        } else {
            const unsigned place = place_of(item, items), at = kQuarter ? from + place / 4 : place;
            e = g.expert_of(at, lane);
            const unsigned begin = __builtin_amdgcn_readfirstlane(g.start(e));
            end = __builtin_amdgcn_readfirstlane(g.start(e + 1));
            locate(at - __builtin_amdgcn_readfirstlane(g.firsts[e]), tp, (end - begin + OF::QT - 1) / OF::QT);
            row0 += begin;
            length = a.length;
            if constexpr (kQuarter) {
                col0 += place % 2 * S::PT, row0 += place / 2 % 2 * S::QT;
                if (col0 >= a.cols || row0 >= end) length = 0, col0 = min(col0, a.cols), row0 = min(row0, end);       // (nothing)
            }
            p = a.p + e * a.sp;
            p = DOES == Does::kForward ? cell(p, col0, a.ldp, 0) : p + col0;
            q = cell(a.q, row0, a.ldq, 0);
            out = a.out;
        }
        stages = (length + kSteps - 1) / kSteps;
        in_p.init(wave, lane, a.ldp, a.cols - col0 < S::PT ? a.cols - col0 : S::PT);
        in_q.init(wave, lane, a.ldq, end - row0 < S::QT ? end - row0 : S::QT);
    }
    __device__ __forceinline__ void fetch(const ExpertArgs<T>& a, unsigned s, unsigned lds) const {
        const uint64_t step_p = DOES == Does::kForward ? kStageBytes : uint64_t{kSteps} * W * a.ldp;
        const uint64_t step_q = DOES == Does::kDw ? uint64_t{kSteps} * W * a.ldq : kStageBytes;
        const int left = static_cast<int>(length - s * kSteps);
        in_p.fetch(reinterpret_cast<uint64_t>(p) + s * step_p, 0, left, lds);
        in_q.fetch(reinterpret_cast<uint64_t>(q) + s * step_q, 0, left, lds + S::PT * kStageBytes);
    }
};

// Two numbers of 16 bits in a word: one instruction for bf16, as a vector (two and more of a structure's members).
template <typename T>
__device__ __forceinline__ int pack(float a, float b) {
    using Two = T __attribute__((ext_vector_type(2)));
    using Floats = float __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(int, __builtin_convertvector(Floats{a, b}, Two));
}

// A lane's sums of 16 rows of a strip, as they go out: `pieces` of 16 bytes at (row, column of the strip).
//
// The matrix instructions leave a lane four neighbouring columns of each of its blocks in row r, r the lane's number within 16.  fp32: these
// are 16 bytes.  16-bit types: neighbouring quarters of the wave exchange halves of a pair of blocks, after which a lane has eight
// neighbouring columns, of two pairs; then neighbouring lanes exchange pairs, after which the even one has a piece of 128 neighbouring bytes of row r for
// itself and r + 1, and the odd one of r - 1 and r.  So an instruction writes whole lines of 128 bytes.
template <typename T, class S>
struct Strip {
    static constexpr bool kNarrow = sizeof(T) == 2;
    static constexpr int kPieces = kNarrow ? S::PB / 2 : S::PB;
    static_assert(!kNarrow || S::PB == 4, "lines of 128 bytes");
    using Words2 = unsigned __attribute__((ext_vector_type(2)));
    int4v v[kPieces];

    static __device__ __forceinline__ int row(int piece, int lane) { return kNarrow ? (lane & 14) + piece : lane & 15; }
    static __device__ __forceinline__ int col(int piece, int lane) {
        const int quarter = lane >> 4;
        return kNarrow ? (lane & 1) * 32 + (quarter & 1) * 16 + (quarter >> 1) * 8 : piece * 16 + quarter * 4;
    }
    __device__ __forceinline__ void take(const float4v (&acc)[S::PB][S::QB], int j, int lane) {
        if constexpr (kNarrow) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4v a = acc[2 * i][j], b = acc[2 * i + 1][j];
                const Words2 low = __builtin_amdgcn_permlane16_swap(pack<T>(a[0], a[1]), pack<T>(b[0], b[1]), false, false);
                const Words2 high = __builtin_amdgcn_permlane16_swap(pack<T>(a[2], a[3]), pack<T>(b[2], b[3]), false, false);
                v[i] = int4v{static_cast<int>(low[0]), static_cast<int>(high[0]), static_cast<int>(low[1]), static_cast<int>(high[1])};
            }
            const bool odd = lane & 1;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int own = odd ? v[1][w] : v[0][w], given = odd ? v[0][w] : v[1][w];
                const int got = __builtin_amdgcn_update_dpp(0, given, 0xB1, 0xF, 0xF, false);        // the neighbour's
                v[0][w] = odd ? got : own;
                v[1][w] = odd ? own : got;
            }
        } else {
#pragma unroll
            for (int i = 0; i < S::PB; ++i) v[i] = __builtin_bit_cast(int4v, acc[i][j]);
        }
    }
};

// A wave's strip of a tile goes out, by straight code where it is whole: a branch for each store, and what is rare between them, cost 2 us a tile.
template <typename T, class S>
__device__ __forceinline__ void store_strip(T* out, unsigned ldo, unsigned rows, unsigned cols, unsigned row0, unsigned col0, int lane, const float4v (&acc)[S::PB][S::QB]) {
    using Out = Strip<T, S>;
    constexpr int kPer = 16 / sizeof(T);
    if (row0 + S::QB * 16 <= rows && col0 + S::PB * 16 <= cols) {
        T* at = cell(out, row0 + Out::row(0, lane), ldo, col0 + Out::col(0, lane));
        const size_t next = Out::kNarrow ? ldo : 16, step = size_t{16} * ldo;
#pragma unroll
        for (int j = 0; j < S::QB; ++j, at += step) {
            Out strip;
            strip.take(acc, j, lane);
#pragma unroll
            for (int i = 0; i < Out::kPieces; ++i) __builtin_memcpy(at + i * next, &strip.v[i], 16);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < S::QB; ++j) {
        Out strip;
        strip.take(acc, j, lane);
#pragma unroll
        for (int i = 0; i < Out::kPieces; ++i) {
            const unsigned row = row0 + j * 16 + Out::row(i, lane), col = col0 + Out::col(i, lane);
            if (row >= rows) continue;
            T* const at = cell(out, row, ldo, col);
            const Pack<T> f = __builtin_bit_cast(Pack<T>, strip.v[i]);
            if (col + kPer <= cols) {
                __builtin_memcpy(at, &f, 16);
            } else {
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (col + e < cols) at[e] = f.v[e];
            }
        }
    }
}

// Four neighbouring sums, `left` of which are columns; `any`: one at least.
template <typename T>
__device__ __forceinline__ void store_four(T* at, float4v sum, unsigned left, bool any) {
    struct Four { T v[4]; };
    Four f;
#pragma unroll
    for (int e = 0; e < 4; ++e) f.v[e] = static_cast<T>(sum[e]);
    if (!any) return;
    if (left >= 4) {
        __builtin_memcpy(at, &f, sizeof f);
    } else {
#pragma unroll
        for (unsigned e = 0; e < 4; ++e)
            if (e < left) at[e] = f.v[e];
    }
}

// The sums of a stage that lies in LDS.
template <typename T, Does DOES, class S>
struct Multiplier {
    using Where = Tile<T, DOES, S>;
    using ReadP = Reader<T, Where::kP, S::PT, S::PB, false>;
    using ReadQ = Reader<T, Where::kQ, S::QT, S::QB, false>;
    using Frag = typename Fragment<T>::type;
    ReadP out_p;
    ReadQ out_q;
    Frag a[2][S::PB], b[2][S::QB];
    float4v acc[S::PB][S::QB];

    __device__ __forceinline__ void init(unsigned base, int wp, int wq, int lane) {
        out_p.init(base, wp, lane);
        out_q.init(base + S::PT * kStageBytes, wq, lane);
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < S::PB; ++i)
#pragma unroll
            for (int j = 0; j < S::QB; ++j) acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};
    }
    template <int HALF>
    __device__ __forceinline__ void read(unsigned stage) {
#pragma unroll
        for (int i = 0; i < S::PB; ++i) a[HALF][i] = out_p.read(i, HALF, stage);
#pragma unroll
        for (int j = 0; j < S::QB; ++j) b[HALF][j] = out_q.read(j, HALF, stage);
    }
    template <int HALF>
    __device__ __forceinline__ void product() {
#pragma unroll
        for (int j = 0; j < S::QB; ++j)
#pragma unroll
            for (int i = 0; i < S::PB; ++i) acc[i][j] = multiply(a[HALF][i], b[HALF][j], acc[i][j]);
        interleave<ReadP::kReads + ReadQ::kReads, S::PB * S::QB * (sizeof(T) == 4 ? 4 : 1)>();
    }
};

using Large = Shape<4, 2, 4, 8, 2>;             // 256 x 256, eight waves
using Quarter = Shape<2, 4, 4, 2, 4>;           // 128 x 128, eight waves, four stages in the same room

// Workgroups take tiles until there are none left; the next tile's first stages are on their way while a tile is finished.
//
// A stage of 128 bytes along the sum goes straight to LDS.  In large tiles, 256 x 256 by eight waves, a wave reads 24 KB of it for 64 products of
// 16 x 16 x 32, and a stage takes 1.47, which is 1460 TFLOP/s (4096 x 4096, one tile a compute unit: a sum over 4096 107, over 2048 60).  The matrix cores are busy for 64 % of such a
// loop (a sum over 65536: 1797), and its waves wait for 40 % of their cycles: with two places each stage ends in a wait for all loads and a barrier.  What a tile
// costs beside its stages, 10 of the 57 that a sum over 2048 takes, is the latency of its first stage and 128 KB that go out through L2 (dW of 16384 x 5632 x 2048 of 32 experts: 443,
// without its stores 334).  Tried and slower for that dW: stores past the caches (745 where it took 576 without), stores before the next tile's first loads (484), tiles of
// 256 x 128 by four waves, two workgroups a compute unit (484).  Tiles cut to the rows that an expert has left gain nothing:
// fewer products leave a stage's loads and its wait as they are.
template <typename T, Does DOES, class S, class OF = S, typename Next>
__device__ __forceinline__ void work(const ExpertArgs<T>& p, const Groups& groups, unsigned items, unsigned base, int lane, Next next, unsigned from = 0) {
    using Where = Tile<T, DOES, S, OF>;
    constexpr int kRing = S::kRing;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wp = wave % S::WP, wq = wave / S::WP;
    Multiplier<T, DOES, S> x;
    x.init(base, wp, wq, lane);
    Where tile;
    const auto begin = [&](unsigned item) {
        tile.init(p, groups, items, from, item, wave, lane);
#pragma unroll
        for (unsigned i = 0; i < kRing; ++i)
            if (i < tile.stages) tile.fetch(p, i, base + i * S::kStage);
    };
    // Waits until the loads of `stages` stages at most are on their way, if as many as the ring holds were asked for.
    constexpr int kLoads = Where::InP::kLoads + Where::InQ::kLoads;
    const auto wait_stages = [&](auto stages, bool full) {
        constexpr int kLeft = decltype(stages)::value * kLoads;
        if (kLeft != 0 && full) wait_loads<kLeft>();
        else wait_loads<0>();
    };
    const auto place = [&](unsigned s) { return (s & (kRing - 1)) * S::kStage; };
    static_assert((kRing & (kRing - 1)) == 0, "stages take places in turn");
    unsigned item = next();
    if (item == kNone) return;
    begin(item);
    while (item != kNone) {
        x.clear();
        // A stage is multiplied in two halves.  While a half's products run, the next half is read from LDS; between
        // the halves everyone has read the stage, and its place takes the one after the ring's last.
        if (tile.stages != 0) {                  // (dW of an expert without rows: 0)
            wait_stages(std::integral_constant<int, kRing - 1>{}, kRing <= tile.stages);
            group_barrier();
            x.template read<0>(0);
            for (unsigned s = 0; s < tile.stages; ++s) {
                x.template read<1>(place(s));
                x.template product<0>();
                wait_stages(std::integral_constant<int, kRing - 2>{}, s + kRing <= tile.stages);
                group_barrier();                 // stage s + 1 is there, and everyone has read stage s
                if (s + kRing < tile.stages) tile.fetch(p, s + kRing, base + place(s));
                x.template read<0>(place(s + 1));    // (behind the last stage: what the place held, for nothing)
                x.template product<1>();
            }
        }
        const unsigned row0 = tile.row0, col0 = tile.col0, end = tile.end;
        T* const out = tile.out;
        item = next();
        group_barrier();                         // (the reads for nothing are done)
        if (item != kNone) begin(item);
        store_strip<T, S>(out, p.ldo, end, p.cols, row0 + wq * S::QB * 16, col0 + wp * S::PB * 16, lane, x.acc);
    }
}

// A ring's places, and the experts' tables behind them.
template <class S>
__device__ __forceinline__ unsigned char* room_of() {
    __shared__ alignas(1024) unsigned char lds[S::kRing * S::kStage + 2 * ZVC_EXPERTS_MAX * sizeof(unsigned)];
    static_assert(S::kPerUnit * sizeof lds <= 160 << 10, "a compute unit's LDS");
    return lds;
}
template <class S>
__device__ __forceinline__ Groups tables(const int64_t* offsets, unsigned experts, unsigned m, unsigned cols, unsigned char* lds) {
    return groups_of<S::kThreads>(offsets, experts, m, (cols + S::PT - 1) / S::PT, S::QT, reinterpret_cast<unsigned*>(lds + S::kRing * S::kStage),
                                  reinterpret_cast<unsigned*>(lds));
}
__device__ __forceinline__ unsigned address(unsigned char* lds) { return static_cast<unsigned>(reinterpret_cast<uintptr_t>((LdsByte*)lds)); }

// y.  8192 x 5632 x 2048 of 16 experts, bf16: 217, 870 TFLOP/s.  The rows would fill 2.75 rounds of tiles; the experts' ragged ends make them 3.4.  The matrix
// cores are busy for half of the dispatch.
// Large tiles that do not fill a round go in quarters, with a deeper ring, where those are two rounds or less: one of large tiles takes 57 with a sum over 2048,
// one of quarters some 20 (16 x 512 rows, 5632 x 2048, 3.4 rounds: 229.6 without, 217).
template <typename T, class S>
__global__ __launch_bounds__(S::kThreads, S::kPerUnit) void expert_product_kernel(ExpertArgs<T> p) {
    unsigned char* const lds = room_of<S>();
    const Groups g = tables<S>(p.offsets, p.experts, p.m, p.cols, lds);
    const int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0));
    if constexpr (std::is_same_v<S, Large>) {
        const unsigned over = g.items % gridDim.x, rest = 2 * over <= gridDim.x ? over : 0, whole = g.items - rest;
        work<T, Does::kForward, S>(p, g, whole, address(lds), lane, Turns{blockIdx.x, whole});
        work<T, Does::kForward, Quarter, Large>(p, g, 4 * rest, address(lds), lane, Turns{blockIdx.x, 4 * rest}, whole);
    } else {
        work<T, Does::kForward, S>(p, g, g.items, address(lds), lane, Turns{blockIdx.x, g.items});
    }
}

// dx, and behind it dW, in one go: either alone leaves compute units idle in its last round (16384 x 5632 x 2048 of 32 experts, bf16: 810, 930 TFLOP/s;
// 849 where idle workgroups do not go ahead with dW).  dw_tiles: of one expert; it, and dx.cols, may be 0.
template <typename T, class S>
__global__ __launch_bounds__(S::kThreads, S::kPerUnit) void expert_gradients_kernel(ExpertArgs<T> dx, ExpertArgs<T> dw, unsigned dw_tiles) {
    unsigned char* const lds = room_of<S>();
    const Groups g = tables<S>(dx.offsets, dx.experts, dx.m, dx.cols, lds);
    // (a lane's number that is had again at any time: no register holds the thread's through both)
    const int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0));
    work<T, Does::kDx, S>(dx, g, g.items, address(lds), lane, Turns{blockIdx.x, g.items});
    // (a tile's time: its stages, and as much as seven to begin and finish)
    constexpr unsigned kSteps = Tile<T, Does::kDw, S>::kSteps;
    const unsigned stages_dx = (dx.length + kSteps - 1) / kSteps + 7, stages_dw = (g.end / dx.experts + kSteps - 1) / kSteps + 7;
    const unsigned xcd = blockIdx.x % 8, busy = g.items / 8 + (xcd < g.items % 8 ? 1 : 0), width = gridDim.x / 8;
    const unsigned ahead = busy % width != 0 ? (stages_dx + stages_dw / 2) / stages_dw : 0;
    work<T, Does::kDw, S>(dw, g, dw_tiles, address(lds), lane, Parts(dw_tiles, dw.experts, busy, ahead));
}

// ------------------------------------------------------------------ operands that do not take 16-byte accesses
// x moved towards its low end by `bytes`, 0 to 16, zeros behind it.
__device__ __forceinline__ int4v moved_down(int4v x, int bytes) {
    const auto whole = __builtin_bit_cast(unsigned __int128, x);
    return __builtin_bit_cast(int4v, bytes < 16 ? whole >> (8 * bytes) : static_cast<unsigned __int128>(0));
}

// The same places in LDS by way of registers: 16 bytes at any element, zeros beyond an operand's ends.  Where a row ends within the 16 bytes, the row's
// last 16 are read and moved into place; rows of fewer are read element by element.
template <typename T, Lies LIES, int SIDE, int WAVES>
struct LooseOperand {
    using Op = Operand<T, LIES, SIDE, WAVES, false>;
    static constexpr int kPer = 16 / sizeof(T);
    Op op;
    int4v v[Op::kLoads];

    // Elements of unit i that exist: `left` of the reduction, `side` rows (kAlong) or columns (kAcross).
    __device__ __forceinline__ int there(int i, int side, int left, int* row) const {
        *row = (op.first + i) * Op::kRowsPerLoad + op.lane_row;
        const int col = op.logical(*row) / static_cast<int>(sizeof(T));
        return *row < (LIES == Lies::kAlong ? side : left) ? (LIES == Lies::kAlong ? left : side) - col : 0;
    }
    // `shorter`: rows have less than 16 bytes in all.
    __device__ __forceinline__ void load(const T* base, size_t ld, int side, int left, bool shorter) {
#pragma unroll
        for (int i = 0; i < Op::kLoads; ++i) {
            int row;
            const int have = there(i, side, left, &row);
            v[i] = int4v{0, 0, 0, 0};
            if (have <= 0) continue;
            const T* const at = base + row * ld + op.logical(row) / static_cast<int>(sizeof(T));
            if (!shorter) {
                __builtin_memcpy(&v[i], at - (have < kPer ? kPer - have : 0), 16);
            } else {
                Pack<T> one = {};
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    if (j < have) one.v[j] = at[j];
                v[i] = __builtin_bit_cast(int4v, one);
            }
        }
    }
    // With load's arguments: what was read too far in front goes into place.  (Not in load, where each load would be waited for.)
    __device__ __forceinline__ void settle(int side, int left, bool shorter) {
        if (shorter || (LIES == Lies::kAlong ? left >= Op::kSteps : side >= SIDE)) return;
#pragma unroll
        for (int i = 0; i < Op::kLoads; ++i) {
            int row;
            const int have = there(i, side, left, &row);
            if (have > 0 && have < kPer) v[i] = moved_down(v[i], (kPer - have) * static_cast<int>(sizeof(T)));
        }
    }
    __device__ __forceinline__ void store(unsigned lds, int lane) const {
#pragma unroll
        for (int i = 0; i < Op::kLoads; ++i)
            *reinterpret_cast<__attribute__((address_space(3))) int4v*>(lds_at(lds + (op.first + i) * 1024 + lane * 16)) = v[i];
    }
};

// The next stage is in registers while one is multiplied.  16-byte loads at any element take the loads' unit longer, and every 16 bytes pass the registers: dW of
// 1956 rows, 32 experts, 2672 x 704, bf16, takes 56 here and 44 straight to LDS, which an operand that is not aligned has no other way to.
template <typename T, Does DOES, class S>
__global__ __launch_bounds__(S::kThreads, S::kPerUnit) void loose_kernel(ExpertArgs<T> p, unsigned dw_tiles) {
    static_assert(S::kRing == 2, "one stage is read while the next is written");
    unsigned char* const lds = room_of<S>();
    const Groups g = tables<S>(p.offsets, p.experts, p.m, p.cols, lds);
    using Where = Tile<T, DOES, S>;
    constexpr int kSteps = Where::kSteps;
    const unsigned base = address(lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wp = wave % S::WP, wq = wave / S::WP;
    Multiplier<T, DOES, S> x;
    x.init(base, wp, wq, lane);
    Where tile;
    LooseOperand<T, Where::kP, S::PT, S::kWavesAll> in_p;
    LooseOperand<T, Where::kQ, S::QT, S::kWavesAll> in_q;
    in_p.op.init(wave, lane, 0, 0);
    in_q.op.init(wave, lane, 0, 0);
    Turns turns{blockIdx.x, g.items};
    Parts parts(dw_tiles, p.experts, 0, 0);
    const auto next = [&]() { return DOES == Does::kDw ? parts() : turns(); };
    for (unsigned item = next(); item != kNone; item = next()) {
        tile.init(p, g, g.items, 0, item, wave, lane);
        const int side_p = min(static_cast<int>(p.cols - tile.col0), S::PT), side_q = min(static_cast<int>(tile.end - tile.row0), S::QT);
        const bool short_p = (DOES == Does::kForward ? p.length : p.cols) * sizeof(T) < 16;
        const bool short_q = (DOES == Does::kDw ? p.rows : p.length) * sizeof(T) < 16;
        const auto load = [&](unsigned s) {
            const size_t step_p = size_t{s} * kSteps * (DOES == Does::kForward ? 1 : p.ldp), step_q = size_t{s} * kSteps * (DOES == Does::kDw ? p.ldq : 1);
            const int left = static_cast<int>(tile.length - s * kSteps);
            in_p.load(tile.p + step_p, p.ldp, side_p, left, short_p);
            in_q.load(tile.q + step_q, p.ldq, side_q, left, short_q);
        };
        const auto store = [&](unsigned s) {
            const int left = static_cast<int>(tile.length - s * kSteps);
            in_p.settle(side_p, left, short_p);
            in_q.settle(side_q, left, short_q);
            in_p.store(base + (s & 1) * S::kStage, lane);
            in_q.store(base + (s & 1) * S::kStage + S::PT * kStageBytes, lane);
        };
        x.clear();
        if (tile.stages != 0) {
            load(0);
            store(0);
            __syncthreads();
        }
        for (unsigned s = 0; s < tile.stages; ++s) {
            if (s + 1 < tile.stages) load(s + 1);
            x.template read<0>((s & 1) * S::kStage);
            x.template read<1>((s & 1) * S::kStage);
            x.template product<0>();
            x.template product<1>();
            if (s + 1 < tile.stages) store(s + 1);
            __syncthreads();
        }
        store_strip<T, S>(tile.out, p.ldo, tile.end, p.cols, tile.row0 + wq * S::QB * 16, tile.col0 + wp * S::PB * 16, lane, x.acc);
    }
}

// ------------------------------------------------------------------ small products
// What a small kernel's workgroup works on.
struct Place {
    unsigned expert, begin, end, at;         // its rows; the tile's number among the expert's
};

// The expert and its tile that number `item` is, `across` tiles for every `tile_rows` rows of an expert; false behind the last.  Each wave looks for itself:
// a lane has some neighbouring experts.
__device__ __forceinline__ bool find_tile(const int64_t* offsets, unsigned experts, unsigned m, unsigned across, unsigned tile_rows, unsigned item, int lane, Place* out) {
    const unsigned each = (experts + 63) / 64, first = lane * each;
    const auto offset = [&](unsigned e) { return static_cast<unsigned>(min(max(offsets[min(e, experts)], int64_t{0}), static_cast<int64_t>(m))); };
    unsigned most = 0;
    for (unsigned j = 0; j < each; ++j) most = max(most, offset(first + j));
    unsigned through = most;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const unsigned before = __shfl_up(through, d);
        through = lane >= d ? max(through, before) : through;
    }
    const unsigned carried = __shfl_up(through, 1);
    const unsigned entry = lane != 0 ? carried : 0;
    const auto tiles = [&](unsigned begin, unsigned end) { return (end - begin + tile_rows - 1) / tile_rows * across; };
    unsigned sum = 0, begin = max(entry, offset(first));
    for (unsigned j = 0; j < each && first + j < experts; ++j) {
        const unsigned end = max(begin, offset(first + j + 1));
        sum += tiles(begin, end);
        begin = end;
    }
    unsigned total = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const unsigned before = __shfl_up(total, d);
        total += lane >= d ? before : 0;
    }
    const uint64_t behind = __ballot(total > item);
    if (behind == 0) return false;
    const int owner = __ffsll(static_cast<unsigned long long>(behind)) - 1;
    Place p{0, 0, 0, item - (total - sum)};
    if (lane == owner) {
        begin = max(entry, offset(first));
        for (unsigned j = 0; j < each && first + j < experts; ++j) {
            const unsigned end = max(begin, offset(first + j + 1)), own = tiles(begin, end);
            if (p.at < own) {
                p.expert = first + j, p.begin = begin, p.end = end;
                break;
            }
            p.at -= own;
            begin = end;
        }
    }
    *out = {static_cast<unsigned>(__builtin_amdgcn_readlane(p.expert, owner)), static_cast<unsigned>(__builtin_amdgcn_readlane(p.begin, owner)),
            static_cast<unsigned>(__builtin_amdgcn_readlane(p.end, owner)), static_cast<unsigned>(__builtin_amdgcn_readlane(p.at, owner))};
    return true;
}

// An expert's rows.
__device__ __forceinline__ void find_rows(const int64_t* offsets, unsigned expert, unsigned m, int lane, unsigned* begin, unsigned* end) {
    int64_t most = 0;
    for (unsigned e = lane; e <= expert; e += 64) most = max(most, offsets[e]);
    unsigned start = static_cast<unsigned>(min(most, static_cast<int64_t>(m)));
#pragma unroll
    for (int d = 1; d < 64; d *= 2) start = max(start, static_cast<unsigned>(__shfl_xor(start, d)));
    const int64_t next = offsets[expert + 1];
    *begin = __builtin_amdgcn_readfirstlane(start);
    *end = __builtin_amdgcn_readfirstlane(max(start, static_cast<unsigned>(min(max(next, int64_t{0}), static_cast<int64_t>(m)))));
}

constexpr int kSoloWaves = 4, kSoloCols = 64;

struct SoloSplit {
    float* sums;                         // part by part, tile by tile
    unsigned tiles, parts, dw_tiles;     // at most, of all experts; of a tile's sum; dW: of one expert
};

// Tiles of 64 columns and 16 QB rows.  The workgroup's waves take turns along the reduction, each with a place of its own in LDS for a stage, and meet there at
// the end; no wave waits for another.  What hides a wave's wait for its next stage are the other waves: four workgroups of 16 rows fit a compute unit, two of
// 64.  One token's 8 rows through 8 of 64 experts, 2816 x 1024, bf16: 9.9, reading the weights at 4.7 TB/s.  (With two places a wave, and half as
// many waves, 16 x 512 rows, 1024 x 1024, bf16 took 58.8 instead of 40.0; 8 x 128, 2048 x 2048 29.3 and 24.6.)
// LOOSE: operands come by way of registers, a stage ahead (two ahead: the dx of 777 x 1000 x 682 of 7 experts, fp32, 40.1 instead of 28.2, other products 0 to
// 17 % slower: not their latency bounds them, but what unaligned loads cost).  An expert's tiles of dW lie side by side in the grid: taken from all experts in
// turn, both gradients of that size took 73.8 instead of 65.7; a run of them for each XCD gains nothing.
template <typename T, Does DOES, int QB, bool LOOSE>
__global__ __launch_bounds__(64 * kSoloWaves, QB == 1 ? (LOOSE ? 3 : 4) : 2) void solo_kernel(ExpertArgs<T> p, SoloSplit split) {
    using S = Shape<1, 1, 4, QB, 2>;
    constexpr Lies kP = DOES == Does::kForward ? Lies::kAlong : Lies::kAcross, kQ = DOES == Does::kDw ? Lies::kAcross : Lies::kAlong;
    constexpr int W = sizeof(T), kSteps = kStageBytes / W, kRow = kSoloCols + 4;
    constexpr int kSums = kSoloWaves * S::QT * kRow * 4, kStages = kSoloWaves * S::kStage;
    __shared__ alignas(1024) unsigned char lds[kSums > kStages ? kSums : kStages];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // (dW: an expert's tiles are spread over the XCDs, since experts differ in what a tile costs)
    const unsigned tp = (p.cols + kSoloCols - 1) / kSoloCols, id = DOES == Does::kDw ? blockIdx.x : place_of(blockIdx.x, gridDim.x);
    const unsigned item = id / split.parts, part = id - item * split.parts;
    Place place;
    unsigned length, rows_end, row0, col0;
    const T *from_p, *from_q;
    T* out = p.out;
    if constexpr (DOES == Does::kDw) {
        place.expert = item / split.dw_tiles, place.at = item - place.expert * split.dw_tiles;
        find_rows(p.offsets, place.expert, p.m, lane, &place.begin, &place.end);
        const unsigned tq = (p.rows + S::QT - 1) / S::QT;
        col0 = place.at / tq * kSoloCols, row0 = place.at % tq * S::QT;
        length = place.end - place.begin, rows_end = p.rows;
        out += place.expert * p.so;
    } else {
        if (!find_tile(p.offsets, p.experts, p.m, tp, S::QT, item, lane, &place)) return;
        const unsigned tq = (place.end - place.begin + S::QT - 1) / S::QT;
        col0 = place.at / tq * kSoloCols, row0 = place.begin + place.at % tq * S::QT;
        length = p.length, rows_end = place.end;
    }
    if constexpr (DOES == Does::kDw) {
        from_p = cell(p.p, place.begin, p.ldp, col0), from_q = cell(p.q, place.begin, p.ldq, row0);
    } else {
        from_p = p.p + place.expert * p.sp;
        from_p = DOES == Does::kForward ? cell(from_p, col0, p.ldp, 0) : from_p + col0;
        from_q = cell(p.q, row0, p.ldq, 0);
    }
    const unsigned stages = (length + kSteps - 1) / kSteps, begin = static_cast<unsigned>(uint64_t{stages} * part / split.parts),
                   end = static_cast<unsigned>(uint64_t{stages} * (part + 1) / split.parts);
    const unsigned first = begin + wave, mine = first < end ? (end - first + kSoloWaves - 1) / kSoloWaves : 0;
    const size_t step_p = size_t{kSteps} * (DOES == Does::kForward ? 1 : p.ldp), step_q = size_t{kSteps} * (DOES == Does::kDw ? p.ldq : 1);
    const unsigned base = address(lds) + wave * S::kStage;
    const int side_p = min(static_cast<int>(p.cols - col0), kSoloCols), side_q = min(static_cast<int>(rows_end - row0), S::QT);
    Multiplier<T, DOES, S> x;
    x.init(base, 0, 0, lane);
    x.clear();
    if constexpr (LOOSE) {
        LooseOperand<T, kP, S::PT, 1> in_p;
        LooseOperand<T, kQ, S::QT, 1> in_q;
        in_p.op.init(0, lane, 0, 0);
        in_q.op.init(0, lane, 0, 0);
        const bool short_p = (DOES == Does::kForward ? p.length : p.cols) * W < 16, short_q = (DOES == Does::kDw ? p.rows : p.length) * W < 16;
        const auto load = [&](unsigned i) {
            const unsigned s = first + i * kSoloWaves;
            const int left = static_cast<int>(length - s * kSteps);
            in_p.load(from_p + s * step_p, p.ldp, side_p, left, short_p);
            in_q.load(from_q + s * step_q, p.ldq, side_q, left, short_q);
        };
        if (mine != 0) load(0);
        for (unsigned i = 0; i < mine; ++i) {
            const int left = static_cast<int>(length - (first + i * kSoloWaves) * kSteps);
            in_p.settle(side_p, left, short_p);
            in_q.settle(side_q, left, short_q);
            in_p.store(base, lane);
            in_q.store(base + S::PT * kStageBytes, lane);
            if (i + 1 < mine) load(i + 1);
            wait_reads();                                            // (what was stored is there)
            x.template read<0>(0);
            x.template read<1>(0);
            x.template product<0>();
            x.template product<1>();
        }
    } else {
        Operand<T, kP, S::PT, 1, false> in_p;
        Operand<T, kQ, S::QT, 1, false> in_q;
        in_p.init(0, lane, p.ldp, side_p);
        in_q.init(0, lane, p.ldq, side_q);
        const auto fetch = [&](unsigned i) {
            const unsigned s = first + i * kSoloWaves;
            const int left = static_cast<int>(length - s * kSteps);
            in_p.fetch(reinterpret_cast<uint64_t>(from_p + s * step_p), 0, left, base);
            in_q.fetch(reinterpret_cast<uint64_t>(from_q + s * step_q), 0, left, base + S::PT * kStageBytes);
        };
        if (mine != 0) fetch(0);
        for (unsigned i = 0; i < mine; ++i) {
            wait_loads<0>();
            x.template read<0>(0);
            x.template read<1>(0);
            wait_reads();                                            // before the place is written again
            if (i + 1 < mine) fetch(i + 1);
            x.template product<0>();
            x.template product<1>();
        }
    }
    __syncthreads();
    float* const sums = reinterpret_cast<float*>(lds);
    const int r = lane & 15, quarter = lane >> 4;
#pragma unroll
    for (int j = 0; j < QB; ++j)
#pragma unroll
        for (int i = 0; i < S::PB; ++i)
            *reinterpret_cast<float4v*>(sums + (wave * S::QT + j * 16 + r) * kRow + i * 16 + quarter * 4) = x.acc[i][j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < QB; ++j) {                               // 16 rows of 64 columns: four neighbouring ones a thread
        const unsigned row_in = j * 16 + threadIdx.x / 16, col_in = threadIdx.x % 16 * 4, row = row0 + row_in, col = col0 + col_in;
        float4v sum = *reinterpret_cast<const float4v*>(sums + row_in * kRow + col_in);
#pragma unroll
        for (int w = 1; w < kSoloWaves; ++w) sum += *reinterpret_cast<const float4v*>(sums + (w * S::QT + row_in) * kRow + col_in);
        if (split.parts > 1) {
            *reinterpret_cast<float4v*>(split.sums + ((size_t{part} * split.tiles + item) * S::QT + row_in) * kSoloCols + col_in) = sum;
        } else if (row < rows_end) {
            store_four(cell(out, row, p.ldo, col), sum, p.cols - col, col < p.cols);
        }
    }
}

// The parts' sums of tiles of 64 columns and 16 QB rows, joined in the order of the parts: a workgroup takes 16 rows of a tile.  A launch and a read of the sums, 3 to 5.
template <typename T, Does DOES, int QB>
__global__ __launch_bounds__(256) void solo_join_kernel(ExpertArgs<T> p, SoloSplit split) {
    constexpr unsigned kRows = 16 * QB;
    const int lane = threadIdx.x & 63;
    const unsigned item = blockIdx.x / QB, row_in = blockIdx.x % QB * 16 + threadIdx.x / 16, col_in = threadIdx.x % 16 * 4;
    Place place;
    unsigned row, col, rows_end;
    T* out = p.out;
    if constexpr (DOES == Does::kDw) {
        const unsigned tq = (p.rows + kRows - 1) / kRows, expert = item / split.dw_tiles, at = item - expert * split.dw_tiles;
        out += expert * p.so;
        row = at % tq * kRows + row_in, col = at / tq * kSoloCols + col_in, rows_end = p.rows;
    } else {
        if (!find_tile(p.offsets, p.experts, p.m, (p.cols + kSoloCols - 1) / kSoloCols, kRows, item, lane, &place)) return;
        const unsigned tq = (place.end - place.begin + kRows - 1) / kRows;
        row = place.begin + place.at % tq * kRows + row_in, col = place.at / tq * kSoloCols + col_in, rows_end = place.end;
    }
    if (row >= rows_end || col >= p.cols) return;
    float4v sum{0.f, 0.f, 0.f, 0.f};
    for (unsigned part = 0; part < split.parts; ++part)
        sum += *reinterpret_cast<const float4v*>(split.sums + ((size_t{part} * split.tiles + item) * kRows + row_in) * kSoloCols + col_in);
    store_four(cell(out, row, p.ldo, col), sum, p.cols - col, true);
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
        if (zvc_status st = launch(route_sums_kernel, dim3(p.experts), kSumThreads, stream, p)) return st;
        return launch(route_places_kernel, dim3(p.blocks), kRouteThreads, stream, p);
    });
}

template <typename T>
zvc_status route_backward_as(const RouteBackArgs& p, hipStream_t stream) {
    return with_chunks<T>(p.experts, [&](auto chunks) {
        return launch(route_backward_kernel<T, decltype(chunks)::value>, dim3(div_up(p.m, 256 / kRowLanes)), 256, stream, p);
    });
}

using Eights = Shape<2, 4, 4, 2, 2>;            // 128 x 128, eight waves
using Small = Shape<2, 2, 4, 4, 2>;             // 128 x 128, four waves

// Which kernel takes a product: persistent tiles of 256 x 256 or 128 x 128, the latter by way of registers, or the small kernels by their rows.
enum class Kind { kLarge, kSmall, kLoose, kSolo16, kSolo64 };

struct Choice {
    Kind kind;
    unsigned parts;                             // of a small kernel's sums (their bytes: within what most_row_sums and most_dw_sums say)
    double cost;
};

// Upper bound of the tiles by rows: every expert's last one may be short.
size_t row_tiles(size_t m, size_t experts, size_t tile) { return m / tile + (experts < m ? experts : m); }
// How many there will be: an expert's last tile is half full on the average.
double expected_tiles(size_t m, size_t experts, size_t tile) {
    const double used = static_cast<double>(experts < m ? experts : m), each = used > 0 ? static_cast<double>(m) / used / tile + 0.5 : 0;
    return used * (each > 1 ? each : 1);
}

// The account that chooses, in us: tiles in rounds of those that run at a time, each its stages and something to begin and finish.  Fitted to calls
// with every kernel forced in turn (m rows evenly over E experts, n, k; weights from memory), L large, S small tiles, s16 and s64 the small kernels:
//   bf16 forward  8 x 32, 2048, 2048: S 25.6, s16 18.3, s64 25.5    8 x 128, 2048, 2048: S 27.3, s16 34.9, s64 24.6    64 x 64, 2048, 128: S 14.2, s16 35.5, s64 38.1
//                 2 x 256, 512, 2048: S 24.0, s16 9.4, s64 13.1     16 x 512, 1024, 1024: L 30.7, S 29.4, s64 40.0     16 x 512, 5632, 2048: L 217, S 251
//   fp32 forward  8 x 32, 2048, 2048: S 132, s16 43.6, s64 81.9     8 x 128, 2048, 2048: S 136, s16 109, s64 131       16 x 512, 1024, 1024: S 188, s16 195, s64 181
//   dW            bf16 5 x 600, 1024, 512: S 17.2, s64 14.4         bf16 8 x 128, 2048, 2048: S 26.3, s64 69.6         fp32 5 x 600, 1024, 512: S 80.2, s64 47.6
//                 fp32 11 x 271, 256, 512: S 48.0, s16 17.6, s64 22.2     fp32 8 x 816, 3656, 520: S 258, s16 339, s64 276
// Against the fastest kernel forced, the one that is chosen takes, over 120 drawn sizes and more: y and dx 1.01 times as long in fp32, with 16 bits
// 1.04 (y) and 1.02 (dx), dW 1.03 and 1.05.
//   (tiles of 256 x 32 and small kernels with a tile for each wave were slower than these or the same everywhere)
constexpr double kLaunchUs = 5, kJoinUs = 3, kSumsPerUs = 3e6;

// (a part of a round of large tiles goes in quarters, see expert_product_kernel)
Choice large_choice(double tiles, double stages, bool quarters) {
    const double whole = std::floor(tiles / kUnits), part = tiles / kUnits - whole;
    const double rounds = whole + (part == 0 ? 0 : quarters && part <= 0.5 ? 0.4 * std::ceil(4 * part) : 1);
    return {Kind::kLarge, 1, kLaunchUs + rounds * (1.45 * stages + 10)};
}

Choice small_choice(double tiles, double stages, size_t w, bool loose) {
    double us;
    if (w == 4) us = std::ceil(tiles / kUnits) * (1.95 * stages + 2);                  // the matrix instructions bound it: two on a compute unit take twice as long
    else us = std::fmax(1, tiles / (2 * kUnits)) * ((tiles <= 2 * kUnits ? 0.72 : 1.35) * stages + 2);
    return {loose ? Kind::kLoose : Kind::kSmall, 1, kLaunchUs + (loose ? (w == 4 ? 1.3 : 1.5) : 1) * us};
}

// Parts of a small kernel's sums where its tiles do not fill the compute units.  More tiles never make it more parts, nor do fewer stages.
size_t solo_parts(double tiles, size_t stages) {
    size_t parts = tiles < 1 ? 1 : static_cast<size_t>(2 * kUnits / tiles);
    if (parts > stages / (2 * kSoloWaves)) parts = stages / (2 * kSoloWaves);
    if (parts > 16) parts = 16;
    return parts < 2 ? 1 : parts;
}
size_t solo_rows(Kind kind) { return kind == Kind::kSolo16 ? 16 : 64; }
size_t solo_tile_bytes(Kind kind) { return solo_rows(kind) * kSoloCols * sizeof(float); }

// most: tiles at most.
Choice solo_choice(Kind kind, size_t most, double tiles, size_t stages, size_t slots, double stage_us, double item_us) {
    if (most > size_t{1} << 20) return {kind, 1, HUGE_VAL};      // (a dimension of a grid holds fewer than 2^32 lanes)
    const size_t parts = solo_parts(tiles, stages), sums = parts > 1 ? parts * most * solo_tile_bytes(kind) : 0;
    const double each = item_us + stage_us * static_cast<double>(stages) / parts;
    return {kind, static_cast<unsigned>(parts), kLaunchUs + std::fmax(1, tiles * parts / slots) * each + (parts > 1 ? kJoinUs + sums / kSumsPerUs : 0)};
}

Choice cheaper(const Choice& a, const Choice& b) { return b.cost < a.cost ? b : a; }

// No sooner than the weights, `bytes`, are read at `rate` bytes a us.
Choice reading(Choice c, double bytes, double rate) {
    c.cost = std::fmax(c.cost, bytes / rate);
    return c;
}

// Of y (forward) or dx: `cols` columns, sums over `length`.  Small kernels read dx's weights in pieces of 64 columns of a row, and slower than others (dx of 645 rows, 28
// experts, 3248 x 2776, bf16: s16 167, S 89; y of 991 rows, 94 experts, 2336 x 1608: s16 161, S 114).
Choice choose_rows(size_t m, size_t experts, size_t cols, size_t length, size_t w, bool loose, bool forward) {
    const size_t stages = div_up(length, kStageBytes / w), across = div_up(cols, kSoloCols);
    const double bytes = static_cast<double>((experts < m ? experts : m) * cols * length * w);
    Choice best = reading(small_choice(expected_tiles(m, experts, 128) * div_up(cols, 128), stages, w, loose), bytes, 5.5e6);
    if (w == 2 && !loose)
        best = cheaper(best, reading(large_choice(expected_tiles(m, experts, 256) * div_up(cols, 256), stages, forward), bytes, 5e6));
    const Choice by16 = solo_choice(Kind::kSolo16, row_tiles(m, experts, 16) * across, expected_tiles(m, experts, 16) * across, stages, 4 * kUnits,
                                    w == 4 ? 0.65 : 0.4, w == 4 ? 4.1 : 2.8);
    const Choice by64 = solo_choice(Kind::kSolo64, row_tiles(m, experts, 64) * across, expected_tiles(m, experts, 64) * across, stages, 2 * kUnits,
                                    w == 4 ? 1.2 : 0.4, w == 4 ? 7.8 : 5);
    return cheaper(cheaper(best, reading(by16, bytes, forward ? 5e6 : 3.5e6)), reading(by64, bytes, forward ? 5.2e6 : 3.2e6));
}

// Of dW.  An expert may have several times the average of rows: a kernel does not end before its tiles have.
Choice choose_dw(size_t m, size_t experts, size_t n, size_t k, size_t w, bool loose) {
    const size_t stages = div_up(div_up(m, experts), kStageBytes / w), across = div_up(k, kSoloCols) * experts;
    const size_t tiles16 = div_up(n, 16) * across, tiles64 = div_up(n, 64) * across;
    const double longest = experts > 1 ? 3.0 * stages : stages;
    Choice best = small_choice(static_cast<double>(div_up(n, 128) * div_up(k, 128) * experts), stages, w, loose);
    if (w == 4) best.cost += 6;
    best.cost = std::fmax(best.cost, kLaunchUs + longest * (w == 4 ? 1.95 : 0.72) * (loose ? 1.4 : 1));
    if (w == 2 && !loose) best = cheaper(best, large_choice(static_cast<double>(div_up(n, 256) * div_up(k, 256) * experts), stages, false));
    // (16-bit types: tiles of 16 rows were faster than the others by 10 % in one of 120 drawn sizes)
    if (w == 4) best = cheaper(best, solo_choice(Kind::kSolo16, tiles16, static_cast<double>(tiles16), stages, 4 * kUnits, 0.5, 2.2));
    return cheaper(best, solo_choice(Kind::kSolo64, tiles64, static_cast<double>(tiles64), stages, 2 * kUnits, w == 4 ? 1.5 : 0.42, w == 4 ? 3.6 : 2.9));
}

// Bytes that the sums' parts take of m rows at most, however many fewer there are and whichever kernel the account chooses for them.
//
// y and dx: the fewer rows the more parts, up to those of one expert's few.  With u experts that have rows there are t >= u tiles expected and t >= m / tile + u / 2 (each
// times the tiles across), and parts <= 512 / t; room is made for m / tile + u tiles, at most 1.5 t of them, so for parts of 768 tiles at most.
size_t most_row_sums(size_t m, size_t experts, size_t cols, size_t length, size_t w) {
    const size_t across = div_up(cols, kSoloCols), parts = solo_parts(static_cast<double>(across), div_up(length, kStageBytes / w));
    size_t most = 0;
    for (const Kind kind : {Kind::kSolo16, Kind::kSolo64}) {
        const size_t tiles = parts * row_tiles(m, experts, solo_rows(kind)) * across, sums = parts > 1 ? (tiles < 3 * kUnits ? tiles : 3 * kUnits) * solo_tile_bytes(kind) : 0;
        most = sums > most ? sums : most;
    }
    return most;
}
// dW: the tiles are the same for any m, and more rows make more parts.
size_t most_dw_sums(size_t m, size_t experts, size_t n, size_t k, size_t w) {
    const size_t stages = div_up(div_up(m, experts), kStageBytes / w), across = div_up(k, kSoloCols) * experts;
    size_t most = 0;
    for (const Kind kind : {Kind::kSolo16, Kind::kSolo64}) {
        const size_t tiles = div_up(n, solo_rows(kind)) * across, parts = solo_parts(static_cast<double>(tiles), stages), sums = parts > 1 ? parts * tiles * solo_tile_bytes(kind) : 0;
        most = sums > most ? sums : most;
    }
    return most;
}

// (as many workgroups on each XCD: `room` is a multiple of 8)
unsigned grid_of(size_t items, unsigned room) { return static_cast<unsigned>(items < room ? round_up(items, 8) : room); }

template <typename T, class S>
zvc_status product_of(const ExpertArgs<T>& p, hipStream_t stream) {
    const size_t items = row_tiles(p.m, p.experts, S::QT) * div_up(p.cols, S::PT);
    return launch(expert_product_kernel<T, S>, dim3(grid_of(std::is_same_v<S, Large> ? 4 * items : items, kUnits * S::kPerUnit)), S::kThreads, stream, p);
}

template <typename T, class S>
zvc_status gradients_of(const ExpertArgs<T>& dx, const ExpertArgs<T>& dw, hipStream_t stream) {
    const size_t dw_tiles = div_up(dw.cols, S::PT) * div_up(dw.rows, S::QT);
    const size_t items = row_tiles(dx.m, dx.experts, S::QT) * div_up(dx.cols, S::PT) + dw_tiles * dw.experts;
    return launch(expert_gradients_kernel<T, S>, dim3(grid_of(items, kUnits * S::kPerUnit)), S::kThreads, stream, dx, dw, static_cast<unsigned>(dw_tiles));
}

template <typename T, Does DOES>
zvc_status loose_of(const ExpertArgs<T>& p, hipStream_t stream) {
    using S = Small;
    const size_t dw_tiles = DOES == Does::kDw ? div_up(p.cols, S::PT) * div_up(p.rows, S::QT) : 0;
    const size_t items = DOES == Does::kDw ? dw_tiles * p.experts : row_tiles(p.m, p.experts, S::QT) * div_up(p.cols, S::PT);
    return launch(loose_kernel<T, DOES, S>, dim3(grid_of(items, kUnits * S::kPerUnit)), S::kThreads, stream, p, static_cast<unsigned>(dw_tiles));
}

template <typename T, Does DOES, int QB, bool LOOSE>
zvc_status solo_as(const ExpertArgs<T>& p, unsigned parts, float* sums, hipStream_t stream) {
    const size_t across = div_up(p.cols, kSoloCols), dw_tiles = across * div_up(p.rows, 16 * QB);
    const size_t tiles = DOES == Does::kDw ? dw_tiles * p.experts : row_tiles(p.m, p.experts, 16 * QB) * across;
    const SoloSplit split = {sums, static_cast<unsigned>(tiles), parts, static_cast<unsigned>(dw_tiles)};
    const zvc_status st = launch(solo_kernel<T, DOES, QB, LOOSE>, dim3(static_cast<unsigned>(tiles * parts)), 64 * kSoloWaves, stream, p, split);
    if (st != ZVC_OK || parts == 1) return st;
    return launch(solo_join_kernel<T, DOES, QB>, dim3(static_cast<unsigned>(tiles * QB)), 256, stream, p, split);
}

template <typename T, Does DOES, int QB>
zvc_status solo_of(const ExpertArgs<T>& p, const Choice& choice, bool loose, float* sums, hipStream_t stream) {
    return loose ? solo_as<T, DOES, QB, true>(p, choice.parts, sums, stream) : solo_as<T, DOES, QB, false>(p, choice.parts, sums, stream);
}

// Whether an operand's rows take 16-byte accesses.
template <typename T>
bool takes_16(const T* at, size_t ld, size_t stride) { return aligned_to(at, 16) && ld * sizeof(T) % 16 == 0 && stride * sizeof(T) % 16 == 0; }

template <typename T>
zvc_status forward_as(const ExpertArgs<T>& p, float* sums, hipStream_t stream) {
    const bool loose = !takes_16(p.p, p.ldp, p.sp) || !takes_16(p.q, p.ldq, 0) || p.length * sizeof(T) % 16 != 0;
    const Choice choice = choose_rows(p.m, p.experts, p.cols, p.length, sizeof(T), loose, true);
    if (choice.kind == Kind::kSolo16) return solo_of<T, Does::kForward, 1>(p, choice, loose, sums, stream);
    if (choice.kind == Kind::kSolo64) return solo_of<T, Does::kForward, 4>(p, choice, loose, sums, stream);
    if (choice.kind == Kind::kLoose) return loose_of<T, Does::kForward>(p, stream);
    if constexpr (sizeof(T) == 2)
        if (choice.kind == Kind::kLarge) return product_of<T, Large>(p, stream);
    return product_of<T, Eights>(p, stream);
}

template <typename T>
zvc_status backward_as(ExpertArgs<T> dx, ExpertArgs<T> dw, float* sums, hipStream_t stream) {
    const bool loose_dx = !takes_16(dx.p, dx.ldp, dx.sp) || !takes_16(dx.q, dx.ldq, 0) || dx.length * sizeof(T) % 16 != 0;
    const bool loose_dw = !takes_16(dw.p, dw.ldp, 0) || !takes_16(dw.q, dw.ldq, 0);
    const Choice of_dx = choose_rows(dx.m, dx.experts, dx.cols, dx.length, sizeof(T), loose_dx, false);
    const Choice of_dw = choose_dw(dw.m, dw.experts, dw.rows, dw.cols, sizeof(T), loose_dw);
    const auto tiles = [](const Choice& c) { return c.kind == Kind::kLarge || c.kind == Kind::kSmall; };
    if (dx.cols != 0 && !tiles(of_dx)) {
        const zvc_status st = of_dx.kind == Kind::kSolo16   ? solo_of<T, Does::kDx, 1>(dx, of_dx, loose_dx, sums, stream)
                              : of_dx.kind == Kind::kSolo64 ? solo_of<T, Does::kDx, 4>(dx, of_dx, loose_dx, sums, stream)
                                                            : loose_of<T, Does::kDx>(dx, stream);
        if (st != ZVC_OK) return st;
        dx.cols = 0;
    }
    if (dw.cols != 0 && !tiles(of_dw)) {
        const zvc_status st = [&] {
            if constexpr (sizeof(T) == 4)
                if (of_dw.kind == Kind::kSolo16) return solo_of<T, Does::kDw, 1>(dw, of_dw, loose_dw, sums, stream);
            return of_dw.kind == Kind::kSolo64 ? solo_of<T, Does::kDw, 4>(dw, of_dw, loose_dw, sums, stream) : loose_of<T, Does::kDw>(dw, stream);
        }();
        if (st != ZVC_OK) return st;
        dw.cols = 0;
    }
    if (dx.cols == 0 && dw.cols == 0) return ZVC_OK;
    if constexpr (sizeof(T) == 2)
        if ((dx.cols != 0 ? of_dx : of_dw).kind == Kind::kLarge) return gradients_of<T, Large>(dx, dw, stream);
    return gradients_of<T, Small>(dx, dw, stream);
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
    const size_t w = type_bytes(type);
    if (w == 0 || !expert_sizes_ok(m, experts, n, k)) return 0;
    const size_t rows = backward == 0 ? most_row_sums(m, experts, n, k, w) : most_row_sums(m, experts, k, n, w);
    const size_t dw = backward == 0 ? 0 : most_dw_sums(m, experts, n, k, w);
    return 256 + round_up(rows > dw ? rows : dw, 256);
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
        p.p = static_cast<const T*>(d_w), p.ldp = static_cast<unsigned>(ldw), p.sp = sw;
        p.q = static_cast<const T*>(d_x), p.ldq = static_cast<unsigned>(ldx);
        p.out = static_cast<T*>(d_y), p.ldo = static_cast<unsigned>(ldy), p.offsets = d_offsets;
        p.m = static_cast<unsigned>(m), p.experts = static_cast<unsigned>(experts), p.cols = static_cast<unsigned>(n), p.length = static_cast<unsigned>(k);
        return forward_as(p, static_cast<float*>(d_ws), stream);
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
        p.offsets = d_offsets, p.m = static_cast<unsigned>(m), p.experts = static_cast<unsigned>(experts);
        ExpertArgs<T> dx = p, dw = p;
        dx.p = static_cast<const T*>(d_w), dx.ldp = static_cast<unsigned>(ldw), dx.sp = sw;
        dx.q = static_cast<const T*>(d_dy), dx.ldq = static_cast<unsigned>(lddy);
        dx.out = static_cast<T*>(d_dx), dx.ldo = static_cast<unsigned>(lddx);
        dx.cols = want_dx ? static_cast<unsigned>(k) : 0, dx.length = static_cast<unsigned>(n);
        dw.p = static_cast<const T*>(d_x), dw.ldp = static_cast<unsigned>(ldx);
        dw.q = static_cast<const T*>(d_dy), dw.ldq = static_cast<unsigned>(lddy);
        dw.out = static_cast<T*>(d_dw), dw.ldo = static_cast<unsigned>(lddw), dw.so = sdw;
        dw.cols = want_dw ? static_cast<unsigned>(k) : 0, dw.rows = static_cast<unsigned>(n);
        return backward_as(dx, dw, static_cast<float*>(d_ws), stream);
    };
    return type == ZVC_FP32 ? as(0.f) : type == ZVC_FP16 ? as(fp16{}) : as(bf16{});
}

}  // extern "C"
