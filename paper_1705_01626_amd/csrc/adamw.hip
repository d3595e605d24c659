// AdamW over many tensors in one launch, states in 32 bits or in 8, for AMD gfx950 (wave64): kernel and C ABI
// (include/zvc_adamw.h has the formulas).
//
// A step reads and writes everything once and is bound by that: what is here keeps the rest out of the way.  A workgroup takes 2048 neighbouring elements of one tensor, a lane
// eight of them, whatever the tensors' number and sizes (256 lanes; 128 and 512 took the same); it finds its tensor in the plan by comparing 64 first pieces at a time.
// Times in the comments are us on one MI355X, where a large copy moves 5.0 TB/s: 138 M fp32 elements 729 (5.3 TB/s), 138 M bf16 elements with masters and
// states of 8 bits 443 (5.0 TB/s), 0.74 M elements in many odd tensors 9.6, of which a launch and two chained reads are most.

#include "elements.h"
#include "zvc_adamw.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

namespace {

constexpr int kThreads = 256;
constexpr unsigned kPiece = 8 * kThreads;              // elements of a workgroup
constexpr uint64_t kCacheBytes = uint64_t{256} << 20;   // in front of the memory
constexpr uint64_t kMostPieces = (1u << 24) - 1;       // a dimension of a grid holds fewer than 2^32 lanes
constexpr uint64_t kMagic = 0x7a76635f6164616dull;

// A plan: this, then the first piece of each tensor and the number of pieces behind the last one (64 entries of filling), then the
// tensors as the caller described them.
struct Header {
    uint64_t magic, tensors, pieces, bytes, weights, unused;      // weights: their bytes
};
inline size_t starts_bytes(size_t tensors) { return round_up((tensors + 65) * sizeof(unsigned), 16); }

struct Now {
    float shrink, step_size, beta1, beta2, gain1, gain2, root_scale, eps, factor;
    double rate, decay, wide_beta1, wide_beta2;
    uint64_t step, seed;
    const uint64_t* d_step;
    const float* d_factors;
    bool past;                            // weights go past the caches
};

// beta^t by squaring: the same on the host and on the device.
__host__ __device__ inline double power(double beta, uint64_t t) {
    double out = 1.0;
    for (; t != 0; t >>= 1, beta *= beta)
        if (t & 1) out *= beta;
    return out;
}

// What depends on the step's number and the factors.
__host__ __device__ inline void settle(Now* now, uint64_t t, double rate, float factor) {
    now->step = t;
    now->shrink = static_cast<float>(1.0 - rate * now->decay);
    now->step_size = static_cast<float>(rate / (1.0 - power(now->wide_beta1, t)));
    now->root_scale = static_cast<float>(1.0 / sqrt(1.0 - power(now->wide_beta2, t)));
    now->factor = factor;
}

__device__ __forceinline__ unsigned bits_of(float x) { return __builtin_bit_cast(unsigned, x); }
__device__ __forceinline__ float float_of(unsigned x) { return __builtin_bit_cast(float, x); }

// The largest of 16 neighbouring lanes, in all of them.
__device__ __forceinline__ unsigned most_of_16(unsigned x) {
    x = max(x, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x128, 0xF, 0xF, false)));    // rotated within 16 by 8
    x = max(x, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x124, 0xF, 0xF, false)));
    x = max(x, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x122, 0xF, 0xF, false)));
    return max(x, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x121, 0xF, 0xF, false)));
}

struct Codes {
    unsigned char v[8];
};
__device__ __forceinline__ Codes load_codes(const unsigned char* at, int there, bool full) {
    Codes c = {};
    if (full) {
        __builtin_memcpy(&c, at, 8);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < there) c.v[j] = at[j];
    }
    return c;
}
__device__ __forceinline__ void store_codes(unsigned char* at, const Codes& c, int there, bool full, bool past) {
    if (full && past) {
        uint64_t all;
        __builtin_memcpy(&all, &c, 8);
        __builtin_nontemporal_store(all, reinterpret_cast<uint64_t*>(at));
    } else if (full) {
        __builtin_memcpy(at, &c, 8);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < there) at[j] = c.v[j];
    }
}

// The numbers of codes: e4m3's exponent and significand are float's, moved up by 20 bits, but for the bias.
__device__ __forceinline__ Eight widen(const Codes& c, float scale) {
    Eight e;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        e.v[j] = float_of((c.v[j] & 0x7Fu) << 20 | (c.v[j] & 0x80u) << 24) * 0x1p120f * scale;
    return e;
}

// A lane's eight of a block's values as codes, and the block's scale.  Over the scale and with e4m3's bias a value's upper bits are its code
// and the 20 below are what is cut off; a random half on top of those carries with the right probability.
template <bool LEAST>
__device__ __forceinline__ Codes narrow(const Eight& e, const Words& random, float* scale) {
    unsigned most = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const unsigned size = bits_of(e.v[j]) & 0x7FFFFFFFu;
        most = max(most, size < 0x7F800000u ? size : 0u);
    }
    const unsigned exponent = max(most_of_16(most) >> 23, 32u);
    *scale = float_of((exponent - 7) << 23);
    const float inverse = float_of((261 - exponent) << 23);
    Codes c;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float size = fabsf(e.v[j]);
        unsigned code = 0x7E;
        if (size < INFINITY) code = min((bits_of(size * inverse * 0x1p-120f) + (half_of(random, j) << 4)) >> 20, 0x7Eu);
        if (LEAST && size > 0.f) code = max(code, 1u);
        c.v[j] = static_cast<unsigned char>(code | (bits_of(e.v[j]) >> 24 & 0x80u));
    }
    return c;
}

// past: past the caches' replacement; `at` is then a multiple of 16 bytes.
template <typename T>
__device__ __forceinline__ void store_past(T* at, const Eight& e, int there, bool full, bool past) {
    if (full && past) store8(at, e, true);
    else store_some(at, e, there, full);
}

// Eight neighbouring elements from `i` on, `there` of which exist.
template <typename P, typename G, bool MASTER, int BITS>
__device__ __forceinline__ void update(const zvc_adamw_tensor& t, const Now& now, unsigned number, uint64_t i, int there) {
#pragma clang fp contract(off)
    const bool full = __all(there == 8);
    // What no one reads before the next step goes past the caches, and so do weights that those cannot hold (`now.past`), of which the forward pass
    // would find little there: 138 M fp32 elements 729, by way of the caches 792; with states of 8 bits 443 and 489.
    const auto address = [](const void* at) { return reinterpret_cast<uintptr_t>(at); };
    const bool past = (address(t.d_m) | address(t.d_v) | address(t.d_master)) % 16 == 0;
    P* const param = static_cast<P*>(t.d_param) + i;
    float* const master = t.d_master + i;
    const Eight grad = load_some(static_cast<const G*>(t.d_grad) + i, there, full);
    Eight p = MASTER ? load_some(static_cast<const float*>(master), there, full) : load_some(static_cast<const P*>(param), there, full);
    Eight m, v;
    const uint64_t block = i / ZVC_ADAMW_BLOCK;
    if constexpr (BITS == 8) {
        const Codes cm = load_codes(static_cast<const unsigned char*>(t.d_m) + i, there, full);
        const Codes cr = load_codes(static_cast<const unsigned char*>(t.d_v) + i, there, full);
        m = widen(cm, there > 0 ? t.d_m_scale[block] : 0.f), v = widen(cr, there > 0 ? t.d_v_scale[block] : 0.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) v.v[j] = v.v[j] * v.v[j];
    } else {
        m = load_some(static_cast<const float*>(t.d_m) + i, there, full);
        v = load_some(static_cast<const float*>(t.d_v) + i, there, full);
    }
    const float shrink = t.decays != 0 ? now.shrink : 1.f;
    // (the reciprocal is off by a unit of 32 bits' last place at most; a division instead: bf16 with states of 8 bits and no masters 640, as it is 600)
    Eight root;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float g = grad.v[j] * now.factor;
        m.v[j] = now.beta1 * m.v[j] + now.gain1 * g;
        v.v[j] = now.beta2 * v.v[j] + now.gain2 * (g * g);
        root.v[j] = sqrtf(v.v[j]);
        p.v[j] = p.v[j] * shrink - now.step_size * (m.v[j] * __builtin_amdgcn_rcpf(root.v[j] * now.root_scale + now.eps));
    }
    if constexpr (MASTER) store_past(master, p, there, full, past);
    store_past(param, p, there, full, now.past && address(param) % 16 == 0);
    if constexpr (BITS == 8) {
        const Words random = philox(i / 8 | static_cast<uint64_t>(number) << 32, now.step, now.seed);
        float scale_m, scale_r;
        const Codes cm = narrow<false>(m, random, &scale_m), cr = narrow<true>(root, random, &scale_r);
        store_codes(static_cast<unsigned char*>(t.d_m) + i, cm, there, full, past);
        store_codes(static_cast<unsigned char*>(t.d_v) + i, cr, there, full, past);
        if (i % ZVC_ADAMW_BLOCK == 0 && there > 0) t.d_m_scale[block] = scale_m, t.d_v_scale[block] = scale_r;
    } else {
        store_past(static_cast<float*>(t.d_m) + i, m, there, full, past);
        store_past(static_cast<float*>(t.d_v) + i, v, there, full, past);
    }
}

template <typename P, typename G, bool MASTER>
__device__ __forceinline__ void update_as(const zvc_adamw_tensor& t, const Now& now, unsigned number, uint64_t i, int there) {
    if (t.state_bits == 8) update<P, G, MASTER, 8>(t, now, number, i, there);
    else update<P, G, MASTER, 32>(t, now, number, i, there);
}

template <typename P>
__device__ __forceinline__ void update_16(const zvc_adamw_tensor& t, const Now& now, unsigned number, uint64_t i, int there) {
    if (t.grad_type == ZVC_FP32) {
        if (t.d_master != nullptr) update_as<P, float, true>(t, now, number, i, there);
        else update_as<P, float, false>(t, now, number, i, there);
    } else {
        if (t.d_master != nullptr) update_as<P, P, true>(t, now, number, i, there);
        else update_as<P, P, false>(t, now, number, i, there);
    }
}

// A workgroup takes one piece of one tensor.
__global__ __launch_bounds__(kThreads) void adamw_kernel(const unsigned* starts, const zvc_adamw_tensor* tensors, unsigned count, Now now) {
    const unsigned piece = blockIdx.x, lane = threadIdx.x & 63;
    // The last tensor whose first piece is not behind this one: 64 of them are compared at a time.
    unsigned low = 0, left = count;
    while (left > 1) {
        const unsigned stride = (left + 63) / 64, at = lane * stride;
        const bool before = at < left && starts[low + at] <= piece;
        const unsigned last = static_cast<unsigned>(__popcll(__ballot(before))) - 1;
        low += last * stride;
        left = min(stride, left - last * stride);
    }
    low = __builtin_amdgcn_readfirstlane(low);
    const zvc_adamw_tensor t = tensors[low];
    if (now.d_step != nullptr || now.d_factors != nullptr) {
        const uint64_t step = now.step + (now.d_step != nullptr ? *now.d_step : 0);
        const float rate = now.d_factors != nullptr ? now.d_factors[0] : 1.f, factor = now.d_factors != nullptr ? now.d_factors[1] : 1.f;
        settle(&now, step == 0 ? 1 : step, now.rate * rate, now.factor * factor);
    }
    const uint64_t i = static_cast<uint64_t>(piece - starts[low]) * kPiece + threadIdx.x * 8;
    const int there = i >= t.count ? 0 : t.count - i < 8 ? static_cast<int>(t.count - i) : 8;
    if (__all(there == 0)) return;
    if (t.type == ZVC_FP32) update_as<float, float, false>(t, now, low, i, there);
    else if (t.type == ZVC_FP16) update_16<fp16>(t, now, low, i, there);
    else update_16<bf16>(t, now, low, i, there);
}

// ------------------------------------------------------------------ host side
struct Span {
    uintptr_t begin, end;
    bool written;
};

zvc_status check_tensor(const zvc_adamw_tensor& t) {
    const size_t w = type_bytes(t.type), g = type_bytes(t.grad_type);
    if (w == 0 || g == 0 || (t.grad_type != t.type && t.grad_type != ZVC_FP32) || (t.state_bits != 8 && t.state_bits != 32) ||
        t.count > ZVC_ADAMW_MAX_ELEMENTS || (t.d_master != nullptr && w == 4))
        return ZVC_E_ARG;
    if (t.count == 0) return ZVC_OK;
    if (t.d_param == nullptr || t.d_grad == nullptr || t.d_m == nullptr || t.d_v == nullptr ||
        (t.d_m_scale != nullptr) != (t.state_bits == 8) || (t.d_v_scale != nullptr) != (t.state_bits == 8))
        return ZVC_E_ARG;
    const size_t s = t.state_bits / 8;
    if (!aligned_to(t.d_param, w) || !aligned_to(t.d_grad, g) || !aligned_to(t.d_master, 4) || !aligned_to(t.d_m, s) || !aligned_to(t.d_v, s) ||
        !aligned_to(t.d_m_scale, 4) || !aligned_to(t.d_v_scale, 4))
        return ZVC_E_ALIGN;
    return ZVC_OK;
}

// Whether what is written overlaps anything.
bool clashes(Span* spans, size_t count) {
    std::sort(spans, spans + count, [](const Span& a, const Span& b) { return a.begin < b.begin; });
    uintptr_t all = 0, written = 0;
    for (size_t i = 0; i < count; ++i) {
        if (spans[i].begin < (spans[i].written ? all : written)) return true;
        all = std::max(all, spans[i].end);
        if (spans[i].written) written = std::max(written, spans[i].end);
    }
    return false;
}

}  // namespace

// ------------------------------------------------------------------ C ABI
extern "C" {

size_t zvc_adamw_plan_bytes(size_t tensors) {
    return tensors > ZVC_ADAMW_MAX_TENSORS ? 0 : sizeof(Header) + starts_bytes(tensors) + tensors * sizeof(zvc_adamw_tensor);
}

zvc_status zvc_adamw_plan(const zvc_adamw_tensor* tensors, size_t count, void* plan, size_t bytes) {
    if (count > ZVC_ADAMW_MAX_TENSORS || (count != 0 && tensors == nullptr) || plan == nullptr) return ZVC_E_ARG;
    if (!aligned_to(plan, 8)) return ZVC_E_ALIGN;
    const size_t need = zvc_adamw_plan_bytes(count);
    if (bytes < need) return ZVC_E_CAPACITY;
    uint64_t pieces = 0, weights = 0;
    for (size_t i = 0; i < count; ++i) {
        if (zvc_status st = check_tensor(tensors[i])) return st;
        pieces += div_up(tensors[i].count, kPiece);
        weights += tensors[i].count * type_bytes(tensors[i].type);
    }
    if (pieces > kMostPieces) return ZVC_E_ARG;
    Span* const spans = new (std::nothrow) Span[7 * count + 1];
    if (spans == nullptr) return ZVC_E_CAPACITY;
    size_t used = 0;
    bool wraps = false;
    const auto add = [&](const void* at, uint64_t size, bool written) {
        const uintptr_t begin = reinterpret_cast<uintptr_t>(at);
        if (at == nullptr || size == 0) return;
        wraps |= begin + size < begin;
        spans[used++] = {begin, begin + size, written};
    };
    for (size_t i = 0; i < count; ++i) {
        const zvc_adamw_tensor& t = tensors[i];
        const uint64_t state = t.count * (t.state_bits / 8), scales = div_up(t.count, ZVC_ADAMW_BLOCK) * 4;
        add(t.d_param, t.count * type_bytes(t.type), true);
        add(t.d_master, t.count * 4, true);
        add(t.d_grad, t.count * type_bytes(t.grad_type), false);
        add(t.d_m, state, true), add(t.d_v, state, true);
        if (t.state_bits == 8) add(t.d_m_scale, scales, true), add(t.d_v_scale, scales, true);
    }
    const bool bad = wraps || clashes(spans, used);
    delete[] spans;
    if (bad) return ZVC_E_ARG;
    unsigned char* const out = static_cast<unsigned char*>(plan);
    const Header header = {kMagic, count, pieces, need, weights, 0};
    std::memcpy(out, &header, sizeof header);
    unsigned* const starts = reinterpret_cast<unsigned*>(out + sizeof header);
    unsigned at = 0;
    for (size_t i = 0; i < starts_bytes(count) / sizeof(unsigned); ++i) {
        starts[i] = at;
        if (i < count) at += static_cast<unsigned>(div_up(tensors[i].count, kPiece));
    }
    if (count != 0) std::memcpy(out + sizeof header + starts_bytes(count), tensors, count * sizeof(zvc_adamw_tensor));
    return ZVC_OK;
}

zvc_status zvc_adamw(const void* plan, const void* d_plan, const zvc_adamw_now* now, hipStream_t stream) {
    if (plan == nullptr || now == nullptr) return ZVC_E_ARG;
    if (!aligned_to(plan, 8) || !aligned_to(now, 8)) return ZVC_E_ALIGN;
    Header header;
    std::memcpy(&header, plan, sizeof header);
    if (header.magic != kMagic || header.tensors > ZVC_ADAMW_MAX_TENSORS || header.bytes != zvc_adamw_plan_bytes(header.tensors)) return ZVC_E_ARG;
    const double values[] = {now->rate, now->decay, now->eps, now->factor};
    for (const double v : values)
        if (!std::isfinite(static_cast<float>(v))) return ZVC_E_ARG;
    const auto share = [](double v) { return v >= 0.0 && v < 1.0; };
    if (!share(now->beta1) || !share(now->beta2) || now->eps < 0.0) return ZVC_E_ARG;
    if (now->d_step == nullptr && now->step == 0) return ZVC_E_ARG;
    if (!aligned_to(now->d_step, 8) || !aligned_to(now->d_factors, 4)) return ZVC_E_ALIGN;
    if (header.pieces == 0) return ZVC_OK;
    if (d_plan == nullptr) return ZVC_E_ARG;
    if (!aligned_to(d_plan, 16)) return ZVC_E_ALIGN;
    Now n{};
    n.rate = now->rate, n.decay = now->decay, n.eps = static_cast<float>(now->eps);
    n.beta1 = static_cast<float>(now->beta1), n.beta2 = static_cast<float>(now->beta2);
    n.gain1 = static_cast<float>(1.0 - now->beta1), n.gain2 = static_cast<float>(1.0 - now->beta2);
    n.wide_beta1 = now->beta1, n.wide_beta2 = now->beta2;
    n.seed = now->seed, n.d_step = now->d_step, n.d_factors = now->d_factors;
    settle(&n, now->step == 0 ? 1 : now->step, n.rate, static_cast<float>(now->factor));
    n.step = now->step;
    n.past = header.weights >= kCacheBytes;
    const unsigned char* const at = static_cast<const unsigned char*>(d_plan) + sizeof(Header);
    return launch(adamw_kernel, dim3(static_cast<unsigned>(header.pieces)), kThreads, stream, reinterpret_cast<const unsigned*>(at),
                  reinterpret_cast<const zvc_adamw_tensor*>(at + starts_bytes(header.tensors)), static_cast<unsigned>(header.tensors), n);
}

}  // extern "C"
