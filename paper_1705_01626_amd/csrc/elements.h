// What the kernels of the training operators share (csrc/ffn.hip, csrc/experts.hip, csrc/adamw.hip): element types, the counter-based generator,
// eight neighbouring elements in registers, and the host's launches and checks of regions.
#pragma once

#include "zvc_ffn.h"

#include <hip/hip_runtime.h>

#include <cstdint>
#include <tuple>
#include <type_traits>
#include <utility>

namespace {

using bf16 = __bf16;
using fp16 = _Float16;

__host__ __device__ inline size_t div_up(size_t a, size_t b) { return (a + b - 1) / b; }
inline size_t round_up(size_t a, size_t b) { return div_up(a, b) * b; }

// ------------------------------------------------------------------ the generator
struct Words {
    unsigned w[4];
};

// a ^ b ^ c, one instruction.
__device__ __forceinline__ unsigned xor3(unsigned a, unsigned b, unsigned c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011): a block cipher's rounds of two 32 x 32 bit products each.
__device__ __forceinline__ Words philox(uint64_t index, uint64_t offset, uint64_t seed) {
    unsigned c0 = static_cast<unsigned>(index), c1 = static_cast<unsigned>(index >> 32);
    unsigned c2 = static_cast<unsigned>(offset), c3 = static_cast<unsigned>(offset >> 32);
    unsigned k0 = static_cast<unsigned>(seed), k1 = static_cast<unsigned>(seed >> 32);
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t a = static_cast<uint64_t>(0xD2511F53u) * c0, b = static_cast<uint64_t>(0xCD9E8D57u) * c2;
        c0 = xor3(static_cast<unsigned>(b >> 32), c1, k0);
        c1 = static_cast<unsigned>(b);
        c2 = xor3(static_cast<unsigned>(a >> 32), c3, k1);
        c3 = static_cast<unsigned>(a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

__device__ __forceinline__ unsigned half_of(const Words& r, int j) { return (r.w[j / 2] >> (16 * (j % 2))) & 0xFFFFu; }

// ------------------------------------------------------------------ eight elements
// Eight consecutive elements, held in 32 bits.
struct Eight {
    float v[8];
};

// 16 bytes at any element: the instruction takes them wherever they lie.
template <typename T>
struct Pack {
    T v[16 / sizeof(T)];
};

template <typename T>
__device__ __forceinline__ Eight load8(const T* at) {
    Eight out;
    constexpr int kPer = 16 / sizeof(T);
#pragma unroll
    for (int h = 0; h < 8 / kPer; ++h) {
        Pack<T> p;
        __builtin_memcpy(&p, at + h * kPer, 16);
#pragma unroll
        for (int j = 0; j < kPer; ++j) out.v[h * kPer + j] = static_cast<float>(p.v[j]);
    }
    return out;
}

// past: past the caches' replacement, for an output that they cannot hold; `at` is then a multiple of 16 bytes.  (Stores of
// different alignment: of equal ones behind a branch the compiler makes one, an ordinary one.)
template <typename T>
__device__ __forceinline__ void store8(T* at, const Eight& e, bool past = false) {
    constexpr int kPer = 16 / sizeof(T);
    using Quad = unsigned __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int h = 0; h < 8 / kPer; ++h) {
        Pack<T> p;
#pragma unroll
        for (int j = 0; j < kPer; ++j) p.v[j] = static_cast<T>(e.v[h * kPer + j]);
        if (past) {
            Quad q;
            __builtin_memcpy(&q, &p, 16);
            __builtin_nontemporal_store(q, reinterpret_cast<Quad*>(at + h * kPer));
        } else {
            __builtin_memcpy(at + h * kPer, &p, 16);
        }
    }
}

template <typename T>
__device__ __forceinline__ T* cell(T* at, unsigned row, unsigned ld, unsigned col) { return at + (static_cast<uint64_t>(row) * ld + col); }

// Zero where the mask's bit is clear, whatever is there (without a branch: an element's chain of exp and reciprocal is long, and
// only the chains of several elements side by side hide it).
__device__ __forceinline__ void drop8(unsigned keep, Eight& x) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
        x.v[j] = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, x.v[j]) & (0u - (keep >> j & 1u)));
}

// The first `there` of eight elements; `full`: eight, in all of a wave's lanes (a branch that the wave takes as one: with masks
// for lanes that have fewer, a tile's stores cost 3 us more).
template <typename T>
__device__ __forceinline__ Eight load_some(const T* at, int there, bool full) {
    if (full) return load8(at);
    Eight e = {};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < there) e.v[j] = static_cast<float>(at[j]);
    return e;
}
template <typename T>
__device__ __forceinline__ void store_some(T* at, const Eight& e, int there, bool full) {
    if (full) return store8(at, e);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < there) at[j] = static_cast<T>(e.v[j]);
}

// How many of eight columns from `col` on there are.
__device__ __forceinline__ int columns_left(unsigned n, unsigned col) { return col + 8 <= n ? 8 : col < n ? static_cast<int>(n - col) : 0; }

// ------------------------------------------------------------------ host side
// A launch that reports its own status (hipGetLastError would also report, and clear, an earlier error of the calling thread).
template <typename... Params, size_t... I>
zvc_status launch_as(void (*kernel)(Params...), dim3 grid, unsigned threads, hipStream_t stream, std::tuple<Params...>& values,
                     std::index_sequence<I...>) {
    void* pointers[] = {static_cast<void*>(&std::get<I>(values))...};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), pointers, 0, stream) == hipSuccess ? ZVC_OK : ZVC_E_HIP;
}
template <typename... Params, typename... Args>
zvc_status launch(void (*kernel)(Params...), dim3 grid, unsigned threads, hipStream_t stream, Args... args) {
    static_assert(sizeof...(Params) == sizeof...(Args), "one argument per kernel parameter");
    std::tuple<Params...> values(static_cast<Params>(args)...);
    return launch_as(kernel, grid, threads, stream, values, std::index_sequence_for<Params...>{});
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
inline bool overlap(const Region& a, const Region& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
    if (a.at == nullptr || b.at == nullptr || a.bytes() == 0 || b.bytes() == 0) return false;
    if (x + a.bytes() <= y || y + b.bytes() <= x) return false;
    if (a.ld != b.ld || a.rows <= 1 || b.rows <= 1) return true;
    const size_t gap = y >= x ? (y - x) % a.ld : (a.ld - (x - y) % a.ld) % a.ld;
    return !(gap >= a.cols && gap + b.cols <= a.ld);
}

}  // namespace
