// Matrix products by tiles on the matrix cores of gfx950: how an operand is staged from memory to LDS and read from there, and the
// order that tiles are walked in.  Used by csrc/ffn.hip and csrc/experts.hip.
#pragma once

#include "elements.h"

namespace {

// ------------------------------------------------------------------ products on the matrix cores
//
// Every product here is  out[row][col] = sum over t of Q(row, t) P(col, t),  with `col` the output's contiguous
// index.  Gated block:  forward  P = Wg and Wu, Q = x;  dx  P = Wg then Wu by columns, Q = dg then du;  dW  P = x by columns,
// Q = dg or du by columns.  Experts, of one expert at a time:  forward  P = W, Q = x;  dx  P = W by columns, Q = dy;  dW  P = x by columns, Q = dy by columns.  P is the matrix instruction's first operand, so a lane holds four neighbouring columns
// of one row and stores them together.
//
// An operand lies either along the reduction (its rows are contiguous in t) or across it (its rows are the t).
// Both are staged as they lie, 128 bytes of reduction or as many of its rows at a time, straight from memory to LDS,
// and read from LDS as the instruction wants them: along by 16-byte reads, across by reads that transpose (16-bit
// types) or by element (fp32).  Units are exchanged within LDS rows so that the lanes of a read hit different banks;
// since the hardware writes a wave's 64 x 16 bytes in lane order, it is the lanes' global addresses that carry the exchange.
using float4v = float __attribute__((ext_vector_type(4)));
using int4v = int __attribute__((ext_vector_type(4)));
using short4v = short __attribute__((ext_vector_type(4)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using fp16x8 = _Float16 __attribute__((ext_vector_type(8)));

template <typename T> struct Fragment;
template <> struct Fragment<bf16> { using type = bf16x8; };
template <> struct Fragment<fp16> { using type = fp16x8; };
template <> struct Fragment<float> { using type = float4v; };

__device__ __forceinline__ float4v multiply(bf16x8 p, bf16x8 q, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, q, c, 0, 0, 0);
}
__device__ __forceinline__ float4v multiply(fp16x8 p, fp16x8 q, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(p, q, c, 0, 0, 0);
}
__device__ __forceinline__ float4v multiply(float4v p, float4v q, float4v c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(p[i], q[i], c, 0, 0, 0);
    return c;
}

constexpr unsigned kReach = 0x80000000u;       // bytes behind a tile's base that loads may reach
constexpr unsigned kNowhere = 0xC0000000u;     // an offset past that: such a load brings zeros
constexpr int kRawBuffer = 0x00020000;
constexpr int kStageBytes = 128;               // bytes of reduction per stage and row

// `address` is the same in all of a wave's lanes.
__device__ __forceinline__ int4v buffer_at(uint64_t address) {
    return int4v{__builtin_amdgcn_readfirstlane(static_cast<int>(address)),
                 __builtin_amdgcn_readfirstlane(static_cast<int>(address >> 32 & 0xFFFF)), static_cast<int>(kReach), kRawBuffer};
}

// 16 bytes a lane from memory to LDS, lane l's at lds + 16 l.  (No register is written: the wait is wait_loads()'s.  m0 is a register
// that the compiler keeps for itself and cannot be told of as overwritten; a test reads from the assembly that nothing else uses it.)
__device__ __forceinline__ void load_to_lds(int4v buffer, unsigned offset, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(buffer)
                 : "memory");
}

using LdsByte = __attribute__((address_space(3))) unsigned char;
__device__ __forceinline__ LdsByte* lds_at(unsigned offset) { return (LdsByte*)static_cast<uintptr_t>(offset); }

template <int LEFT>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void group_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

enum class Lies { kAlong, kAcross };

// The workgroup's tile: WP x WQ waves of PB x QB blocks of 16 x 16, and the stages that are in LDS at a time.
template <int WP_, int WQ_, int PB_, int QB_, int RING>
struct Shape {
    static constexpr int kRing = RING;
    static constexpr int WP = WP_, WQ = WQ_, PB = PB_, QB = QB_;
    static constexpr int kWavesAll = WP * WQ, kThreads = 64 * kWavesAll;
    static constexpr int PT = WP * PB * 16, QT = WQ * QB * 16;
    static constexpr int kStage = (PT + QT) * kStageBytes;
    static constexpr int kPerUnit = 2 * kRing * kStage > 160 << 10 ? 1 : 2;     // workgroups that a compute unit's LDS holds
};

// How one operand's tile of SIDE rows (kAlong) or columns (kAcross) is staged and read.  FOLD: the projections' P, in
// which 32 rows of Wg and 32 of Wu take turns, and a 16 x 16 block takes rows {8 a + 4 j + b : a, b < 4} of the 32, j = 0 | 1, so
// that a lane's two blocks are eight neighbouring columns.
template <typename T, Lies LIES, int SIDE, int WAVES, bool FOLD>
struct Operand {
    static constexpr int W = sizeof(T);
    static constexpr int kSteps = kStageBytes / W;                    // reduction per stage: 64 | 32
    static constexpr int kLoads = SIDE * kStageBytes / 1024 / WAVES;  // per wave and stage
    static constexpr int kRowBytes = LIES == Lies::kAlong ? kStageBytes : SIDE * W;
    static constexpr int kLanesPerRow = kRowBytes / 16;
    static constexpr int kRowsPerLoad = 1024 / kRowBytes;
    static constexpr int kUnit = LIES == Lies::kAlong ? 16 : W == 2 ? 32 : 64;   // what is exchanged within a row
    static constexpr int kUnitMask = kRowBytes / kUnit - 1;
    static_assert(kLoads * WAVES * 1024 == SIDE * kStageBytes, "whole loads");

    static __device__ __forceinline__ int exchange(int row) {
        if constexpr (LIES == Lies::kAlong)
            return FOLD ? (row & 3) | (row >> 3 & 1) << 2 : row & 7;
        else
            return (W == 2 ? (row & 3) | (row >> 3 & 3) << 2 : row >> 2 & 3) & kUnitMask;
    }

    unsigned offset[kLoads];            // of this lane's 16 bytes from the tile's base
    int first, lane_row, unit16;        // this wave's first load; the lane's row within a load, its 16 bytes' place

    // `left`: rows (kAlong) or columns (kAcross) of the tile that exist.  `ld` in elements.
    __device__ __forceinline__ void init(int wave, int lane, unsigned ld, unsigned left) {
        first = wave * kLoads;
        lane_row = lane / kLanesPerRow;
        unit16 = lane % kLanesPerRow;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = (first + i) * kRowsPerLoad + lane_row;
            const int place = logical(row);
            if constexpr (LIES == Lies::kAlong) {
                const unsigned r = FOLD ? (row >> 6) * 32 + (row & 31) : row;
                offset[i] = r < left ? r * ld * W + place : kNowhere;
            } else {
                offset[i] = place / W < static_cast<int>(left) ? row * ld * W + place : kNowhere;
            }
        }
    }
    // The byte within the row that the lane fetches for the place that it fills.
    __device__ __forceinline__ int logical(int row) const {
        const int place = unit16 * 16;
        return ((place / kUnit) ^ exchange(row)) * kUnit + place % kUnit;
    }
    // Whether load i of a stage with `left` of the reduction brings something.
    __device__ __forceinline__ bool within(int i, int left) const {
        const int row = (first + i) * kRowsPerLoad + lane_row;
        return LIES == Lies::kAlong ? logical(row) / W < left : row < left;
    }
    // Stage: `left` of the reduction remain at `base` (FOLD: at `base` for Wg's rows, at `other` for Wu's).
    __device__ __forceinline__ void fetch(uint64_t base, uint64_t other, int left, unsigned lds) const {
        constexpr int kRun = 32 / kRowsPerLoad;             // loads that bring 32 rows
        const bool odd = FOLD && kLoads <= kRun && (first / kRun & 1);
        const int4v buffers[] = {buffer_at(odd ? other : base), buffer_at(other)};
        const auto from = [&](int i) { return buffers[FOLD && kRun > 0 && i >= kRun]; };
        if (left >= kSteps) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) load_to_lds(from(i), offset[i], lds + (first + i) * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                load_to_lds(from(i), within(i, left) ? offset[i] : kNowhere, lds + (first + i) * 1024);
        }
    }
};

// A wave's reads of its strip of an operand from LDS: block b, half s of the stage.
template <typename T, Lies LIES, int SIDE, int BLOCKS, bool FOLD>
struct Reader {
    using Frag = typename Fragment<T>::type;
    using Op = Operand<T, LIES, SIDE, 1, FOLD>;
    static constexpr int W = sizeof(T);
    static constexpr int kReads = BLOCKS * (LIES == Lies::kAlong ? 1 : W);       // LDS instructions per half
    unsigned at[LIES == Lies::kAlong ? 2 : BLOCKS];

    __device__ __forceinline__ void init(unsigned lds, int strip, int lane) {
        const int r = lane & 15, q = lane >> 4;
        if constexpr (LIES == Lies::kAlong) {
            const int row = strip * BLOCKS * 16 + (FOLD ? (r >> 2) * 8 + (r & 3) : r);
            at[0] = lds + row * kStageBytes + (q ^ Op::exchange(row)) * 16;
            at[1] = lds + row * kStageBytes + ((q + 4) ^ Op::exchange(row)) * 16;
        } else {
            const int row = W == 2 ? q * 8 + (r >> 2) : q * 4;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
                at[b] = lds + row * Op::kRowBytes + ((strip * BLOCKS + b) ^ Op::exchange(row)) * Op::kUnit + (W == 2 ? (r & 3) * 8 : r * 4);
        }
    }
    __device__ __forceinline__ Frag read(int b, int s, unsigned stage) const {
        if constexpr (LIES == Lies::kAlong) {
            const int rows = FOLD ? (b >> 1) * 32 + (b & 1) * 4 : b * 16;
            return *reinterpret_cast<__attribute__((address_space(3))) Frag*>(lds_at(at[s] + stage + rows * kStageBytes));
        } else if constexpr (W == 2) {
            LdsByte* const p = lds_at(at[b] + stage + s * 32 * Op::kRowBytes);
            const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)p);
            const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(p + 4 * Op::kRowBytes));
            return __builtin_bit_cast(Frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            Frag f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                f[i] = *reinterpret_cast<__attribute__((address_space(3))) float*>(lds_at(at[b] + stage + (s * 16 + i) * Op::kRowBytes));
            return f;
        }
    }
};

// Asks the compiler to put the LDS reads of a block of straight code between its matrix instructions, evenly.
template <int READS, int PRODUCTS>
__device__ __forceinline__ void interleave() {
    constexpr int kEach = PRODUCTS / READS > 0 ? PRODUCTS / READS : 1;
#pragma unroll
    for (int i = 0; i < READS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);       // one LDS read
        __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);   // matrix instructions
    }
    __builtin_amdgcn_sched_group_barrier(0x008, PRODUCTS, 0);
}

// The place of work item `id` of `count` in the order that they are walked in: workgroups go to the eight XCDs in turn, so
// that each XCD takes a contiguous run of it.
__device__ __forceinline__ unsigned place_of(unsigned id, unsigned count) {
    const unsigned xcd = id % 8, per = count / 8, more = count % 8;
    return xcd * per + (xcd < more ? xcd : more) + id / 8;
}

constexpr unsigned kNone = ~0u;                  // no work item

template <class S>
__device__ __forceinline__ unsigned ring() {
    __shared__ alignas(1024) unsigned char lds[S::kRing * S::kStage];
    return static_cast<unsigned>(reinterpret_cast<uintptr_t>((LdsByte*)lds));
}

// Every gridDim.x-th item from `first` on.
struct Turns {
    unsigned at, items;
    __device__ __forceinline__ unsigned operator()() {
        const unsigned item = at;
        at += gridDim.x;
        return item < items ? item : kNone;
    }
};

constexpr unsigned kUnits = 256;                // compute units

}  // namespace
