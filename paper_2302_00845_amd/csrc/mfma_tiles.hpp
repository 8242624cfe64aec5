// Tiles of 16-bit elements in LDS and MFMAs of 32 x 32 x 16 on them: what products of long rows share.
#pragma once
#include "layer_common.hpp"

namespace cdgrab {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma32(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// Memory to LDS without registers, sixteen bytes a lane, NS stages of 32 k on their way or in use.  LDS rows are dense (a wave
// fills 1 KB in a row); sixteen-byte pieces are swapped within a row by its number, so that the lanes of a read hit different banks.
template <int T> struct LdsTile {
    static constexpr int KC = 32, PLANE = T * KC, CALLS = PLANE / 8 / 64 / 4;  // elements; a wavefront's loads per plane
    // piece c of row r of an [T][KC] plane / of a [KC][T] plane (pairs of pieces stay together for the transposing read)
    static __device__ __forceinline__ int along(int r, int c) { return c ^ ((r >> 2) & 3); }
    static __device__ __forceinline__ int across(int r, int c) { return T == 128 ? c ^ ((r & 7) << 1) : c ^ (((r >> 1) & 3) << 1); }
};

// Waits until at most LEFT of this wavefront's loads are on their way and its LDS reads are done, then for the workgroup.
// (By builtins: the compiler then knows that the reads are done, and does not wait for the next ones instead.)
template <int LEFT>
__device__ __forceinline__ void stage_barrier() {
    static_assert(LEFT < 64, "six bits");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_s_waitcnt((LEFT & 15) | (LEFT >> 4) << 14 | 7 << 4);  // vmcnt LEFT, lgkmcnt 0, expcnt any
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    __builtin_amdgcn_sched_barrier(0);
}

// A wavefront's share of a stage's loads of one plane: `from` is the same for all lanes, a lane adds `at[q]` bytes for its q-th load.
template <typename E, int T, bool ACROSS>
struct TileFetch {
    typedef LdsTile<T> O;
    uint32_t at[O::CALLS];
    __device__ __forceinline__ TileFetch(int64_t ld, int wave, int lane) {
        constexpr int PIECES = ACROSS ? T / 8 : O::KC / 8, ROWS = 64 / PIECES;
#pragma unroll
        for (int q = 0; q < O::CALLS; ++q) {
            const int row = (q * 4 + wave) * ROWS + lane / PIECES, slot = lane % PIECES;
            at[q] = (uint32_t)(row * (int)ld + (ACROSS ? O::across(row, slot) : O::along(row, slot)) * 8) * 2u;
        }
    }
    __device__ __forceinline__ void operator()(const E *from, E *lds, int wave) const {
        typedef __attribute__((address_space(3))) void *Lds;
        typedef const __attribute__((address_space(1))) void *Mem;
#pragma unroll
        for (int q = 0; q < O::CALLS; ++q)
            __builtin_amdgcn_global_load_lds((Mem)(reinterpret_cast<const char *>(from) + at[q]), (Lds)(lds + (q * 4 + wave) * 512), 16, 0, 0);
    }
};

// A lane's operands of 32 x 32 x 16 MFMAs: `at[k / 16]` is where those of the tile's first 32 rows (columns) lie in a plane,
// those of the i-th next are a constant further, as the planes and stages are.
template <typename E, int T, bool ACROSS>
struct TileRead {
    typedef LdsTile<T> O;
    int at[2], at4[2];  // (in elements; at4: the second half of a transposing read)
    __device__ __forceinline__ TileRead(int first, int lane) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (!ACROSS) {  // row first + lane % 32, elements 16 h + 8 (lane / 32) ..
                const int row = first + (lane & 31);
                at[h] = row * O::KC + O::along(row, 2 * h + (lane >> 5)) * 8;
            } else {
                const int row = 16 * h + (lane >> 5) * 8 + ((lane & 15) >> 2), col = first + (lane & 16) + (lane & 3) * 4;
                at[h] = row * T + O::across(row, col >> 3) * 8 + (col & 4);
                at4[h] = (row + 4) * T + O::across(row + 4, col >> 3) * 8 + (col & 4);
            }
        }
    }
    // (ACROSS: columns are swapped by exclusive or, and so are those 32 further, since `first` is a multiple of 64)
    typedef E Vec __attribute__((ext_vector_type(8)));
    __device__ __forceinline__ Vec operator()(const E *plane, int h, int i) const {
        if constexpr (!ACROSS) {
            return *reinterpret_cast<const Vec *>(plane + at[h] + i * 32 * O::KC);
        } else {
            typedef __attribute__((address_space(3))) s16x4 *Ptr;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(plane + (at[h] ^ (i * 32))));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(plane + (at4[h] ^ (i * 32))));
            return __builtin_bit_cast(Vec, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

}  // namespace cdgrab
