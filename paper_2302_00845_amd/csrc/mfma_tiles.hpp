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

// Tiles of pairs: a matrix of pairs of fp16 lies as rows of 32 high parts, their 32 low parts, the next 32 high parts, .., so that a
// stage of 32 k takes whole lines of 128 bytes.  (In planes of their own 64 bytes at a time; a CU has about fifty requests on their
// way, whatever their size, and waited for those.  12 products of 768 x 768 and 768 x 2304: 69 -> 51 million busy cycles of the
// CUs.  The time hardly fell: under that load the clock does, from 2.0 to 1.5 GHz.)
// T x 32 of a matrix whose rows run along k (each row 128 bytes), or 32 x T of one whose rows run across.  Memory to LDS without
// registers, sixteen bytes a lane.  LDS rows are dense (a wave fills 1 KB in a row); sixteen-byte pieces are swapped within a row
// by its number, so that the lanes of a read hit different banks.
template <int T> struct PairTile {
    static constexpr int KC = 32, LEN = 2 * T * KC, CALLS = LEN / 8 / 64 / 4;  // fp16; a wavefront's loads
    static __device__ __forceinline__ int along(int r, int c) { return c ^ ((r >> 1) & 7); }
    static __device__ __forceinline__ int across(int r, int c) { return c ^ ((r & 7) << 1); }  // (pairs of pieces stay together)
};
// Where element (row, col) of such a matrix is, of `ld` elements per row; its low part is 32 further.
__device__ __forceinline__ int64_t pair_at(int64_t row, int64_t col, int64_t ld) { return row * 2 * ld + (col >> 5) * 64 + (col & 31); }

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

// A wavefront's share of a tile's loads: `from` is the same for all lanes, a lane adds `at[q]` bytes for its q-th load.
template <int T, bool ACROSS>
struct PairFetch {
    typedef PairTile<T> O;
    uint32_t at[O::CALLS];
    __device__ __forceinline__ PairFetch(int64_t ld, int wave, int lane) {
        constexpr int PIECES = ACROSS ? T / 4 : 8, ROWS = 64 / PIECES;
#pragma unroll
        for (int q = 0; q < O::CALLS; ++q) {
            const int row = (q * 4 + wave) * ROWS + lane / PIECES, slot = lane % PIECES;
            at[q] = (uint32_t)(row * 2 * (int)ld + (ACROSS ? O::across(row, slot) : O::along(row, slot)) * 8) * 2u;
        }
    }
    __device__ __forceinline__ void operator()(const f16_t *from, f16_t *lds, int wave) const {
        typedef __attribute__((address_space(3))) void *Lds;
        typedef const __attribute__((address_space(1))) void *Mem;
#pragma unroll
        for (int q = 0; q < O::CALLS; ++q)
            __builtin_amdgcn_global_load_lds((Mem)(reinterpret_cast<const char *>(from) + at[q]), (Lds)(lds + (q * 4 + wave) * 512), 16, 0, 0);
    }
};

// A lane's operands of 32 x 32 x 16 MFMAs: `at[k / 16]` is where those of the tile's first 32 rows (columns) lie, those of the i-th
// next are a constant further.
template <int T, bool ACROSS>
struct PairRead {
    typedef PairTile<T> O;
    int hi[2], lo[2], hi4[2], lo4[2];  // (hi4, lo4: the second half of a transposing read)
    __device__ __forceinline__ PairRead(int first, int lane) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (!ACROSS) {  // row first + lane % 32, elements 16 h + 8 (lane / 32) ..
                const int row = first + (lane & 31), piece = 2 * h + (lane >> 5);
                hi[h] = row * 64 + O::along(row, piece) * 8;
                lo[h] = row * 64 + O::along(row, piece + 4) * 8;
            } else {
                const int row = 16 * h + (lane >> 5) * 8 + ((lane & 15) >> 2), col = (lane & 16) + (lane & 3) * 4;
                const int piece = (first >> 5) * 8 + (col >> 3);
                hi[h] = row * 2 * T + O::across(row, piece) * 8 + (col & 4);
                lo[h] = row * 2 * T + O::across(row, piece + 4) * 8 + (col & 4);
                hi4[h] = (row + 4) * 2 * T + O::across(row + 4, piece) * 8 + (col & 4);
                lo4[h] = (row + 4) * 2 * T + O::across(row + 4, piece + 4) * 8 + (col & 4);
            }
        }
    }
    __device__ __forceinline__ f16x8 get(const f16_t *tile, int at, int at4, int i) const {
        if constexpr (!ACROSS) {
            return *reinterpret_cast<const f16x8 *>(tile + at + i * 32 * 64);
        } else {  // (pieces are swapped by exclusive or, and 32 columns further are eight pieces: another one, since `first` is a multiple of 64)
            typedef __attribute__((address_space(3))) s16x4 *Ptr;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(tile + (at ^ (i * 64))));
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(tile + (at4 ^ (i * 64))));
            return __builtin_bit_cast(f16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
    __device__ __forceinline__ f16x8 high(const f16_t *tile, int h, int i) const { return get(tile, hi[h], hi4[h], i); }
    __device__ __forceinline__ f16x8 low(const f16_t *tile, int h, int i) const { return get(tile, lo[h], lo4[h], i); }
};

}  // namespace cdgrab
