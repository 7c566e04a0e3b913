// Rows of elements in pieces of 16 bytes, aligned to an element, requested without a branch: behind one each, the loads of a tile leave one by one (a
// branch that may write the same registers makes the next load wait for all before it: a step of 1024 environments, 127 us with branches, 85 without).
#pragma once

#include "numeric.h"

typedef uint32_t piece_t __attribute__((ext_vector_type(4), aligned(2)));

// The piece of a row of D elements that begins at element col; elements from D on are zero.  WHOLE: D is a multiple of a piece.
// Where col >= D (or nothing is wanted: `in`), zeros; what is requested then lies in the row all the same.
template <typename T, bool WHOLE>
struct RowPiece {
    static constexpr int VE = 16 / sizeof(T);
    uint4 u;
    __device__ inline void load(const T* row, int col, int D) {
        if constexpr (WHOLE) {
            const piece_t w = *reinterpret_cast<const piece_t*>(row + (col < D ? col : 0));
            u = make_uint4(w[0], w[1], w[2], w[3]);
        } else if (D >= VE) {  // (the last one of a row: the 16 bytes that end with it, moved down below)
            const piece_t w = *reinterpret_cast<const piece_t*>(row + (col < D - VE ? col : D - VE));
            u = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                const T* p = row + (i < D ? i : D - 1);
                if constexpr (sizeof(T) == 2) w[i / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p) << (16 * (i & 1));
                else w[i] = *reinterpret_cast<const uint32_t*>(p);
            }
            u = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    __device__ inline uint4 get(int col, int D, bool in = true) const {
        uint4 v = u;
        if constexpr (!WHOLE) {
            const int first = D >= VE ? (col < D - VE ? col : D - VE) : 0, bits = (col - first) * (int)sizeof(T) * 8;
            uint64_t lo = ((uint64_t)v.y << 32) | v.x, hi = ((uint64_t)v.w << 32) | v.z;
            const int s = bits & 63;
            lo = (lo >> s) | ((hi << 1) << (63 - s));
            hi >>= s;
            if (bits >= 64) {
                lo = hi;
                hi = 0;
            }
            if (D < VE) {  // (the row's last element stood in for those behind it)
                const int keep = D * (int)sizeof(T) * 8;
                lo &= keep >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << keep) - 1;
                hi &= keep > 64 ? ((uint64_t)1 << (keep - 64)) - 1 : 0;
            }
            v = make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
        }
        const bool there = in & (col < D);
        return make_uint4(there ? v.x : 0, there ? v.y : 0, there ? v.z : 0, there ? v.w : 0);
    }
};
