// Tiles of rows in LDS as operands of the matrix instructions, and operands that a lane computed.
#pragma once

#include "mlp_device.h"
#include "pieces.h"

typedef short short4_t __attribute__((ext_vector_type(4)));
#define ATTN_K 64      // rows of a tile that is walked through (keys; in the pass over the keys, queries)
constexpr float kLog2e = 1.4426950408889634f;

// No instruction moves across (left to itself the scheduler starts the reads of a whole tile at once, and two hundred registers hold them).
__device__ inline void phase() { __builtin_amdgcn_sched_barrier(0); }
// The lane, as a value that the compiler cannot know to be the same for the next tile: or it computes the addresses of all of a tile's
// accesses once, ahead of the loop, and keeps them in registers.
__device__ inline int lane_now() {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}

// A tile of ATTN_K rows of up to DP elements in LDS, rows 16 bytes apart beyond their length: reads of whole pieces along a row and transposed
// reads (16 x 16 elements bf16, single ones fp32) both touch every bank equally often.
template <typename T, int DP>
struct Tile {
    static constexpr int ES = sizeof(T), VE = 16 / ES, PITCH = DP * ES + 16, CPR = DP / VE, KS = DP * ES / 64, NB = DP / 16;
    static constexpr int TU = ES == 2 ? 32 : 16, NU = ATTN_K / TU;  // rows of one transposed operand, operands of a tile
    static constexpr int NX = TU / 16;                              // blocks of 16 of one
    static constexpr int NP = ES == 2 ? 3 : 1;                      // parts of a computed operand (see Computed)
    static constexpr int BYTES = ATTN_K * PITCH;
    // the lane's operand of rows row .. row + 15, contraction indices of piece ks along the row
    static __device__ inline uint4 rows(const unsigned char* lds, int row, int ks, int lane) {
        return *reinterpret_cast<const uint4*>(lds + (row + (lane & 15)) * PITCH + ks * 64 + (lane >> 4) * 16);
    }
    // columns 16 dt .. + 15 as the rows of an operand, contraction over the rows u TU .. : in the order in which a lane holds the products'
    // results (bf16: 4 g + r of two blocks of 16; fp32: of one)
    static __device__ inline uint4 turned(const unsigned char* lds, int u, int dt, int lane) {
        const int a = lane & 15, gr = lane >> 4;
        if constexpr (ES == 2) {
            typedef __attribute__((address_space(3))) short4_t lds_s4;
            const unsigned char* s = lds + (32 * u + 4 * gr + (a >> 2)) * PITCH + (16 * dt + 4 * (a & 3)) * 2;
            const uint2 u0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)s));
            const uint2 u1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(s + 16 * PITCH)));
            return make_uint4(u0.x, u0.y, u1.x, u1.y);
        } else {
            const unsigned char* s = lds + (16 * u + 4 * gr) * PITCH + (16 * dt + a) * 4;
            return make_uint4(*reinterpret_cast<const uint32_t*>(s), *reinterpret_cast<const uint32_t*>(s + PITCH),
                              *reinterpret_cast<const uint32_t*>(s + 2 * PITCH), *reinterpret_cast<const uint32_t*>(s + 3 * PITCH));
        }
    }
    static __device__ inline float at(const unsigned char* lds, int row, int d) {
        return to_f(*reinterpret_cast<const T*>(lds + row * PITCH + d * ES));
    }
};

// A lane's computed operand of four values a block: bf16 in two parts (off by 2^-18 of the value at most), so that the one rounding that counts is the
// output's (one part: y off by 2.0e-3 of its size instead of 1.6e-3; the second costs nothing that can be measured).  The forward of a training
// pass takes a third: delta comes of y, and what it is off by adds up in the bias's gradient, which is an fp32 sum.
template <typename T, int DP>
struct Computed {
    typedef Tile<T, DP> L;
    uint4 part[L::NP];
    __device__ inline void set(const float4_t (&p)[L::NX]) {
        if constexpr (L::ES == 2) {
            float v[8] = {p[0][0], p[0][1], p[0][2], p[0][3], p[1][0], p[1][1], p[1][2], p[1][3]};
#pragma unroll
            for (int q = 0; q < L::NP; ++q) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] = pack2(v[2 * i], v[2 * i + 1]);
                    v[2 * i] -= __uint_as_float(w[i] << 16);
                    v[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
                }
                part[q] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        } else {
            const float4_t a = p[0];
            part[0] = make_uint4(__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(a[2]), __float_as_uint(a[3]));
        }
    }
    template <bool FINE>
    __device__ inline void product(const uint4& turned, float4_t& acc) const {
#pragma unroll
        for (int i = 0; i < (FINE || L::NP < 3 ? L::NP : 2); ++i) Mma16<T>::run(turned, part[i], acc);
    }
};

