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

// Operands hold bf16 values; an fp32 one is the sum of three (split3), a product of two the six larger ones of nine products: fp32 results, at 96 cycles
// for 16 x 16 x 32 where the fp32 instructions take 256 (forward of a history of 4099 steps, 2 x 4 heads of 32, in one piece: 149 us, 175 on those).
// The five smaller products are summed apart and added at the end: a matrix instruction drops of what it adds what lies far below its
// accumulator, always to one side (all six in one accumulator: 11% faster, but the bias's gradient, a sum in which most cancels, off by 8.5e-7 instead
// of 2.4e-7; 129 environments, 67 of 101 steps, 6 heads of 40).
template <typename T>
struct Operand {
    static constexpr int N = sizeof(T) == 4 ? 3 : 1;
    uint4 p[N];
};
template <int N, int M>
__device__ inline void multiply(const uint4 (&a)[N], const uint4 (&b)[M], float4_t& acc) {
    if constexpr (N == 1) {  // the second operand in parts, or none
#pragma unroll
        for (int i = 0; i < M; ++i) Mma16<bf16_t>::run(a[0], b[i], acc);
    } else {
        float4_t low = {0.f, 0.f, 0.f, 0.f};
        Mma16<bf16_t>::run(a[0], b[2], low);
        Mma16<bf16_t>::run(a[2], b[0], low);
        Mma16<bf16_t>::run(a[1], b[1], low);
        Mma16<bf16_t>::run(a[0], b[1], low);
        Mma16<bf16_t>::run(a[1], b[0], low);
        Mma16<bf16_t>::run(a[0], b[0], acc);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[r] += low[r];
    }
}
// Eight elements of a row from element d on, as they are in memory
template <typename T, bool WHOLE>
struct RowOperand {
    RowPiece<T, WHOLE> u[sizeof(T) / 2];
    __device__ inline void load(const T* row, int d, int D) {
        u[0].load(row, d, D);
        if constexpr (sizeof(T) == 4) u[1].load(row, d + 4, D);
    }
    __device__ inline void values(int d, int D, bool in, float (&v)[8]) const {
        static_assert(sizeof(T) == 4, "");
        const uint4 a = u[0].get(d, D, in), b = u[sizeof(T) / 2 - 1].get(d + 4, D, in);
        v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
        v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
    }
    __device__ inline Operand<T> get(int d, int D, bool in = true) const {
        Operand<T> r;
        if constexpr (sizeof(T) == 2) {
            r.p[0] = u[0].get(d, D, in);
        } else {
            float v[8];
            values(d, D, in, v);
            split3<true>(v, r.p);
        }
        return r;
    }
};

// A tile of ATTN_K rows of up to DP values in LDS, a plane for each part, rows 16 bytes apart beyond their length: reads of whole pieces along a row and
// transposed reads of 16 x 16 values both touch every bank equally often.
template <typename T, int DP>
struct Tile {
    static constexpr int ES = sizeof(T), VE = 16 / ES, CPR = DP / VE;  // in memory: pieces of a row
    static constexpr int N = Operand<T>::N, PITCH = DP * 2 + 16, PLANE = ATTN_K * PITCH, BYTES = N * PLANE;
    static constexpr int KS = DP / 32, NB = DP / 16, TU = 32, NU = ATTN_K / TU, NX = TU / 16;  // rows of a transposed operand, operands of a tile, blocks of one
    static constexpr int OPITCH = DP * ES + 16;                                                // rows of results on their way out
    // the lane's operand of rows row .. row + 15, contraction over the values 32 ks .. of the rows
    static __device__ inline Operand<T> rows(const unsigned char* lds, int row, int ks, int lane) {
        Operand<T> r;
#pragma unroll
        for (int q = 0; q < N; ++q) r.p[q] = *reinterpret_cast<const uint4*>(lds + q * PLANE + (row + (lane & 15)) * PITCH + ks * 64 + (lane >> 4) * 16);
        return r;
    }
    // columns 16 dt .. + 15 as the rows of an operand, contraction over the rows 32 u .., in the order in which a lane holds the products' results
    // (4 g + r of two blocks of 16)
    static __device__ inline Operand<T> turned(const unsigned char* lds, int u, int dt, int lane) {
        typedef __attribute__((address_space(3))) short4_t lds_s4;
        const int a = lane & 15, gr = lane >> 4;
        Operand<T> r;
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const unsigned char* s = lds + q * PLANE + (32 * u + 4 * gr + (a >> 2)) * PITCH + (16 * dt + 4 * (a & 3)) * 2;
            const uint2 u0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)s));
            const uint2 u1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(s + 16 * PITCH)));
            r.p[q] = make_uint4(u0.x, u0.y, u1.x, u1.y);
        }
        return r;
    }
    // a piece from memory, columns col .. of a row
    static __device__ inline void put(unsigned char* lds, int row, int col, const uint4& u) {
        if constexpr (ES == 2) {
            *reinterpret_cast<uint4*>(lds + row * PITCH + col * 2) = u;
        } else {
            uint2 part[3];
            split3<true>(u, part);
#pragma unroll
            for (int q = 0; q < 3; ++q) *reinterpret_cast<uint2*>(lds + q * PLANE + row * PITCH + col * 2) = part[q];
        }
    }
};

// A lane's computed operand of four values a block.  For bf16 tensors in PARTS = 2 (off by 2^-18 of the value at most), so that the one rounding that
// counts is the output's (one part: y off by 2.0e-3 of its size instead of 1.6e-3; the second costs nothing that can be measured).  The forward of
// a training pass takes a third: delta comes of y, and what it is off by adds up in the bias's gradient, which is an fp32 sum.  fp32: three.
template <int PARTS>
struct Computed {
    uint4 p[PARTS];
    __device__ inline void set(const float4_t (&f)[2]) {
        float v[8] = {f[0][0], f[0][1], f[0][2], f[0][3], f[1][0], f[1][1], f[1][2], f[1][3]};
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = pack2(v[2 * i], v[2 * i + 1]);
                v[2 * i] -= __uint_as_float(w[i] << 16);
                v[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
            }
            p[q] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
};
