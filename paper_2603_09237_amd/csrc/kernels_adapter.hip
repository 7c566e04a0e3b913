// A shared projection with a low-rank adapter per preference, every row naming its own (the factors of Sec. III-B's
// W_l(p) = W0_l + A_l(p) B_l(p), applied without ever forming W_l(p)):
//
//   forward    u_m = B_p x_m,   y_m = W0 x_m + bias + A_p u_m                     p = index[m]
//   backward   v_m = A_p^T dy_m,  dx_m = W0^T dy_m + B_p^T v_m
//              dW0 = sum_m dy_m x_m^T,  dbias = sum_m dy_m,
//              dA_p = sum_{m of p} dy_m u_m^T,  dB_p = sum_{m of p} v_m x_m^T
//
// An index outside [0, n_adapters) is a row without an adapter.  u and v are fp32.  Rows may come in any order: the products
// with W0 take rows as they lie and add the adapters' part block by block of 32 rows, once for every adapter that a block
// holds; the gradients of the factors walk the rows sorted by adapter (k_ad_plan), pieces of at most AD_PIECE rows each, and
// what a piece leaves is added in order, so results repeat bit for bit.
#include "mlp_device.h"

typedef short short4_t __attribute__((ext_vector_type(4)));

#define AD_PIECE 256    // sorted rows of a factor-gradient workgroup

struct AdArgs {
    const void *x, *w0, *A, *B, *dy;
    const float* bias;
    const int32_t* index;
    void *y, *dx;
    float *dw0, *dbias, *dA, *dB;
    int64_t ld_x, ld_y;
    int M, I, O, r, P;
    // scratch
    float *u, *v;        // [M][rp]
    int32_t *seg, *perm; // [P + 2], [M]
    int32_t* table;      // [chunks][P + 1]: rows of each segment in a chunk, or NULL
    float *pw, *pA, *pB, *pb;  // partial sums: [split][O][I], [slot][O][r], [slot][r][I], [piece][O]
    const int32_t* order;  // perm where rows are taken sorted by adapter (u and v are then in that order), or NULL: as they lie
    int rp, split, kchunk, pieces, bf16, chunk, chunks;
    __device__ inline int row(int s) const { return order ? order[s] : s; }
    // adapter of the row at position s, or -1
    __device__ inline int adapter(int s) const {
        const int p = s < M ? index[row(s)] : -1;
        return p >= 0 && p < P ? p : -1;
    }
};

// sixteen consecutive values of a matrix row, of which the first `avail` exist (the others are zero): vector loads where VEC
// says that the row's address allows them
template <typename T>
__device__ inline void load16(const T* p, int avail, bool vec, uint4 (&v)[sizeof(T)]) {
    constexpr int VE = 16 / (int)sizeof(T);
#pragma unroll
    for (int q = 0; q < (int)sizeof(T); ++q) {
        v[q] = make_uint4(0, 0, 0, 0);
        if (vec && avail >= (q + 1) * VE) {
            v[q] = *reinterpret_cast<const uint4*>(p + q * VE);
        } else if (avail > q * VE) {
            T e[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) e[i] = q * VE + i < avail ? p[q * VE + i] : (T)0.f;
            v[q] = *reinterpret_cast<uint4*>(e);
        }
    }
}
// the bf16 parts of them: one (the values) or three (split3), 32 bytes each
template <bool BOUNDED = false>
__device__ inline void parts16(const uint4 (&v)[2], uint4 (&lo)[1], uint4 (&hi)[1]) { lo[0] = v[0]; hi[0] = v[1]; }
template <bool BOUNDED = false>
__device__ inline void parts16(const uint4 (&v)[4], uint4 (&lo)[3], uint4 (&hi)[3]) {
    uint2 p[4][3];
#pragma unroll
    for (int q = 0; q < 4; ++q) split3<BOUNDED>(v[q], p[q]);
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        lo[q] = make_uint4(p[0][q].x, p[0][q].y, p[1][q].x, p[1][q].y);
        hi[q] = make_uint4(p[2][q].x, p[2][q].y, p[3][q].x, p[3][q].y);
    }
}

// One operand of a tiled product: `rows` x `kdim`, element (row, k) at base[row * ld + k] (KC, contraction contiguous) or
// base[k * ld + row] (KS).  A stage is 128 rows x 32 k, in LDS as bf16 planes: KC [row][32 k], 80 bytes a row (the sixteen rows of
// a fragment read start in different groups of four banks); KS [k][128 rows], 320 bytes a k, read transposed.
enum { KC = 0, KS = 1 };
template <typename T, int KIND>
struct AdOperand {
    static constexpr int NP = sizeof(T) == 4 ? 3 : 1;
    static constexpr int PLANE = 10240;
    const T* base;
    int64_t ld;
    int rows, kdim;
    bool vec;
    const int32_t* order;  // KC: rows through it, or NULL
    uint4 reg[sizeof(T)];

    __device__ inline int64_t at(int row) const { return (order ? order[row] : row) * ld; }
    __device__ inline void init(const void* b, int64_t l, int r, int k) {
        base = reinterpret_cast<const T*>(b);
        ld = l; rows = r; kdim = k; order = nullptr;
        vec = ((reinterpret_cast<uintptr_t>(b) | (uintptr_t)(l * (int64_t)sizeof(T))) & 15) == 0;
    }
    __device__ inline float elem(int row, int k) const {
        if (row >= rows || k >= kdim) return 0.f;
        return to_f(base[KIND == KC ? at(row) + k : (int64_t)k * ld + row]);
    }
    __device__ inline void fetch(int t0, int k0) {
        const int tid = threadIdx.x;
        if (KIND == KC) {
            const int row = t0 + tid / 2, k = k0 + 16 * (tid % 2);
            load16(base + (row < rows ? at(row) : 0) + k, row < rows ? kdim - k : 0, vec, reg);
        } else {
            const int k = k0 + tid / 8, row = t0 + 16 * (tid % 8);
            load16(base + (int64_t)k * ld + row, k < kdim ? rows - row : 0, vec, reg);
        }
    }
    __device__ inline void put(unsigned char* lds) const {
        const int tid = threadIdx.x;
        uint4 lo[NP], hi[NP];
        parts16(reg, lo, hi);
        unsigned char* d = lds + (KIND == KC ? (tid / 2) * 80 + (tid % 2) * 32 : (tid / 8) * 320 + (tid % 8) * 32);
#pragma unroll
        for (int q = 0; q < NP; ++q) {
            *reinterpret_cast<uint4*>(d + q * PLANE) = lo[q];
            *reinterpret_cast<uint4*>(d + q * PLANE + 16) = hi[q];
        }
    }
    // the lane's operand of the 32-row block at `row`, contraction indices 16 ks + 8 lg + [0, 8)
    __device__ static inline void frag(const unsigned char* lds, int row, int ks, uint4 (&f)[NP]) {
        const int lane = threadIdx.x & 63, lr = lane & 31, lg = lane >> 5;
#pragma unroll
        for (int q = 0; q < NP; ++q) {
            if (KIND == KC) {
                f[q] = *reinterpret_cast<const uint4*>(lds + q * PLANE + (row + lr) * 80 + ks * 32 + lg * 16);
            } else {
                typedef __attribute__((address_space(3))) short4_t lds_s4;
                const int a = lane & 15, q0 = (lane >> 4) & 1, e = a >> 2, c = a & 3;
                const unsigned char* s = lds + q * PLANE + (16 * ks + 8 * lg + e) * 320 + (row + 16 * q0 + 4 * c) * 2;
                const uint2 u0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)s));
                const uint2 u1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(s + 4 * 320)));
                f[q] = make_uint4(u0.x, u0.y, u1.x, u1.y);
            }
        }
    }
};

// acc += a b^T for operands of one part, or of three each (six products, the five small ones into `low`)
__device__ inline void mma_parts(const uint4 (&a)[1], const uint4 (&b)[1], float16_t& acc, float16_t&) { Mma32<bf16_t>::run(a[0], b[0], acc); }
__device__ inline void mma_parts(const uint4 (&a)[3], const uint4 (&b)[3], float16_t& acc, float16_t& low) {
#pragma unroll
    for (int t = 0; t < 6; ++t) split_mma(t, a, b, acc, low);
}
__device__ inline float16_t zero16() {
    float16_t z;
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = 0.f;
    return z;
}

// Factor (n, j) of adapter p for output column n: forward A_p [O][r], backward B_p [r][I].
template <typename T, bool BWD>
struct AdFactor {
    const T* base;
    int N, r;
    __device__ inline const T* at(int p, int n, int j) const {
        return base + (int64_t)p * N * r + (BWD ? (int64_t)j * N + n : (int64_t)n * r + j);
    }
    // zero for j >= r; columns beyond the last one repeat it.  No branch goes by the lane: the loads of a block leave together
    __device__ inline T get(int p, int n, int j) const {
        const T v = *at(p, n < N ? n : N - 1, j < r ? j : 0);
        return j < r ? v : (T)0.f;
    }
    // eight j of column n (vec: r is a multiple of 8)
    __device__ inline uint4 frag(int p, int n, int j0, bool vec) const {
        if (!BWD && vec) {
            const uint4 u = *reinterpret_cast<const uint4*>(at(p, n < N ? n : N - 1, j0 < r ? j0 : 0));
            return j0 < r ? u : make_uint4(0, 0, 0, 0);
        }
        T e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = get(p, n, j0 + i);
        return *reinterpret_cast<uint4*>(e);
    }
};

// The adapters' part of a wave's 32 x 64 outputs, a lane holding row m0 + lr (accumulator: columns n0 + 8 (e / 4) + 4 lg + e % 4): one product
// of the block per adapter among its rows, which goes to its own rows' lanes only -- so an undefined factor of one adapter stays out of
// the others' rows, and these bits of a row do not depend on whose rows lie beside it.  The next adapter's factors are requested before
// this one's product (one after the other, 64 rows with an adapter each waited 32 times for memory: 116 us a launch of 64 x 2048 x 2048).
// bf16: u as two bf16 parts, the leading one cut, so that both have its sign, and the second never zero where u is not: an infinite factor's
// two products are then both what its product with u is.  What is left out is 2^-16 of u (rounding u to one part would double the error of y);
// fp32 on the fp32 instructions.
template <typename T, bool BWD, int RP>
struct AdExpand {
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int K16 = RP / 16, KF = RP / 2;
    AdFactor<T, BWD> F;
    bool vec;
    int kf;  // fp32: half the rank, rounded up; lane group lg takes values kf lg ..
    uint4 fb[BF ? 2 * K16 : 1];
    float ff[BF ? 1 : 2 * KF];
    __device__ inline void fetch(int p, int n0) {
        const int lane = threadIdx.x & 63, lr = lane & 31, lg = lane >> 5;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int n = n0 + 32 * b + lr;
            if constexpr (BF) {
#pragma unroll
                for (int s = 0; s < K16; ++s) fb[b * K16 + s] = F.frag(p, n, 16 * s + 8 * lg, vec);
            } else {
#pragma unroll
                for (int s = 0; s < KF; ++s)
                    if (s < kf) ff[b * KF + s] = to_f(F.get(p, n, kf * lg + s));
            }
        }
    }
    __device__ inline void run(const AdArgs& g, const float* u, int p, int m0, int n0, float16_t (&acc)[2]) {  // p: the lane's row's adapter
        const int lane = threadIdx.x & 63, lr = lane & 31, lg = lane >> 5, m = m0 + lr;
        uint64_t todo = __ballot(p >= 0) & 0xffffffffull;
        if (!todo) return;
        vec = (F.r & 7) == 0;
        kf = (F.r + 1) / 2;
        const float* um = u + (int64_t)(m < g.M ? m : g.M - 1) * RP;
        uint4 hi[BF ? K16 : 1], lo[BF ? K16 : 1];
        float uf[BF ? 1 : KF];
        if constexpr (BF) {
#pragma unroll
            for (int s = 0; s < K16; ++s) {
                const float4 a = *reinterpret_cast<const float4*>(um + 16 * s + 8 * lg), b = *reinterpret_cast<const float4*>(um + 16 * s + 8 * lg + 4);
                float t[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}, l[8];
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(__float_as_uint(t[2 * i + 1]), __float_as_uint(t[2 * i]), 0x07060302);
                hi[s] = make_uint4(w[0], w[1], w[2], w[3]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float d = t[i] - __uint_as_float(__float_as_uint(t[i]) & 0xffff0000u);
                    l[i] = __builtin_amdgcn_classf(d, 0x267) ? t[i] * 0x1p-20f : d;  // (zero, or t infinite or undefined)
                }
                lo[s] = pack_chunk<bf16_t>(l);
            }
        } else {
#pragma unroll
            for (int s = 0; s < KF; ++s)
                if (s < kf) uf[s] = um[kf * lg + s];
        }
        auto next = [&]() {
            const int q = __builtin_amdgcn_readlane(p, __ffsll((unsigned long long)todo) - 1);
            todo &= ~__ballot(p == q);
            return q;
        };
        int q = next();
        fetch(q, n0);
        for (;;) {
            AdExpand now = *this;
            const int mine = q;
            const bool more = todo != 0;
            if (more) {
                q = next();
                fetch(q, n0);
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                float16_t t = zero16();
                if constexpr (BF) {
#pragma unroll
                    for (int s = 0; s < K16; ++s) Mma32<bf16_t>::run(now.fb[b * K16 + s], lo[s], t);
#pragma unroll
                    for (int s = 0; s < K16; ++s) Mma32<bf16_t>::run(now.fb[b * K16 + s], hi[s], t);
                } else {
#pragma unroll
                    for (int s = 0; s < KF; ++s)
                        if (s < kf) t = __builtin_amdgcn_mfma_f32_32x32x2f32(now.ff[b * KF + s], uf[s], t, 0, 0, 0);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[b][e] += p == mine ? t[e] : 0.f;
            }
            if (!more) break;
        }
    }
};

// A wave's 32 x 64 outputs (row m0 + lr of lane lr) through a patch of LDS into whole row segments of C, rows through g.order for DX.
#define AD_PATCH (32 * 272)
template <typename T, bool GATHER>
__device__ inline void ad_store(const AdArgs& g, const float16_t (&acc)[2], unsigned char* patch, T* C, int64_t ldc, int M, int N, int m0, int n0, bool vec) {
    constexpr int VE = 16 / (int)sizeof(T), PITCH = 64 * (int)sizeof(T) + 16, CH = 64 / VE;
    const int lane = threadIdx.x & 63, lr = lane & 31, lg = lane >> 5;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4) {
            unsigned char* d = patch + lr * PITCH + (32 * b + 8 * g4 + 4 * lg) * (int)sizeof(T);
            if (sizeof(T) == 2)
                *reinterpret_cast<uint2*>(d) = make_uint2(pack2(acc[b][4 * g4], acc[b][4 * g4 + 1]), pack2(acc[b][4 * g4 + 2], acc[b][4 * g4 + 3]));
            else
                *reinterpret_cast<float4*>(d) = make_float4(acc[b][4 * g4], acc[b][4 * g4 + 1], acc[b][4 * g4 + 2], acc[b][4 * g4 + 3]);
        }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 32 * CH / 64; ++i) {
        const int pos = 64 * i + lane, row = pos / CH, n = n0 + (pos % CH) * VE;
        const uint4 v = *reinterpret_cast<const uint4*>(patch + row * PITCH + (pos % CH) * 16);
        if (m0 + row < M && n < N) {
            T* d = C + (int64_t)(GATHER ? g.row(m0 + row) : m0 + row) * ldc + n;
            if (vec && n + VE <= N) {
                *reinterpret_cast<uint4*>(d) = v;
            } else {
                T e[VE];
                *reinterpret_cast<uint4*>(e) = v;
#pragma unroll
                for (int k = 0; k < VE; ++k)
                    if (n + k < N) d[k] = e[k];
            }
        }
    }
    __builtin_amdgcn_wave_barrier();
}
static __device__ inline bool ad_vec(const void* p, int64_t ld, int size) {
    return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size)) & 15) == 0;
}
// The three products with or of W0, on 128 x 128 tiles of four waves of 64 x 64: any size, stride and alignment.  fp32 as three bf16 parts
// a value (split3: what the six products leave out is below 2^-24 of the largest term), two thirds of the fp32 instructions' cycles; the
// split's arithmetic and the waits for registers on their way to LDS bound it (dW of 584 x 256 over 2051 rows: 15 us).
enum { AD_FWD = 0, AD_DX = 1, AD_DW = 2 };
template <int ROLE> struct AdRole;
template <> struct AdRole<AD_FWD> { static constexpr int KA = KC, KB = KC; };
template <> struct AdRole<AD_DX> { static constexpr int KA = KC, KB = KS; };
template <> struct AdRole<AD_DW> { static constexpr int KA = KS, KB = KS; };

// what a wave does with its 32 x 64 sums
template <typename T, int ROLE, int RP>
__device__ inline void ad_finish(const AdArgs& g, float16_t (&acc)[2], unsigned char* patch, int p, int range, int m0, int n0) {
    const int lg = (threadIdx.x >> 5) & 1;
    if constexpr (ROLE == AD_FWD) {
        if (g.bias) {
            asm volatile("" : "+v"(n0));  // (its values are read again for the next rows: held, they would cost the product its registers)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int n = n0 + 32 * j + 8 * (e / 4) + 4 * lg + e % 4;
                    acc[j][e] += g.bias[n < g.O ? n : g.O - 1];
                }
        }
        AdExpand<T, false, RP> x;
        x.F = {reinterpret_cast<const T*>(g.A), g.O, g.r};
        x.run(g, g.u, p, m0, n0, acc);
        ad_store<T, false>(g, acc, patch, reinterpret_cast<T*>(g.y), g.ld_y, g.M, g.O, m0, n0, ad_vec(g.y, g.ld_y, sizeof(T)));
    } else if constexpr (ROLE == AD_DX) {
        AdExpand<T, true, RP> x;
        x.F = {reinterpret_cast<const T*>(g.B), g.I, g.r};
        x.run(g, g.v, p, m0, n0, acc);
        ad_store<T, true>(g, acc, patch, reinterpret_cast<T*>(g.dx), g.ld_x, g.M, g.I, m0, n0, ad_vec(g.dx, g.ld_x, sizeof(T)));
    } else {
        float* C = g.split > 1 ? g.pw + (int64_t)range * g.O * g.I : g.dw0;
        ad_store<float, false>(g, acc, patch, C, g.I, g.O, g.I, m0, n0, (g.I & 3) == 0);
    }
}

template <typename T, int ROLE, int RP>
__global__ __launch_bounds__(256, 2) void k_ad_gemm(AdArgs g) {
    constexpr int KA = AdRole<ROLE>::KA, KB = AdRole<ROLE>::KB;
    typedef AdOperand<T, KA> OpA;
    typedef AdOperand<T, KB> OpB;
    constexpr int NP = OpA::NP;
    __shared__ __align__(16) unsigned char lds[(2 * NP * OpA::PLANE > 4 * AD_PATCH) ? 2 * NP * OpA::PLANE : 4 * AD_PATCH];
    const int wave = threadIdx.x >> 6, lr = threadIdx.x & 31;
    const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
    const int tiles_n = ((ROLE == AD_FWD ? g.O : g.I) + 127) / 128;
    const int tile = blockIdx.x;
    const int tm = (tile / tiles_n) * 128, tn = (tile % tiles_n) * 128;
    OpA a;
    OpB b;
    int kdim;
    if (ROLE == AD_FWD) {
        kdim = g.I;
        a.init(g.x, g.ld_x, g.M, kdim);
        b.init(g.w0, g.I, g.O, kdim);
    } else if (ROLE == AD_DX) {
        kdim = g.O;
        a.init(g.dy, g.ld_y, g.M, kdim);
        a.order = g.order;
        b.init(g.w0, g.I, g.I, kdim);
    } else {
        const int k0 = blockIdx.y * g.kchunk;
        kdim = g.M - k0 < g.kchunk ? g.M - k0 : g.kchunk;
        if (kdim < 0) kdim = 0;
        a.init(reinterpret_cast<const T*>(g.dy) + (int64_t)k0 * g.ld_y, g.ld_y, g.O, kdim);
        b.init(reinterpret_cast<const T*>(g.x) + (int64_t)k0 * g.ld_x, g.ld_x, g.I, kdim);
    }
    unsigned char* lb = lds + NP * OpA::PLANE;
    float16_t acc[2][2], low[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = low[i][j] = zero16();
    if (kdim > 0) {
        a.fetch(tm, 0);
        b.fetch(tn, 0);
    }
    for (int k = 0; k < kdim; k += 32) {
        a.put(lds);
        b.put(lb);
        __syncthreads();
        if (k + 32 < kdim) {
            a.fetch(tm, k + 32);
            b.fetch(tn, k + 32);
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            uint4 fa[2][NP], fb[2][NP];
#pragma unroll
            for (int i = 0; i < 2; ++i) OpA::frag(lds, wm + 32 * i, ks, fa[i]);
#pragma unroll
            for (int j = 0; j < 2; ++j) OpB::frag(lb, wn + 32 * j, ks, fb[j]);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) mma_parts(fb[j], fa[i], acc[i][j], low[i][j]);
        }
        __syncthreads();
    }
    if (NP == 3) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] += low[i][j][e];
                if (any_undefined(acc[i][j])) {  // those sums again on the fp32 instructions, from memory; the others stay as they are
                    const int lg = (threadIdx.x >> 5) & 1;
                    float16_t t = zero16();
#pragma unroll 1
                    for (int k = 0; k < kdim; k += 2)
                        t = __builtin_amdgcn_mfma_f32_32x32x2f32(b.elem(tn + wn + 32 * j + lr, k + lg), a.elem(tm + wm + 32 * i + lr, k + lg), t, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (!(__builtin_fabsf(acc[i][j][e]) < __builtin_inff())) acc[i][j][e] = t[e];
                }
            }
    }
    unsigned char* patch = lds + wave * AD_PATCH;
#pragma unroll
    for (int i = 0; i < 2; ++i) ad_finish<T, ROLE, RP>(g, acc[i], patch, ROLE == AD_DW ? 0 : g.adapter(tm + wm + 32 * i + lr), blockIdx.y, tm + wm + 32 * i, tn + wn);
}

// ---- bf16 operands whose rows are whole 16-byte pieces: direct-to-LDS loads, three stages of 32 contraction indices -------------------
// Tiles of 64 MB x 128, four waves of 32 MB x 64.  A stage's pieces lie as the loads leave them, one KB an instruction; which piece a lane
// fetches is free, and the bank swizzle is there: KC, piece (row, c) of four a row at position 4 row + (c ^ row's bits 2, 3); KS, piece
// (k, c) of ROWS / 8 a contraction index at (ROWS / 8) k + (c ^ 4 (k mod 4)), read transposed.  A contraction that is no multiple of 32
// begins with the rest of it, loaded through registers.  Half a stage's products run while the other half's operands and the loads of the third
// next stage are issued between them, with no branch in the loop.
// 16384 x 512 x 1160, 20.3 GFLOP: 40 us, 0.5 PFLOP/s; dX and dW of 32768 x 512 x 1160, 39 GFLOP each: 62 and 61 us, 0.63 PFLOP/s.  Bound by the
// loads: without the matrix instructions 37 of 40 and 55 of 62 us are left (rows of 64 bytes a request keep the L2 busy), without the loads 30
// and 44; the last tiles' outputs, which nothing overlaps, take 10.  Tiles of 256 x 256 at a wave a SIMD took 67 and 57 (and 5 more to add up).
template <int KIND, int ROWS>
struct AdTile {
    static constexpr int NI = ROWS / 16 / 4, CPR = ROWS / 8, BYTES = ROWS * 64;
    const char* base;
    uint32_t voff[NI];
    int64_t kstep;
    __device__ inline void init(const void* b, int64_t ld, int rows, int t0, const int32_t* order) {
        base = reinterpret_cast<const char*>(b);
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int j = NI * wave + i;
            if (KIND == KC) {
                const int row = 16 * j + lane / 4, c = (lane % 4) ^ ((row >> 2) & 3);
                int r = t0 + row < rows ? t0 + row : rows - 1;
                if (order) r = order[r];
                voff[i] = (uint32_t)r * (uint32_t)(ld * 2) + 16 * c;
            } else {
                const int pos = 64 * j + lane, k = pos / CPR, c = (pos % CPR) ^ (4 * (k & 3));
                const int r = t0 + 8 * c < rows - 8 ? t0 + 8 * c : rows - 8;
                voff[i] = (uint32_t)k * (uint32_t)(ld * 2) + (uint32_t)r * 2;
            }
        }
        kstep = KIND == KC ? 64 : 64 * ld;
    }
    __device__ inline void issue(int i, int64_t from, uint32_t tile) const {  // from: bytes along the contraction
        const int wave = threadIdx.x >> 6;
        dma16(base + from, voff[i], __builtin_amdgcn_readfirstlane(tile + (uint32_t)(NI * wave + i) * 1024u));
    }
    // the first `rest` (a multiple of 8 for KC) contraction indices, zeros behind them
    __device__ inline void put_rest(int rest, unsigned char* tile) const {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int j = NI * wave + i;
            const int k = KIND == KC ? 8 * ((lane % 4) ^ (((16 * j + lane / 4) >> 2) & 3)) : (64 * j + lane) / CPR;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (k < rest) v = *reinterpret_cast<const uint4*>(base + voff[i]);
            *reinterpret_cast<uint4*>(tile + j * 1024 + lane * 16) = v;
        }
    }
    __device__ static inline uint4 frag(const unsigned char* tile, int row0, int ks) {
        const int lane = threadIdx.x & 63, lr = lane & 31, lg = lane >> 5;
        if (KIND == KC) {
            const int row = row0 + lr;
            return *reinterpret_cast<const uint4*>(tile + row * 64 + (((2 * ks + lg) ^ ((row >> 2) & 3)) * 16));
        } else {
            typedef __attribute__((address_space(3))) short4_t lds_s4;
            const int a = lane & 15, q0 = (lane >> 4) & 1, e = a >> 2, c = a & 3, col = row0 + 16 * q0 + 4 * c, k = 16 * ks + 8 * lg + e;
            const unsigned char* s = tile + (k * CPR + ((col >> 3) ^ (4 * (k & 3)))) * 16 + ((col >> 2) & 1) * 8;
            const uint2 u0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)s));
            const uint2 u1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(s + 4 * CPR * 16)));
            return make_uint4(u0.x, u0.y, u1.x, u1.y);
        }
    }
};
template <int MB, int NB> struct AdDma {
    static constexpr int STAGE = 64 * (MB + NB) * 64, LDS = 3 * STAGE > 4 * AD_PATCH ? 3 * STAGE : 4 * AD_PATCH, LOADS = MB + NB;
};

template <int ROLE, int MB, int NB, int RP>
__global__ __launch_bounds__(256, MB == 2 ? 3 : 2) void k_ad_gemm_dma(AdArgs g) {
    constexpr int KA = AdRole<ROLE>::KA, KB = AdRole<ROLE>::KB, TM = 64 * MB, TN = 64 * NB;
    typedef AdTile<KA, TM> TA;
    typedef AdTile<KB, TN> TB;
    typedef AdDma<MB, NB> S;
    __shared__ __align__(16) unsigned char lds[S::LDS];
    const int wave = threadIdx.x >> 6;
    const int wm = (wave >> 1) * 32 * MB, wn = (wave & 1) * 32 * NB;
    const int rows_a = ROLE == AD_DW ? g.O : g.M, rows_b = ROLE == AD_FWD ? g.O : g.I;
    // consecutive workgroups of an XCD: the tiles of one range of the contraction, or of the same rows
    const int tiles_n = (rows_b + TN - 1) / TN, id = xcd_remap(blockIdx.x, gridDim.x);
    const int tiles = ROLE == AD_DW ? ((rows_a + TM - 1) / TM) * tiles_n : gridDim.x, tile = id % tiles, range = id / tiles;
    const int tm = (tile / tiles_n) * TM, tn = (tile % tiles_n) * TN;
    TA a;
    TB b;
    int kdim;
    if (ROLE == AD_FWD) {
        kdim = g.I;
        a.init(g.x, g.ld_x, rows_a, tm, nullptr);
        b.init(g.w0, g.I, rows_b, tn, nullptr);
    } else if (ROLE == AD_DX) {
        kdim = g.O;
        a.init(g.dy, g.ld_y, rows_a, tm, g.order);
        b.init(g.w0, g.I, rows_b, tn, nullptr);
    } else {
        const int k0 = range * g.kchunk;
        kdim = g.M - k0 < g.kchunk ? g.M - k0 : g.kchunk;
        a.init(reinterpret_cast<const bf16_t*>(g.dy) + (int64_t)k0 * g.ld_y, g.ld_y, rows_a, tm, nullptr);
        b.init(reinterpret_cast<const bf16_t*>(g.x) + (int64_t)k0 * g.ld_x, g.ld_x, rows_b, tn, nullptr);
    }
    int owner[MB];  // the adapters of the wave's rows
#pragma unroll
    for (int i = 0; i < MB; ++i) owner[i] = ROLE == AD_DW ? 0 : g.adapter(tm + wm + 32 * i + (threadIdx.x & 31));
    const uint32_t lbase = (uint32_t)(size_t)lds;
    const int rest = kdim & 31, steps = (kdim + 31) / 32, shift = rest ? 1 : 0;
    const int64_t skip_a = KA == KC ? 2 * rest : a.kstep / 32 * rest, skip_b = KB == KC ? 2 * rest : b.kstep / 32 * rest;
    auto issue_one = [&](int from, int s, int i) {
        const uint32_t to = lbase + (uint32_t)(s % 3) * S::STAGE;
        const int64_t d = from - shift;
        if (i < MB) a.issue(i, skip_a + d * a.kstep, to);
        else b.issue(i - MB, skip_b + d * b.kstep, to + TA::BYTES);
    };
    auto issue = [&](int from, int s) {
#pragma unroll
        for (int i = 0; i < MB + NB; ++i) issue_one(from, s, i);
    };
    if (rest) {
        a.put_rest(rest, lds);
        b.put_rest(rest, lds + TA::BYTES);
    } else {
        issue(0, 0);
    }
    // Behind the last stage it is requested again: the loop has no branch, and as many loads are on their way at every wait.  (A range of fewer
    // than 32 indices has its rest alone.)
    const bool full = ROLE != AD_DW || kdim >= 32;
    if (full)
        for (int s = 1; s < 3; ++s) issue(s < steps ? s : steps - 1, s);
    float16_t acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = zero16();
    uint4 fa[2][MB], fb[2][NB];
    auto load_one = [&](int s, int ks, int f) {
        const unsigned char *ta = lds + (s % 3) * S::STAGE, *tb = ta + TA::BYTES;
        if (f < NB) fb[ks][f] = TB::frag(tb, wn + 32 * f, ks);
        else fa[ks][f - NB] = TA::frag(ta, wm + 32 * (f - NB), ks);
    };
    // the products of half a stage, `PIECES` pieces of other work between them, two or more behind each
    auto products = [&](int ks, auto pieces, auto piece) {
        constexpr int Q = MB * NB, PIECES = decltype(pieces)::value, EACH = (PIECES + Q - 1) / Q < 2 ? 2 : (PIECES + Q - 1) / Q;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            Mma32<bf16_t>::run(fb[ks][q % NB], fa[ks][q / NB], acc[q / NB][q % NB]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int e = 0; e < EACH; ++e)
                if (q * EACH + e < PIECES) piece(q * EACH + e);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    constexpr int F = MB + NB;
    wait_vm<2 * S::LOADS>();
    __syncthreads();
#pragma unroll
    for (int f = 0; f < F; ++f) load_one(0, 0, f);
    if (!full) {
#pragma unroll
        for (int f = 0; f < F; ++f) load_one(0, 1, f);
        products(0, std::integral_constant<int, 0>{}, [](int) {});
        products(1, std::integral_constant<int, 0>{}, [](int) {});
    }
    for (int s = 0; full && s < steps; ++s) {
        products(0, std::integral_constant<int, F>{}, [&](int f) { load_one(s, 1, f); });
        wait_vm<S::LOADS>();
        __syncthreads();  // stage s is in registers, stage s + 1 complete
        const int from = s + 3 < steps ? s + 3 : steps - 1;
        products(1, std::integral_constant<int, 2 * F>{}, [&](int f) {
            if (f < F) load_one(s + 1, 0, f);
            else issue_one(from, s + 3, f - F);
        });
    }
    wait_vm<0>();
    __syncthreads();
    unsigned char* patch = lds + wave * AD_PATCH;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; j += 2) ad_finish<bf16_t, ROLE, RP>(g, *reinterpret_cast<float16_t(*)[2]>(&acc[i][j]), patch, owner[i], range, tm + wm + 32 * i, tn + wn + 32 * j);
}

// ---- few rows: every workgroup sixteen columns of the output for 32 rows, its eight waves sharing the contraction --------------------
// Bound by the latency of its few loads and the stream of W0, each row of which is read once; operands go straight into registers, 16
// bytes a lane, and the waves' sums meet in LDS, where the adapters' part joins them in fp32: with so few rows each may have its own.
// Sixteen bytes of a row of K values from k on, zero where it ends or `on` is false: one access where whole pieces make up the row (WHOLE;
// with the alignment of one element only), else one a value; no branch goes by the lane.
template <bool WHOLE, typename T>
__device__ inline uint4 ad_piece(const T* row, int k, int K, bool on) {
    constexpr int VE = 16 / (int)sizeof(T);
    typedef T vec_t __attribute__((ext_vector_type(VE), aligned(sizeof(T))));
    if constexpr (WHOLE) {
        const bool have = on && k < K;
        const uint4 u = __builtin_bit_cast(uint4, *reinterpret_cast<const vec_t*>(row + (have ? k : 0)));
        return make_uint4(have ? u.x : 0, have ? u.y : 0, have ? u.z : 0, have ? u.w : 0);
    }
    T e[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) {
        const bool have = on && k + i < K;
        const T v = row[have ? k + i : 0];
        e[i] = have ? v : (T)0.f;
    }
    return *reinterpret_cast<uint4*>(e);
}
template <typename T>
__device__ inline uint4 ad_piece_of(bool whole, const T* row, int k, int K, bool on) {
    return whole ? ad_piece<true>(row, k, K, on) : ad_piece<false>(row, k, K, on);
}
// the same of a column: values `stride` apart
template <typename T>
__device__ inline uint4 ad_column(const T* col, int64_t stride, int k, int K) {
    constexpr int VE = 16 / (int)sizeof(T);
    T e[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) {
        const T v = col[(int64_t)(k + i < K ? k + i : 0) * stride];
        e[i] = k + i < K ? v : (T)0.f;
    }
    return *reinterpret_cast<uint4*>(e);
}
// A workgroup has 16 columns x 32 rows, an output a thread; rows beyond the last one repeat it.  64 rows x 2048 x 2048 bf16 with an adapter each:
// 9 us; 4099 x 27 x 523 fp32: 25 us, where a value of a row of 27 is a load of its own.
template <typename T, bool BWD, int RP, bool WHOLE>
__global__ __launch_bounds__(512) void k_ad_few(AdArgs g) {
    constexpr int VE = 16 / (int)sizeof(T), STEP = 4 * VE, U = BWD ? 2 : 4;  // contraction indices of a step; steps requested together
    __shared__ float red[8][32][17];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, l16 = lane & 15, kg = lane >> 4;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 32;
    const int K = BWD ? g.O : g.I, N = BWD ? g.I : g.O;
    const int64_t ld = BWD ? g.ld_y : g.ld_x;
    const T *src = reinterpret_cast<const T*>(BWD ? g.dy : g.x), *w0 = reinterpret_cast<const T*>(g.w0);
    const int m = m0 + (int)threadIdx.x / 16, c = n0 + (int)threadIdx.x % 16, cc = c < N ? c : N - 1;
    const int adapter = g.adapter(m);
    const int n = n0 + l16 < N ? n0 + l16 : N - 1;
    const T* wrow = w0 + (BWD ? (int64_t)n : (int64_t)n * g.I);
    const T* xrow[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = m0 + 16 * i + l16;
        xrow[i] = src + (int64_t)g.row(r < g.M ? r : g.M - 1) * ld;
    }
    float4_t acc[2] = {};
    auto steps = [&](auto count, int k) {
        constexpr int C = decltype(count)::value;
        uint4 fw[C], fx[C][2];
#pragma unroll
        for (int s = 0; s < C; ++s) {
            const int kk = k + 8 * STEP * s + VE * kg;
            fw[s] = BWD ? ad_column(wrow, g.I, kk, K) : ad_piece<WHOLE>(wrow, kk, K, true);
#pragma unroll
            for (int i = 0; i < 2; ++i) fx[s][i] = ad_piece<WHOLE>(xrow[i], kk, K, true);
        }
#pragma unroll
        for (int s = 0; s < C; ++s)
#pragma unroll
            for (int i = 0; i < 2; ++i) Mma16<T>::run(fw[s], fx[s][i], acc[i]);
    };
    int k = wave * STEP;
    for (; k + 8 * STEP * (U - 1) < K; k += 8 * STEP * U) steps(std::integral_constant<int, U>{}, k);
    for (; k < K; k += 8 * STEP) steps(std::integral_constant<int, 1>{}, k);
    // the adapter's part
    const AdFactor<T, BWD> F = {reinterpret_cast<const T*>(BWD ? g.B : g.A), N, g.r};
    const T* fp = F.at(adapter < 0 ? 0 : adapter, cc, 0);
    uint4 f[RP / VE];
#pragma unroll
    for (int j = 0; j < RP / VE; ++j) f[j] = BWD ? ad_column(fp, N, j * VE, g.r) : ad_piece_of(g.r % VE == 0, fp, j * VE, g.r, true);
    const float4* um = reinterpret_cast<const float4*>((BWD ? g.v : g.u) + (int64_t)(m < g.M ? m : g.M - 1) * g.rp);
    float4 uv[RP / 4];
#pragma unroll
    for (int j = 0; j < RP / 4; ++j) uv[j] = um[j];
    const float bias = !BWD && g.bias ? g.bias[cc] : 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) red[wave][16 * i + l16][4 * kg + e] = acc[i][e];
    __syncthreads();
    float s = 0.f, t = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) s += red[q][threadIdx.x / 16][threadIdx.x % 16];
    s += bias;
#pragma unroll
    for (int j = 0; j < RP; ++j) {
        const float4 q = uv[j / 4];
        const T* e = reinterpret_cast<const T*>(&f[j / VE]);
        t += (j % 4 == 0 ? q.x : j % 4 == 1 ? q.y : j % 4 == 2 ? q.z : q.w) * to_f(e[j % VE]);
    }
    if (adapter >= 0) s += t;
    if (m < g.M && c < N) {
        if (BWD) reinterpret_cast<T*>(g.dx)[(int64_t)g.row(m) * g.ld_x + c] = cvt<T>(s);
        else reinterpret_cast<T*>(g.y)[(int64_t)m * g.ld_y + c] = cvt<T>(s);
    }
}

// ---- u (or v): the rows' products with their adapters' short factor ------------------------------------------------------------------
// A thread's part of row position m's: WPR waves (four, or one) share the contraction, a factor's values are used once.
template <typename T, bool BWD, int RP, int WPR, bool WHOLE>
__device__ inline void shrink_row(const AdArgs& g, int m, int p, int tid, float (&acc)[RP]) {
    constexpr int VE = 16 / (int)sizeof(T);
    const int K = BWD ? g.O : g.I;
    const T* row = reinterpret_cast<const T*>(BWD ? g.dy : g.x) + (int64_t)g.row(m) * (BWD ? g.ld_y : g.ld_x);
#pragma unroll
    for (int j = 0; j < RP; ++j) acc[j] = 0.f;
    if (p < 0) return;
    {
        const T* f = reinterpret_cast<const T*>(BWD ? g.A : g.B) + (int64_t)p * K * g.r;
        if (BWD) {  // A_p [O][r]: a thread's rows of it, two requested together
            for (int k = tid; k < K; k += 2 * 64 * WPR) {
                float v[2];
                uint4 q[2][RP / VE];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int kk = k + 64 * WPR * u < K ? k + 64 * WPR * u : k;
                    v[u] = to_f(row[kk]);
#pragma unroll
                    for (int j = 0; j < RP / VE; ++j) q[u][j] = ad_piece<WHOLE>(f + (int64_t)kk * g.r, j * VE, g.r, true);
                }
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int j = 0; j < RP; ++j)
                        acc[j] += j < g.r && k + 64 * WPR * u < K ? v[u] * to_f(reinterpret_cast<const T*>(&q[u][j / VE])[j % VE]) : 0.f;
            }
        } else if constexpr (!WHOLE) {  // B_p [r][I], rows that end inside a piece: a value a lane
            for (int k = tid; k < K; k += 64 * WPR) {
                T q[RP];
                const T xv = row[k];
#pragma unroll
                for (int j = 0; j < RP; ++j) q[j] = f[(int64_t)(j < g.r ? j : 0) * K + k];
#pragma unroll
                for (int j = 0; j < RP; ++j) acc[j] += j < g.r ? to_f(xv) * to_f(q[j]) : 0.f;
            }
        } else {  // B_p [r][I]
            for (int k = tid * VE; k < K; k += 64 * WPR * VE) {
                uint4 q[RP];
                const uint4 xq = ad_piece<true>(row, k, K, true);
#pragma unroll
                for (int j = 0; j < RP; ++j) q[j] = ad_piece<true>(f + (int64_t)(j < g.r ? j : 0) * K, k, K, true);
#pragma unroll
                for (int j = 0; j < RP; ++j)
#pragma unroll
                    for (int i = 0; i < VE; ++i)
                        acc[j] += j < g.r ? to_f(reinterpret_cast<const T*>(&xq)[i]) * to_f(reinterpret_cast<const T*>(&q[j])[i]) : 0.f;
            }
        }
    }
}
// their sums over the wave: of RP values, a lane keeps fewer and fewer (bits 5, 4, .. of the lane select the halves of j); value
// lane / (64 / RP) is returned
template <int RP>
__device__ inline float shrink_sum(float (&acc)[RP]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int h = RP / 2, o = 32; h >= 1; h /= 2, o /= 2)
#pragma unroll
        for (int j = 0; j < h; ++j) {
            const bool up = lane & o;
            const float give = up ? acc[j] : acc[j + h];
            acc[j] = (up ? acc[j + h] : acc[j]) + __shfl_xor(give, o);
        }
    float s = acc[0];
#pragma unroll
    for (int o = 64 / RP / 2; o >= 1; o /= 2) s += __shfl_xor(s, o);
    return s;
}
// Few rows, or small factors: WPR waves a row.  Latency: index, row and factor one after the other; 64 rows x 2048 bf16 8 us, 2051 x 584 fp32 of
// rank 8 backward 8 us.
template <typename T, bool BWD, int RP, int WPR, bool WHOLE>
__global__ __launch_bounds__(256) void k_ad_shrink_row(AdArgs g) {
    __shared__ float part[4][RP];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int m = WPR == 4 ? blockIdx.x : blockIdx.x * 4 + wave;
    if (WPR == 1 && m >= g.M) return;
    const int p = __builtin_amdgcn_readfirstlane(g.adapter(m));
    float acc[RP];
    shrink_row<T, BWD, RP, WPR, WHOLE>(g, m, p, WPR == 4 ? threadIdx.x : lane, acc);
    const float s = shrink_sum<RP>(acc);
    float* out = (BWD ? g.v : g.u) + (int64_t)m * g.rp;
    const int j = lane / (64 / RP);
    if (RP == 8 && threadIdx.x % (64 * WPR) >= 8 && threadIdx.x % (64 * WPR) < 16) out[threadIdx.x % (64 * WPR)] = 0.f;  // (g.rp is 16)
    if (WPR == 1) {
        if (lane % (64 / RP) == 0) out[j] = j < g.r && p >= 0 ? s : 0.f;
        return;
    }
    if (lane % (64 / RP) == 0) part[wave][j] = s;
    __syncthreads();
    if (threadIdx.x < RP) {
        const int i = threadIdx.x;
        out[i] = i < g.r && p >= 0 ? part[0][i] + part[1][i] + part[2][i] + part[3][i] : 0.f;
    }
}

// acc += F^T x for the contraction indices [k0, k1) of a wave (k0 a multiple of 64), 64 at a time, the next ones on their way.  A load takes
// whole lines, eight lanes 128 bytes of a row (rows 8 i + lane / 8 for i = 0 .. 3), and the rows reach their lanes through LDS (`stage`, 32
// rows x 64, piece c of a row at c ^ (row mod 8)).  Backward: A [K][r], r a multiple of 8, sixty-four rows of it turned in `turn`; forward:
// B [r][K], a row a lane.
template <bool BWD>
__device__ inline void shrink_staged(const bf16_t* f, const bf16_t* const (&rows)[4], int K, int r, int k0, int k1, bf16_t* stage, bf16_t* turn,
                                     float16_t& acc) {
    const int lane = threadIdx.x & 63, lr = lane & 31, lg = lane >> 5, a = lane & 15, q0 = (lane >> 4) & 1, e = a >> 2, c = a & 3, pieces = r / 8;
    uint4 fq[4], xq[4];
    auto fetch = [&](int k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) xq[i] = ad_piece<true>(rows[i], k + 8 * (lane & 7), K, true);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (BWD) {
                if (q < pieces) fq[q] = ad_piece<true>(f, k * r + 8 * (lane + 64 * q), K * r, true);
            } else {
                fq[q] = ad_piece<true>(f + (int64_t)(lr < r ? lr : 0) * K, k + 32 * lg + 8 * q, K, lr < r);
            }
        }
    };
    if (k0 < k1) fetch(k0);
    for (int k = k0; k < k1; k += 64) {
        uint4 fs[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint4*>(stage + (8 * i + lane / 8) * 64 + ((lane ^ lane / 8) & 7) * 8) = xq[i];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (BWD) {
                if (q < pieces) {
                    const int at = lane + 64 * q;
                    *reinterpret_cast<uint4*>(turn + at / pieces * 32 + at % pieces * 8) = fq[q];
                }
            } else {
                fs[q] = fq[q];
            }
        }
        __builtin_amdgcn_wave_barrier();
        if (k + 64 < k1) fetch(k + 64);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if constexpr (BWD) {
                typedef __attribute__((address_space(3))) short4_t lds_s4;
                const bf16_t* p = turn + (32 * lg + 8 * s + e) * 32 + 16 * q0 + 4 * c;
                const uint2 u0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)p));
                const uint2 u1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(p + 4 * 32)));
                fs[s] = make_uint4(u0.x, u0.y, u1.x, u1.y);
            }
            const uint4 x = *reinterpret_cast<const uint4*>(stage + lr * 64 + (((4 * lg + s) ^ lr) & 7) * 8);
            Mma32<bf16_t>::run(fs[s], x, acc);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// adapters among 32 rows beyond which these are taken one by one.  us of the forward, rows mixed: 2048 x 1160 x 1160 fp32 of 8 adapters 146
// one by one, 292 adapter by adapter; 16384 x 512 x 1160 bf16 of 128 142 and 162; of 4 adapters 57 and 56 (above four are one by one).  The two
// add up a row's products in different orders: its u has other last bits among other rows, which the header says.  One order for both costs more
// than it gives: fp32 one by one throughout 237 -> 263 for 16384 x 512 x 1160 grouped, and 78 -> 207 for 8192 x 512 x 512 of rank 32.
#define AD_ONE_BY_ONE 4
// Many rows: 32 a workgroup, its four waves a quarter of the contraction each, one pass over the rows per adapter among them.  bf16 on
// 32x32x16, fp32 on 32x32x2 (the factor's 32 rows are at most `rank` real ones; the pass is bound by its reads).  The backward's factor,
// [O][r], is turned in LDS.  bf16, whole lines: 32768 x 512 13 us (2.6 TB/s), 32768 x 1160 backward 29 us (2.7 TB/s); a lane taking 64 bytes of
// its own row at a time, as fp32 and rows of odd sizes do, needed 17 and 36.
template <typename T, bool BWD, int RP, bool WHOLE>
__global__ __launch_bounds__(256, RP == 32 ? 2 : 4) void k_ad_shrink(AdArgs g) {
    constexpr int VE = 16 / (int)sizeof(T), KI = 8 * VE;  // contraction indices of an iteration: four pieces of either lane group
    // a wave's: the rows' pieces on their way (bf16), the factor turned (backward), then its sums
    __shared__ __align__(16) unsigned char lds[4][BWD ? 8192 : 32 * 33 * 4];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, lr = lane & 31, lg = lane >> 5;
    const int m0 = blockIdx.x * 32, m = m0 + lr;
    const int K = BWD ? g.O : g.I;
    const int64_t ld = BWD ? g.ld_y : g.ld_x;
    const T* base = reinterpret_cast<const T*>(BWD ? g.dy : g.x);
    const T* row = base + (int64_t)g.row(m < g.M ? m : g.M - 1) * ld;
    const T* rows[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int l = m0 + 8 * i + lane / 8;
        rows[i] = base + (int64_t)g.row(l < g.M ? l : g.M - 1) * ld;
    }
    float(*part)[33] = reinterpret_cast<float(*)[33]>(lds[wave]);
    T(*turn)[32] = reinterpret_cast<T(*)[32]>(lds[wave]);
    const T* fac = reinterpret_cast<const T*>(BWD ? g.A : g.B);
    float* out = BWD ? g.v : g.u;
    const int p = g.adapter(m);
    uint64_t todo = __ballot(p >= 0) & 0xffffffffull;
    int others = 0;  // adapters among the rows
    for (uint64_t left = todo; left; ++others) left &= ~__ballot(p == __builtin_amdgcn_readlane(p, __ffsll((unsigned long long)left) - 1));
    if (others > AD_ONE_BY_ONE) {
        for (int i = 0; i < 8; ++i) {
            const int mi = m0 + 8 * wave + i, pi = __builtin_amdgcn_readlane(p, 8 * wave + i);
            if (mi >= g.M) break;
            float acc[RP];
            shrink_row<T, BWD, RP, 1, WHOLE>(g, mi, pi, lane, acc);
            const float s = shrink_sum<RP>(acc);
            const int j = lane / (64 / RP);
            if (lane % (64 / RP) == 0) out[(int64_t)mi * g.rp + j] = j < g.r && pi >= 0 ? s : 0.f;
            if (RP == 8 && lane >= 8 && lane < 16) out[(int64_t)mi * g.rp + lane] = 0.f;  // (g.rp is 16)
        }
        return;
    }
    const bool whole = K % VE == 0;
    const int kw = ((K + 4 * KI - 1) / (4 * KI)) * KI;  // contraction indices of a wave
    const int k0 = wave * kw, k1 = k0 + kw < K ? k0 + kw : K;
    while (todo) {
        const int q = __builtin_amdgcn_readlane(p, __ffsll((unsigned long long)todo) - 1);
        const uint64_t mine = __ballot(p == q) & 0xffffffffull;
        todo &= ~mine;
        const T* f = fac + (int64_t)q * K * g.r;
        float16_t acc = zero16();
        bool done = false;
        if constexpr (sizeof(T) == 2) {
            done = whole && (!BWD || (g.r & 7) == 0);
            if (done) shrink_staged<BWD>(f, rows, K, g.r, k0, k1, reinterpret_cast<T*>(lds[wave] + (BWD ? 4096 : 0)), &turn[0][0], acc);
        }
        for (int k = k0; k < k1 && !done; k += KI) {
            if (BWD) {  // KI rows of the factor, r values each, one after the other in memory
                const int n = (k1 - k < KI ? k1 - k : KI) * g.r;
                const T* s = f + (int64_t)k * g.r;
                const int rr = g.r;
                if ((rr * (int)sizeof(T)) % 16 == 0) {
                    for (int i = lane * VE; i < n; i += 64 * VE)
                        *reinterpret_cast<uint4*>(&turn[i / rr][i % rr]) = *reinterpret_cast<const uint4*>(s + i);
                } else {
                    for (int i = lane; i < n; i += 64) turn[i / rr][i % rr] = s[i];
                }
                __builtin_amdgcn_wave_barrier();
            }
            uint4 xq[4], fq[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int kk = k + 4 * VE * lg + VE * s;
                xq[s] = ad_piece_of(whole, row, kk, K, true);
                if (!BWD) {
                    fq[s] = ad_piece_of(whole, f + (int64_t)(lr < g.r ? lr : 0) * K, kk, K, lr < g.r);
                } else {
                    T e[VE];
#pragma unroll
                    for (int i = 0; i < VE; ++i) e[i] = kk + i < K && lr < g.r ? turn[kk - k + i][lr] : (T)0.f;
                    fq[s] = *reinterpret_cast<uint4*>(e);
                }
            }
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if constexpr (sizeof(T) == 2) {
                    Mma32<bf16_t>::run(fq[s], xq[s], acc);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(chunk_f32(fq[s], i), chunk_f32(xq[s], i), acc, 0, 0, 0);
                }
            }
            if (BWD) __builtin_amdgcn_wave_barrier();
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int e = 0; e < 16; ++e) part[8 * (e / 4) + 4 * lg + e % 4][lr] = acc[e];
        __syncthreads();
        auto sum = [&](int j, int ml) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) s += reinterpret_cast<const float(*)[33]>(lds[w])[j][ml];
            return s;
        };
        for (int i = threadIdx.x; i < 32 * g.rp; i += 256) {
            const int ml = i / g.rp, j = i % g.rp;
            if (mine >> ml & 1)
                out[(int64_t)(m0 + ml) * g.rp + j] = j < g.r ? sum(j, ml) : 0.f;
        }
        __syncthreads();
    }
    const uint64_t none = __ballot(p < 0) & 0xffffffffull;  // rows without an adapter
    for (int i = threadIdx.x; i < 32 * g.rp; i += 256) {
        const int ml = i / g.rp;
        if ((none >> ml & 1) && m0 + ml < g.M) out[(int64_t)(m0 + ml) * g.rp + i % g.rp] = 0.f;
    }
}

// Rows sorted by adapter, order kept among a preference's own: workgroup q walks the index twice, to count the rows that come
// before its own, and to place them, a wave a contiguous sixteenth of the rows (and the last one those behind the last whole four).  q = P:
// the rows without one.  Bound by latency: a lane takes four rows at a time and has four such pieces on their way (32768 rows of 128: 8 us, one at
// a time 13).
__global__ __launch_bounds__(1024) void k_ad_plan(AdArgs g) {
    __shared__ int s_less[16], s_mine[16];
    const int q = blockIdx.x, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int quads = g.M / 4, len = (quads + 1023) / 1024 * 64, lo = wave * len, hi = lo + len < quads ? lo + len : quads;
    const int4* index = reinterpret_cast<const int4*>(g.index);
    auto segment = [&](int p) { return p >= 0 && p < g.P ? p : g.P; };
    // run(first row, its four's segments; -1: no row)
    auto walk = [&](auto run) {
        for (int i0 = lo; i0 < hi; i0 += 256) {
            int4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = index[i0 + 64 * u + lane < hi ? i0 + 64 * u + lane : hi - 1];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + 64 * u + lane;
                const int p[4] = {i < hi ? segment(v[u].x) : -1, i < hi ? segment(v[u].y) : -1, i < hi ? segment(v[u].z) : -1, i < hi ? segment(v[u].w) : -1};
                run(4 * i, p);
            }
        }
        if (wave == 15 && (g.M & 3)) {
            const int m = 4 * quads + lane;
            const int p[4] = {m < g.M ? segment(g.index[m < g.M ? m : 0]) : -1, -1, -1, -1};
            run(m, p);
        }
    };
    int less = 0, mine = 0;
    walk([&](int, const int(&p)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            less += p[e] >= 0 && p[e] < q;
            mine += p[e] == q;
        }
    });
    for (int o = 32; o; o >>= 1) {
        less += __shfl_xor(less, o);
        mine += __shfl_xor(mine, o);
    }
    if (lane == 0) {
        s_less[wave] = less;
        s_mine[wave] = mine;
    }
    __syncthreads();
    int start = 0, at = 0;
    for (int w = 0; w < 16; ++w) {
        start += s_less[w];
        at += w < wave ? s_mine[w] : 0;
    }
    if (threadIdx.x == 0) {
        g.seg[q] = start;
        if (q == g.P) g.seg[g.P + 1] = g.M;
    }
    if (mine == 0) return;
    at += start;
    walk([&](int m, const int(&p)[4]) {
        const uint64_t below = (1ull << lane) - 1;
        int to = at;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint64_t hits = __ballot(p[e] == q);
            to += __popcll(hits & below);
            at += __popcll(hits);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (p[e] == q) g.perm[to++] = m + e;
    });
}

// The same order where rows times adapters are too many for every workgroup to walk all rows: chunks of at least 4096 rows and an
// eighth as many as there are adapters, each with a count of every segment's rows in it (at most 8 a row and adapter in all); the counts to places,
// over the chunks and then over the segments; and every chunk's rows to their places, 64 at a time in order.
__device__ inline int ad_segment(const AdArgs& g, int64_t m) {
    const int p = g.index[m];
    return p >= 0 && p < g.P ? p : g.P;
}
__global__ __launch_bounds__(1024) void k_ad_plan_count(AdArgs g) {
    const int64_t lo = (int64_t)blockIdx.x * g.chunk, hi = lo + g.chunk < g.M ? lo + g.chunk : g.M;
    int32_t* mine = g.table + (int64_t)blockIdx.x * (g.P + 1);
    for (int p = threadIdx.x; p <= g.P; p += 1024) mine[p] = 0;
    __threadfence();
    __syncthreads();
    for (int64_t m = lo + threadIdx.x; m < hi; m += 1024) atomicAdd(mine + ad_segment(g, m), 1);
}
// a thread a segment: rows in earlier chunks for every chunk, all rows into seg
__global__ __launch_bounds__(256) void k_ad_plan_chunks(AdArgs g) {
    const int p = blockIdx.x * 256 + threadIdx.x;
    if (p > g.P) return;
    int sum = 0;
    for (int c0 = 0; c0 < g.chunks; c0 += 8) {
        int v[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) v[c] = g.table[(int64_t)(c0 + c < g.chunks ? c0 + c : 0) * (g.P + 1) + p];
#pragma unroll
        for (int c = 0; c < 8; ++c)
            if (c0 + c < g.chunks) {
                g.table[(int64_t)(c0 + c) * (g.P + 1) + p] = sum;
                sum += v[c];
            }
    }
    g.seg[p] = sum;
}
// seg: from counts to starts, a thread a run of segments
__global__ __launch_bounds__(1024) void k_ad_plan_starts(AdArgs g) {
    __shared__ int sums[1024];
    const int tid = threadIdx.x, each = g.P / 1024 + 1, p0 = tid * each, p1 = p0 + each < g.P + 1 ? p0 + each : g.P + 1;
    int sum = 0;
    for (int p = p0; p < p1; ++p) sum += g.seg[p];
    sums[tid] = sum;
    __syncthreads();
    for (int o = 1; o < 1024; o <<= 1) {
        const int before = tid >= o ? sums[tid - o] : 0;
        __syncthreads();
        sums[tid] += before;
        __syncthreads();
    }
    int at = sums[tid] - sum;
    for (int p = p0; p < p1; ++p) {
        const int n = g.seg[p];
        g.seg[p] = at;
        at += n;
    }
    if (tid == 0) g.seg[g.P + 1] = g.M;
}
__global__ __launch_bounds__(64) void k_ad_plan_place(AdArgs g) {
    const int64_t lo = (int64_t)blockIdx.x * g.chunk, hi = lo + g.chunk < g.M ? lo + g.chunk : g.M;
    const int lane = threadIdx.x;
    int32_t* mine = g.table + (int64_t)blockIdx.x * (g.P + 1);
    for (int64_t m0 = lo; m0 < hi; m0 += 64) {
        const int64_t m = m0 + lane;
        const int p = m < hi ? ad_segment(g, m) : -1;
        int first = 0, rank = 0, rows = 0;  // of the lanes with this lane's segment: the first one, those before this lane, all
        for (uint64_t todo = __ballot(p >= 0); todo;) {
            const int l = __ffsll((unsigned long long)todo) - 1, q = __builtin_amdgcn_readlane(p, l);
            const uint64_t same = __ballot(p == q);
            if (p == q) {
                first = l;
                rank = __popcll(same & ((1ull << lane) - 1));
                rows = __popcll(same);
            }
            todo &= ~same;
        }
        int at = 0;
        if (p >= 0 && first == lane) at = atomicAdd(mine + p, rows) + g.seg[p];
        at = __shfl(at, first);
        if (p >= 0) g.perm[at + rank] = (int)m;
        __threadfence_block();  // the next 64 rows' places follow these
    }
}

// The gradients of the factors and of the bias, one piece of sorted rows and 128 columns of dy (role 0: dA, dbias) or x (role 1:
// dB) a workgroup: out[c][j] = sum_m src[m][c] w[m][j] with w = u or v in three bf16 parts; a column of ones beside u's gives dbias.
// The parts of an infinite value add up to an undefined one, as do its products with the zeros beside the one of the column of ones: sums that are
// not finite are taken again on the fp32 instructions, from memory.
// Bound by its reads, dy and x once more, and their way through LDS: 32768 x (1160 + 512) bf16, 110 MB, 37 us (2.9 TB/s).
// Piece c of the sorted rows: segment p and block b = c - p of AD_PIECE rows, p the last one with seg[p] / AD_PIECE + p <= c.  A segment of one piece
// leaves its sums in the gradient, others in slots, of which a block needs two: for a segment that began in an earlier one, and for one that began
// in it and goes on.
__device__ inline int ad_slot(int b, bool began_earlier) { return 2 * b + (began_earlier ? 0 : 1); }
template <typename T, int JB>
__global__ __launch_bounds__(256, sizeof(T) == 4 ? 5 - JB : 8 - 2 * JB) void k_ad_factor_grad(AdArgs g, int col_blocks_y) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1;
    constexpr int SP = 32 * 320;                 // a plane of 32 rows x 128 columns
    constexpr int WP = (JB * 32) * 2 + 16;       // bytes of a row of w
    __shared__ __align__(16) unsigned char src[NP * SP], wts[3 * 32 * WP];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, lr = lane & 31, lg = lane >> 5;
    const int c = blockIdx.x;
    int lo = 0, hi = g.P;  // last segment p in [0, P] with seg[p] / AD_PIECE + p <= c: 64 places looked at together
    while (lo < hi) {
        const int step = (hi - lo + 64) / 64, at = lo + lane * step;
        const bool under = at <= hi && g.seg[at <= hi ? at : hi] / AD_PIECE + at <= c;
        lo += (__popcll(__ballot(under)) - 1) * step;
        hi = lo + step - 1 < hi ? lo + step - 1 : hi;
    }
    const int p = lo, b = c - p;
    const int s0 = g.seg[p] > b * AD_PIECE ? g.seg[p] : b * AD_PIECE;
    const int s1 = g.seg[p + 1] < (b + 1) * AD_PIECE ? g.seg[p + 1] : (b + 1) * AD_PIECE;
    const bool empty = b < 0 || s0 >= s1;  // no such piece: nothing but its zeros in dbias
    const bool whole = s0 == g.seg[p] && s1 == g.seg[p + 1];
    const bool is_y = (int)blockIdx.y < col_blocks_y;
    const int C = is_y ? g.O : g.I;
    const int c0 = (is_y ? blockIdx.y : blockIdx.y - col_blocks_y) * 128;
    if (!is_y && (empty || p == g.P)) return;
    if (empty) {
        if (g.dbias && threadIdx.x < 128 && c0 + (int)threadIdx.x < C) g.pb[(int64_t)c * g.O + c0 + threadIdx.x] = 0.f;
        return;
    }
    const T* base = reinterpret_cast<const T*>(is_y ? g.dy : g.x);
    const int64_t ld = is_y ? g.ld_y : g.ld_x;
    const float* w = is_y ? g.u : g.v;
    const bool weighed = p < g.P && (is_y ? g.dA : g.dB);  // (u is not there where dA is not asked for)
    const bool vec = ((reinterpret_cast<uintptr_t>(base) | (uintptr_t)(ld * (int64_t)sizeof(T))) & 15) == 0;
    float16_t acc[JB];
#pragma unroll
    for (int j = 0; j < JB; ++j) acc[j] = zero16();
    // 32 rows x 128 columns of src and their weights: eight threads a row, sixteen columns and 4 JB weights each.  Requested a step ahead, the
    // rows' places two
    const int row = tid / 8, cc = c0 + 16 * (tid % 8);
    uint4 reg[sizeof(T)];
    float wt[JB][4];
    auto place = [&](int s) { return s + row < s1 ? g.perm[s + row] : -1; };
    auto fetch = [&](int s, int m) {
        load16(base + (int64_t)(m < 0 ? 0 : m) * ld + cc, m < 0 ? 0 : C - cc, vec, reg);
#pragma unroll
        for (int jj = 0; jj < JB; ++jj) {
            const int j = 32 * jj + 4 * (tid % 8);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                wt[jj][i] = m < 0 ? 0.f : j + i < g.r ? (weighed ? w[(int64_t)(s + row) * g.rp + j + i] : 0.f) : j + i == g.r ? 1.f : 0.f;
        }
    };
    int next = place(s0);
    fetch(s0, next);
    next = place(s0 + 32);
    for (int s = s0; s < s1; s += 32) {
        {
            uint4 l[NP], h[NP];
            parts16<true>(reg, l, h);
#pragma unroll
            for (int q = 0; q < NP; ++q) {
                *reinterpret_cast<uint4*>(src + q * SP + row * 320 + (tid % 8) * 32) = l[q];
                *reinterpret_cast<uint4*>(src + q * SP + row * 320 + (tid % 8) * 32 + 16) = h[q];
            }
#pragma unroll
            for (int jj = 0; jj < JB; ++jj) {
                const int j = 32 * jj + 4 * (tid % 8);
                uint2 parts[3];
                split3<true>(make_uint4(__float_as_uint(wt[jj][0]), __float_as_uint(wt[jj][1]), __float_as_uint(wt[jj][2]), __float_as_uint(wt[jj][3])), parts);
#pragma unroll
                for (int q = 0; q < 3; ++q) *reinterpret_cast<uint2*>(wts + q * 32 * WP + row * WP + j * 2) = parts[q];
            }
        }
        __syncthreads();
        if (s + 32 < s1) {
            fetch(s + 32, next);
            next = place(s + 64);
        }
        typedef __attribute__((address_space(3))) short4_t lds_s4;
        const int a = lane & 15, q0 = (lane >> 4) & 1, e = a >> 2, cw = a & 3;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const int k = 16 * ks + 8 * lg + e;
            uint4 fs[NP];
#pragma unroll
            for (int q = 0; q < NP; ++q) {
                const unsigned char* at = src + q * SP + k * 320 + (32 * wave + 16 * q0 + 4 * cw) * 2;
                const uint2 u0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)at));
                const uint2 u1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(at + 4 * 320)));
                fs[q] = make_uint4(u0.x, u0.y, u1.x, u1.y);
            }
#pragma unroll
            for (int j = 0; j < JB; ++j) {
                uint4 fw[3];
#pragma unroll
                for (int q = 0; q < 3; ++q) {
                    const unsigned char* at = wts + q * 32 * WP + k * WP + (32 * j + 16 * q0 + 4 * cw) * 2;
                    const uint2 u0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)at));
                    const uint2 u1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(at + 4 * WP)));
                    fw[q] = make_uint4(u0.x, u0.y, u1.x, u1.y);
                }
                // lane: column of src; accumulator: j
#pragma unroll
                for (int q = 2; q >= 0; --q)
#pragma unroll
                    for (int r = NP - 1; r >= 0; --r)
                        if (q + r <= 2) Mma32<bf16_t>::run(fw[q], fs[r], acc[j]);
            }
        }
        __syncthreads();
    }
    const int col = c0 + 32 * wave + lr;
#pragma unroll
    for (int j = 0; j < JB; ++j)
        if (any_undefined(acc[j])) {
            const int jj = 32 * j + lr;
            float16_t t = zero16();
#pragma unroll 1
            for (int s = s0 + lg; s < s1 + lg; s += 2) {
                const bool on = s < s1;
                const float wv = !on ? 0.f : jj < g.r ? (weighed ? w[(int64_t)s * g.rp + jj] : 0.f) : jj == g.r ? 1.f : 0.f;
                const float sv = on && col < C ? to_f(base[(int64_t)g.perm[s] * ld + col]) : 0.f;
                t = __builtin_amdgcn_mfma_f32_32x32x2f32(wv, sv, t, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (!(__builtin_fabsf(acc[j][e]) < __builtin_inff())) acc[j][e] = t[e];
        }
    if (col >= C) return;
    float* out = is_y ? g.dA : g.dB;
    if (out && !whole) out = is_y ? g.pA : g.pB;
    const int64_t pi = whole ? p : ad_slot(b, g.seg[p] < b * AD_PIECE);
#pragma unroll
    for (int j = 0; j < JB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int jj = 32 * j + 8 * (e / 4) + 4 * lg + e % 4;
            if (jj < g.r) {
                if (out && p < g.P) out[is_y ? (pi * g.O + col) * g.r + jj : (pi * g.r + jj) * g.I + col] = acc[j][e];
            } else if (jj == g.r && is_y && g.dbias) {
                g.pb[(int64_t)c * g.O + col] = acc[j][e];
            }
        }
}

// (32768 x 512 x 1160: 12 ranges of dW0, 28 MB, 12 us.)
// What is left in pieces, added in order: split dW0; factor gradients of preferences with several pieces (none: zero); dbias.
__global__ __launch_bounds__(256) void k_ad_final(AdArgs g, int64_t n_w, int64_t n_f, int blocks_w, int blocks_f) {
    if ((int)blockIdx.x < blocks_w) {
        const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
        if ((n_w & 3) == 0) {
            if (i >= n_w) return;
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
            for (int q = 0; q < g.split; ++q) {
                const float4 v = *reinterpret_cast<const float4*>(g.pw + q * n_w + i);
                s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            }
            *reinterpret_cast<float4*>(g.dw0 + i) = s;
        } else {
            for (int64_t e = i; e < i + 4 && e < n_w; ++e) {
                float s = 0.f;
#pragma unroll 8
                for (int q = 0; q < g.split; ++q) s += g.pw[q * n_w + e];
                g.dw0[e] = s;
            }
        }
    } else if ((int)blockIdx.x < blocks_w + blocks_f) {
        // of [P][r (O + I)]: most adapters have no rows in two pieces, and nothing is to be done for them
        for (int64_t i = (int64_t)(blockIdx.x - blocks_w) * 256 + threadIdx.x; i < n_f; i += (int64_t)blocks_f * 256) {
            const int64_t per = (int64_t)g.r * (g.O + g.I);
            const int p = (int)(i / per);
            int64_t k = i % per;
            const int s0 = g.seg[p], s1 = g.seg[p + 1];
            const int b0 = s0 / AD_PIECE, b1 = s1 > s0 ? (s1 - 1) / AD_PIECE : b0 - 1;
            const bool in_a = k < (int64_t)g.r * g.O;
            if (!in_a) k -= (int64_t)g.r * g.O;
            const int64_t n = (int64_t)g.r * (in_a ? g.O : g.I);
            float* out = in_a ? g.dA : g.dB;
            const float* part = in_a ? g.pA : g.pB;
            if (b1 == b0 || !out) continue;
            float s = 0.f;
            for (int b = b0; b <= b1; ++b) s += part[ad_slot(b, b > b0) * n + k];
            out[p * n + k] = s;
        }
    } else {
        // 32 columns of dbias, eight groups of threads a contiguous eighth of the pieces each
        __shared__ float sums[8][32];
        const int o = (blockIdx.x - blocks_w - blocks_f) * 32 + threadIdx.x % 32, q = threadIdx.x / 32;
        const int each = (g.pieces + 7) / 8, c1 = (q + 1) * each < g.pieces ? (q + 1) * each : g.pieces;
        float s = 0.f;
        if (o < g.O)
#pragma unroll 16
            for (int c = q * each; c < c1; ++c) s += g.pb[(int64_t)c * g.O + o];
        sums[q][threadIdx.x % 32] = s;
        __syncthreads();
        if (q == 0 && o < g.O) {
            for (int i = 1; i < 8; ++i) s += sums[i][threadIdx.x];
            g.dbias[o] = s;
        }
    }
}

static int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// rows times segments beyond which the plan takes its four launches.  us of a call for dbias alone, one launch and four:
// 131072 rows of 2048 adapters 201 and 277, 16384 of 16384 230 and 373, 1048576 of 512 493 and 420, of 4096 2510 and 483
#define AD_PLAN_WORK ((int64_t)1 << 29)
static bool ad_plan_is_large(const AdArgs& g) { return (int64_t)g.M * (g.P + 1) > AD_PLAN_WORK; }
// sizes of the scratch regions for these dimensions; carve(nullptr) gives the total
static int64_t ad_carve(AdArgs& g, bool bwd, void* ws) {
    char* at = reinterpret_cast<char*>(ws);
    int64_t off = 0;
    auto take = [&](int64_t bytes) {
        void* q = ws ? at + off : nullptr;
        off += align_up(bytes, 256);
        return q;
    };
    g.rp = g.r <= 16 ? 16 : 32;
    g.u = (float*)take((int64_t)g.M * g.rp * 4);
    if (bwd) {
        g.v = (float*)take((int64_t)g.M * g.rp * 4);
        g.seg = (int32_t*)take(((int64_t)g.P + 2) * 4);
        g.perm = (int32_t*)take((int64_t)g.M * 4);
        if (ad_plan_is_large(g)) {
            const int64_t least = cdiv(g.M, 1024) > 4096 ? cdiv(g.M, 1024) : 4096, by_p = cdiv(g.P + 1, 8);
            g.chunk = (int)(by_p > least ? by_p : least);
            g.chunks = (int)cdiv(g.M, g.chunk);
            g.table = (int32_t*)take((int64_t)g.chunks * (g.P + 1) * 4);
        }
        // dW0's contraction in ranges: bf16, one workgroup of the large tiles a CU (32768 x 512 x 1160, us: 12 ranges 65 and 13 for their sum, 25
        // ranges 65 and 17, on small tiles 13 ranges 83 and 13); fp32, two of the small ones
        int64_t split = g.bf16 ? 256 / (cdiv(g.O, 256) * cdiv(g.I, 128)) : cdiv(512, cdiv(g.O, 128) * cdiv(g.I, 128));
        const int64_t most = cdiv(g.M, 64);
        if (split > most) split = most;
        if (split < 1) split = 1;
        g.kchunk = (int)align_up(cdiv(g.M > 0 ? g.M : 1, split), 32);
        g.split = (int)cdiv(g.M > 0 ? g.M : 1, g.kchunk);
        g.pw = (float*)take(g.split > 1 ? (int64_t)g.split * g.O * g.I * 4 : 0);
        g.pieces = (int)(g.M / AD_PIECE + 1 + g.P);  // ids run to (M - 1) / AD_PIECE + P
        const int64_t slots = g.M > AD_PIECE ? 2 * cdiv(g.M, AD_PIECE) : 0;
        g.pA = (float*)take(slots * g.O * g.r * 4);
        g.pB = (float*)take(slots * g.I * g.r * 4);
        g.pb = (float*)take((int64_t)g.pieces * g.O * 4);
    }
    return off > 0 ? off : 256;
}
static AdArgs ad_args(const morlax_adapter_dims& d) {
    AdArgs g = {};
    g.M = d.rows; g.I = d.d_in; g.O = d.d_out; g.r = d.rank; g.P = d.n_adapters;
    g.ld_x = d.ld_x; g.ld_y = d.ld_y; g.bf16 = d.dtype;
    return g;
}
int64_t adapter_ws_bytes(const morlax_adapter_dims& d, bool bwd) {
    AdArgs g = ad_args(d);
    return ad_carve(g, bwd, nullptr);
}

static bool on16(const void* p, int64_t ld, int size) { return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size)) & 15) == 0; }
// u and v take a workgroup a row where the factors that the rows read, each its own copy, are at most so many bytes (of the L2).  us of a forward of
// 512 x 1160 bf16, rank 16, with and without: mixed rows 256 15 and 56, 1024 44 and 84, 4096 (64 MiB) 75 and 112; grouped 1024 19 and 22, 4096 30
// and 22 -- who mixes rows gains more than who groups them loses.
#define AD_ROW_BYTES (64 << 20)

// run(padded rank, whole) with both as constants
template <typename F>
static void pick_rank(const AdArgs& g, bool whole, F run) {
    typedef std::integral_constant<int, 8> R8;
    typedef std::integral_constant<int, 16> R16;
    typedef std::integral_constant<int, 32> R32;
    if (g.r <= 8) {
        if (whole) run(R8{}, std::true_type{});
        else run(R8{}, std::false_type{});
    } else if (g.rp == 16) {
        if (whole) run(R16{}, std::true_type{});
        else run(R16{}, std::false_type{});
    } else {
        if (whole) run(R32{}, std::true_type{});
        else run(R32{}, std::false_type{});
    }
}
template <typename T, bool BWD>
static void shrink(const AdArgs& g, hipStream_t s) {
    const int K = BWD ? g.O : g.I;
    const bool whole = (BWD ? g.r : K) % (16 / (int)sizeof(T)) == 0;
    if ((int64_t)g.M * g.r * K * (int64_t)sizeof(T) <= AD_ROW_BYTES) {
        const bool one = K <= (BWD ? 256 : 128 * 16 / (int)sizeof(T)) && g.M > 256;  // a wave a row: two rounds of its lanes or four, and waves enough
        auto run = [&](auto rp, auto w) {
            constexpr int RP = decltype(rp)::value;
            constexpr bool W = decltype(w)::value;
            if (one) k_ad_shrink_row<T, BWD, RP, 1, W><<<cdiv(g.M, 4), 256, 0, s>>>(g);
            else k_ad_shrink_row<T, BWD, RP, 4, W><<<g.M, 256, 0, s>>>(g);
        };
        pick_rank(g, whole, run);
    } else {
        pick_rank(g, whole, [&](auto rp, auto w) { k_ad_shrink<T, BWD, decltype(rp)::value, decltype(w)::value><<<cdiv(g.M, 32), 256, 0, s>>>(g); });
    }
}
// Which kernel multiplies with W0.  Few rows: 16 columns a workgroup where 128 x 128 tiles would leave most CUs without one.  us, few rows' kernel
// and tiles, 512 to 1160: bf16 64 rows 11 and 20, 256 14 and 21, 512 (40 tiles) 18 and 21, 2048 (160) 45 and 24; fp32 1024 41 and 72, 2048 (160)
// 70 and 76; 64 to 512, where a tile has two steps: bf16 4099 rows (132) 23 and 37, 16384 (512) 89 and 55; fp32 4099 49 and 122.  Else tiles:
// direct-to-LDS loads for bf16 rows of whole 16-byte pieces within 32-bit offsets, the general kernel for the rest.
template <typename T, int ROLE>
static void product(const AdArgs& g, hipStream_t s) {
    const int rows_a = ROLE == AD_DW ? g.O : g.M, rows_b = ROLE == AD_FWD ? g.O : g.I, K = ROLE == AD_FWD ? g.I : ROLE == AD_DX ? g.O : g.M;
    const int64_t tiles = cdiv(rows_a, 128) * cdiv(rows_b, 128);
    const int split = ROLE == AD_DW ? g.split : 1;
    if constexpr (ROLE != AD_DW)
        if ((tiles <= (sizeof(T) == 4 && ROLE == AD_FWD ? 160 : 64) || (K <= 64 && (sizeof(T) == 4 || tiles <= 256))) && cdiv(g.M, 32) <= 65535) {
            pick_rank(g, K % (16 / (int)sizeof(T)) == 0, [&](auto rp, auto w) {
                k_ad_few<T, ROLE == AD_DX, decltype(rp)::value, decltype(w)::value><<<dim3(cdiv(rows_b, 16), cdiv(g.M, 32)), 512, 0, s>>>(g);
            });
            return;
        }
    if constexpr (sizeof(T) == 2) {
        const bool x_ok = on16(g.x, g.ld_x, 2) && (int64_t)g.M * g.ld_x * 2 < (int64_t)1 << 32;
        const bool y_ok = on16(g.dy, g.ld_y, 2) && (int64_t)g.M * g.ld_y * 2 < (int64_t)1 << 32;
        const bool w_ok = g.I % 8 == 0;  // (d_in, d_out <= 65536: W0 has at most 2^33 bytes)
        const bool small_w = (int64_t)g.O * g.I * 2 < (int64_t)1 << 32;
        const bool ok = ROLE == AD_FWD ? x_ok && w_ok && small_w : ROLE == AD_DX ? y_ok && w_ok && small_w && g.O % 8 == 0 : x_ok && y_ok && w_ok && g.O % 8 == 0;
        if (ok && K >= 32) {
            const int64_t big = cdiv(rows_a, 256) * cdiv(rows_b, 128);
            // Large tiles do a product in 7/8 of the small ones' time and go two to a CU at a time, the small ones three; the CU with most tiles
            // decides.  us: 16384 x 1160 x 512 (640 or 1280 tiles) 48 large, 40 small; dX of 32768 x 512 x 1160 (512 or 1024) 64 and 73
            if (2 * 7 * cdiv(big * split, 256) <= 8 * cdiv(tiles * split, 256)) {
                if (g.rp == 16) k_ad_gemm_dma<ROLE, 4, 2, 16><<<big * split, 256, 0, s>>>(g);
                else k_ad_gemm_dma<ROLE, 4, 2, 32><<<big * split, 256, 0, s>>>(g);
            } else {
                if (g.rp == 16) k_ad_gemm_dma<ROLE, 2, 2, 16><<<tiles * split, 256, 0, s>>>(g);
                else k_ad_gemm_dma<ROLE, 2, 2, 32><<<tiles * split, 256, 0, s>>>(g);
            }
            return;
        }
    }
    if (g.rp == 16) k_ad_gemm<T, ROLE, 16><<<dim3(tiles, split), 256, 0, s>>>(g);
    else k_ad_gemm<T, ROLE, 32><<<dim3(tiles, split), 256, 0, s>>>(g);
}

template <typename T>
static void fwd(const AdArgs& g, hipStream_t s) {
    shrink<T, false>(g, s);
    product<T, AD_FWD>(g, s);
}
void launch_adapter_fwd(const morlax_adapter_dims& d, const void* x, const void* w0, const float* bias, const void* A, const void* B,
                        const int32_t* index, void* y, void* ws, hipStream_t s) {
    AdArgs g = ad_args(d);
    if (g.M == 0) return;
    ad_carve(g, false, ws);
    g.x = x; g.w0 = w0; g.bias = bias; g.A = A; g.B = B; g.index = index; g.y = y;
    if (d.dtype) fwd<bf16_t>(g, s);
    else fwd<float>(g, s);
}

template <typename T>
static void bwd(AdArgs& g, hipStream_t s) {
    const bool factors = g.dA || g.dB || g.dbias;
    if (factors || g.dx) {
        if (ad_plan_is_large(g)) {
            k_ad_plan_count<<<g.chunks, 1024, 0, s>>>(g);
            k_ad_plan_chunks<<<cdiv(g.P + 1, 256), 256, 0, s>>>(g);
            k_ad_plan_starts<<<1, 1024, 0, s>>>(g);
            k_ad_plan_place<<<g.chunks, 64, 0, s>>>(g);
        } else {
            k_ad_plan<<<g.P + 1, 1024, 0, s>>>(g);
        }
        g.order = g.perm;
    }
    if (g.M > 0) {
        if (g.dA) shrink<T, false>(g, s);
        if (g.dx || g.dB) shrink<T, true>(g, s);
        if (g.dx) product<T, AD_DX>(g, s);
    }
    if (g.dw0) product<T, AD_DW>(g, s);
    if (factors) {
        const int by = g.dA || g.dbias ? (int)cdiv(g.O, 128) : 0, bx = g.dB ? (int)cdiv(g.I, 128) : 0;
        if (g.r < 32) k_ad_factor_grad<T, 1><<<dim3(g.pieces, by + bx), 256, 0, s>>>(g, by);
        else k_ad_factor_grad<T, 2><<<dim3(g.pieces, by + bx), 256, 0, s>>>(g, by);
    }
    const int64_t n_w = g.dw0 && g.split > 1 ? (int64_t)g.O * g.I : 0, n_f = g.dA || g.dB ? (int64_t)g.P * g.r * (g.O + g.I) : 0;
    const int64_t bw = cdiv(n_w, 1024), bf = cdiv(n_f, 256) < 2048 ? cdiv(n_f, 256) : 2048, bb = g.dbias ? cdiv(g.O, 32) : 0;
    if (bw + bf + bb > 0) k_ad_final<<<bw + bf + bb, 256, 0, s>>>(g, n_w, n_f, (int)bw, (int)bf);
}
void launch_adapter_bwd(const morlax_adapter_dims& d, const void* x, const void* w0, const void* A, const void* B, const int32_t* index,
                        const void* dy, void* dx, float* dw0, float* dbias, float* dA, float* dB, void* ws, hipStream_t s) {
    AdArgs g = ad_args(d);
    ad_carve(g, true, ws);
    g.x = x; g.w0 = w0; g.A = A; g.B = B; g.index = index; g.dy = dy;
    g.dx = dx; g.dw0 = dw0; g.dbias = dbias; g.dA = dA; g.dB = dB;
    if (d.dtype) bwd<bf16_t>(g, s);
    else bwd<float>(g, s);
}
