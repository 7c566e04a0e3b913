// What stands between two blocks of a stack, row by row:
//   n = u r_u w_post,  y = x + scale sigmoid(gate) n,  h = y r_y w_pre,    r_v = 1 / sqrt(mean(v^2) + eps)
// and its gradients, with dY = dy + r_y (w_pre dh) - y r_y^3 mean(w_pre dh y):
//   dx = dY,  dscale = sum dY sigmoid(gate) n,  dgate = dY scale n s (1 - s),  dn = dY scale s,
//   dw_post = sum dn u r_u,  du = r_u (w_post dn) - u r_u^3 mean(w_post dn u),  dw_pre = sum dh y r_y.
// Bound: HBM.  Every tensor goes through registers once: a row lies along the lanes of a wave (or of four, beyond 128 pieces of 16 bytes), the
// backward computes n, y and both means again, and a workgroup keeps the three columns' sums of its rows in registers until its last row.
#include "mlp_device.h"

static int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct NormArgs {
    const void *x, *u, *gate, *dy, *dh;
    const float *scale, *w_post, *w_pre;
    void *y, *h, *dx, *du, *dgate;
    float *dscale, *dw_post, *dw_pre, *part;  // part [blocks, 3, width]
    int64_t ld_x, ld_u, ld_g, ld_h;
    float eps, over;  // over = 1 / width
    int rows, width, blocks;
};

template <typename T> struct Run16 {  // 16 bytes of elements, aligned to one
    static constexpr int V = 16 / sizeof(T);
    typedef T vec_t __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
template <typename T>
__device__ inline void load_run(const T* p, int n, float (&v)[16 / sizeof(T)]) {
    constexpr int V = Run16<T>::V;
    if (n >= V) {
        const typename Run16<T>::vec_t u = *reinterpret_cast<const typename Run16<T>::vec_t*>(p);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (float)u[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = i < n ? to_f(p[i]) : 0.f;
    }
}
template <typename T>
__device__ inline void save_run(T* p, int n, const float (&v)[16 / sizeof(T)]) {
    constexpr int V = Run16<T>::V;
    if (n >= V) {
        typename Run16<T>::vec_t u;
#pragma unroll
        for (int i = 0; i < V; ++i) u[i] = (T)v[i];
        *reinterpret_cast<typename Run16<T>::vec_t*>(p) = u;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) p[i] = cvt<T>(v[i]);
    }
}
// sum over the W waves of a row
template <int W>
__device__ inline float row_sum(float v, float* lds) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if constexpr (W == 1) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}
// sigmoid, and what it lacks to one (from the exponential of -|v|, so that neither loses its digits or overflows)
__device__ inline float2 sigmoid_of(float v) {
    const float e = __expf(-__builtin_fabsf(v)), r = __builtin_amdgcn_rcpf(1.f + e);
    return v >= 0.f ? make_float2(r, e * r) : make_float2(e * r, v == v ? r : v);
}

// A row of up to W * 64 * V * CH elements, W waves of 64 lanes
template <typename T, int W, int CH>
struct NormRow {
    static constexpr int V = 16 / sizeof(T);
    float x[CH][V], u[CH][V], s[CH][V], n[CH][V];  // s: the gate; after value(): x is y, n the normed u
    float r_u, r_y;
    __device__ static inline int col(int c) { return (c * W * 64 + (W == 1 ? threadIdx.x & 63 : threadIdx.x)) * V; }
    __device__ inline void load(const NormArgs& g, int64_t row) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = col(c), left = g.width - at;
            load_run(reinterpret_cast<const T*>(g.x) + row * g.ld_x + at, left, x[c]);
            if (g.u) load_run(reinterpret_cast<const T*>(g.u) + row * g.ld_u + at, left, u[c]);
            if (g.gate) load_run(reinterpret_cast<const T*>(g.gate) + row * g.ld_g + at, left, s[c]);
        }
    }
    __device__ inline void value(const NormArgs& g, const float (&sc)[CH][V], const float (&wo)[CH][V], float* lds) {
        r_u = 1.f;
        if (g.u) {
            if (g.w_post) {
                float q = 0.f;
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < V; ++i) q = __builtin_fmaf(u[c][i], u[c][i], q);
                r_u = 1.f / sqrtf(row_sum<W>(q, lds) * g.over + g.eps);
            }
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    n[c][i] = u[c][i] * r_u * wo[c][i];
                    x[c][i] = __builtin_fmaf(g.gate ? sc[c][i] * sigmoid_of(s[c][i]).x : sc[c][i], n[c][i], x[c][i]);
                }
        }
        r_y = 1.f;
        if (g.w_pre) {
            float q = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < V; ++i) q = __builtin_fmaf(x[c][i], x[c][i], q);
            r_y = 1.f / sqrtf(row_sum<W>(q, lds) * g.over + g.eps);
        }
    }
};
template <typename T, int W, int CH>
__device__ inline void columns(const NormArgs& g, const float* p, float (&v)[CH][16 / sizeof(T)]) {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 16 / (int)sizeof(T); ++i) {
            const int at = NormRow<T, W, CH>::col(c) + i;
            v[c][i] = at < g.width ? (p ? p[at] : 1.f) : 0.f;
        }
}

template <typename T, int W, int CH>
__global__ __launch_bounds__(256) void k_norm_fwd(NormArgs g) {
    constexpr int V = 16 / sizeof(T);
    __shared__ float lds[4];
    float sc[CH][V], wo[CH][V], wi[CH][V];
    columns<T, W, CH>(g, g.scale, sc);
    columns<T, W, CH>(g, g.w_post, wo);
    columns<T, W, CH>(g, g.w_pre, wi);
    const int64_t per = W == 1 ? 4 : 1;
    for (int64_t row = blockIdx.x * per + (W == 1 ? threadIdx.x >> 6 : 0); row < g.rows; row += gridDim.x * per) {
        NormRow<T, W, CH> r;
        r.load(g, row);
        r.value(g, sc, wo, lds);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = r.col(c), left = g.width - at;
            if (g.y) save_run(reinterpret_cast<T*>(g.y) + row * g.ld_x + at, left, r.x[c]);
            if (g.h) {
                float h[V];
#pragma unroll
                for (int i = 0; i < V; ++i) h[i] = r.x[c][i] * r.r_y * wi[c][i];
                save_run(reinterpret_cast<T*>(g.h) + row * g.ld_h + at, left, h);
            }
        }
    }
}

template <typename T, int W, int CH>
__global__ __launch_bounds__(256) void k_norm_bwd(NormArgs g) {
    constexpr int V = 16 / sizeof(T), CAP = 64 * V * CH;  // columns of a wave
    __shared__ float lds[4];
    __shared__ float sums[W == 1 ? 3 * CAP : 1];
    float sc[CH][V], wo[CH][V], wi[CH][V], ds[CH][V], dwo[CH][V], dwi[CH][V];
    columns<T, W, CH>(g, g.scale, sc);
    columns<T, W, CH>(g, g.w_post, wo);
    columns<T, W, CH>(g, g.w_pre, wi);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) ds[c][i] = dwo[c][i] = dwi[c][i] = 0.f;
    const int64_t per = W == 1 ? 4 : 1;
    for (int64_t row = blockIdx.x * per + (W == 1 ? threadIdx.x >> 6 : 0); row < g.rows; row += gridDim.x * per) {
        NormRow<T, W, CH> r;
        float dy[CH][V], dh[CH][V];
        r.load(g, row);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = r.col(c), left = g.width - at;
            load_run(reinterpret_cast<const T*>(g.dy) + row * g.ld_x + at, g.dy ? left : 0, dy[c]);
            load_run(reinterpret_cast<const T*>(g.dh) + row * g.ld_h + at, g.dh ? left : 0, dh[c]);
        }
        r.value(g, sc, wo, lds);
        if (g.dh) {
            float q = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    dwi[c][i] = __builtin_fmaf(dh[c][i], r.x[c][i] * r.r_y, dwi[c][i]);
                    dh[c][i] *= wi[c][i];
                    q = __builtin_fmaf(dh[c][i], r.x[c][i], q);
                }
            q = row_sum<W>(q, lds) * g.over * r.r_y * r.r_y;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < V; ++i) dy[c][i] = __builtin_fmaf(r.r_y, __builtin_fmaf(-q, r.x[c][i], dh[c][i]), dy[c][i]);
        }
        float q = 0.f;
        if (g.dx) {
#pragma unroll
            for (int c = 0; c < CH; ++c) save_run(reinterpret_cast<T*>(g.dx) + row * g.ld_x + r.col(c), g.width - r.col(c), dy[c]);
        }
        if (!g.u) continue;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float dg[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float2 sig = g.gate ? sigmoid_of(r.s[c][i]) : make_float2(1.f, 0.f);
                const float t = dy[c][i] * sig.x, dn = t * sc[c][i];
                ds[c][i] = __builtin_fmaf(t, r.n[c][i], ds[c][i]);
                dg[i] = dn * r.n[c][i] * sig.y;
                dwo[c][i] = __builtin_fmaf(dn, r.u[c][i] * r.r_u, dwo[c][i]);
                dy[c][i] = dn * wo[c][i];
                q = __builtin_fmaf(dy[c][i], r.u[c][i], q);
            }
            if (g.dgate) save_run(reinterpret_cast<T*>(g.dgate) + row * g.ld_g + r.col(c), g.width - r.col(c), dg);
        }
        if (!g.du) continue;
        if (g.w_post) {
            q = row_sum<W>(q, lds) * g.over * r.r_u * r.r_u;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < V; ++i) dy[c][i] = r.r_u * __builtin_fmaf(-q, r.u[c][i], dy[c][i]);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) save_run(reinterpret_cast<T*>(g.du) + row * g.ld_u + r.col(c), g.width - r.col(c), dy[c]);
    }
    if (!g.part) return;
    float* out = g.part + (int64_t)blockIdx.x * 3 * g.width;
    if constexpr (W == 1) {  // the four waves' sums, one wave after the other
        const int lane = threadIdx.x & 63;
#pragma unroll 1
        for (int w = 0; w < 4; ++w) {
            if ((int)(threadIdx.x >> 6) == w) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int at = (c * V + i) * 64 + lane;  // (a lane's own place: no bank twice)
                        sums[at] = (w ? sums[at] : 0.f) + ds[c][i];
                        sums[CAP + at] = (w ? sums[CAP + at] : 0.f) + dwo[c][i];
                        sums[2 * CAP + at] = (w ? sums[2 * CAP + at] : 0.f) + dwi[c][i];
                    }
            }
            __syncthreads();
        }
        for (int x = threadIdx.x; x < 3 * CAP; x += 256) {
            const int k = x / CAP, at = x % CAP, lane_ = at & 63, ci = at >> 6, col = (ci / V * 64 + lane_) * V + ci % V;
            if (col < g.width) out[(int64_t)k * g.width + col] = sums[x];
        }
    } else {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int col = NormRow<T, W, CH>::col(c) + i;
                if (col >= g.width) continue;
                out[col] = ds[c][i];
                out[g.width + col] = dwo[c][i];
                out[2 * (int64_t)g.width + col] = dwi[c][i];
            }
    }
}
// the workgroups' sums: 64 columns of the three to a block, four threads a column
__global__ __launch_bounds__(256) void k_norm_columns(NormArgs g) {
    __shared__ float part[4][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6, all = 3 * g.width;
    float sum = 0.f;
    if (c < all) {
#pragma unroll 8
        for (int b = w; b < g.blocks; b += 4) sum += g.part[(int64_t)b * all + c];
    }
    part[w][threadIdx.x & 63] = sum;
    __syncthreads();
    if (w || c >= all) return;
    sum = (part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]);
    const int k = c / g.width, at = c - k * g.width;
    float* out = k == 0 ? g.dscale : k == 1 ? g.dw_post : g.dw_pre;
    if (out) out[at] = sum;
}

static NormArgs norm_args(const morlax_norm_dims& d) {
    NormArgs g = {};
    g.rows = d.rows; g.width = d.width; g.eps = d.eps; g.over = 1.f / d.width;
    g.ld_x = d.ld_x; g.ld_u = d.ld_u; g.ld_g = d.ld_g; g.ld_h = d.ld_h;
    return g;
}
// pieces of 16 bytes of a row; a wave holds two a lane
static int norm_pieces(const morlax_norm_dims& d) { return (int)cdiv(d.width, d.dtype ? 8 : 4); }
static int norm_blocks(const morlax_norm_dims& d) {
    const int64_t all = cdiv(d.rows, norm_pieces(d) <= 128 ? 4 : 1);
    return (int)(all < 1 ? 1 : all < 1024 ? all : 1024);
}
int64_t norm_ws_bytes(const morlax_norm_dims& d) { return (int64_t)norm_blocks(d) * 3 * d.width * 4; }

template <typename T, int W, int CH>
static void norm_pass(const NormArgs& g, bool back, hipStream_t s) {
    if (back) {
        k_norm_bwd<T, W, CH><<<dim3(g.blocks), 256, 0, s>>>(g);
    } else {
        const int64_t all = cdiv(g.rows, W == 1 ? 4 : 1);
        k_norm_fwd<T, W, CH><<<dim3((uint32_t)(all < 4096 ? all : 4096)), 256, 0, s>>>(g);
    }
}
template <typename T>
static void norm_pick(const NormArgs& g, int pieces, bool back, hipStream_t s) {
    if (pieces <= 64) norm_pass<T, 1, 1>(g, back, s);
    else if (pieces <= 128) norm_pass<T, 1, 2>(g, back, s);
    else if (pieces <= 256) norm_pass<T, 4, 1>(g, back, s);
    else if (pieces <= 512) norm_pass<T, 4, 2>(g, back, s);
    else if (sizeof(T) == 2 || pieces <= 1024) norm_pass<T, 4, 4>(g, back, s);
    else norm_pass<T, 4, sizeof(T) == 2 ? 4 : 8>(g, back, s);
}
void launch_norm_fwd(const morlax_norm_dims& d, const void* x, const void* u, const void* gate, const float* scale, const float* w_post,
                     const float* w_pre, void* y, void* h, hipStream_t s) {
    NormArgs g = norm_args(d);
    g.x = x; g.u = u; g.gate = gate; g.scale = scale; g.w_post = w_post; g.w_pre = w_pre; g.y = y; g.h = h;
    if (d.dtype) norm_pick<bf16_t>(g, norm_pieces(d), false, s);
    else norm_pick<float>(g, norm_pieces(d), false, s);
}
void launch_norm_bwd(const morlax_norm_dims& d, const void* x, const void* u, const void* gate, const float* scale, const float* w_post,
                     const float* w_pre, const void* dy, const void* dh, void* dx, void* du, void* dgate, float* dscale, float* dw_post, float* dw_pre,
                     void* ws, hipStream_t s) {
    NormArgs g = norm_args(d);
    g.x = x; g.u = u; g.gate = gate; g.scale = scale; g.w_post = w_post; g.w_pre = w_pre; g.dy = dy; g.dh = dh;
    g.dx = dx; g.du = du; g.dgate = dgate; g.dscale = dscale; g.dw_post = dw_post; g.dw_pre = dw_pre;
    g.blocks = norm_blocks(d);
    if (dscale || dw_post || dw_pre) g.part = reinterpret_cast<float*>(ws);
    if (d.dtype) norm_pick<bf16_t>(g, norm_pieces(d), true, s);
    else norm_pick<float>(g, norm_pieces(d), true, s);
    if (g.part) k_norm_columns<<<dim3((uint32_t)cdiv(3 * (int64_t)d.width, 64)), 256, 0, s>>>(g);
}
