// What stands between two blocks of a stack, row by row:
//   n = u r_u w_post,  y = x + scale sigmoid(gate) n,  h = y r_y w_pre,    r_v = 1 / sqrt(mean(v^2) + eps)
// and its gradients, with dY = dy + r_y (w_pre dh) - y r_y^3 mean(w_pre dh y):
//   dx = dY,  dscale = sum dY sigmoid(gate) n,  dgate = dY scale n s (1 - s),  dn = dY scale s,
//   dw_post = sum dn u r_u,  du = r_u (w_post dn) - u r_u^3 mean(w_post dn u),  dw_pre = sum dh y r_y.
// Bound: HBM.  Every tensor goes through registers once: a row lies along the lanes of a wave, 16 bytes each (or of up to sixteen waves), the
// backward computes n, y and both means again, and a workgroup keeps the three columns' sums of its rows in registers until its last row.  65536 rows of
// 512 with gradients: bf16 182 us (4.3 and 5.1 TB/s), fp32 128 and 224 (5.2, 4.8).  Rows that take sixteen waves have 128 registers for all of that and
// 58 to 72 of their backward's in memory: 4096 rows of 8192 bf16 281 us, 1.9 TB/s, of the same elements in rows of 4096 132.
#include "mlp_device.h"
#include "pieces.h"

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
// sum over the W waves of a row, the same in all lanes
template <int CTRL, int ROWS>
__device__ inline float moved(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xf, true)); }
template <int W>
__device__ inline float row_sum(float v, float* lds) {
    v += moved<0x111, 0xf>(v);  // along 16 lanes, into the last of them
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);  // from the row before, from the two before
    v += moved<0x143, 0xc>(v);
    v = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
    if constexpr (W == 1) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float all = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) all += lds[w];
    return all;
}
__device__ inline float sigmoid_of(float v) { return __builtin_amdgcn_rcpf(1.f + __expf(-v)); }
// and what it lacks to one, all digits of it: neither the infinite exponential of a low gate nor the sigmoid of a high one leaves any
__device__ inline float2 sigmoid_both(float v) {
    const float e = __expf(-v), s = __builtin_amdgcn_rcpf(1.f + e);
    return make_float2(s, v < 0.f ? 1.f - s : e * s);
}
template <typename T>
__device__ inline void values(const uint4& u, float (&v)[16 / sizeof(T)]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 16 / (int)sizeof(T); ++i) {
        if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(w[i]);
        else v[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
}
// A row of up to W * 64 * V * CH elements, W waves of 64 lanes: what is requested of it ...
template <typename T, int W, int CH, bool WHOLE, bool BACK>
struct NormInput {
    typedef RowPiece<T, WHOLE> piece;
    piece x[CH], u[CH], s[CH], dy[BACK ? CH : 1], dh[BACK ? CH : 1];
    __device__ static inline int col(int c) { return (c * W * 64 + (W == 1 ? threadIdx.x & 63 : threadIdx.x)) * piece::VE; }
    // tensors that are not there stand for x (what comes of them is not used, or taken for zero)
    __device__ inline void load(const NormArgs& g, int64_t row) {
        row = row < g.rows ? row : g.rows - 1;
        const T* px = reinterpret_cast<const T*>(g.x) + row * g.ld_x;
        const T* pu = g.u ? reinterpret_cast<const T*>(g.u) + row * g.ld_u : px;
        const T* ps = g.gate ? reinterpret_cast<const T*>(g.gate) + row * g.ld_g : px;
        const T* py = g.dy ? reinterpret_cast<const T*>(g.dy) + row * g.ld_x : px;
        const T* ph = g.dh ? reinterpret_cast<const T*>(g.dh) + row * g.ld_h : px;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            x[c].load(px, col(c), g.width);
            u[c].load(pu, col(c), g.width);
            s[c].load(ps, col(c), g.width);
            if (BACK) {
                dy[c].load(py, col(c), g.width);
                dh[c].load(ph, col(c), g.width);
            }
        }
    }
};
// ... and what becomes of it
template <typename T, int W, int CH>
struct NormRow {
    static constexpr int V = 16 / sizeof(T);
    float x[CH][V], u[CH][V], s[CH][V], n[CH][V];  // s: the gate; after value(): x is y, n the normed u
    float r_u, r_y;
    __device__ static inline int col(int c) { return NormInput<T, W, CH, true, false>::col(c); }
    template <bool WHOLE, bool BACK>
    __device__ inline void take(const NormInput<T, W, CH, WHOLE, BACK>& in, int width) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            values<T>(in.x[c].get(col(c), width), x[c]);
            values<T>(in.u[c].get(col(c), width), u[c]);
            values<T>(in.s[c].get(col(c), width), s[c]);
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
                r_u = __builtin_amdgcn_rsqf(row_sum<W>(q, lds) * g.over + g.eps);
            }
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    n[c][i] = u[c][i] * r_u * wo[c][i];
                    x[c][i] = __builtin_fmaf(g.gate ? sc[c][i] * sigmoid_of(s[c][i]) : sc[c][i], n[c][i], x[c][i]);
                }
        }
        r_y = 1.f;
        if (g.w_pre) {
            float q = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < V; ++i) q = __builtin_fmaf(x[c][i], x[c][i], q);
            r_y = __builtin_amdgcn_rsqf(row_sum<W>(q, lds) * g.over + g.eps);
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

template <typename T, int W, int CH, bool WHOLE>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void k_norm_fwd(NormArgs g) {
    constexpr int V = 16 / sizeof(T);
    __shared__ float lds[W];
    float sc[CH][V], wo[CH][V], wi[CH][V];
    columns<T, W, CH>(g, g.scale, sc);
    columns<T, W, CH>(g, g.w_post, wo);
    columns<T, W, CH>(g, g.w_pre, wi);
    const int64_t per = W == 1 ? 4 : 1, first = blockIdx.x * per + (W == 1 ? threadIdx.x >> 6 : 0);
    NormInput<T, W, CH, WHOLE, false> in;
    if (first < g.rows) in.load(g, first);
    for (int64_t row = first; row < g.rows; row += gridDim.x * per) {
        NormRow<T, W, CH> r;
        r.take(in, g.width);
        in.load(g, row + gridDim.x * per);  // the next one's
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

template <typename T, int W, int CH, bool WHOLE>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void k_norm_bwd(NormArgs g) {
    constexpr int V = 16 / sizeof(T), CAP = 64 * V * CH;  // columns of a wave
    __shared__ float lds[W];
    __shared__ float sums[W == 1 ? 3 * CAP : 1];
    float sc[CH][V], wo[CH][V], wi[CH][V], ds[CH][V], dwo[CH][V], dwi[CH][V];
    columns<T, W, CH>(g, g.scale, sc);
    columns<T, W, CH>(g, g.w_post, wo);
    columns<T, W, CH>(g, g.w_pre, wi);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) ds[c][i] = dwo[c][i] = dwi[c][i] = 0.f;
    const int64_t per = W == 1 ? 4 : 1, first = blockIdx.x * per + (W == 1 ? threadIdx.x >> 6 : 0);
    NormInput<T, W, CH, WHOLE, true> in;
    if (first < g.rows) in.load(g, first);
    for (int64_t row = first; row < g.rows; row += gridDim.x * per) {
        NormRow<T, W, CH> r;
        float dy[CH][V], dh[CH][V];
        r.take(in, g.width);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            values<T>(in.dy[c].get(r.col(c), g.width, g.dy != nullptr), dy[c]);
            values<T>(in.dh[c].get(r.col(c), g.width, g.dh != nullptr), dh[c]);
        }
        in.load(g, row + gridDim.x * per);  // the next one's
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
                const float2 sig = g.gate ? sigmoid_both(r.s[c][i]) : make_float2(1.f, 0.f);
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
// the workgroups' sums: 16 columns of the three to a block, 64 threads a column
__global__ __launch_bounds__(1024) void k_norm_columns(NormArgs g) {
    __shared__ float part[64][17];
    const int lane = threadIdx.x & 15, w = threadIdx.x >> 4, c = blockIdx.x * 16 + lane, all = 3 * g.width;
    float sum = 0.f;
    if (c < all) {
#pragma unroll 8
        for (int b = w; b < g.blocks; b += 64) sum += g.part[(int64_t)b * all + c];
    }
    part[w][lane] = sum;
    __syncthreads();
    for (int o = 32; o; o >>= 1) {
        if (w < o) part[w][lane] += part[w + o][lane];
        __syncthreads();
    }
    if (w || c >= all) return;
    const int k = c / g.width, at = c - k * g.width;
    float* out = k == 0 ? g.dscale : k == 1 ? g.dw_post : g.dw_pre;
    if (out) out[at] = part[0][lane];
}

static NormArgs norm_args(const morlax_norm_dims& d) {
    NormArgs g = {};
    g.rows = d.rows; g.width = d.width; g.eps = d.eps; g.over = 1.f / d.width;
    g.ld_x = d.ld_x; g.ld_u = d.ld_u; g.ld_g = d.ld_g; g.ld_h = d.ld_h;
    return g;
}
// Waves along a row: a lane holds one piece of 16 bytes (two in rows of more than 16 KB), as the backward keeps a piece's five tensors, their columns'
// weights and sums and the next row's pieces in registers (two pieces a lane: 304 of them).  Workgroups of four rows where one wave is enough.
static int norm_waves(const morlax_norm_dims& d) {
    const int pieces = (int)cdiv(d.width, d.dtype ? 8 : 4);
    int w = 1;
    while (w < 16 && 64 * w < pieces) w *= 2;
    return w;
}
static int norm_blocks(const morlax_norm_dims& d) {
    const int w = norm_waves(d);
    const int64_t all = cdiv(d.rows, w == 1 ? 4 : 1), most = w == 1 ? 768 : 4096 / w;  // (what the last launch adds up stays a few per cent of the rows)
    return (int)(all < 1 ? 1 : all < most ? all : most);
}
int64_t norm_ws_bytes(const morlax_norm_dims& d) { return (int64_t)norm_blocks(d) * 3 * d.width * 4; }

template <typename T, int W, int CH, bool WHOLE>
static void norm_run(const NormArgs& g, bool back, hipStream_t s) {
    constexpr int THREADS = W == 1 ? 256 : W * 64;
    if (back) {
        k_norm_bwd<T, W, CH, WHOLE><<<dim3(g.blocks), THREADS, 0, s>>>(g);
    } else {
        const int64_t all = cdiv(g.rows, W == 1 ? 4 : 1), most = W == 1 ? 4096 : 16384 / W;
        k_norm_fwd<T, W, CH, WHOLE><<<dim3((uint32_t)(all < most ? all : most)), THREADS, 0, s>>>(g);
    }
}
template <typename T, int W, int CH>
static void norm_pass(const NormArgs& g, bool back, hipStream_t s) {
    g.width % (16 / (int)sizeof(T)) == 0 ? norm_run<T, W, CH, true>(g, back, s) : norm_run<T, W, CH, false>(g, back, s);
}
template <typename T>
static void norm_pick(const NormArgs& g, int waves, bool back, hipStream_t s) {
    switch (waves) {
        case 1: norm_pass<T, 1, 1>(g, back, s); break;
        case 2: norm_pass<T, 2, 1>(g, back, s); break;
        case 4: norm_pass<T, 4, 1>(g, back, s); break;
        case 8: norm_pass<T, 8, 1>(g, back, s); break;
        default:
            if (sizeof(T) == 2 || g.width <= 4096) norm_pass<T, 16, 1>(g, back, s);
            else norm_pass<T, 16, sizeof(T) == 2 ? 1 : 2>(g, back, s);
    }
}
void launch_norm_fwd(const morlax_norm_dims& d, const void* x, const void* u, const void* gate, const float* scale, const float* w_post,
                     const float* w_pre, void* y, void* h, hipStream_t s) {
    NormArgs g = norm_args(d);
    g.x = x; g.u = u; g.gate = gate; g.scale = scale; g.w_post = w_post; g.w_pre = w_pre; g.y = y; g.h = h;
    if (d.dtype) norm_pick<bf16_t>(g, norm_waves(d), false, s);
    else norm_pick<float>(g, norm_waves(d), false, s);
}
void launch_norm_bwd(const morlax_norm_dims& d, const void* x, const void* u, const void* gate, const float* scale, const float* w_post,
                     const float* w_pre, const void* dy, const void* dh, void* dx, void* du, void* dgate, float* dscale, float* dw_post, float* dw_pre,
                     void* ws, hipStream_t s) {
    NormArgs g = norm_args(d);
    g.x = x; g.u = u; g.gate = gate; g.scale = scale; g.w_post = w_post; g.w_pre = w_pre; g.dy = dy; g.dh = dh;
    g.dx = dx; g.du = du; g.dgate = dgate; g.dscale = dscale; g.dw_post = dw_post; g.dw_pre = dw_pre;
    g.blocks = norm_blocks(d);
    if (dscale || dw_post || dw_pre) g.part = reinterpret_cast<float*>(ws);
    if (d.dtype) norm_pick<bf16_t>(g, norm_waves(d), true, s);
    else norm_pick<float>(g, norm_waves(d), true, s);
    if (g.part) k_norm_columns<<<dim3((uint32_t)cdiv(3 * (int64_t)d.width, 16)), 1024, 0, s>>>(g);
}
