// Memory over time for the policies: a short causal convolution and a selective state space scan, on time-major tensors [T, N, .]
// of N environments whose episodes begin where `first` says so (as the GAE scan's episode ends, a select: nothing before an
// episode's first step reaches it).
//
//   convolution  y[t, c] = act(b[c] + sum_k w[c, k] x[t - (width - 1) + k, c])        taps of the same episode
//   scan         h_t = e_t h_{t-1} + dt_t x_t B_t^T,  y_t = (h_t C_t + D x_t) silu(z_t),  dt = softplus(dt_raw + dt_bias), e = exp(dt a),
//                a = -exp(a_log), per environment and head; h [head_dim, state] fp32; e_t h_{t-1} is zero where an episode begins
//
// The scan runs on the matrix instructions, 32 steps at a time: with l_t the sum of dt a since the chunk's (or the episode's) start,
//   y_t = exp(l_t) C_t h_in + sum_{s <= t} exp(l_t - l_s) dt_s (C_t . B_s) x_s,   h_out = exp(l_31) h_in + sum_s exp(l_31 - l_s) dt_s B_s x_s^T.
// Every operand that is computed here (states, decays times scores) is fp32 and enters a product as bf16 parts (split3): the results are
// fp32 ones, rounded once where they are stored as bf16.
#include "mlp_device.h"
#include "memory_shape.h"

typedef short short4_t __attribute__((ext_vector_type(4)));

#define MEM_Q 32  // time steps of a chunk

// The end of a phase of a chunk's work: what one lane left in LDS is there for the others, and no instruction moves across (left to itself
// the scheduler starts every phase's reads at once, and hundreds of registers spill).
__device__ inline void phase() {
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_sched_barrier(0);
}
// The lane, as a value that the compiler cannot know to be the same in the next chunk: or it computes the addresses of all of a chunk's
// accesses once, ahead of the loop, and keeps some hundred of them in registers.
__device__ inline int lane_now() {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}

static int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

__device__ inline float silu_f(float v) { return v * __builtin_amdgcn_rcpf(1.f + __expf(-v)); }
__device__ inline float sigmoid_f(float v) { return __builtin_amdgcn_rcpf(1.f + __expf(-v)); }

// V consecutive values as they are in memory: one access, with the alignment of one element
template <typename T, int V> struct Run {
    typedef T vec_t __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    vec_t u;
    __device__ inline void load(const T* p) { u = *reinterpret_cast<const vec_t*>(p); }
    __device__ inline float get(int i) const { return (float)u[i]; }
};
template <typename T> struct Run<T, 1> {
    T u;
    __device__ inline void load(const T* p) { u = *p; }
    __device__ inline float get(int) const { return to_f(u); }
};
template <typename T, int V>
__device__ inline void store_run(T* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        *p = cvt<T>(v[0]);
    } else {
        typename Run<T, V>::vec_t u;
#pragma unroll
        for (int i = 0; i < V; ++i) u[i] = (T)v[i];
        *reinterpret_cast<typename Run<T, V>::vec_t*>(p) = u;
    }
}

// ---- convolution ----------------------------------------------------------------------------------------------------
#define CONV_W 4  // taps that a thread keeps: a shorter convolution's leading ones are absent
#define CONV_U 8      // time steps whose inputs a thread requests together: forward
#define CONV_U_BWD 4  // backward, which keeps more beside them (eight: 61 us instead of 45 for 32 x 1023 x 274 fp32)

struct ConvArgs {
    const void *x, *dy;
    const float *w, *b;
    const uint8_t* first;
    const void *state_in, *dstate_out;
    void *y, *state_out, *dx, *dstate_in;
    float *dw, *db, *part;
    int64_t x_t, x_n, y_t, y_n;
    int T, N, C, width, act, run, runs, nblocks;
};

// One thread's filters and the last inputs of its V channels (from channel c on) of one environment.
template <typename T, int V>
struct Taps {
    float w[CONV_W][V], b[V], win[CONV_W][V];
    __device__ inline void init(const ConvArgs& g, int c) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            b[i] = g.b ? g.b[c + i] : 0.f;
            if (g.width == CONV_W) {  // (w is 16-byte aligned: so is a filter of four)
                const float4_t f = *reinterpret_cast<const float4_t*>(g.w + (int64_t)(c + i) * CONV_W);
#pragma unroll
                for (int k = 0; k < CONV_W; ++k) w[k][i] = f[k];
            } else {
#pragma unroll
                for (int k = 0; k < CONV_W; ++k) {
                    const int q = k - (CONV_W - g.width);
                    const float f = g.w[(int64_t)(c + i) * g.width + (q < 0 ? 0 : q)];
                    w[k][i] = q < 0 ? 0.f : f;
                }
            }
        }
    }
    __device__ inline void push(const Run<T, V>& x, bool begins) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
#pragma unroll
            for (int k = 0; k + 1 < CONV_W; ++k) win[k][i] = begins ? 0.f : win[k + 1][i];
            win[CONV_W - 1][i] = x.get(i);
        }
    }
    // the inputs before step t0; returns the step among them at which an episode began last, or a very early one
    __device__ inline int before(const ConvArgs& g, const T* x, int n, int c, int t0) {
        const int before = g.width - 1;
        int e = -(1 << 30);
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int k = 0; k < CONV_W; ++k) win[k][i] = 0.f;
        Run<T, V> v[CONV_W - 1];
        bool begins[CONV_W - 1];
#pragma unroll
        for (int k = 0; k < CONV_W - 1; ++k) {  // input t0 - (CONV_W - 1) + k
            const int s = t0 - (CONV_W - 1) + k;
            begins[k] = false;
            v[k].u = (T)0.f;
            if (s < t0 - before) continue;
            if (s >= 0) {
                v[k].load(x + (int64_t)s * g.x_t);
                begins[k] = g.first && g.first[(int64_t)s * g.N + n];
            } else if (g.state_in) {
                v[k].load(reinterpret_cast<const T*>(g.state_in) + ((int64_t)n * before + s + before) * g.C + c);
            }
        }
#pragma unroll
        for (int k = 0; k < CONV_W - 1; ++k) {
            if (begins[k]) e = t0 - (CONV_W - 1) + k;
            push(v[k], begins[k]);
        }
        return e;
    }
    __device__ inline float sum(const ConvArgs& g, int i) const {
        float s = b[i];
#pragma unroll
        for (int k = 0; k < CONV_W; ++k)
            if (k >= CONV_W - g.width) s += w[k][i] * win[k][i];
        return s;
    }
};

// A thread takes V channels of one environment and a run of time steps, the last inputs in registers, the next CONV_U requested together.
// (The last V channels overlap with those before where V does not divide them: both threads write the same values.)  Bound by its
// reads and writes: a run's first width - 1 inputs are read again.  64 steps x 1024 environments x 640 channels bf16, 168 MB: 53 us, 3.2 TB/s.
template <typename T, int V>
__global__ __launch_bounds__(256) void k_conv_fwd(ConvArgs g) {
    const int cols = (g.C + V - 1) / V;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int n = (int)(id / cols);
    int c = (int)(id % cols) * V;
    c = c + V <= g.C ? c : g.C - V;
    if (n >= g.N) return;
    const int t0 = blockIdx.y * g.run, t1 = t0 + g.run < g.T ? t0 + g.run : g.T, before = g.width - 1;
    const T* x = reinterpret_cast<const T*>(g.x) + (int64_t)n * g.x_n + c;
    T* y = reinterpret_cast<T*>(g.y) + (int64_t)n * g.y_n + c;
    Taps<T, V> a;
    a.init(g, c);
    a.before(g, x, n, c, t0);
    for (int t = t0; t < t1; t += CONV_U) {
        Run<T, V> v[CONV_U];
        uint32_t first[CONV_U];
#pragma unroll
        for (int u = 0; u < CONV_U; ++u) {
            const int tt = t + u < t1 ? t + u : t1 - 1;
            v[u].load(x + (int64_t)tt * g.x_t);
            first[u] = g.first ? g.first[(int64_t)tt * g.N + n] : 0;
        }
#pragma unroll
        for (int u = 0; u < CONV_U; ++u) {
            if (t + u >= t1) break;
            a.push(v[u], first[u] != 0);
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float s = a.sum(g, i);
                o[i] = g.act ? silu_f(s) : s;
            }
            store_run<T, V>(y + (int64_t)(t + u) * g.y_t, o);
        }
    }
    if (t1 == g.T && g.state_out)
#pragma unroll
        for (int k = 1; k < CONV_W; ++k)
            if (k > CONV_W - g.width)
                store_run<T, V>(reinterpret_cast<T*>(g.state_out) + ((int64_t)n * before + k - (CONV_W - g.width) - 1) * g.C + c, a.win[k]);
}

// A thread's V channels of one environment after the other (n, n + stride, ..) and a run of time steps; it walks width - 1 steps
// beyond its run, whose gradients reach back into it.  dw and db: registers over its environments, then over the
// environments of its workgroup, then k_conv_final over the workgroups.  32 steps x 1023 x 274 channels fp32, 108 MB: 38 us and 5.
template <typename T, int V>
__global__ __launch_bounds__(256) void k_conv_bwd(ConvArgs g, int cols, int rows) {
    extern __shared__ float red[];  // [rows][CONV_W + 1][cols][V]
    const int col = threadIdx.x % cols, row = threadIdx.x / cols, chunk = blockIdx.x * cols + col;
    const bool live = row < rows && chunk * V < g.C;
    const int c = chunk * V + V <= g.C ? chunk * V : g.C - V;
    const int t0 = blockIdx.z * g.run, t1 = t0 + g.run < g.T ? t0 + g.run : g.T, before = g.width - 1;
    float dw[CONV_W + 1][V];
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int k = 0; k <= CONV_W; ++k) dw[k][i] = 0.f;
    if (live) {
        Taps<T, V> a;
        a.init(g, c);
        for (uint32_t at = blockIdx.y * rows + row; at < (uint32_t)g.N; at += gridDim.y * rows) {  // (N may be next to 2^31)
            const int n = (int)at;
            const T* x = reinterpret_cast<const T*>(g.x) + (int64_t)n * g.x_n + c;
            const T* dy = reinterpret_cast<const T*>(g.dy) + (int64_t)n * g.y_n + c;
            T* dx = reinterpret_cast<T*>(g.dx) + (int64_t)n * g.x_n + c;
            float pend[CONV_W][V];  // pend[k]: gradient so far of step t - (CONV_W - 1) + k
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int k = 0; k < CONV_W; ++k) pend[k][i] = 0.f;
            int e = a.before(g, x, n, c, t0);  // the step at which the episode of t began
            // gradient of input s is complete: what the state behind the last step passes back is added
            auto done = [&](int s, const float(&v)[V]) {
                float o[V];
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = v[i];
                if (g.dstate_out && s >= g.T - before && s >= e) {
                    Run<T, V> d;
                    d.load(reinterpret_cast<const T*>(g.dstate_out) + ((int64_t)n * before + s - (g.T - before)) * g.C + c);
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] += d.get(i);
                }
                if (s >= t0 && s < t1) store_run<T, V>(dx + (int64_t)s * g.x_t, o);
                else if (s < 0 && s >= -before && t0 == 0 && g.dstate_in)
                    store_run<T, V>(reinterpret_cast<T*>(g.dstate_in) + ((int64_t)n * before + s + before) * g.C + c, o);
            };
            const int end = t1 + before < g.T ? t1 + before : g.T;
            for (int t4 = t0; t4 < end; t4 += CONV_U_BWD) {
                Run<T, V> v[CONV_U_BWD], q[CONV_U_BWD];
                uint32_t first[CONV_U_BWD];
#pragma unroll
                for (int u = 0; u < CONV_U_BWD; ++u) {
                    const int tt = t4 + u < end ? t4 + u : end - 1;
                    v[u].load(x + (int64_t)tt * g.x_t);
                    q[u].load(dy + (int64_t)tt * g.y_t);
                    first[u] = g.first ? g.first[(int64_t)tt * g.N + n] : 0;
                }
#pragma unroll
                for (int u = 0; u < CONV_U_BWD; ++u) {
                    const int t = t4 + u;
                    if (t >= end) break;
                    if (first[u]) e = t;
                    a.push(v[u], first[u] != 0);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float d = q[u].get(i);
                        if (g.act) {
                            const float s = a.sum(g, i), sg = sigmoid_f(s);
                            d *= sg * (1.f + s * (1.f - sg));
                        }
                        if (t < t1) {
#pragma unroll
                            for (int k = 0; k < CONV_W; ++k)
                                if (k >= CONV_W - g.width) dw[k][i] += d * a.win[k][i];
                            dw[CONV_W][i] += d;
                        }
#pragma unroll
                        for (int k = 0; k < CONV_W; ++k)
                            if (k >= CONV_W - g.width && t - (CONV_W - 1) + k >= e) pend[k][i] += a.w[k][i] * d;
                    }
                    done(t - (CONV_W - 1), pend[0]);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
#pragma unroll
                        for (int k = 0; k + 1 < CONV_W; ++k) pend[k][i] = pend[k + 1][i];
                        pend[CONV_W - 1][i] = 0.f;
                    }
                }
            }
#pragma unroll
            for (int k = 0; k + 1 < CONV_W; ++k) done(end - (CONV_W - 1) + k, pend[k]);  // (end is T, or these lie beyond the run)
        }
    }
    const int per = cols * V * (CONV_W + 1);
    if (row < rows)
#pragma unroll
        for (int k = 0; k <= CONV_W; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) red[row * per + (k * cols + col) * V + i] = dw[k][i];
    __syncthreads();
    const int blk = blockIdx.z * gridDim.y + blockIdx.y;
    for (int i = threadIdx.x; i < per; i += 256) {
        const int k = i / (cols * V), ch = blockIdx.x * cols + i % (cols * V) / V;
        if (ch * V >= g.C) continue;
        float s = 0.f;
        for (int r = 0; r < rows; ++r) s += red[r * per + i];
        g.part[((int64_t)blk * (CONV_W + 1) + k) * g.C + (ch * V + V <= g.C ? ch * V : g.C - V) + i % V] = s;
    }
}
// the workgroups' sums: 32 of them a workgroup, eight groups of threads a contiguous eighth each, in order
__global__ __launch_bounds__(256) void k_conv_final(ConvArgs g) {
    __shared__ float sums[8][32];
    const int total = (CONV_W + 1) * g.C, i = blockIdx.x * 32 + threadIdx.x % 32, q = threadIdx.x / 32;
    const int each = (g.nblocks + 7) / 8, b1 = (q + 1) * each < g.nblocks ? (q + 1) * each : g.nblocks;
    float s = 0.f;
    if (i < total)
#pragma unroll 8
        for (int b = q * each; b < b1; ++b) s += g.part[(int64_t)b * total + i];
    sums[q][threadIdx.x % 32] = s;
    __syncthreads();
    if (q != 0 || i >= total) return;
    for (int j = 1; j < 8; ++j) s += sums[j][threadIdx.x];
    const int k = i / g.C, c = i % g.C;
    if (k == CONV_W) {
        if (g.db) g.db[c] = s;
    } else if (k >= CONV_W - g.width && g.dw) {
        g.dw[(int64_t)c * g.width + k - (CONV_W - g.width)] = s;
    }
}

// ---- scan: one wave a head of an environment ----------------------------------------------------------------------------
struct ScanArgs {
    const void *x, *b, *c, *dt, *z, *dy;
    const float *a_log, *d_skip, *dt_bias;
    const uint8_t* first;
    const float *state_in, *dstate_out;
    void *y, *dx, *db, *dc, *ddt, *dz;
    float *state_out, *dstate_in, *da_log, *dd_skip, *ddt_bias;
    float *saved;        // per (n, h): the state before each chunk, as the registers hold it
    float *pb, *pc;      // [head block][T][N][G][S] sums of dB, dC where a group's heads need several workgroups
    float *ph;           // [3][H][N][spans] sums of da, dD, ddt_bias
    float *ends;         // [N H][spans] states that a span leaves or takes over, as the registers hold them
    float *left;         // [N H][spans] what is left of a state over a span
    int64_t x_t, x_n, z_t, z_n, dt_t, dt_n, y_t, y_n;
    int T, N, H, P, G, S, chunks, head_blocks;
    int span, spans;     // time steps that one wave takes, a multiple of MEM_Q, and their number
};

template <typename T> struct Planes { static constexpr int N = sizeof(T) == 4 ? 3 : 1; };

// Eight consecutive values of a row of `width` at column 8 c8 as they are in memory, zero where the row ends or `on` is false.  No branch
// goes by the lane: rows that are whole pieces of eight take one access (to the start of a row that exists, where there is none), others
// one a value.  (16-byte accesses need the alignment of one element only.)
template <typename T>
struct Eight {
    uint4 u[sizeof(T) / 2];
    typedef T vec_t __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    __device__ inline void load(const T* p) {
        const vec_t v = *reinterpret_cast<const vec_t*>(p);
        __builtin_memcpy(u, &v, sizeof(u));
    }
    __device__ inline void load(const T* row0, int64_t off, int c8, int width, bool on) {
        if (width % 8 == 0) {
            const bool have = on && 8 * c8 < width;
            const vec_t v = *reinterpret_cast<const vec_t*>(row0 + (have ? off + 8 * c8 : 0));
            __builtin_memcpy(u, &v, sizeof(u));
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) u[i] = make_uint4(have ? u[i].x : 0, have ? u[i].y : 0, have ? u[i].z : 0, have ? u[i].w : 0);
        } else {
            T e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool have = on && 8 * c8 + i < width;
                const T v = row0[have ? off + 8 * c8 + i : 0];
                e[i] = have ? v : (T)0.f;
            }
            __builtin_memcpy(u, e, sizeof(u));
        }
    }
    __device__ inline void get(float (&v)[8]) const {
        const uint32_t w[8] = {u[0].x, u[0].y, u[0].z, u[0].w, u[sizeof(T) / 2 - 1].x, u[sizeof(T) / 2 - 1].y, u[sizeof(T) / 2 - 1].z, u[sizeof(T) / 2 - 1].w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = sizeof(T) == 4 ? __uint_as_float(w[i]) : __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    // the larger of `top` and the magnitudes here, as bits: infinite and undefined values are the largest
    __device__ inline uint32_t largest(uint32_t top) const {
        const uint32_t w[8] = {u[0].x, u[0].y, u[0].z, u[0].w, u[sizeof(T) / 2 - 1].x, u[sizeof(T) / 2 - 1].y, u[sizeof(T) / 2 - 1].z, u[sizeof(T) / 2 - 1].w};
        typedef unsigned short half_t __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < (sizeof(T) == 4 ? 8 : 4); ++i) {
            if (sizeof(T) == 4) {
                const uint32_t m = w[i] & 0x7fffffffu;
                top = m > top ? m : top;
            } else {
                top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(half_t, w[i] & 0x7fff7fffu), __builtin_bit_cast(half_t, top)));
            }
        }
        return top;
    }
    __device__ static inline bool finite(uint32_t top) { return sizeof(T) == 4 ? top < 0x7f800000u : (top & 0xffffu) < 0x7f80u && top >> 16 < 0x7f80u; }
};
__device__ inline void parts8(const Eight<bf16_t>& e, uint4 (&p)[1]) { p[0] = e.u[0]; }
__device__ inline void parts8(const Eight<float>& e, uint4 (&p)[3]) {
    float v[8];
    e.get(v);
    split3(v, p);
}
// eight values as two or three parts: two leave out 2^-17 of them, where the result is rounded to bf16 anyway
__device__ inline void split_parts(const float (&v)[8], uint4 (&p)[3]) { split3(v, p); }
__device__ inline void split_parts(const float (&v)[8], uint4 (&p)[2]) {
    float l[8];
    p[0] = pack_chunk<bf16_t>(v);
    const uint32_t w[4] = {p[0].x, p[0].y, p[0].z, p[0].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) l[i] = v[i] - __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    p[1] = pack_chunk<bf16_t>(l);
}
// a += sum of products of parts i, j with i + j <= 2, smallest first.  MIRROR: in the order that gives each element the bits that the product
// with a and b exchanged gives it.
template <bool MIRROR = false, int NA, int NB>
__device__ inline void mma_p(const uint4 (&a)[NA], const uint4 (&b)[NB], float16_t& c) {
#pragma unroll
    for (int s = (NA + NB - 2 < 2 ? NA + NB - 2 : 2); s >= 0; --s)
#pragma unroll
        for (int k = 0; k <= s; ++k) {
            const int i = MIRROR ? s - k : k;
            if (i < NA && s - i < NB) Mma32<bf16_t>::run(a[i], b[s - i], c);
        }
}
// The same with all but the leading product in a sum of their own.  A matrix instruction cuts what lies below its sum's last place, towards the
// lower value: six on one sum left it lower by a tenth of its rounding errors' size, always, and a sum over all steps of such values, as the
// decays' gradient is, kept it: da_log's error was 3.6e-6 of 64 x 512 x 8 heads, 6.5e-7 with this and the pairs' sum (between) of either sign.
template <bool MIRROR = false, int NA, int NB>
__device__ inline void mma_p2(const uint4 (&a)[NA], const uint4 (&b)[NB], float16_t& c, float16_t& low) {
#pragma unroll
    for (int s = (NA + NB - 2 < 2 ? NA + NB - 2 : 2); s >= 1; --s)
#pragma unroll
        for (int k = 0; k <= s; ++k) {
            const int i = MIRROR ? s - k : k;
            if (i < NA && s - i < NB) Mma32<bf16_t>::run(a[i], b[s - i], low);
        }
    Mma32<bf16_t>::run(a[0], b[0], c);
}
__device__ inline void zero(float16_t& c) {
#pragma unroll
    for (int e = 0; e < 16; ++e) c[e] = 0.f;
}

// A tile of 32 time steps x 32 B columns in LDS, NP planes of bf16.  Contraction order of all products here: the sixteen indices of step
// kk are, for lane group lg, 16 kk + 4 lg + [0, 4) and 16 kk + 8 + 4 lg + [0, 4) -- the rows that a lane of an accumulator holds, so that
// accumulators become operands without moving between lanes.
template <int B, int NP>
struct Tile {
    static constexpr int PITCH = 64 * B + 16, PLANE = 32 * PITCH, BYTES = NP * PLANE;
    unsigned char* at;
    // operand: row lr, contraction over the columns
    __device__ inline void rows(int kk, uint4 (&f)[NP]) const {
        const int lane = lane_now(), lr = lane & 31, lg = lane >> 5;
#pragma unroll
        for (int q = 0; q < NP; ++q) {
            const unsigned char* s = at + q * PLANE + lr * PITCH + kk * 32 + lg * 8;
            const uint2 u = *reinterpret_cast<const uint2*>(s), v = *reinterpret_cast<const uint2*>(s + 16);
            f[q] = make_uint4(u.x, u.y, v.x, v.y);
        }
    }
    // operand: column 32 blk + lr, contraction over the time steps
    __device__ inline void cols(int blk, int kk, uint4 (&f)[NP]) const {
        typedef __attribute__((address_space(3))) short4_t lds_s4;
        const int lane = threadIdx.x & 63, lg = lane >> 5, a = lane & 15, q0 = (lane >> 4) & 1, e = a >> 2, c = a & 3;
#pragma unroll
        for (int q = 0; q < NP; ++q) {
            const unsigned char* s = at + q * PLANE + (16 * kk + 4 * lg + e) * PITCH + (32 * blk + 16 * q0 + 4 * c) * 2;
            const uint2 u = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)s));
            const uint2 v = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(s + 8 * PITCH)));
            f[q] = make_uint4(u.x, u.y, v.x, v.y);
        }
    }
    __device__ inline void put(int row, int c8, const uint4 (&p)[NP]) const {
#pragma unroll
        for (int q = 0; q < NP; ++q) *reinterpret_cast<uint4*>(at + q * PLANE + row * PITCH + c8 * 16) = p[q];
    }
    // four consecutive values of a row (whole again: the parts of a value add up to it)
    __device__ inline void get4(int row, int col, float (&v)[4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = 0.f;
#pragma unroll
        for (int q = NP - 1; q >= 0; --q) {
            const uint2 u = *reinterpret_cast<const uint2*>(at + q * PLANE + row * PITCH + col * 2);
            v[0] += __uint_as_float(u.x << 16); v[1] += __uint_as_float(u.x & 0xffff0000u);
            v[2] += __uint_as_float(u.y << 16); v[3] += __uint_as_float(u.y & 0xffff0000u);
        }
    }
};

// The rows t0 .. t0 + cnt - 1 of a tensor on their way to a tile (others zero), 2 B pieces of eight values a lane.  All of a chunk's tensors
// are requested before the first is put down: one latency, not one each.
template <typename T, int B>
struct Fetch {
    static constexpr int CH = 4 * B;
    Eight<T> v[2 * B];
    __device__ inline void request(const T* base, int64_t st, int t0, int cnt, int width) {
        const int lane = lane_now();
        if (cnt == MEM_Q && width == 32 * B) {  // a whole tile: nothing to leave out
            const T* p = base + (int64_t)t0 * st + (int64_t)(lane / CH) * st + lane % CH * 8;
            const int64_t step = (64 / CH) * st;
#pragma unroll
            for (int i = 0; i < 2 * B; ++i) v[i].load(p + i * step);
            return;
        }
#pragma unroll
        for (int i = 0; i < 2 * B; ++i) {
            const int row = i * (64 / CH) + lane / CH;
            v[i].load(base + (int64_t)t0 * st, row * st, lane % CH, width, row < cnt);
        }
    }
    // into the tile; whether a value is undefined or infinite
    template <int NP>
    __device__ inline bool put(const Tile<B, NP>& tile) const {
        const int lane = lane_now();
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 2 * B; ++i) {
            uint4 p[NP];
            parts8(v[i], p);
            tile.put(i * (64 / CH) + lane / CH, lane % CH, p);
            top = v[i].largest(top);
        }
        return !Eight<T>::finite(top);
    }
};
// dy silu(z) (without a gate: dy) into a tile, in three parts
template <typename T, int B>
__device__ inline bool put_dy(const Tile<B, 3>& tile, const Fetch<T, B>& dy, const Fetch<T, B>& z, bool gate) {
    constexpr int CH = 4 * B;
    const int lane = lane_now();
    float bad = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * B; ++i) {
        float v[8], zv[8];
        dy.v[i].get(v);
        if (gate) {
            z.v[i].get(zv);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= silu_f(zv[k]);
        }
        uint4 p[3];
        split3(v, p);
        tile.put(i * (64 / CH) + lane / CH, lane % CH, p);
#pragma unroll
        for (int k = 0; k < 8; ++k) bad += v[k] * 0.f;
    }
    return !(bad == 0.f);
}

// Time steps of a chunk: lane lr (both halves alike) holds step t0 + lr.
struct Steps {
    float dt, raw, hi, lo;  // dt; dt_raw + dt_bias; log2 of the decay since the chunk's or the episode's start, in two parts
    int e;                  // chunk step at which the episode of this step began, or -1: before the chunk
    bool begins;
};
__device__ inline float last_of(float v) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 31)); }
// small per-chunk arrays in LDS, for lanes that need them by accumulator row
struct StepLds { float hi[32], lo[32], dt[32], w[32]; };

template <typename T>
__device__ inline Steps steps(const ScanArgs& g, int n, int h, int t0, int cnt, double a2, float bias, StepLds* sl) {
    const int lane = lane_now(), lr = lane & 31;
    Steps s;
    const int r = lr < cnt ? lr : 0;
    const float raw = to_f(reinterpret_cast<const T*>(g.dt)[(int64_t)(t0 + r) * g.dt_t + (int64_t)n * g.dt_n + h]) + bias;
    const float soft = log1pf(expf(raw));
    s.raw = lr < cnt ? raw : 0.f;
    s.dt = lr < cnt ? (raw > 20.f ? raw : soft) : 0.f;
    s.begins = false;
    if (g.first) s.begins = lr < cnt && g.first[(int64_t)(t0 + r) * g.N + n] != 0;
    const uint32_t begun = (uint32_t)__ballot(s.begins) & (uint32_t)((2ull << lr) - 1);
    s.e = begun ? 31 - __clz(begun) : -1;
    // in 64 bits: a difference of two sums keeps its precision whatever they have grown to
    double l = s.begins ? 0.0 : (double)s.dt * a2;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double up = __shfl_up(l, o, 32);
        if (lr - o >= (s.e < 0 ? 0 : s.e)) l += up;
    }
    s.hi = (float)l;
    s.lo = (float)(l - (double)s.hi);
    if (!(__builtin_fabsf(s.lo) < __builtin_inff())) s.lo = 0.f;
    if (lane < 32) {
        sl->hi[lr] = s.hi;
        sl->lo[lr] = s.lo;
        sl->dt[lr] = s.dt;
    }
    return s;
}
__device__ inline float decay(float hi1, float lo1, float hi0, float lo0) { return __builtin_amdgcn_exp2f((hi1 - hi0) + (lo1 - lo0)); }
// v w, and zero where w is zero whatever v is: a step that does not count may hold anything.  (The instruction by the compiler's own name
// for it: written as assembly, it reads matrix results before they are there, since nobody puts the waits between.)
extern "C" __device__ float mul_zero_wins(float, float) __asm("llvm.amdgcn.fmul.legacy");
__device__ inline float counted(float v, float w) { return mul_zero_wins(v, w); }
__device__ inline int acc_row(int e, int lg) { return 8 * (e / 4) + 4 * lg + e % 4; }

template <int PB, int SB> constexpr int64_t per_state() { return (int64_t)SB * PB * 1024; }  // floats of one as the registers hold it
// a state [state][head_dim] of a head as accumulators: rows n, column p = lr
template <int PB, int SB>
struct State {
    float16_t v[SB][PB];
    __device__ inline void clear() {
#pragma unroll
        for (int s = 0; s < SB; ++s)
#pragma unroll
            for (int p = 0; p < PB; ++p) zero(v[s][p]);
    }
    // from / to [head_dim][state] in memory, whole lines an access: 32 rows at a time turned in `patch`, 32 rows of 32 SB + 4 floats
    static constexpr int TP = 32 * SB + 4;
    __device__ inline void load(const float* m, int P, int S, float* patch) {
        const int lane = threadIdx.x & 63, lr = lane & 31, lg = lane >> 5;
        const bool vec = S % 4 == 0 && (reinterpret_cast<uintptr_t>(m) & 15) == 0;
#pragma unroll
        for (int p = 0; p < PB; ++p) {
            const int rows = P - 32 * p < 32 ? P - 32 * p : 32, n = rows > 0 ? rows * S : 0;
            const float* from = m + (int64_t)32 * p * S;
            if (vec && S == 32 * SB && rows == 32) {
                float4_t f[4 * SB];
#pragma unroll
                for (int i = 0; i < 4 * SB; ++i) f[i] = *reinterpret_cast<const float4_t*>(from + 256 * i + 4 * lane);
#pragma unroll
                for (int i = 0; i < 4 * SB; ++i) *reinterpret_cast<float4_t*>(patch + (256 * i + 4 * lane) / (32 * SB) * TP + 4 * lane % (32 * SB)) = f[i];
            } else if (vec)
                for (int i = 4 * lane; i < n; i += 256) *reinterpret_cast<float4*>(patch + i / S * TP + i % S) = *reinterpret_cast<const float4*>(from + i);
            else
                for (int i = lane; i < n; i += 64) patch[i / S * TP + i % S] = from[i];
            phase();
#pragma unroll
            for (int s = 0; s < SB; ++s)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int nn = 32 * s + 8 * k + 4 * lg;
                    const float4 f = *reinterpret_cast<const float4*>(patch + lr * TP + nn);
                    v[s][p][4 * k] = nn < S && lr < rows ? f.x : 0.f;
                    v[s][p][4 * k + 1] = nn + 1 < S && lr < rows ? f.y : 0.f;
                    v[s][p][4 * k + 2] = nn + 2 < S && lr < rows ? f.z : 0.f;
                    v[s][p][4 * k + 3] = nn + 3 < S && lr < rows ? f.w : 0.f;
                }
            phase();
        }
    }
    __device__ inline void store(float* m, int P, int S, float* patch) const {
        const int lane = threadIdx.x & 63, lr = lane & 31, lg = lane >> 5;
        const bool vec = S % 4 == 0 && (reinterpret_cast<uintptr_t>(m) & 15) == 0;
#pragma unroll
        for (int p = 0; p < PB; ++p) {
            const int rows = P - 32 * p < 32 ? P - 32 * p : 32, n = rows > 0 ? rows * S : 0;
            float* to = m + (int64_t)32 * p * S;
#pragma unroll
            for (int s = 0; s < SB; ++s)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    *reinterpret_cast<float4*>(patch + lr * TP + 32 * s + 8 * k + 4 * lg) =
                        make_float4(v[s][p][4 * k], v[s][p][4 * k + 1], v[s][p][4 * k + 2], v[s][p][4 * k + 3]);
            phase();
            if (vec && S == 32 * SB && rows == 32) {
#pragma unroll
                for (int i = 0; i < 4 * SB; ++i)
                    *reinterpret_cast<float4*>(to + 256 * i + 4 * lane) =
                        *reinterpret_cast<const float4*>(patch + (256 * i + 4 * lane) / (32 * SB) * TP + 4 * lane % (32 * SB));
            } else if (vec)
                for (int i = 4 * lane; i < n; i += 256) *reinterpret_cast<float4*>(to + i) = *reinterpret_cast<const float4*>(patch + i / S * TP + i % S);
            else
                for (int i = lane; i < n; i += 64) to[i] = patch[i / S * TP + i % S];
            phase();
        }
    }
    // from / to the registers' own order: whole kilobytes an access
    __device__ inline void dump(float* m) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < SB * PB * 4; ++i)
            reinterpret_cast<float4*>(m)[i * 64 + lane] = make_float4(v[i / 4 / PB][i / 4 % PB][i % 4 * 4], v[i / 4 / PB][i / 4 % PB][i % 4 * 4 + 1],
                                                                      v[i / 4 / PB][i / 4 % PB][i % 4 * 4 + 2], v[i / 4 / PB][i / 4 % PB][i % 4 * 4 + 3]);
    }
    __device__ inline void undump(const float* m) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < SB * PB * 4; ++i) {
            const float4 f = reinterpret_cast<const float4*>(m)[i * 64 + lane];
            v[i / 4 / PB][i / 4 % PB][i % 4 * 4] = f.x;
            v[i / 4 / PB][i / 4 % PB][i % 4 * 4 + 1] = f.y;
            v[i / 4 / PB][i / 4 % PB][i % 4 * 4 + 2] = f.z;
            v[i / 4 / PB][i / 4 % PB][i % 4 * 4 + 3] = f.w;
        }
    }
};
// eight accumulator values (the second or first half of a block) as an operand's parts
template <int NP>
__device__ inline void acc_parts(const float16_t& a, int half, uint4 (&p)[NP]) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = a[8 * half + i];
    split_parts(v, p);
}
// the values of an operand's parts times eight factors, as parts again
template <int NP>
__device__ inline void scaled_parts(const uint4 (&f)[NP], const float (&w)[8], uint4 (&p)[3]) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
#pragma unroll
    for (int q = NP - 1; q >= 0; --q) {
        const uint32_t u[4] = {f[q].x, f[q].y, f[q].z, f[q].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] += __uint_as_float(u[i] << 16);
            v[2 * i + 1] += __uint_as_float(u[i] & 0xffff0000u);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = counted(v[i], w[i]);
    split3(v, p);
}
__device__ inline void eight(const float* a, int kk, float (&v)[8]) {  // values of the contraction indices of step kk
    const int lg = (threadIdx.x >> 5) & 1;
    const float4 u = *reinterpret_cast<const float4*>(a + 16 * kk + 4 * lg), w = *reinterpret_cast<const float4*>(a + 16 * kk + 8 + 4 * lg);
    v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w; v[4] = w.x; v[5] = w.y; v[6] = w.z; v[7] = w.w;
}

// results [column | time step] of a wave into `patch` as rows of 32 B + 4 floats
template <int B>
__device__ inline void to_rows(const float16_t (&o)[B], float* patch) {
    const int lane = threadIdx.x & 63, lr = lane & 31, lg = lane >> 5;
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            *reinterpret_cast<float4*>(patch + lr * (32 * B + 4) + 32 * b + 8 * k + 4 * lg) =
                make_float4(o[b][4 * k], o[b][4 * k + 1], o[b][4 * k + 2], o[b][4 * k + 3]);
}
// eight of a row's values to memory, as many as exist
template <typename T>
__device__ inline void store8_row(T* p, const float (&v)[8], int c8, int width, bool on) {
    typedef T vec_t __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    if (width % 8 == 0) {
        vec_t u;
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = (T)v[i];
        if (on && 8 * c8 < width) *reinterpret_cast<vec_t*>(p + 8 * c8) = u;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (on && 8 * c8 + i < width) p[8 * c8 + i] = cvt<T>(v[i]);
    }
}
// piece i of a lane's rows of a chunk: store(row pointer) where the tile is whole, as few address steps as the loads take
template <typename T, int B, typename F>
__device__ inline void store_tile(T* base, int64_t st, int t0, int cnt, int width, bool live, F values) {
    constexpr int CH = 4 * B;
    typedef T vec_t __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    const int lane = lane_now();
    if (cnt == MEM_Q && width == 32 * B && live) {
        T* p = base + (int64_t)t0 * st + (int64_t)(lane / CH) * st + lane % CH * 8;
        const int64_t step = (64 / CH) * st;
#pragma unroll
        for (int i = 0; i < 2 * B; ++i) {
            float v[8];
            values(i, i * (64 / CH) + lane / CH, lane % CH, v);
            vec_t u;
#pragma unroll
            for (int k = 0; k < 8; ++k) u[k] = (T)v[k];
            *reinterpret_cast<vec_t*>(p + i * step) = u;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 2 * B; ++i) {
        const int row = i * (64 / CH) + lane / CH;
        float v[8];
        values(i, row, lane % CH, v);
        store8_row(base + (int64_t)(t0 + row) * st, v, lane % CH, width, live && row < cnt);
    }
}
__device__ inline void patch8(const float* row, int c8, float (&v)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(row + 8 * c8), b = *reinterpret_cast<const float4*>(row + 8 * c8 + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
// The wave's index as a scalar: environment, head and every pointer that follows from it are then in scalar registers, and a branch on
// them is a scalar one.  (With the index in the lanes, `if (z)` cost a mask of lanes, and the compiler, out of registers in the
// backward, moved 26 of them into the accumulation file ahead of the place where the lanes come back: with no gate, none was on.)
__device__ inline int wave_index() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

template <typename T, int PB, int SB>
struct ScanFwdLds {
    static constexpr int NP = Planes<T>::N;
    static constexpr int NW = sizeof(T) == 4 ? 2 : 4;  // waves of a workgroup
    static constexpr int X = Tile<PB, NP>::BYTES, N = Tile<SB, NP>::BYTES;
    static constexpr int WAVE = X + 2 * N + (int)sizeof(StepLds);
};

// Bound by its reads and writes, half of them the states: 64 steps x 1024 environments x 8 heads of 64 x 64 bf16, 487 MB in 121 us, 4.0 TB/s.
// One wave a head keeps the state in registers over the whole segment.  Rounding: operands as bf16 parts (three in fp32 and where a state
// follows; two, which leave out 2^-17, where only a bf16 y does), sums and states in fp32, y once.
// LOCAL: only the state that a span of time leaves when nothing enters it, and what it leaves of a state that does.  (Where environments
// and heads are too few to fill the machine, time is cut into spans: LOCAL for all of them at once, k_scan_join one after the other, then the
// outputs of all of them at once.)
template <typename T, int PB, int SB, bool LOCAL>
__global__ __launch_bounds__((ScanFwdLds<T, PB, SB>::NW * 64), 2) void k_scan_fwd(ScanArgs g) {
    typedef ScanFwdLds<T, PB, SB> L;
    constexpr int NP = L::NP, NY = sizeof(T) == 4 ? 3 : 2;  // parts of what only y sees
    extern __shared__ __align__(16) unsigned char lds[];
    const int wave = wave_index(), lane = threadIdx.x & 63, lr = lane & 31, lg = lane >> 5;
    const int64_t unit = (int64_t)blockIdx.x * L::NW + wave;
    if (unit >= (int64_t)g.N * g.H * g.spans) return;
    const int64_t id = unit / g.spans;
    const int span = (int)(unit % g.spans), t_begin = span * g.span, t_end = t_begin + g.span < g.T ? t_begin + g.span : g.T;
    const int n = (int)(id / g.H), h = (int)(id % g.H), grp = h / (g.H / g.G);
    unsigned char* own = lds + wave * L::WAVE;
    float* patch = reinterpret_cast<float*>(own);  // over the tiles, once they are done with
    const Tile<PB, NP> X = {own};
    const Tile<SB, NP> B = {own + L::X}, C = {own + L::X + L::N};
    StepLds* sl = reinterpret_cast<StepLds*>(own + L::X + 2 * L::N);
    const T* x = reinterpret_cast<const T*>(g.x) + (int64_t)n * g.x_n + (int64_t)h * g.P;
    const T* b = reinterpret_cast<const T*>(g.b) + (int64_t)n * g.x_n + (int64_t)grp * g.S;
    const T* c = reinterpret_cast<const T*>(g.c) + (int64_t)n * g.x_n + (int64_t)grp * g.S;
    const T* z = g.z ? reinterpret_cast<const T*>(g.z) + (int64_t)n * g.z_n + (int64_t)h * g.P : nullptr;
    T* y_out = reinterpret_cast<T*>(g.y) + (int64_t)n * g.y_n + (int64_t)h * g.P;
    const double a2 = -(double)expf(g.a_log[h]) * 1.4426950408889634;
    const float dskip = g.d_skip ? g.d_skip[h] : 0.f, bias = g.dt_bias ? g.dt_bias[h] : 0.f;
    const int64_t per = (int64_t)SB * PB * 1024;
    State<PB, SB> st;
    if (LOCAL) st.clear();
    else if (g.spans > 1) st.undump(g.ends + unit * per);
    else if (g.state_in) st.load(g.state_in + id * g.P * g.S, g.P, g.S, patch);
    else st.clear();
    float* saved = !LOCAL && g.saved ? g.saved + id * g.chunks * per : nullptr;
    float all = 1.f;  // LOCAL: what is left of a state that enters the span
    int slow = 0;  // steps to take one by one: a chunk with an undefined or infinite input, which would reach others through products with zero
    for (int t = t_begin; t < t_end;) {
        int cnt = t_end - t < MEM_Q ? t_end - t : MEM_Q;
        if (slow) cnt = 1;
        Fetch<T, PB> fx, fz;
        Fetch<T, SB> fb, fc;
        fx.request(x, g.x_t, t, cnt, g.P);
        fb.request(b, g.x_t, t, cnt, g.S);
        if (!LOCAL) {
            fc.request(c, g.x_t, t, cnt, g.S);
            if (z) fz.request(z, g.z_t, t, cnt, g.P);
        }
        phase();
        if (__any(fx.put(X)) && cnt > 1) {
            slow = cnt;
            continue;
        }
        fb.put(B);
        if (!LOCAL) fc.put(C);
        phase();
        const Steps s = steps<T>(g, n, h, t, cnt, a2, bias, sl);
        // the last step's sums: decay to the chunk's end
        const float hiq = last_of(s.hi), loq = last_of(s.lo);
        const int eq = __builtin_amdgcn_readlane(s.e, 31);
        const float w = lr >= eq ? s.dt * decay(hiq, loq, s.hi, s.lo) : 0.f;
        if (lane < 32) sl->w[lr] = w;
        phase();
        if (saved && t % MEM_Q == 0) st.dump(saved + (t / MEM_Q) * per);
        // scores [s | t] and what the state gives, [p | t]
        float16_t m, y[PB];
        if (!LOCAL) {
            zero(m);
#pragma unroll
            for (int p = 0; p < PB; ++p) zero(y[p]);
#pragma unroll
            for (int kk = 0; kk < 2 * SB; ++kk) {
                uint4 ob[NP], oc[NP], fh[NY];
                C.rows(kk, oc);
                B.rows(kk, ob);
                mma_p(ob, oc, m);
#pragma unroll
                for (int p = 0; p < PB; ++p) {
                    acc_parts(st.v[kk / 2][p], kk % 2, fh);
                    mma_p(fh, oc, y[p]);
                }
            }
            const float in = s.e < 0 ? __builtin_amdgcn_exp2f(s.hi + s.lo) : 0.f;
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int e = 0; e < 16; ++e) y[p][e] = counted(y[p][e], in);
#pragma unroll
            for (int k4 = 0; k4 < 4; ++k4) {
                const int r0 = 8 * k4 + 4 * lg;
                const float4 hi = *reinterpret_cast<const float4*>(sl->hi + r0), lo = *reinterpret_cast<const float4*>(sl->lo + r0),
                             dt = *reinterpret_cast<const float4*>(sl->dt + r0);
                const float a[4] = {hi.x, hi.y, hi.z, hi.w}, bb[4] = {lo.x, lo.y, lo.z, lo.w}, d[4] = {dt.x, dt.y, dt.z, dt.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool on = r0 + i <= lr && r0 + i >= s.e;
                    m[4 * k4 + i] = counted(m[4 * k4 + i], on ? d[i] * decay(s.hi, s.lo, a[i], bb[i]) : 0.f);
                }
            }
        }
        phase();
        // state to the chunk's end: what is left of the old one
        const float left = eq < 0 ? __builtin_amdgcn_exp2f(hiq + loq) : 0.f;
        if (LOCAL) all = counted(all, left);  // (an episode's begin wins over an undefined step of another chunk)
#pragma unroll
        for (int i = 0; i < SB; ++i)
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int e = 0; e < 16; ++e) st.v[i][p][e] = counted(st.v[i][p][e], left);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            uint4 fm[NY], ox[PB][NP];
            if (!LOCAL) acc_parts(m, kk, fm);
#pragma unroll
            for (int p = 0; p < PB; ++p) {
                X.cols(p, kk, ox[p]);
                if (!LOCAL) mma_p(ox[p], fm, y[p]);
            }
            float wk[8];
            eight(sl->w, kk, wk);
#pragma unroll
            for (int i = 0; i < SB; ++i) {
                uint4 ob[NP], fw[3];
                B.cols(i, kk, ob);
                scaled_parts(ob, wk, fw);
#pragma unroll
                for (int p = 0; p < PB; ++p) mma_p(fw, ox[p], st.v[i][p]);
            }
        }
        phase();
        if (!LOCAL) {  // d x joins y; then rows, gated, eight values a lane
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int k4 = 0; k4 < 4; ++k4) {
                    float xv[4];
                    X.get4(lr, 32 * p + 8 * k4 + 4 * lg, xv);
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[p][4 * k4 + i] += dskip * xv[i];
                }
            phase();
            to_rows(y, patch);
            phase();
            store_tile<T, PB>(y_out, g.y_t, t, cnt, g.P, true, [&](int i, int row, int c8, float(&v)[8]) {
                patch8(patch + row * (32 * PB + 4), c8, v);
                if (z) {
                    float zv[8];
                    fz.v[i].get(zv);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] *= silu_f(zv[k]);
                }
            });
        }
        phase();
        t += cnt;
        if (slow) --slow;
    }
    if (LOCAL) {
        st.dump(g.ends + unit * per);
        if (lane == 0) g.left[unit] = all;
        return;
    }
    if (g.state_out && g.spans == 1)  // (of several spans k_scan_join has left it)
        st.store(g.state_out + id * g.P * g.S, g.P, g.S, patch);
}

// The states between the spans of an environment's head, a thread four values of the register order: what span i leaves is replaced by what
// enters it.  REVERSE: the gradients of states, from the last span to the first.
template <int PB, int SB, bool REVERSE>
__global__ __launch_bounds__(256) void k_scan_join(ScanArgs g) {
    constexpr int per = SB * PB * 1024;
    const int64_t id = blockIdx.x;
    const int i = blockIdx.y * 256 + threadIdx.x, blk = i / 256, lane = i % 64;
    // values 4 k .. 4 k + 3 of block (s, p), k = i / 64 % 4: states 32 s + 8 k + 4 lg + [0, 4) of channel 32 p + lr
    const int nn = 32 * (blk / PB) + 8 * (i / 64 % 4) + 4 * (lane / 32), pp = 32 * (blk % PB) + lane % 32;
    const float* from = REVERSE ? g.dstate_out : g.state_in;
    float* to = REVERSE ? g.dstate_in : g.state_out;
    const int64_t at = (id * g.P + pp) * g.S + nn;
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = from && pp < g.P && nn + k < g.S ? from[at + k] : 0.f;
    float4* ends = reinterpret_cast<float4*>(g.ends + id * g.spans * per) + i;
    const float* left = g.left + id * g.spans;
#pragma unroll 4
    for (int q = 0; q < g.spans; ++q) {
        const int span = REVERSE ? g.spans - 1 - q : q;
        const float4 gave = ends[(int64_t)span * (per / 4)];
        const float l = left[span];
        ends[(int64_t)span * (per / 4)] = make_float4(v[0], v[1], v[2], v[3]);
        v[0] = (l != 0.f ? l * v[0] : 0.f) + gave.x;
        v[1] = (l != 0.f ? l * v[1] : 0.f) + gave.y;
        v[2] = (l != 0.f ? l * v[2] : 0.f) + gave.z;
        v[3] = (l != 0.f ? l * v[3] : 0.f) + gave.w;
    }
    if (to && pp < g.P)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (nn + k < g.S) to[at + k] = v[k];
}

// ---- backward of the scan: the chunks in reverse, a workgroup of NW waves taking heads of one group, whose dB and dC it adds up ----
// With dh the gradient of the state behind a chunk, R[t, s] = dy_t . x_s, E[t, s] the decay between steps, u_s that to the chunk's end and q_t that
// from its start (zero across an episode's begin):
//   dC_t = sum_s E R dt_s B_s + q_t h_in dy_t,           dB_s = dt_s dB'_s,  dB'_s = sum_t E R C_t + u_s dh x_s,
//   dx_s = dt_s (sum_t E (C_t . B_s) dy_t + u_s dh^T B_s) + D dy_s,   dh_in = exp(l_31) dh + sum_t q_t C_t dy_t^T,
// and for the decays' exponents, whose gradient at step i is the sum over the pairs (t, s) that it lies between,
//   d(dt_i a) = sum_{s < i <= t} E (C_t . B_s) dt_s R[t, s] + sum_{t >= i} C_t . q_t h_in dy_t + sum_{s < i} dt_s B_s . u_s dh x_s + exp(l_31) <h_in, dh>,
// the first sum as a product of the pairs with a triangle of ones over t, then those s of i's own episode: every term is there once and nothing
// is taken away again.  (As a sum over t >= i of what the pairs with earlier steps give less what those with later ones do, all pairs of later steps
// come in and go out again: what they round to, and a step of a later episode that is undefined, stayed in the earlier steps' gradients.)
// Half the environments of the forward's example: 301 us.  Bound by instructions and their waits: 61 million of the vector unit's (99 us of its
// time) at one wave a SIMD, whose 477 registers and 37 KB of LDS leave no room for a second; 34 % of the cycles wait.
template <typename T, int PB, int SB>
struct ScanBwdLds {
    static constexpr int NP = Planes<T>::N;
    static constexpr int NW = sizeof(T) == 4 ? 2 : 4;
    static constexpr int X = Tile<PB, NP>::BYTES, N = Tile<SB, NP>::BYTES, DY = Tile<PB, 3>::BYTES;
    static constexpr int RED = 32 * (32 * (SB > PB ? SB : PB) + 4) * 4;  // one of dB, dC of a wave for the sum over the waves; dx, dz on their way to rows
    static constexpr int WAVE = X + 2 * N + DY + RED + (int)sizeof(StepLds);
};

template <typename T, int PB, int SB>
__global__ __launch_bounds__((ScanBwdLds<T, PB, SB>::NW * 64)) void k_scan_bwd(ScanArgs g) {
    typedef ScanBwdLds<T, PB, SB> L;
    constexpr bool FOLD = sizeof(T) == 4 && PB * SB == 4;  // no registers for both blocks' small products: with it and without, us: 256 environments fp32 64 x 64 469 and 498, 512 bf16 389 and 387
    constexpr int NP = L::NP, NW = L::NW, RP = 32 * SB + 4, NY = sizeof(T) == 4 ? 3 : 2;  // NY: parts of what only dz and dx see
    extern __shared__ __align__(16) unsigned char lds[];
    const int wave = wave_index(), lane = threadIdx.x & 63, lr = lane & 31, lg = lane >> 5;
    const int rep = g.H / g.G;
    int64_t blk = blockIdx.x;
    const int hb = (int)(blk % g.head_blocks);
    blk /= g.head_blocks;
    const int grp = (int)(blk % g.G);
    blk /= g.G;
    const int span = (int)(blk % g.spans), n = (int)(blk / g.spans);
    const int t_begin = span * g.span, t_last = t_begin + g.span < g.T ? t_begin + g.span : g.T;
    const bool live = hb * NW + wave < rep;   // (a wave without a head runs along on another's inputs and leaves nothing)
    const int h = grp * rep + (live ? hb * NW + wave : rep - 1);
    const int64_t id = (int64_t)n * g.H + h;
    unsigned char* own = lds + wave * L::WAVE;
    const Tile<PB, NP> X = {own};
    const Tile<SB, NP> B = {own + L::X}, C = {own + L::X + L::N};
    const Tile<PB, 3> D = {own + L::X + 2 * L::N};
    float* red = reinterpret_cast<float*>(own + L::X + 2 * L::N + L::DY);
    StepLds* sl = reinterpret_cast<StepLds*>(own + L::X + 2 * L::N + L::DY + L::RED);
    const T* x = reinterpret_cast<const T*>(g.x) + (int64_t)n * g.x_n + (int64_t)h * g.P;
    const T* b = reinterpret_cast<const T*>(g.b) + (int64_t)n * g.x_n + (int64_t)grp * g.S;
    const T* c = reinterpret_cast<const T*>(g.c) + (int64_t)n * g.x_n + (int64_t)grp * g.S;
    const T* dy = reinterpret_cast<const T*>(g.dy) + (int64_t)n * g.y_n + (int64_t)h * g.P;
    const T* z = g.z ? reinterpret_cast<const T*>(g.z) + (int64_t)n * g.z_n + (int64_t)h * g.P : nullptr;
    const float av = -expf(g.a_log[h]);
    const double a2 = (double)av * 1.4426950408889634;
    const float dskip = g.d_skip ? g.d_skip[h] : 0.f, bias = g.dt_bias ? g.dt_bias[h] : 0.f;
    const int64_t per = (int64_t)SB * PB * 1024;
    const float* saved = g.saved + id * g.chunks * per;
    State<PB, SB> dh1;
    if (g.spans > 1) dh1.undump(g.ends + (id * g.spans + span) * per);
    else if (g.dstate_out) dh1.load(g.dstate_out + id * g.P * g.S, g.P, g.S, red);
    else dh1.clear();
    float sum_a = 0.f, sum_d = 0.f, sum_b = 0.f;  // per lane: of its steps
    int slow = 0;
    for (int t_end = t_last; t_end > t_begin;) {
        const int base = (t_end - 1) / MEM_Q * MEM_Q;
        int t = base, cnt = t_end - base;
        if (slow) {
            t = t_end - 1;
            cnt = 1;
        }
        Fetch<T, PB> fx, fdy, fz;
        Fetch<T, SB> fb, fc;
        fx.request(x, g.x_t, t, cnt, g.P);
        fb.request(b, g.x_t, t, cnt, g.S);
        fc.request(c, g.x_t, t, cnt, g.S);
        fdy.request(dy, g.y_t, t, cnt, g.P);
        if (z) fz.request(z, g.z_t, t, cnt, g.P);
        // the state before step t
        State<PB, SB> hin;
        hin.undump(saved + (int64_t)(base / MEM_Q) * per);
        phase();
        bool bad = fx.put(X);
        bad |= fb.put(B);
        bad |= fc.put(C);
        bad |= put_dy(D, fdy, fz, z != nullptr);
        phase();
        if (__syncthreads_or(bad) && cnt > 1) {  // all waves step by step together
            slow = cnt;
            continue;
        }
        for (int q = base; q < t; ++q) {  // step by step: forward again from the chunk's start
            const float raw = to_f(reinterpret_cast<const T*>(g.dt)[(int64_t)q * g.dt_t + (int64_t)n * g.dt_n + h]) + bias;
            const float dt = raw > 20.f ? raw : log1pf(expf(raw)), e = __builtin_amdgcn_exp2f((float)((double)dt * a2));
            const bool begins = g.first && g.first[(int64_t)q * g.N + n];
#pragma unroll
            for (int p = 0; p < PB; ++p) {
                const float xv = 32 * p + lr < g.P ? to_f(x[(int64_t)q * g.x_t + 32 * p + lr]) * dt : 0.f;
#pragma unroll
                for (int i = 0; i < SB; ++i)
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const int nn = 32 * i + acc_row(k, lg);
                        const float bv = nn < g.S ? to_f(b[(int64_t)q * g.x_t + nn]) : 0.f;
                        hin.v[i][p][k] = (begins ? 0.f : e * hin.v[i][p][k]) + xv * bv;
                    }
            }
        }
        float through = 0.f;  // <h_in, dh>: the chunk's first state in its last
#pragma unroll
        for (int i = 0; i < SB; ++i)
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int e = 0; e < 16; ++e) through += hin.v[i][p][e] * dh1.v[i][p][e];
        for (int o = 32; o; o >>= 1) through += __shfl_xor(through, o);
        through = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(through)));
        phase();
        const Steps s = steps<T>(g, n, h, t, cnt, a2, bias, sl);
        const float hiq = last_of(s.hi), loq = last_of(s.lo);
        const int eq = __builtin_amdgcn_readlane(s.e, 31);
        const float us = lr >= eq ? decay(hiq, loq, s.hi, s.lo) : 0.f;                     // to the chunk's end
        const float qs = s.e < 0 ? __builtin_amdgcn_exp2f(s.hi + s.lo) : 0.f;              // from its start
        const float left = eq < 0 ? __builtin_amdgcn_exp2f(hiq + loq) : 0.f;                // over all of it
        if (lane < 32) sl->w[lr] = qs;
        phase();
        // scores and dy . x in both layouts: [s | t] (lane: the later step) and [t | s] (lane: the earlier one)
        float16_t g1, g2, r1, r2, l2;  // (r2 enters the decays' gradients, r1 dC alone)
        zero(g1); zero(g2); zero(r1); zero(r2); zero(l2);
#pragma unroll
        for (int kk = 0; kk < 2 * SB; ++kk) {
            uint4 ob[NP], oc[NP];
            C.rows(kk, oc);
            B.rows(kk, ob);
            mma_p(ob, oc, g1);
            mma_p<true>(oc, ob, g2);
        }
#pragma unroll
        for (int kk = 0; kk < 2 * PB; ++kk) {
            uint4 ox[NP], fd[3];
            X.rows(kk, ox);
            D.rows(kk, fd);
            mma_p(ox, fd, r1);
            mma_p2<true>(fd, ox, r2, l2);
        }
        phase();
        float col_tot = 0.f;  // B_s . dB'_s: the sum over the step and later ones of E scores R, and end_tot below
        // m1: scores that give y [s | t]; r1: E R dt_s [s | t]; g2: E scores [t | s]; r2: E R [t | s]; pairs: E scores R dt_s [t | s]
        float16_t m1, pairs;
        // the accumulator's rows (bit 8 (e / 4) + e % 4) that are steps of this one's episode: before it, up to it, from it on
        const uint32_t begun = (uint32_t)__ballot(s.begins), below = (1u << lr) - 1, next = begun & ~(2 * below + 1);
        const uint32_t rows_before = (below & ~(s.e < 0 ? 0u : (1u << s.e) - 1)) >> 4 * lg, rows_t = rows_before | (1u << lr) >> 4 * lg,
                       rows_s = (((next & -next) - 1) & ~below) >> 4 * lg;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int r = acc_row(e, lg);
            r2[e] += l2[e];
            const float rhi = sl->hi[r], rlo = sl->lo[r], rdt = sl->dt[r];
            const uint32_t bit = 1u << acc_row(e, 0);
            const bool on1 = (rows_t & bit) != 0, on2 = (rows_s & bit) != 0;
            const float x = (s.hi - rhi) + (s.lo - rlo), d = __builtin_amdgcn_exp2f(on1 ? x : -x);  // (one of the two, or a step and itself)
            const float d1 = on1 ? d * rdt : 0.f, d2 = on2 ? d : 0.f;
            m1[e] = counted(g1[e], d1);
            r1[e] = counted(r1[e], d1);
            g2[e] = counted(g2[e], d2);
            const float pair = counted(r2[e], g2[e]);
            col_tot += pair;
            pairs[e] = counted(pair, s.dt);
            r2[e] = counted(r2[e], d2);
        }
        float between = 0.f;  // the pairs of an earlier step with this or a later one: pairs [s | i] summed over t >= i, then over s < i
        {
            float16_t o;  // the first half of it added, the second taken from its opposite: what each is cut by has either sign
            zero(o);
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                uint4 fp[3];
                if (kk) o = -o;
                uint32_t w[4];  // ones where the contraction's step is i or later
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int t2 = acc_row(8 * kk + 2 * k, lg);
                    w[k] = (t2 >= lr ? 0x3f80u : 0u) | (t2 + 1 >= lr ? 0x3f800000u : 0u) | (kk ? 0x80008000u : 0u);
                }
                const uint4 ones = make_uint4(w[0], w[1], w[2], w[3]);
                acc_parts(pairs, kk, fp);
#pragma unroll
                for (int q = 2; q >= 0; --q) Mma32<bf16_t>::run(fp[q], ones, o);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) between -= rows_before & (1u << acc_row(e, 0)) ? o[e] : 0.f;
        }
        phase();
        // dz needs y again
        if (z && g.dz) {
            float16_t y[PB];
#pragma unroll
            for (int p = 0; p < PB; ++p) zero(y[p]);
#pragma unroll
            for (int kk = 0; kk < 2 * SB; ++kk) {
                uint4 oc[NP], fh[NY];
                C.rows(kk, oc);
#pragma unroll
                for (int p = 0; p < PB; ++p) {
                    acc_parts(hin.v[kk / 2][p], kk % 2, fh);
                    mma_p(fh, oc, y[p]);
                }
            }
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int e = 0; e < 16; ++e) y[p][e] = counted(y[p][e], qs);
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                uint4 fm[NY], ox[NP];
                acc_parts(m1, kk, fm);
#pragma unroll
                for (int p = 0; p < PB; ++p) {
                    X.cols(p, kk, ox);
                    mma_p(ox, fm, y[p]);
                }
            }
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int k4 = 0; k4 < 4; ++k4) {
                    float xv[4];
                    X.get4(lr, 32 * p + 8 * k4 + 4 * lg, xv);
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[p][4 * k4 + i] += dskip * xv[i];
                }
            to_rows(y, red);
            phase();
            T* dzo = reinterpret_cast<T*>(g.dz) + (int64_t)n * g.z_n + (int64_t)h * g.P;
            store_tile<T, PB>(dzo, g.z_t, t, cnt, g.P, live, [&](int i, int row, int c8, float(&v)[8]) {
                float dv[8], zv[8];
                patch8(red + row * (32 * PB + 4), c8, v);
                fdy.v[i].get(dv);
                fz.v[i].get(zv);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float sg = sigmoid_f(zv[k]);
                    v[k] *= dv[k] * sg * (1.f + zv[k] * (1.f - sg));
                }
            });
            phase();
        }
        phase();
        // dx [p | s]
        {
            float16_t o[PB];
#pragma unroll
            for (int p = 0; p < PB; ++p) zero(o[p]);
#pragma unroll
            for (int kk = 0; kk < 2 * SB; ++kk) {
                uint4 ob[NP], fh[NY];
                B.rows(kk, ob);
#pragma unroll
                for (int p = 0; p < PB; ++p) {
                    acc_parts(dh1.v[kk / 2][p], kk % 2, fh);
                    mma_p(fh, ob, o[p]);
                }
            }
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[p][e] = counted(o[p][e], us);
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                uint4 fm[NY], fd[3];
                acc_parts(g2, kk, fm);
#pragma unroll
                for (int p = 0; p < PB; ++p) {
                    D.cols(p, kk, fd);
                    mma_p(fd, fm, o[p]);
                }
            }
            phase();
            float dd = 0.f;
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int k4 = 0; k4 < 4; ++k4) {
                    float dv[4], xv[4];
                    D.get4(lr, 32 * p + 8 * k4 + 4 * lg, dv);
                    X.get4(lr, 32 * p + 8 * k4 + 4 * lg, xv);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        o[p][4 * k4 + i] = s.dt * o[p][4 * k4 + i] + dskip * dv[i];
                        dd += dv[i] * xv[i];
                    }
                }
            if (lr < cnt) sum_d += dd;
            to_rows(o, red);
            phase();
            T* dxo = reinterpret_cast<T*>(g.dx) + (int64_t)n * g.x_n + (int64_t)h * g.P;
            store_tile<T, PB>(dxo, g.x_t, t, cnt, g.P, live, [&](int, int row, int c8, float(&v)[8]) { patch8(red + row * (32 * PB + 4), c8, v); });
            phase();
        }
        // dC [n | t], dB' [n | s]
        float state_tot = 0.f, end_tot = 0.f;  // C_t . q_t h_in dy_t, B_s . u_s dh x_s
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float16_t o[SB], low[SB];
#pragma unroll
            for (int i = 0; i < SB; ++i) {
                zero(o[i]);
                zero(low[i]);
            }
            // contraction over p: h_in dy_t, dh x_s; both have p in their lanes, their blocks are turned in LDS
#pragma unroll
            for (int p = 0; p < PB; ++p) {
                uint4 ox[2][NP], od[2][3];
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    if (which) X.rows(2 * p + kk, ox[kk]);
                    else D.rows(2 * p + kk, od[kk]);
                }
#pragma unroll
                for (int i = 0; i < SB; ++i) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) red[acc_row(e, lg) * 36 + lr] = which ? dh1.v[i][p][e] : hin.v[i][p][e];
                    phase();
#pragma unroll
                    for (int kk = 0; kk < 2; ++kk) {
                        float v[8];
                        uint4 fh[3];
                        eight(red + lr * 36, kk, v);
                        split3(v, fh);
                        if (which) mma_p2(fh, ox[kk], o[i], low[i]);
                        else mma_p2(fh, od[kk], o[i], low[i]);
                    }
                    if (FOLD) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[i][e] += low[i][e];
                        zero(low[i]);
                    }
                    phase();
                }
            }
            phase();
            const float lane_scale = which ? us : qs;
#pragma unroll
            for (int i = 0; i < SB; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[i][e] = counted(FOLD ? o[i][e] : o[i][e] + low[i][e], lane_scale);
            {
                float tot = 0.f;
#pragma unroll
                for (int i = 0; i < SB; ++i)
#pragma unroll
                    for (int k4 = 0; k4 < 4; ++k4) {
                        float v[4];
                        if (which) B.get4(lr, 32 * i + 8 * k4 + 4 * lg, v);
                        else C.get4(lr, 32 * i + 8 * k4 + 4 * lg, v);
#pragma unroll
                        for (int k = 0; k < 4; ++k) tot += v[k] * o[i][4 * k4 + k];
                    }
                if (which) end_tot = tot;
                else state_tot = tot;
            }
            phase();
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                uint4 fv[3], f[NP];
                acc_parts(which ? r2 : r1, kk, fv);
#pragma unroll
                for (int i = 0; i < SB; ++i) {
                    if (which) C.cols(i, kk, f);
                    else B.cols(i, kk, f);
                    mma_p(f, fv, o[i]);
                }
            }
            phase();
#pragma unroll
            for (int i = 0; i < SB; ++i)
#pragma unroll
                for (int k4 = 0; k4 < 4; ++k4) {
                    const int n0 = 32 * i + 8 * k4 + 4 * lg;
                    float4 r;
                    const float sc = live ? (which ? s.dt : 1.f) : 0.f;
                    r.x = o[i][4 * k4] * sc; r.y = o[i][4 * k4 + 1] * sc; r.z = o[i][4 * k4 + 2] * sc; r.w = o[i][4 * k4 + 3] * sc;
                    *reinterpret_cast<float4*>(red + lr * RP + n0) = r;
                }
            __syncthreads();
            for (int i = threadIdx.x; i < cnt * 32 * SB; i += NW * 64) {
                const int tt = i / (32 * SB), nn = i % (32 * SB);
                if (nn >= g.S) continue;
                float v = 0.f;
#pragma unroll
                for (int q = 0; q < NW; ++q)
                    if (hb * NW + q < rep) v += reinterpret_cast<const float*>(lds + q * L::WAVE + L::X + 2 * L::N + L::DY)[tt * RP + nn];
                if (g.head_blocks == 1) {
                    T* o2 = reinterpret_cast<T*>(which ? g.db : g.dc) + (int64_t)(t + tt) * g.x_t + (int64_t)n * g.x_n + (int64_t)grp * g.S + nn;
                    *o2 = cvt<T>(v);
                } else {
                    (which ? g.pb : g.pc)[((((int64_t)hb * g.T + t + tt) * g.N + n) * g.G + grp) * g.S + nn] = v;
                }
            }
            __syncthreads();
        }
        // gradients of the steps
        {
            float acc = state_tot;
            col_tot += end_tot;
            acc += __shfl_xor(acc, 32);
            between += __shfl_xor(between, 32);
            col_tot += __shfl_xor(col_tot, 32);
            end_tot += __shfl_xor(end_tot, 32);
            float before = lr >= eq ? s.dt * end_tot : 0.f;  // (a select: a step of an episode that ends in the chunk may be undefined)
            if (lr >= cnt) acc = before = 0.f;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const float dn = __shfl_down(acc, o, 32), up = __shfl_up(before, o, 32);
                if (lr + o < 32) acc += dn;
                if (lr >= o) before += up;
            }
            before = __shfl_up(before, 1, 32);
            if (lr > 0) acc += before;
            acc += between + counted(through, left);
            if (s.begins) acc = 0.f;
            const float ddt = col_tot + av * acc;
            const float draw = s.raw > 20.f ? ddt : ddt * sigmoid_f(s.raw);
            if (lr < cnt && lg == 0) {
                sum_a += s.dt * acc;
                sum_b += draw;
                if (live) reinterpret_cast<T*>(g.ddt)[(int64_t)(t + lr) * g.dt_t + (int64_t)n * g.dt_n + h] = cvt<T>(draw);
            }
        }
        phase();
        // dh before the chunk
#pragma unroll
        for (int i = 0; i < SB; ++i)
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    dh1.v[i][p][e] = counted(dh1.v[i][p][e], left);
                }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            float qk[8];
            eight(sl->w, kk, qk);
            uint4 fd[PB][3];
#pragma unroll
            for (int p = 0; p < PB; ++p) D.cols(p, kk, fd[p]);
#pragma unroll
            for (int i = 0; i < SB; ++i) {
                uint4 f[NP], fq[3];
                C.cols(i, kk, f);
                scaled_parts(f, qk, fq);
#pragma unroll
                for (int p = 0; p < PB; ++p) mma_p(fq, fd[p], dh1.v[i][p]);
            }
        }
        __syncthreads();
        t_end -= cnt;
        if (slow) --slow;
    }
    if (!live) return;
    if (g.dstate_in && g.spans == 1) dh1.store(g.dstate_in + id * g.P * g.S, g.P, g.S, red);
    for (int o = 32; o; o >>= 1) {
        sum_a += __shfl_xor(sum_a, o);
        sum_d += __shfl_xor(sum_d, o);
        sum_b += __shfl_xor(sum_b, o);
    }
    if (lane == 0) {
        const int64_t parts = (int64_t)g.N * g.spans, at = (int64_t)n * g.spans + span;
        g.ph[h * parts + at] = sum_a * av;
        g.ph[((int64_t)g.H + h) * parts + at] = sum_d;
        g.ph[((int64_t)2 * g.H + h) * parts + at] = sum_b;
    }
}

// What a span of time adds to the gradient of the state before it when none enters from behind, and what it leaves of one that does.
template <typename T, int PB, int SB>
struct ScanBwdLocalLds {
    static constexpr int NP = Planes<T>::N;
    static constexpr int N = Tile<SB, NP>::BYTES, DY = Tile<PB, 3>::BYTES;
    static constexpr int WAVE = N + DY + (int)sizeof(StepLds);
};
template <typename T, int PB, int SB>
__global__ __launch_bounds__(256) void k_scan_bwd_local(ScanArgs g) {
    typedef ScanBwdLocalLds<T, PB, SB> L;
    constexpr int NP = L::NP;
    extern __shared__ __align__(16) unsigned char lds[];
    const int wave = wave_index(), lane = threadIdx.x & 63, lr = lane & 31;
    const int64_t unit = (int64_t)blockIdx.x * 4 + wave;
    if (unit >= (int64_t)g.N * g.H * g.spans) return;
    const int64_t id = unit / g.spans;
    const int span = (int)(unit % g.spans), t_begin = span * g.span, t_last = t_begin + g.span < g.T ? t_begin + g.span : g.T;
    const int n = (int)(id / g.H), h = (int)(id % g.H), grp = h / (g.H / g.G);
    unsigned char* own = lds + wave * L::WAVE;
    const Tile<SB, NP> C = {own};
    const Tile<PB, 3> D = {own + L::N};
    StepLds* sl = reinterpret_cast<StepLds*>(own + L::N + L::DY);
    const T* c = reinterpret_cast<const T*>(g.c) + (int64_t)n * g.x_n + (int64_t)grp * g.S;
    const T* dy = reinterpret_cast<const T*>(g.dy) + (int64_t)n * g.y_n + (int64_t)h * g.P;
    const T* z = g.z ? reinterpret_cast<const T*>(g.z) + (int64_t)n * g.z_n + (int64_t)h * g.P : nullptr;
    const double a2 = -(double)expf(g.a_log[h]) * 1.4426950408889634;
    const float bias = g.dt_bias ? g.dt_bias[h] : 0.f;
    State<PB, SB> dh;
    dh.clear();
    float all = 1.f;
    int slow = 0;
    for (int t_end = t_last; t_end > t_begin;) {
        int t = (t_end - 1) / MEM_Q * MEM_Q, cnt = t_end - t;
        if (slow) {
            t = t_end - 1;
            cnt = 1;
        }
        Fetch<T, SB> fc;
        Fetch<T, PB> fdy, fz;
        fc.request(c, g.x_t, t, cnt, g.S);
        fdy.request(dy, g.y_t, t, cnt, g.P);
        if (z) fz.request(z, g.z_t, t, cnt, g.P);
        phase();
        bool bad = fc.put(C);
        bad |= put_dy(D, fdy, fz, z != nullptr);
        if (__any(bad) && cnt > 1) {
            slow = cnt;
            continue;
        }
        const Steps s = steps<T>(g, n, h, t, cnt, a2, bias, sl);
        const float hiq = last_of(s.hi), loq = last_of(s.lo);
        const int eq = __builtin_amdgcn_readlane(s.e, 31);
        if (lane < 32) sl->w[lr] = s.e < 0 ? __builtin_amdgcn_exp2f(s.hi + s.lo) : 0.f;
        phase();
        const float left = eq < 0 ? __builtin_amdgcn_exp2f(hiq + loq) : 0.f;
        all = counted(all, left);
#pragma unroll
        for (int i = 0; i < SB; ++i)
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int e = 0; e < 16; ++e) dh.v[i][p][e] = counted(dh.v[i][p][e], left);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            float qk[8];
            eight(sl->w, kk, qk);
            uint4 fd[PB][3];
#pragma unroll
            for (int p = 0; p < PB; ++p) D.cols(p, kk, fd[p]);
#pragma unroll
            for (int i = 0; i < SB; ++i) {
                uint4 f[NP], fq[3];
                C.cols(i, kk, f);
                scaled_parts(f, qk, fq);
#pragma unroll
                for (int p = 0; p < PB; ++p) mma_p(fq, fd[p], dh.v[i][p]);
            }
        }
        phase();
        t_end -= cnt;
        if (slow) --slow;
    }
    dh.dump(g.ends + unit * per_state<PB, SB>());
    if (lane == 0) g.left[unit] = all;
}

// the sums over a group's head blocks, in order
template <typename T>
__global__ __launch_bounds__(256) void k_scan_bc(ScanArgs g) {
    const int64_t per = (int64_t)g.T * g.N * g.G * g.S;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < per; i += (int64_t)gridDim.x * 256) {
        const int s = (int)(i % g.S);
        int64_t k = i / g.S;
        const int grp = (int)(k % g.G);
        k /= g.G;
        const int n = (int)(k % g.N);
        const int64_t t = k / g.N, to = t * g.x_t + (int64_t)n * g.x_n + (int64_t)grp * g.S + s;
        float b = 0.f, c = 0.f;
        for (int q = 0; q < g.head_blocks; ++q) {
            b += g.pb[q * per + i];
            c += g.pc[q * per + i];
        }
        reinterpret_cast<T*>(g.db)[to] = cvt<T>(b);
        reinterpret_cast<T*>(g.dc)[to] = cvt<T>(c);
    }
}
// gradients of a_log, D and dt_bias: a head's sums over the environments
__global__ __launch_bounds__(256) void k_scan_heads(ScanArgs g) {
    __shared__ float part[4];
    const int h = blockIdx.x % g.H, which = blockIdx.x / g.H;
    float* out = which == 0 ? g.da_log : which == 1 ? g.dd_skip : g.ddt_bias;
    if (!out) return;
    const int64_t parts = (int64_t)g.N * g.spans;
    float s = 0.f;
    for (int64_t n = threadIdx.x; n < parts; n += 256) s += g.ph[((int64_t)which * g.H + h) * parts + n];
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) out[h] = part[0] + part[1] + part[2] + part[3];
}

// ---- a single time step: convolution, state and output of a head in one launch ------------------------------------------
struct StepArgs {
    ScanArgs s;
    const void *xbc, *conv_in;
    const float *conv_w, *conv_b;
    void* conv_out;
    int width;
    StepLayout lay;
};
// A wave takes a head of an environment, or one of `parts` equal runs of its channels where there are few heads in all (each computes the
// head's B and C for itself).  The convolution's outputs stay in fp32 in LDS; a row of the state (the state values of one channel) is shared
// by lpr lanes of four values each, or of single ones where rows are not whole 16-byte pieces; STEP_U rows a lane are requested together.
// Bound by the states, read and written once: 4096 environments x 8 heads of 64 x 64, 1.09 GB in 240 us, 4.5 TB/s; one environment 7.9 us.
// Runs of channels, us with and without: 1 environment 8 and 15, 127 13 and 19, 192 16 and 20, 255 24 and 21.
#define STEP_U 4
template <typename T>
__global__ __launch_bounds__(256) void k_memory_step(StepArgs a, int lpr, int vec, int parts) {
    extern __shared__ __align__(16) float slds[];
    const ScanArgs& g = a.s;
    const int wave = wave_index(), lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + wave;
    if (unit >= (int64_t)g.N * g.H * parts) return;
    const int64_t id = unit / parts;
    const int each = a.lay.each, q0 = (int)(unit % parts) * each, q1 = q0 + each < g.P ? q0 + each : g.P;  // its channels
    const int n = (int)(id / g.H), h = (int)(id % g.H), rep = g.H / g.G, grp = h / rep, D = g.H * g.P;
    const int chans = D + 2 * g.G * g.S, before = a.width - 1, np = q1 > q0 ? q1 - q0 : 0;
    float *bs = slds + wave * a.lay.wave + a.lay.b, *cs = bs + g.S, *xs = bs - np;  // one run of values
    const bool begins = g.first && g.first[n];
    const T* row = reinterpret_cast<const T*>(a.xbc) + (int64_t)n * g.x_n;
    const T* old = reinterpret_cast<const T*>(a.conv_in) + (int64_t)n * before * chans;
    T* kept = reinterpret_cast<T*>(a.conv_out) + (int64_t)n * before * chans;
    for (int i = lane; i < np + 2 * g.S; i += 64) {
        const int c = i < np ? h * g.P + q0 + i : i < np + g.S ? D + grp * g.S + i - np : D + g.G * g.S + grp * g.S + i - np - g.S;
        float v = a.conv_b ? a.conv_b[c] : 0.f;
        const bool mine = i < np || (h == grp * rep && q0 == 0);  // one wave of a group keeps its B and C
        T in[CONV_W];
        float w[CONV_W];
#pragma unroll
        for (int k = 0; k < CONV_W; ++k) {
            in[k] = (T)0.f;
            w[k] = 0.f;
            if (k < a.width) {
                w[k] = a.conv_w[(int64_t)c * a.width + k];
                if (k == before) in[k] = row[c];
                else if (a.conv_in && !begins) in[k] = old[(int64_t)k * chans + c];
            }
        }
#pragma unroll
        for (int k = 0; k < CONV_W; ++k) {
            if (k == before || (k < before && !begins)) v += w[k] * to_f(in[k]);
            if (k > 0 && k < a.width && mine && a.conv_out) kept[(int64_t)(k - 1) * chans + c] = in[k];
        }
        xs[i] = silu_f(v);
    }
    __builtin_amdgcn_wave_barrier();
    const float raw = to_f(reinterpret_cast<const T*>(g.dt)[(int64_t)n * g.dt_n + h]) + (g.dt_bias ? g.dt_bias[h] : 0.f);
    const float dt = raw > 20.f ? raw : log1pf(expf(raw));
    const float e = expf(-dt * expf(g.a_log[h])), dskip = g.d_skip ? g.d_skip[h] : 0.f;
    const bool have = g.state_in && !begins;
    const float* hi = have ? g.state_in + (id * g.P + q0) * g.S : g.state_out;  // (never read where there is none)
    float* ho = g.state_out + (id * g.P + q0) * g.S;
    const int sub = lane % lpr, rows = 64 / lpr;
    const T* z = reinterpret_cast<const T*>(g.z) + (int64_t)n * g.z_n + (int64_t)h * g.P + q0;
    T* yo = reinterpret_cast<T*>(g.y) + (int64_t)n * g.y_n + (int64_t)h * g.P + q0;
    float4_t bv = {}, cv = {};
    if (vec && 4 * sub < g.S) {
        bv = *reinterpret_cast<const float4_t*>(bs + 4 * sub);
        cv = *reinterpret_cast<const float4_t*>(cs + 4 * sub);
    }
    for (int p0 = 0; p0 < np; p0 += STEP_U * rows) {
        float y[STEP_U];
        if (vec) {
            float4_t v[STEP_U];
#pragma unroll
            for (int u = 0; u < STEP_U; ++u) {
                const int p = p0 + u * rows + lane / lpr;
                v[u] = float4_t{};
                if (have && p < np && 4 * sub < g.S) v[u] = *reinterpret_cast<const float4_t*>(hi + (int64_t)p * g.S + 4 * sub);
            }
#pragma unroll
            for (int u = 0; u < STEP_U; ++u) {
                const int p = p0 + u * rows + lane / lpr;
                const float xv = dt * xs[p < np ? p : 0];
                y[u] = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    v[u][k] = e * v[u][k] + xv * bv[k];
                    y[u] += v[u][k] * cv[k];
                }
                if (p < np && 4 * sub < g.S) *reinterpret_cast<float4_t*>(ho + (int64_t)p * g.S + 4 * sub) = v[u];
            }
        } else {
#pragma unroll
            for (int u = 0; u < STEP_U; ++u) {
                const int p = p0 + u * rows + lane / lpr;
                y[u] = 0.f;
                if (p < np && sub < g.S) {
                    const float v = (have ? e * hi[(int64_t)p * g.S + sub] : 0.f) + dt * xs[p] * bs[sub];
                    ho[(int64_t)p * g.S + sub] = v;
                    y[u] = v * cs[sub];
                }
            }
        }
#pragma unroll
        for (int u = 0; u < STEP_U; ++u) {
            for (int o = lpr / 2; o; o >>= 1) y[u] += __shfl_xor(y[u], o);
            const int p = p0 + u * rows + lane / lpr;
            if (p < np && sub == 0) {
                float v = y[u] + dskip * xs[p];
                if (g.z) v *= silu_f(to_f(z[p]));
                yo[p] = cvt<T>(v);
            }
        }
    }
}

// ---- host side ------------------------------------------------------------------------------------------------------
static void conv_runs(ConvArgs& g, int64_t threads) {
    // runs of time steps long enough that the steps before them, read again, do not count, where there are threads enough without
    int run = g.T;
    // (and no more runs than a grid has along y)
    while (run > 16 && threads * cdiv(g.T, run) < 256 * 1024 && g.T / 65535 < run / 4) run = (run + 1) / 2;
    g.run = run;
    g.runs = (int)cdiv(g.T, run);
}
static ConvArgs conv_args(const morlax_conv_dims& d) {
    ConvArgs g = {};
    g.T = d.T; g.N = d.N; g.C = d.channels; g.width = d.width; g.act = d.act;
    g.x_t = d.x_t; g.x_n = d.x_n; g.y_t = d.y_t; g.y_n = d.y_n;
    return g;
}
#define CONV_BLOCKS 512  // workgroups that leave sums, at most
int64_t conv_ws_bytes(const morlax_conv_dims& d) { return (int64_t)CONV_BLOCKS * (CONV_W + 1) * d.channels * 4; }
template <typename T, int V>
static void conv_fwd(ConvArgs& g, hipStream_t s) {
    const int64_t threads = cdiv(g.C, V) * g.N;
    conv_runs(g, threads);
    k_conv_fwd<T, V><<<dim3(cdiv(threads, 256), g.runs), 256, 0, s>>>(g);
}
void launch_conv_fwd(const morlax_conv_dims& d, const void* x, const float* w, const float* b, const uint8_t* first, const void* state_in, void* y,
                     void* state_out, hipStream_t s) {
    ConvArgs g = conv_args(d);
    g.x = x; g.w = w; g.b = b; g.first = first; g.state_in = state_in; g.y = y; g.state_out = state_out;
    if (d.dtype) {
        if (g.C >= 8) conv_fwd<bf16_t, 8>(g, s);
        else conv_fwd<bf16_t, 1>(g, s);
    } else {
        if (g.C >= 4) conv_fwd<float, 4>(g, s);
        else conv_fwd<float, 1>(g, s);
    }
}
template <typename T, int V>
static void conv_bwd(ConvArgs& g, hipStream_t s) {
    const int chunks = (int)cdiv(g.C, V);
    const int cols = (int)cdiv(chunks, cdiv(chunks, 64)), rows = 256 / cols;
    conv_runs(g, (int64_t)chunks * g.N);
    if (g.runs > CONV_BLOCKS) {
        g.run = (int)cdiv(g.T, CONV_BLOCKS);
        g.runs = (int)cdiv(g.T, g.run);
    }
    int64_t by = cdiv(g.N, rows);
    const int64_t most = CONV_BLOCKS / g.runs;
    if (by > most) by = most;
    g.nblocks = (int)(by * g.runs);
    k_conv_bwd<T, V><<<dim3(cdiv(chunks, cols), by, g.runs), 256, rows * cols * V * (CONV_W + 1) * 4, s>>>(g, cols, rows);
    k_conv_final<<<cdiv((CONV_W + 1) * (int64_t)g.C, 32), 256, 0, s>>>(g);
}
void launch_conv_bwd(const morlax_conv_dims& d, const void* x, const float* w, const float* b, const uint8_t* first, const void* state_in,
                     const void* dy, const void* dstate_out, void* dx, float* dw, float* db, void* dstate_in, void* ws, hipStream_t s) {
    ConvArgs g = conv_args(d);
    g.x = x; g.w = w; g.b = b; g.first = first; g.state_in = state_in; g.dy = dy; g.dstate_out = dstate_out;
    g.dx = dx; g.dw = dw; g.db = db; g.dstate_in = dstate_in; g.part = (float*)ws;
    if (d.dtype) {
        if (g.C >= 4) conv_bwd<bf16_t, 4>(g, s);
        else conv_bwd<bf16_t, 1>(g, s);
    } else {
        if (g.C >= 4) conv_bwd<float, 4>(g, s);
        else conv_bwd<float, 1>(g, s);
    }
}

// Spans of time: one where environments and heads fill the machine's SIMDs, or the segment is short; else as many as give every SIMD a
// wave, of two chunks at least (a span costs its inputs once more and a state to write and read).  us with and without, 64 x 64 bf16: 64
// waves of 32 chunks 38 and 190, 256 of 8 39 and 53, 512 of 32 169 and 196; but 384 of 8 57 and 54, 512 of 8 62 and 55.
static void scan_spans(ScanArgs& g) {
    const int64_t waves = (int64_t)g.N * g.H;
    g.spans = 1;
    g.span = g.chunks * MEM_Q;
    if (waves > 512 || g.chunks < (waves > 256 ? 32 : 8)) return;
    int64_t spans = cdiv(1024, waves);
    if (spans > g.chunks / 2) spans = g.chunks / 2;
    g.span = (int)(cdiv(g.chunks, spans) * MEM_Q);
    g.spans = (int)cdiv(g.T, g.span);
}
static ScanArgs scan_args(const morlax_scan_dims& d) {
    ScanArgs g = {};
    g.T = d.T; g.N = d.N; g.H = d.heads; g.P = d.head_dim; g.G = d.groups; g.S = d.state;
    g.x_t = d.x_t; g.x_n = d.x_n; g.z_t = d.z_t; g.z_n = d.z_n; g.dt_t = d.dt_t; g.dt_n = d.dt_n; g.y_t = d.y_t; g.y_n = d.y_n;
    g.chunks = (int)cdiv(d.T, MEM_Q);
    g.head_blocks = (int)cdiv(d.heads / d.groups, d.dtype ? 4 : 2);
    scan_spans(g);
    return g;
}
static int64_t scan_blocks(const ScanArgs& g) { return cdiv(g.P, 32) * cdiv(g.S, 32); }
int64_t scan_saved_bytes(const morlax_scan_dims& d) {
    const int64_t blocks = cdiv(d.head_dim, 32) * cdiv(d.state, 32);
    return (int64_t)d.N * d.heads * cdiv(d.T, MEM_Q) * blocks * 4096;
}
static int64_t scan_carve(ScanArgs& g, bool back, void* ws) {
    char* at = reinterpret_cast<char*>(ws);
    int64_t off = 0;
    auto take = [&](int64_t bytes) {
        float* q = ws ? (float*)(at + off) : nullptr;
        off += align_up(bytes, 256);
        return q;
    };
    if (g.spans > 1) {
        g.ends = take((int64_t)g.N * g.H * g.spans * scan_blocks(g) * 4096);
        g.left = take((int64_t)g.N * g.H * g.spans * 4);
    }
    if (back) {
        g.ph = take((int64_t)3 * g.H * g.N * g.spans * 4);
        const int64_t n = g.head_blocks > 1 ? (int64_t)g.head_blocks * g.T * g.N * g.G * g.S * 4 : 0;
        g.pb = take(n);
        g.pc = take(n);
    }
    return off > 0 ? off : 256;
}
int64_t scan_ws_bytes(const morlax_scan_dims& d, bool back) {
    ScanArgs g = scan_args(d);
    return scan_carve(g, back, nullptr);
}
// allows a kernel its LDS; 0 on success
static int allow_lds(const void* kernel, int bytes) {
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess) return 0;
    (void)hipGetLastError();
    return -1;
}
template <typename T, int PB, int SB, bool LOCAL>
static int scan_fwd_pass(const ScanArgs& g, hipStream_t s) {
    typedef ScanFwdLds<T, PB, SB> L;
    constexpr int lds = L::NW * L::WAVE;
    if (allow_lds(reinterpret_cast<const void*>(k_scan_fwd<T, PB, SB, LOCAL>), lds) != 0) return -1;
    k_scan_fwd<T, PB, SB, LOCAL><<<cdiv((int64_t)g.N * g.H * g.spans, L::NW), L::NW * 64, lds, s>>>(g);
    return 0;
}
template <typename T, int PB, int SB>
static int scan_fwd(const ScanArgs& g, hipStream_t s) {
    if (g.spans > 1) {
        if (scan_fwd_pass<T, PB, SB, true>(g, s) != 0) return -1;
        k_scan_join<PB, SB, false><<<dim3((int64_t)g.N * g.H, PB * SB), 256, 0, s>>>(g);
    }
    return scan_fwd_pass<T, PB, SB, false>(g, s);
}
template <typename T, int PB, int SB>
static int scan_bwd(const ScanArgs& g, hipStream_t s) {
    typedef ScanBwdLds<T, PB, SB> L;
    if (g.spans > 1) {
        constexpr int lds = 4 * ScanBwdLocalLds<T, PB, SB>::WAVE;
        if (allow_lds(reinterpret_cast<const void*>(k_scan_bwd_local<T, PB, SB>), lds) != 0) return -1;
        k_scan_bwd_local<T, PB, SB><<<cdiv((int64_t)g.N * g.H * g.spans, 4), 256, lds, s>>>(g);
        k_scan_join<PB, SB, true><<<dim3((int64_t)g.N * g.H, PB * SB), 256, 0, s>>>(g);
    }
    constexpr int lds = L::NW * L::WAVE;
    if (allow_lds(reinterpret_cast<const void*>(k_scan_bwd<T, PB, SB>), lds) != 0) return -1;
    k_scan_bwd<T, PB, SB><<<(int64_t)g.N * g.G * g.head_blocks * g.spans, L::NW * 64, lds, s>>>(g);
    if (g.head_blocks > 1) {
        int64_t nb = cdiv((int64_t)g.T * g.N * g.G * g.S, 256);
        k_scan_bc<T><<<nb < 8192 ? nb : 8192, 256, 0, s>>>(g);
    }
    k_scan_heads<<<3 * g.H, 256, 0, s>>>(g);
    return 0;
}
template <typename T>
static int scan_pick(const ScanArgs& g, bool back, hipStream_t s) {
    const bool p2 = g.P > 32, s2 = g.S > 32;
    if (back) return p2 ? (s2 ? scan_bwd<T, 2, 2>(g, s) : scan_bwd<T, 2, 1>(g, s)) : (s2 ? scan_bwd<T, 1, 2>(g, s) : scan_bwd<T, 1, 1>(g, s));
    return p2 ? (s2 ? scan_fwd<T, 2, 2>(g, s) : scan_fwd<T, 2, 1>(g, s)) : (s2 ? scan_fwd<T, 1, 2>(g, s) : scan_fwd<T, 1, 1>(g, s));
}
int launch_scan_fwd(const morlax_scan_dims& d, const void* x, const void* b, const void* c, const void* dt, const void* z, const float* a_log,
                    const float* d_skip, const float* dt_bias, const uint8_t* first, const float* state_in, void* y, float* state_out, void* saved,
                    void* ws, hipStream_t s) {
    ScanArgs g = scan_args(d);
    scan_carve(g, false, ws);
    g.x = x; g.b = b; g.c = c; g.dt = dt; g.z = z; g.a_log = a_log; g.d_skip = d_skip; g.dt_bias = dt_bias; g.first = first;
    g.state_in = state_in; g.y = y; g.state_out = state_out; g.saved = (float*)saved;
    return d.dtype ? scan_pick<bf16_t>(g, false, s) : scan_pick<float>(g, false, s);
}
int launch_scan_bwd(const morlax_scan_dims& d, const void* x, const void* b, const void* c, const void* dt, const void* z, const float* a_log,
                    const float* d_skip, const float* dt_bias, const uint8_t* first, const void* saved, const void* dy, const float* dstate_out,
                    void* dx, void* db, void* dc, void* ddt, void* dz, float* da_log, float* dd_skip, float* ddt_bias, float* dstate_in, void* ws,
                    hipStream_t s) {
    ScanArgs g = scan_args(d);
    scan_carve(g, true, ws);
    g.x = x; g.b = b; g.c = c; g.dt = dt; g.z = z; g.a_log = a_log; g.d_skip = d_skip; g.dt_bias = dt_bias; g.first = first;
    g.saved = (float*)saved; g.dy = dy; g.dstate_out = dstate_out; g.dx = dx; g.db = db; g.dc = dc; g.ddt = ddt; g.dz = dz;
    g.da_log = da_log; g.dd_skip = dd_skip; g.ddt_bias = ddt_bias; g.dstate_in = dstate_in;
    return d.dtype ? scan_pick<bf16_t>(g, true, s) : scan_pick<float>(g, true, s);
}
void launch_memory_step(const morlax_scan_dims& d, int width, const void* xbc, const void* dt, const void* z, const float* conv_w, const float* conv_b,
                        const float* a_log, const float* d_skip, const float* dt_bias, const uint8_t* first, const void* conv_in, const float* state_in,
                        void* y, void* conv_out, float* state_out, hipStream_t s) {
    StepArgs a = {};
    a.s = scan_args(d);
    ScanArgs& g = a.s;
    a.xbc = xbc; a.conv_in = conv_in; a.conv_w = conv_w; a.conv_b = conv_b; a.conv_out = conv_out; a.width = width;
    g.dt = dt; g.z = z; g.a_log = a_log; g.d_skip = d_skip; g.dt_bias = dt_bias; g.first = first; g.state_in = state_in; g.y = y; g.state_out = state_out;
    const int vec = g.S % 4 == 0;
    int lpr = 1;
    while (lpr < 64 && lpr * (vec ? 4 : 1) < g.S) lpr *= 2;
    const int parts = (int64_t)g.N * g.H <= 1536 && g.P >= 4 ? 4 : 1;  // a wave for every SIMD, or nearly
    a.lay = step_layout(g.P, g.S, parts);
    const int lds = 4 * a.lay.wave * (int)sizeof(float);
    const int64_t blocks = cdiv((int64_t)g.N * g.H * parts, 4);
    if (d.dtype) k_memory_step<bf16_t><<<blocks, 256, lds, s>>>(a, lpr, vec, parts);
    else k_memory_step<float><<<blocks, 256, lds, s>>>(a, lpr, vec, parts);
}
