// Attention of a rollout segment's steps over the past steps of their own episode, on time-major tensors of N environments, with a learned
// bias by buckets of the distance in time.
//
//   a[t, s] = scale q_t . k_s + bias[h, bucket(p_t - s)],   p_t = S - T + t,   seen where lo_t <= s <= p_t,
//   y_t = sum_s P[t, s] v_s,   P = exp(a - L),   L_t = log sum_s exp(a[t, s]);     lo_t: the episode's begin or p_t - window + 1, the later one
//   dP = dy_t . v_s,   dA = P (dP - delta_t),   delta_t = dy_t . y_t,
//   dq_t = scale sum_s dA k_s,   dk_s = scale sum_t dA q_t,   dv_s = sum_t P dy_t,   dbias[h, b] = sum of dA over the pairs in bucket b
//
// One pass over the keys with the running maximum and sum; scores never leave the registers.  Products run on the matrix instructions with
// the operands turned so that a computed operand (P, dA) is already where the next product wants it: keys lie along a lane's registers,
// queries along the lanes (the other way round in the pass over the keys), and the other operand is read transposed out of LDS.  What is seen of
// a row is an interval, [lo_t, p_t], and every mask is a select: what an unseen key, value or row holds never counts (see `clean`
// below).
// Query heads that share a head of keys are rows of the same tile (`pack` of them), so the keys are read once for all of them and the sums over
// heads in dk and dv are sums over rows.
#include "attn_tile.h"

static int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

#define ATTN_THREADS 256
#define ATTN_ROOM(rows, keys) ((rows) + 4 * (keys))  // table entries of a tile: pack <= 4 heads, each its distances
// Waves of a SIMD that the registers are to leave room for (forward, backward of queries, of keys)
constexpr int attn_waves(int pass, int es, int dp) {
    return es == 4 && dp == 128 ? 1 : dp == 128 || pass == 2 || (es == 4 && dp == 64) ? 2 : pass == 0 && dp == 32 ? 4 : 3;
}
constexpr int kNever = 1 << 30;  // begin of the seen interval of a row that is not there

// Few long walks are cut into `chunks` of `span` tiles each, whose parts are joined by a launch of their own (see `cut` below)
struct Cut {
    int chunks, span;
    float* o;         // forward: [chunks, N H T, DP] outputs ahead of their division; queries: the same of dq; keys: [2, chunks, S N KV, DP] dk and dv
    float2* m;        // forward: [chunks, N H T] maximum (in units of log2) and sum, -1: no part
    int32_t* there;   // backward: [chunks, workgroups of a chunk] is there a part
};

struct AttnArgs {
    const void *q, *k, *v, *y, *dy;
    void *out, *dq, *dk, *dv;
    const float* bias;
    const int32_t* edges;
    const uint8_t* first;
    int32_t* lo;      // [N, S] begin of every step's episode; NULL: no episodes
    float* table;     // [H, reach] bias by distance, in units of log2; NULL: no bias
    int32_t* bucket;  // [reach]
    float* lse;       // [N, H, T] L, in units of log2; NULL: not wanted
    uint16_t* low;    // [T, N, H, D] what y's rounding to bf16 took away: the fp32 value's bits less the rounded one's
    float* delta;     // [N, H, T]
    float* part;      // [H, B, parts] sums of dA of each workgroup
    float* dbias;
    float scale;
    int T, S, N, H, KV, D, B, window, reach, lgp, tiles;
    int64_t q_t, q_n, k_t, k_n, y_t, y_n;
    uint32_t total;   // workgroups of a chunk
    uint32_t own;     // heads of an XCD where these are few, or 0
    RowDiv by_total, by_tiles, by_own, by_heads;
    uint32_t before;  // workgroups of the launch that do something else
    int64_t parts;    // of a sum of dbias
    int share;        // query heads to a head of keys
    Cut cut, cut_q;  // of the forward or of the backward's pass over the keys; of its pass over the queries
    int whole;  // rows hold whole pieces of 16 bytes
};

// ---- episodes and the bias by distance --------------------------------------------------------------------------------
// A launch ahead of the others, which are bound by what they read once per tile of theirs, not once per pair.  Bound by latency: 5 us
// (8 environments of 2048 steps in one workgroup, in runs of 16 steps: 14).
// Blocks below `spans`: 2^lgn environments at a time, the threads of an environment taking a run of steps each; the others: the table.
__global__ __launch_bounds__(1024) void k_attn_prepare(AttnArgs g, int spans, int lgn) {
    __shared__ int last[1024];
    if ((int)blockIdx.x < spans) {
        const int NB = 1 << lgn, lanes = 1024 >> lgn, e = threadIdx.x & (NB - 1), c = threadIdx.x >> lgn;
        const int64_t n = (int64_t)blockIdx.x * NB + e;
        const int run = (g.S + lanes - 1) / lanes, s0 = c * run, s1 = s0 + run < g.S ? s0 + run : g.S;
        int mine = -1;
        if (n < g.N) {
#pragma unroll 16
            for (int s = s0; s < s1; ++s)
                if (g.first[(int64_t)s * g.N + n]) mine = s;
        }
        last[threadIdx.x] = mine;
        __syncthreads();
        for (int o = 1; o < lanes; o <<= 1) {  // the last begin up to and with each run
            const int v = c >= o ? last[((c - o) << lgn) + e] : -1;
            __syncthreads();
            if (v > last[threadIdx.x]) last[threadIdx.x] = v;
            __syncthreads();
        }
        if (n >= g.N) return;
        int begin = c ? last[((c - 1) << lgn) + e] : 0;
        begin = begin < 0 ? 0 : begin;
        for (int s = s0; s < s1; ++s) {
            if (mine >= 0 && g.first[(int64_t)s * g.N + n]) begin = s;
            g.lo[n * g.S + s] = begin;
        }
        return;
    }
    const int i = ((int)blockIdx.x - spans) * 1024 + threadIdx.x, h = i / g.reach, d = i - h * g.reach;
    if (threadIdx.x < g.B) last[threadIdx.x] = g.edges[threadIdx.x];
    __syncthreads();
    if (h >= g.H) return;
    int b = 0;
    for (int j = 1; j < g.B; ++j) b += last[j] <= d;
    if (h == 0) g.bucket[d] = b;
    g.table[i] = g.bias[h * g.B + b] * kLog2e;
}

// ---- tiles ------------------------------------------------------------------------------------------------------------
// A computed zero times an infinite or undefined element would reach rows that do not see it.  So such elements are put down as zeros in
// the tiles that computed operands are multiplied with, and a workgroup that met one adds them in the end, one by one, to what sees them
// (as they are: the products of the definition are infinite or undefined too).
__device__ inline bool finite(float v) { return __builtin_fabsf(v) < __builtin_inff(); }
template <typename T>
__device__ inline uint4 clean(const uint4& u) {
    uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) {
            if (!finite(__uint_as_float(w[i] << 16))) w[i] &= 0xffff0000u;
            if (!finite(__uint_as_float(w[i] & 0xffff0000u))) w[i] &= 0xffffu;
        } else if (!finite(__uint_as_float(w[i]))) {
            w[i] = 0;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// Has any of the pieces looked at held such an element
template <typename T> struct Probe {
    float z = 0.f;
    __device__ inline void look(const uint4& u) {
        z = __builtin_fmaf(__uint_as_float(u.x), 0.f, __builtin_fmaf(__uint_as_float(u.y), 0.f, z));
        z = __builtin_fmaf(__uint_as_float(u.z), 0.f, __builtin_fmaf(__uint_as_float(u.w), 0.f, z));
    }
    __device__ inline bool met() const { return z != 0.f; }
};
template <> struct Probe<bf16_t> {  // (the largest of the magnitudes as integers, two at a time)
    typedef uint16_t pair_t __attribute__((ext_vector_type(2)));
    pair_t m = {0, 0};
    __device__ inline void look(uint32_t w) { m = __builtin_elementwise_max(m, __builtin_bit_cast(pair_t, w & 0x7fff7fffu)); }
    __device__ inline void look(const uint4& u) {
        look(u.x); look(u.y); look(u.z); look(u.w);
    }
    __device__ inline bool met() const { return (m[0] >= 0x7f80) | (m[1] >= 0x7f80); }
};
// does a row hold such an element
template <typename T>
__device__ inline bool tainted(const T* row, int D) {
    bool t = false;
    for (int d = 0; d < D; ++d) t |= !finite(to_f(row[d]));
    return t;
}

// A thread's pieces of a tile on their way: requested before the tile ahead of it is worked on, put down after.  Rows [r0, end) are there; the
// requests for others go to the last row, without a branch (behind one each they would leave one by one), and zeros are put down for them.
template <typename T, int DP, bool WHOLE>
struct Stage {
    typedef Tile<T, DP> L;
    static constexpr int CH = ATTN_K * L::CPR / ATTN_THREADS, STEP = ATTN_THREADS / L::CPR;  // pieces, rows from one to the next
    RowPiece<T, WHOLE> in[CH];
    int64_t mine;  // the first piece's row in a tile
    __device__ static inline int row() { return threadIdx.x / L::CPR; }
    __device__ static inline int col() { return threadIdx.x % L::CPR * L::VE; }
    // row r (r0 a multiple of four) lies at base + (r >> lgp) * stride + (r & (pack - 1)) * D
    __device__ inline void init(int64_t stride, int lgp, int D) {
        mine = (int64_t)(row() >> lgp) * stride + (row() & ((1 << lgp) - 1)) * D;
    }
    __device__ inline void load(const T* base, int64_t stride, int r0, int end, int lgp, int D) {
        if (r0 + ATTN_K <= end) {
            const T* p = base + (int64_t)(r0 >> lgp) * stride;
            int64_t at = mine;
            asm volatile("" : "+v"(at));  // (or every piece's place is kept in registers of its own)
#pragma unroll
            for (int c = 0; c < CH; ++c) in[c].load(p + (int64_t)(c * STEP >> lgp) * stride + at, col(), D);
        } else {
            int first = r0 + row();
            asm volatile("" : "+v"(first));
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                int r = first + c * STEP;
                r = r < end ? r : end - 1;
                in[c].load(base + (int64_t)(r >> lgp) * stride + (r & ((1 << lgp) - 1)) * D, col(), D);
            }
        }
    }
    // CLEAN: infinite and undefined elements as zeros; returns whether there were any
    template <bool CLEAN>
    __device__ inline bool put(unsigned char* lds, int r0, int end, int D) {
        uint4 u[CH];
        if (WHOLE && r0 + ATTN_K <= end && D == DP) {
#pragma unroll
            for (int c = 0; c < CH; ++c) u[c] = in[c].u;
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c) u[c] = in[c].get(col(), D, r0 + row() + c * STEP < end);
        }
        bool met = false;
        if (CLEAN) {
            Probe<T> probe;
#pragma unroll
            for (int c = 0; c < CH; ++c) probe.look(u[c]);
            met = probe.met();
            if (__any(met)) {
#pragma unroll
                for (int c = 0; c < CH; ++c) u[c] = clean<T>(u[c]);
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) L::put(lds, row() + c * STEP, col(), u[c]);
        return met;
    }
};

// acc[b][dt] (rows: columns 16 dt + 4 g + r of the tile; column: lane & 15) += rows^T p[b] over the tile's rows u TU .., for NBLK blocks of 16
// lanes' columns
template <typename T, int DP, int NBLK, bool FINE = false>
__device__ inline void fold(const unsigned char* lds, int u, const float4_t (&p)[NBLK][Tile<T, DP>::NX], float4_t (&acc)[NBLK][DP / 16], int lane) {
    typedef Tile<T, DP> L;
    Computed<sizeof(T) == 4 || FINE ? 3 : 2> c[NBLK];
#pragma unroll
    for (int b = 0; b < NBLK; ++b) c[b].set(p[b]);
#pragma unroll
    for (int dt = 0; dt < L::NB; ++dt) {
        if (dt && dt % 4 == 0) phase();
        const Operand<T> f = L::turned(lds, u, dt, lane);
#pragma unroll
        for (int b = 0; b < NBLK; ++b) multiply(f.p, c[b].p, acc[b][dt]);
    }
    phase();
}

// Rows of results go out as what no workgroup here reads again, and leave the L2 to the tiles that others share (512 environments, 64 of 128 steps, 8
// heads of 64: dk and dv 131 -> 117 us, the passes over the queries 5% less; requests of what is read once marked so too: 10% more).
template <typename T, int DP, bool WHOLE, typename F>
__device__ inline void send_rows(const unsigned char* lds, int D, F to) {
    typedef Tile<T, DP> L;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < 16 * L::CPR / 64; ++i) {
        const int p = i * 64 + lane, row = p / L::CPR, col = p % L::CPR * L::VE;
        T* dst = reinterpret_cast<T*>(to(row));
        const uint4 u = *reinterpret_cast<const uint4*>(lds + row * L::OPITCH + col * L::ES);
        if (!dst) continue;
        if (WHOLE ? col < D : col + L::VE <= D) {
            __builtin_nontemporal_store(piece_t{u.x, u.y, u.z, u.w}, reinterpret_cast<piece_t*>(dst + col));
        } else if (!WHOLE) {
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int e = 0; e < L::VE; ++e) {
                if (col + e >= D) continue;
                if constexpr (L::ES == 2) reinterpret_cast<uint16_t*>(dst)[col + e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
                else reinterpret_cast<uint32_t*>(dst)[col + e] = w[e];
            }
        }
    }
}
// A wave's block of 16 rows goes out by whole rows: laid down in LDS as its lanes hold it (row: the lane's; columns 16 dt + 4 g + r), read back in
// pieces along the rows (8 bytes a lane straight from the registers touch 32 bytes of each line four times over).
// lds: 16 rows of the wave's own; to(row): where a row of D elements begins, or NULL
template <typename T, int DP, bool WHOLE, typename F>
__device__ inline void put_rows(unsigned char* lds, const float4_t (&v)[DP / 16], float scale, int D, F to) {
    typedef Tile<T, DP> L;
    const int lane = threadIdx.x & 63, a = lane & 15, gr = lane >> 4;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int dt = 0; dt < L::NB; ++dt) {
        unsigned char* at = lds + a * L::OPITCH + (16 * dt + 4 * gr) * L::ES;
        if constexpr (L::ES == 2) *reinterpret_cast<uint2*>(at) = make_uint2(pack2(v[dt][0] * scale, v[dt][1] * scale), pack2(v[dt][2] * scale, v[dt][3] * scale));
        else *reinterpret_cast<float4_t*>(at) = float4_t{v[dt][0] * scale, v[dt][1] * scale, v[dt][2] * scale, v[dt][3] * scale};
    }
    __builtin_amdgcn_wave_barrier();
    send_rows<T, DP, WHOLE>(lds, D, to);
}

// Which tile of which environment and heads (`rest`) a workgroup takes.  Workgroups go round the eight XCDs, and what belongs to one `rest` goes to the
// same one, where its keys are in the L2.  Later rows see more keys (earlier keys are seen by more rows): the longest tiles first, of all that an
// XCD has where these are few, so that the last ones to end are short.
struct Place {
    uint32_t rest;
    int tile, chunk;
    __device__ inline Place(const AttnArgs& g) {
        const uint32_t index = blockIdx.x - g.before;
        chunk = (int)g.by_total.quotient(index);
        const uint32_t at = index - chunk * g.total, x = at & 7, i = at >> 3;
        if (g.own) {
            const uint32_t row = g.by_own.quotient(i);
            rest = x + 8 * (i - row * g.own);
            tile = g.tiles - 1 - (int)row;
        } else {
            const uint32_t each = g.total >> 3, over = g.total & 7, w = x * each + (x < over ? x : over) + i;
            rest = g.by_tiles.quotient(w);
            tile = g.tiles - 1 - (int)(w - rest * g.tiles);
        }
    }
};

// A workgroup's rows of queries: (step, head of the pack), heads next to each other
struct Rows {
    int n, kv, h0, r0, rows, past, chunk;
    __device__ inline void init(const AttnArgs& g, int per) {
        const Place at(g);
        n = (int)g.by_heads.quotient(at.rest);
        h0 = (int)(at.rest - n * (g.H >> g.lgp)) << g.lgp;
        kv = h0 / g.share;
        r0 = at.tile * per;
        chunk = at.chunk;
        rows = g.T << g.lgp;
        past = g.S - g.T;
    }
    __device__ inline int lo(const AttnArgs& g, int p) const {
        const int b = g.lo ? g.lo[(int64_t)n * g.S + p] : 0, w = p - g.window + 1, v = b > w ? b : w;
        return v < 0 ? 0 : v > p ? p : v;  // (within the row whatever `saved` holds)
    }
};

// The bias of a tile by distance: entry [head][j] belongs to the distance `far` - j (or `far` + j), clamped to those there are
template <int NR>  // entries that a thread stages
struct Table {
    float v[NR];
    int b[NR];
    template <bool BUCKET>
    __device__ inline void load(const AttnArgs& g, int h0, int each, int far, int dir) {
        const int count = each << g.lgp;
#pragma unroll
        for (int c = 0; c < NR; ++c) {
            int i = threadIdx.x + c * ATTN_THREADS;
            i = i < count ? i : count - 1;
            const int hh = (i >= each) + (i >= 2 * each) + (i >= 3 * each);
            int d = far + dir * (i - hh * each);
            d = d < 0 ? 0 : d >= g.reach ? g.reach - 1 : d;
            v[c] = g.table[(int64_t)(h0 + hh) * g.reach + d];
            if (BUCKET) {  // (a bucket whatever `saved` holds)
                const int i = g.bucket[d];
                b[c] = i < 0 ? 0 : i >= g.B ? g.B - 1 : i;
            }
        }
    }
    template <bool BUCKET>
    __device__ inline void put(const AttnArgs& g, int each, float* tab, int* idx) const {
        const int count = each << g.lgp;
#pragma unroll
        for (int c = 0; c < NR; ++c) {
            const int i = threadIdx.x + c * ATTN_THREADS;
            if (i >= count) break;  // (behind the loads)
            tab[i] = v[c];
            if (BUCKET && i < each) idx[i] = b[c];
        }
    }
};

// ---- forward ------------------------------------------------------------------------------------------------------------
// Four waves, 16 rows each (32: see below), and a tile of 64 keys at a time, the next one's requests on their way.  Bound by instructions, and by what is
// read and written where there are few keys to a row: 1024 environments, 64 of 128 steps, 8 heads of 64 to 2 of keys 72 us (201 MB; 2.8 TB/s);
// for training 512 of them, 8 heads of keys 48 us (235 MB, 4.9 TB/s); 2048 x 8 x 8 heads of 128 190 us (137 GF of parts, 0.7 PFLOP/s; 30 to 43 of this
// variant's 256 registers lie in memory).
template <typename T, int DP, int QB>
struct FwdLds {
    static constexpr int ROOM = ATTN_ROOM(64 * QB, ATTN_K), NR = (ROOM + ATTN_THREADS - 1) / ATTN_THREADS;
    static constexpr int K = 0, V = Tile<T, DP>::BYTES, TAB = 2 * V, FLAG = TAB + ROOM * 4, TOTAL = FLAG + 16;
};
template <typename T, int DP, int QB, bool WHOLE, bool FINE, int LGP>
__global__ __launch_bounds__(ATTN_THREADS, attn_waves(0, sizeof(T), DP)) void k_attn_fwd(AttnArgs given) {
    AttnArgs g = given;
    g.lgp = LGP;
    typedef Tile<T, DP> L;
    typedef FwdLds<T, DP, QB> M;
    extern __shared__ __align__(16) unsigned char lds[];
    float* tab = reinterpret_cast<float*>(lds + M::TAB);
    int* flag = reinterpret_cast<int*>(lds + M::FLAG);
    constexpr int BQ = 64 * QB;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, a = lane & 15, gr = lane >> 4;
    Rows R;
    R.init(g, BQ);
    int t[QB], p[QB], lo[QB];
    Operand<T> qf[QB][L::KS];
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int r = R.r0 + (wave * QB + b) * 16 + a;
        const bool in = r < R.rows;
        t[b] = in ? r >> g.lgp : -1;
        p[b] = in ? R.past + t[b] : -1;
        lo[b] = in ? R.lo(g, p[b]) : kNever;
        const T* src = reinterpret_cast<const T*>(g.q) + (int64_t)(in ? t[b] : 0) * g.q_t + (int64_t)R.n * g.q_n +
                       (int64_t)(R.h0 + (r & ((1 << g.lgp) - 1))) * g.D;
#pragma unroll
        for (int ks = 0; ks < L::KS; ++ks) {
            const int d = ks * 32 + gr * 8;
            RowOperand<T, WHOLE> u;
            u.load(src, d, g.D);
            qf[b][ks] = u.get(d, g.D, in);
        }
    }
    const int first_p = R.past + (R.r0 >> g.lgp), each = (BQ >> g.lgp) + ATTN_K, far = first_p + (BQ >> g.lgp) - 1;
    const int last_row = (R.r0 + BQ < R.rows ? R.r0 + BQ : R.rows) - 1;
    int k_begin = R.lo(g, first_p), k_end = R.past + (last_row >> g.lgp) + 1;
    if (g.cut.chunks > 1) {
        k_begin += R.chunk * g.cut.span * ATTN_K;
        const int end = k_begin + g.cut.span * ATTN_K;
        k_end = end < k_end ? end : k_end;
    }
    const int last_edge = g.table ? g.edges[g.B - 1] : 0;
    const float beyond = g.table ? g.bias[(int64_t)(R.h0 + (lane & ((1 << g.lgp) - 1))) * g.B + g.B - 1] * kLog2e : 0.f;
    const T* kb = reinterpret_cast<const T*>(g.k) + (int64_t)R.n * g.k_n + (int64_t)R.kv * g.D;
    const T* vb = reinterpret_cast<const T*>(g.v) + (int64_t)R.n * g.k_n + (int64_t)R.kv * g.D;
    const float c = g.scale * kLog2e;
    float m[QB], l[QB];
    float4_t o[QB][L::NB];
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        m[b] = -__builtin_inff();
        l[b] = 0.f;
#pragma unroll
        for (int dt = 0; dt < L::NB; ++dt) o[b][dt] = float4_t{0.f, 0.f, 0.f, 0.f};
    }
    if (threadIdx.x == 0) *flag = 0;
    if (!g.table)
        for (int i = threadIdx.x; i < M::ROOM; i += ATTN_THREADS) tab[i] = 0.f;
    Stage<T, DP, WHOLE> sk, sv;
    Table<M::NR> st;
    sk.init(g.k_t, 0, g.D);
    sv.init(g.k_t, 0, g.D);
    auto request = [&](int k0) {
        sk.load(kb, g.k_t, k0, k_end, 0, g.D);
        sv.load(vb, g.k_t, k0, k_end, 0, g.D);
        if (g.table) st.template load<false>(g, R.h0, each, far - k0, -1);
    };
    if (k_begin < k_end) request(k_begin);  // (a chunk may be empty)
    __syncthreads();
    for (int k0 = k_begin; k0 < k_end; k0 += ATTN_K) {
        const bool near = g.table && first_p - (k0 + ATTN_K - 1) < last_edge;
        sk.template put<false>(lds + M::K, k0, k_end, g.D);
        if (sv.template put<true>(lds + M::V, k0, k_end, g.D)) *flag = 1;
        if (g.table) st.template put<false>(g, each, tab, nullptr);
        __syncthreads();
        if (k0 + ATTN_K < k_end) request(k0 + ATTN_K);
        bool any = false, all = true;
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            any |= (p[b] >= k0) & (lo[b] < k0 + ATTN_K);
            all &= (lo[b] <= k0) & (p[b] >= k0 + ATTN_K - 1);
        }
        // FAST: all of the tile is seen, at distances beyond the last edge
        auto tile = [&](auto fast) {
            constexpr bool FAST = decltype(fast)::value;
            float4_t s[QB][4];
            const int now = lane_now();
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                phase();
#pragma unroll
                for (int b = 0; b < QB; ++b) s[b][x] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < L::KS; ++ks) {
                    const Operand<T> f = L::rows(lds + M::K, 16 * x, ks, now);
#pragma unroll
                    for (int b = 0; b < QB; ++b) multiply(f.p, qf[b][ks].p, s[b][x]);
                }
            }
            phase();
#pragma unroll
            for (int b = 0; b < QB; ++b) {
                const float* row = tab + (now & ((1 << g.lgp) - 1)) * each + 4 * (now >> 4) + (t[b] < 0 ? 0 : far - p[b]);
                const int from = lo[b] - k0 - 4 * (now >> 4);
                const uint32_t span = p[b] - lo[b];
                float top = m[b];
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float v = __builtin_fmaf(s[b][x][r], c, FAST ? beyond : row[16 * x + r]);
                        if (!FAST) v = ((t[b] >= 0) & ((uint32_t)(16 * x + r - from) <= span)) ? v : -__builtin_inff();
                        s[b][x][r] = v;
                        top = fmaxf(top, v);
                    }
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float base = top == -__builtin_inff() ? 0.f : top;  // nothing seen yet
                float sum = 0.f;
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        s[b][x][r] = __builtin_amdgcn_exp2f(s[b][x][r] - base);
                        sum += s[b][x][r];
                    }
                if (__any(top != m[b])) {
                    const float fade = __builtin_amdgcn_exp2f(m[b] - base);
                    l[b] *= fade;
#pragma unroll
                    for (int dt = 0; dt < L::NB; ++dt)
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[b][dt][r] *= fade;
                }
                l[b] += sum;
                m[b] = top;
            }
#pragma unroll
            for (int u = 0; u < L::NU; ++u) {
                float4_t part[QB][L::NX];
#pragma unroll
                for (int b = 0; b < QB; ++b)
#pragma unroll
                    for (int i = 0; i < L::NX; ++i) part[b][i] = s[b][u * L::NX + i];
                fold<T, DP, QB, FINE>(lds + M::V, u, part, o, now);
            }
        };
        if (__any(any)) {
            if (!near && __all(all)) tile(std::true_type{});
            else tile(std::false_type{});
        }
        __syncthreads();
    }
    if (*flag) {
        for (int k = k_begin; k < k_end; ++k)
#pragma unroll
            for (int b = 0; b < QB; ++b) {
                const bool see = (t[b] >= 0) & (k >= lo[b]) & (k <= p[b]);
                if (!see) continue;
#pragma unroll
                for (int dt = 0; dt < L::NB; ++dt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int d = 16 * dt + 4 * gr + r;
                        const float v = d < g.D ? to_f(vb[(int64_t)k * g.k_t + d]) : 0.f;
                        o[b][dt][r] += finite(v) ? 0.f : v;
                    }
            }
    }
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        l[b] += __shfl_xor(l[b], 16);
        l[b] += __shfl_xor(l[b], 32);
        if (g.cut.chunks > 1) {
            if (t[b] < 0) continue;
            const int64_t row = ((int64_t)R.n * g.H + R.h0 + (a & ((1 << g.lgp) - 1))) * g.T + t[b], all = (int64_t)g.N * g.H * g.T;
            if (gr == 0) g.cut.m[R.chunk * all + row] = make_float2(m[b], k_begin < k_end ? l[b] : -1.f);
            float* dst = g.cut.o + (R.chunk * all + row) * DP + 4 * gr;
            if (k_begin < k_end)
#pragma unroll
                for (int dt = 0; dt < L::NB; ++dt) *reinterpret_cast<float4_t*>(dst + 16 * dt) = o[b][dt];
            continue;
        }
        const float inv = 1.f / l[b];
        if (g.lse && gr == 0 && t[b] >= 0)
            g.lse[((int64_t)R.n * g.H + R.h0 + (a & ((1 << g.lgp) - 1))) * g.T + t[b]] = m[b] + __builtin_amdgcn_logf(l[b]);
        unsigned char* mine = lds + wave * 16 * L::OPITCH;
        const int first = R.r0 + (wave * QB + b) * 16;
        put_rows<T, DP, WHOLE>(mine, o[b], inv, g.D, [&](int row) -> T* {
            const int r = first + row;
            if (r >= R.rows) return nullptr;
            return reinterpret_cast<T*>(g.out) + (int64_t)(r >> g.lgp) * g.y_t + (int64_t)R.n * g.y_n + (int64_t)(R.h0 + (r & ((1 << g.lgp) - 1))) * g.D;
        });
        if constexpr (FINE) {  // what the rounding took: the fp32 value's bits less the rounded one's (a tie that went down is one more)
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int dt = 0; dt < L::NB; ++dt) {
                uint32_t rest[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float y = o[b][dt][r] * inv;
                    const int d = __float_as_int(y) - __float_as_int((float)(bf16_t)y);
                    rest[r] = (uint32_t)(d < 0x7fff ? d : 0x7fff) & 0xffff;
                }
                *reinterpret_cast<uint2*>(mine + a * L::OPITCH + (16 * dt + 4 * gr) * 2) = make_uint2(rest[0] | rest[1] << 16, rest[2] | rest[3] << 16);
            }
            __builtin_amdgcn_wave_barrier();
            send_rows<T, DP, WHOLE>(mine, g.D, [&](int row) -> T* {
                const int r = first + row;
                if (r >= R.rows) return nullptr;
                return reinterpret_cast<T*>(g.low) + (((int64_t)(r >> g.lgp) * g.N + R.n) * g.H + R.h0 + (r & ((1 << g.lgp) - 1))) * g.D;
            });
        }
    }
}

// The parts of a row, joined: DP / 4 lanes a row, four columns each
template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attn_fwd_join(AttnArgs g) {
    constexpr int LANES = DP / 4;
    const int64_t all = (int64_t)g.N * g.H * g.T, row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    if (row >= all) return;
    const int d = threadIdx.x % LANES * 4, t = (int)(row % g.T), h = (int)(row / g.T % g.H), n = (int)(row / g.T / g.H);
    float top = -__builtin_inff();
    for (int c = 0; c < g.cut.chunks; ++c) top = fmaxf(top, g.cut.m[c * all + row].x);
    const float base = top == -__builtin_inff() ? 0.f : top;
    float sum = 0.f;
    float4_t y = {0.f, 0.f, 0.f, 0.f};
    for (int c = 0; c < g.cut.chunks; ++c) {
        const float2 p = g.cut.m[c * all + row];
        if (p.y < 0.f) continue;  // (an empty chunk, which wrote no part)
        const float f = __builtin_amdgcn_exp2f(p.x - base);
        const float4_t o = *reinterpret_cast<const float4_t*>(g.cut.o + (c * all + row) * DP + d);
        sum = __builtin_fmaf(f, p.y, sum);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __builtin_fmaf(f, o[i], y[i]);
    }
    if (g.lse && d == 0) g.lse[row] = top + __builtin_amdgcn_logf(sum);
    T* dst = reinterpret_cast<T*>(g.out) + (int64_t)t * g.y_t + (int64_t)n * g.y_n + (int64_t)h * g.D;
    uint16_t* low = g.low ? g.low + (((int64_t)t * g.N + n) * g.H + h) * g.D : nullptr;
    const float inv = 1.f / sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (d + i >= g.D) continue;
        const float v = y[i] * inv;
        dst[d + i] = cvt<T>(v);
        if (sizeof(T) == 2 && low) {
            const int rest = __float_as_int(v) - __float_as_int((float)(bf16_t)v);
            low[d + i] = (uint16_t)(rest < 0x7fff ? rest : 0x7fff);
        }
    }
}

// Sums of a block of 16 keys and 16 rows along its slants (pairs of one distance): lane (a, g) holds the keys 4 g + r, r = 0 .. 3, of row a, that is
// of step a / PACK, and key 4 g + r of step t + r is as far as key 4 g of step t.  x: the lane's, distance a / PACK - 4 g; y: those that lie
// 16 / PACK steps further on, distance a / PACK - 16 / PACK - 4 g.
template <int CTRL>
__device__ inline float shifted(float v) {  // another lane's of the same 16, zero from beyond them
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int PACK>
struct Slant {
    static __device__ inline float2 sum(const float4_t& v) {
        constexpr int SHL = 0x100, SHR = 0x110;
        return make_float2((v[0] + shifted<SHL + PACK>(v[1])) + (shifted<SHL + 2 * PACK>(v[2]) + shifted<SHL + 3 * PACK>(v[3])),
                           (shifted<SHR + 16 - PACK>(v[1]) + shifted<SHR + 16 - 2 * PACK>(v[2])) + shifted<SHR + 16 - 3 * PACK>(v[3]));
    }
};
// Four values of distances 16 apart into a lane's bins: those of one bucket together first, so that the reads of the bins need not wait for each other
// (the last write of a bin is the one with the sum)
// at: the first one's entry in the table; entries from `end` on are distances that no pair of the tile has.  LANES 32: two lanes have a bin in common,
// and add to it one after the other.
template <int LANES, typename F>
__device__ inline void by_halves(F add) {
    if constexpr (LANES == 64) {
        add();
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if ((int)(threadIdx.x >> 5 & 1) == h) add();
            __builtin_amdgcn_wave_barrier();
        }
    }
}
template <int LANES>
__device__ inline void add_to_bins(float* bins, const int* idx, int at, int end, float4_t v) {
    int b[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) b[x] = idx[at + 16 * x < end ? at + 16 * x : end - 1] * LANES;
#pragma unroll
    for (int x = 3; x > 0; --x) {
        const bool same = b[x] == b[x - 1];
        v[x - 1] += same ? v[x] : 0.f;
        v[x] = same ? 0.f : v[x];
    }
    by_halves<LANES>([&] {
        float old[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) old[x] = bins[b[x]];
#pragma unroll
        for (int x = 3; x >= 0; --x) bins[b[x]] = old[x] + v[x];
    });
}

// ---- backward, queries: dq, the sums of dA by bucket, and delta ---------------------------------------------------------------
// As the forward, with dP beside the scores.  512 environments, 64 of 128 steps, 8 heads of 64: 73 us (302 MB, 4.1 TB/s); 2048 x 8 x 8 heads of 128
// to 2 of keys: 230 us (0.6 PFLOP/s of parts): instructions, the matrix ones a third of the time.
template <typename T, int DP, int QB>
struct DqLds {
    static constexpr int ROOM = ATTN_ROOM(64 * QB, ATTN_K), NR = (ROOM + ATTN_THREADS - 1) / ATTN_THREADS;
    static constexpr int K = 0, V = Tile<T, DP>::BYTES, TAB = 2 * V, IDX = TAB + ROOM * 4, FLAG = IDX + (64 * QB + ATTN_K) * 4, BINS = FLAG + 16;
    static constexpr int LANES = BINS > 48 * 1024 ? 32 : 64;  // bins of a bucket and wave: beside the largest tiles fewer have to do
};
template <typename T, int DP, int QB, bool WHOLE, int LGP>
__global__ __launch_bounds__(ATTN_THREADS, attn_waves(1, sizeof(T), DP)) void k_attn_dq(AttnArgs given) {
    AttnArgs g = given;
    g.lgp = LGP;
    typedef Tile<T, DP> L;
    typedef DqLds<T, DP, QB> M;
    extern __shared__ __align__(16) unsigned char lds[];
    float* tab = reinterpret_cast<float*>(lds + M::TAB);
    int* idx = reinterpret_cast<int*>(lds + M::IDX);
    int* flag = reinterpret_cast<int*>(lds + M::FLAG);
    constexpr int BQ = 64 * QB, LANES = M::LANES;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, a = lane & 15, gr = lane >> 4, hh = lane & ((1 << g.lgp) - 1);
    // Sums of dA by bucket.  A lane adds up what it and its neighbours hold of one distance (see Slant) and adds that to a bin of its own: no two
    // lanes have a bin in common, so the order of every sum is the program's.  (Added pair by pair by LDS atomics: 174 cycles for 64 of them, half
    // of this kernel's time on 2048 x 8 x 8 heads of 128; laid out by distance in LDS and added up there: still a third.)
    float* bins = reinterpret_cast<float*>(lds + M::BINS) + (int64_t)wave * g.B * LANES + (lane & (LANES - 1));
    Rows R;
    R.init(g, BQ);
    int t[QB], p[QB], lo[QB];
    float lse[QB], delta[QB];
    Operand<T> qf[QB][L::KS], of[QB][L::KS];
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int r = R.r0 + (wave * QB + b) * 16 + a;
        const bool in = r < R.rows;
        t[b] = in ? r >> g.lgp : -1;
        p[b] = in ? R.past + t[b] : -1;
        lo[b] = in ? R.lo(g, p[b]) : kNever;
        const int64_t at = in ? t[b] : 0, h = R.h0 + hh;
        const T* src = reinterpret_cast<const T*>(g.q) + at * g.q_t + (int64_t)R.n * g.q_n + h * g.D;
        const T* dsrc = reinterpret_cast<const T*>(g.dy) + at * g.y_t + (int64_t)R.n * g.y_n + h * g.D;
        const T* ysrc = reinterpret_cast<const T*>(g.y) + at * g.y_t + (int64_t)R.n * g.y_n + h * g.D;
        const uint16_t* lsrc = g.low ? g.low + ((at * g.N + R.n) * g.H + h) * g.D : nullptr;
        float sum = 0.f;
#pragma unroll
        for (int ks = 0; ks < L::KS; ++ks) {
            const int d = ks * 32 + gr * 8;
            RowOperand<T, WHOLE> uq, uo, uy;
            uq.load(src, d, g.D);
            uo.load(dsrc, d, g.D);
            uy.load(ysrc, d, g.D);
            RowPiece<uint16_t, WHOLE> ul;
            if constexpr (L::ES == 2) ul.load(lsrc, d, g.D);
            qf[b][ks] = uq.get(d, g.D, in);
            of[b][ks] = uo.get(d, g.D, in);
            if constexpr (L::ES == 2) {
                const uint4 yf = uy.u[0].get(d, g.D, in), lf = ul.get(d, g.D, in), df = of[b][ks].p[0];
                const uint32_t wy[4] = {yf.x, yf.y, yf.z, yf.w}, wd[4] = {df.x, df.y, df.z, df.w}, wl[4] = {lf.x, lf.y, lf.z, lf.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sum = __builtin_fmaf(__uint_as_float(wd[i] << 16), __int_as_float((int)(wy[i] << 16) + ((int)(wl[i] << 16) >> 16)), sum);
                    sum = __builtin_fmaf(__uint_as_float(wd[i] & 0xffff0000u), __int_as_float((int)(wy[i] & 0xffff0000u) + ((int)wl[i] >> 16)), sum);
                }
            } else {
                float vy[8], vd[8];
                uy.values(d, g.D, in, vy);
                uo.values(d, g.D, in, vd);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(vd[i], vy[i], sum);
            }
        }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        delta[b] = sum;
        lse[b] = 0.f;
        if (in) {
            const int64_t row = ((int64_t)R.n * g.H + h) * g.T + t[b];
            lse[b] = g.lse[row];
            if (gr == 0 && R.chunk == 0) g.delta[row] = sum;
        }
    }
    const int first_p = R.past + (R.r0 >> g.lgp), each = (BQ >> g.lgp) + ATTN_K, far = first_p + (BQ >> g.lgp) - 1;
    const int last_row = (R.r0 + BQ < R.rows ? R.r0 + BQ : R.rows) - 1;
    int k_begin = R.lo(g, first_p), k_end = R.past + (last_row >> g.lgp) + 1;
    if (g.cut_q.chunks > 1) {
        k_begin += R.chunk * g.cut_q.span * ATTN_K;
        const int end = k_begin + g.cut_q.span * ATTN_K;
        k_end = end < k_end ? end : k_end;
    }
    const int last_edge = g.table ? g.edges[g.B - 1] : 0;
    const float beyond = g.table ? g.bias[(int64_t)(R.h0 + hh) * g.B + g.B - 1] * kLog2e : 0.f;
    const T* kb = reinterpret_cast<const T*>(g.k) + (int64_t)R.n * g.k_n + (int64_t)R.kv * g.D;
    const T* vb = reinterpret_cast<const T*>(g.v) + (int64_t)R.n * g.k_n + (int64_t)R.kv * g.D;
    const float c = g.scale * kLog2e;
    float outer = 0.f;  // sum of dA over tiles beyond the last edge
    float4_t o[QB][L::NB];
#pragma unroll
    for (int b = 0; b < QB; ++b)
#pragma unroll
        for (int dt = 0; dt < L::NB; ++dt) o[b][dt] = float4_t{0.f, 0.f, 0.f, 0.f};
    if (threadIdx.x == 0) *flag = 0;
    if (!g.table)
        for (int i = threadIdx.x; i < M::ROOM; i += ATTN_THREADS) tab[i] = 0.f;
    if (g.part)
        for (int b = 0; b < g.B; ++b) bins[b * LANES] = 0.f;
    float carry[QB];  // of the tile before, of distances that go on with the key `carry_k` (one head a tile)
    int carry_k = 0;
    bool lone[QB];    // sees itself only: its probability is one whatever the score, and dA nothing, not what two sums' roundings leave
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        carry[b] = 0.f;
        lone[b] = lo[b] == p[b];
    }
    Stage<T, DP, WHOLE> sk, sv;
    Table<M::NR> st;
    sk.init(g.k_t, 0, g.D);
    sv.init(g.k_t, 0, g.D);
    auto request = [&](int k0) {
        sk.load(kb, g.k_t, k0, k_end, 0, g.D);
        sv.load(vb, g.k_t, k0, k_end, 0, g.D);
        if (g.table) st.template load<true>(g, R.h0, each, far - k0, -1);
    };
    if (k_begin < k_end) request(k_begin);
    __syncthreads();
    for (int k0 = k_begin; k0 < k_end; k0 += ATTN_K) {
        const bool near = g.table && first_p - (k0 + ATTN_K - 1) < last_edge;
        if (sk.template put<true>(lds + M::K, k0, k_end, g.D)) *flag = 1;
        sv.template put<false>(lds + M::V, k0, k_end, g.D);
        if (g.table) st.template put<true>(g, each, tab, idx);
        __syncthreads();
        if (k0 + ATTN_K < k_end) request(k0 + ATTN_K);
        bool any = false, all = true;
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            any |= (p[b] >= k0) & (lo[b] < k0 + ATTN_K);
            all &= (lo[b] <= k0) & (p[b] >= k0 + ATTN_K - 1);
        }
        auto tile = [&](auto fast) {
            constexpr bool FAST = decltype(fast)::value;
            const int now = lane_now(), an = now & 15, gn = now >> 4;
            float4_t main[QB], over[QB];  // by block of 16 keys: sums along a slant
#pragma unroll
            for (int u = 0; u < L::NU; ++u) {
                float4_t s[QB][L::NX], dp[QB][L::NX];
                phase();
#pragma unroll
                for (int i = 0; i < L::NX; ++i) {
                    const int x = u * L::NX + i;
                    if (i && DP > 64) phase();
#pragma unroll
                    for (int b = 0; b < QB; ++b) s[b][i] = dp[b][i] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int ks = 0; ks < L::KS; ++ks) {
                        const Operand<T> f = L::rows(lds + M::K, 16 * x, ks, now), fv = L::rows(lds + M::V, 16 * x, ks, now);
#pragma unroll
                        for (int b = 0; b < QB; ++b) {
                            multiply(f.p, qf[b][ks].p, s[b][i]);
                            multiply(fv.p, of[b][ks].p, dp[b][i]);
                        }
                    }
                }
                phase();
#pragma unroll
                for (int i = 0; i < L::NX; ++i)
#pragma unroll
                    for (int b = 0; b < QB; ++b) {
                        const int x = u * L::NX + i, place = hh * each + 4 * gn + (t[b] < 0 ? 0 : far - p[b]);
                        const int from = lo[b] - k0 - 4 * gn;
                        const uint32_t span = p[b] - lo[b];
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i][r], c, FAST ? beyond : tab[place + 16 * x + r]) - lse[b]);
                            float da = e * (dp[b][i][r] - delta[b]);
                            if (!FAST) da = ((t[b] >= 0) & !lone[b] & ((uint32_t)(16 * x + r - from) <= span)) ? da : 0.f;
                            s[b][i][r] = da;
                            if (FAST) outer += da;
                        }
                        if (!FAST && g.part) {
                            const float2 v = g.lgp == 0 ? Slant<1>::sum(s[b][i]) : g.lgp == 1 ? Slant<2>::sum(s[b][i]) : Slant<4>::sum(s[b][i]);
                            main[b][x] = v.x;
                            over[b][x] = v.y;
                        }
                    }
                phase();
                fold<T, DP, QB>(lds + M::K, u, s, o, now);
            }
            if (FAST) {
#pragma unroll
                for (int b = 0; b < QB; ++b) {
                    outer += carry[b];
                    carry[b] = 0.f;
                }
            }
            if (!FAST && g.part) {
#pragma unroll
                for (int b = 0; b < QB; ++b) {
                    // entry of the table: (the tile's last step) - (the lane's step) + (its first key)
                    const int at = far - R.past - (((R.r0 + (wave * QB + b) * 16 + an) >> g.lgp)) + 4 * gn;
                    if (g.lgp == 0) {  // what lies beyond a block's first query goes with the next block of keys, of the same lane
                        const float4_t v = {main[b][0] + carry[b], main[b][1] + over[b][0], main[b][2] + over[b][1], main[b][3] + over[b][2]};
                        carry[b] = over[b][3];
                        carry_k = k0 + ATTN_K;
                        add_to_bins<LANES>(bins, idx, at, each, v);
                    } else {
                        add_to_bins<LANES>(bins, idx, at, each, main[b]);
                        add_to_bins<LANES>(bins, idx, at + (16 >> g.lgp), each, over[b]);
                    }
                }
            }
        };
        if (__any(any)) {
            if (!near && __all(all)) tile(std::true_type{});
            else tile(std::false_type{});
        }
        __syncthreads();
    }
    if (*flag) {  // a row that sees such a key has a score that is not finite: no part of its gradient is
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            bool hit = false;
            for (int k = k_begin; k < k_end; ++k) hit |= (t[b] >= 0) & (k >= lo[b]) & (k <= p[b]) && tainted(kb + (int64_t)k * g.k_t, g.D);
            if (!hit) continue;
            const float nan = __builtin_nanf("");
#pragma unroll
            for (int dt = 0; dt < L::NB; ++dt) o[b][dt] = float4_t{nan, nan, nan, nan};
            if (!g.part) continue;
            for (int d = 0, end = p[b] - lo[b] + 1; d < end;) {  // the buckets of the distances that it sees, each by its first one
                const int i = g.bucket[d];
                bins[(i < 0 ? 0 : i >= g.B ? g.B - 1 : i) * LANES] = nan;
                int next = end;
                while (next - d > 1) {
                    const int mid = d + (next - d) / 2;
                    if (g.bucket[mid] > i) next = mid;
                    else d = mid;
                }
                d = next;
            }
        }
    }
    if (g.cut_q.chunks > 1) {
        if (threadIdx.x == 0) g.cut_q.there[R.chunk * g.total + (R.n * (g.H >> g.lgp) + (R.h0 >> g.lgp)) * g.tiles + R.r0 / BQ] = k_begin < k_end;
        const int64_t all = (int64_t)g.N * g.H * g.T;
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            if (t[b] < 0 || k_begin >= k_end) continue;
            float* to = g.cut_q.o + (R.chunk * all + ((int64_t)R.n * g.H + R.h0 + hh) * g.T + t[b]) * DP + 4 * gr;
#pragma unroll
            for (int dt = 0; dt < L::NB; ++dt) *reinterpret_cast<float4_t*>(to + 16 * dt) = o[b][dt];
        }
    } else {
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            const int first = R.r0 + (wave * QB + b) * 16;
            put_rows<T, DP, WHOLE>(lds + wave * 16 * L::OPITCH, o[b], g.scale, g.D, [&](int row) -> T* {
                const int r = first + row;
                if (r >= R.rows) return nullptr;
                return reinterpret_cast<T*>(g.dq) + (int64_t)(r >> g.lgp) * g.q_t + (int64_t)R.n * g.q_n + (int64_t)(R.h0 + (r & ((1 << g.lgp) - 1))) * g.D;
            });
        }
    }
    if (!g.part) return;
    by_halves<LANES>([&] { bins[(g.B - 1) * LANES] += outer; });
    if (g.lgp == 0) {
#pragma unroll
        for (int b = 0; b < QB; ++b) {  // (rows that are not there may lie between the last tile's keys and the block's last row)
            int d = R.past + R.r0 + (wave * QB + b) * 16 + a - carry_k - 4 * gr;
            d = d < 0 ? 0 : d >= g.reach ? g.reach - 1 : d;
            const int i = g.bucket[d];
            by_halves<LANES>([&] { bins[(i < 0 ? 0 : i >= g.B ? g.B - 1 : i) * LANES] += carry[b]; });
        }
    }
    __syncthreads();
    // eight threads a bucket: each adds up an eighth of its lanes (of one head, in an order that touches no bank twice) of all four waves
    const int64_t parts = g.parts, mine = ((int64_t)R.n * g.tiles + R.r0 / BQ) * g.cut_q.chunks + R.chunk;
    const int part = threadIdx.x & 7, head = part & ((1 << g.lgp) - 1), eighth = part >> g.lgp;
    for (int b0 = 0; b0 < g.B; b0 += 32) {
        const int b = b0 + (threadIdx.x >> 3);
        float sum = 0.f;
        if (b < g.B) {
            constexpr int EACH = LANES / 8;
            const float* from = reinterpret_cast<const float*>(lds + M::BINS) + b * LANES + head;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int at = (eighth * EACH + ((i + b) & (EACH - 1))) << g.lgp, wave_ = g.B * LANES;
                sum += (from[at] + from[at + wave_]) + (from[at + 2 * wave_] + from[at + 3 * wave_]);
            }
        }
        for (int o = 1 << g.lgp; o < 8; o <<= 1) sum += __shfl_xor(sum, o);
        if (b < g.B && part < 1 << g.lgp) g.part[((int64_t)(R.h0 + head) * g.B + b) * parts + mine] = sum;
    }
}

// dbias[h, b]: the workgroups' sums, a workgroup of the next launch each (of a launch of their own: 5 us)
__device__ inline void add_bias(const AttnArgs& g, float* part) {
    const float* src = g.part + (int64_t)blockIdx.x * g.parts;
    float sum = 0.f;
    for (int64_t i = threadIdx.x; i < g.parts; i += ATTN_THREADS) sum += src[i];
#pragma unroll
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) g.dbias[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// ---- backward, keys: dk and dv ---------------------------------------------------------------------------------------------------
// Four waves, 16 keys each in registers, and a tile of 64 rows of queries at a time.  512 environments, 64 of 128 steps, 8 heads of 64: 110 us (330 MB,
// 3.0 TB/s: one tile to a workgroup, most of its time is the wait for it; workgroups that go on to a next tile and ask for it ahead 133, three waves
// a SIMD 140); 2048 x 8 x 8 heads of 128 to 2 of keys: 345 us (206 GF of parts, 0.6 PFLOP/s): two waves a SIMD, 14 to 46 registers in memory, half of the
// time in waits.
template <typename T, int DP, int KB>
struct DkvLds {
    static constexpr int ROOM = ATTN_ROOM(ATTN_K, 64 * KB), NR = (ROOM + ATTN_THREADS - 1) / ATTN_THREADS;
    static constexpr int Q = 0, O = Tile<T, DP>::BYTES, TAB = 2 * O, INFO = TAB + ROOM * 4, FLAG = INFO + 3 * ATTN_K * 4, TOTAL = FLAG + 16;
};
template <typename T, int DP, int KB, bool WHOLE, int LGP>
__global__ __launch_bounds__(ATTN_THREADS, attn_waves(2, sizeof(T), DP)) void k_attn_dkv(AttnArgs given) {
    AttnArgs g = given;
    g.lgp = LGP;
    typedef Tile<T, DP> L;
    typedef DkvLds<T, DP, KB> M;
    extern __shared__ __align__(16) unsigned char lds[];
    float* tab = reinterpret_cast<float*>(lds + M::TAB);
    float* row_lse = reinterpret_cast<float*>(lds + M::INFO);
    float* row_delta = row_lse + ATTN_K;
    int* row_lo = reinterpret_cast<int*>(row_delta + ATTN_K);
    int* flag = reinterpret_cast<int*>(lds + M::FLAG);
    if (blockIdx.x < g.before) return add_bias(g, reinterpret_cast<float*>(lds));
    constexpr int BK = 64 * KB;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, a = lane & 15, gr = lane >> 4;
    const Place at(g);
    Rows R;
    R.n = (int)g.by_heads.quotient(at.rest);
    R.kv = (int)(at.rest - R.n * g.KV);
    R.past = g.S - g.T;
    const int k0 = (g.tiles - 1 - at.tile) * BK, k_last = (k0 + BK < g.S ? k0 + BK : g.S) - 1;
    Operand<T> kf[KB][L::KS], vf[KB][L::KS];
    int key[KB];
    float4_t dk[KB][L::NB], dv[KB][L::NB];
#pragma unroll
    for (int b = 0; b < KB; ++b) {
        key[b] = k0 + (wave * KB + b) * 16 + a;
        const bool in = key[b] < g.S;
        const int64_t at = (int64_t)(in ? key[b] : 0) * g.k_t + (int64_t)R.n * g.k_n + (int64_t)R.kv * g.D;
#pragma unroll
        for (int ks = 0; ks < L::KS; ++ks) {
            const int d = ks * 32 + gr * 8;
            RowOperand<T, WHOLE> uk, uv;
            uk.load(reinterpret_cast<const T*>(g.k) + at, d, g.D);
            uv.load(reinterpret_cast<const T*>(g.v) + at, d, g.D);
            kf[b][ks] = uk.get(d, g.D, in);
            vf[b][ks] = uv.get(d, g.D, in);
        }
#pragma unroll
        for (int dt = 0; dt < L::NB; ++dt) dk[b][dt] = dv[b][dt] = float4_t{0.f, 0.f, 0.f, 0.f};
    }
    if (threadIdx.x == 0) *flag = 0;
    if (!g.table)
        for (int i = threadIdx.x; i < M::ROOM; i += ATTN_THREADS) tab[i] = 0.f;
    const int pack = 1 << g.lgp, share = g.share, each = (ATTN_K >> g.lgp) + BK;
    const int last_edge = g.table ? g.edges[g.B - 1] : 0;
    const float c = g.scale * kLog2e;
    const int t_begin = k0 > R.past ? k0 - R.past : 0;
    // The steps that may see a key here end where the window or an episode does (lo never falls).  The walk is one from its end: workgroups of one
    // environment then meet at the same rows at the same time, which the L2 holds (2048 x 8 x 8 heads of 128 to 2 of keys: 1.6 million requests miss it,
    // from each one's own first row on 5.9 million; 3% of the time).
    const int64_t t_far = (int64_t)k_last + g.window - R.past;
    int t_end = t_far < g.T ? (int)t_far : g.T;
    if (g.lo && (t_end - t_begin) << g.lgp > 4 * ATTN_K) {
        int from = t_begin;
        while (from < t_end) {
            const int stride = (t_end - from + 63) / 64, t = from + lane * stride;
            const uint64_t over = __ballot(t >= t_end || R.lo(g, R.past + (t < t_end ? t : t_end - 1)) > k_last);
            const int one = over ? __ffsll((long long)over) - 1 : 64;
            if (one == 0) {
                t_end = from;
            } else {
                const int upto = from + one * stride;
                t_end = upto < t_end ? upto : t_end;
                from += (one - 1) * stride + 1;
            }
        }
    }
    int r_begin = (t_begin << g.lgp) & ~3, r_end = t_end << g.lgp;
    if (g.cut.chunks > 1) {
        const int tiles = r_end > r_begin ? (r_end - r_begin + ATTN_K - 1) / ATTN_K : 0, upto = tiles - at.chunk * g.cut.span, from = upto - g.cut.span;
        r_end = at.chunk == 0 ? r_end : r_begin + (upto > 0 ? upto : 0) * ATTN_K;
        r_begin += (from > 0 ? from : 0) * ATTN_K;
    }
    const int r_last = r_begin < r_end ? r_begin + (r_end - 1 - r_begin) / ATTN_K * ATTN_K : r_begin - ATTN_K;  // where the last tile of rows begins
    bool some = false;  // (of a chunk: has a row been looked at)
    for (int h0 = R.kv * share; h0 < (R.kv + 1) * share; h0 += pack) {
        const T* qb = reinterpret_cast<const T*>(g.q) + (int64_t)R.n * g.q_n + (int64_t)h0 * g.D;
        const T* ob = reinterpret_cast<const T*>(g.dy) + (int64_t)R.n * g.y_n + (int64_t)h0 * g.D;
        Stage<T, DP, WHOLE> sq, so;
        Table<M::NR> st;
        sq.init(g.q_t, g.lgp, g.D);
        so.init(g.y_t, g.lgp, g.D);
        float i_lse = 0.f, i_delta = 0.f;
        int i_lo = kNever;
        float beyond[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) beyond[r] = g.table ? g.bias[(int64_t)(h0 + (r & (pack - 1))) * g.B + g.B - 1] * kLog2e : 0.f;
        auto near_at = [&](int r0) { return g.table && R.past + (r0 >> g.lgp) - k_last < last_edge; };
        auto request = [&](int r0) {
            sq.load(qb, g.q_t, r0, r_end, g.lgp, g.D);
            so.load(ob, g.y_t, r0, r_end, g.lgp, g.D);
            if (g.table) st.template load<false>(g, h0, each, R.past + (r0 >> g.lgp) - (k0 + BK - 1), 1);
            if (threadIdx.x < ATTN_K) {
                const int r = r0 + threadIdx.x;
                i_lo = kNever;
                if (r < r_end) {
                    const int tt = r >> g.lgp;
                    const int64_t row = ((int64_t)R.n * g.H + h0 + (r & (pack - 1))) * g.T + tt;
                    i_lse = g.lse[row];
                    i_delta = g.delta[row];
                    i_lo = R.lo(g, R.past + tt);
                }
            }
        };
        if (r_begin < r_end) request(r_last);
        __syncthreads();
        for (int r0 = r_last; r0 >= r_begin; r0 -= ATTN_K) {
            const bool near = near_at(r0);
            const bool mq = sq.template put<true>(lds + M::Q, r0, r_end, g.D), mo = so.template put<true>(lds + M::O, r0, r_end, g.D);
            if (mq | mo) *flag = 1;
            if (g.table) st.template put<false>(g, each, tab, nullptr);
            if (threadIdx.x < ATTN_K) {
                row_lse[threadIdx.x] = i_lse;
                row_delta[threadIdx.x] = i_delta;
                row_lo[threadIdx.x] = i_lo;
            }
            __syncthreads();
            if (r0 > r_begin) request(r0 - ATTN_K);
            const bool seen = row_lo[0] <= k_last;  // (of a short walk: an episode may end it earlier)
            some |= seen;
            const int p0 = R.past + (r0 >> g.lgp);
            auto tile = [&](auto fast) {
                constexpr bool FAST = decltype(fast)::value;
                const int now = lane_now();
#pragma unroll
                for (int u = 0; u < L::NU; ++u) {
                    float4_t s[KB][L::NX], e[KB][L::NX];
                    phase();
#pragma unroll
                    for (int i = 0; i < L::NX; ++i) {
                        const int x = u * L::NX + i;
                        if (i && DP > 64) phase();
#pragma unroll
                        for (int b = 0; b < KB; ++b) s[b][i] = e[b][i] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int ks = 0; ks < L::KS; ++ks) {
                            const Operand<T> f = L::rows(lds + M::Q, 16 * x, ks, now), fo = L::rows(lds + M::O, 16 * x, ks, now);
#pragma unroll
                            for (int b = 0; b < KB; ++b) {
                                multiply(f.p, kf[b][ks].p, s[b][i]);
                                multiply(fo.p, vf[b][ks].p, e[b][i]);
                            }
                        }
                    }
                    phase();
#pragma unroll
                    for (int i = 0; i < L::NX; ++i) {
                        const int row = 16 * (u * L::NX + i) + 4 * (now >> 4);
                        const float4_t lse = *reinterpret_cast<const float4_t*>(row_lse + row), delta = *reinterpret_cast<const float4_t*>(row_delta + row);
                        const int4 lo4 = *reinterpret_cast<const int4*>(row_lo + row);
                        const int lo[4] = {lo4.x, lo4.y, lo4.z, lo4.w};
#pragma unroll
                        for (int b = 0; b < KB; ++b) {
                            const float* place = tab + (row >> g.lgp) + (k0 + BK - 1 - key[b]);
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const int step = r >> g.lgp;
                                const float shift = FAST ? beyond[r] : place[(r & (pack - 1)) * each + step];
                                float v = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i][r], c, shift) - lse[r]), da = v * (e[b][i][r] - delta[r]);
                                if (!FAST) {
                                    const int p = p0 + (row >> g.lgp) + step;
                                    const bool see = (lo[r] <= key[b]) & (key[b] <= p);
                                    v = see ? v : 0.f;
                                    da = (see & (lo[r] != p)) ? da : 0.f;  // (a row that sees itself only: nothing, see above)
                                }
                                e[b][i][r] = v;
                                s[b][i][r] = da;
                            }
                        }
                    }
                    phase();
                    fold<T, DP, KB>(lds + M::O, u, e, dv, now);
                    fold<T, DP, KB>(lds + M::Q, u, s, dk, now);
                }
            };
            if (seen) {
                if (!near && row_lo[ATTN_K - 1] <= k0 && p0 >= k0 + BK - 1) tile(std::true_type{});
                else tile(std::false_type{});
            }
            __syncthreads();
        }
        if (*flag) {  // an undefined q: undefined probabilities; an undefined dy: undefined dA, and itself in dv
            for (int r = r_begin; r < r_end; ++r) {
                const int tt = r >> g.lgp, p = R.past + tt, lo = R.lo(g, p);
                const T *qr = qb + (int64_t)tt * g.q_t + (r & (pack - 1)) * g.D, *orow = ob + (int64_t)tt * g.y_t + (r & (pack - 1)) * g.D;
                const bool bad_q = tainted(qr, g.D), bad_o = tainted(orow, g.D);
                if (!(bad_q | bad_o)) continue;
                const float nan = __builtin_nanf("");
#pragma unroll
                for (int b = 0; b < KB; ++b) {
                    const bool see = (lo <= key[b]) & (key[b] <= p);
                    if (!see) continue;
#pragma unroll
                    for (int dt = 0; dt < L::NB; ++dt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int d = 16 * dt + 4 * gr + e;
                            const float v = d < g.D ? to_f(orow[d]) : 0.f;
                            dk[b][dt][e] = nan;
                            dv[b][dt][e] += bad_q ? nan : finite(v) ? 0.f : v;
                        }
                }
            }
            __syncthreads();  // (the next heads' walk may set it again)
        }
    }
    if (g.cut.chunks > 1) {
        if (threadIdx.x == 0) g.cut.there[at.chunk * g.total + at.rest * g.tiles + k0 / BK] = some;
        if (!some) return;
        const int64_t all = (int64_t)g.S * g.N * g.KV;
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            if (key[b] >= g.S) continue;
            float* to = g.cut.o + (at.chunk * all + ((int64_t)key[b] * g.N + R.n) * g.KV + R.kv) * DP + 4 * gr;
#pragma unroll
            for (int dt = 0; dt < L::NB; ++dt) {
                *reinterpret_cast<float4_t*>(to + 16 * dt) = dk[b][dt];
                *reinterpret_cast<float4_t*>(to + g.cut.chunks * all * DP + 16 * dt) = dv[b][dt];
            }
        }
        return;
    }
#pragma unroll
    for (int b = 0; b < KB; ++b) {
        const int first = k0 + (wave * KB + b) * 16;
        const auto place = [&](void* base, int row) -> T* {
            return first + row < g.S ? reinterpret_cast<T*>(base) + (int64_t)(first + row) * g.k_t + (int64_t)R.n * g.k_n + (int64_t)R.kv * g.D : nullptr;
        };
        put_rows<T, DP, WHOLE>(lds + wave * 16 * L::OPITCH, dk[b], g.scale, g.D, [&](int row) { return place(g.dk, row); });
        put_rows<T, DP, WHOLE>(lds + wave * 16 * L::OPITCH, dv[b], 1.f, g.D, [&](int row) { return place(g.dv, row); });
    }
}

// The parts of a row's gradient, added up in the chunks' order: DP / 4 lanes a row, four columns each
template <int DP>
__device__ inline float4_t add_parts(const Cut& c, const float* from, int64_t rows, uint32_t total, uint32_t workgroup) {
    float4_t sum = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < c.chunks; ++i) {
        if (!c.there[i * total + workgroup]) continue;
        const float4_t v = *reinterpret_cast<const float4_t*>(from + i * rows * DP);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += v[e];
    }
    return sum;
}
template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attn_dq_join(AttnArgs g, int queries) {
    constexpr int LANES = DP / 4;
    const int64_t all = (int64_t)g.N * g.H * g.T, row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    if (row >= all) return;
    const int d = threadIdx.x % LANES * 4, t = (int)(row % g.T), h = (int)(row / g.T % g.H), n = (int)(row / g.T / g.H);
    const uint32_t workgroup = (n * (g.H >> g.lgp) + (h >> g.lgp)) * g.tiles + ((t << g.lgp) + (h & ((1 << g.lgp) - 1))) / queries;
    const float4_t v = add_parts<DP>(g.cut_q, g.cut_q.o + row * DP + d, all, g.total, workgroup);
    T* to = reinterpret_cast<T*>(g.dq) + (int64_t)t * g.q_t + (int64_t)n * g.q_n + (int64_t)h * g.D;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (d + i < g.D) to[d + i] = cvt<T>(v[i] * g.scale);
}
template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attn_dkv_join(AttnArgs g, int keys) {
    constexpr int LANES = DP / 4;
    const int64_t all = (int64_t)g.S * g.N * g.KV, row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    if (row >= all) return;
    const int d = threadIdx.x % LANES * 4, kv = (int)(row % g.KV), n = (int)(row / g.KV % g.N), s = (int)(row / g.KV / g.N);
    const uint32_t workgroup = (n * g.KV + kv) * g.tiles + s / keys;
    const float* from = g.cut.o + row * DP + d;
    const float4_t dk = add_parts<DP>(g.cut, from, all, g.total, workgroup), dv = add_parts<DP>(g.cut, from + g.cut.chunks * all * DP, all, g.total, workgroup);
    const int64_t at = (int64_t)s * g.k_t + (int64_t)n * g.k_n + (int64_t)kv * g.D;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (d + i >= g.D) continue;
        reinterpret_cast<T*>(g.dk)[at + d + i] = cvt<T>(dk[i] * g.scale);
        reinterpret_cast<T*>(g.dv)[at + d + i] = cvt<T>(dv[i]);
    }
}

// ---- host -------------------------------------------------------------------------------------------------------------------
// query heads of a tile: the power of two that divides the heads of a head of keys, up to 4
static int pack_bits(const morlax_attn_dims& d) {
    const int share = d.heads / d.kv_heads;
    return share % 4 == 0 ? 2 : share % 2 == 0 ? 1 : 0;
}
static int padded(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : 128; }
// rows of queries that a workgroup of the forward takes: two blocks of 16 a wave in long bf16 heads where there are rows for them
static int fwd_rows(const morlax_attn_dims& d) { return d.dtype && d.head_dim > 64 && ((int64_t)d.T << pack_bits(d)) > 64 ? 128 : 64; }
// Where the workgroups are no more than the chip holds at once, the time is that of the longest walk (earlier keys are seen by more rows, later rows see
// more keys), and most of the chip is idle at its end: such walks are cut until there is work for the chip twice over, into no chunk of under eight
// tiles, as each part is written and read again.  4099 steps of 2 x 4 fp32 heads of 32, forward (260 workgroups, 1024 places): 149 us in one piece,
// 99 in seven (with today's sums of products 110); dk and dv of 2048 x 8 x 8 heads of 128 to 2 of keys (512 workgroups, 512 places): 519 in one piece, 382 in two, 433
// in four.  The forward of the latter (1024 workgroups of twice the rows): 200 in one piece, 308 in four.
// One environment's 4096 steps, 4 bf16 heads of 64 (256 workgroups): forward 105, dq 102, dk and dv 150 us in one piece; 66, 75 and 105 cut, with their
// joins.
static Cut cut(int waves, int64_t workgroups, int64_t tiles) {
    int64_t c = 2 * 256 * waves / workgroups;
    c = c < tiles / 8 ? c : tiles / 8;
    c = c < 8 ? c : 8;
    Cut r = {};
    r.chunks = c > 1 ? (int)c : 1;
    r.span = (int)cdiv(tiles, r.chunks);
    return r;
}
// pass 0, 1: `rows` rows of queries to a workgroup, along the keys; 2: 64 keys, along the queries
static Cut cut_of(const morlax_attn_dims& d, int pass, int rows) {
    const int lgp = pack_bits(d), waves = attn_waves(pass, d.dtype ? 2 : 4, padded(d.head_dim));
    const int64_t reach = (int64_t)d.window + (pass == 2 ? rows : rows >> lgp), most = pass == 2 ? d.T : d.S, seen = reach < most ? reach : most;
    return pass == 2 ? cut(waves, cdiv(d.S, rows) * d.N * d.kv_heads, cdiv((seen << lgp) + 3, ATTN_K))
                     : cut(waves, cdiv((int64_t)d.T << lgp, rows) * d.N * (d.heads >> lgp), cdiv(seen, ATTN_K));
}
static AttnArgs attn_args(const morlax_attn_dims& d) {
    AttnArgs g = {};
    g.T = d.T; g.S = d.S; g.N = d.N; g.H = d.heads; g.KV = d.kv_heads; g.D = d.head_dim; g.B = d.buckets; g.window = d.window;
    g.reach = d.window < d.S ? d.window : d.S;
    g.scale = d.scale;
    g.whole = d.head_dim % (d.dtype ? 8 : 4) == 0;
    g.lgp = pack_bits(d);
    g.share = d.heads / d.kv_heads;
    g.q_t = d.q_t; g.q_n = d.q_n; g.k_t = d.k_t; g.k_n = d.k_n; g.y_t = d.y_t; g.y_n = d.y_n;
    return g;
}
template <typename P>
static int64_t carve(P*& p, int64_t at, void* base, int64_t bytes) {
    p = base ? reinterpret_cast<P*>(reinterpret_cast<char*>(base) + at) : nullptr;
    return at + align_up(bytes, 256);
}
// episodes and the bias by distance: in `saved` where there is one, else in the workspace
static int64_t attn_carve_prepared(AttnArgs& g, void* base, int64_t at) {
    at = carve(g.lo, at, base, (int64_t)g.N * g.S * 4);
    if (g.B) {
        at = carve(g.table, at, base, (int64_t)g.H * g.reach * 4);
        at = carve(g.bucket, at, base, (int64_t)g.reach * 4);
    }
    return at;
}
static int64_t attn_carve_saved(AttnArgs& g, const morlax_attn_dims& d, void* saved) {
    int64_t at = carve(g.lse, 0, saved, (int64_t)g.N * g.H * g.T * 4);
    if (d.dtype) at = carve(g.low, at, saved, (int64_t)g.T * g.N * g.H * g.D * 2);
    return attn_carve_prepared(g, saved, at);
}
#define ATTN_ROWS 64  // the fewest rows of queries of a workgroup
static int64_t attn_carve_fwd(AttnArgs& g, const morlax_attn_dims& d, void* ws, int64_t at) {
    g.cut = cut_of(d, 0, fwd_rows(d));
    if (g.cut.chunks == 1) return at;
    const int64_t rows = (int64_t)g.cut.chunks * g.N * g.H * g.T;
    at = carve(g.cut.m, at, ws, rows * 8);
    return carve(g.cut.o, at, ws, rows * padded(g.D) * 4);
}
static int64_t attn_carve_bwd(AttnArgs& g, const morlax_attn_dims& d, void* ws) {
    int64_t at = carve(g.delta, 0, ws, (int64_t)g.N * g.H * g.T * 4);
    g.cut_q = cut_of(d, 1, ATTN_ROWS);
    if (g.cut_q.chunks > 1) {
        at = carve(g.cut_q.there, at, ws, (int64_t)g.cut_q.chunks * g.N * (g.H >> g.lgp) * cdiv((int64_t)g.T << g.lgp, ATTN_ROWS) * 4);
        at = carve(g.cut_q.o, at, ws, (int64_t)g.cut_q.chunks * g.N * g.H * g.T * padded(g.D) * 4);
    }
    g.cut = cut_of(d, 2, 64);
    if (g.cut.chunks > 1) {
        at = carve(g.cut.there, at, ws, (int64_t)g.cut.chunks * g.N * g.KV * cdiv(g.S, 64) * 4);
        at = carve(g.cut.o, at, ws, 2 * (int64_t)g.cut.chunks * g.S * g.N * g.KV * padded(g.D) * 4);
    }
    if (g.B) at = carve(g.part, at, ws, (int64_t)g.H * g.B * g.N * cdiv((int64_t)g.T << g.lgp, ATTN_ROWS) * g.cut_q.chunks * 4);
    return at;
}
int64_t attn_saved_bytes(const morlax_attn_dims& d) {
    AttnArgs g = attn_args(d);
    return attn_carve_saved(g, d, nullptr);
}
int64_t attn_ws_bytes(const morlax_attn_dims& d, bool back) {
    AttnArgs g = attn_args(d);
    return back ? attn_carve_bwd(g, d, nullptr) : attn_carve_fwd(g, d, nullptr, attn_carve_prepared(g, nullptr, 0));
}

static int run_kernel(void (*kernel)(AttnArgs), AttnArgs& g, int64_t total, int chunks, int lds, hipStream_t s) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return 1;
    g.total = (uint32_t)total;
    const uint32_t rests = g.total / g.tiles;
    g.own = rests % 8 == 0 && rests <= 128 ? rests / 8 : 0;
    g.by_total = row_div((int)g.total);
    g.by_tiles = row_div(g.tiles);
    g.by_own = row_div(g.own ? (int)g.own : 1);
    g.by_heads = row_div((int)(rests / g.N));
    if (g.before + total * chunks >= 1 << 24) {  // (a launch holds fewer than 2^32 threads: what else there is to do in one of its own)
        kernel<<<dim3(g.before), ATTN_THREADS, lds, s>>>(g);
        g.before = 0;
    }
    kernel<<<dim3((uint32_t)(g.before + total * chunks)), ATTN_THREADS, lds, s>>>(g);
    return 0;
}
template <typename T, int DP, int QB, bool WHOLE, int LGP, bool FINE = false>
static int attn_fwd_pass(AttnArgs& g, hipStream_t s) {
    if constexpr (!FINE && sizeof(T) == 2) {
        if (g.low) return attn_fwd_pass<T, DP, QB, WHOLE, LGP, true>(g, s);
    }
    g.tiles = (int)cdiv((int64_t)g.T << g.lgp, 64 * QB);
    if (run_kernel(k_attn_fwd<T, DP, QB, WHOLE, FINE, LGP>, g, (int64_t)g.tiles * g.N * (g.H >> g.lgp), g.cut.chunks, FwdLds<T, DP, QB>::TOTAL, s)) return 1;
    if (g.cut.chunks > 1) k_attn_fwd_join<T, DP><<<dim3((uint32_t)cdiv((int64_t)g.N * g.H * g.T * (DP / 4), 256)), 256, 0, s>>>(g);
    return 0;
}
template <typename T, int DP, int QB, bool WHOLE, int LGP>
static int attn_dq_pass(AttnArgs& g, hipStream_t s) {
    g.tiles = (int)cdiv((int64_t)g.T << g.lgp, 64 * QB);
    g.parts = (int64_t)g.N * g.tiles * g.cut_q.chunks;
    if (run_kernel(k_attn_dq<T, DP, QB, WHOLE, LGP>, g, (int64_t)g.tiles * g.N * (g.H >> g.lgp), g.cut_q.chunks,
                   DqLds<T, DP, QB>::BINS + (g.part ? g.B * DqLds<T, DP, QB>::LANES * 16 : 0), s))
        return 1;
    if (g.cut_q.chunks > 1) k_attn_dq_join<T, DP><<<dim3((uint32_t)cdiv((int64_t)g.N * g.H * g.T * (DP / 4), 256)), 256, 0, s>>>(g, 64 * QB);
    if (g.part) g.before = (uint32_t)(g.H * g.B);  // (of the next launch)
    return 0;
}
template <typename T, int DP, int KB, bool WHOLE, int LGP>
static int attn_dkv_pass(AttnArgs& g, hipStream_t s) {
    g.tiles = (int)cdiv(g.S, 64 * KB);
    if (run_kernel(k_attn_dkv<T, DP, KB, WHOLE, LGP>, g, (int64_t)g.tiles * g.N * g.KV, g.cut.chunks, DkvLds<T, DP, KB>::TOTAL, s)) return 1;
    if (g.cut.chunks > 1) k_attn_dkv_join<T, DP><<<dim3((uint32_t)cdiv((int64_t)g.S * g.N * g.KV * (DP / 4), 256)), 256, 0, s>>>(g, 64 * KB);
    return 0;
}
// A wave takes one block of 16 rows; in the forward pass of long bf16 heads two where there are rows for them, as what is read of a tile then serves
// both (2048 x 8 x 8 heads of 128: 167 us, one block 186; heads of 64, 64 steps: 77, one block 72; the backward kernels run out of registers).
template <typename T, int DP, bool WHOLE, int LGP>
static int attn_packed(AttnArgs& g, bool back, hipStream_t s) {
    constexpr int MORE = sizeof(T) == 2 && DP == 128 ? 2 : 1;  // (fwd_rows says the same)
    if (!back) return ((int64_t)g.T << LGP) > 64 ? attn_fwd_pass<T, DP, MORE, WHOLE, LGP>(g, s) : attn_fwd_pass<T, DP, 1, WHOLE, LGP>(g, s);
    return attn_dq_pass<T, DP, 1, WHOLE, LGP>(g, s) || attn_dkv_pass<T, DP, 1, WHOLE, LGP>(g, s);
}
template <typename T, int DP, bool WHOLE>
static int attn_whole(AttnArgs& g, bool back, hipStream_t s) {
    return g.lgp == 0 ? attn_packed<T, DP, WHOLE, 0>(g, back, s) : g.lgp == 1 ? attn_packed<T, DP, WHOLE, 1>(g, back, s) : attn_packed<T, DP, WHOLE, 2>(g, back, s);
}
template <typename T, int DP>
static int attn_rows(AttnArgs& g, bool back, hipStream_t s) {
    return g.whole ? attn_whole<T, DP, true>(g, back, s) : attn_whole<T, DP, false>(g, back, s);
}
template <typename T>
static int attn_pick(AttnArgs& g, bool back, hipStream_t s) {
    if (g.D <= 32) return attn_rows<T, 32>(g, back, s);
    if (g.D <= 64) return attn_rows<T, 64>(g, back, s);
    return attn_rows<T, 128>(g, back, s);
}

int launch_attn_fwd(const morlax_attn_dims& d, const void* q, const void* k, const void* v, const float* bias, const int32_t* edges,
                    const uint8_t* first, void* y, void* saved, void* ws, hipStream_t s) {
    AttnArgs g = attn_args(d);
    g.q = q; g.k = k; g.v = v; g.bias = bias; g.edges = edges; g.first = first; g.out = y;
    const int64_t at = attn_carve_prepared(g, ws, 0);
    attn_carve_fwd(g, d, ws, at);
    if (saved) attn_carve_saved(g, d, saved);
    if (!first) g.lo = nullptr;
    if (first || g.B) {
        // up to 16 environments to a workgroup, whose flags lie next to each other; of few with long histories fewer, for runs of two steps
        int lgn = 0;
        while (lgn < 4 && 1 << lgn < d.N && (1024 >> lgn >= d.S || d.N >> lgn > 64)) ++lgn;
        const int64_t spans = first ? cdiv(d.N, 1 << lgn) : 0;
        k_attn_prepare<<<dim3((uint32_t)(spans + (g.B ? cdiv((int64_t)g.H * g.reach, 1024) : 0))), 1024, 0, s>>>(g, (int)spans, lgn);
    }
    return d.dtype ? attn_pick<bf16_t>(g, false, s) : attn_pick<float>(g, false, s);
}
int launch_attn_bwd(const morlax_attn_dims& d, const void* q, const void* k, const void* v, const float* bias, const int32_t* edges,
                    const uint8_t* first, const void* y, const void* saved, const void* dy, void* dq, void* dk, void* dv, float* dbias, void* ws,
                    hipStream_t s) {
    AttnArgs g = attn_args(d);
    g.q = q; g.k = k; g.v = v; g.bias = bias; g.edges = edges; g.first = first; g.y = y; g.dy = dy;
    g.dq = dq; g.dk = dk; g.dv = dv; g.dbias = dbias;
    attn_carve_saved(g, d, const_cast<void*>(saved));
    attn_carve_bwd(g, d, ws);
    if (!first) g.lo = nullptr;
    if (!dbias) g.part = nullptr;
    return d.dtype ? attn_pick<bf16_t>(g, true, s) : attn_pick<float>(g, true, s);
}
