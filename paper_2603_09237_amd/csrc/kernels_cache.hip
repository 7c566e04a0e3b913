// A paged cache of keys and values, one step at a time: the pages' bookkeeping, and the attention of every environment's new step over it.
#include "attn_tile.h"

static int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---- pages --------------------------------------------------------------------------------------------------------------
// Integers only: a workgroup owns 64 environments (256 of many), one a thread of its first waves; ranks (whose turn at the queue it is, where a page that goes back lies) are
// sums over the workgroups before, which a first launch leaves where there is more than one.  Bound by latency for a few thousand environments
// (two dependent launches of some microseconds), by the copy of the tables where they go into other buffers (16384 environments of 64 slots: 14 us, in
// place 9.5).
// A page may come late, in the middle of its rows or a round of the slots later: the rows that its steps have not reached hold what others left.  `since`
// says from which step on a slot's page is the episode's: the step that took it.
#define PAGES_THREADS 256
#define PAGES_AHEAD 8
struct PagesArgs {
    const uint8_t* first;
    const int32_t *length_in, *table_in, *queue_in, *state_in;
    int32_t *length, *table, *queue, *state, *slot;
    const int32_t* since_in;
    int32_t* since;    // [N, slots], or NULL
    int2* sums;        // of each workgroup: environments that need a page, pages that go back
    int32_t* was;      // [2] the state before
    int N, lgp, lge, slots, pages, blocks;  // lge: 2^lge environments to a workgroup
    RowDiv by_slots;
};

// of two values at once, over a workgroup of 256: the sums before a thread's, and of all (x, y; z, w)
__device__ inline int4 block_before(int u, int v, int2* lds4) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int a = u, b = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int c = __shfl_up(a, o), d = __shfl_up(b, o);
        if (lane >= o) {
            a += c;
            b += d;
        }
    }
    if (lane == 63) lds4[wave] = make_int2(a, b);
    __syncthreads();
    int4 r = make_int4(a - u, b - v, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int2 w = lds4[i];
        if (i < wave) {
            r.x += w.x;
            r.y += w.y;
        }
        r.z += w.x;
        r.w += w.y;
    }
    return r;
}

struct PageOf {  // what one environment does
    bool live, begins, needs;
    int at, column, entry;
    __device__ inline void look(const PagesArgs& g, int n) {
        live = begins = needs = false;
        at = column = 0;
        entry = -1;
        if (n >= g.N) return;
        at = g.length_in[n];
        live = at >= 0;
        if (!live) return;
        begins = g.first && g.first[n];
        if (begins) at = 0;
        column = (int)((uint32_t)(at >> g.lgp) % (uint32_t)g.slots);
        entry = g.table_in[(int64_t)n * g.slots + column];
        needs = (uint32_t)entry >= (uint32_t)g.pages;
    }
};
// The pages that the environments of this wave give back, an environment at a time, all lanes along its slots: each(place among the wave's, page);
// returns how many for this lane's environment.
template <typename F>
__device__ inline int wave_gives(const PagesArgs& g, int n, bool begins, F each) {
    const int lane = threadIdx.x & 63;
    uint64_t todo = __ballot(begins);
    int mine = 0, done = 0;
    while (todo) {
        const int who = __ffsll((long long)todo) - 1;
        todo &= todo - 1;
        const int32_t* row = g.table_in + (int64_t)__shfl(n, who) * g.slots;
        int count = 0;
        for (int j0 = 1; j0 < g.slots; j0 += 64) {
            const int j = j0 + lane;
            const int e = j < g.slots ? row[j] : -1;
            const bool held = (uint32_t)e < (uint32_t)g.pages;
            const uint64_t set = __ballot(held);
            if (held) each(done + count + __popcll(set & (((uint64_t)1 << lane) - 1)), e);
            count += __popcll(set);
        }
        if (lane == who) mine = count;
        done += count;
    }
    return mine;
}

__global__ __launch_bounds__(PAGES_THREADS) void k_pages_count(PagesArgs g) {
    __shared__ int2 part[4];
    const int n = (int)threadIdx.x < 1 << g.lge ? ((int)blockIdx.x << g.lge) + (int)threadIdx.x : g.N;
    PageOf e;
    e.look(g, n);
    const int gives = wave_gives(g, n, e.begins, [](int, int) {});
    const int4 own = block_before(e.needs, gives, part);
    if (threadIdx.x == 0) {
        g.sums[blockIdx.x] = make_int2(own.z, own.w);
        if (blockIdx.x == 0) {
            g.was[0] = g.state_in[0];
            g.was[1] = g.state_in[1];
        }
    }
}

__global__ __launch_bounds__(PAGES_THREADS) void k_pages_apply(PagesArgs g) {
    __shared__ int2 part[4], sums[4], totals[4];
    __shared__ int wave_back[4];
    __shared__ int32_t column[PAGES_THREADS], entry[PAGES_THREADS], from[PAGES_THREADS];
    const int n0 = (int)blockIdx.x << g.lge, wave = threadIdx.x >> 6;
    const int n = (int)threadIdx.x < 1 << g.lge ? n0 + (int)threadIdx.x : g.N;
    const int here = g.N - n0 < 1 << g.lge ? g.N - n0 : 1 << g.lge, cells = here * g.slots;
    // the tables' first entries and the workgroups' sums, requested ahead of what they wait for
    int32_t ahead[PAGES_AHEAD];
    if (g.table != g.table_in)
#pragma unroll
        for (int i = 0; i < PAGES_AHEAD; ++i) {
            const int at = threadIdx.x + i * PAGES_THREADS;
            ahead[i] = g.table_in[(int64_t)n0 * g.slots + (at < cells ? at : 0)];
        }
    int a = 0, b = 0, c = 0, d = 0, head, count;
    if (g.blocks > 1) {
        for (int i = threadIdx.x; i < g.blocks; i += PAGES_THREADS) {
            const int2 s = g.sums[i];
            a += i < (int)blockIdx.x ? s.x : 0;
            b += i < (int)blockIdx.x ? s.y : 0;
            c += s.x;
            d += s.y;
        }
        head = g.was[0];
        count = g.was[1];
    } else {
        head = g.state_in[0];
        count = g.state_in[1];
    }
    PageOf e;
    e.look(g, n);
    const int gives = wave_gives(g, n, e.begins, [](int, int) {});  // (each pushes them below, once the place is known)
    const int4 own = block_before(e.needs, gives, part);  // (its barrier stands between the state's reads and its write: it may be its own output)
    int needs_before = 0, back_before = 0, needs_all = own.z, back_all = own.w;
    if (g.blocks > 1) {
        const int4 u = block_before(a, b, sums), v = block_before(c, d, totals);
        needs_before = u.z;
        back_before = u.w;
        needs_all = v.z;
        back_all = v.w;
    }
    head = (int)((uint32_t)head % (uint32_t)g.pages);
    count = count < 0 ? 0 : count > g.pages ? g.pages : count;
    auto ring = [&](int64_t i) { return (int)((uint64_t)i % (uint32_t)g.pages); };
    const int rank = needs_before + own.x;
    if (e.needs && rank < count) e.entry = g.queue_in[ring((int64_t)head + rank)];
    column[threadIdx.x] = !e.live ? -1 : e.begins ? -2 - e.column : e.column;  // (an episode that begins is at slot 0)
    entry[threadIdx.x] = e.entry;
    if ((threadIdx.x & 63) == 0) wave_back[wave] = own.y;
    if (g.since && e.live) {  // (a step that is still to come kept nothing)
        const int old = g.since_in[(int64_t)n * g.slots + e.column], now = e.begins | e.needs | (old > e.at) ? e.at : old;
        from[threadIdx.x] = now;
        if (g.since == g.since_in) g.since[(int64_t)n * g.slots + e.column] = now;
    }
    if (n < g.N) {
        const bool has = (uint32_t)e.entry < (uint32_t)g.pages;
        g.length[n] = e.live ? e.at + 1 : e.at;
        g.slot[n] = e.live && has ? (e.entry << g.lgp) + (e.at & ((1 << g.lgp) - 1)) : -1;
    }
    const int64_t tail = (int64_t)head + count + back_before;
    __syncthreads();
    const int64_t base = tail + wave_back[wave];
    wave_gives(g, n, e.begins, [&](int at, int page) { g.queue[ring(base + at)] = page; });
    __syncthreads();  // (the rows of episodes that begin have been read: they may be written)
    if (g.table != g.table_in) {
        const int32_t* old = g.table_in + (int64_t)n0 * g.slots;
        int32_t* to = g.table + (int64_t)n0 * g.slots;
        auto put = [&](int i, int was) {
            const int r = (int)g.by_slots.quotient((uint32_t)i), j = i - r * g.slots, c = column[r], now = entry[r];
            to[i] = c <= -2 ? (j == 0 ? now : -1) : c == j ? now : was;
        };
#pragma unroll
        for (int i = 0; i < PAGES_AHEAD; ++i) {
            const int at = threadIdx.x + i * PAGES_THREADS;
            if (at < cells) put(at, ahead[i]);
        }
#pragma unroll 4
        for (int i = threadIdx.x + PAGES_AHEAD * PAGES_THREADS; i < cells; i += PAGES_THREADS) put(i, old[i]);
    } else if (n < g.N && e.live) {
        if (e.begins)
            for (int j = 1; j < g.slots; ++j) g.table[(int64_t)n * g.slots + j] = -1;
        g.table[(int64_t)n * g.slots + e.column] = e.entry;
    }
    if (g.since != g.since_in)
        for (int i = threadIdx.x; i < cells; i += PAGES_THREADS) {
            const int r = (int)g.by_slots.quotient((uint32_t)i), j = i - r * g.slots, c = column[r];
            const int64_t at = (int64_t)n0 * g.slots + i;
            g.since[at] = j == (c <= -2 ? 0 : c) ? from[r] : g.since_in[at];
        }
    if (g.queue != g.queue_in) {  // what no page went back to
        const int64_t per = ((int64_t)g.pages + g.blocks - 1) / g.blocks, i0 = blockIdx.x * per, i1 = i0 + per < g.pages ? i0 + per : g.pages;
        const int tail0 = ring((int64_t)head + count);
        for (int64_t i = i0 + threadIdx.x; i < i1; i += PAGES_THREADS) {
            const int64_t d = i - tail0 < 0 ? i - tail0 + g.pages : i - tail0;
            if (d >= back_all) g.queue[i] = g.queue_in[i];
        }
    }
    if ((int)blockIdx.x == g.blocks - 1 && threadIdx.x == 0) {
        const int taken = needs_all < count ? needs_all : count;
        const int64_t left = (int64_t)count - taken + back_all;
        g.state[0] = ring((int64_t)head + taken);
        g.state[1] = left > g.pages ? g.pages : (int)left;
    }
}

// ---- one new step over the cache ------------------------------------------------------------------------------------------------
// Bound: HBM, every key and value of the window once (the query heads that share a head of keys share what is read), split over the length and joined
// where few environments have to fill the chip.  fp32: a key lies along LPK lanes, 16 bytes each, so a wave takes 64 / LPK keys at a time; every group
// of LPK lanes carries a running maximum, sum and output of its own, which are joined once at the end, across the groups, the waves and the
// workgroups of a length (33 environments, 384 steps, 6 heads of 40: 9 us and 3.5 for the join, latency of dependent loads: length, table, key).
struct StepArgs {
    const void *q, *k, *v;
    const float* bias;
    const int32_t *edges, *table, *length, *since;
    void *k_cache, *v_cache, *y;
    float* part_o;   // [N, H, splits, D]
    float2* part_m;  // [N, H, splits] maximum (in units of log2) and sum
    float scale;
    int N, H, KV, D, B, window, lgp, slots, pages, splits, chunks, whole;
    int64_t q_n, k_n, y_n;
};

__device__ inline float element(const uint4& u, int i) { return __uint_as_float(i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w); }  // i known after unrolling

#define STEP_U 4  // keys that a group of lanes requests together

template <int CTRL>
__device__ inline float moved(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true)); }
// the sum over a group of L lanes, in all of them: within four, then the other four (mirrored), the other eight, the other sixteen
template <int L>
__device__ inline float group_sum(float v) {
    v += moved<0xb1>(v);
    v += moved<0x4e>(v);
    if (L > 4) v += moved<0x141>(v);
    if (L > 8) v += moved<0x140>(v);
    if (L > 16) v += __shfl_xor(v, 16);
    return v;
}

// SINCE: pages may have come late, and steps from before are not seen (an instance of its own, as the word of each key costs 1024 environments 1 us of
// 54 in bf16, 4 of 122 in fp32).
template <int DP, int GQ, bool WHOLE, bool SINCE>
__global__ __launch_bounds__(256) void k_attn_step(StepArgs g) {
    typedef float T;
    constexpr int VE = 4, LPK = DP / VE, KPW = 64 / LPK, STRIDE = 4 * KPW * STEP_U;
    __shared__ float bias[GQ][64];
    __shared__ int32_t edges[64];  // those that are not there: no distance reaches them
    __shared__ float2 wave_m[4][GQ];
    __shared__ float wave_o[4][GQ][DP];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % LPK, key = lane / LPK;
    const int split = blockIdx.x % g.splits, rest = blockIdx.x / g.splits, chunk = rest % g.chunks, rest2 = rest / g.chunks;
    const int kv = rest2 % g.KV, n = rest2 / g.KV, share = g.H / g.KV, h0 = kv * share + chunk * GQ, heads = share - chunk * GQ < GQ ? share - chunk * GQ : GQ;
    const int length = g.length[n], pos = length - 1;
    const int d = sub * VE;
    T* y = reinterpret_cast<T*>(g.y) + (int64_t)n * g.y_n;
    if (length <= 0) {
        if (g.splits == 1)
            for (int i = threadIdx.x; i < heads * g.D; i += 256) y[(int64_t)h0 * g.D + i] = (T)0.f;
        return;
    }
    const int begin = pos - g.window + 1 > 0 ? pos - g.window + 1 : 0;
    // this workgroup's part of the window, a whole number of keys of its waves
    const uint32_t count = pos - begin + 1, per = ((count + g.splits - 1) / g.splits + 4 * KPW - 1) / (4 * KPW) * (4 * KPW);  // (sums pass 2^31)
    const int64_t s0 = begin + (int64_t)split * per;
    const int s1 = s0 + per < pos + 1 ? (int)(s0 + per) : pos + 1;
    const int32_t *table = g.table + (int64_t)n * g.slots, *since = SINCE ? g.since + (int64_t)n * g.slots : nullptr;
    const int64_t row = (int64_t)g.KV * g.D;
    const T *kn = reinterpret_cast<const T*>(g.k) + (int64_t)n * g.k_n + (int64_t)kv * g.D, *vn = reinterpret_cast<const T*>(g.v) + (int64_t)n * g.k_n + (int64_t)kv * g.D;
    T *kc = reinterpret_cast<T*>(g.k_cache) + (int64_t)kv * g.D, *vc = reinterpret_cast<T*>(g.v_cache) + (int64_t)kv * g.D;
    const int slot0 = (begin >> g.lgp) % g.slots, page0 = begin >> g.lgp, in_page = (1 << g.lgp) - 1;
    auto slot_of = [&](int s) {  // (the window's pages lie once round the slots at most)
        const int j = slot0 + (s >> g.lgp) - page0;
        return j >= g.slots ? j - g.slots : j;
    };
    if (split == 0 && chunk == 0) {  // the step goes into its page; no workgroup reads it there
        const int id = table[slot_of(pos)];
        if ((uint32_t)id < (uint32_t)g.pages) {
            const int64_t at = (((int64_t)id << g.lgp) + (pos & in_page)) * row;
            for (int i = threadIdx.x; i < g.D; i += 256) {
                kc[at + i] = kn[i];
                vc[at + i] = vn[i];
            }
        }
    }
    float qf[GQ][VE];
#pragma unroll
    for (int i = 0; i < GQ; ++i) {
        RowPiece<T, WHOLE> in;
        in.load(reinterpret_cast<const T*>(g.q) + (int64_t)n * g.q_n + (int64_t)(h0 + (i < heads ? i : 0)) * g.D, d, g.D);
        const uint4 u = in.get(d, g.D);
#pragma unroll
        for (int e = 0; e < VE; ++e) qf[i][e] = element(u, e);
    }
    int last_edge = 0;
    if (g.B) {
        if (threadIdx.x < 64) edges[threadIdx.x] = (int)threadIdx.x < g.B ? g.edges[threadIdx.x] : 0x7fffffff;
        for (int i = threadIdx.x; i < GQ * g.B; i += 256) bias[i / g.B][i % g.B] = i / g.B < heads ? g.bias[(int64_t)(h0 + i / g.B) * g.B + i % g.B] * kLog2e : 0.f;
        last_edge = g.edges[g.B - 1];
    }
    __syncthreads();
    const float c = g.scale * kLog2e;
    float m[GQ], l[GQ], o[GQ][VE];
#pragma unroll
    for (int i = 0; i < GQ; ++i) {
        m[i] = -__builtin_inff();
        l[i] = 0.f;
#pragma unroll
        for (int e = 0; e < VE; ++e) o[i][e] = 0.f;
    }
    const int my = wave * KPW + key;
    int id[STEP_U], from[SINCE ? STEP_U : 1];
    auto look = [&](int64_t at) {
#pragma unroll
        for (int u = 0; u < STEP_U; ++u) {
            const int64_t s = at + my + u * 4 * KPW;
            const int j = slot_of((int)(s < s1 ? s : s1 - 1));
            id[u] = table[j];
            if (SINCE) from[u] = since[j];
        }
    };
    if (s0 < s1) look(s0);
    for (int64_t at = s0; at < s1; at += STRIDE) {
        RowPiece<T, WHOLE> kp[STEP_U], vp[STEP_U];
        bool in[STEP_U];
#pragma unroll
        for (int u = 0; u < STEP_U; ++u) {
            const int64_t s = at + my + u * 4 * KPW;
            const bool now = s == pos;
            in[u] = (s < s1) & (now | (((uint32_t)id[u] < (uint32_t)g.pages) & (!SINCE || s >= from[SINCE ? u : 0])));
            const int64_t off = (((int64_t)id[u] << g.lgp) + ((int)s & in_page)) * row;
            const bool held = in[u] & !now;
            kp[u].load(held ? kc + off : kn, d, g.D);
            vp[u].load(held ? vc + off : vn, d, g.D);
        }
        if (at + STRIDE < s1) look(at + STRIDE);
        float s[STEP_U][GQ];
#pragma unroll
        for (int u = 0; u < STEP_U; ++u) {
#pragma unroll
            for (int i = 0; i < GQ; ++i) s[u][i] = 0.f;
            const uint4 ku = kp[u].get(d, g.D, in[u]);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float x = element(ku, e);
#pragma unroll
                for (int i = 0; i < GQ; ++i) s[u][i] = __builtin_fmaf(x, qf[i][e], s[u][i]);
            }
#pragma unroll
            for (int i = 0; i < GQ; ++i) s[u][i] = group_sum<LPK>(s[u][i]);
            int b = g.B - 1;
            const int dist = pos - (int)(at + my + u * 4 * KPW);
            if (dist < last_edge) {  // the last edge that is not beyond the distance (one by one: 5 us of a workgroup's time)
                b = 0;
#pragma unroll
                for (int x = 32; x; x >>= 1) b += edges[b + x] <= dist ? x : 0;
            }
#pragma unroll
            for (int i = 0; i < GQ; ++i) {
                const float a = __builtin_fmaf(s[u][i], c, g.B ? bias[i][b] : 0.f);
                s[u][i] = in[u] ? a : -__builtin_inff();
            }
        }
#pragma unroll
        for (int i = 0; i < GQ; ++i) {
            float top = m[i];
#pragma unroll
            for (int u = 0; u < STEP_U; ++u) top = fmaxf(top, s[u][i]);
            const float base = top == -__builtin_inff() ? 0.f : top, fade = __builtin_amdgcn_exp2f(m[i] - base);
            m[i] = top;
            l[i] *= fade;
#pragma unroll
            for (int e = 0; e < VE; ++e) o[i][e] *= fade;
#pragma unroll
            for (int u = 0; u < STEP_U; ++u) {
                s[u][i] = __builtin_amdgcn_exp2f(s[u][i] - base);
                l[i] += s[u][i];
            }
        }
#pragma unroll
        for (int u = 0; u < STEP_U; ++u) {
            const uint4 vu = vp[u].get(d, g.D, in[u]);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float x = element(vu, e);
#pragma unroll
                for (int i = 0; i < GQ; ++i) o[i][e] = __builtin_fmaf(s[u][i], x, o[i][e]);
            }
        }
    }
    // joined: the groups of a wave, then the waves
#pragma unroll
    for (int i = 0; i < GQ; ++i) {
        float top = m[i];
#pragma unroll
        for (int x = LPK; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
        const float base = top == -__builtin_inff() ? 0.f : top, w = __builtin_amdgcn_exp2f(m[i] - base);
        l[i] *= w;
#pragma unroll
        for (int x = LPK; x < 64; x <<= 1) l[i] += __shfl_xor(l[i], x);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            o[i][e] *= w;
#pragma unroll
            for (int x = LPK; x < 64; x <<= 1) o[i][e] += __shfl_xor(o[i][e], x);
        }
        if (lane < LPK) {
            if (lane == 0) wave_m[wave][i] = make_float2(top, l[i]);
#pragma unroll
            for (int e = 0; e < VE; ++e) wave_o[wave][i][d + e] = o[i][e];
        }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < heads * DP; x += 256) {
        const int i = x / DP, dd = x % DP;
        if (dd >= g.D) continue;
        float top = wave_m[0][i].x;
#pragma unroll
        for (int w = 1; w < 4; ++w) top = fmaxf(top, wave_m[w][i].x);
        const float base = top == -__builtin_inff() ? 0.f : top;
        float sum = 0.f, out = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(wave_m[w][i].x - base);
            sum = __builtin_fmaf(f, wave_m[w][i].y, sum);
            out = __builtin_fmaf(f, wave_o[w][i][dd], out);
        }
        if (g.splits == 1) {
            y[(int64_t)(h0 + i) * g.D + dd] = cvt<T>(out / sum);
        } else {
            const int64_t at = ((int64_t)n * g.H + h0 + i) * g.splits + split;
            if (dd == 0) g.part_m[at] = make_float2(top, sum);
            g.part_o[at * g.D + dd] = out;
        }
    }
}

// ---- one new step over the cache, bf16: on the matrix instructions ------------------------------------------------------------------
// Up to sixteen query heads that share a head of keys are the columns of a product's result, 32 keys its rows: the arithmetic of a key is then a
// few instructions of a wave whatever the number of heads (one lane's products and sums for every head: a step of 1024 environments, four heads to a
// head of keys, 82 us, bound by them; so 55, 4.9 TB/s, step after step over the same cache, and 67, 4.0 TB/s, where every step finds another one, as the 256 MB
// beside the HBM then hold nothing of it; one environment of 8192 steps 6.4 and 4.4 for the join, latency).  A lane's two rows of keys and values come straight from the cache; values go through LDS, which turns them.
template <int DP>
struct StepLds {
    typedef Tile<bf16_t, DP> L;
    static constexpr int V = 32 * L::PITCH, OUT = 16 * (DP + 1) * 4, WAVE = V > OUT ? V : OUT;  // (a wave's output lies where its values lay)
};
template <int DP, bool WHOLE, bool SINCE>
__global__ __launch_bounds__(256, DP == 128 ? 2 : 3) void k_attn_step_bf16(StepArgs g) {
    typedef bf16_t T;
    typedef Tile<T, DP> L;
    __shared__ __align__(16) unsigned char lds[4 * StepLds<DP>::WAVE];
    __shared__ float bias[16][65];
    __shared__ int32_t edges[64];  // those that are not there: no distance reaches them
    __shared__ __align__(16) int32_t buckets[4][32];
    __shared__ float2 wave_m[4][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, a = lane & 15, gr = lane >> 4;
    const int split = blockIdx.x % g.splits, rest = blockIdx.x / g.splits, chunk = rest % g.chunks, rest2 = rest / g.chunks;
    const int kv = rest2 % g.KV, n = rest2 / g.KV, share = g.H / g.KV, h0 = kv * share + chunk * 16, heads = share - chunk * 16 < 16 ? share - chunk * 16 : 16;
    const int length = g.length[n], pos = length - 1;
    T* y = reinterpret_cast<T*>(g.y) + (int64_t)n * g.y_n;
    if (length <= 0) {
        if (g.splits == 1)
            for (int i = threadIdx.x; i < heads * g.D; i += 256) y[(int64_t)h0 * g.D + i] = (T)0.f;
        return;
    }
    const int begin = pos - g.window + 1 > 0 ? pos - g.window + 1 : 0;
    const uint32_t count = pos - begin + 1, per = ((count + g.splits - 1) / g.splits + 127) / 128 * 128;  // a whole number of keys of the four waves
    const int64_t s0 = begin + (int64_t)split * per;
    const int s1 = s0 + per < pos + 1 ? (int)(s0 + per) : pos + 1;
    const int32_t *table = g.table + (int64_t)n * g.slots, *since = SINCE ? g.since + (int64_t)n * g.slots : nullptr;
    const int64_t row = (int64_t)g.KV * g.D;
    const T *kn = reinterpret_cast<const T*>(g.k) + (int64_t)n * g.k_n + (int64_t)kv * g.D, *vn = reinterpret_cast<const T*>(g.v) + (int64_t)n * g.k_n + (int64_t)kv * g.D;
    T *kc = reinterpret_cast<T*>(g.k_cache) + (int64_t)kv * g.D, *vc = reinterpret_cast<T*>(g.v_cache) + (int64_t)kv * g.D;
    const int slot0 = (begin >> g.lgp) % g.slots, page0 = begin >> g.lgp, in_page = (1 << g.lgp) - 1;
    auto slot_of = [&](int s) {  // (the window's pages lie once round the slots at most)
        const int j = slot0 + (s >> g.lgp) - page0;
        return j >= g.slots ? j - g.slots : j;
    };
    if (split == 0 && chunk == 0) {  // the step goes into its page; no workgroup reads it there
        const int id = table[slot_of(pos)];
        if ((uint32_t)id < (uint32_t)g.pages) {
            const int64_t at = (((int64_t)id << g.lgp) + (pos & in_page)) * row;
            for (int i = threadIdx.x; i < g.D; i += 256) {
                kc[at + i] = kn[i];
                vc[at + i] = vn[i];
            }
        }
    }
    Operand<T> qf[L::KS];
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks) {
        const int d = 32 * ks + 8 * gr;
        RowPiece<T, WHOLE> u;
        u.load(reinterpret_cast<const T*>(g.q) + (int64_t)n * g.q_n + (int64_t)(h0 + (a < heads ? a : 0)) * g.D, d, g.D);
        qf[ks].p[0] = u.get(d, g.D, a < heads);
    }
    int last_edge = 0;
    float beyond = 0.f;
    if (g.B) {
        if (threadIdx.x < 64) edges[threadIdx.x] = (int)threadIdx.x < g.B ? g.edges[threadIdx.x] : 0x7fffffff;
        for (int i = threadIdx.x; i < 16 * g.B; i += 256) {
            const int h = i / g.B, b = i - h * g.B;
            bias[h][b] = h < heads ? g.bias[(int64_t)(h0 + h) * g.B + b] * kLog2e : 0.f;
        }
        last_edge = g.edges[g.B - 1];
    }
    __syncthreads();
    if (g.B) beyond = bias[a][g.B - 1];
    const float c = g.scale * kLog2e;
    unsigned char* mine = lds + wave * StepLds<DP>::WAVE;
    float m = -__builtin_inff(), l = 0.f;
    float4_t o[1][L::NB];
#pragma unroll
    for (int dt = 0; dt < L::NB; ++dt) o[0][dt] = float4_t{0.f, 0.f, 0.f, 0.f};
    int id[2], from[SINCE ? 2 : 1];
    RowPiece<T, WHOLE> kp[2][L::KS], vp[2][L::KS];
    bool in[2];
    auto look = [&](int64_t at) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int64_t s = at + 16 * x + a;
            const int j = slot_of((int)(s < s1 ? s : s1 - 1));
            id[x] = table[j];
            if (SINCE) from[x] = since[j];
        }
    };
    auto request = [&](int64_t at) {  // (its pages' numbers are there) and the next one's numbers
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int64_t s = at + 16 * x + a;
            const bool now = s == pos;
            in[x] = (s < s1) & (now | (((uint32_t)id[x] < (uint32_t)g.pages) & (!SINCE || s >= from[SINCE ? x : 0])));
            const bool held = in[x] & !now;
            const int64_t off = (((int64_t)id[x] << g.lgp) + ((int)s & in_page)) * row;
            const T *pk = held ? kc + off : kn, *pv = held ? vc + off : vn;
#pragma unroll
            for (int ks = 0; ks < L::KS; ++ks) {
                kp[x][ks].load(pk, 32 * ks + 8 * gr, g.D);
                vp[x][ks].load(pv, 32 * ks + 8 * gr, g.D);
            }
        }
        look(at + 128);
    };
    int64_t at = s0 + 32 * wave;
    if (at < s1) {
        look(at);
        request(at);
    }
    for (; at < s1; at += 128) {
        float4_t s[1][2];
        // which of the 32 keys are there, a bit each (a lane's keys: 4 gr + r of both halves)
        const uint32_t there0 = (uint32_t)__ballot(in[0]) & 0xffff, there1 = (uint32_t)__ballot(in[1]) & 0xffff;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            s[0][x] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < L::KS; ++ks) {
                const int d = 32 * ks + 8 * gr;
                Mma16<T>::run(kp[x][ks].get(d, g.D, in[x]), qf[ks].p[0], s[0][x]);
                *reinterpret_cast<uint4*>(mine + (16 * x + a) * L::PITCH + d * 2) = vp[x][ks].get(d, g.D, in[x]);
            }
        }
        if (at + 128 < s1) request(at + 128);
        const bool near = g.B && pos - (int)(at + 31) < last_edge;
        if (near && lane < 32) {  // the bucket of a key: the last edge that is not beyond its distance
            const int dist = pos - (int)(at + lane);
            int b = 0;
#pragma unroll
            for (int x = 32; x; x >>= 1) b += edges[b + x] <= dist ? x : 0;
            buckets[wave][lane] = b;
        }
        __builtin_amdgcn_wave_barrier();
        float top = m;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint32_t bits = (x ? there1 : there0) >> (4 * gr);
            int4 b4 = make_int4(0, 0, 0, 0);
            if (near) b4 = *reinterpret_cast<const int4*>(&buckets[wave][16 * x + 4 * gr]);
            const int b[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float v = __builtin_fmaf(s[0][x][r], c, near ? bias[a][b[r]] : beyond);
                s[0][x][r] = (bits >> r) & 1 ? v : -__builtin_inff();
                top = fmaxf(top, s[0][x][r]);
            }
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float base = top == -__builtin_inff() ? 0.f : top;
        if (__any(top != m)) {
            const float fade = __builtin_amdgcn_exp2f(m - base);
            l *= fade;
#pragma unroll
            for (int dt = 0; dt < L::NB; ++dt)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[0][dt][r] *= fade;
        }
        m = top;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[0][x][r] = __builtin_amdgcn_exp2f(s[0][x][r] - base);
                l += s[0][x][r];
            }
        Computed<2> p;
        p.set(s[0]);
#pragma unroll
        for (int dt = 0; dt < L::NB; ++dt) multiply(L::turned(mine, 0, dt, lane).p, p.p, o[0][dt]);
        __builtin_amdgcn_wave_barrier();
    }
    // joined: the waves
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (gr == 0) wave_m[wave][a] = make_float2(m, l);
    float* out = reinterpret_cast<float*>(mine);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int dt = 0; dt < L::NB; ++dt)
#pragma unroll
        for (int r = 0; r < 4; ++r) out[a * (DP + 1) + 16 * dt + 4 * gr + r] = o[0][dt][r];
    __syncthreads();
    for (int x = threadIdx.x; x < heads * DP; x += 256) {
        const int i = x / DP, dd = x % DP;
        if (dd >= g.D) continue;
        float top = wave_m[0][i].x;
#pragma unroll
        for (int w = 1; w < 4; ++w) top = fmaxf(top, wave_m[w][i].x);
        const float base = top == -__builtin_inff() ? 0.f : top;
        float sum = 0.f, acc = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(wave_m[w][i].x - base);
            sum = __builtin_fmaf(f, wave_m[w][i].y, sum);
            acc = __builtin_fmaf(f, *reinterpret_cast<const float*>(lds + w * StepLds<DP>::WAVE + (i * (DP + 1) + dd) * 4), acc);
        }
        if (g.splits == 1) {
            y[(int64_t)(h0 + i) * g.D + dd] = cvt<T>(acc / sum);
        } else {
            const int64_t p = ((int64_t)n * g.H + h0 + i) * g.splits + split;
            if (dd == 0) g.part_m[p] = make_float2(top, sum);
            g.part_o[p * g.D + dd] = acc;
        }
    }
}

// the parts of an environment and head, joined: a workgroup each, every wave a quarter of them
template <typename T>
__global__ __launch_bounds__(256) void k_attn_join(StepArgs g) {
    __shared__ float sums[4], outs[4][128];
    const int64_t i = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = (int)(i / g.H), h = (int)(i % g.H);
    T* y = reinterpret_cast<T*>(g.y) + (int64_t)n * g.y_n + (int64_t)h * g.D;
    if (g.length[n] <= 0) {
        if ((int)threadIdx.x < g.D) y[threadIdx.x] = (T)0.f;
        return;
    }
    const float2* pm = g.part_m + i * g.splits;
    const float* po = g.part_o + i * g.splits * g.D;
    const int d0 = lane < g.D ? lane : 0, d1 = lane + 64 < g.D ? lane + 64 : 0;
    float top = -__builtin_inff();
    for (int s = lane; s < g.splits; s += 64) top = fmaxf(top, pm[s].x);
#pragma unroll
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float base = top == -__builtin_inff() ? 0.f : top;
    float sum = 0.f, out[2] = {0.f, 0.f};
#pragma unroll 8
    for (int s = wave; s < g.splits; s += 4) {
        const float2 p = pm[s];
        const float a = po[(int64_t)s * g.D + d0], b = po[(int64_t)s * g.D + d1];
        const float f = __builtin_amdgcn_exp2f(p.x - base);
        sum = __builtin_fmaf(f, p.y, sum);
        out[0] = __builtin_fmaf(f, a, out[0]);
        out[1] = __builtin_fmaf(f, b, out[1]);
    }
    if (lane == 0) sums[wave] = sum;
    outs[wave][lane] = out[0];
    outs[wave][lane + 64] = out[1];
    __syncthreads();
    const int d = threadIdx.x;
    if (d < g.D) y[d] = cvt<T>(((outs[0][d] + outs[1][d]) + (outs[2][d] + outs[3][d])) / ((sums[0] + sums[1]) + (sums[2] + sums[3])));
}

// ---- host ---------------------------------------------------------------------------------------------------------------------------
static int log2_of(int v) {
    int l = 0;
    while (1 << l < v) ++l;
    return l;
}
static int64_t pages_carve(PagesArgs& g, const morlax_pages_dims& d, void* ws) {
    g.N = d.N; g.lgp = log2_of(d.page); g.slots = d.slots; g.pages = d.pages;
    g.lge = d.N <= 65536 ? 6 : 8;
    g.blocks = (int)cdiv(d.N, 1 << g.lge);
    g.by_slots = row_div((uint32_t)d.slots);
    g.was = reinterpret_cast<int32_t*>(ws);
    g.sums = reinterpret_cast<int2*>(reinterpret_cast<char*>(ws) + 256);
    return 256 + (int64_t)g.blocks * 8;
}
int64_t pages_ws_bytes(const morlax_pages_dims& d) {
    PagesArgs g = {};
    return pages_carve(g, d, nullptr);
}
void launch_cache_pages(const morlax_pages_dims& d, const uint8_t* first, const int32_t* length_in, const int32_t* table_in, const int32_t* queue_in,
                        const int32_t* state_in, const int32_t* since_in, int32_t* length, int32_t* table, int32_t* queue, int32_t* state, int32_t* since,
                        int32_t* slot, void* ws, hipStream_t s) {
    PagesArgs g = {};
    g.first = first; g.length_in = length_in; g.table_in = table_in; g.queue_in = queue_in; g.state_in = state_in;
    g.length = length; g.table = table; g.queue = queue; g.state = state; g.slot = slot;
    g.since_in = since_in; g.since = since;
    pages_carve(g, d, ws);
    if (g.blocks > 1) k_pages_count<<<dim3(g.blocks), PAGES_THREADS, 0, s>>>(g);
    k_pages_apply<<<dim3(g.blocks), PAGES_THREADS, 0, s>>>(g);
}

static int heads_of_workgroup(int share) { return share >= 5 ? 8 : share >= 3 ? 4 : share; }
static int64_t step_carve(StepArgs& g, const morlax_cache_dims& d, void* ws) {
    g.N = d.N; g.H = d.heads; g.KV = d.kv_heads; g.D = d.head_dim; g.B = d.buckets; g.window = d.window; g.lgp = log2_of(d.page);
    g.slots = d.slots; g.pages = d.pages; g.scale = d.scale; g.whole = d.head_dim % (d.dtype ? 8 : 4) == 0;
    g.q_n = d.q_n; g.k_n = d.k_n; g.y_n = d.y_n;
    const int share = d.heads / d.kv_heads;
    g.chunks = (int)cdiv(share, d.dtype ? 16 : heads_of_workgroup(share));
    // few environments: the window in as many parts as fill the chip, of 128 keys at least
    const int64_t blocks = (int64_t)d.N * d.kv_heads * g.chunks;
    int64_t splits = 1024 / blocks, most = cdiv(d.window, 128);
    splits = splits < most ? splits : most;
    g.splits = splits < 1 ? 1 : (int)splits;
    if (g.splits == 1) return 16;
    g.part_m = reinterpret_cast<float2*>(ws);
    const int64_t m = align_up((int64_t)d.N * d.heads * g.splits * 8, 256);
    g.part_o = reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + m);
    return m + (int64_t)d.N * d.heads * g.splits * d.head_dim * 4;
}
int64_t attn_step_ws_bytes(const morlax_cache_dims& d) {
    StepArgs g = {};
    return step_carve(g, d, nullptr);
}
template <typename T, int DP, bool WHOLE, bool SINCE>
static void step_run(const StepArgs& g, hipStream_t s) {
    const dim3 grid((uint32_t)((int64_t)g.splits * g.chunks * g.KV * g.N));
    if constexpr (sizeof(T) == 2) k_attn_step_bf16<DP, WHOLE, SINCE><<<grid, 256, 0, s>>>(g);
    else switch (heads_of_workgroup(g.H / g.KV)) {
        case 1: k_attn_step<DP, 1, WHOLE, SINCE><<<grid, 256, 0, s>>>(g); break;
        case 2: k_attn_step<DP, 2, WHOLE, SINCE><<<grid, 256, 0, s>>>(g); break;
        case 4: k_attn_step<DP, 4, WHOLE, SINCE><<<grid, 256, 0, s>>>(g); break;
        default: k_attn_step<DP, 8, WHOLE, SINCE><<<grid, 256, 0, s>>>(g);
    }
    if (g.splits > 1) k_attn_join<T><<<dim3((uint32_t)((int64_t)g.N * g.H)), 256, 0, s>>>(g);
}
template <typename T, int DP, bool WHOLE>
static void step_pass(const StepArgs& g, hipStream_t s) {
    g.since ? step_run<T, DP, WHOLE, true>(g, s) : step_run<T, DP, WHOLE, false>(g, s);
}
template <typename T>
static void step_pick(const StepArgs& g, hipStream_t s) {
    if (g.D <= 32) g.whole ? step_pass<T, 32, true>(g, s) : step_pass<T, 32, false>(g, s);
    else if (g.D <= 64) g.whole ? step_pass<T, 64, true>(g, s) : step_pass<T, 64, false>(g, s);
    else g.whole ? step_pass<T, 128, true>(g, s) : step_pass<T, 128, false>(g, s);
}
void launch_attn_step(const morlax_cache_dims& d, const void* q, const void* k, const void* v, const float* bias, const int32_t* edges,
                      const int32_t* table, const int32_t* length, const int32_t* since, void* k_cache, void* v_cache, void* y, void* ws, hipStream_t s) {
    StepArgs g = {};
    step_carve(g, d, ws);
    g.q = q; g.k = k; g.v = v; g.bias = bias; g.edges = edges; g.table = table; g.length = length; g.since = since; g.k_cache = k_cache; g.v_cache = v_cache; g.y = y;
    if (d.dtype) step_pick<bf16_t>(g, s);
    else step_pick<float>(g, s);
}
