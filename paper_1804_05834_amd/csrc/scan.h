// Gated linear recurrence over time, h_t = a_t k_t h_{t-1} + (1 - a_t) x_t, and its gradients.
//
// A stretch of steps maps the state before it to the state after it by s -> A s + H, and two stretches after
// one another compose to such a map again; going back, what comes from the right goes through by m -> A m + P
// with the same A, the product of the gates.  So a long sequence is cut into short runs of steps, one per thread:
// a thread finds the map of its run, the maps are joined across the threads, and each thread then goes through
// its run once more from the state that enters it.  A run that begins an episode (reset) lets nothing through: its
// A is 0, and what enters is not multiplied by it but dropped, so that a state that is not finite ends there.
//
// Bound by memory: forward reads f and x and writes h once, backward reads f, x and dh and writes df and dx; the
// states are not kept but computed again from one in every tile of steps (`carry`).
#pragma once
#include "seq_common.h"

namespace seq {

struct ScanArgs {
    const void *f, *x;
    long f_bs, f_ts, x_bs, x_ts;
    const float *h0;
    const uint8_t *reset;
    long r_bs, r_ts;
    void *h;
    long h_bs, h_ts;
    float *h_last, *carry;
    long T;
    int B, C;
    // Ranges: few sequences of few channels are cut over time, so that there are enough workgroups.  A first launch finds
    // the map of every range but the last, a second one takes each range from the state that enters it on.
    long range;      // steps of a range (a multiple of the tile)
    int ranges;
    float *totals;   // [B][ranges][2][C]: A (-1: an episode starts in the range) and H of each; the last A: a copy of h0,
                     // which the last range may overwrite (h_last) before the first has read it
    long tiles;      // states per sequence in `carry`
};
struct ScanGradArgs {
    const void *f, *x, *dh;
    long f_bs, f_ts, x_bs, x_ts, dh_bs, dh_ts;
    const float *carry, *dlast;
    const uint8_t *reset;
    long r_bs, r_ts;
    void *df, *dx;
    long df_bs, df_ts, dx_bs, dx_ts;
    float *dh0;
    long T;
    int B, C;
    long range;
    int ranges;
    float *totals;   // A and P of every range but the first
    long tiles;
};

constexpr int SCAN_RUN = 16;        // elements of a thread in a tile: 16 steps of a channel or 4 steps of 4 channels
constexpr int SCAN_STRIP = 64;      // channels of a workgroup
constexpr int SCAN_WAVES = 8;       // most waves of a workgroup
constexpr int SCAN_SHORT = 8;       // longest sequence that a thread goes through alone

// sigmoid(f) and 1 - sigmoid(f).  The second is computed apart: 1 - a of an `a` near one, a memory that lasts, would keep
// few of its digits.
__device__ __forceinline__ void gates(float f, float &a, float &i)
{
    const float e = __builtin_amdgcn_exp2f(-1.44269504088896341f * fabsf(f));
    const float r = __builtin_amdgcn_rcpf(1.f + e), s = e * r;
    a = f < 0.f ? s : r;
    i = f < 0.f ? r : s;
}

// What a thread works on: V channels from c on of sequence b, clamped to the tensor where c is beyond it (then `live` is
// false and nothing is stored).
template <int V> struct Lane {
    int c;
    bool live;
    __device__ Lane(int first, int C) : c(min(first, C - V)), live(first < C) {}
};

template <int V, class T> __device__ __forceinline__ vec<T, V> load(const T *p)
{
    if constexpr (V == 1) return vec<T, 1>{*p};
    else return *reinterpret_cast<const vec<T, V> *>(p);
}
template <int V, class T> __device__ __forceinline__ void store(T *p, vec<T, V> v)
{
    if constexpr (V == 1) *p = v[0];
    else *reinterpret_cast<vec<T, V> *>(p) = v;
}
template <class E, int V> __device__ __forceinline__ vec<E, V> narrow(const float (&v)[V])
{
    vec<E, V> o;
#pragma unroll
    for (int k = 0; k < V; ++k) o[k] = (E)v[k];
    return o;
}
template <int V> __device__ __forceinline__ void state(const float *p, float (&s)[V])
{
    const auto v = load<V>(p);
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = v[k];
}
template <int V> __device__ __forceinline__ void keep_state(float *p, const float (&s)[V]) { store<V>(p, narrow<float, V>(s)); }

// ------------------------------------------------------------ short sequences
__device__ __forceinline__ long sequence_of(long id, long all, int per)   // id / per; in 32 bits where that is enough
{
    return all >> 32 ? id / per : (long)((unsigned)id / (unsigned)per);
}

// A thread takes V channels of a sequence through all of its at most SCAN_SHORT steps; all of its loads go out before
// the first is used.  The step of an acting agent is T = 1.
template <class E, int V> __global__ __launch_bounds__(256) void k_scan_short(ScanArgs A)
{
    const long id = (long)blockIdx.x * 256 + threadIdx.x, all = (long)A.B * (A.C / V);
    if (id >= all) return;
    const long b = sequence_of(id, all, A.C / V);
    const int c = (int)(id - b * (A.C / V)) * V, T = (int)A.T;
    const E *f = (const E *)A.f + b * A.f_bs + c, *x = (const E *)A.x + b * A.x_bs + c;
    vec<E, V> fr[SCAN_SHORT], xr[SCAN_SHORT];
#pragma unroll
    for (int j = 0; j < SCAN_SHORT; ++j)
        if (j < T) { fr[j] = load<V>(f + j * A.f_ts); xr[j] = load<V>(x + j * A.x_ts); }
    float s[V] = {};
    if (A.h0) state<V>(A.h0 + b * A.C + c, s);
    if (A.carry) keep_state<V>(A.carry + b * A.C + c, s);
#pragma unroll
    for (int j = 0; j < SCAN_SHORT; ++j)
        if (j < T) {
            const bool cut = A.reset && A.reset[b * A.r_bs + j * A.r_ts];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                float a, i;
                gates((float)fr[j][k], a, i);
                s[k] = fmaf(a, cut ? 0.f : s[k], i * (float)xr[j][k]);
            }
            store<V>((E *)A.h + b * A.h_bs + j * A.h_ts + c, narrow<E, V>(s));
        }
    if (A.h_last) keep_state<V>(A.h_last + b * A.C + c, s);
}

template <class E, int V> __global__ __launch_bounds__(256) void k_scan_grad_short(ScanGradArgs A)
{
    const long id = (long)blockIdx.x * 256 + threadIdx.x, all = (long)A.B * (A.C / V);
    if (id >= all) return;
    const long b = sequence_of(id, all, A.C / V);
    const int c = (int)(id - b * (A.C / V)) * V, T = (int)A.T;
    const E *f = (const E *)A.f + b * A.f_bs + c, *x = (const E *)A.x + b * A.x_bs + c, *dh = (const E *)A.dh + b * A.dh_bs + c;
    vec<E, V> fr[SCAN_SHORT], xr[SCAN_SHORT], gr[SCAN_SHORT];
    bool cut[SCAN_SHORT];
#pragma unroll
    for (int j = 0; j < SCAN_SHORT; ++j)
        if (j < T) {
            fr[j] = load<V>(f + j * A.f_ts); xr[j] = load<V>(x + j * A.x_ts); gr[j] = load<V>(dh + j * A.dh_ts);
            cut[j] = A.reset && A.reset[b * A.r_bs + j * A.r_ts];
        }
    float mu[V] = {}, s[V] = {}, before[SCAN_SHORT][V];
    if (T) state<V>(A.carry + b * A.C + c, s);
    if (A.dlast) state<V>(A.dlast + b * A.C + c, mu);
#pragma unroll
    for (int j = 0; j < SCAN_SHORT; ++j)
        if (j < T) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                float a, i;
                gates((float)fr[j][k], a, i);
                before[j][k] = cut[j] ? 0.f : s[k];
                s[k] = fmaf(a, before[j][k], i * (float)xr[j][k]);
            }
        }
#pragma unroll
    for (int j = SCAN_SHORT - 1; j >= 0; --j)
        if (j < T) {
            float df[V], dx[V];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                float a, i;
                gates((float)fr[j][k], a, i);
                const float l = (float)gr[j][k] + mu[k];
                dx[k] = i * l;
                df[k] = a * dx[k] * (before[j][k] - (float)xr[j][k]);
                mu[k] = cut[j] ? 0.f : a * l;
            }
            store<V>((E *)A.df + b * A.df_bs + j * A.df_ts + c, narrow<E, V>(df));
            store<V>((E *)A.dx + b * A.dx_bs + j * A.dx_ts + c, narrow<E, V>(dx));
        }
    if (A.dh0) keep_state<V>(A.dh0 + b * A.C + c, mu);
}

// ------------------------------------------------------------ strips
// A workgroup takes a strip of 64 channels through a range of steps, tile by tile.  In a tile a thread has V channels
// and L = 16 / V steps: with V = 4 sixteen lanes are a row of the strip and a wave holds four runs of four steps, with
// V = 1 (sizes, strides or addresses that are not multiples of 4 elements) a wave is one run of sixteen.
template <int V> struct Strip {
    static constexpr int L = SCAN_RUN / V, G = SCAN_STRIP / V, S = 64 / G;
};

// flags of the L steps of a run: bit j is set where step j starts an episode
template <int L> __device__ __forceinline__ unsigned resets(const uint8_t *reset, long r_ts, long t, long end)
{
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < L; ++j) m |= (unsigned)(t + j < end && reset[min(t + j, end - 1) * r_ts] != 0) << j;
    return m;
}

// The maps of the runs of a wave before (UP) or after this lane's: inclusive to exclusive composition across its S runs.
// In: the run's own map, `cuts` a bit per lane whose run starts an episode.  Out: (A, H) of the whole wave, valid in the
// lanes of its last run in this direction, and (xa, xh, xcut) of the runs ahead of this one.
template <int V, bool UP> __device__ __forceinline__ void across(float (&A)[V], float (&H)[V], unsigned long cuts, float (&xa)[V], float (&xh)[V], bool &xcut)
{
    constexpr int G = Strip<V>::G, S = Strip<V>::S;
    const int lane = threadIdx.x & 63, run = UP ? lane / G : S - 1 - lane / G;
    // bit r: run r (counted in this direction) starts an episode
    unsigned c = 0;
#pragma unroll
    for (int r = 0; r < S; ++r) c |= (unsigned)(cuts >> (UP ? r : S - 1 - r) * G & 1) << r;
#pragma unroll
    for (int d = 1; d < S; d *= 2) {
        const bool mine = c >> max(run - d + 1, 0) & ((1u << min(d, run + 1)) - 1);   // an episode starts in what has been joined so far
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float a = UP ? __shfl_up(A[k], d * G) : __shfl_down(A[k], d * G), h = UP ? __shfl_up(H[k], d * G) : __shfl_down(H[k], d * G);
            if (run >= d) {
                H[k] = mine ? H[k] : fmaf(A[k], h, H[k]);
                A[k] = mine ? 0.f : A[k] * a;
            }
        }
    }
    xcut = (c & ((1u << run) - 1)) != 0;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const float a = UP ? __shfl_up(A[k], G) : __shfl_down(A[k], G), h = UP ? __shfl_up(H[k], G) : __shfl_down(H[k], G);
        xa[k] = run ? a : 1.f;
        xh[k] = run ? h : 0.f;
    }
}

template <int V> __device__ __forceinline__ void through(float (&s)[V], const float *A, const float *H, bool cut)
{
    const auto a = load<V>(A), h = load<V>(H);
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = cut ? h[k] : fmaf(a[k], s[k], h[k]);
}

// the same past a range of another workgroup
template <int V> __device__ __forceinline__ void past_range(float (&s)[V], const float *p, int C)
{
    const auto a = load<V>(p), h = load<V>(p + C);
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = a[k] < 0.f ? h[k] : fmaf(a[k], s[k], h[k]);
}

template <class E, int V> struct Rows {   // what a thread reads of a tensor in a tile
    vec<E, V> v[Strip<V>::L];
    // rows t .. t + L - 1, clamped into [0, end)
    __device__ __forceinline__ void load_rows(const E *p, long ts, long t, long end)
    {
#pragma unroll
        for (int j = 0; j < Strip<V>::L; ++j) v[j] = load<V>(p + min(t + j, end - 1) * ts);
    }
};

// TOTAL: nothing is written but the map of the range, for the launch that then takes the ranges from their states on.
template <class E, int V, bool TOTAL> __global__ __launch_bounds__(64 * SCAN_WAVES) void k_scan(ScanArgs A)
{
    constexpr int L = Strip<V>::L, G = Strip<V>::G, S = Strip<V>::S;
    __shared__ float tot[2][2][SCAN_WAVES][SCAN_STRIP];
    __shared__ int cuts[2][SCAN_WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, W = blockDim.x >> 6, g = lane % G, tile = W * S * L;
    const Lane<V> me(blockIdx.x * SCAN_STRIP + g * V, A.C);
    const int z = blockIdx.z;
    const long b = blockIdx.y, t0 = z * A.range, end = min(A.T, t0 + A.range), at = b * A.C + me.c;
    float *totals = A.totals + b * A.ranges * 2 * A.C + me.c;   // (A, H) of range r at 2 r C and (2 r + 1) C
    const E *f = (const E *)A.f + b * A.f_bs + me.c, *x = (const E *)A.x + b * A.x_bs + me.c;
    const uint8_t *reset = A.reset ? A.reset + b * A.r_bs : nullptr;
    const long mine = (long)(wave * S + lane / G) * L;   // first step of this thread in a tile

    float s[V] = {}, all[V];   // state entering the tile; TOTAL: the map so far is s -> all s + s
    bool allcut = false;
#pragma unroll
    for (int k = 0; k < V; ++k) all[k] = 1.f;
    if constexpr (!TOTAL) {
        if (A.ranges > 1) state<V>(totals + (long)(2 * A.ranges - 2) * A.C, s);
        else if (A.h0) state<V>(A.h0 + at, s);
#pragma unroll 8
        for (int r = 0; r < z; ++r) past_range<V>(s, totals + 2l * r * A.C, A.C);
    }
    Rows<E, V> fr, xr;
    unsigned rs = 0;
    fr.load_rows(f, A.f_ts, t0 + mine, end);
    xr.load_rows(x, A.x_ts, t0 + mine, end);
    if (reset) rs = resets<L>(reset, A.r_ts, t0 + mine, end);
    int buf = 0;
    for (long t = t0; t < end; t += tile, buf ^= 1) {
        const long ts = t + mine;
        float ga[L][V], gx[L][V], a[V], h[V];
        const unsigned r = rs;
#pragma unroll
        for (int k = 0; k < V; ++k) { a[k] = 1.f; h[k] = 0.f; }
#pragma unroll
        for (int j = 0; j < L; ++j) {
            const bool in = ts + j < end;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                float i;
                gates((float)fr.v[j][k], ga[j][k], i);
                gx[j][k] = in ? i * (float)xr.v[j][k] : 0.f;     // beyond the end: the map that changes nothing
                if (!in) ga[j][k] = 1.f;
                h[k] = fmaf(ga[j][k], r >> j & 1 ? 0.f : h[k], gx[j][k]);
                a[k] = r >> j & 1 ? 0.f : a[k] * ga[j][k];
            }
        }
        if (t + tile < end) {   // the next tile's loads are in flight behind everything below
            fr.load_rows(f, A.f_ts, ts + tile, end);
            xr.load_rows(x, A.x_ts, ts + tile, end);
            if (reset) rs = resets<L>(reset, A.r_ts, ts + tile, end);
        }
        float xa[V], xh[V];
        bool xcut;
        const unsigned long ball = __ballot(r != 0);
        across<V, true>(a, h, ball, xa, xh, xcut);
        if (lane / G == S - 1) {
            keep_state<V>(&tot[buf][0][wave][g * V], a);
            keep_state<V>(&tot[buf][1][wave][g * V], h);
            if (g == 0) cuts[buf][wave] = ball != 0;
        }
        lds_barrier();
        float in[V];
        for (int w = 0; w < W; ++w) {
            if (w == wave) {
#pragma unroll
                for (int k = 0; k < V; ++k) in[k] = s[k];
            }
            const bool cut = cuts[buf][w];
            if constexpr (TOTAL) {
                const auto m = load<V>(&tot[buf][0][w][g * V]);
#pragma unroll
                for (int k = 0; k < V; ++k) all[k] *= m[k];
                allcut |= cut;
            }
            through<V>(s, &tot[buf][0][w][g * V], &tot[buf][1][w][g * V], cut);
        }
        if constexpr (!TOTAL) {
            if (A.carry && wave == 0 && lane < G && me.live) keep_state<V>(A.carry + (b * A.tiles + t / tile) * A.C + me.c, in);
#pragma unroll
            for (int k = 0; k < V; ++k) in[k] = xcut ? xh[k] : fmaf(xa[k], in[k], xh[k]);
#pragma unroll
            for (int j = 0; j < L; ++j) {
#pragma unroll
                for (int k = 0; k < V; ++k) in[k] = fmaf(ga[j][k], r >> j & 1 ? 0.f : in[k], gx[j][k]);
                if (me.live && ts + j < end) store<V>((E *)A.h + b * A.h_bs + (ts + j) * A.h_ts + me.c, narrow<E, V>(in));
            }
        }
    }
    if (wave || lane >= G || !me.live) return;
    if constexpr (TOTAL) {
#pragma unroll
        for (int k = 0; k < V; ++k) all[k] = allcut ? -1.f : all[k];
        keep_state<V>(totals + 2l * z * A.C, all);
        keep_state<V>(totals + (2l * z + 1) * A.C, s);
        if (z == 0) {
            float h0[V] = {};
            if (A.h0) state<V>(A.h0 + at, h0);
            keep_state<V>(totals + (long)(2 * A.ranges - 2) * A.C, h0);
        }
    } else if (A.h_last && end == A.T) {
        keep_state<V>(A.h_last + at, s);
    }
}

template <class E, int V, bool TOTAL> __global__ __launch_bounds__(64 * SCAN_WAVES) void k_scan_grad(ScanGradArgs A)
{
    constexpr int L = Strip<V>::L, G = Strip<V>::G, S = Strip<V>::S;
    __shared__ float tot[2][3][SCAN_WAVES][SCAN_STRIP];   // A, P and H of the waves
    __shared__ int cuts[2][SCAN_WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, W = blockDim.x >> 6, g = lane % G, tile = W * S * L;
    const Lane<V> me(blockIdx.x * SCAN_STRIP + g * V, A.C);
    const int z = blockIdx.z + (TOTAL ? 1 : 0);
    const long b = blockIdx.y, t0 = z * A.range, end = min(A.T, t0 + A.range), at = b * A.C + me.c;
    float *totals = A.totals + b * A.ranges * 2 * A.C + me.c;
    const E *f = (const E *)A.f + b * A.f_bs + me.c, *x = (const E *)A.x + b * A.x_bs + me.c, *dh = (const E *)A.dh + b * A.dh_bs + me.c;
    const uint8_t *reset = A.reset ? A.reset + b * A.r_bs : nullptr;
    const long mine = (long)(wave * S + lane / G) * L;

    float mu[V] = {}, all[V];   // what comes from the right into the tile; TOTAL: the map so far is m -> all m + mu
    bool allcut = false;
#pragma unroll
    for (int k = 0; k < V; ++k) all[k] = 1.f;
    if constexpr (!TOTAL) {
        if (A.dlast) state<V>(A.dlast + at, mu);
#pragma unroll 8
        for (int r = A.ranges - 1; r > z; --r) past_range<V>(mu, totals + 2l * r * A.C, A.C);
    }
    const long last = t0 + (end - t0 - 1) / tile * tile;
    Rows<E, V> fr, xr, gr;
    unsigned rs = 0;
    float first[V];
    auto fetch = [&](long t) {
        fr.load_rows(f, A.f_ts, t + mine, end);
        if constexpr (!TOTAL) {
            xr.load_rows(x, A.x_ts, t + mine, end);
            state<V>(A.carry + (b * A.tiles + t / tile) * A.C + me.c, first);
        }
        gr.load_rows(dh, A.dh_ts, t + mine, end);
        if (reset) rs = resets<L>(reset, A.r_ts, t + mine, end);
    };
    fetch(last);
    int buf = 0;
    for (long t = last; t >= t0; t -= tile, buf ^= 1) {
        const long ts = t + mine;
        float ga[L][V], gi[L][V], xv[L][V], gv[L][V], a[V], h[V], p[V], s[V];
        const unsigned r = rs;
#pragma unroll
        for (int k = 0; k < V; ++k) { a[k] = 1.f; h[k] = p[k] = 0.f; if constexpr (!TOTAL) s[k] = first[k]; }
#pragma unroll
        for (int j = 0; j < L; ++j) {
            const bool in = ts + j < end;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                gates((float)fr.v[j][k], ga[j][k], gi[j][k]);
                if (!in) { ga[j][k] = 1.f; gi[j][k] = 0.f; }
                gv[j][k] = in ? (float)gr.v[j][k] : 0.f;
                if constexpr (!TOTAL) {
                    xv[j][k] = in ? (float)xr.v[j][k] : 0.f;
                    h[k] = fmaf(ga[j][k], r >> j & 1 ? 0.f : h[k], gi[j][k] * xv[j][k]);
                }
                a[k] = r >> j & 1 ? 0.f : a[k] * ga[j][k];
            }
        }
#pragma unroll
        for (int j = L - 1; j >= 0; --j)
#pragma unroll
            for (int k = 0; k < V; ++k) p[k] = r >> j & 1 ? 0.f : ga[j][k] * (gv[j][k] + p[k]);
        if (t > t0) fetch(t - tile);
        const unsigned long ball = __ballot(r != 0);
        float xa[V], xh[V], ya[V], yp[V], aa[V];
        bool xcut = false, ycut;
#pragma unroll
        for (int k = 0; k < V; ++k) aa[k] = a[k];
        if constexpr (!TOTAL) across<V, true>(aa, h, ball, xa, xh, xcut);
        across<V, false>(a, p, ball, ya, yp, ycut);
        if constexpr (!TOTAL) {
            if (lane / G == S - 1) keep_state<V>(&tot[buf][2][wave][g * V], h);
        }
        if (lane / G == 0) {
            keep_state<V>(&tot[buf][0][wave][g * V], a);
            keep_state<V>(&tot[buf][1][wave][g * V], p);
            if (g == 0) cuts[buf][wave] = ball != 0;
        }
        lds_barrier();
        float in[V];
        for (int w = W - 1; w >= 0; --w) {
            if (w == wave) {
#pragma unroll
                for (int k = 0; k < V; ++k) in[k] = mu[k];
            }
            const bool cut = cuts[buf][w];
            if constexpr (TOTAL) {
                const auto m = load<V>(&tot[buf][0][w][g * V]);
#pragma unroll
                for (int k = 0; k < V; ++k) all[k] *= m[k];
                allcut |= cut;
            }
            through<V>(mu, &tot[buf][0][w][g * V], &tot[buf][1][w][g * V], cut);
        }
        if constexpr (!TOTAL) {
            for (int w = 0; w < wave; ++w) through<V>(s, &tot[buf][0][w][g * V], &tot[buf][2][w][g * V], cuts[buf][w]);
            float before[L][V];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                s[k] = xcut ? xh[k] : fmaf(xa[k], s[k], xh[k]);
                in[k] = ycut ? yp[k] : fmaf(ya[k], in[k], yp[k]);
            }
#pragma unroll
            for (int j = 0; j < L; ++j)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    before[j][k] = r >> j & 1 ? 0.f : s[k];
                    s[k] = fmaf(ga[j][k], before[j][k], gi[j][k] * xv[j][k]);
                }
#pragma unroll
            for (int j = L - 1; j >= 0; --j) {
                float df[V], dx[V];
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float l = gv[j][k] + in[k];
                    dx[k] = gi[j][k] * l;
                    df[k] = ga[j][k] * dx[k] * (before[j][k] - xv[j][k]);
                    in[k] = r >> j & 1 ? 0.f : ga[j][k] * l;
                }
                if (me.live && ts + j < end) {
                    store<V>((E *)A.df + b * A.df_bs + (ts + j) * A.df_ts + me.c, narrow<E, V>(df));
                    store<V>((E *)A.dx + b * A.dx_bs + (ts + j) * A.dx_ts + me.c, narrow<E, V>(dx));
                }
            }
        }
    }
    if (wave || lane >= G || !me.live) return;
    if constexpr (TOTAL) {
#pragma unroll
        for (int k = 0; k < V; ++k) all[k] = allcut ? -1.f : all[k];
        keep_state<V>(totals + 2l * z * A.C, all);
        keep_state<V>(totals + (2l * z + 1) * A.C, mu);
    } else if (A.dh0 && z == 0) {
        keep_state<V>(A.dh0 + at, mu);
    }
}

}  // namespace seq
