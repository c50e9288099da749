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

constexpr int SCAN_RUN = 16;        // elements of a thread in a tile: 8 steps of 2 channels or 16 steps of one
constexpr int SCAN_STRIP = 64;      // channels of a workgroup
constexpr int SCAN_WAVES = 8;       // most waves of a workgroup
constexpr int SCAN_SHORT = 8;       // longest sequence that a thread goes through alone

// sigmoid(f) = 1 / (1 + e) and 1 - sigmoid(f) = e / (1 + e) with e = exp(-f).  The second is not taken from the first: 1 - a
// of an `a` near one, a memory that lasts, would keep few of its digits.  Where e is infinite, infinity times zero is
// the one that it should be (fminf drops the NaN); a gate that is NaN has a = NaN.
__device__ __forceinline__ void gates(float f, float &a, float &i)
{
    const float e = __builtin_amdgcn_exp2f(-1.44269504088896341f * f);
    a = __builtin_amdgcn_rcpf(1.f + e);
    i = fminf(e * a, 1.f);
}

// What a thread works on: V channels from c on of sequence b, clamped to the tensor where c is beyond it (then `live` is
// false and nothing is stored).
template <int V> struct Lane {
    int c;
    bool live;
    __device__ Lane(int first, int C) : c(min(first, C - V)), live(first < C) {}
};

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
// and L = 16 / V steps: with V = 2 half a wave is a row of the strip and a wave holds two runs of eight steps, with
// V = 1 (a size, a stride or an address that is not a multiple of two elements) a wave is one run of sixteen.
//
// Vector instructions cost as much as memory does here (about thirty per element, two of them exp and the reciprocal), so
// the choices that few tiles need are kept out of the others' way: a tile that ends beyond the range or that holds
// the start of an episode takes the careful form of the loops (EDGE), the rest the one without tests.
template <int V> struct Strip {
    static constexpr int L = SCAN_RUN / V, G = SCAN_STRIP / V, S = 64 / G;
};
using Plain = std::false_type;
using Edge = std::true_type;

// The reset flags of a wave's 16 steps from t on, a step per lane; flags() makes bits of them, bit j for step j.
struct Resets {
    uint8_t v = 0;
    __device__ __forceinline__ void fetch(const uint8_t *reset, long r_ts, long t, long end)
    {
        const int lane = threadIdx.x & 63;
        v = lane < SCAN_RUN && t + lane < end ? reset[(t + lane) * r_ts] : 0;
    }
    __device__ __forceinline__ unsigned flags() const { return (unsigned)__ballot(v != 0); }
};

// s through a map (a, h) that starts an episode (cut) or not
__device__ __forceinline__ float through(float s, float a, float h, bool cut) { return cut ? h : fmaf(a, s, h); }
template <int V> __device__ __forceinline__ void through(float (&s)[V], const float *A, const float *H, bool cut)
{
    const auto a = load<V>(A), h = load<V>(H);
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = through(s[k], a[k], h[k], cut);
}
// the same past a range of another workgroup
template <int V> __device__ __forceinline__ void past_range(float (&s)[V], const float *p, int C)
{
    const auto a = load<V>(p), h = load<V>(p + C);
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = through(s[k], a[k], h[k], a[k] < 0.f);
}

// The runs of one wave: each lane's map in, the map of the whole wave out (in all lanes).  FORWARD: the lower half is
// first, else the upper.  (fa, fh, fcut): the map of the half that is first, which what enters the wave goes through
// on its way to the other half.  `cuts`: bit 0 the lower half, bit 1 the upper.
template <int V, bool FORWARD> struct Across {
    float fa[V], fh[V];
    bool fcut;
    __device__ __forceinline__ void join(float (&A)[V], float (&H)[V], unsigned cuts)
    {
        if constexpr (Strip<V>::S == 2) {
            const bool scut = cuts & (FORWARD ? 2 : 1);
            fcut = cuts & (FORWARD ? 1 : 2);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                float la, ha, lh, hh;
                halves(A[k], la, ha);
                halves(H[k], lh, hh);
                fa[k] = FORWARD ? la : ha;
                fh[k] = FORWARD ? lh : hh;
                A[k] = la * ha;
                H[k] = through(fh[k], FORWARD ? ha : la, FORWARD ? hh : lh, scut);
            }
        }
    }
    // what enters the wave -> what enters this lane's run
    __device__ __forceinline__ void enter(float (&s)[V]) const
    {
        if constexpr (Strip<V>::S == 2) {
            const bool second = ((threadIdx.x & 32) != 0) == FORWARD;
#pragma unroll
            for (int k = 0; k < V; ++k) s[k] = second ? through(s[k], fa[k], fh[k], fcut) : s[k];
        }
    }
};

// A wave's window onto the 16 rows of a tensor from `row` on: a buffer that ends with the last step of the range, so that
// loads beyond it give zeros and stores are dropped.  A thread's place in the window is that of its first row, in bytes;
// one that lies outside the tensor has the place NOWHERE.  FULL: all 16 rows are there, and the way from row to row
// is the instruction's scalar offset, which costs no vector instruction; else it is part of the place, since the
// buffer's end is compared with the place alone.
constexpr int NOWHERE = 0x7FFFFFF0;
template <class E> struct Window {
    __amdgpu_buffer_rsrc_t rsrc;
    int step;   // bytes from row to row
    __device__ __forceinline__ Window(const E *p, long ts, long row, long end, int C)
    {
        const long bytes = ((end - row - 1) * ts + C) * (long)sizeof(E);
        rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<E *>(p + row * ts), 0, row < end ? (int)min(bytes, (long)NOWHERE) : 0, 0x00020000);
        step = (int)ts * (int)sizeof(E);
    }
    template <int V, bool FULL> __device__ __forceinline__ vec<E, V> get(int place, int j) const
    {
        constexpr int bytes = V * sizeof(E);
        const int ahead = FULL ? j * step : 0;
        if (!FULL) place += j * step;
        vec<E, V> v;
        if constexpr (bytes == 2) { const auto x = __builtin_amdgcn_raw_buffer_load_b16(rsrc, place, ahead, 0); __builtin_memcpy(&v, &x, bytes); }
        else if constexpr (bytes == 4) { const auto x = __builtin_amdgcn_raw_buffer_load_b32(rsrc, place, ahead, 0); __builtin_memcpy(&v, &x, bytes); }
        else { const auto x = __builtin_amdgcn_raw_buffer_load_b64(rsrc, place, ahead, 0); __builtin_memcpy(&v, &x, bytes); }
        return v;
    }
    template <int V, bool FULL> __device__ __forceinline__ void put(int place, int j, const float (&f)[V]) const
    {
        constexpr int bytes = V * sizeof(E);
        const int ahead = FULL ? j * step : 0;
        if (!FULL) place += j * step;
        const vec<E, V> v = narrow<E, V>(f);
        if constexpr (bytes == 2) { unsigned short x; __builtin_memcpy(&x, &v, bytes); __builtin_amdgcn_raw_buffer_store_b16(x, rsrc, place, ahead, 0); }
        else if constexpr (bytes == 4) { unsigned x; __builtin_memcpy(&x, &v, bytes); __builtin_amdgcn_raw_buffer_store_b32(x, rsrc, place, ahead, 0); }
        else { vec<unsigned, 2> x; __builtin_memcpy(&x, &v, bytes); __builtin_amdgcn_raw_buffer_store_b64(x, rsrc, place, ahead, 0); }
    }
};
template <class E, int V> struct Rows {   // what a thread reads of a tensor in a tile
    vec<E, V> v[Strip<V>::L];
    __device__ __forceinline__ void load_rows(const Window<E> &w, int place, bool full)
    {
        if (full) {
#pragma unroll
            for (int j = 0; j < Strip<V>::L; ++j) v[j] = w.template get<V, true>(place, j);
        } else {
#pragma unroll
            for (int j = 0; j < Strip<V>::L; ++j) v[j] = w.template get<V, false>(place, j);
        }
    }
};

// bits 0 and 1: whether an episode starts in the run of the wave's lower / upper half (V = 1: one run, bit 0)
template <int V> __device__ __forceinline__ unsigned cuts_of(unsigned flags)
{
    constexpr unsigned run = (1u << Strip<V>::L) - 1;
    return ((flags & run) != 0) | (flags >> Strip<V>::L != 0) << 1;
}

// TOTAL: nothing is written but the map of the range, for the launch that then takes the ranges from their states on.
template <class E, int V, bool TOTAL> __global__ __launch_bounds__(64 * SCAN_WAVES) void k_scan(ScanArgs A)
{
    constexpr int L = Strip<V>::L, G = Strip<V>::G, S = Strip<V>::S;
    __shared__ __attribute__((aligned(16))) float tot[2][2][SCAN_WAVES][SCAN_STRIP];
    __shared__ unsigned cuts[2][SCAN_WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = blockDim.x >> 6, g = lane % G, tile = W * S * L;
    const Lane<V> me(blockIdx.x * SCAN_STRIP + g * V, A.C);
    const int z = blockIdx.z;
    const long b = blockIdx.y, t0 = z * A.range, end = min(A.T, t0 + A.range), at = b * A.C + me.c;
    float *totals = A.totals + b * A.ranges * 2 * A.C + me.c;   // (A, H) of range r at 2 r C and (2 r + 1) C
    const E *f = (const E *)A.f + b * A.f_bs, *x = (const E *)A.x + b * A.x_bs;
    E *hs = (E *)A.h + b * A.h_bs;
    const uint8_t *reset = A.reset ? A.reset + b * A.r_bs : nullptr;
    const int wrow = wave * SCAN_RUN, half = lane / G * L;   // first step of the wave in a tile, of this thread's run in the wave
    auto place = [&](long ts) { return me.live ? (me.c + half * (int)ts) * (int)sizeof(E) : NOWHERE; };
    const int fplace = place(A.f_ts), xplace = place(A.x_ts), hplace = place(A.h_ts);
    float *carry = A.carry ? A.carry + (b * A.tiles + t0 / tile) * A.C + me.c : nullptr;

    float s[V] = {}, all[V];   // state entering the tile; TOTAL: the map so far is s -> all s + s
    bool allcut = false;
#pragma unroll
    for (int k = 0; k < V; ++k) all[k] = 1.f;
    Rows<E, V> fr, xr;
    Resets rs;
    auto fetch = [&](long t) {
        fr.load_rows(Window<E>(f, A.f_ts, t + wrow, end, A.C), fplace, t + tile <= end);
        xr.load_rows(Window<E>(x, A.x_ts, t + wrow, end, A.C), xplace, t + tile <= end);
        if (reset) rs.fetch(reset, A.r_ts, t + wrow, end);
    };
    fetch(t0);
    if constexpr (!TOTAL) {
        if (A.ranges > 1) state<V>(totals + (long)(2 * A.ranges - 2) * A.C, s);
        else if (A.h0) state<V>(A.h0 + at, s);
#pragma unroll 8
        for (int r = 0; r < z; ++r) past_range<V>(s, totals + 2l * r * A.C, A.C);
    }
    int buf = 0;
    for (long t = t0; t < end; t += tile, buf ^= 1) {
        const unsigned flags = rs.flags(), r = flags >> half, mycuts = cuts_of<V>(flags);
        const bool edge = flags || t + tile > end;
        const int left = (int)min((long)L, end - t - wrow - half);   // steps of this thread that are in the range
        float ga[L][V], gx[L][V], a[V], h[V];
        auto maps = [&](auto e) {
#pragma unroll
            for (int k = 0; k < V; ++k) { a[k] = 1.f; h[k] = 0.f; }
#pragma unroll
            for (int j = 0; j < L; ++j) {
                const bool cut = e.value && (r >> j & 1), in = !e.value || j < left;
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    float i;
                    gates((float)fr.v[j][k], ga[j][k], i);
                    gx[j][k] = i * (float)xr.v[j][k];
                    if (!in) { ga[j][k] = 1.f; gx[j][k] = 0.f; }     // beyond the end: the map that changes nothing
                    h[k] = fmaf(ga[j][k], cut ? 0.f : h[k], gx[j][k]);
                    a[k] = cut ? 0.f : a[k] * ga[j][k];
                }
            }
        };
        edge ? maps(Edge{}) : maps(Plain{});
        if (t + tile < end) fetch(t + tile);   // the next tile's loads are in flight behind everything below
        Across<V, true> up;
        up.join(a, h, mycuts);
        if (lane < G) {
            keep_state<V>(&tot[buf][0][wave][g * V], a);
            keep_state<V>(&tot[buf][1][wave][g * V], h);
            if (lane == 0) cuts[buf][wave] = mycuts;
        }
        lds_barrier();
        float in[V];
        // the waves that start an episode, one bit each
        const unsigned starts = (unsigned)__ballot(lane < W && cuts[buf][lane % SCAN_WAVES] != 0);
        for (int w = 0; w < W; ++w) {
            if (w == wave) {
#pragma unroll
                for (int k = 0; k < V; ++k) in[k] = s[k];
            }
            if constexpr (TOTAL) {
                const auto m = load<V>(&tot[buf][0][w][g * V]);
#pragma unroll
                for (int k = 0; k < V; ++k) all[k] *= m[k];
            }
            if (starts >> w & 1) through<V>(s, &tot[buf][0][w][g * V], &tot[buf][1][w][g * V], true);
            else through<V>(s, &tot[buf][0][w][g * V], &tot[buf][1][w][g * V], false);
        }
        allcut |= starts != 0;
        if constexpr (!TOTAL) {
            if (carry) {
                if (wave == 0 && lane < G && me.live) keep_state<V>(carry, in);
                carry += A.C;
            }
            up.enter(in);
            const Window<E> hw(hs, A.h_ts, t + wrow, end, A.C);
            auto steps = [&](auto e) {
#pragma unroll
                for (int j = 0; j < L; ++j) {
                    const bool cut = e.value && r >> j & 1;
#pragma unroll
                    for (int k = 0; k < V; ++k) in[k] = fmaf(ga[j][k], cut ? 0.f : in[k], gx[j][k]);
                    hw.template put<V, !e.value>(hplace, j, in);
                }
            };
            edge ? steps(Edge{}) : steps(Plain{});
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
    __shared__ __attribute__((aligned(16))) float tot[2][3][SCAN_WAVES][SCAN_STRIP];   // A, P and H of the waves
    __shared__ unsigned cuts[2][SCAN_WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = blockDim.x >> 6, g = lane % G, tile = W * S * L;
    const Lane<V> me(blockIdx.x * SCAN_STRIP + g * V, A.C);
    const int z = blockIdx.z + (TOTAL ? 1 : 0);
    const long b = blockIdx.y, t0 = z * A.range, end = min(A.T, t0 + A.range), at = b * A.C + me.c;
    float *totals = A.totals + b * A.ranges * 2 * A.C + me.c;
    const E *f = (const E *)A.f + b * A.f_bs, *x = (const E *)A.x + b * A.x_bs, *dh = (const E *)A.dh + b * A.dh_bs;
    E *dfs = (E *)A.df + b * A.df_bs, *dxs = (E *)A.dx + b * A.dx_bs;
    const uint8_t *reset = A.reset ? A.reset + b * A.r_bs : nullptr;
    const int wrow = wave * SCAN_RUN, half = lane / G * L;
    const long last = t0 + (end - t0 - 1) / tile * tile;
    auto place = [&](long ts) { return me.live ? (me.c + half * (int)ts) * (int)sizeof(E) : NOWHERE; };
    const int fplace = place(A.f_ts), xplace = place(A.x_ts), gplace = place(A.dh_ts), dfplace = place(A.df_ts), dxplace = place(A.dx_ts);
    const float *carry = A.carry + (b * A.tiles + last / tile) * A.C + me.c;

    float mu[V] = {}, all[V];   // what comes from the right into the tile; TOTAL: the map so far is m -> all m + mu
    bool allcut = false;
#pragma unroll
    for (int k = 0; k < V; ++k) all[k] = 1.f;
    Rows<E, V> fr, xr, gr;
    Resets rs;
    float first[V];   // state before the tile
    auto fetch = [&](long t) {
        fr.load_rows(Window<E>(f, A.f_ts, t + wrow, end, A.C), fplace, t + tile <= end);
        if constexpr (!TOTAL) xr.load_rows(Window<E>(x, A.x_ts, t + wrow, end, A.C), xplace, t + tile <= end);
        gr.load_rows(Window<E>(dh, A.dh_ts, t + wrow, end, A.C), gplace, t + tile <= end);
        if constexpr (!TOTAL) {
            state<V>(carry, first);
            carry -= A.C;
        }
        if (reset) rs.fetch(reset, A.r_ts, t + wrow, end);
    };
    fetch(last);
    if constexpr (!TOTAL) {
        if (A.dlast) state<V>(A.dlast + at, mu);
#pragma unroll 8
        for (int r = A.ranges - 1; r > z; --r) past_range<V>(mu, totals + 2l * r * A.C, A.C);
    }
    int buf = 0;
    for (long t = last; t >= t0; t -= tile, buf ^= 1) {
        const unsigned flags = rs.flags(), r = flags >> half, mycuts = cuts_of<V>(flags);
        const bool edge = flags || t + tile > end;
        const int left = (int)min((long)L, end - t - wrow - half);
        float ga[L][V], gi[L][V], gv[L][V], a[V], h[V], p[V], s[V];
        vec<E, V> xv[L];
        auto maps = [&](auto e) {
#pragma unroll
            for (int k = 0; k < V; ++k) { a[k] = 1.f; h[k] = p[k] = 0.f; }
#pragma unroll
            for (int j = 0; j < L; ++j) {
                const bool cut = e.value && (r >> j & 1), in = !e.value || j < left;
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    gates((float)fr.v[j][k], ga[j][k], gi[j][k]);
                    gv[j][k] = (float)gr.v[j][k];
                    if (!in) { ga[j][k] = 1.f; gi[j][k] = gv[j][k] = 0.f; }
                    if constexpr (!TOTAL) {
                        xv[j][k] = in ? xr.v[j][k] : (E)0.f;
                        h[k] = fmaf(ga[j][k], cut ? 0.f : h[k], gi[j][k] * (float)xv[j][k]);
                    }
                    a[k] = cut ? 0.f : a[k] * ga[j][k];
                }
            }
#pragma unroll
            for (int j = L - 1; j >= 0; --j)
#pragma unroll
                for (int k = 0; k < V; ++k) p[k] = e.value && r >> j & 1 ? 0.f : ga[j][k] * (gv[j][k] + p[k]);
        };
        edge ? maps(Edge{}) : maps(Plain{});
        if constexpr (!TOTAL) {
#pragma unroll
            for (int k = 0; k < V; ++k) s[k] = first[k];
        }
        if (t > t0) fetch(t - tile);
        Across<V, true> up;
        Across<V, false> down;
        float aa[V];
#pragma unroll
        for (int k = 0; k < V; ++k) aa[k] = a[k];
        if constexpr (!TOTAL) up.join(aa, h, mycuts);
        down.join(a, p, mycuts);
        if (lane < G) {
            keep_state<V>(&tot[buf][0][wave][g * V], a);
            keep_state<V>(&tot[buf][1][wave][g * V], p);
            if constexpr (!TOTAL) keep_state<V>(&tot[buf][2][wave][g * V], h);
            if (lane == 0) cuts[buf][wave] = mycuts;
        }
        lds_barrier();
        float in[V];
        const unsigned starts = (unsigned)__ballot(lane < W && cuts[buf][lane % SCAN_WAVES] != 0);
        for (int w = W - 1; w >= 0; --w) {
            if (w == wave) {
#pragma unroll
                for (int k = 0; k < V; ++k) in[k] = mu[k];
            }
            if constexpr (TOTAL) {
                const auto m = load<V>(&tot[buf][0][w][g * V]);
#pragma unroll
                for (int k = 0; k < V; ++k) all[k] *= m[k];
            }
            if (starts >> w & 1) through<V>(mu, &tot[buf][0][w][g * V], &tot[buf][1][w][g * V], true);
            else through<V>(mu, &tot[buf][0][w][g * V], &tot[buf][1][w][g * V], false);
        }
        allcut |= starts != 0;
        if constexpr (!TOTAL) {
            for (int w = 0; w < wave; ++w) {
                if (starts >> w & 1) through<V>(s, &tot[buf][0][w][g * V], &tot[buf][2][w][g * V], true);
                else through<V>(s, &tot[buf][0][w][g * V], &tot[buf][2][w][g * V], false);
            }
            up.enter(s);
            down.enter(in);
            const Window<E> dfw(dfs, A.df_ts, t + wrow, end, A.C), dxw(dxs, A.dx_ts, t + wrow, end, A.C);
            auto steps = [&](auto e) {
                float before[L][V];
#pragma unroll
                for (int j = 0; j < L; ++j)
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        before[j][k] = e.value && r >> j & 1 ? 0.f : s[k];
                        s[k] = fmaf(ga[j][k], before[j][k], gi[j][k] * (float)xv[j][k]);
                    }
#pragma unroll
                for (int j = L - 1; j >= 0; --j) {
                    float df[V], dx[V];
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        const float l = gv[j][k] + in[k], m = ga[j][k] * l;
                        dx[k] = gi[j][k] * l;
                        df[k] = gi[j][k] * m * (before[j][k] - (float)xv[j][k]);
                        in[k] = e.value && r >> j & 1 ? 0.f : m;
                    }
                    dfw.template put<V, !e.value>(dfplace, j, df);
                    dxw.template put<V, !e.value>(dxplace, j, dx);
                }
            };
            edge ? steps(Edge{}) : steps(Plain{});
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
