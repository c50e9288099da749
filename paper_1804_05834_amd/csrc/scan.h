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
    long tiles;      // states per sequence in `carry`
    long range;      // lines: steps of a range, ranges, and their maps (see there)
    int ranges;
    float *totals;
    bool apart;      // lines: no wave may hold parts of two ranges
    bool torn;       // rows are not aligned to the caches' lines
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
    long tiles;
    long range;
    int ranges;
    float *totals;
    bool apart;      // lines: no wave may hold parts of two ranges
    bool torn;       // rows are not aligned to the caches' lines
};

constexpr int SCAN_RUN = 16;        // elements of a thread in a tile: 8 steps of 2 channels or 16 steps of one
constexpr int SCAN_STRIP = 64;      // channels of a workgroup
constexpr int SCAN_WAVES = 8;       // most waves of a workgroup
constexpr int SCAN_SHORT = 8;       // longest sequence that a thread goes through alone

// sigmoid(f) = 1 / (1 + e) and 1 - sigmoid(f) = e / (1 + e) with e = exp(-f).  The second is not taken from the first: 1 - a
// of an `a` near one, a memory that lasts, would keep few of its digits.  Nor is it the product e a where e is large: the
// instruction gives zero for a reciprocal below 2^-126, from f = -87.4 on, and infinity times zero is NaN.  From e = 2^24
// on it is one to the last digit.  A gate that is NaN makes both NaN: no comparison with it holds.
__device__ __forceinline__ void gates(float f, float &a, float &i)
{
    const float e = __builtin_amdgcn_exp2f(-1.44269504088896341f * f);
    a = __builtin_amdgcn_rcpf(1.f + e);
    i = e > 0x1p24f ? 1.f : e * a;
}

// What a thread works on: V channels from c on of sequence b, clamped to the tensor where c is beyond it (then `live` is
// false and nothing is stored).
template <int V> struct Lane {
    int c;
    bool live;
    __device__ Lane(int first, int C) : c(min(first, C - V)), live(first < C) {}
};

// Which of `all` items (a sequence or a group of ranges) and which strip of its channels a workgroup has.  Workgroups with the same
// id modulo 8 share a cache.  Where rows are torn, that is where strips have lines of memory in common, those of an item
// share a cache (7 x 4099 x 261 in fp32 with gradients: 101 -> 93 us); else they are dealt out in turn (131072 x 512 in bf16:
// 127 -> 123 us).
struct Dealt {
    unsigned item;
    int strip;
    __device__ __forceinline__ Dealt(unsigned strips, unsigned all, bool torn)
    {
        const unsigned even = torn ? all / 8 * 8 : 0;   // the others do not make eight
        if (blockIdx.x < even * strips) {
            const unsigned k = blockIdx.x / 8;
            item = k / strips * 8 + blockIdx.x % 8;
            strip = k % strips;
        } else {
            const unsigned k = blockIdx.x - even * strips;
            item = even + k / strips;
            strip = k % strips;
        }
    }
};

// a state of V channels, at any address of a float
template <int V> __device__ __forceinline__ void state(const float *p, float (&s)[V]) { __builtin_memcpy(s, p, sizeof(s)); }
template <int V> __device__ __forceinline__ void keep_state(float *p, const float (&s)[V]) { __builtin_memcpy(p, s, sizeof(s)); }

// ------------------------------------------------------------ short sequences
// A thread takes V channels of a sequence through all of its at most SCAN_SHORT steps; all of its loads go out before
// the first is used.  The step of an acting agent is T = 1 (32 environments of 512 channels: 3.1 us, a launch and two trips
// to memory).
template <class E, int V> __global__ __launch_bounds__(256) void k_scan_short(ScanArgs A)
{
    const long id = (long)blockIdx.x * 256 + threadIdx.x, all = (long)A.B * (A.C / V);
    if (id >= all) return;
    const long b = (unsigned)id / (unsigned)(A.C / V);   // there are at most 2^28
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
    const long b = (unsigned)id / (unsigned)(A.C / V);   // there are at most 2^28
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
// Vector instructions cost nearly as much as memory does here (about twenty-one per element, two of them exp and the
// reciprocal), so the choices that few tiles need are kept out of the others' way: a tile that ends beyond the sequence or
// that holds the start of an episode takes the careful form of the loops (Edge), the rest the one without tests.
// Measured, 32 sequences of 512 steps of 512 channels in bf16: forward 14.8 us (3.4 TB/s), backward 21.8 (3.8).
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

// Results are stored as a stream: they are read next by another kernel, on any of the eight XCDs, and pass through memory (or
// its cache) anyway (32 sequences of 512 steps with gradients: 37.6 -> 34.6 us).
//
// A wave's window onto the 16 rows of a tensor from `row` on: a buffer that ends with the last step of the range, so that
// loads beyond it give zeros and stores are dropped.  A thread's place in the window is that of its first row, in bytes;
// one that lies outside the tensor has the place NOWHERE.  FULL: all 16 rows are there, and the way from row to row
// is the instruction's scalar offset, which costs no vector instruction; else it is part of the place, since the
// buffer's end is compared with the place alone.
constexpr int NOWHERE = 0x7FFFFFF0;
constexpr int STREAM = 2;   // the instructions' hint that nothing near by reads this again
template <class E> struct Window {
    __amdgpu_buffer_rsrc_t rsrc;
    int step;   // bytes from row to row
    __device__ __forceinline__ Window(const E *p, long ts, long row, long end, int C)
    {
        const long bytes = ((end - row - 1) * ts + C) * (long)sizeof(E);
        rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<E *>(p + row * ts), 0, row < end ? (int)min(bytes, (long)NOWHERE) : 0, 0x00020000);
        step = (int)ts * (int)sizeof(E);
    }
    template <int V, bool FULL, int LOAD = 0> __device__ __forceinline__ vec<E, V> get(int place, int j) const
    {
        constexpr int bytes = V * sizeof(E);
        const int ahead = FULL ? j * step : 0;
        if (!FULL) place += j * step;
        vec<E, V> v;
        if constexpr (bytes == 2) { const auto x = __builtin_amdgcn_raw_buffer_load_b16(rsrc, place, ahead, LOAD); __builtin_memcpy(&v, &x, bytes); }
        else if constexpr (bytes == 4) { const auto x = __builtin_amdgcn_raw_buffer_load_b32(rsrc, place, ahead, LOAD); __builtin_memcpy(&v, &x, bytes); }
        else { const auto x = __builtin_amdgcn_raw_buffer_load_b64(rsrc, place, ahead, LOAD); __builtin_memcpy(&v, &x, bytes); }
        return v;
    }
    template <int V, bool FULL> __device__ __forceinline__ void put(int place, int j, const float (&f)[V]) const
    {
        constexpr int bytes = V * sizeof(E);
        const int ahead = FULL ? j * step : 0;
        if (!FULL) place += j * step;
        const vec<E, V> v = narrow<E, V>(f);
        if constexpr (bytes == 2) { unsigned short x; __builtin_memcpy(&x, &v, bytes); __builtin_amdgcn_raw_buffer_store_b16(x, rsrc, place, ahead, STREAM); }
        else if constexpr (bytes == 4) { unsigned x; __builtin_memcpy(&x, &v, bytes); __builtin_amdgcn_raw_buffer_store_b32(x, rsrc, place, ahead, STREAM); }
        else { vec<unsigned, 2> x; __builtin_memcpy(&x, &v, bytes); __builtin_amdgcn_raw_buffer_store_b64(x, rsrc, place, ahead, STREAM); }
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

template <class E, int V> __global__ __launch_bounds__(64 * SCAN_WAVES) void k_scan(ScanArgs A)
{
    constexpr int L = Strip<V>::L, G = Strip<V>::G, S = Strip<V>::S;
    __shared__ __attribute__((aligned(16))) float tot[2][2][SCAN_WAVES][SCAN_STRIP];
    __shared__ unsigned cuts[2][SCAN_WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = blockDim.x >> 6, g = lane % G, tile = W * S * L;
    const Dealt to((A.C + SCAN_STRIP - 1) / SCAN_STRIP, A.B, A.torn);
    const Lane<V> me(to.strip * SCAN_STRIP + g * V, A.C);
    const long b = to.item, end = A.T, at = b * A.C + me.c;
    const E *f = (const E *)A.f + b * A.f_bs, *x = (const E *)A.x + b * A.x_bs;
    E *hs = (E *)A.h + b * A.h_bs;
    const uint8_t *reset = A.reset ? A.reset + b * A.r_bs : nullptr;
    const int wrow = wave * SCAN_RUN, half = lane / G * L;   // first step of the wave in a tile, of this thread's run in the wave
    auto place = [&](long ts) { return me.live ? (me.c + half * (int)ts) * (int)sizeof(E) : NOWHERE; };
    const int fplace = place(A.f_ts), xplace = place(A.x_ts), hplace = place(A.h_ts);
    float *carry = A.carry ? A.carry + b * A.tiles * A.C + me.c : nullptr;

    float s[V] = {};   // state entering the tile
    Rows<E, V> fr, xr;
    Resets rs;
    auto fetch = [&](long t) {
        fr.load_rows(Window<E>(f, A.f_ts, t + wrow, end, A.C), fplace, t + tile <= end);
        xr.load_rows(Window<E>(x, A.x_ts, t + wrow, end, A.C), xplace, t + tile <= end);
        if (reset) rs.fetch(reset, A.r_ts, t + wrow, end);
    };
    fetch(0);
    if (A.h0) {   // all waves read it, and the first may write h_last there behind the first barrier
        state<V>(A.h0 + at, s);
        arrived(s);
    }
    int buf = 0;
    for (long t = 0; t < end; t += tile, buf ^= 1) {
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
            if (starts >> w & 1) through<V>(s, &tot[buf][0][w][g * V], &tot[buf][1][w][g * V], true);
            else through<V>(s, &tot[buf][0][w][g * V], &tot[buf][1][w][g * V], false);
        }
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
    if (A.h_last && wave == 0 && lane < G && me.live) keep_state<V>(A.h_last + at, s);
}

template <class E, int V> __global__ __launch_bounds__(64 * SCAN_WAVES) void k_scan_grad(ScanGradArgs A)
{
    constexpr int L = Strip<V>::L, G = Strip<V>::G, S = Strip<V>::S;
    __shared__ __attribute__((aligned(16))) float tot[2][3][SCAN_WAVES][SCAN_STRIP];   // A, P and H of the waves
    __shared__ unsigned cuts[2][SCAN_WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = blockDim.x >> 6, g = lane % G, tile = W * S * L;
    const Dealt to((A.C + SCAN_STRIP - 1) / SCAN_STRIP, A.B, A.torn);
    const Lane<V> me(to.strip * SCAN_STRIP + g * V, A.C);
    const long b = to.item, end = A.T, at = b * A.C + me.c;
    const E *f = (const E *)A.f + b * A.f_bs, *x = (const E *)A.x + b * A.x_bs, *dh = (const E *)A.dh + b * A.dh_bs;
    E *dfs = (E *)A.df + b * A.df_bs, *dxs = (E *)A.dx + b * A.dx_bs;
    const uint8_t *reset = A.reset ? A.reset + b * A.r_bs : nullptr;
    const int wrow = wave * SCAN_RUN, half = lane / G * L;
    const long last = (A.tiles - 1) * tile;
    auto place = [&](long ts) { return me.live ? (me.c + half * (int)ts) * (int)sizeof(E) : NOWHERE; };
    const int fplace = place(A.f_ts), xplace = place(A.x_ts), gplace = place(A.dh_ts), dfplace = place(A.df_ts), dxplace = place(A.dx_ts);
    const float *carry = A.carry + ((b + 1) * A.tiles - 1) * A.C + me.c;

    float mu[V] = {};   // what comes from the right into the tile
    Rows<E, V> fr, xr, gr;
    Resets rs;
    float first[V];   // state before the tile
    auto fetch = [&](long t) {
        fr.load_rows(Window<E>(f, A.f_ts, t + wrow, end, A.C), fplace, t + tile <= end);
        xr.load_rows(Window<E>(x, A.x_ts, t + wrow, end, A.C), xplace, t + tile <= end);
        gr.load_rows(Window<E>(dh, A.dh_ts, t + wrow, end, A.C), gplace, t + tile <= end);
        state<V>(carry, first);
        carry -= A.C;
        if (reset) rs.fetch(reset, A.r_ts, t + wrow, end);
    };
    fetch(last);
    if (A.dlast) state<V>(A.dlast + at, mu);
    int buf = 0;
    for (long t = last; t >= 0; t -= tile, buf ^= 1) {
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
                    xv[j][k] = in ? xr.v[j][k] : (E)0.f;
                    h[k] = fmaf(ga[j][k], cut ? 0.f : h[k], gi[j][k] * (float)xv[j][k]);
                    a[k] = cut ? 0.f : a[k] * ga[j][k];
                }
            }
#pragma unroll
            for (int j = L - 1; j >= 0; --j)
#pragma unroll
                for (int k = 0; k < V; ++k) p[k] = e.value && r >> j & 1 ? 0.f : ga[j][k] * (gv[j][k] + p[k]);
        };
        edge ? maps(Edge{}) : maps(Plain{});
#pragma unroll
        for (int k = 0; k < V; ++k) s[k] = first[k];
        if (t > 0) fetch(t - tile);
        Across<V, true> up;
        Across<V, false> down;
        float aa[V];
#pragma unroll
        for (int k = 0; k < V; ++k) aa[k] = a[k];
        up.join(aa, h, mycuts);
        down.join(a, p, mycuts);
        if (lane < G) {
            keep_state<V>(&tot[buf][0][wave][g * V], a);
            keep_state<V>(&tot[buf][1][wave][g * V], p);
            keep_state<V>(&tot[buf][2][wave][g * V], h);
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
            if (starts >> w & 1) through<V>(mu, &tot[buf][0][w][g * V], &tot[buf][1][w][g * V], true);
            else through<V>(mu, &tot[buf][0][w][g * V], &tot[buf][1][w][g * V], false);
        }
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
    if (A.dh0 && wave == 0 && lane < G && me.live) keep_state<V>(A.dh0 + at, mu);
}

// ------------------------------------------------------------ lines
// A lane takes two channels through a range of steps, step after step, LINE steps' loads ahead: no work but the
// recurrence itself (fifteen vector instructions per element, where a strip takes twenty-one).  With enough sequences
// and channels a wave takes whole sequences.  Else time is cut into ranges, and the state that enters one is not known yet:
// a first launch finds the map of every range, a second composes the maps of those before and then runs.  f and x
// are read twice then, which long sequences of few channels have to: the other way would be to wait for the
// workgroup before, a thousand times in turn.
//
// LINE_GROUP ranges of a sequence in turn are a group: maps are kept of ranges and of groups, and a group's lanes compose the
// groups before it among them.  A group's strip of 64 pairs of channels is a workgroup and a range of it a wave.  In a strip that is
// half as wide, or less, the lanes of the group's ranges follow one another, so that a wave holds parts of several
// (100 sequences of 900 steps of 64 channels in bf16: 18 us forward, 22 backward; a wave a range: 26 and 40).
// Channels are taken in pairs at any alignment: what the first pair of a row begins with need not be aligned to two elements,
// and of an odd number of channels the last lane has the last two but stores the last alone (`half`).
//
// Measured: 512 sequences of 64 steps of 512 channels in bf16, a wave each, 18 us forward (5.6 TB/s), 36 backward (4.7); one
// sequence of 131072 steps of 512 channels, in ranges, 58 for the maps (4.6 TB/s) and 70 for the states (5.8).
constexpr int LINE = 8;         // steps between two states of `carry`, and of a wave's loads
constexpr int LINE_GROUP = 8;   // ranges of a workgroup; waves of one whose waves take whole sequences

// V values that lie at any address of a float
__device__ __forceinline__ void pair(const float *p, float (&s)[2]) { __builtin_memcpy(s, p, 8); }
__device__ __forceinline__ void keep_pair(float *p, const float (&s)[2], bool half)
{
    if (half) p[1] = s[1];
    else __builtin_memcpy(p, s, 8);
}

// Maps in memory: [B][ranges + groups][2][C], A (-1: an episode starts there) and H of each range, then of each group.  A map
// is made and composed in registers as (a, h).  The last range's map (forward; backward the first's) is not needed.
// Forward, range 0 runs from h0 on and counts as the start of an episode, and a copy of h0 stands in place of the last
// range's A: the last range may write h_last where h0 was before the first has read it.
struct Map {
    float a[2] = {1.f, 1.f}, h[2] = {};
    bool cut = false;
    __device__ __forceinline__ void put(float *p, int C, bool half) const
    {
        const float m[2] = {cut ? -1.f : a[0], cut ? -1.f : a[1]};
        keep_pair(p, m, half);
        keep_pair(p + C, h, half);
    }
    // this map, then (pa, ph) if `there`
    __device__ __forceinline__ void then(const float (&pa)[2], const float (&ph)[2], bool there)
    {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float nh = through(h[k], pa[k], ph[k], pa[k] < 0.f), na = pa[k] < 0.f || a[k] < 0.f ? -1.f : a[k] * pa[k];
            h[k] = there ? nh : h[k];
            a[k] = there ? na : a[k];
        }
    }
    // this map, then the one at p
    __device__ __forceinline__ void then(const float *p, int C)
    {
        float pa[2], ph[2];
        pair(p, pa);
        pair(p + C, ph);
        then(pa, ph, true);
    }
    __device__ __forceinline__ void apply(float (&s)[2]) const
    {
#pragma unroll
        for (int k = 0; k < 2; ++k) s[k] = through(s[k], a[k], h[k], a[k] < 0.f);
    }
};

// lanes of a strip of so many pairs of channels: a power of two, so that the parts of rows that a wave has are not cut anew
__host__ __device__ __forceinline__ int line_width(int pairs)
{
    int width = 64;
    while (width > 1 && width / 2 >= pairs) width /= 2;
    return width;
}

// Where a lane stands.
struct Line {
    int c, lane, q, z;          // its channels; in ranges: place in the strip, range in the group and in the sequence
    int z0, z1, group, groups;  // first and last range of the wave, the workgroup's group, all groups
    int width;                  // lanes of the strip
    long b, range;
    bool live, half, idle;      // idle: the wave has nothing to do, but the workgroup's barriers
    bool halves;                // a lane of the wave is half
    __device__ __forceinline__ Line(int B, int C, int ranges, long range, bool apart, bool torn) : range(range)
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        groups = (ranges + LINE_GROUP - 1) / LINE_GROUP;
        const int pairs = (C + 1) / 2, strips = (pairs + 63) / 64;
        int first;
        if (ranges == 1) {   // a wave per strip
            const long id = (long)blockIdx.x * LINE_GROUP + wave;
            b = id / strips;
            lane = threadIdx.x & 63;
            first = ((int)(id - b * strips) * 64 + lane) * 2;
            q = z = z0 = z1 = group = 0;
            width = 64;
            idle = b >= B;
            live = first < C && !idle;
        } else {             // a workgroup per strip and group
            const Dealt to(strips, (unsigned)B * groups, torn);
            const unsigned id = to.item;
            const int strip = to.strip;
            b = id / groups;
            group = id - (unsigned)b * groups;
            width = apart ? 64 : line_width(pairs - strip * 64);
            q = threadIdx.x / (unsigned)width;
            lane = threadIdx.x % (unsigned)width;
            first = (strip * 64 + lane) * 2;
            z = group * LINE_GROUP + q;
            z0 = __builtin_amdgcn_readfirstlane(z);
            const int last = min((group + 1) * LINE_GROUP, ranges) - 1;
            z1 = min(__builtin_amdgcn_readlane(z, 63), last);
            idle = z0 > last;
            live = z <= last && first < C;
        }
        c = min(first, C - 2);
        half = live && first > c;
        halves = __ballot(half) != 0;
    }
    // the lane's step when the wave's first one is at `t`
    __device__ __forceinline__ long step(long t) const { return t + (z - z0) * range; }
    // Its bytes from the wave's first row on.  The host sees to it that they fit.
    __device__ __forceinline__ int place(long ts, int size) const { return (int)(((z - z0) * range * ts + c) * size); }
    // whether LINE steps from the wave's step t on are there in all of its lanes
    __device__ __forceinline__ bool whole(long t, long T) const { return t + (z1 - z0) * range + LINE <= T; }
    // batches of LINE steps
    __device__ __forceinline__ long batches(int ranges, long T) const
    {
        return ((z0 < ranges - 1 ? range : T - z0 * range) + LINE - 1) / LINE;
    }
};

// Rows t .. t + LINE - 1 of a tensor
template <class E, int LOAD = 0> struct LineRows {
    vec<E, 2> v[LINE];
    __device__ __forceinline__ void fetch(const E *p, long ts, long t, long T, int C, int place, bool whole)
    {
        const Window<E> w(p, ts, t, T, C);
        if (whole) {
#pragma unroll
            for (int j = 0; j < LINE; ++j) v[j] = w.template get<2, true, LOAD>(place, j);
        } else {
#pragma unroll
            for (int j = 0; j < LINE; ++j) v[j] = w.template get<2, false, LOAD>(place, j);
        }
    }
};
// A row's results; `one`: the place of a lane's second channel where that is stored alone, if a lane of the wave has such.
template <bool FULL, class E> __device__ __forceinline__ void put_line(const Window<E> &w, int place, int one, bool halves, int j, const float (&v)[2])
{
    w.template put<2, FULL>(place, j, v);
    if (halves) w.template put<1, FULL>(one, j, {v[1]});
}

// The reset flags of a wave's next LINE steps, lane l having step l % 8 of range z0 + l / 8.
struct LineResets {
    uint8_t v = 0;
    __device__ __forceinline__ void fetch(const uint8_t *reset, long r_ts, long t, long T, const Line &me)
    {
        const int lane = threadIdx.x & 63, z = lane / LINE;
        const long row = t + z * me.range + lane % LINE;
        v = z <= me.z1 - me.z0 && row < T ? reset[row * r_ts] : 0;
    }
    __device__ __forceinline__ uint64_t flags() const { return __ballot(v != 0); }
};
__device__ __forceinline__ unsigned of_lane(uint64_t flags, const Line &me) { return (unsigned)(flags >> ((me.z - me.z0) * LINE & 63)) & ((1u << LINE) - 1); }

// The state that enters a lane's range: the lanes of every range of the group compose a share of the groups on the way to it,
// then the ranges before theirs in the workgroup.
template <bool FORWARD> __device__ __forceinline__ void enter_range(float (&s)[2], const Line &me, const float *maps, int ranges, int C)
{
    __shared__ float sh[2 * LINE_GROUP * 2 * 128];   // [2 LINE_GROUP][2][the strip's channels]
    const int row = me.width * 2, before = FORWARD ? me.group : me.groups - 1 - me.group;
    float *at = sh + me.lane * 2;
    const int order = me.q >= LINE_GROUP ? 0 : FORWARD ? me.q : LINE_GROUP - 1 - me.q;   // (lanes beyond the last range: any)
    if (me.q < LINE_GROUP) {
        const int share = (before + LINE_GROUP - 1) / LINE_GROUP;
        Map m;
        for (int k = 0; k < share; k += 8) {   // eight maps' loads go out at once: one after the other they were 6 us of 14 at 256 groups
            float a[8][2], h[8][2];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int q = min(order * share + k + j, me.groups - 1);
                const float *p = maps + (long)(ranges + (FORWARD ? q : me.groups - 1 - q)) * 2 * C;
                pair(p, a[j]);
                pair(p + C, h[j]);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool mine = k + j < share && order * share + k + j < before;
                m.then(a[j], h[j], mine);
            }
        }
        Map own;
        if (me.live && me.z != (FORWARD ? ranges - 1 : 0)) own.then(maps + (long)me.z * 2 * C, C);
        m.put(at + order * 2 * row, row, false);
        own.put(at + (LINE_GROUP + order) * 2 * row, row, false);
    }
    __syncthreads();
    if (me.idle) return;
    for (int q = 0; q < LINE_GROUP + order; ++q) {
        Map step;
        pair(at + q * 2 * row, step.a);
        pair(at + q * 2 * row + row, step.h);
        step.apply(s);
    }
}

// the maps of a workgroup's ranges: each to its place, and all composed to the group's
template <bool FORWARD> __device__ __forceinline__ void leave_maps(const Map &m, const Line &me, float *maps, int ranges, int C)
{
    __shared__ float sh[LINE_GROUP * 2 * 128];
    const int row = me.width * 2;
    float *at = sh + me.lane * 2;
    if (me.q < LINE_GROUP) m.put(at + (FORWARD ? me.q : LINE_GROUP - 1 - me.q) * 2 * row, row, false);
    if (me.live && me.z != (FORWARD ? ranges - 1 : 0)) m.put(maps + (long)me.z * 2 * C, C, me.half);
    __syncthreads();
    if (me.q || !me.live) return;
    Map all;
    for (int q = 0; q < LINE_GROUP; ++q) all.then(at + q * 2 * row, row);
    float *p = maps + (long)(ranges + me.group) * 2 * C;
    keep_pair(p, all.a, me.half);
    keep_pair(p + C, all.h, me.half);
}

template <class E> __global__ __launch_bounds__(64 * LINE_GROUP) void k_line_maps(ScanArgs A)
{
    const Line me(A.B, A.C, A.ranges, A.range, A.apart, A.torn);
    const E *f = (const E *)A.f + me.b * A.f_bs, *x = (const E *)A.x + me.b * A.x_bs;
    const uint8_t *reset = A.reset ? A.reset + me.b * A.r_bs : nullptr;
    const bool wanted = me.live && me.z < A.ranges - 1;   // a range that is not the last is whole: a multiple of LINE steps
    const int fp = wanted ? me.place(A.f_ts, sizeof(E)) : NOWHERE, xp = wanted ? me.place(A.x_ts, sizeof(E)) : NOWHERE;
    float *maps = A.totals + me.b * (A.ranges + me.groups) * 2 * A.C + me.c;
    Map m;
    if (!me.idle && me.z0 < A.ranges - 1) {
        const long t0 = me.z0 * A.range, end = t0 + A.range;
        LineRows<E> fr, xr;
        LineResets rs;
        auto fetch = [&](long t) {
            fr.fetch(f, A.f_ts, t, A.T, A.C, fp, true);
            xr.fetch(x, A.x_ts, t, A.T, A.C, xp, true);
            if (reset) rs.fetch(reset, A.r_ts, t, A.T, me);
        };
        fetch(t0);
        if (me.z == 0) {
            m.cut = true;
            if (A.h0) pair(A.h0 + me.b * A.C + me.c, m.h);
        }
        for (long t = t0; t < end; t += LINE) {
            const uint64_t flags = rs.flags();
            const LineRows<E> fv = fr, xv = xr;
            if (t + LINE < end) fetch(t + LINE);
            auto steps = [&](auto e) {
                const unsigned mine = e.value ? of_lane(flags, me) : 0;
#pragma unroll
                for (int j = 0; j < LINE; ++j) {
                    const bool cut = e.value && mine >> j & 1;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float a, i;
                        gates((float)fv.v[j][k], a, i);
                        m.h[k] = fmaf(a, cut ? 0.f : m.h[k], i * (float)xv.v[j][k]);
                        m.a[k] *= a;
                    }
                }
                if (e.value) m.cut |= mine != 0;
            };
            flags ? steps(Edge{}) : steps(Plain{});
        }
        if (!wanted) m = Map{};
    }
    leave_maps<true>(m, me, maps, A.ranges, A.C);
    if (me.z == A.ranges - 1 && me.live) {
        float s[2] = {};
        if (A.h0) pair(A.h0 + me.b * A.C + me.c, s);
        keep_pair(maps + (long)(A.ranges - 1) * 2 * A.C, s, me.half);
    }
}

// LOAD = STREAM: f and x together are more than the last-level cache holds, so that the second reading finds nothing of the
// first there any more, and does better not to look (131072 steps of 512 channels, 268 MB: 75 -> 63 us; below that it loses 10 %).
template <class E, int LOAD> __global__ __launch_bounds__(64 * LINE_GROUP) void k_lines(ScanArgs A)
{
    const Line me(A.B, A.C, A.ranges, A.range, A.apart, A.torn);
    if (A.ranges == 1 && me.idle) return;
    const E *f = (const E *)A.f + me.b * A.f_bs, *x = (const E *)A.x + me.b * A.x_bs;
    E *h = (E *)A.h + me.b * A.h_bs;
    const uint8_t *reset = A.reset ? A.reset + me.b * A.r_bs : nullptr;
    const int fp = me.live ? me.place(A.f_ts, sizeof(E)) : NOWHERE, xp = me.live ? me.place(A.x_ts, sizeof(E)) : NOWHERE;
    const int out = me.live ? me.place(A.h_ts, sizeof(E)) : NOWHERE, hp = me.half ? NOWHERE : out, one = me.half ? out + (int)sizeof(E) : NOWHERE;
    const long at = me.b * A.C + me.c, t0 = me.z0 * A.range, end = t0 + me.batches(A.ranges, A.T) * LINE, mine = min(A.T, (me.z + 1) * A.range);
    LineRows<E, LOAD> fr, xr;
    LineResets rs;
    auto fetch = [&](long t) {
        const bool whole = me.whole(t, A.T);
        fr.fetch(f, A.f_ts, t, A.T, A.C, fp, whole);
        xr.fetch(x, A.x_ts, t, A.T, A.C, xp, whole);
        if (reset) rs.fetch(reset, A.r_ts, t, A.T, me);
    };
    if (!me.idle) fetch(t0);
    float s[2] = {};
    if (A.ranges > 1) {
        const float *maps = A.totals + me.b * (A.ranges + me.groups) * 2 * A.C + me.c;
        pair(maps + (long)(A.ranges - 1) * 2 * A.C, s);
        enter_range<true>(s, me, maps, A.ranges, A.C);
        if (me.idle) return;
    } else if (A.h0) {
        pair(A.h0 + at, s);
    }
    float *carry = A.carry ? A.carry + (me.b * A.tiles + me.step(t0) / LINE) * A.C + me.c : nullptr;
    for (long t = t0; t < end; t += LINE) {
        const uint64_t flags = rs.flags();
        const bool whole = me.whole(t, A.T);
        const LineRows<E, LOAD> fv = fr, xv = xr;
        if (t + LINE < end) fetch(t + LINE);
        if (carry) {
            if (me.live && (whole || me.step(t) < mine)) keep_pair(carry, s, me.half);
            carry += A.C;
        }
        const Window<E> hw(h, A.h_ts, t, A.T, A.C);
        auto steps = [&](auto e) {
            const unsigned cuts = e.value ? of_lane(flags, me) : 0;
            const long left = e.value ? mine - me.step(t) : LINE;
#pragma unroll
            for (int j = 0; j < LINE; ++j) {
                const bool cut = e.value && cuts >> j & 1, there = !e.value || j < left;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float a, i;
                    gates((float)fv.v[j][k], a, i);
                    const float n = fmaf(a, cut ? 0.f : s[k], i * (float)xv.v[j][k]);
                    s[k] = there ? n : s[k];
                }
                put_line<!e.value>(hw, hp, one, me.halves, j, s);
            }
        };
        flags || !whole ? steps(Edge{}) : steps(Plain{});
    }
    if (A.h_last && me.z == A.ranges - 1 && me.live) keep_pair(A.h_last + at, s, me.half);
}

template <class E> __global__ __launch_bounds__(64 * LINE_GROUP) void k_line_grad_maps(ScanGradArgs A)
{
    const Line me(A.B, A.C, A.ranges, A.range, A.apart, A.torn);
    const E *f = (const E *)A.f + me.b * A.f_bs, *dh = (const E *)A.dh + me.b * A.dh_bs;
    const uint8_t *reset = A.reset ? A.reset + me.b * A.r_bs : nullptr;
    const bool wanted = me.live && me.z > 0;
    const int fp = wanted ? me.place(A.f_ts, sizeof(E)) : NOWHERE, gp = wanted ? me.place(A.dh_ts, sizeof(E)) : NOWHERE;
    float *maps = A.totals + me.b * (A.ranges + me.groups) * 2 * A.C + me.c;
    Map m;
    if (!me.idle && me.z1 > 0) {
        LineRows<E> fr, gr;
        LineResets rs;
        auto fetch = [&](long t) {
            const bool whole = me.whole(t, A.T);
            fr.fetch(f, A.f_ts, t, A.T, A.C, fp, whole);
            gr.fetch(dh, A.dh_ts, t, A.T, A.C, gp, whole);
            if (reset) rs.fetch(reset, A.r_ts, t, A.T, me);
        };
        const long t0 = me.z0 * A.range, last = t0 + (me.batches(A.ranges, A.T) - 1) * LINE, mine = min(A.T, (me.z + 1) * A.range);
        fetch(last);
        for (long t = last; t >= t0; t -= LINE) {
            const uint64_t flags = rs.flags();
            const bool whole = me.whole(t, A.T);
            const LineRows<E> fv = fr, gv = gr;
            if (t > t0) fetch(t - LINE);
            auto steps = [&](auto e) {
                const long left = e.value ? mine - me.step(t) : LINE;
                const unsigned cuts = e.value ? of_lane(flags, me) : 0;
#pragma unroll
                for (int j = LINE - 1; j >= 0; --j) {
                    const bool cut = e.value && cuts >> j & 1, there = !e.value || j < left;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float a, i;
                        gates((float)fv.v[j][k], a, i);
                        const float n = cut ? 0.f : a * ((float)gv.v[j][k] + m.h[k]);
                        m.h[k] = there ? n : m.h[k];
                        m.a[k] *= there ? a : 1.f;
                    }
                }
                if (e.value) m.cut |= cuts != 0;
            };
            flags || !whole ? steps(Edge{}) : steps(Plain{});
        }
        if (!wanted) m = Map{};
    }
    leave_maps<false>(m, me, maps, A.ranges, A.C);
}

template <class E> __global__ __launch_bounds__(64 * LINE_GROUP) void k_line_grad(ScanGradArgs A)
{
    const Line me(A.B, A.C, A.ranges, A.range, A.apart, A.torn);
    if (A.ranges == 1 && me.idle) return;
    const E *f = (const E *)A.f + me.b * A.f_bs, *x = (const E *)A.x + me.b * A.x_bs, *dh = (const E *)A.dh + me.b * A.dh_bs;
    E *df = (E *)A.df + me.b * A.df_bs, *dx = (E *)A.dx + me.b * A.dx_bs;
    const uint8_t *reset = A.reset ? A.reset + me.b * A.r_bs : nullptr;
    constexpr int size = sizeof(E);
    const int fp = me.live ? me.place(A.f_ts, size) : NOWHERE, xp = me.live ? me.place(A.x_ts, size) : NOWHERE, gp = me.live ? me.place(A.dh_ts, size) : NOWHERE;
    const int dfo = me.live ? me.place(A.df_ts, size) : NOWHERE, dfp = me.half ? NOWHERE : dfo, df1 = me.half ? dfo + size : NOWHERE;
    const int dxo = me.live ? me.place(A.dx_ts, size) : NOWHERE, dxp = me.half ? NOWHERE : dxo, dx1 = me.half ? dxo + size : NOWHERE;
    const long at = me.b * A.C + me.c, t0 = me.z0 * A.range, last = t0 + (me.batches(A.ranges, A.T) - 1) * LINE, mine = min(A.T, (me.z + 1) * A.range);
    const float *final = A.carry + ((me.b + 1) * A.tiles - 1) * A.C + me.c, *carry = A.carry + (me.b * A.tiles + (me.live ? me.step(last) : last) / LINE) * A.C + me.c;   // a lane that is not live reads what the first does
    LineRows<E> fr, xr, gr;
    LineResets rs;
    float first[2];
    auto fetch = [&](long t) {
        const bool whole = me.whole(t, A.T);
        fr.fetch(f, A.f_ts, t, A.T, A.C, fp, whole);
        xr.fetch(x, A.x_ts, t, A.T, A.C, xp, whole);
        gr.fetch(dh, A.dh_ts, t, A.T, A.C, gp, whole);
        if (reset) rs.fetch(reset, A.r_ts, t, A.T, me);
        pair(whole || carry < final ? carry : final, first);   // a range that has ended reads what is there
        carry -= A.C;
    };
    if (!me.idle) fetch(last);
    float mu[2] = {};
    if (A.dlast) pair(A.dlast + at, mu);
    if (A.ranges > 1) {
        enter_range<false>(mu, me, A.totals + me.b * (A.ranges + me.groups) * 2 * A.C + me.c, A.ranges, A.C);
        if (me.idle) return;
    }
    for (long t = last; t >= t0; t -= LINE) {
        const uint64_t flags = rs.flags();
        const bool whole = me.whole(t, A.T);
        const LineRows<E> fv = fr, xv = xr, gv = gr;
        float s[2] = {first[0], first[1]}, before[LINE][2], ga[LINE][2], gi[LINE][2];
        if (t > t0) fetch(t - LINE);
        const Window<E> dfw(df, A.df_ts, t, A.T, A.C), dxw(dx, A.dx_ts, t, A.T, A.C);
        auto steps = [&](auto e) {
            const unsigned cuts = e.value ? of_lane(flags, me) : 0;
            const long left = e.value ? mine - me.step(t) : LINE;
#pragma unroll
            for (int j = 0; j < LINE; ++j) {
                const bool cut = e.value && cuts >> j & 1;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    gates((float)fv.v[j][k], ga[j][k], gi[j][k]);
                    before[j][k] = cut ? 0.f : s[k];
                    s[k] = fmaf(ga[j][k], before[j][k], gi[j][k] * (float)xv.v[j][k]);
                }
            }
#pragma unroll
            for (int j = LINE - 1; j >= 0; --j) {
                const bool cut = e.value && cuts >> j & 1, there = !e.value || j < left;
                float odf[2], odx[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float l = (float)gv.v[j][k] + mu[k], n = ga[j][k] * l;
                    odx[k] = gi[j][k] * l;
                    odf[k] = gi[j][k] * n * (before[j][k] - (float)xv.v[j][k]);
                    mu[k] = !there ? mu[k] : cut ? 0.f : n;
                }
                put_line<!e.value>(dfw, dfp, df1, e.value && me.halves, j, odf);
                put_line<!e.value>(dxw, dxp, dx1, e.value && me.halves, j, odx);
            }
        };
        flags || !whole || me.halves ? steps(Edge{}) : steps(Plain{});
    }
    if (A.dh0 && me.z == 0 && me.live) keep_pair(A.dh0 + at, mu, me.half);
}

// ------------------------------------------------------------ narrow sequences
// Few channels: a wave of a strip or a line would have few lanes at work.  Here a thread takes one channel through a range of
// steps, neighbouring threads the channels and then the ranges, and time is cut as far as it takes to have enough
// threads (83 sequences of 95456 steps of one channel in bf16: 139 us forward, 179 backward, 0.4 TB/s: a load of a wave
// touches 64 lines there).  Maps of ranges first, then one wave per channel of a sequence joins them into the states that enter the ranges
// (in place of the maps' H), then the ranges.  `totals` is [2][B][ranges][C]: A (-1: an episode starts there), H.
struct Thread {
    long b;
    int z, c;
    bool none;
    __device__ __forceinline__ Thread(int B, int ranges, int C)
    {
        const long id = (long)blockIdx.x * 256 + threadIdx.x;
        const long q = id / C;
        c = (int)(id - q * C);
        b = q / ranges;
        z = (int)(q - b * ranges);
        none = b >= B;
    }
};
// Steps t .. t + N - 1 of a thread, those from `end` on being the last one: what it loads of a tensor, and bit j of the
// flags for step j.  N is 32 (16 backward) for many steps of one or two channels, so that a line of memory, which holds the steps one
// after the other there, is used whole while it is in the first cache; else 8.
template <int N, class E> __device__ __forceinline__ void steps_of(E (&v)[N], const E *p, long ts, long t, long end)
{
    if (t + N <= end) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = p[(t + j) * ts];
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = p[min(t + j, end - 1) * ts];
    }
}
template <int N, class Args> __device__ __forceinline__ unsigned flags_of(const Args &A, long b, long t, long end)
{
    unsigned m = 0;
    if (!A.reset) return m;
    const uint8_t *p = A.reset + b * A.r_bs;
    if (A.r_ts == 1 && t + N <= end) {   // eight flags at a time, at any address
#pragma unroll
        for (int k = 0; k < N; k += 8) {
            uint64_t v;
            __builtin_memcpy(&v, p + t + k, 8);
            if (!v) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j) m |= (unsigned)((v >> 8 * j & 255) != 0) << (k + j);
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) m |= (unsigned)(t + j < end && p[min(t + j, end - 1) * A.r_ts] != 0) << j;
    }
    return m;
}

// The map of steps t0 .. end - 1 of a channel, forward and backward.
template <class E, int N> __device__ __forceinline__ void narrow_map(const ScanArgs &A, long b, int c, long t0, long end, float &pa, float &ph, bool &cut)
{
    const E *f = (const E *)A.f + b * A.f_bs + c, *x = (const E *)A.x + b * A.x_bs + c;
    unsigned all = 0;
    pa = 1.f;
    ph = 0.f;
    for (long t = t0; t < end; t += N) {
        E fv[N], xv[N];
        steps_of<N>(fv, f, A.f_ts, t, end);
        steps_of<N>(xv, x, A.x_ts, t, end);
        const unsigned flags = flags_of<N>(A, b, t, end);
        all |= flags;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (t + j >= end) break;
            float a, i;
            gates((float)fv[j], a, i);
            ph = fmaf(a, flags >> j & 1 ? 0.f : ph, i * (float)xv[j]);
            pa *= a;
        }
    }
    cut = all;
}
template <class E, int N> __device__ __forceinline__ void narrow_map(const ScanGradArgs &A, long b, int c, long t0, long end, float &pa, float &pp, bool &cut)
{
    const E *f = (const E *)A.f + b * A.f_bs + c, *dh = (const E *)A.dh + b * A.dh_bs + c;
    unsigned all = 0;
    pa = 1.f;
    pp = 0.f;
    for (long t = t0 + (end - t0 - 1) / N * N; t >= t0; t -= N) {
        E fv[N], gv[N];
        steps_of<N>(fv, f, A.f_ts, t, end);
        steps_of<N>(gv, dh, A.dh_ts, t, end);
        const unsigned flags = flags_of<N>(A, b, t, end);
        all |= flags;
#pragma unroll
        for (int j = N - 1; j >= 0; --j) {
            if (t + j >= end) continue;
            float a, i;
            gates((float)fv[j], a, i);
            pp = flags >> j & 1 ? 0.f : a * ((float)gv[j] + pp);
            pa *= a;
        }
    }
    cut = all;
}

// The steps themselves, from the state s that enters them; t0 is a multiple of LINE.  s: the state after them.
template <class E, int N> __device__ __forceinline__ void narrow_run(const ScanArgs &A, long b, int c, long t0, long end, float &s)
{
    const E *f = (const E *)A.f + b * A.f_bs + c, *x = (const E *)A.x + b * A.x_bs + c;
    E *h = (E *)A.h + b * A.h_bs + c;
    float *carry = A.carry ? A.carry + (b * A.tiles + t0 / LINE) * A.C + c : nullptr;
    for (long t = t0; t < end; t += N) {
        E fv[N], xv[N];
        steps_of<N>(fv, f, A.f_ts, t, end);
        steps_of<N>(xv, x, A.x_ts, t, end);
        const unsigned flags = flags_of<N>(A, b, t, end);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (t + j >= end) break;
            if (j % LINE == 0 && carry) { *carry = s; carry += A.C; }
            float a, i;
            gates((float)fv[j], a, i);
            s = fmaf(a, flags >> j & 1 ? 0.f : s, i * (float)xv[j]);
            h[(t + j) * A.h_ts] = (E)s;
        }
    }
}
template <class E, int N> __device__ __forceinline__ void narrow_run(const ScanGradArgs &A, long b, int c, long t0, long end, float &mu)
{
    const E *f = (const E *)A.f + b * A.f_bs + c, *x = (const E *)A.x + b * A.x_bs + c, *dh = (const E *)A.dh + b * A.dh_bs + c;
    E *df = (E *)A.df + b * A.df_bs + c, *dx = (E *)A.dx + b * A.dx_bs + c;
    for (long t = t0 + (end - t0 - 1) / N * N; t >= t0; t -= N) {
        float s = A.carry[(b * A.tiles + t / LINE) * A.C + c], before[N], ga[N], gi[N];
        E fv[N], xv[N], gv[N];
        steps_of<N>(fv, f, A.f_ts, t, end);
        steps_of<N>(xv, x, A.x_ts, t, end);
        steps_of<N>(gv, dh, A.dh_ts, t, end);
        const unsigned flags = flags_of<N>(A, b, t, end);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            gates((float)fv[j], ga[j], gi[j]);
            before[j] = flags >> j & 1 ? 0.f : s;
            s = fmaf(ga[j], before[j], gi[j] * (float)xv[j]);
        }
#pragma unroll
        for (int j = N - 1; j >= 0; --j) {
            if (t + j >= end) continue;
            const float l = (float)gv[j] + mu, n = ga[j] * l;
            dx[(t + j) * A.dx_ts] = (E)(gi[j] * l);
            df[(t + j) * A.df_ts] = (E)(gi[j] * n * (before[j] - (float)xv[j]));
            mu = flags >> j & 1 ? 0.f : n;
        }
    }
}
// what enters a sequence and where what leaves it goes
__host__ __device__ __forceinline__ const float *entering(const ScanArgs &A) { return A.h0; }
__host__ __device__ __forceinline__ const float *entering(const ScanGradArgs &A) { return A.dlast; }
__device__ __forceinline__ float *leaving(const ScanArgs &A) { return A.h_last; }
__device__ __forceinline__ float *leaving(const ScanGradArgs &A) { return A.dh0; }

// A workgroup takes a sequence of up to NARROW_BLOCK elements: a thread a channel and a run of steps, maps joined in LDS, the
// second reading from the caches.  One launch where ranges take three, and its lines are read by one unit.  us forward /
// backward here against ranges, B x T x C in bf16: 32 x 333 x 3: 8 / 10, 25 / 31; 300 x 250 x 16: 11 / 19, 22 / 25; 300 x 4000 x 1: 21 / 33,
// 34 / 45; past its limit one workgroup a sequence is too few: 32 x 16000 x 1: 39 / 62, 33 / 42; 32 x 4062 x 16: 37 / 67, 23 / 27.
constexpr int NARROW_BLOCK = 8192;
template <class Args> constexpr int BLOCK_THREADS = std::is_same<Args, ScanArgs>::value ? 1024 : 512;   // as many as have registers
template <class E, class Args> __global__ __launch_bounds__(BLOCK_THREADS<Args>) void k_narrow_block(Args A)
{
    constexpr bool FORWARD = std::is_same<Args, ScanArgs>::value;
    __shared__ float sa[BLOCK_THREADS<Args>], sh[BLOCK_THREADS<Args>];
    const int c = threadIdx.x % A.C, runs = blockDim.x / A.C, run = threadIdx.x / A.C, order = FORWARD ? run : runs - 1 - run;
    const long b = blockIdx.x, range = ((A.T + runs - 1) / runs + LINE - 1) / LINE * LINE, t0 = min(A.T, run * range), end = min(A.T, t0 + range);
    const bool mine = run < runs;
    const int at = order * A.C + c;   // place of this run's map among those of its channel
    const float *first = entering(A);
    float s = first ? first[b * A.C + c] : 0.f;   // every run reads it, and the last may write its own state there: before the joins
    float a = 1.f, h = 0.f;
    bool cut = false;
    if (mine && t0 < end) narrow_map<E, 8>(A, b, c, t0, end, a, h, cut);
    if (cut) a = -1.f;
    for (int d = 1; d < runs; d *= 2) {   // maps of all runs up to this one
        if (mine) { sa[at] = a; sh[at] = h; }
        __syncthreads();
        if (mine && order >= d) {
            const float oa = sa[at - d * A.C], oh = sh[at - d * A.C];
            h = through(oh, a, h, a < 0.f);
            a = a < 0.f || oa < 0.f ? -1.f : a * oa;
        }
        __syncthreads();
    }
    if (mine) { sa[at] = a; sh[at] = h; }
    arrived(s);
    __syncthreads();
    if (!mine) return;
    if (order) s = through(s, sa[at - A.C], sh[at - A.C], sa[at - A.C] < 0.f);
    if (t0 < end) narrow_run<E, 8>(A, b, c, t0, end, s);
    float *last = leaving(A);
    if (last && order == runs - 1) last[b * A.C + c] = s;
}

template <class E, int N, class Args> __global__ __launch_bounds__(256) void k_narrow_maps(Args A)
{
    const Thread me(A.B, A.ranges, A.C);
    if (me.none) return;
    const long t0 = me.z * A.range, end = min(A.T, t0 + A.range), at = (me.b * A.ranges + me.z) * A.C + me.c;
    float a, h;
    bool cut;
    narrow_map<E, N>(A, me.b, me.c, t0, end, a, h, cut);
    A.totals[at] = cut ? -1.f : a;
    A.totals[(long)A.B * A.ranges * A.C + at] = h;
}

// One wave per channel of a sequence: lane l has the ranges from ranges l / 64 on (backward: from the other end).  `first`
// ([B][C] or NULL): what enters the first of them.  In: maps; out: in place of H what enters each range.
template <bool FORWARD> __global__ __launch_bounds__(64) void k_narrow_join(float *totals, const float *first, int B, int ranges, int C)
{
    const int lane = threadIdx.x, c = blockIdx.x % C;
    const long b = blockIdx.x / C;
    float *A = totals + b * ranges * C + c, *H = A + (long)B * ranges * C;
    const int lo = (int)((long)ranges * lane / 64), hi = (int)((long)ranges * (lane + 1) / 64);
    auto at = [&](int q) { return (long)(FORWARD ? q : ranges - 1 - q) * C; };
    float a = 1.f, h = 0.f;      // the map of this lane's ranges
#pragma unroll 4
    for (int q = lo; q < hi; ++q) {
        const float qa = A[at(q)], qh = H[at(q)];
        h = through(h, qa, qh, qa < 0.f);
        a = qa < 0.f || a < 0.f ? -1.f : a * qa;
    }
    for (int d = 1; d < 64; d *= 2) {   // of all up to this lane's
        const float oa = __shfl_up(a, d), oh = __shfl_up(h, d);
        if (lane >= d) {
            h = through(oh, a, h, a < 0.f);
            a = a < 0.f || oa < 0.f ? -1.f : a * oa;
        }
    }
    const float ea = __shfl_up(a, 1), eh = __shfl_up(h, 1);
    float s = first ? first[b * C + c] : 0.f;
    if (lane) s = through(s, ea, eh, ea < 0.f);
#pragma unroll 4
    for (int q = lo; q < hi; ++q) {
        const float qa = A[at(q)], qh = H[at(q)];
        H[at(q)] = s;
        s = through(s, qa, qh, qa < 0.f);
    }
}

template <class E, int N, class Args> __global__ __launch_bounds__(256) void k_narrow(Args A)
{
    constexpr bool FORWARD = std::is_same<Args, ScanArgs>::value;
    const Thread me(A.B, A.ranges, A.C);
    if (me.none) return;
    const long t0 = me.z * A.range, end = min(A.T, t0 + A.range);
    const float *first = entering(A);
    float s = A.ranges > 1 ? A.totals[((long)A.B + me.b) * A.ranges * A.C + (long)me.z * A.C + me.c] : first ? first[me.b * A.C + me.c] : 0.f;
    narrow_run<E, N>(A, me.b, me.c, t0, end, s);
    float *last = leaving(A);
    if (last && (FORWARD ? end == A.T : me.z == 0)) last[me.b * A.C + me.c] = s;
}

}  // namespace seq
