// Product of 8-bit rows with 8-bit weights, y = (a w^T) a_scale w_scale + bias.
//
// The matrix instructions on e4m3 (16 x 16 outputs, 128 k) run at twice the rate of those on bf16, but they do not add up
// in 32 bits: products are cut off 16 bits below the largest one's exponent (of products of 7.875 beside 256 x 256 and
// its opposite each counted as 7: measured, 880 for 992).  So 128 of them are off by up to 2^-9 of the largest, which the
// rounding of its operands to e4m3 has moved by up to 2^-4; over random numbers the sums are 1.5e-5 off in the 2-norm at every K,
// where the same numbers as bf16, which holds them exactly, are 5e-8 off.  An output that is rounded to bf16 loses a hundred
// times that anyway and takes them; an fp32 output, for which a caller may ask, takes the numbers as bf16.
//
// Operands are swapped, weights as the instruction's rows: a lane then has four neighbouring columns of a row of y and
// stores them at once.  A lane holds 32 bytes of one row of either operand, lane l of row l % 16 bytes 32 (l / 16) and
// on of every 128; which k the instruction takes them for is the same on both sides and does not matter.
#pragma once
#include "seq_common.h"

namespace seq {

struct ProductArgs {
    const uint8_t *a, *w;
    long a_rs, w_rs;
    const float *a_scale, *w_scale, *bias;
    void *y;
    long y_rs, M;
    int N, K;
    int wide;   // columns of y that can be stored at once: 1, 4 or, in bf16, 8
};

using Bytes32 = vec<int, 8>;
using Acc = vec<float, 4>;

// 16 bytes of a row from k on (a multiple of 16), those from K on set to zero; nothing is read if k >= K
__device__ __forceinline__ vec<uint32_t, 4> row_piece(const uint8_t *row, int k, int K)
{
    vec<uint32_t, 4> v = {};
    if (k < K) {
        v = *reinterpret_cast<const vec<uint32_t, 4> *>(row + k);
        const int left = K - k;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = left - 4 * i;   // bytes of this word that count
            v[i] = n >= 4 ? v[i] : n <= 0 ? 0u : v[i] & ~(~0u << 8 * n);
        }
    }
    return v;
}
__device__ __forceinline__ Bytes32 joined(vec<uint32_t, 4> lo, vec<uint32_t, 4> hi)
{
    return Bytes32{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// An operand's 32 bytes in the form in which the outputs' type wants them multiplied.
template <class E> struct Operand;
template <> struct Operand<bf16> {
    Bytes32 v;
    __device__ __forceinline__ void set(Bytes32 b) { v = b; }
};
template <> struct Operand<float> {
    vec<bf16, 8> v[4];
    __device__ __forceinline__ void set(Bytes32 b)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const auto lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b[i], 1.f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b[i], 1.f, true);
            v[i / 2][i % 2 * 4] = lo[0]; v[i / 2][i % 2 * 4 + 1] = lo[1]; v[i / 2][i % 2 * 4 + 2] = hi[0]; v[i / 2][i % 2 * 4 + 3] = hi[1];
        }
    }
};
__device__ __forceinline__ Acc mac(const Operand<bf16> &w, const Operand<bf16> &a, Acc s)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.v, a.v, s, 0, 0, 0, 0, 0, 0);   // e4m3 both, no scales
}
__device__ __forceinline__ Acc mac(const Operand<float> &w, const Operand<float> &a, Acc s)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.v[i], a.v[i], s, 0, 0, 0);
    return s;
}

// columns n .. n + 3 of row m; w: their scales, b: their biases
template <class E> __device__ __forceinline__ void put(const ProductArgs &A, long m, int n, Acc s, float sa, Acc w, Acc b)
{
    if (m >= A.M || n >= A.N) return;
    vec<E, 4> v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = (E)(s[j] * sa * w[j] + b[j]);
    E *p = (E *)A.y + m * A.y_rs + n;
    if (A.wide >= 4 && n + 4 <= A.N) {
        *reinterpret_cast<vec<E, 4> *>(p) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n + j < A.N) p[j] = v[j];
    }
}
__device__ __forceinline__ Acc four_of(const float *p, int n, int N)   // p[n .. n + 3], or zeros where p is NULL or ends
{
    Acc v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = p && n + j < N ? p[n + j] : 0.f;
    return v;
}

// ------------------------------------------------------------ few outputs
// A workgroup takes MI x 16 rows and NI x 16 columns; its waves share K, 128 bytes in turn, straight from memory into
// registers, and add up in LDS.  For products that would not give every compute unit a tile of the kernel below: what
// counts then is that much is in flight at once (32 x 1024 x 512: 3.3 us; 1 x 4096 x 8192, 34 MB of weights: 7.4 us, 8.8 from memory).
constexpr int FEW_WAVES = 8;
template <class E, int MI, int NI> __global__ __launch_bounds__(64 * FEW_WAVES) void k_product_few(ProductArgs A)
{
    __shared__ Acc part[FEW_WAVES][MI * NI][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const int tiles = (A.N + 16 * NI - 1) / (16 * NI);
    const long m0 = (long)(blockIdx.x / tiles) * (16 * MI);
    const int n0 = (int)(blockIdx.x % tiles) * (16 * NI);
    const uint8_t *a[MI], *w[NI];
#pragma unroll
    for (int x = 0; x < MI; ++x) a[x] = A.a + min(m0 + 16 * x + i, A.M - 1) * A.a_rs;
#pragma unroll
    for (int x = 0; x < NI; ++x) w[x] = A.w + (long)min(n0 + 16 * x + i, A.N - 1) * A.w_rs;
    Acc s[MI][NI] = {};
    for (int k = wave * 128; k < A.K; k += FEW_WAVES * 128) {
        const int at = k + 32 * g;
        vec<uint32_t, 4> va[MI][2], vw[NI][2];
        if (k + 128 <= A.K) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int x = 0; x < MI; ++x) va[x][h] = *reinterpret_cast<const vec<uint32_t, 4> *>(a[x] + at + 16 * h);
#pragma unroll
                for (int x = 0; x < NI; ++x) vw[x][h] = *reinterpret_cast<const vec<uint32_t, 4> *>(w[x] + at + 16 * h);
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int x = 0; x < MI; ++x) va[x][h] = row_piece(a[x], at + 16 * h, A.K);
#pragma unroll
                for (int x = 0; x < NI; ++x) vw[x][h] = row_piece(w[x], at + 16 * h, A.K);
            }
        }
        Operand<E> oa[MI];
#pragma unroll
        for (int x = 0; x < MI; ++x) oa[x].set(joined(va[x][0], va[x][1]));
#pragma unroll
        for (int y = 0; y < NI; ++y) {
            Operand<E> ow;
            ow.set(joined(vw[y][0], vw[y][1]));
#pragma unroll
            for (int x = 0; x < MI; ++x) s[x][y] = mac(ow, oa[x], s[x][y]);
        }
    }
#pragma unroll
    for (int x = 0; x < MI; ++x)
#pragma unroll
        for (int y = 0; y < NI; ++y) part[wave][x * NI + y][lane] = s[x][y];
    __syncthreads();
    for (int t = wave; t < MI * NI; t += FEW_WAVES) {   // a 16 x 16 tile per wave
        Acc sum = part[0][t][lane];
#pragma unroll
        for (int v = 1; v < FEW_WAVES; ++v) sum += part[v][t][lane];
        const long m = m0 + t / NI * 16 + i;
        const int n = n0 + t % NI * 16 + 4 * g;
        put<E>(A, m, n, sum, A.a_scale[min(m, A.M - 1)], four_of(A.w_scale, n, A.N), four_of(A.bias, n, A.N));
    }
}

// ------------------------------------------------------------ tiles
// BM x BN outputs per workgroup, WM x WN waves, 128 k a step, two steps' operands in LDS: while one is multiplied, the
// next comes from memory past the registers.  Measured, 256 x 256 tiles of 8192 x 4096 outputs in bf16: 23.4 us per 1024 of K
// (2.9 PFLOP/s) and 20 us to begin and end; K = 2048 66 us.  A row of a step is 128 bytes in eight pieces of 16; piece c of row r has
// the place c ^ (r / 2 % 8), so that the sixteen lanes that LDS serves together, a piece of sixteen rows, meet each of
// its 64 banks once.

// Which tile a workgroup takes: neighbouring ones on the same XCD (workgroups go round the eight), eight tiles high
// bands of them, so that an XCD's L2 holds what its workgroups read together.
struct Tile {
    long m;
    int n;
    __device__ __forceinline__ Tile(int tm, int tn)
    {
        const int all = tm * tn, x = blockIdx.x & 7, q = all / 8, r = all % 8;
        const int t = x * q + min(x, r) + (int)(blockIdx.x >> 3);
        const int band = t / (8 * tn), first = band * 8, high = min(tm - first, 8), in = t - band * 8 * tn;
        m = first + in % high;
        n = in / high;
    }
};

template <class E, int BM, int BN, int WM, int WN> __global__ __launch_bounds__(64 * WM * WN) void k_product_tile(ProductArgs A)
{
    constexpr int WAVES = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16, LOADS = (BM + BN) / 8 / WAVES, STAGE = (BM + BN) * 128;
    static_assert((BM + BN) % (8 * WAVES) == 0 && BM % 8 == 0, "a wave's loads are eight rows of one operand each");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];   // [2][BM rows of a, BN rows of w][128]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
    const Tile tile((int)((A.M + BM - 1) / BM), (A.N + BN - 1) / BN);
    const long m0 = tile.m * BM;
    const int n0 = tile.n * BN, full = A.K / 128, steps = (A.K + 127) / 128;

    const uint8_t *src[LOADS];   // row and piece of this lane in the wave's loads
    static_assert(LOADS % 2 == 0, "a wave's loads begin at a multiple of sixteen rows");
    auto piece = [&](int q) { return ((lane & 7) ^ (lane >> 4) ^ (q & 1) * 4) * 16; };
#pragma unroll
    for (int q = 0; q < LOADS; ++q) {
        const int r = (wave * LOADS + q) * 8 + (lane >> 3);
        src[q] = (r < BM ? A.a + min(m0 + r, A.M - 1) * A.a_rs : A.w + (long)min(n0 + r - BM, A.N - 1) * A.w_rs) + piece(q);
    }
    auto fetch = [&](int step) {
        uint8_t *to = lds + (step & 1) * STAGE + wave * LOADS * 1024;
        if (step < full) {
#pragma unroll
            for (int q = 0; q < LOADS; ++q) to_lds(src[q] + (long)step * 128, to + q * 1024);
        } else {   // the last step, where K ends within it
#pragma unroll
            for (int q = 0; q < LOADS; ++q)
                *reinterpret_cast<vec<uint32_t, 4> *>(to + q * 1024 + lane * 16) = row_piece(src[q] - piece(q), step * 128 + piece(q), A.K);
        }
    };
    const int wm = wave % WM * MI * 16, wn = wave / WM * NI * 16;
    const int place = i * 128 + ((2 * g) ^ (i >> 1)) * 16;   // of this lane's first piece among 16 rows; the second: place ^ 16
    Acc s[MI][NI] = {};
    if (steps) fetch(0);
    for (int step = 0; step < steps; ++step) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (step + 1 < steps) fetch(step + 1);
        const uint8_t *la = lds + (step & 1) * STAGE + wm * 128, *lw = lds + (step & 1) * STAGE + (BM + wn) * 128;
        auto piece32 = [&](const uint8_t *rows) {
            return joined(*reinterpret_cast<const vec<uint32_t, 4> *>(rows + place), *reinterpret_cast<const vec<uint32_t, 4> *>(rows + (place ^ 16)));
        };
        Operand<E> w[NI];
#pragma unroll
        for (int y = 0; y < NI; ++y) w[y].set(piece32(lw + y * 2048));
        Bytes32 next = piece32(la);
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * NI + 2, 0);
#pragma unroll
        for (int x = 0; x < MI; ++x) {   // the next 16 rows are read behind the products of these
            Operand<E> a;
            a.set(next);
            if (x + 1 < MI) next = piece32(la + (x + 1) * 2048);
#pragma unroll
            for (int y = 0; y < NI; ++y) s[x][y] = mac(w[y], a, s[x][y]);
            if (x + 1 < MI) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, NI * (sizeof(E) == 2 ? 1 : 4), 0);
        }
    }
    // 64 columns of a row are a line or two of memory.  Stored as the lanes hold them, 8 bytes of each of sixteen rows, they
    // took 19 us of a tile of 8192 x 4096 outputs in bf16.  So they change places through LDS, whose operands are done
    // with: rows of 64 columns, in pieces of 16 bytes with places as the operands' have.  Then a lane stores a piece; where
    // y's rows are not aligned to pieces or end within the columns, a lane a column.
    if constexpr (NI == 4) {
        constexpr int ES = sizeof(E), ROW = 64 * ES, PIECES = ROW / 16, SHARE = 2 * STAGE / WAVES, XP = SHARE / (16 * ROW) < MI ? SHARE / (16 * ROW) : MI;
        static_assert(MI % XP == 0, "passes of whole 16 rows");
        auto swap = [](int r) { return ES == 2 ? r >> 1 & 7 : r & 15; };
        uint8_t *mine = lds + wave * SHARE;
        const bool whole = A.wide == 16 / ES && n0 + wn + 64 <= A.N;
        __syncthreads();
#pragma unroll
        for (int pass = 0; pass < MI; pass += XP) {   // the wave reads what it wrote itself: its own LDS accesses are in order
#pragma unroll
            for (int y = 0; y < NI; ++y) {
                const int n = n0 + wn + 16 * y + 4 * g;
                const Acc sw = four_of(A.w_scale, n, A.N), b = four_of(A.bias, n, A.N);
#pragma unroll
                for (int x = 0; x < XP; ++x) {
                    const float sa = A.a_scale[min(m0 + wm + 16 * (pass + x) + i, A.M - 1)];
                    vec<E, 4> v;
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = (E)(s[pass + x][y][j] * sa * sw[j] + b[j]);
                    const int at = (16 * y + 4 * g) * ES;
                    *reinterpret_cast<vec<E, 4> *>(mine + (16 * x + i) * ROW + ((at / 16) ^ swap(i)) * 16 + at % 16) = v;
                }
            }
            const long m1 = m0 + wm + 16 * pass;
            E *out = (E *)A.y + m1 * A.y_rs + n0 + wn;
            if (whole) {
#pragma unroll
                for (int q = 0; q < XP * 16 * PIECES / 64; ++q) {
                    const int r = q * (64 / PIECES) + lane / PIECES, c = lane % PIECES;
                    const auto v = *reinterpret_cast<const vec<uint32_t, 4> *>(mine + r * ROW + (c ^ swap(r)) * 16);
                    if (m1 + r < A.M) *reinterpret_cast<vec<uint32_t, 4> *>(out + r * A.y_rs + c * (16 / ES)) = v;
                }
            } else if (n0 + wn + lane < A.N) {
                const int left = (int)min((long)(16 * XP), A.M - m1);
#pragma unroll 8
                for (int r = 0; r < left; ++r)
                    out[r * A.y_rs + lane] = *reinterpret_cast<const E *>(mine + r * ROW + ((lane * ES / 16) ^ swap(r)) * 16 + lane * ES % 16);
            }
        }
        return;
    }
#pragma unroll
    for (int y = 0; y < NI; ++y) {
        const int n = n0 + wn + 16 * y + 4 * g;
        const Acc sw = four_of(A.w_scale, n, A.N), b = four_of(A.bias, n, A.N);
#pragma unroll
        for (int x = 0; x < MI; ++x) {
            const long m = m0 + wm + 16 * x + i;
            put<E>(A, m, n, s[x][y], A.a_scale[min(m, A.M - 1)], sw, b);
        }
    }
}

}  // namespace seq
