// A step for matrices whose momentum is made orthogonal by products of itself: the optimizer, and the three coefficients of its Newton-Schulz rounds, of
// Jordan et al. 2024, "Muon: An optimizer for hidden layers in neural networks".
//
// With m <- mu m + g and u = g + mu m (or m) of r <= c (the transposed where there are more rows than columns): X = u / (|u| + eps), then `rounds`
// times  A = X X^T,  B = b A + c A^2,  X <- a X + B X, which takes all singular values near one.  At last p <- p (1 - lr decay) - lr s X.
//
// The products are the cost, 2 r^2 c + 2 r^3 + 2 r^2 c operations a round, a fourth less with A and A^2 formed on one side of their
// diagonal.  Operands are pairs of bf16, hi + lo, which hold 16 bits of a number, and a product takes three matrix instructions,
// hi hi + hi lo + lo hi: rounding X or A to one bf16 would put the result 2^-9 off at every round, pairs are 2^-17 off, and fp32
// instructions have a sixteenth of the rate.  Sums are fp32.
//
// X is kept as its transposed Y [c][r] alone.  B X has rows of B and rows of Y as operands, whose inner dimension lies in one piece; what a lane
// holds of a result is four neighbours of a row of the new Y.  X X^T has columns of Y on both sides, which the transposing LDS reads take.
// A row lies in memory as 32 numbers' hi, the same numbers' lo, the next 32 numbers: 128 bytes, a line, for 32 of the inner dimension.
// Sizes are padded with zeros to multiples of PAD, so that no product looks at bounds of the inner dimension.
#pragma once
#include "seq_common.h"

namespace seq {

constexpr int PAD = 64;
constexpr int MUON_CHUNK = 4096;        // elements of a partial sum of squares
constexpr int TILES[3] = {64, 128, 256};       // rows and columns of a workgroup's part of a product

struct MuonMatrix {
    float *p, *m;
    const void *g;
    uint16_t *copy;
    bf16 *y[2], *a, *b;
    double *sums;
    long rows, cols;
    int rp, cp;                         // the shorter and the longer side, padded
    int tall;                           // more rows than columns: y is the matrix, else its transposed
    float decay, scale;
    int chunks;                         // of its elements
    int first_chunk, first_start;       // its first workgroup in a launch over chunks, over parts of 64 x 64,
    int first_half[3], first_whole[3];  // over parts of A on and below the diagonal, over parts of X, by their size
};
struct MuonArgs {
    const MuonMatrix *matrices;
    int count, nesterov, from;          // from: which Y holds X
    float mu, eps, lr, a, b, c;
};

// The matrix that workgroup `i` of a launch belongs to.
template <class F> __device__ __forceinline__ const MuonMatrix &matrix_of(const MuonArgs &A, int i, F &&first)
{
    int lo = 0, hi = A.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        (first(A.matrices[mid]) <= i ? lo : hi) = mid;
    }
    return A.matrices[lo];
}

template <class G> __global__ __launch_bounds__(256) void k_muon_momentum(MuonArgs A)
{
    __shared__ double sh[4];
    const MuonMatrix &M = matrix_of(A, blockIdx.x, [](const MuonMatrix &m) { return m.first_chunk; });
    const int chunk = blockIdx.x - M.first_chunk;
    const long first = (long)chunk * MUON_CHUNK, n = min((long)MUON_CHUNK, M.rows * M.cols - first);
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) {
        const float g = (float)((const G *)M.g)[first + i], m = fmaf(A.mu, M.m[first + i], g), u = A.nesterov ? fmaf(A.mu, m, g) : m;
        M.m[first + i] = m;
        sum += (double)u * u;           // squares of what fp32 holds may pass its range
    }
#pragma unroll
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) M.sums[chunk] = (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

__device__ __forceinline__ void halves_of(float v, bf16 &hi, bf16 &lo)
{
    hi = (bf16)v;
    lo = (bf16)(v - (float)hi);
}

// where the hi of number (row, col) of a matrix `width` wide lies; its lo is 32 further
__device__ __forceinline__ long hi_at(long row, int col, int width) { return row * 2 * width + (col >> 5) * 64 + (col & 31); }

// Y, 64 x 64 of it per workgroup.
template <class G> __global__ __launch_bounds__(256) void k_muon_start(MuonArgs A)
{
    __shared__ float t[64][65];
    __shared__ double sh[4];
    const MuonMatrix &M = matrix_of(A, blockIdx.x, [](const MuonMatrix &m) { return m.first_start; });
    const int tile = blockIdx.x - M.first_start, across = M.rp / 64, ti = tile / across, tj = tile % across;      // rows of Y 64 ti.., columns 64 tj..
    double sum = 0.0;
    for (int i = threadIdx.x; i < M.chunks; i += 256) sum += M.sums[i];
#pragma unroll
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = sum;
    __syncthreads();
    const float inv = 1.f / ((float)sqrt((sh[0] + sh[1]) + (sh[2] + sh[3])) + A.eps);
    const int c = threadIdx.x & 63;
    for (int r = threadIdx.x >> 6; r < 64; r += 4) {
        const long row = (long)(M.tall ? ti : tj) * 64 + r, col = (long)(M.tall ? tj : ti) * 64 + c;      // as they lie in memory
        float v = 0.f;
        if (row < M.rows && col < M.cols) {
            const long at = row * M.cols + col;
            const float m = M.m[at];
            v = (A.nesterov ? fmaf(A.mu, m, (float)((const G *)M.g)[at]) : m) * inv;
        }
        (M.tall ? t[r][c] : t[c][r]) = v;
    }
    __syncthreads();
    for (int r = threadIdx.x >> 6; r < 64; r += 4) {
        bf16 *y = M.y[0] + hi_at(ti * 64 + r, tj * 64 + c, M.rp);
        halves_of(t[r][c], y[0], y[32]);
    }
}

using f4 = vec<float, 4>;
using b4 = vec<bf16, 4>;
using b8 = vec<bf16, 8>;
struct Pair4 {
    b4 hi, lo;
    __device__ __forceinline__ f4 whole() const
    {
        return f4{(float)hi[0] + (float)lo[0], (float)hi[1] + (float)lo[1], (float)hi[2] + (float)lo[2], (float)hi[3] + (float)lo[3]};
    }
};
__device__ __forceinline__ Pair4 pair_at(const bf16 *hi) { return Pair4{load<4>(hi), load<4>(hi + 32)}; }
__device__ __forceinline__ void put_halves(bf16 *hi, f4 v)
{
    b4 a, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        a[e] = (bf16)v[e];
        b[e] = (bf16)(v[e] - (float)a[e]);
    }
    store<4>(hi, a);
    store<4>(hi + 32, b);
}

// N x N numbers of L R^T (COLUMNS false: rows i0.. of L, j0.. of R, both K wide) or of L^T R (COLUMNS: columns i0.., j0.. of the same matrix of K rows,
// `width` wide), `steps` steps of 32 of K from k0 on, by WM x WN waves, a wave having MI x NI results of 16 x 16, a lane rows 4 (l / 16).. of column l % 16 of each.  32 of K a step,
// STAGES steps' operands in LDS: while one is multiplied, the next ones come from memory past the registers (four stages of 64 x 64, which are often
// few and wait for memory: a step 0.49 us with two, 0.36 with four).
// LDS, rows: a row's 128 bytes in eight pieces of 16, four of hi and four of lo; piece c of row r has the place c ^ (r / 2 % 8).  Columns: a row has 4 N
// bytes in pieces of 32, sixteen columns' hi or lo; piece c of row r has the place c ^ (r % 8).  So the lanes that LDS serves together meet each of
// its banks once.
constexpr int muon_stages(int n) { return n == 64 ? 4 : 2; }
constexpr int muon_lds(int n) { return muon_stages(n) * 256 * n; }
template <int N, int WM, int WN, bool COLUMNS> struct MuonProduct {
    static constexpr int WAVES = WM * WN, MI = N / WM / 16, NI = N / WN / 16, SIDE = N * 128, STAGE = 2 * SIDE, LOADS = STAGE / 1024 / WAVES, STAGES = muon_stages(N);
    static_assert(STAGE % (1024 * WAVES) == 0 && LOADS >= 1, "whole loads of a wave");
    f4 acc[MI][NI];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int x = 0; x < MI; ++x)
#pragma unroll
            for (int y = 0; y < NI; ++y) acc[x][y] = f4{};
    }
    __device__ __forceinline__ void run(uint8_t *lds, const bf16 *L, const bf16 *R, int i0, int j0, int rows_l, int rows_r, int width, int K, int k0, int steps)
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
        const uint8_t *src[LOADS];
        const long pitch = COLUMNS ? 4l * width : 4l * K, step_bytes = COLUMNS ? 32 * pitch : 128;
#pragma unroll
        for (int q = 0; q < LOADS; ++q) {
            const int at = (wave * LOADS + q) * 1024 + lane * 16, side = at / SIDE, in = at % SIDE;
            const bf16 *from = side ? R : L;
            const int first = side ? j0 : i0, last = side ? rows_r : rows_l;
            if (COLUMNS) {
                const int r = in / (4 * N), piece = in % (4 * N) / 32 ^ (r & 7);
                const int block = min(first / 32 + piece / 4, width / 32 - 1);        // beyond the last columns: numbers that nobody keeps
                src[q] = (const uint8_t *)from + r * pitch + block * 128 + (piece & 3) * 32 + (in & 16);
            } else {
                const int r = in / 128, piece = in % 128 / 16 ^ (r >> 1 & 7);
                src[q] = (const uint8_t *)from + min(first + r, last - 1) * pitch + piece * 16;
            }
        }
        auto fetch = [&](int step) {
            uint8_t *to = lds + step % STAGES * STAGE + wave * LOADS * 1024;
            const long from = (k0 / 32 + min(step, steps - 1)) * step_bytes;      // behind the last step it again, so that the same number is under way always
#pragma unroll
            for (int q = 0; q < LOADS; ++q) to_lds(src[q] + from, to + q * 1024);
        };
        // 16 rows (columns) from `first` on as an operand, its hi and its lo
        auto operand = [&](const uint8_t *side, int first, b8 (&v)[2]) {
            if constexpr (COLUMNS) {
                using s4 = vec<short, 4>;
                typedef __attribute__((address_space(3))) s4 *At;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int piece = first / 32 * 4 + 2 * h + (first >> 4 & 1), r = 8 * g + (i >> 2);
                    const uint8_t *a = side + r * (4 * N) + (piece ^ (i >> 2)) * 32 + (i & 3) * 8;
                    const uint8_t *b = side + (r + 4) * (4 * N) + (piece ^ ((i >> 2) + 4)) * 32 + (i & 3) * 8;
                    const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)a), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)b);
                    v[h] = __builtin_bit_cast(b8, (vec<short, 8>){x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]});
                }
            } else {
                const int place = (first + i) * 128 + (g ^ (i >> 1)) * 16;
                v[0] = *reinterpret_cast<const b8 *>(side + place);
                v[1] = *reinterpret_cast<const b8 *>(side + (place ^ 64));
            }
        };
        clear();
        const int wm = wave % WM * MI * 16, wn = wave / WM * NI * 16;
#pragma unroll
        for (int n = 0; n + 1 < STAGES; ++n) fetch(n);
        for (int step = 0; step < steps; ++step) {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * LOADS) : "memory");
            fetch(step + STAGES - 1);
            const uint8_t *l = lds + step % STAGES * STAGE, *r = l + SIDE;
            constexpr int READS = COLUMNS ? 4 : 2;      // of LDS for an operand
            b8 b[NI][2], next[2];
#pragma unroll
            for (int y = 0; y < NI; ++y) operand(r, wn + 16 * y, b[y]);
            operand(l, wm, next);
            __builtin_amdgcn_sched_group_barrier(0x100, READS * (NI + 1), 0);
#pragma unroll
            for (int x = 0; x < MI; ++x) {      // the next 16 rows are read behind the products of these
                const b8 a[2] = {next[0], next[1]};
                if (x + 1 < MI) operand(l, wm + 16 * (x + 1), next);
#pragma unroll
                for (int y = 0; y < NI; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[1], b[y][0], acc[x][y], 0, 0, 0);
#pragma unroll
                for (int y = 0; y < NI; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[0], b[y][1], acc[x][y], 0, 0, 0);
#pragma unroll
                for (int y = 0; y < NI; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[0], b[y][0], acc[x][y], 0, 0, 0);
                if (x + 1 < MI) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 3 * NI, 0);
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // nothing may arrive in LDS that another workgroup has by then
    }
    // f(row, column, the four numbers of rows row.. and that column, get(row, column)); what several get() read is asked for before the first is waited for
    template <class G, class F> __device__ __forceinline__ void each(G &&get, F &&f)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave % WM * MI * 16 + 4 * (lane >> 4), wn = wave / WM * NI * 16 + (lane & 15);
#pragma unroll
        for (int x = 0; x < MI; ++x) {
            decltype(get(0, 0)) old[NI];
#pragma unroll
            for (int y = 0; y < NI; ++y) old[y] = get(wm + 16 * x, wn + 16 * y);
#pragma unroll
            for (int y = 0; y < NI; ++y) f(wm + 16 * x, wn + 16 * y, acc[x][y], old[y]);
        }
    }
};
constexpr int muon_wn(int n) { return n == 256 ? 4 : 2; }
constexpr int muon_threads(int n) { return 128 * muon_wn(n); }

// The part of a matrix that workgroup `i` of its `n` takes: neighbouring parts on the same XCD (workgroups go round the eight), whose L2 holds what
// they read together, and every matrix, its inner dimension being its own, spread over all of them (twelve of two kinds: 537 us for B X where the
// eight took an eighth of all parts each, 424 so).
__device__ __forceinline__ int muon_part(int i, int n)
{
    const int x = i & 7, q = n / 8, r = n % 8;
    return x * q + min(x, r) + (i >> 3);
}

// SQUARE: B = b A + c A A, else A = X X^T; a part on or below the diagonal and its mirror.  Where parts are few and K is long, it is cut: SPLIT leaves `cuts` sums of
// each part, JOIN adds them up in their order.
enum Gram { WHOLE, SQUARE, SPLIT, JOIN };
template <Gram G, int T> __global__ __launch_bounds__(muon_threads(TILES[T])) void k_muon_gram(MuonArgs A, f4 *sums, int cuts)
{
    constexpr int N = TILES[T], THREADS = muon_threads(N);
    extern __shared__ __align__(16) uint8_t lds[];
    const int group = blockIdx.x, which = G == SPLIT ? group / cuts : group;
    const MuonMatrix &M = matrix_of(A, which, [](const MuonMatrix &m) { return m.first_half[T]; });
    const int rp = M.rp, down = (rp + N - 1) / N, part = G == SPLIT || G == JOIN ? which - M.first_half[T] : muon_part(which - M.first_half[T], down * (down + 1) / 2);
    int ti = (int)((sqrtf(8.f * part + 1.f) - 1.f) * 0.5f);
    while (ti * (ti + 1) / 2 > part) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= part) ++ti;
    const int tj = part - ti * (ti + 1) / 2, i0 = ti * N, j0 = tj * N;
    MuonProduct<N, 2, muon_wn(N), G != SQUARE> P;
    constexpr int MI = decltype(P)::MI, NI = decltype(P)::NI;
    if (G == SQUARE) P.run(lds, M.a, M.a, i0, j0, rp, rp, rp, rp, 0, rp / 32);
    if (G == WHOLE) P.run(lds, M.y[A.from], M.y[A.from], i0, j0, rp, rp, rp, M.cp, 0, M.cp / 32);
    if (G == SPLIT) {
        const int steps = M.cp / 32, per = (steps + cuts - 1) / cuts, first = min(group % cuts * per, steps), n = min(per, steps - first);
        if (n > 0) P.run(lds, M.y[A.from], M.y[A.from], i0, j0, rp, rp, rp, M.cp, 32 * first, n);
        else P.clear();
#pragma unroll
        for (int x = 0; x < MI; ++x)
#pragma unroll
            for (int y = 0; y < NI; ++y) sums[((long)group * MI * NI + x * NI + y) * THREADS + threadIdx.x] = P.acc[x][y];
        return;
    }
    if (G == JOIN) {
        P.clear();
        for (int k = 0; k < cuts; ++k)
#pragma unroll
            for (int x = 0; x < MI; ++x)
#pragma unroll
                for (int y = 0; y < NI; ++y) P.acc[x][y] += sums[(((long)which * cuts + k) * MI * NI + x * NI + y) * THREADS + threadIdx.x];
    }
    bf16 *out = G == SQUARE ? M.b : M.a;
    P.each([&](int r, int c) { return G == SQUARE ? pair_at(M.a + hi_at(min(j0 + c, rp - 1), min(i0 + r, rp - 4), rp)) : Pair4{}; },
           [&](int r, int c, f4 v, const Pair4 &old) {
        const int row = i0 + r, col = j0 + c;
        if (row >= rp || col >= rp) return;
        const long mirror = hi_at(col, row, rp);
        if (G == SQUARE) v = A.b * old.whole() + A.c * v;
        put_halves(out + mirror, v);
        if (ti != tj)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                bf16 *p = out + hi_at(row + e, col, rp);
                halves_of(v[e], p[0], p[32]);
            }
    });
}

// X <- a X + B X, into the other Y; the last time into the parameters.
template <bool LAST, int T> __global__ __launch_bounds__(muon_threads(TILES[T])) void k_muon_apply(MuonArgs A)
{
    constexpr int N = TILES[T];
    extern __shared__ __align__(16) uint8_t lds[];
    const MuonMatrix &M = matrix_of(A, blockIdx.x, [](const MuonMatrix &m) { return m.first_whole[T]; });
    const int down = (M.rp + N - 1) / N, part = muon_part((int)blockIdx.x - M.first_whole[T], down * ((M.cp + N - 1) / N)), i0 = part % down * N, j0 = part / down * N;
    MuonProduct<N, 2, muon_wn(N), false> P;
    P.run(lds, M.b, M.y[A.from], i0, j0, M.rp, M.cp, M.rp, M.rp, 0, M.rp / 32);
    if (!LAST) {
        P.each([&](int r, int c) { return pair_at(M.y[A.from] + hi_at(min(j0 + c, M.cp - 1), min(i0 + r, M.rp - 4), M.rp)); },
               [&](int r, int c, f4 v, const Pair4 &old) {
            const int row = i0 + r, col = j0 + c;       // of X
            if (row < M.rp && col < M.cp) put_halves(M.y[A.from ^ 1] + hi_at(col, row, M.rp), A.a * old.whole() + v);
        });
        return;
    }
    struct Old {
        Pair4 x;
        float p[4];
    };
    const long down_p = M.tall ? 1 : M.cols, across_p = M.tall ? M.cols : 1;       // from row to row, column to column of X in the parameters
    const int r_end = (int)(M.tall ? M.cols : M.rows), c_end = (int)(M.tall ? M.rows : M.cols);
    P.each([&](int r, int c) {
               const int row = i0 + r, col = j0 + c;
               Old o;
               o.x = pair_at(M.y[A.from] + hi_at(min(col, M.cp - 1), min(row, M.rp - 4), M.rp));
#pragma unroll
               for (int e = 0; e < 4; ++e) o.p[e] = M.p[min(row + e, r_end - 1) * down_p + min(col, c_end - 1) * across_p];
               return o;
           },
           [&](int r, int c, f4 v, const Old &old) {
        const int row = i0 + r, col = j0 + c;
        v = A.a * old.x.whole() + v;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (row + e < r_end && col < c_end) {
                const long to = (row + e) * down_p + col * across_p;
                const float n = old.p[e] - A.lr * (M.decay * old.p[e] + M.scale * v[e]);
                M.p[to] = n;
                if (M.copy) M.copy[to] = __builtin_bit_cast(uint16_t, (bf16)n);
            }
    });
}

}  // namespace seq
