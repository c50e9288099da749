// A step for matrices whose momentum is made orthogonal by products of itself.
//
// With m <- mu m + g and u = g + mu m (or m) of r <= c (the transposed where there are more rows than columns): X = u / (|u| + eps), then `rounds`
// times  A = X X^T,  B = b A + c A^2,  X <- a X + B X, which takes all singular values near one.  At last p <- p (1 - lr decay) - lr s X.
//
// The products are the cost, 2 r^2 c + 2 r^3 + 2 r^2 c operations a round, a fourth less with A and A^2 formed on one side of their
// diagonal.  Operands are pairs of bf16, hi + lo, which hold 16 bits of a number, and a product takes three matrix instructions,
// hi hi + hi lo + lo hi: rounding X or A to one bf16 would put the result 2^-9 off at every round, pairs are 2^-17 off, and fp32
// instructions have a sixteenth of the rate.  Sums are fp32.  All operands lie with their inner dimension in one piece: A and B are
// symmetric, and X is kept as its transposed as well.  Sizes are padded with zeros to multiples of TILE, so that no product looks at bounds.
#pragma once
#include "seq_common.h"

namespace seq {

constexpr int MT = 64;                  // rows and columns of a tile of a product
constexpr int MUON_CHUNK = 4096;        // elements of a partial sum of squares

struct MuonMatrix {
    float *p, *m;
    const void *g;
    uint16_t *copy;
    bf16 *x, *xt[2], *a, *b;            // planes: all hi, then all lo
    double *sums;
    long rows, cols;
    int rp, cp;                         // the shorter and the longer side, padded
    int tall;                           // more rows than columns: x is the transposed
    float decay, scale;
    int chunks;                         // of its elements
    int first_chunk, first_half, first_whole;   // its first workgroup in a launch over chunks, tiles on and below the diagonal of A, tiles of X
};
struct MuonArgs {
    const MuonMatrix *matrices;
    int count, nesterov;
    float mu, eps, lr, a, b, c;
};

// The matrix that workgroup `i` of a launch belongs to.
template <int MuonMatrix::*FIRST> __device__ __forceinline__ const MuonMatrix &matrix_of(const MuonArgs &A, int i)
{
    int lo = 0, hi = A.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        (A.matrices[mid].*FIRST <= i ? lo : hi) = mid;
    }
    return A.matrices[lo];
}

template <class G> __global__ __launch_bounds__(256) void k_muon_momentum(MuonArgs A)
{
    __shared__ double sh[4];
    const MuonMatrix &M = matrix_of<&MuonMatrix::first_chunk>(A, blockIdx.x);
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

// X and its transposed, a tile of 64 x 64 per workgroup.
template <class G> __global__ __launch_bounds__(256) void k_muon_start(MuonArgs A)
{
    __shared__ float t[MT][MT + 1];
    __shared__ double sh[4];
    const MuonMatrix &M = matrix_of<&MuonMatrix::first_whole>(A, blockIdx.x);
    const int tile = blockIdx.x - M.first_whole, across = M.cp / MT, ti = tile / across, tj = tile % across;
    double sum = 0.0;
    for (int i = threadIdx.x; i < M.chunks; i += 256) sum += M.sums[i];
#pragma unroll
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = sum;
    __syncthreads();
    const float inv = 1.f / ((float)sqrt((sh[0] + sh[1]) + (sh[2] + sh[3])) + A.eps);
    const int c = threadIdx.x & 63;
    for (int r = threadIdx.x >> 6; r < MT; r += 4) {
        // row and column as they lie in memory; in t as they lie in x
        const long row = (long)(M.tall ? tj : ti) * MT + r, col = (long)(M.tall ? ti : tj) * MT + c;
        float v = 0.f;
        if (row < M.rows && col < M.cols) {
            const long at = row * M.cols + col;
            const float m = M.m[at];
            v = (A.nesterov ? fmaf(A.mu, m, (float)((const G *)M.g)[at]) : m) * inv;
        }
        (M.tall ? t[c][r] : t[r][c]) = v;
    }
    __syncthreads();
    const long plane = (long)M.rp * M.cp;
    for (int r = threadIdx.x >> 6; r < MT; r += 4) {
        bf16 hi, lo;
        halves_of(t[r][c], hi, lo);
        bf16 *x = M.x + (long)(ti * MT + r) * M.cp + tj * MT + c;
        x[0] = hi;
        x[plane] = lo;
        halves_of(t[c][r], hi, lo);
        x = M.xt[0] + (long)(tj * MT + r) * M.rp + ti * MT + c;
        x[0] = hi;
        x[plane] = lo;
    }
}

using f4 = vec<float, 4>;

// Rows i0.. of L times rows j0.. of R, both [.][K] in planes, inner dimension in one piece: 32 x 32 of each wave's, lane l holding rows
// 4 (l / 16).. of column l % 16 of each of four 16 x 16.
constexpr int MK = 64, MLD = MK + 8;    // inner dimension of a step, and its rows' distance in LDS
struct MuonTiles {
    bf16 l[2][MT * MLD], r[2][MT * MLD];
};
__device__ __forceinline__ void muon_product(MuonTiles &s, const bf16 *L, long lplane, int i0, const bf16 *R, long rplane, int j0, int K, f4 (&acc)[2][2])
{
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, wi = 32 * (w >> 1), wj = 32 * (w & 1);
    for (int k0 = 0; k0 < K; k0 += MK) {
        __syncthreads();
        for (int e = tid; e < MT * MK / 8; e += 256) {
            const int r = e / (MK / 8), c = e % (MK / 8) * 8;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                *reinterpret_cast<vec<bf16, 8> *>(s.l[h] + r * MLD + c) = *reinterpret_cast<const vec<bf16, 8> *>(L + h * lplane + (long)(i0 + r) * K + k0 + c);
                *reinterpret_cast<vec<bf16, 8> *>(s.r[h] + r * MLD + c) = *reinterpret_cast<const vec<bf16, 8> *>(R + h * rplane + (long)(j0 + r) * K + k0 + c);
            }
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < MK; kk += 32) {
            vec<bf16, 8> a[2][2], b[2][2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    a[h][n] = *reinterpret_cast<const vec<bf16, 8> *>(s.l[h] + (wi + 16 * n + (lane & 15)) * MLD + kk + 8 * (lane >> 4));
                    b[h][n] = *reinterpret_cast<const vec<bf16, 8> *>(s.r[h] + (wj + 16 * n + (lane & 15)) * MLD + kk + 8 * (lane >> 4));
                }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[1][i], b[0][j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[0][i], b[1][j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[0][i], b[0][j], acc[i][j], 0, 0, 0);
                }
        }
    }
}

// SQUARE: B = b A + c A A, else A = X X^T; a tile on or below the diagonal and its mirror.
template <bool SQUARE> __global__ __launch_bounds__(256) void k_muon_gram(MuonArgs A)
{
    __shared__ __align__(16) MuonTiles s;
    const MuonMatrix &M = matrix_of<&MuonMatrix::first_half>(A, blockIdx.x);
    const int tile = blockIdx.x - M.first_half;
    int ti = (int)((sqrtf(8.f * tile + 1.f) - 1.f) * 0.5f);
    while (ti * (ti + 1) / 2 > tile) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= tile) ++ti;
    const int tj = tile - ti * (ti + 1) / 2, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const long plane = (long)M.rp * M.rp;
    f4 acc[2][2] = {};
    if (SQUARE) muon_product(s, M.a, plane, ti * MT, M.a, plane, tj * MT, M.rp, acc);
    else muon_product(s, M.x, (long)M.rp * M.cp, ti * MT, M.x, (long)M.rp * M.cp, tj * MT, M.cp, acc);
    bf16 *out = SQUARE ? M.b : M.a;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const long row = ti * MT + 32 * (w >> 1) + 16 * i + 4 * (lane >> 4), col = tj * MT + 32 * (w & 1) + 16 * j + (lane & 15);
            vec<bf16, 4> hi, lo;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const long at = (row + e) * M.rp + col;
                float v = acc[i][j][e];
                if (SQUARE) v = A.b * ((float)M.a[at] + (float)M.a[at + plane]) + A.c * v;
                bf16 h, l;
                halves_of(v, h, l);
                out[at] = hi[e] = h;
                out[at + plane] = lo[e] = l;
            }
            if (ti != tj) {
                *reinterpret_cast<vec<bf16, 4> *>(out + col * M.rp + row) = hi;
                *reinterpret_cast<vec<bf16, 4> *>(out + col * M.rp + row + plane) = lo;
            }
        }
}

// X <- a X + B X, from the transposed number `from` into the other; the last time into the parameters.
template <bool LAST> __global__ __launch_bounds__(256) void k_muon_apply(MuonArgs A, int from)
{
    __shared__ __align__(16) MuonTiles s;
    const MuonMatrix &M = matrix_of<&MuonMatrix::first_whole>(A, blockIdx.x);
    const int tile = blockIdx.x - M.first_whole, across = M.cp / MT, ti = tile / across, tj = tile % across, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const long plane = (long)M.rp * M.cp;
    f4 acc[2][2] = {};
    muon_product(s, M.b, (long)M.rp * M.rp, ti * MT, M.xt[from], plane, tj * MT, M.rp, acc);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const long row = ti * MT + 32 * (w >> 1) + 16 * i + 4 * (lane >> 4), col = tj * MT + 32 * (w & 1) + 16 * j + (lane & 15);
            vec<bf16, 4> hi, lo;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const long at = (row + e) * M.cp + col;
                const float v = A.a * ((float)M.x[at] + (float)M.x[at + plane]) + acc[i][j][e];
                if (LAST) {
                    const long r = M.tall ? col : row + e, c = M.tall ? row + e : col;
                    if (r < M.rows && c < M.cols) {
                        const long to = r * M.cols + c;
                        const float p = M.p[to], n = p - A.lr * (M.decay * p + M.scale * v);
                        M.p[to] = n;
                        if (M.copy) M.copy[to] = __builtin_bit_cast(uint16_t, (bf16)n);
                    }
                } else {
                    bf16 h, l;
                    halves_of(v, h, l);
                    M.x[at] = hi[e] = h;
                    M.x[at + plane] = lo[e] = l;
                }
            }
            if (!LAST) {
                bf16 *to = M.xt[from ^ 1] + col * M.rp + row;
                *reinterpret_cast<vec<bf16, 4> *>(to) = hi;
                *reinterpret_cast<vec<bf16, 4> *>(to + plane) = lo;
            }
        }
}

}  // namespace seq
