// C ABI of the recurrent network's operators (see include/dqn.h): checks of arguments and launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <algorithm>
#include <atomic>
#include <initializer_list>
#include <new>
#include <type_traits>
#include <vector>

#include "adamw.h"
#include "checks.h"
#include "norm.h"
#include "rows_product.h"
#include "scan.h"

struct dqn_adamw {
    seq::AdamArgs args;
    int64_t chunks;
    int bits, grad_dtype;
};

namespace {

// Which form a recurrence takes, by how many lines (sequences times strips of 128 channels) and strips (of 64) there are; us
// forward / backward in bf16, C = 512, B x T:
//   512 x 64, 2048 lines:  whole lines 18 / 36              256 x 128, 1024 lines: strips 31 / 44, lines 24 / 46
//   128 x 256, 512 lines:  strips 27 / 40, lines 44 / 73     32 x 512, 256 strips: strips 13 / 21, ranges 20 / 26
// below that ranges, see SCAN_UNITS.  A compute unit holds one workgroup of a strip, so that strips go in turns of 256: B x 512, strips and
// ranges, 31: 13 / 20, 19 / 27; 33: 23 / 35, 28 / 35; 63: 25 / 38, 33 / 43; 65: 35 / 53, 44 / 65; 100: 46 / 71, 50 / 71.  Below 256, and for
// long sequences in a part of a turn (40 x 4000: 166 / 285, 145 / 240), the other form than the one taken is the faster.
// Narrow sequences: up to 16 channels, up to 32 of more than 1000 steps; us forward / backward, narrow against ranges of lines,
// B x T x C in bf16: 2000 x 3000 x 8: 184 / 283, 240 / 298; 200 x 4000 x 5: 38 / 51, 48 / 70; 574 x 2844 x 17: 125 / 160, 150 / 189.  Ranges
// of lines where a strip is filled for five eighths (100 x 3000 x 32: 42 / 52, 26 / 35; 2000 x 1000 x 16: 122 / 166, 89 / 120) or sequences and
// steps are few (1 x 131072 x 2: 44 / 53, 25 / 31; 10 x 30000 x 3: 29 / 34, 22 / 26; 64 x 20000 x 4: 35 / 49, 56 / 79).  Short ones a
// workgroup each (see there).
constexpr int64_t SCAN_FEW = 1 << 18, SCAN_LINES = 2048, SCAN_STRIPS = 256, SCAN_WANT = 4096, SCAN_LEAST = 32;
// Ranges of lines: the compute units hold one workgroup of eight waves each of the backward kernel, two of the lines' other kernels, and a
// second turn of a few workgroups takes as long as the first.  So ranges are as short as leaves one workgroup for each unit, or two
// if that is still 64 steps a range (131072 x 512 in bf16, forward: 122 us, 125 with one).  us forward / backward by the
// steps of a range (workgroups), in bf16:
//   7 x 4099 x 256:  16 (462) 21 / 30   24 (308) 24 / 35   32 (238) 20 / 26   48 (154) 24 / 31
//   7 x 4099 x 320:  16 (693) 25 / 36   24 (462) 25 / 36   32 (357) 27 / 40   48 (231) 25 / 33
// Every range composes the maps of all groups before it, so that more than 2048 cost more than they give (1 x 65536 x 64: 24 / 29 us
// with 1024, 20 / 22 with 2048; before the loads went out in eights 27 / 29 with 2048, 34 / 34 with 4096).
constexpr int64_t SCAN_UNITS = 256, SCAN_MOST = 2048;
constexpr long SCAN_LONG_RANGE = 64;
// One or two channels: 32 steps of a thread at a time rather than 8 from this many elements on (83 x 95456 x 1: 139 / 179 us against
// 166 / 400; 60 x 25811 x 1: 55 / 61 against 38 / 48).
constexpr int64_t SCAN_LONG = 6 << 20;
constexpr int64_t LAST_LEVEL = 256 << 20;   // bytes of the cache in front of memory


// Called with elements present: a [B][T][C] tensor, its strides no shorter than what they step over, and apart for a
// tensor that is written (no element twice).  Where there is one step, or one sequence, its stride is not taken.
const char *check_steps(const void *p, int64_t bs, int64_t ts, const dqn_scan_args &s, bool written)
{
    if (s.B == 1) bs = 0;
    if (s.T == 1) ts = 0;
    if (!p || !at(p, bytes_of(s.dtype))) return "a tensor is NULL or not aligned to its elements";
    if (bs < 0 || ts < 0 || bs > MOST || ts > 1 << 24) return "a stride is negative or too large";   // 16 rows are within 2^30 bytes
    if (ts > 0 && s.T - 1 > MOST / ts) return "T times a stride is too large";
    if (bs > 0 && s.B - 1 > MOST / bs) return "B times a stride is too large";
    if (!written) return nullptr;
    const bool apart = (s.T == 1 || ts >= s.C) && (s.B == 1 || bs >= s.C) &&
                       (s.T == 1 || s.B == 1 || bs >= (s.T - 1) * ts + s.C || ts >= (s.B - 1) * bs + s.C);
    return apart ? nullptr : "rows of an output lie on top of each other";
}

const char *check_scan(const dqn_scan_args &s)
{
    if (!dtype_ok(s.dtype)) return "dtype must be DQN_F32 or DQN_BF16";
    if (s.B < 0 || s.C < 0 || s.T < 0 || s.B > 65535 || s.C > 1 << 24 || (int64_t)s.B * s.C > 1 << 28 || !size_ok(s.B, s.T, s.C))
        return "B must be in 0..65535, C in 0..2^24, B C in 0..2^28, T >= 0";
    if (!at(s.h0, 4) || !at(s.h_last, 4) || !at(s.carry, 4)) return "a state is not aligned to its elements";
    if (s.reset && (s.reset_bs < 0 || s.reset_ts < 0 || s.reset_bs > MOST || s.reset_ts > MOST ||
                    (s.reset_ts > 0 && s.T - 1 > MOST / s.reset_ts))) return "a stride of reset is negative or too large";
    return nullptr;
}

// waves of a workgroup of lines in ranges
int line_waves(int32_t C) { return C > 128 ? seq::LINE_GROUP : (seq::line_width((C + 1) / 2) * seq::LINE_GROUP + 63) / 64; }

// How a recurrence of these sizes is cut: a function of the sizes alone, the same for both directions.
struct ScanCut {
    enum { SHORT, BLOCK, NARROW, STRIPS, LINES } form;
    int waves;         // of a workgroup of the strips
    long tile, tiles;  // steps between two states of `carry`, states of a sequence
    long range;        // lines: steps of a range
    int ranges;
};
ScanCut scan_cut(int32_t B, int64_t T, int32_t C)
{
    if (T <= seq::SCAN_SHORT) return ScanCut{ScanCut::SHORT, 0, seq::SCAN_SHORT, T ? 1 : 0, (long)T, 1};
    const int pairs = (C + 1) / 2;
    const bool narrow = C <= 16 || (C <= 32 && T > 1000), filled = C >= 16 && pairs * 8 >= seq::line_width(pairs) * 5;
    const bool few = narrow && B < SCAN_LINES && (filled || (C >= 2 && B * T <= SCAN_FEW));   // ranges of lines all the same
    if (narrow && (!few || T * C <= seq::NARROW_BLOCK)) {
        if (C && T * C <= seq::NARROW_BLOCK) return ScanCut{ScanCut::BLOCK, 0, seq::LINE, (long)((T + seq::LINE - 1) / seq::LINE), (long)T, 1};
        const int64_t all = std::max<int64_t>(1, (int64_t)B * C), want = std::max<int64_t>(1, std::min<int64_t>(SCAN_WANT * 64 / all, T / SCAN_LEAST));
        const long per = (T + want - 1) / want, range = (per + seq::LINE - 1) / seq::LINE * seq::LINE;
        return ScanCut{ScanCut::NARROW, 0, seq::LINE, (long)((T + seq::LINE - 1) / seq::LINE), range, (int)((T + range - 1) / range)};
    }
    const int64_t strips = (int64_t)B * ((C + seq::SCAN_STRIP - 1) / seq::SCAN_STRIP), lines = (int64_t)B * ((C + 127) / 128);
    if (!few && lines < SCAN_LINES && strips >= SCAN_STRIPS) {
        int waves = 1;
        while (waves < seq::SCAN_WAVES && 16 * waves < T) waves *= 2;
        const long tile = 16 * waves;
        return ScanCut{ScanCut::STRIPS, waves, tile, (long)((T + tile - 1) / tile), (long)T, 1};
    }
    long range = (T + seq::LINE - 1) / seq::LINE * seq::LINE;
    if (lines && lines < SCAN_LINES) {
        const int64_t groups = (int64_t)B * ((C + 127) / 128), slots = SCAN_UNITS * seq::LINE_GROUP / line_waves(C);
        auto cut = [&](int64_t all) {
            const int64_t n = std::min(std::max<int64_t>(1, all / groups) * seq::LINE_GROUP, SCAN_MOST);
            return (long)(((T + n - 1) / n + seq::LINE - 1) / seq::LINE * seq::LINE);
        };
        range = cut(2 * slots);
        if (range < SCAN_LONG_RANGE) range = cut(slots);
    }
    return ScanCut{ScanCut::LINES, 0, seq::LINE, (long)((T + seq::LINE - 1) / seq::LINE), range, (int)((T + range - 1) / range)};
}
size_t scan_workspace(const ScanCut &c, int32_t B, int32_t C)
{
    if (c.ranges == 1) return 0;
    if (c.form == ScanCut::NARROW) return ((size_t)B * c.ranges * 2 * C * 4 + 15) / 16 * 16;
    const size_t maps = c.ranges + (c.ranges + seq::LINE_GROUP - 1) / seq::LINE_GROUP;
    return ((size_t)B * maps * 2 * C * 4 + 15) / 16 * 16;
}

// whether `n` elements of every tensor can be taken at once
bool together(int n, int32_t dtype, int32_t C, std::initializer_list<const void *> tensors, std::initializer_list<int64_t> strides, std::initializer_list<const void *> states)
{
    if (C % n) return false;
    for (const void *p : tensors)
        if (!at(p, n * bytes_of(dtype))) return false;
    for (int64_t s : strides)
        if (s % n) return false;
    for (const void *p : states)
        if (!at(p, n * 4)) return false;
    return true;
}

template <class E, int V> void launch_short(const seq::ScanArgs &A, hipStream_t st)
{
    seq::k_scan_short<E, V><<<dim3((unsigned)(((int64_t)A.B * (A.C / V) + 255) / 256)), 256, 0, st>>>(A);
}
template <class E, int V> void launch_short(const seq::ScanGradArgs &A, hipStream_t st)
{
    seq::k_scan_grad_short<E, V><<<dim3((unsigned)(((int64_t)A.B * (A.C / V) + 255) / 256)), 256, 0, st>>>(A);
}
dim3 line_grid(int32_t B, int32_t C, int ranges)
{
    const int64_t strips = ((C + 1) / 2 + 63) / 64;
    return dim3((unsigned)(ranges == 1 ? (B * strips + seq::LINE_GROUP - 1) / seq::LINE_GROUP : strips * B * ((ranges + seq::LINE_GROUP - 1) / seq::LINE_GROUP)));
}
// whether a group's ranges are too far from one another to count the distance in 32 bits: eight of them within 2^30 bytes
bool far_ranges(int64_t range, std::initializer_list<int64_t> steps)
{
    const int64_t most = std::max(steps);
    return most && range > (1 << 25) / most;
}
// whether a row of a tensor begins within a line of the caches, of 128 bytes
bool torn_rows(std::initializer_list<const void *> tensors, size_t size, std::initializer_list<int64_t> strides)
{
    for (const void *p : tensors)
        if (!at(p, 128)) return true;
    for (int64_t s : strides)
        if (s * (int64_t)size % 128) return true;
    return false;
}
template <class E> void launch_lines(seq::ScanArgs A, hipStream_t st)
{
    A.apart = far_ranges(A.range, {A.f_ts, A.x_ts, A.h_ts});
    const dim3 grid = line_grid(A.B, A.C, A.ranges), block(64 * (A.ranges == 1 || A.apart ? seq::LINE_GROUP : line_waves(A.C)));
    if (A.ranges > 1) seq::k_line_maps<E><<<grid, block, 0, st>>>(A);
    if (2 * (int64_t)sizeof(E) * A.B * A.T * A.C >= LAST_LEVEL) seq::k_lines<E, seq::STREAM><<<grid, block, 0, st>>>(A);
    else seq::k_lines<E, 0><<<grid, block, 0, st>>>(A);
}
template <class E> void launch_lines(seq::ScanGradArgs A, hipStream_t st)
{
    A.apart = far_ranges(A.range, {A.f_ts, A.x_ts, A.dh_ts, A.df_ts, A.dx_ts});
    const dim3 grid = line_grid(A.B, A.C, A.ranges), block(64 * (A.ranges == 1 || A.apart ? seq::LINE_GROUP : line_waves(A.C)));
    if (A.ranges > 1) seq::k_line_grad_maps<E><<<grid, block, 0, st>>>(A);
    seq::k_line_grad<E><<<grid, block, 0, st>>>(A);
}
template <class E, int V> void launch_strips(const seq::ScanArgs &A, int waves, hipStream_t st)
{
    seq::k_scan<E, V><<<dim3((unsigned)((A.C + seq::SCAN_STRIP - 1) / seq::SCAN_STRIP * A.B)), 64 * waves, 0, st>>>(A);
}
template <class E, int V> void launch_strips(const seq::ScanGradArgs &A, int waves, hipStream_t st)
{
    seq::k_scan_grad<E, V><<<dim3((unsigned)((A.C + seq::SCAN_STRIP - 1) / seq::SCAN_STRIP * A.B)), 64 * waves, 0, st>>>(A);
}
template <class E, int N, class Args> void launch_narrow(const Args &A, hipStream_t st)
{
    constexpr bool FORWARD = std::is_same<Args, seq::ScanArgs>::value;
    const dim3 grid((unsigned)(((int64_t)A.B * A.ranges * A.C + 255) / 256));
    if (A.ranges > 1) {
        seq::k_narrow_maps<E, N, Args><<<grid, 256, 0, st>>>(A);
        seq::k_narrow_join<FORWARD><<<dim3((unsigned)(A.B * A.C)), 64, 0, st>>>(A.totals, seq::entering(A), A.B, A.ranges, A.C);
    }
    seq::k_narrow<E, FORWARD ? N : std::min(N, 16), Args><<<grid, 256, 0, st>>>(A);
}
template <class E, class Args> void launch_block(const Args &A, hipStream_t st)
{
    const int64_t threads = std::min<int64_t>(seq::BLOCK_THREADS<Args>, A.tiles * A.C);   // 8 steps each, or more
    seq::k_narrow_block<E, Args><<<dim3((unsigned)A.B), (unsigned)((threads + 63) / 64 * 64), 0, st>>>(A);
}
// fits(n): whether n channels can be taken at once
template <class E, class Args, class F> void launch_recurrence(const Args &A, const ScanCut &c, F &&fits, hipStream_t st)
{
    if (c.form == ScanCut::NARROW) A.C <= 2 && A.T * A.B * A.C >= SCAN_LONG ? launch_narrow<E, 32>(A, st) : launch_narrow<E, 8>(A, st);
    else if (c.form == ScanCut::BLOCK) launch_block<E>(A, st);
    else if (c.form == ScanCut::SHORT) fits(4) ? launch_short<E, 4>(A, st) : launch_short<E, 1>(A, st);
    else if (c.form == ScanCut::STRIPS) fits(2) ? launch_strips<E, 2>(A, c.waves, st) : launch_strips<E, 1>(A, c.waves, st);
    else launch_lines<E>(A, st);
}

const char *check_rows8(const void *p, int64_t rs, int64_t M, int64_t K)
{
    if (!p || !at(p, 16) || rs % 16 || rs < 0 || rs > MOST || (rs > 0 && M - 1 > MOST / rs)) return "8-bit rows must be 16-byte aligned, strides multiples of 16";
    return M == 1 || rs >= K ? nullptr : "the stride of 8-bit rows is shorter than a row";
}

// Partial sums of the weight's gradient, a workgroup each: of 16 rows, or of fewer where there would not be one workgroup per
// compute unit (241 rows of 6497: 16 workgroups 80 us, 241 workgroups 20 us).
int norm_parts(int64_t M, int C)
{
    const int64_t least = std::min<int64_t>(256, C > 1024 ? M : (M + 3) / 4);
    return (int)std::min<int64_t>(seq::NORM_PARTS, std::max<int64_t>((M + seq::NORM_ROWS - 1) / seq::NORM_ROWS, least));
}

// The smallest form of a norm kernel that holds a row of C elements (8-bit rows: up to the next multiple of 16), V being
// 16 bytes' worth of elements or 1.  go(V, K, W, lanes) launches it.  A thread holds up to 16 elements (more cost so many
// registers that few waves fit), a row is one wave's, four waves' or sixteen waves'.
template <int N> using Int = std::integral_constant<int, N>;
template <class E, class F> void norm_form(bool wide, int C, F &&go)
{
    constexpr int V = 16 / (int)sizeof(E);
    auto lanes = [&](int per) {
        int n = 1;
        while (n * per < C) n *= 2;
        return n;
    };
    if (wide) {
        if (C <= 64 * V) go(Int<V>{}, Int<1>{}, Int<1>{}, lanes(V));
        else if (C <= 128 * V) go(Int<V>{}, Int<2>{}, Int<1>{}, 64);
        else if (C <= 64 * 16) go(Int<V>{}, Int<16 / V>{}, Int<1>{}, 64);
        else if (C <= 256 * 16) go(Int<V>{}, Int<16 / V>{}, Int<4>{}, 64);
        else go(Int<V>{}, Int<16 / V>{}, Int<16>{}, 64);
    } else {
        if (C <= 64) go(Int<1>{}, Int<1>{}, Int<1>{}, lanes(1));
        else if (C <= 256) go(Int<1>{}, Int<4>{}, Int<1>{}, 64);
        else if (C <= 1024) go(Int<1>{}, Int<16>{}, Int<1>{}, 64);
        else if (C <= 4096) go(Int<1>{}, Int<16>{}, Int<4>{}, 64);
        else if (C <= 8192) go(Int<1>{}, Int<8>{}, Int<16>{}, 64);
        else go(Int<1>{}, Int<16>{}, Int<16>{}, 64);
    }
}
static_assert(DQN_NORM_MAX == 16 * 64 * 16, "the longest rows that norm_form can hold");

template <class E, bool EIGHT> void launch_norm(seq::NormArgs A, hipStream_t st)
{
    constexpr int n = 16 / (int)sizeof(E);
    const bool wide = together(n, sizeof(E) == 4 ? DQN_F32 : DQN_BF16, A.C, {A.x, A.residual, A.r, A.y}, {A.x_rs, A.residual_rs, A.r_rs, A.y_rs}, {A.weight});
    norm_form<E>(wide, EIGHT ? (A.C + 15) / 16 * 16 : A.C, [&](auto V, auto K, auto W, int lanes) {
        A.lanes = lanes;
        const int64_t rows = W.value > 1 ? 1 : 256 / lanes;
        const unsigned grid = (unsigned)std::min<int64_t>((A.M + rows - 1) / rows, 1 << 20);
        seq::k_norm<E, V.value, K.value, W.value, EIGHT><<<dim3(grid), W.value == 1 ? 256 : 64 * W.value, 0, st>>>(A);
    });
}
template <class E> void launch_norm_grad(seq::NormGradArgs A, int parts, hipStream_t st)
{
    constexpr int n = 16 / (int)sizeof(E);
    const bool wide = together(n, sizeof(E) == 4 ? DQN_F32 : DQN_BF16, A.C, {A.dy, A.x, A.residual, A.dr, A.dx}, {A.dy_rs, A.x_rs, A.residual_rs, A.dr_rs, A.dx_rs}, {A.weight});
    norm_form<E>(wide, A.C, [&](auto V, auto K, auto W, int lanes) {
        A.lanes = lanes;
        seq::k_norm_grad<E, V.value, K.value, W.value><<<dim3((unsigned)parts), W.value == 1 ? 256 : 64 * W.value, 0, st>>>(A);
    });
}

template <class E, int BM, int BN, int WM, int WN> bool launch_tile(const seq::ProductArgs &A, hipStream_t st)
{
    constexpr int bytes = 2 * (BM + BN) * 128;
    auto kernel = seq::k_product_tile<E, BM, BN, WM, WN>;
    static std::atomic<uint64_t> granted{0};
    if (!lds_granted((const void *)kernel, bytes, granted)) return false;
    const int64_t tiles = (A.M + BM - 1) / BM * ((A.N + BN - 1) / BN);
    kernel<<<dim3((unsigned)tiles), 64 * WM * WN, bytes, st>>>(A);
    return true;
}
template <class E, int MI, int NI> bool launch_few(const seq::ProductArgs &A, hipStream_t st)
{
    const int64_t tiles = (A.M + 16 * MI - 1) / (16 * MI) * ((A.N + 16 * NI - 1) / (16 * NI));
    seq::k_product_few<E, MI, NI><<<dim3((unsigned)tiles), 64 * seq::FEW_WAVES, 0, st>>>(A);
    return true;
}
// The largest tiles of which there are enough for the compute units; below that the outputs are few and K is shared.
// Measured, us, bf16 y (M x N x K: 16 x 16 and 32 x 32 few outputs, tiles of 64, 128, 256):
//   32 x 1024 x 512:     3.3   3.9   4.8   7.1  11.4      64 x 4096 x 4096:  17.1  10.3  13.0  23.9  48.2
//   256 x 1024 x 1024:   6.3   4.8   6.3   9.6  17.4     128 x 4096 x 4096:  31.4  17.5  13.1  23.8  48.3
//   2048 x 1024 x 512:  18.3  11.8   6.8   8.0  12.5    2048 x 2048 x 2048: 117    60.2  18.2  16.9  29.8
//   8192 x 1024 x 512:  62.8  43.3  15.7  11.5  14.7    4096 x 4096 x 2048:     -     -  59.9  41.0  36.0
template <class E> bool launch_product(const seq::ProductArgs &A, hipStream_t st)
{
    auto tiles = [&](int64_t n) { return (A.M + n - 1) / n * ((A.N + n - 1) / n); };
    if (tiles(256) >= 192) return launch_tile<E, 256, 256, 2, 4>(A, st);
    if (tiles(128) >= 192) return launch_tile<E, 128, 128, 2, 2>(A, st);
    if (tiles(64) >= 128) return launch_tile<E, 64, 64, 2, 2>(A, st);
    if (tiles(16) > 512) return launch_few<E, 2, 2>(A, st);
    return launch_few<E, 1, 1>(A, st);
}

const char *check_tensors(const dqn_adamw_tensor *t, int32_t count, int32_t bits)
{
    if (!t || count < 1 || count > 65536) return "count must be in 1..65536, tensors not NULL";
    if (bits != 8 && bits != 32) return "bits must be 8 or 32";
    int64_t sum = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (t[i].n < 0 || t[i].n > (1ll << 38)) return "a tensor's size is out of range";
        sum += (t[i].n + seq::ADAM_BLOCK - 1) / seq::ADAM_BLOCK * seq::ADAM_BLOCK;
        if (sum > (1ll << 38)) return "too many elements";
        if (t[i].n && (!t[i].param || !t[i].grad || !at(t[i].param, 4) || !at(t[i].copy, 2))) return "a tensor's pointer is NULL or not aligned to its elements";
        if (!(t[i].decay >= 0.f) || std::isinf(t[i].decay)) return "decay must be finite and >= 0";
    }
    return nullptr;
}

struct AdamSizes {
    int64_t elements, chunks;
};
AdamSizes adamw_sizes(const dqn_adamw_tensor *t, int32_t count)
{
    AdamSizes s{0, 0};
    for (int32_t i = 0; i < count; ++i) {
        s.elements += (t[i].n + seq::ADAM_BLOCK - 1) / seq::ADAM_BLOCK * seq::ADAM_BLOCK;
        s.chunks += (t[i].n + seq::ADAM_CHUNK - 1) / seq::ADAM_CHUNK;
    }
    return s;
}
size_t plan_bytes(const AdamSizes &s) { return ((size_t)std::max<int64_t>(s.chunks, 1) * sizeof(seq::AdamChunk) + 255) / 256 * 256; }

}  // namespace

extern "C" {

// ------------------------------------------------------------ gated linear recurrence
int32_t dqn_scan_sizes(int32_t dtype, int32_t B, int64_t T, int32_t C, size_t *carry, size_t *workspace)
{
    static const char *call = "dqn_scan_sizes";
    dqn_scan_args s{};
    s.dtype = dtype; s.B = B; s.T = T; s.C = C;
    if (!carry || !workspace) return bad(call, "NULL argument");
    if (const char *m = check_scan(s)) return bad(call, m);
    const ScanCut cut = scan_cut(B, T, C);
    *carry = (size_t)B * cut.tiles * C * 4;
    *workspace = scan_workspace(cut, B, C);
    return DQN_OK;
}

int32_t dqn_scan_forward(const dqn_scan_args *args, void *stream)
{
    static const char *call = "dqn_scan_forward";
    if (!args) return bad(call, "NULL argument");
    const dqn_scan_args &s = *args;
    if (const char *m = check_scan(s)) return bad(call, m);
    if (!s.B || !s.C) return DQN_OK;
    if (s.T) {
        for (const char *m : {check_steps(s.f, s.f_bs, s.f_ts, s, false), check_steps(s.x, s.x_bs, s.x_ts, s, false), check_steps(s.h, s.h_bs, s.h_ts, s, true)})
            if (m) return bad(call, m);
    }
    hipStream_t st = (hipStream_t)stream;
    const ScanCut cut = scan_cut(s.B, s.T, s.C);
    if (scan_workspace(cut, s.B, s.C) && (!s.workspace || !at(s.workspace, 16))) return bad(call, "workspace is NULL or not 16-byte aligned");
    const seq::ScanArgs A{s.f, s.x, s.f_bs, s.f_ts, s.x_bs, s.x_ts, s.h0, s.reset, s.reset_bs, s.reset_ts, s.h, s.h_bs, s.h_ts, s.h_last,
                          s.T ? s.carry : nullptr, s.T, s.B, s.C, cut.tiles, cut.range, cut.ranges, (float *)s.workspace, false,
                          torn_rows({s.f, s.x, s.h}, bytes_of(s.dtype), {s.f_bs, s.f_ts, s.x_bs, s.x_ts, s.h_bs, s.h_ts})};
    auto fits = [&](int n) { return together(n, s.dtype, s.C, {s.f, s.x, s.h}, {s.f_bs, s.f_ts, s.x_bs, s.x_ts, s.h_bs, s.h_ts}, {s.h0, s.h_last, s.carry}); };
    s.dtype == DQN_F32 ? launch_recurrence<float>(A, cut, fits, st) : launch_recurrence<seq::bf16>(A, cut, fits, st);
    return launched(call);
}

int32_t dqn_scan_backward(const dqn_scan_grad_args *args, void *stream)
{
    static const char *call = "dqn_scan_backward";
    if (!args) return bad(call, "NULL argument");
    const dqn_scan_grad_args &g = *args;
    dqn_scan_args s{};
    s.dtype = g.dtype; s.B = g.B; s.T = g.T; s.C = g.C;
    s.reset = g.reset; s.reset_bs = g.reset_bs; s.reset_ts = g.reset_ts;
    if (const char *m = check_scan(s)) return bad(call, m);
    if (!at(g.carry, 4) || !at(g.dlast, 4) || !at(g.dh0, 4)) return bad(call, "a state is not aligned to its elements");
    if (!s.B || !s.C) return DQN_OK;
    if (s.T) {
        if (!g.carry) return bad(call, "carry is NULL");
        for (const char *m : {check_steps(g.f, g.f_bs, g.f_ts, s, false), check_steps(g.x, g.x_bs, g.x_ts, s, false), check_steps(g.dh, g.dh_bs, g.dh_ts, s, false),
                              check_steps(g.df, g.df_bs, g.df_ts, s, true), check_steps(g.dx, g.dx_bs, g.dx_ts, s, true)})
            if (m) return bad(call, m);
    }
    hipStream_t st = (hipStream_t)stream;
    const ScanCut cut = scan_cut(s.B, s.T, s.C);
    if (scan_workspace(cut, s.B, s.C) && (!g.workspace || !at(g.workspace, 16))) return bad(call, "workspace is NULL or not 16-byte aligned");
    const seq::ScanGradArgs A{g.f, g.x, g.dh, g.f_bs, g.f_ts, g.x_bs, g.x_ts, g.dh_bs, g.dh_ts, g.carry, g.dlast, g.reset, g.reset_bs, g.reset_ts,
                              g.df, g.dx, g.df_bs, g.df_ts, g.dx_bs, g.dx_ts, g.dh0, g.T, g.B, g.C, cut.tiles, cut.range, cut.ranges, (float *)g.workspace, false,
                              torn_rows({g.f, g.x, g.dh, g.df, g.dx}, bytes_of(g.dtype),
                                        {g.f_bs, g.f_ts, g.x_bs, g.x_ts, g.dh_bs, g.dh_ts, g.df_bs, g.df_ts, g.dx_bs, g.dx_ts})};
    auto fits = [&](int n) {
        return together(n, g.dtype, g.C, {g.f, g.x, g.dh, g.df, g.dx}, {g.f_bs, g.f_ts, g.x_bs, g.x_ts, g.dh_bs, g.dh_ts, g.df_bs, g.df_ts, g.dx_bs, g.dx_ts},
                        {g.carry, g.dlast, g.dh0});
    };
    s.dtype == DQN_F32 ? launch_recurrence<float>(A, cut, fits, st) : launch_recurrence<seq::bf16>(A, cut, fits, st);
    return launched(call);
}

// ------------------------------------------------------------ norm, rows of 8-bit numbers
int32_t dqn_norm_sizes(int64_t M, int32_t C, size_t *workspace)
{
    static const char *call = "dqn_norm_sizes";
    if (!workspace) return bad(call, "NULL argument");
    if (M < 0 || M > INT32_MAX || C < 1 || C > DQN_NORM_MAX) return bad(call, "M must be in 0..2^31-1, C in 1..DQN_NORM_MAX");
    *workspace = (size_t)norm_parts(M, C) * C * 4;
    return DQN_OK;
}

int32_t dqn_norm_forward(const dqn_norm_args *args, void *stream)
{
    static const char *call = "dqn_norm_forward";
    if (!args) return bad(call, "NULL argument");
    const dqn_norm_args &n = *args;
    if (!dtype_ok(n.dtype)) return bad(call, "dtype must be DQN_F32 or DQN_BF16");
    if (n.M < 0 || n.M > INT32_MAX || n.C < 1 || n.C > DQN_NORM_MAX) return bad(call, "M must be in 0..2^31-1, C in 1..DQN_NORM_MAX");
    if (!(n.eps >= 0.f) || std::isinf(n.eps)) return bad(call, "eps must be finite and >= 0");
    if (!n.M) return DQN_OK;
    if (!n.y == !n.q) return bad(call, "one of y and q must be given");
    if (!n.weight || !at(n.weight, 4) || !at(n.rstd, 4)) return bad(call, "weight is NULL or a pointer is not aligned to its elements");
    for (const char *m : {check_rows(n.x, n.x_rs, n.M, n.C, n.dtype, false), n.residual ? check_rows(n.residual, n.residual_rs, n.M, n.C, n.dtype, false) : nullptr,
                          n.r ? check_rows(n.r, n.r_rs, n.M, n.C, n.dtype, true) : nullptr, n.y ? check_rows(n.y, n.y_rs, n.M, n.C, n.dtype, true) : nullptr,
                          n.q ? check_rows8(n.q, n.q_rs, n.M, n.C) : nullptr})
        if (m) return bad(call, m);
    if (n.q && (!n.scale || !at(n.scale, 4))) return bad(call, "scale is NULL or not aligned to its elements");
    const seq::NormArgs A{n.x, n.residual, n.x_rs, n.residual_rs, n.weight, n.eps, n.r, n.y, n.r_rs, n.y_rs, n.q, n.q_rs, n.scale, n.rstd, n.M, n.C, 0};
    hipStream_t st = (hipStream_t)stream;
    if (n.dtype == DQN_F32) n.q ? launch_norm<float, true>(A, st) : launch_norm<float, false>(A, st);
    else n.q ? launch_norm<seq::bf16, true>(A, st) : launch_norm<seq::bf16, false>(A, st);
    return launched(call);
}

int32_t dqn_norm_backward(const dqn_norm_grad_args *args, void *stream)
{
    static const char *call = "dqn_norm_backward";
    if (!args) return bad(call, "NULL argument");
    const dqn_norm_grad_args &n = *args;
    if (!dtype_ok(n.dtype)) return bad(call, "dtype must be DQN_F32 or DQN_BF16");
    if (n.M < 0 || n.M > INT32_MAX || n.C < 1 || n.C > DQN_NORM_MAX) return bad(call, "M must be in 0..2^31-1, C in 1..DQN_NORM_MAX");
    if (!n.dw || !at(n.dw, 4)) return bad(call, "dw is NULL or not aligned to its elements");
    hipStream_t st = (hipStream_t)stream;
    const int parts = norm_parts(n.M, n.C);
    if (n.M) {
        if (!n.weight || !n.rstd || !at(n.weight, 4) || !at(n.rstd, 4)) return bad(call, "weight or rstd is NULL or not aligned to its elements");
        if (!n.workspace || !at(n.workspace, 16)) return bad(call, "workspace is NULL or not 16-byte aligned");
        for (const char *m : {check_rows(n.dy, n.dy_rs, n.M, n.C, n.dtype, false), check_rows(n.x, n.x_rs, n.M, n.C, n.dtype, false),
                              n.residual ? check_rows(n.residual, n.residual_rs, n.M, n.C, n.dtype, false) : nullptr,
                              n.dr ? check_rows(n.dr, n.dr_rs, n.M, n.C, n.dtype, false) : nullptr, check_rows(n.dx, n.dx_rs, n.M, n.C, n.dtype, true)})
            if (m) return bad(call, m);
        const seq::NormGradArgs A{n.dy, n.x, n.residual, n.dr, n.dy_rs, n.x_rs, n.residual_rs, n.dr_rs, n.weight, n.rstd, n.dx, n.dx_rs, n.dw, (float *)n.workspace, n.M, n.C, 0};
        if (n.dtype == DQN_F32) launch_norm_grad<float>(A, parts, st);
        else launch_norm_grad<seq::bf16>(A, parts, st);
    }
    seq::k_norm_grad_join<<<dim3((unsigned)((n.C + 15) / 16)), 1024, 0, st>>>((const float *)n.workspace, parts, n.C, n.dw);
    return launched(call);
}

int32_t dqn_rows_quantize(int32_t dtype, int64_t M, int32_t K, const void *x, int64_t x_rs, uint8_t *q, int64_t q_rs, float *scale, void *stream)
{
    static const char *call = "dqn_rows_quantize";
    if (!dtype_ok(dtype)) return bad(call, "dtype must be DQN_F32 or DQN_BF16");
    if (M < 0 || M > INT32_MAX || K < 1 || K > DQN_NORM_MAX) return bad(call, "M must be in 0..2^31-1, K in 1..DQN_NORM_MAX");
    if (!M) return DQN_OK;
    if (!scale || !at(scale, 4)) return bad(call, "scale is NULL or not aligned to its elements");
    for (const char *m : {check_rows(x, x_rs, M, K, dtype, false), check_rows8(q, q_rs, M, K)})
        if (m) return bad(call, m);
    const seq::NormArgs A{x, nullptr, x_rs, 0, nullptr, 0.f, nullptr, nullptr, 0, 0, q, q_rs, scale, nullptr, M, K, 0};
    if (dtype == DQN_F32) launch_norm<float, true>(A, (hipStream_t)stream);
    else launch_norm<seq::bf16, true>(A, (hipStream_t)stream);
    return launched(call);
}

// ------------------------------------------------------------ product of 8-bit rows
int32_t dqn_rows_product(const dqn_product_args *args, void *stream)
{
    static const char *call = "dqn_rows_product";
    if (!args) return bad(call, "NULL argument");
    const dqn_product_args &p = *args;
    if (!dtype_ok(p.dtype)) return bad(call, "dtype must be DQN_F32 or DQN_BF16");
    if (p.M < 0 || p.N < 0 || p.K < 0 || p.M > INT32_MAX - 1024 || p.N > (1 << 20) || p.K > (1 << 24)) return bad(call, "M must be in 0..2^31-1025, N in 0..2^20, K in 0..2^24");
    if ((p.M + 255) / 256 * ((p.N + 255) / 256) > 1 << 22) return bad(call, "ceil(M / 256) times ceil(N / 256) must be at most 2^22");
    if (!p.M || !p.N) return DQN_OK;
    for (const char *m : {p.K ? check_rows8(p.a, p.a_rs, p.M, p.K) : nullptr, p.K ? check_rows8(p.w, p.w_rs, p.N, p.K) : nullptr,
                          check_rows(p.y, p.y_rs, p.M, p.N, p.dtype, true)})
        if (m) return bad(call, m);
    if (!p.a_scale || !p.w_scale || !at(p.a_scale, 4) || !at(p.w_scale, 4) || !at(p.bias, 4)) return bad(call, "a scale is NULL or a pointer is not aligned to its elements");
    hipStream_t st = (hipStream_t)stream;
    const seq::ProductArgs A{p.a, p.w, p.a_rs, p.w_rs, p.a_scale, p.w_scale, p.bias, p.y, p.y_rs, p.M, p.N, p.K,
                             p.dtype == DQN_BF16 && p.y_rs % 8 == 0 && at(p.y, 16) ? 8 : p.y_rs % 4 == 0 && at(p.y, 4 * bytes_of(p.dtype)) ? 4 : 1};
    const bool ok = p.dtype == DQN_F32 ? launch_product<float>(A, st) : launch_product<seq::bf16>(A, st);
    return ok ? launched(call) : dqn_seq_fail(DQN_ERR_HIP, call, "the LDS of a tile was not granted");
}

// ------------------------------------------------------------ AdamW
int32_t dqn_adamw_sizes(const dqn_adamw_tensor *tensors, int32_t count, int32_t bits, dqn_adamw_bytes *out)
{
    static const char *call = "dqn_adamw_sizes";
    if (!out) return bad(call, "NULL argument");
    if (const char *m = check_tensors(tensors, count, bits)) return bad(call, m);
    const AdamSizes s = adamw_sizes(tensors, count);
    *out = dqn_adamw_bytes{};
    out->elements = s.elements;
    out->m = out->v = (size_t)s.elements * (bits / 8);
    out->m_scale = out->v_scale = bits == 8 ? (size_t)s.elements / seq::ADAM_BLOCK * 4 : 0;
    out->plan = plan_bytes(s);
    return DQN_OK;
}

int32_t dqn_adamw_init(dqn_adamw **out, const dqn_adamw_tensor *tensors, int32_t count, int32_t bits, int32_t grad_dtype,
                       const dqn_adamw_buffers *bufs, void *stream)
{
    static const char *call = "dqn_adamw_init";
    if (!out || !bufs) return bad(call, "NULL argument");
    *out = nullptr;
    if (const char *m = check_tensors(tensors, count, bits)) return bad(call, m);
    if (!dtype_ok(grad_dtype)) return bad(call, "grad_dtype must be DQN_F32 or DQN_BF16");
    const AdamSizes s = adamw_sizes(tensors, count);
    for (const void *p : {(const void *)bufs->plan, s.elements ? (const void *)bufs->m : bufs->plan, s.elements ? (const void *)bufs->v : bufs->plan,
                          s.elements && bits == 8 ? (const void *)bufs->m_scale : bufs->plan, s.elements && bits == 8 ? (const void *)bufs->v_scale : bufs->plan})
        if (!p || !at(p, 256)) return bad(call, "a buffer is NULL or not 256-byte aligned");
    for (int32_t i = 0; i < count; ++i)
        if (tensors[i].n && !at(tensors[i].grad, bytes_of(grad_dtype))) return bad(call, "a gradient is not aligned to its elements");
    if (s.chunks >= 1 << 24) return bad(call, "too many elements");   // a launch has 2^32 threads
    dqn_adamw *o = nullptr;
    try {
        std::vector<uint8_t> table(plan_bytes(s), 0);
        seq::AdamChunk *c = reinterpret_cast<seq::AdamChunk *>(table.data());
        int64_t place = 0;
        for (int32_t i = 0; i < count; ++i) {
            const dqn_adamw_tensor &u = tensors[i];
            const bool wide = at(u.param, 16) && at(u.grad, 4 * bytes_of(grad_dtype)) && at(u.copy, 8);
            for (int64_t k = 0; k < u.n; k += seq::ADAM_CHUNK)
                *c++ = seq::AdamChunk{u.param + k, (const uint8_t *)u.grad + k * bytes_of(grad_dtype), u.copy ? u.copy + k : nullptr, (long)(place + k),
                                      (int)std::min<int64_t>(seq::ADAM_CHUNK, u.n - k), u.decay, wide, 0};
            place += (u.n + seq::ADAM_BLOCK - 1) / seq::ADAM_BLOCK * seq::ADAM_BLOCK;
        }
        hipStream_t st = (hipStream_t)stream;
        if (hipMemcpyAsync(bufs->plan, table.data(), table.size(), hipMemcpyHostToDevice, st) != hipSuccess || hipStreamSynchronize(st) != hipSuccess) {
            (void)hipGetLastError();
            return dqn_seq_fail(DQN_ERR_HIP, call, "copying the table of tensors failed");
        }
        o = new dqn_adamw{};
    } catch (...) {
        return dqn_seq_fail(DQN_ERR_OOM, call, "out of host memory");
    }
    o->args.chunks = (const seq::AdamChunk *)bufs->plan;
    o->args.m = bufs->m; o->args.v = bufs->v; o->args.ms = bufs->m_scale; o->args.vs = bufs->v_scale;
    o->chunks = s.chunks; o->bits = bits; o->grad_dtype = grad_dtype;
    *out = o;
    return DQN_OK;
}

int32_t dqn_adamw_step(dqn_adamw *opt, double lr, double beta_m, double beta_v, double eps, int64_t step, uint64_t seed, void *stream)
{
    static const char *call = "dqn_adamw_step";
    if (!opt) return bad(call, "NULL argument");
    if (!(lr >= 0.0) || lr > 1e30 || !(eps >= 1e-30) || eps > 1e30) return bad(call, "lr in 0..1e30 and eps in 1e-30..1e30 required");
    if (!(beta_m >= 0.0 && beta_m < 1.0 && beta_v >= 0.0 && beta_v < 1.0)) return bad(call, "beta_m and beta_v must be in [0, 1)");
    if (step < 1) return bad(call, "step must be >= 1");
    if (!opt->chunks) return DQN_OK;
    seq::AdamArgs A = opt->args;
    // doubles: 1 - b of the float next to 0.999 is 1.3e-5 off
    A.lr = (float)lr; A.b1 = (float)beta_m; A.c1 = (float)(1.0 - beta_m); A.b2 = (float)beta_v; A.c2 = (float)(1.0 - beta_v); A.eps = (float)eps;
    A.rate = (float)(lr / (1.0 - std::pow(beta_m, (double)step)));
    A.root = (float)(1.0 / std::sqrt(1.0 - std::pow(beta_v, (double)step)));
    A.seed = seed;
    const dim3 grid((unsigned)opt->chunks);
    hipStream_t st = (hipStream_t)stream;
    if (opt->grad_dtype == DQN_F32) {
        if (opt->bits == 8) seq::k_adamw<float, 8><<<grid, 256, 0, st>>>(A);
        else seq::k_adamw<float, 32><<<grid, 256, 0, st>>>(A);
    } else {
        if (opt->bits == 8) seq::k_adamw<seq::bf16, 8><<<grid, 256, 0, st>>>(A);
        else seq::k_adamw<seq::bf16, 32><<<grid, 256, 0, st>>>(A);
    }
    return launched(call);
}

int32_t dqn_adamw_destroy(dqn_adamw *opt)
{
    delete opt;
    return DQN_OK;
}

}  // extern "C"
