// C ABI of the gated delta rule (see include/dqn.h): checks of arguments and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <type_traits>
#include <utility>

#include "../../include/dqn.h"
#include "checks.h"
#include "delta.h"

namespace {

// A tensor [B][T][H][D]: for one that is read any strides, for one that is written none that put an element in two places.  Where a size is 1
// its stride is not taken.
const char *check_heads(const void *p, const int64_t (&stride)[3], int64_t B, int64_t T, int64_t H, int64_t D, int32_t dtype, bool written)
{
    if (!p || !at(p, bytes_of(dtype))) return "a tensor is NULL or not aligned to its elements";
    std::pair<int64_t, int64_t> by[3] = {{stride[0], B}, {stride[1], T}, {stride[2], H}};
    for (auto &d : by) {
        if (d.second == 1) d.first = 0;
        else if (d.first < 0 || d.first > MOST || (d.first > 0 && d.second - 1 > MOST / d.first)) return "a stride is negative or too large";
    }
    if (by[1].first > 1 << 24) return "a stride from step to step is above 2^24";      // 32 steps are within 2^32 bytes
    if (!written) return nullptr;
    std::sort(by, by + 3);
    int64_t extent = D;
    for (const auto &d : by)
        if (d.second > 1) {
            if (d.first < extent) return "rows of an output lie on top of each other";
            extent = (d.second - 1) * d.first + extent;
        }
    return nullptr;
}

struct DeltaSizes {
    int32_t dtype, B, H, Dk, Dv;
    int64_t T;
};
int64_t tiles_of(int64_t T) { return (T + seq::CH - 1) / seq::CH; }
// Keys of 33 to 64 elements cost what 64 cost, of 65 to 128 what 128 cost: their rows are padded in LDS and registers.
int width_of(int32_t Dk) { return Dk <= 32 ? 32 : Dk <= 64 ? 64 : 128; }

const char *check_sizes(const DeltaSizes &s)
{
    if (!dtype_ok(s.dtype)) return "dtype must be DQN_F32 or DQN_BF16";
    if (s.B < 0 || s.H < 0 || s.B > 65535 || s.H > 65535 || (int64_t)s.B * s.H > 1 << 20) return "B and H must be in 0..65535, B H in 0..2^20";
    if (s.Dk < 1 || s.Dv < 1 || s.Dk > DQN_DELTA_MAX || s.Dv > DQN_DELTA_MAX) return "Dk and Dv must be in 1..DQN_DELTA_MAX";
    if (s.T < 0 || s.T > 1ll << 32 || (int64_t)s.B * s.H * tiles_of(s.T) > 1ll << 24) return "T must be >= 0 and B H ceil(T / 32) at most 2^24";
    return nullptr;
}
const char *check_reset(const uint8_t *reset, int64_t bs, int64_t ts, int64_t B, int64_t T)
{
    if (!reset) return nullptr;
    return bs < 0 || ts < 0 || bs > MOST || ts > MOST || (bs > 0 && B - 1 > MOST / bs) || (ts > 0 && T - 1 > MOST / ts) ? "a stride of reset is negative or too large" : nullptr;
}
seq::Strides strides(const int64_t (&s)[3]) { return seq::Strides{(long)s[0], (long)s[1], (long)s[2]}; }
// whether rows of q and k can be read 16 bytes at a time
bool wide_rows(int32_t dtype, int32_t Dk, std::initializer_list<const void *> tensors, std::initializer_list<const int64_t *> strides)
{
    const int n = 16 / (int)bytes_of(dtype);
    if (Dk % n) return false;
    for (const void *p : tensors)
        if (!at(p, 16)) return false;
    for (const int64_t *s : strides)
        if (s[0] % n || s[1] % n || s[2] % n) return false;
    return true;
}
template <class Args> seq::DeltaIn inputs(const Args &d)      // what both directions read
{
    return seq::DeltaIn{d.q, d.k, d.v, d.f, d.b, strides(d.q_s), strides(d.k_s), strides(d.v_s), strides(d.f_s), strides(d.b_s), d.reset, (long)d.reset_bs, (long)d.reset_ts,
                        (long)d.T, (long)tiles_of(d.T), d.B, d.H, d.Dk, d.Dv, d.scale, wide_rows(d.dtype, d.Dk, {d.q, d.k}, {d.q_s, d.k_s})};
}

// go(E, DK): the type of the activations and the width that holds Dk
template <int N> using Int = std::integral_constant<int, N>;
template <class F> bool delta_form(int32_t dtype, int32_t Dk, F &&go)
{
    auto wide = [&](auto e) { return width_of(Dk) == 32 ? go(e, Int<32>{}) : width_of(Dk) == 64 ? go(e, Int<64>{}) : go(e, Int<128>{}); };
    return dtype == DQN_F32 ? wide(float{}) : wide(seq::bf16{});
}
size_t record_bytes(const DeltaSizes &s) { return (size_t)s.B * s.H * tiles_of(s.T) * sizeof(seq::DeltaRecord); }
// a state for each tile, padded as the kernels hold them
size_t state_bytes(const DeltaSizes &s) { return (size_t)s.B * s.H * tiles_of(s.T) * width_of(s.Dk) * ((s.Dv + 15) / 16 * 16) * 4; }

// Ranges of a head's tiles, where there are fewer workgroups of a chain than compute units.  All of its tiles are gone through three times then
// (the maps take as many columns again), so that fewer than four ranges would not pay.  Measured (bf16, 64 x 64, forward / backward): 4 ranges
// (64 heads of 4096 steps) 171 / 376 us, one 257 / 403; 3 (85 heads) 227 / 502, one 268 / 478; 2 (128 heads) 339 / 727, one 302 / 615.  Ranges of
// 4 tiles (4 heads of 1024 steps) 38 / 44 us, of 8 49 / 52, one 68 / 65; of 2 tiles, which makes 64 of them at 4096 steps, 55 / 71 for 53 / 67.
constexpr int64_t UNITS = 256, LEAST_TILES = 4, LEAST_RANGES = 4;
template <class E, int DK> seq::DeltaRanges ranges_of(int64_t heads, int64_t tiles, int Dv)
{
    constexpr int waves = seq::DeltaChain<E, DK>::WAVES;
    const int64_t groups = heads * (((Dv + 15) / 16 + waves - 1) / waves);
    const int64_t n = groups ? std::min({UNITS / groups, tiles / LEAST_TILES, (int64_t)seq::MOST_RANGES}) : 1;
    seq::DeltaRanges R{1, (long)tiles, nullptr, nullptr, nullptr, nullptr};
    if (n < LEAST_RANGES) return R;
    R.per = (long)((tiles + n - 1) / n);
    R.ranges = (int)((tiles + R.per - 1) / R.per);
    return R;
}
// Ranges are joined in groups of 8 where there are many, which takes two launches more: 64 of them (8192 steps, one head of 64 in fp32) 86 / 97 us at once,
// 62 / 72 so; 32 (4096 steps, four heads of 128 in bf16) 124 / 168 and 97 / 142; 20 (2560 steps, two of 64) 46 / 53 and 47 / 54; 16 are slower in groups.
constexpr int LEAST_JOINED = 24, JOINED = 8;
int span_of(int ranges) { return ranges < LEAST_JOINED ? ranges : JOINED; }
seq::DeltaRanges groups_of(const seq::DeltaRanges &R)
{
    const int span = span_of(R.ranges);
    return seq::DeltaRanges{(R.ranges + span - 1) / span, R.per * span, nullptr, nullptr, nullptr, nullptr};
}
size_t range_bytes(const seq::DeltaRanges &R, int64_t heads, int width, int64_t size)
{
    return R.ranges == 1 ? 0 : ((size_t)heads * R.ranges * ((size_t)width * width + 2 * (size_t)size) * 4 + 15) / 16 * 16;
}
size_t ranges_workspace(const DeltaSizes &s)
{
    size_t n = 0;
    delta_form(s.dtype, s.Dk, [&](auto e, auto dk) { const int64_t heads = (int64_t)s.B * s.H, size = (int64_t)s.Dk * s.Dv;
        const seq::DeltaRanges R = ranges_of<decltype(e), dk.value>(heads, tiles_of(s.T), s.Dv);
        n = range_bytes(R, heads, dk.value, size) + range_bytes(groups_of(R), heads, dk.value, size);
        return true;
    });
    return n;
}
// What a forward call keeps of the ranges' maps for a backward call.
size_t map_bytes(const DeltaSizes &s)
{
    size_t n = 0;
    delta_form(s.dtype, s.Dk, [&](auto e, auto dk) {
        const int ranges = ranges_of<decltype(e), dk.value>((int64_t)s.B * s.H, tiles_of(s.T), s.Dv).ranges;
        n = ranges == 1 ? 0 : (size_t)s.B * s.H * ranges * dk.value * dk.value * 4;
        return true;
    });
    return n;
}
template <int DK> void place(seq::DeltaRanges &R, const seq::DeltaIn &A, void *workspace)
{
    const int64_t n = (int64_t)A.B * A.H * R.ranges, size = (int64_t)A.Dk * A.Dv;
    R.m = (float *)workspace;
    R.b = R.m + n * DK * DK;
    R.first = R.b + n * size;
}
template <class E, int DK> seq::DeltaRanges ranges_at(const seq::DeltaIn &A, void *workspace)
{
    seq::DeltaRanges R = ranges_of<E, DK>((int64_t)A.B * A.H, A.tiles, A.Dv);
    place<DK>(R, A, workspace);
    return R;
}
// The states that ranges begin with, from their maps.
template <int DK, bool BACK> void launch_join(const seq::DeltaRanges &R, const seq::DeltaIn &A, const float *given, const seq::DeltaRecord *records, void *workspace, hipStream_t st)
{
    const int64_t heads = (int64_t)A.B * A.H;
    const unsigned blocks = (unsigned)((A.Dv + 15) / 16);
    const int span = span_of(R.ranges);
    auto join = [&](const seq::DeltaRanges &r, int n, const float *from) {
        seq::k_delta_join<DK, BACK, false><<<dim3((unsigned)heads * ((r.ranges + n - 1) / n) * blocks), 8 * DK, 0, st>>>(r, n, from, r, records, A.tiles, A.Dk, A.Dv);
    };
    if (span == R.ranges) return join(R, span, given);
    seq::DeltaRanges G = groups_of(R);
    place<DK>(G, A, (uint8_t *)workspace + range_bytes(R, heads, DK, (int64_t)A.Dk * A.Dv));
    seq::k_delta_join<DK, BACK, true><<<dim3((unsigned)heads * G.ranges * (blocks + DK / 16)), 4 * DK, 0, st>>>(R, span, nullptr, G, records, A.tiles, A.Dk, A.Dv);
    join(G, G.ranges, given);
    join(R, span, G.first);
}
template <class Chain, int DK> unsigned chain_groups(const seq::DeltaIn &A, const seq::DeltaRanges &R, bool maps)
{
    constexpr int waves = Chain::WAVES;
    return (unsigned)((int64_t)A.B * A.H * R.ranges * (((A.Dv + 15) / 16 + (maps ? DK / 16 : 0) + waves - 1) / waves));
}
template <class E, int DK> bool launch_delta(const seq::DeltaArgs &A, void *workspace, float *maps, hipStream_t st)
{
    static std::atomic<uint64_t> granted{0}, maps_granted{0};
    using Chain = seq::DeltaChain<E, DK>;
    using Maps = seq::DeltaMaps<E, DK>;
    constexpr int bytes = sizeof(Chain), maps_bytes = sizeof(Maps);
    static_assert(bytes <= 160 * 1024 && maps_bytes <= 80 * 1024, "one and two within a compute unit's LDS");
    if (!lds_granted((const void *)seq::k_delta<E, DK, false>, bytes, granted) || !lds_granted((const void *)seq::k_delta<E, DK, true>, maps_bytes, maps_granted)) return false;
    const int64_t heads = (int64_t)A.B * A.H;
    if (A.T <= seq::STEPS_MOST && !A.states) {
        seq::k_delta_few<E, DK><<<dim3((unsigned)((heads * ((A.Dv + 15) / 16) + 3) / 4)), 256, 0, st>>>(A);
        return true;
    }
    if (A.tiles) seq::k_delta_tiles<E, DK><<<dim3((unsigned)((heads * A.tiles + 3) / 4)), 256, 0, st>>>(A, (seq::DeltaRecord *)A.records);
    seq::DeltaRanges R = ranges_at<E, DK>(A, workspace);
    R.turned = maps;
    if (R.ranges > 1) {
        seq::k_delta<E, DK, true><<<dim3(chain_groups<Maps, DK>(A, R, true)), seq::threads_of<Maps>, maps_bytes, st>>>(A, R);
        launch_join<DK, false>(R, A, A.s0, (const seq::DeltaRecord *)A.records, workspace, st);
    }
    seq::k_delta<E, DK, false><<<dim3(chain_groups<Chain, DK>(A, R, false)), seq::threads_of<Chain>, bytes, st>>>(A, R);
    return true;
}
constexpr int64_t GRAD_GROUPS = 256;     // a workgroup of the gradients per compute unit, which is all that fits; 512 in two turns: 4 % slower
template <class E, int DK> bool launch_delta_grad(const seq::DeltaGradArgs &A, void *workspace, const float *maps, hipStream_t st)
{
    static std::atomic<uint64_t> back_granted{0}, maps_granted{0}, granted{0};
    constexpr int back = sizeof(seq::DeltaChain<E, DK>), threads = seq::threads_of<seq::DeltaChain<E, DK>>, bytes = sizeof(seq::DeltaGradTile<E, DK>);
    static_assert(bytes <= 160 * 1024 && sizeof(seq::DeltaSteps<E, DK>) <= 65536, "within what a workgroup can have");
    if (!lds_granted((const void *)seq::k_delta_back<E, DK, false>, back, back_granted) || !lds_granted((const void *)seq::k_delta_back<E, DK, true>, back, maps_granted) ||
        !lds_granted((const void *)seq::k_delta_grad<E, DK>, bytes, granted)) return false;
    const int64_t heads = (int64_t)A.B * A.H;
    seq::DeltaRanges R = ranges_at<E, DK>(A, workspace);
    if (R.ranges > 1) {
        R.m = const_cast<float *>(maps);      // read only
        seq::k_delta_back<E, DK, true><<<dim3(chain_groups<seq::DeltaChain<E, DK>, DK>(A, R, false)), threads, back, st>>>(A, R);
        launch_join<DK, true>(R, A, A.dlast, (const seq::DeltaRecord *)A.records, workspace, st);
    }
    seq::k_delta_back<E, DK, false><<<dim3(chain_groups<seq::DeltaChain<E, DK>, DK>(A, R, false)), threads, back, st>>>(A, R);
    if (!A.tiles) return true;
    const int64_t all = heads * A.tiles, per = std::max<int64_t>(1, (all + GRAD_GROUPS - 1) / GRAD_GROUPS);
    seq::k_delta_grad<E, DK><<<dim3((unsigned)((all + per - 1) / per)), 512, bytes, st>>>(A, (int)per);
    seq::k_delta_grad_steps<E, DK><<<dim3((unsigned)((all + seq::AGAIN - 1) / seq::AGAIN)), 256, sizeof(seq::DeltaSteps<E, DK>), st>>>(A);
    return true;
}

}  // namespace

extern "C" {

int32_t dqn_delta_sizes(int32_t dtype, int32_t B, int64_t T, int32_t H, int32_t Dk, int32_t Dv, size_t *carry,
                        size_t *forward_workspace, size_t *backward_workspace)
{
    static const char *call = "dqn_delta_sizes";
    const DeltaSizes s{dtype, B, H, Dk, Dv, T};
    if (!carry || !forward_workspace || !backward_workspace) return bad(call, "NULL argument");
    if (const char *m = check_sizes(s)) return bad(call, m);
    *carry = state_bytes(s) + record_bytes(s) + map_bytes(s);
    *forward_workspace = ranges_workspace(s) + record_bytes(s);      // the records lie in `carry` if there is one
    *backward_workspace = ranges_workspace(s) + state_bytes(s) + (size_t)B * H * tiles_of(T) * 4;
    return DQN_OK;
}

int32_t dqn_delta_forward(const dqn_delta_args *args, void *stream)
{
    static const char *call = "dqn_delta_forward";
    if (!args) return bad(call, "NULL argument");
    const dqn_delta_args &d = *args;
    const DeltaSizes s{d.dtype, d.B, d.H, d.Dk, d.Dv, d.T};
    if (const char *m = check_sizes(s)) return bad(call, m);
    if (const char *m = check_reset(d.reset, d.reset_bs, d.reset_ts, d.B, d.T)) return bad(call, m);
    if (!at(d.s0, 4) || !at(d.s_last, 4) || !at(d.carry, 16)) return bad(call, "a state is not aligned to its elements, or carry to 16 bytes");
    if (!std::isfinite(d.scale)) return bad(call, "scale must be finite");
    if (!d.B || !d.H) return DQN_OK;
    if (d.T && (!d.workspace || !at(d.workspace, 16))) return bad(call, "workspace is NULL or not 16-byte aligned");
    if (d.T)
        for (const char *m : {check_heads(d.q, d.q_s, d.B, d.T, d.H, d.Dk, d.dtype, false), check_heads(d.k, d.k_s, d.B, d.T, d.H, d.Dk, d.dtype, false),
                              check_heads(d.v, d.v_s, d.B, d.T, d.H, d.Dv, d.dtype, false), check_heads(d.f, d.f_s, d.B, d.T, d.H, 1, d.dtype, false),
                              check_heads(d.b, d.b_s, d.B, d.T, d.H, 1, d.dtype, false), check_heads(d.o, d.o_s, d.B, d.T, d.H, d.Dv, d.dtype, true)})
            if (m) return bad(call, m);
    float *records = (float *)(d.carry ? (uint8_t *)d.carry + state_bytes(s) : (uint8_t *)d.workspace + ranges_workspace(s));
    float *maps = d.carry ? (float *)((uint8_t *)d.carry + state_bytes(s) + record_bytes(s)) : nullptr;
    seq::DeltaArgs A{};
    static_cast<seq::DeltaIn &>(A) = inputs(d);
    A.s0 = d.s0; A.o = d.o; A.so = strides(d.o_s); A.last = d.s_last; A.states = d.carry; A.records = records;
    hipStream_t st = (hipStream_t)stream;
    const bool ok = delta_form(d.dtype, d.Dk, [&](auto e, auto dk) { return launch_delta<decltype(e), dk.value>(A, d.workspace, maps, st); });
    return ok ? launched(call) : dqn_seq_fail(DQN_ERR_HIP, call, "the LDS of a tile was not granted");
}

int32_t dqn_delta_backward(const dqn_delta_grad_args *args, void *stream)
{
    static const char *call = "dqn_delta_backward";
    if (!args) return bad(call, "NULL argument");
    const dqn_delta_grad_args &d = *args;
    const DeltaSizes s{d.dtype, d.B, d.H, d.Dk, d.Dv, d.T};
    if (const char *m = check_sizes(s)) return bad(call, m);
    if (const char *m = check_reset(d.reset, d.reset_bs, d.reset_ts, d.B, d.T)) return bad(call, m);
    if (!at(d.carry, 16) || !at(d.dlast, 4) || !at(d.ds0, 4)) return bad(call, "a state is not aligned to its elements, or carry to 16 bytes");
    if (!std::isfinite(d.scale)) return bad(call, "scale must be finite");
    if (!d.B || !d.H) return DQN_OK;
    if (d.T) {
        if (!d.carry) return bad(call, "carry is NULL");
        if (!d.workspace || !at(d.workspace, 16)) return bad(call, "workspace is NULL or not 16-byte aligned");
        for (const char *m : {check_heads(d.q, d.q_s, d.B, d.T, d.H, d.Dk, d.dtype, false), check_heads(d.k, d.k_s, d.B, d.T, d.H, d.Dk, d.dtype, false),
                              check_heads(d.v, d.v_s, d.B, d.T, d.H, d.Dv, d.dtype, false), check_heads(d.f, d.f_s, d.B, d.T, d.H, 1, d.dtype, false),
                              check_heads(d.b, d.b_s, d.B, d.T, d.H, 1, d.dtype, false), check_heads(d.dout, d.dout_s, d.B, d.T, d.H, d.Dv, d.dtype, false),
                              check_heads(d.dq, d.dq_s, d.B, d.T, d.H, d.Dk, d.dtype, true), check_heads(d.dk, d.dk_s, d.B, d.T, d.H, d.Dk, d.dtype, true),
                              check_heads(d.dv, d.dv_s, d.B, d.T, d.H, d.Dv, d.dtype, true), check_heads(d.df, d.df_s, d.B, d.T, d.H, 1, d.dtype, true),
                              check_heads(d.db, d.db_s, d.B, d.T, d.H, 1, d.dtype, true)})
            if (m) return bad(call, m);
    }
    const float *maps = (const float *)((const uint8_t *)d.carry + state_bytes(s) + record_bytes(s));
    seq::DeltaGradArgs A{};
    static_cast<seq::DeltaIn &>(A) = inputs(d);
    A.dout = d.dout; A.sdo = strides(d.dout_s); A.states = d.carry; A.records = (const float *)((const uint8_t *)d.carry + state_bytes(s)); A.dlast = d.dlast;
    A.dq = d.dq; A.dk = d.dk; A.dv = d.dv; A.df = d.df; A.db = d.db;
    A.sdq = strides(d.dq_s); A.sdk = strides(d.dk_s); A.sdv = strides(d.dv_s); A.sdf = strides(d.df_s); A.sdb = strides(d.db_s);
    A.ds0 = d.ds0; A.into = (float *)((uint8_t *)d.workspace + ranges_workspace(s)); A.again = (int *)((uint8_t *)A.into + state_bytes(s));
    hipStream_t st = (hipStream_t)stream;
    const bool ok = delta_form(d.dtype, d.Dk, [&](auto e, auto dk) { return launch_delta_grad<decltype(e), dk.value>(A, d.workspace, maps, st); });
    return ok ? launched(call) : dqn_seq_fail(DQN_ERR_HIP, call, "the LDS of a tile was not granted");
}

}  // extern "C"
