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
int64_t heads_of(const seq::DeltaIn &A) { return (int64_t)A.B * A.H; }
template <class E, int DK> void launch_tiles(const seq::DeltaIn &A, float *records, hipStream_t st)
{
    if (A.tiles) seq::k_delta_tiles<E, DK><<<dim3((unsigned)((heads_of(A) * A.tiles + 3) / 4)), 256, 0, st>>>(A, (seq::DeltaRecord *)records);
}
template <class E, int DK> bool launch_delta(const seq::DeltaArgs &A, hipStream_t st)
{
    static std::atomic<uint64_t> granted{0};
    constexpr int bytes = sizeof(seq::DeltaChain<E, DK>), waves = seq::DeltaChain<E, DK>::WAVES;
    static_assert(bytes <= 160 * 1024, "within a compute unit's LDS");
    if (!lds_granted((const void *)seq::k_delta<E, DK>, bytes, granted)) return false;
    launch_tiles<E, DK>(A, A.records, st);
    seq::k_delta<E, DK><<<dim3((unsigned)(heads_of(A) * ((A.Dv + 16 * waves - 1) / (16 * waves)))), 128 * waves, bytes, st>>>(A);
    return true;
}
constexpr int64_t GRAD_GROUPS = 256;     // a workgroup of the gradients per compute unit
template <class E, int DK> bool launch_delta_grad(const seq::DeltaGradArgs &A, hipStream_t st)
{
    static std::atomic<uint64_t> back_granted{0}, granted{0};
    constexpr int back = sizeof(seq::DeltaChain<E, DK>), waves = seq::DeltaChain<E, DK>::WAVES, bytes = sizeof(seq::DeltaGradTile<E, DK>);
    if (!lds_granted((const void *)seq::k_delta_back<E, DK>, back, back_granted) || !lds_granted((const void *)seq::k_delta_grad<E, DK>, bytes, granted)) return false;
    seq::k_delta_back<E, DK><<<dim3((unsigned)(heads_of(A) * ((A.Dv + 16 * waves - 1) / (16 * waves)))), 128 * waves, back, st>>>(A);
    if (!A.tiles) return true;
    static_assert(sizeof(seq::DeltaSteps<E, DK>) <= 65536, "within what a workgroup gets");
    const int64_t all = heads_of(A) * A.tiles, per = std::max<int64_t>(1, (all + GRAD_GROUPS - 1) / GRAD_GROUPS);
    seq::k_delta_grad<E, DK><<<dim3((unsigned)((all + per - 1) / per)), 512, bytes, st>>>(A, (int)per);
    seq::k_delta_grad_steps<E, DK><<<dim3((unsigned)((heads_of(A) * A.tiles + seq::AGAIN - 1) / seq::AGAIN)), 256, sizeof(seq::DeltaSteps<E, DK>), st>>>(A);
    return true;
}
size_t record_bytes(const DeltaSizes &s) { return (size_t)s.B * s.H * tiles_of(s.T) * sizeof(seq::DeltaRecord); }
// a state for each tile, padded as the kernels hold them
size_t state_bytes(const DeltaSizes &s) { return (size_t)s.B * s.H * tiles_of(s.T) * width_of(s.Dk) * ((s.Dv + 15) / 16 * 16) * 4; }

}  // namespace

extern "C" {

int32_t dqn_delta_sizes(int32_t dtype, int32_t B, int64_t T, int32_t H, int32_t Dk, int32_t Dv, size_t *carry,
                        size_t *forward_workspace, size_t *backward_workspace)
{
    static const char *call = "dqn_delta_sizes";
    const DeltaSizes s{dtype, B, H, Dk, Dv, T};
    if (!carry || !forward_workspace || !backward_workspace) return bad(call, "NULL argument");
    if (const char *m = check_sizes(s)) return bad(call, m);
    *carry = state_bytes(s) + record_bytes(s);
    *forward_workspace = record_bytes(s);
    *backward_workspace = state_bytes(s) + (size_t)B * H * tiles_of(T) * 4;
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
    if (d.T && !d.carry && (!d.workspace || !at(d.workspace, 16))) return bad(call, "workspace is NULL or not 16-byte aligned");
    if (d.T)
        for (const char *m : {check_heads(d.q, d.q_s, d.B, d.T, d.H, d.Dk, d.dtype, false), check_heads(d.k, d.k_s, d.B, d.T, d.H, d.Dk, d.dtype, false),
                              check_heads(d.v, d.v_s, d.B, d.T, d.H, d.Dv, d.dtype, false), check_heads(d.f, d.f_s, d.B, d.T, d.H, 1, d.dtype, false),
                              check_heads(d.b, d.b_s, d.B, d.T, d.H, 1, d.dtype, false), check_heads(d.o, d.o_s, d.B, d.T, d.H, d.Dv, d.dtype, true)})
            if (m) return bad(call, m);
    float *records = (float *)(d.carry ? (uint8_t *)d.carry + state_bytes(s) : (uint8_t *)d.workspace);
    seq::DeltaArgs A{};
    static_cast<seq::DeltaIn &>(A) = inputs(d);
    A.s0 = d.s0; A.o = d.o; A.so = strides(d.o_s); A.last = d.s_last; A.states = d.carry; A.records = records;
    hipStream_t st = (hipStream_t)stream;
    const bool ok = delta_form(d.dtype, d.Dk, [&](auto e, auto dk) { return launch_delta<decltype(e), dk.value>(A, st); });
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
    seq::DeltaGradArgs A{};
    static_cast<seq::DeltaIn &>(A) = inputs(d);
    A.dout = d.dout; A.sdo = strides(d.dout_s); A.states = d.carry; A.records = (const float *)((const uint8_t *)d.carry + state_bytes(s)); A.dlast = d.dlast;
    A.dq = d.dq; A.dk = d.dk; A.dv = d.dv; A.df = d.df; A.db = d.db;
    A.sdq = strides(d.dq_s); A.sdk = strides(d.dk_s); A.sdv = strides(d.dv_s); A.sdf = strides(d.df_s); A.sdb = strides(d.db_s);
    A.ds0 = d.ds0; A.into = (float *)d.workspace; A.again = (int *)((uint8_t *)d.workspace + state_bytes(s));
    hipStream_t st = (hipStream_t)stream;
    const bool ok = delta_form(d.dtype, d.Dk, [&](auto e, auto dk) { return launch_delta_grad<decltype(e), dk.value>(A, st); });
    return ok ? launched(call) : dqn_seq_fail(DQN_ERR_HIP, call, "the LDS of a tile was not granted");
}

}  // extern "C"
