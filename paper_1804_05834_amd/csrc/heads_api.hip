// C ABI of queries and keys per head (see include/dqn.h): checks of arguments and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "../../include/dqn.h"
#include "checks.h"
#include "heads.h"

namespace {

static_assert(DQN_HEADS_MAX == seq::HEADS_MAX, "the widest head");

const char *check_shape(int64_t M, int32_t Hq, int32_t Hk, int32_t D, int32_t R)
{
    if (M < 0 || M > INT32_MAX) return "M must be in 0..2^31-1";
    if (Hq < 0 || Hk < 0 || Hq > 65535 || Hk > 65535) return "Hq and Hk must be in 0..65535";
    if (D < 1 || D > DQN_HEADS_MAX) return "D must be in 1..DQN_HEADS_MAX";
    if (R < 0 || R > D || R % 2) return "R must be even and in 0..D";
    return nullptr;
}

// [M][H][D] with the strides of a row and of a head; an output has no element in two places
const char *check_tensor(const void *p, int64_t rs, int64_t hs, int64_t M, int64_t H, int64_t D, int32_t dtype, bool written)
{
    if (!H) return nullptr;
    if (!p || !at(p, bytes_of(dtype))) return "a tensor is NULL or not aligned to its elements";
    if (M == 1) rs = 0;
    if (H == 1) hs = 0;
    if (rs < 0 || hs < 0 || rs > MOST || hs > MOST || (rs > 0 && M - 1 > MOST / rs) || (hs > 0 && H - 1 > MOST / hs)) return "a stride is negative or too large";
    if (!written) return nullptr;
    const bool apart = (H == 1 || hs >= D) && (M == 1 || rs >= D) && (H == 1 || M == 1 || rs >= (H - 1) * hs + D || hs >= (M - 1) * rs + D);
    return apart ? nullptr : "rows of an output lie on top of each other";
}

const char *fill_turns(const double *turns, int32_t R, uint64_t (&out)[seq::HEADS_MAX / 2])
{
    for (int i = 0; i < R / 2; ++i) {
        if (!std::isfinite(turns[i])) return "turns must be finite";
        const double part = turns[i] - std::floor(turns[i]);      // in [0, 1], 1 where a tiny negative one is rounded
        out[i] = part < 1.0 ? (uint64_t)std::ldexp(part, 64) : 0;
    }
    return nullptr;
}

template <int N> using Int = std::integral_constant<int, N>;
int power_of_two(int n)
{
    int p = 1;
    while (p < n) p *= 2;
    return p;
}

// Units of V elements and their partners; whether V at once are allowed: sizes and strides multiples of V, addresses of 16 bytes.
bool wide(int V, int32_t dtype, const seq::HeadsShape &s, std::initializer_list<const void *> tensors, std::initializer_list<int64_t> strides)
{
    if (s.half % V || s.D % V) return false;
    for (const void *p : tensors)
        if (!at(p, V * bytes_of(dtype))) return false;
    for (int64_t x : strides)
        if (x % V) return false;
    return true;
}
template <class E, class F> void heads_form(bool wide, seq::HeadsShape &s, int64_t waves, F &&go)
{
    constexpr int V = 16 / (int)sizeof(E);
    const int v = wide ? V : 1, units = (s.half + v - 1) / v + (s.D - 2 * s.half + 2 * v - 1) / (2 * v);
    s.lanes = std::min(64, power_of_two(units));
    // groups that share a row: as few as leave `waves` waves, so that angles serve many heads
    const int groups = 64 / s.lanes, most = std::min(groups, power_of_two(std::max(std::max(s.Hq, s.Hk), 1)));
    s.per_row = 1;
    while (s.per_row < most && s.M * s.per_row < waves * groups) s.per_row *= 2;
    if (wide) go(Int<V>{}, Int<1>{});
    else if (units <= 64) go(Int<1>{}, Int<1>{});
    else go(Int<1>{}, Int<2>{});
}
constexpr int64_t WAVES = 4096;     // four per SIMD
int64_t groups_of_rows(const seq::HeadsShape &s) { return (s.M + 256 / s.lanes / s.per_row - 1) / (256 / s.lanes / s.per_row); }

}  // namespace

extern "C" {

int32_t dqn_heads_sizes(int64_t M, int32_t Hq, int32_t Hk, int32_t D, size_t *workspace)
{
    static const char *call = "dqn_heads_sizes";
    if (!workspace) return bad(call, "NULL argument");
    if (const char *m = check_shape(M, Hq, Hk, D, 0)) return bad(call, m);
    *workspace = (size_t)std::min<int64_t>(std::max<int64_t>(M, 1), seq::HEADS_PARTS) * 2 * D * 4;
    return DQN_OK;
}

int32_t dqn_heads_forward(const dqn_heads_args *args, void *stream)
{
    static const char *call = "dqn_heads_forward";
    if (!args) return bad(call, "NULL argument");
    const dqn_heads_args &n = *args;
    if (!dtype_ok(n.dtype)) return bad(call, "dtype must be DQN_F32 or DQN_BF16");
    if (const char *m = check_shape(n.M, n.Hq, n.Hk, n.D, n.R)) return bad(call, m);
    if (!(n.eps >= 0.f) || std::isinf(n.eps)) return bad(call, "eps must be finite and >= 0");
    if (n.R && (!n.turns || (n.M && (!n.position || !at(n.position, 4))))) return bad(call, "R > 0 takes turns and positions");
    if (!at(n.rstd, 4)) return bad(call, "rstd is not aligned to its elements");
    if (!n.M || (!n.Hq && !n.Hk)) return DQN_OK;
    if ((n.Hq && (!n.q_weight || !at(n.q_weight, 4))) || (n.Hk && (!n.k_weight || !at(n.k_weight, 4)))) return bad(call, "a weight is NULL or not aligned to its elements");
    for (const char *m : {check_tensor(n.q, n.q_rs, n.q_hs, n.M, n.Hq, n.D, n.dtype, false), check_tensor(n.k, n.k_rs, n.k_hs, n.M, n.Hk, n.D, n.dtype, false),
                          check_tensor(n.yq, n.yq_rs, n.yq_hs, n.M, n.Hq, n.D, n.dtype, true), check_tensor(n.yk, n.yk_rs, n.yk_hs, n.M, n.Hk, n.D, n.dtype, true)})
        if (m) return bad(call, m);
    seq::HeadsArgs A{n.q, n.k, n.q_rs, n.q_hs, n.k_rs, n.k_hs, n.q_weight, n.k_weight, n.position, n.yq, n.yk, n.yq_rs, n.yq_hs, n.yk_rs, n.yk_hs, n.rstd, n.eps,
                     {(long)n.M, n.Hq, n.Hk, n.D, n.R / 2, 0, 0}, {}};
    if (const char *m = fill_turns(n.turns, n.R, A.turns)) return bad(call, m);
    hipStream_t st = (hipStream_t)stream;
    auto launch = [&](auto e) {
        using E = decltype(e);
        const bool w = wide(16 / (int)sizeof(E), n.dtype, A.s, {n.Hq ? n.q : nullptr, n.Hk ? n.k : nullptr, n.Hq ? n.yq : nullptr, n.Hk ? n.yk : nullptr},
                            {n.q_rs, n.q_hs, n.k_rs, n.k_hs, n.yq_rs, n.yq_hs, n.yk_rs, n.yk_hs});
        heads_form<E>(w, A.s, WAVES, [&](auto V, auto K) {
            seq::k_heads<E, V.value, K.value><<<dim3((unsigned)std::min<int64_t>(groups_of_rows(A.s), 1 << 16)), 256, 0, st>>>(A);
        });
    };
    n.dtype == DQN_F32 ? launch(float{}) : launch(seq::bf16{});
    return launched(call);
}

int32_t dqn_heads_backward(const dqn_heads_grad_args *args, void *stream)
{
    static const char *call = "dqn_heads_backward";
    if (!args) return bad(call, "NULL argument");
    const dqn_heads_grad_args &n = *args;
    if (!dtype_ok(n.dtype)) return bad(call, "dtype must be DQN_F32 or DQN_BF16");
    if (const char *m = check_shape(n.M, n.Hq, n.Hk, n.D, n.R)) return bad(call, m);
    if (n.R && (!n.turns || (n.M && (!n.position || !at(n.position, 4))))) return bad(call, "R > 0 takes turns and positions");
    if ((n.Hq && (!n.dq_weight || !at(n.dq_weight, 4))) || (n.Hk && (!n.dk_weight || !at(n.dk_weight, 4)))) return bad(call, "a weight's gradient is NULL or not aligned to its elements");
    if (!n.Hq && !n.Hk) return DQN_OK;
    hipStream_t st = (hipStream_t)stream;
    int64_t parts = 0;
    if (n.M) {
        if (!n.rstd || !at(n.rstd, 4)) return bad(call, "rstd is NULL or not aligned to its elements");
        if ((n.Hq && (!n.q_weight || !at(n.q_weight, 4))) || (n.Hk && (!n.k_weight || !at(n.k_weight, 4)))) return bad(call, "a weight is NULL or not aligned to its elements");
        if (!n.workspace || !at(n.workspace, 16)) return bad(call, "workspace is NULL or not 16-byte aligned");
        for (const char *m : {check_tensor(n.dyq, n.dyq_rs, n.dyq_hs, n.M, n.Hq, n.D, n.dtype, false), check_tensor(n.dyk, n.dyk_rs, n.dyk_hs, n.M, n.Hk, n.D, n.dtype, false),
                              check_tensor(n.q, n.q_rs, n.q_hs, n.M, n.Hq, n.D, n.dtype, false), check_tensor(n.k, n.k_rs, n.k_hs, n.M, n.Hk, n.D, n.dtype, false),
                              check_tensor(n.dq, n.dq_rs, n.dq_hs, n.M, n.Hq, n.D, n.dtype, true), check_tensor(n.dk, n.dk_rs, n.dk_hs, n.M, n.Hk, n.D, n.dtype, true)})
            if (m) return bad(call, m);
        seq::HeadsGradArgs A{n.dyq, n.dyk, n.q, n.k, n.dyq_rs, n.dyq_hs, n.dyk_rs, n.dyk_hs, n.q_rs, n.q_hs, n.k_rs, n.k_hs, n.q_weight, n.k_weight, n.rstd, n.position,
                             n.dq, n.dk, n.dq_rs, n.dq_hs, n.dk_rs, n.dk_hs, (float *)n.workspace, {(long)n.M, n.Hq, n.Hk, n.D, n.R / 2, 0, 0}, {}};
        if (const char *m = fill_turns(n.turns, n.R, A.turns)) return bad(call, m);
        auto launch = [&](auto e) {
            using E = decltype(e);
            const bool w = wide(16 / (int)sizeof(E), n.dtype, A.s,
                                {n.Hq ? n.dyq : nullptr, n.Hk ? n.dyk : nullptr, n.Hq ? n.q : nullptr, n.Hk ? n.k : nullptr, n.Hq ? n.dq : nullptr, n.Hk ? n.dk : nullptr},
                                {n.dyq_rs, n.dyq_hs, n.dyk_rs, n.dyk_hs, n.q_rs, n.q_hs, n.k_rs, n.k_hs, n.dq_rs, n.dq_hs, n.dk_rs, n.dk_hs});
            const int64_t most = w ? seq::HEADS_PARTS / 2 : seq::HEADS_PARTS;
            heads_form<E>(w, A.s, 4 * most, [&](auto V, auto K) {
                parts = std::min<int64_t>(groups_of_rows(A.s), most);
                seq::k_heads_grad<E, V.value, K.value><<<dim3((unsigned)parts), 256, 0, st>>>(A);
            });
        };
        n.dtype == DQN_F32 ? launch(float{}) : launch(seq::bf16{});
    }
    seq::k_heads_join<<<dim3((unsigned)((2 * n.D + 15) / 16)), 1024, 0, st>>>((const float *)n.workspace, (int)parts, n.D, n.Hq ? n.dq_weight : nullptr, n.Hk ? n.dk_weight : nullptr);
    return launched(call);
}

}  // extern "C"
