// C ABI of the steps for matrices (see include/dqn.h): checks of arguments and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <type_traits>
#include <vector>

#include "../../include/dqn.h"
#include "checks.h"
#include "muon.h"

struct dqn_muon {
    seq::MuonArgs args;
    int64_t chunks, start, half[3], whole[3];       // workgroups of the launches, by the size of their parts
    int grad_dtype;
    seq::f4 *sums;
};

namespace {

constexpr int64_t LONGEST = 1 << 20;    // most rows or columns
// Parts of a product that are enough for 256 compute units, by their size.  us a launch in parts of 64, 128, 256: B X of twelve matrices of 1024 x 4096 and
// 2048 x 2048 (768 parts of 256) 822, 582, 424, their X X^T (224) 434, 307, 311; of a block of 512 channels (196 parts of 128) 22, 26, 64.
// The rule counts parts, not how full they are: 200 matrices of 64 x 64 count as 200 parts of 256, each mostly padding, and take 250 us a step.
constexpr int64_t ENOUGH[3] = {0, 256, 192};
constexpr int64_t MOST_CUTS = 6;

const char *check_matrices(const dqn_muon_matrix *t, int32_t count)
{
    if (!t || count < 1 || count > 65536) return "count must be in 1..65536, matrices not NULL";
    for (int32_t i = 0; i < count; ++i) {
        if (t[i].rows < 0 || t[i].cols < 0 || t[i].rows > LONGEST || t[i].cols > LONGEST || std::min(t[i].rows, t[i].cols) > 65536) return "a matrix's size is out of range";
        if (t[i].rows && t[i].cols && (!t[i].param || !t[i].momentum || !t[i].grad || !at(t[i].param, 4) || !at(t[i].momentum, 4) || !at(t[i].copy, 2)))
            return "a matrix's pointer is NULL or not aligned to its elements";
        if (!(t[i].decay >= 0.f) || std::isinf(t[i].decay)) return "decay must be finite and >= 0";
    }
    return nullptr;
}

// Whether a buffer that a step writes (parameters, momentum, copy) lies on any other, a gradient's too: the same matrix twice, say.
bool overlapping(const dqn_muon_matrix *t, int32_t count, size_t grad_bytes)
{
    struct Range {
        uintptr_t begin, end;
        bool written;
    };
    std::vector<Range> ranges;
    auto add = [&](const void *p, size_t bytes, bool written) { ranges.push_back({(uintptr_t)p, (uintptr_t)p + bytes, written}); };
    for (int32_t i = 0; i < count; ++i) {
        const size_t n = (size_t)t[i].rows * (size_t)t[i].cols;
        if (!n) continue;
        add(t[i].param, 4 * n, true);
        add(t[i].momentum, 4 * n, true);
        add(t[i].grad, grad_bytes * n, false);
        if (t[i].copy) add(t[i].copy, 2 * n, true);
    }
    std::sort(ranges.begin(), ranges.end(), [](const Range &x, const Range &y) { return x.begin < y.begin; });
    uintptr_t any = 0, written = 0;
    for (const Range &r : ranges) {
        if (r.begin < (r.written ? any : written)) return true;
        any = std::max(any, r.end);
        if (r.written) written = std::max(written, r.end);
    }
    return false;
}

// Of one matrix: its padded sides and its parts of the workspace in bytes, in their order.
struct Parts {
    int64_t rp, cp, chunks, x, a, sums;
    int64_t bytes() const { return 2 * x + 2 * a + sums; }
};
int64_t padded(int64_t n) { return (n + seq::PAD - 1) / seq::PAD * seq::PAD; }
Parts parts_of(const dqn_muon_matrix &t)
{
    Parts p{};
    if (!t.rows || !t.cols) return p;
    p.rp = padded(std::min(t.rows, t.cols));
    p.cp = padded(std::max(t.rows, t.cols));
    p.chunks = (t.rows * t.cols + seq::MUON_CHUNK - 1) / seq::MUON_CHUNK;
    p.x = p.rp * p.cp * 4;
    p.a = p.rp * p.rp * 4;
    p.sums = (p.chunks * 8 + 255) / 256 * 256;
    return p;
}

struct Total {
    int64_t plan, workspace, chunks, start, half[3], whole[3];
    void add(const Parts &p)
    {
        workspace += p.bytes();
        chunks += p.chunks;
        start += p.rp / 64 * (p.cp / 64);
        for (int t = 0; t < 3; ++t) {
            const int64_t n = seq::TILES[t], down = (p.rp + n - 1) / n;
            half[t] += down * (down + 1) / 2;
            whole[t] += down * ((p.cp + n - 1) / n);
        }
    }
};
Total total_of(const dqn_muon_matrix *t, int32_t count)
{
    Total s{((int64_t)count * (int64_t)sizeof(seq::MuonMatrix) + 255) / 256 * 256, 0, 0, 0, {}, {}};
    for (int32_t i = 0; i < count; ++i) s.add(parts_of(t[i]));
    return s;
}

// The largest parts of which there is enough for the compute units.
int part_of(const int64_t (&n)[3]) { return n[2] >= ENOUGH[2] ? 2 : n[1] >= ENOUGH[1] ? 1 : 0; }
// Sums that X X^T is cut into where it has few parts (of 64 x 64), for one to two workgroups per compute unit, two being what LDS has place for.  A step with
// 144 parts: uncut 329 us, in two 299, in three 314; with 40 parts: in six 204, in eight 211, in twelve 234.
int cuts_of(int64_t parts) { return parts ? (int)std::max<int64_t>(1, std::min<int64_t>(MOST_CUTS, 384 / parts)) : 1; }
size_t sums_bytes(int64_t parts) { return cuts_of(parts) > 1 ? (size_t)parts * cuts_of(parts) * 64 * 64 * 4 : 0; }
template <int T> bool granted_lds()
{
    static std::atomic<uint64_t> a{0}, b{0}, c{0}, d{0};
    constexpr int bytes = seq::muon_lds(seq::TILES[T]);
    return lds_granted((const void *)seq::k_muon_gram<seq::WHOLE, T>, bytes, a) && lds_granted((const void *)seq::k_muon_gram<seq::SQUARE, T>, bytes, b) &&
           lds_granted((const void *)seq::k_muon_apply<false, T>, bytes, c) && lds_granted((const void *)seq::k_muon_apply<true, T>, bytes, d);
}
template <class F> void with_part(int t, F &&go)
{
    if (t == 2) go(std::integral_constant<int, 2>{});
    else if (t == 1) go(std::integral_constant<int, 1>{});
    else go(std::integral_constant<int, 0>{});
}

template <class G> void launch_begin(const dqn_muon &o, hipStream_t st)
{
    seq::k_muon_momentum<G><<<dim3((unsigned)o.chunks), 256, 0, st>>>(o.args);
    seq::k_muon_start<G><<<dim3((unsigned)o.start), 256, 0, st>>>(o.args);
}

}  // namespace

extern "C" {

int32_t dqn_muon_sizes(const dqn_muon_matrix *matrices, int32_t count, size_t *plan, size_t *workspace)
{
    static const char *call = "dqn_muon_sizes";
    if (!plan || !workspace) return bad(call, "NULL argument");
    if (const char *m = check_matrices(matrices, count)) return bad(call, m);
    const Total s = total_of(matrices, count);
    *plan = (size_t)s.plan;
    *workspace = std::max<size_t>((size_t)s.workspace + sums_bytes(s.half[0]), 256);
    return DQN_OK;
}

int32_t dqn_muon_init(dqn_muon **out, const dqn_muon_matrix *matrices, int32_t count, int32_t grad_dtype, void *plan, void *workspace, void *stream)
{
    static const char *call = "dqn_muon_init";
    if (!out) return bad(call, "NULL argument");
    *out = nullptr;
    if (const char *m = check_matrices(matrices, count)) return bad(call, m);
    if (!dtype_ok(grad_dtype)) return bad(call, "grad_dtype must be DQN_F32 or DQN_BF16");
    if (!plan || !workspace || !at(plan, 256) || !at(workspace, 256)) return bad(call, "plan or workspace is NULL or not 256-byte aligned");
    for (int32_t i = 0; i < count; ++i)
        if (!at(matrices[i].grad, bytes_of(grad_dtype))) return bad(call, "a gradient is not aligned to its elements");
    const Total s = total_of(matrices, count);
    if (s.chunks >= 1 << 24 || s.start >= 1 << 24 || s.half[0] >= 1 << 24 || s.whole[0] >= 1 << 24) return bad(call, "too many elements");   // a launch has 2^32 threads
    dqn_muon *o = nullptr;
    try {
        if (overlapping(matrices, count, bytes_of(grad_dtype))) return bad(call, "a matrix's parameters, momentum or copy lie on another buffer");
        std::vector<seq::MuonMatrix> table;
        table.reserve((size_t)count);
        uint8_t *at = (uint8_t *)workspace;
        Total before{};
        // those whose parts take longest first
        std::vector<int32_t> order;
        for (int32_t i = 0; i < count; ++i)
            if (matrices[i].rows && matrices[i].cols) order.push_back(i);
        std::stable_sort(order.begin(), order.end(), [&](int32_t x, int32_t y) {
            const Parts p = parts_of(matrices[x]), q = parts_of(matrices[y]);
            return p.rp != q.rp ? p.rp > q.rp : p.cp > q.cp;
        });
        for (int32_t i : order) {
            const dqn_muon_matrix &t = matrices[i];
            const Parts p = parts_of(t);
            seq::MuonMatrix m{};
            m.p = t.param; m.m = t.momentum; m.g = t.grad; m.copy = t.copy;
            m.y[0] = (seq::bf16 *)at; m.y[1] = (seq::bf16 *)(at + p.x);
            m.a = (seq::bf16 *)(at + 2 * p.x); m.b = (seq::bf16 *)(at + 2 * p.x + p.a); m.sums = (double *)(at + 2 * p.x + 2 * p.a);
            at += p.bytes();
            m.rows = (long)t.rows; m.cols = (long)t.cols; m.rp = (int)p.rp; m.cp = (int)p.cp; m.tall = t.rows > t.cols;
            m.decay = t.decay; m.scale = (float)std::sqrt(std::max(1.0, (double)t.rows / (double)t.cols)); m.chunks = (int)p.chunks;
            m.first_chunk = (int)before.chunks; m.first_start = (int)before.start;
            for (int k = 0; k < 3; ++k) m.first_half[k] = (int)before.half[k], m.first_whole[k] = (int)before.whole[k];
            before.add(p);
            table.push_back(m);
        }
        hipStream_t st = (hipStream_t)stream;
        if (!table.empty() && (hipMemcpyAsync(plan, table.data(), table.size() * sizeof(table[0]), hipMemcpyHostToDevice, st) != hipSuccess || hipStreamSynchronize(st) != hipSuccess)) {
            (void)hipGetLastError();
            return dqn_seq_fail(DQN_ERR_HIP, call, "copying the table of matrices failed");
        }
        o = new dqn_muon{};
        o->args.count = (int)table.size();
    } catch (...) {
        return dqn_seq_fail(DQN_ERR_OOM, call, "out of host memory");
    }
    o->args.matrices = (const seq::MuonMatrix *)plan;
    o->chunks = s.chunks; o->start = s.start; o->grad_dtype = grad_dtype;
    o->sums = (seq::f4 *)((uint8_t *)workspace + s.workspace);
    std::copy(s.half, s.half + 3, o->half);
    std::copy(s.whole, s.whole + 3, o->whole);
    *out = o;
    return DQN_OK;
}

int32_t dqn_muon_step(dqn_muon *opt, double lr, double momentum, int32_t nesterov, double eps, int32_t rounds, void *stream)
{
    static const char *call = "dqn_muon_step";
    if (!opt) return bad(call, "NULL argument");
    if (!(lr >= 0.0) || lr > 1e30 || !(eps >= 1e-30) || eps > 1e30) return bad(call, "lr in 0..1e30 and eps in 1e-30..1e30 required");
    if (!(momentum >= 0.0 && momentum < 1.0)) return bad(call, "momentum must be in [0, 1)");
    if (rounds < 1 || rounds > 100) return bad(call, "rounds must be in 1..100");
    if (!opt->args.count) return DQN_OK;
    seq::MuonArgs A = opt->args;
    A.nesterov = nesterov != 0; A.mu = (float)momentum; A.eps = (float)eps; A.lr = (float)lr;
    A.a = 3.4445f; A.b = -4.7750f; A.c = 2.0315f;
    hipStream_t st = (hipStream_t)stream;
    dqn_muon now = *opt;
    now.args = A;
    const int half = part_of(opt->half), whole = part_of(opt->whole), cuts = cuts_of(opt->half[0]);
    bool ok = true;
    with_part(half, [&](auto t) { ok = ok && granted_lds<t.value>(); });
    with_part(whole, [&](auto t) { ok = ok && granted_lds<t.value>(); });
    if (!ok) return dqn_seq_fail(DQN_ERR_HIP, call, "the LDS of a part was not granted");
    opt->grad_dtype == DQN_F32 ? launch_begin<float>(now, st) : launch_begin<seq::bf16>(now, st);
    for (int32_t i = 0; i < rounds; ++i) {
        A.from = i & 1;
        with_part(half, [&](auto t) {
            constexpr int n = seq::TILES[t.value];
            const dim3 grid((unsigned)opt->half[t.value]);
            if (t.value == 0 && cuts > 1) {
                seq::k_muon_gram<seq::SPLIT, 0><<<dim3((unsigned)(opt->half[0] * cuts)), seq::muon_threads(64), seq::muon_lds(64), st>>>(A, opt->sums, cuts);
                seq::k_muon_gram<seq::JOIN, 0><<<grid, seq::muon_threads(64), 0, st>>>(A, opt->sums, cuts);
            } else seq::k_muon_gram<seq::WHOLE, t.value><<<grid, seq::muon_threads(n), seq::muon_lds(n), st>>>(A, nullptr, 1);
            seq::k_muon_gram<seq::SQUARE, t.value><<<grid, seq::muon_threads(n), seq::muon_lds(n), st>>>(A, nullptr, 1);
        });
        with_part(whole, [&](auto t) {
            constexpr int n = seq::TILES[t.value];
            const dim3 grid((unsigned)opt->whole[t.value]);
            if (i + 1 < rounds) seq::k_muon_apply<false, t.value><<<grid, seq::muon_threads(n), seq::muon_lds(n), st>>>(A);
            else seq::k_muon_apply<true, t.value><<<grid, seq::muon_threads(n), seq::muon_lds(n), st>>>(A);
        });
    }
    return launched(call);
}

int32_t dqn_muon_destroy(dqn_muon *opt)
{
    delete opt;
    return DQN_OK;
}

}  // extern "C"
