"""A toy task that takes a memory, and a recurrent Q-network that learns it with the operators of seq.py.

The first observation of an episode shows one of K symbols, the last one a signal; in between there is only noise.
The reward comes at the signal: +1 for the action that names the symbol, -1 for another.  A network that sees the
present alone can do no better than -1 + 2 / K.

The network is one block: a residual stream from the observation, a norm, a projection to the gates and inputs of the
gated recurrence (RecurrentQ) or to the queries, keys, values, gates and rates of a matrix memory (MatrixQ), a projection back,
a norm of the sum, Q-values.  It acts one step at a time with 8-bit weights and
rows, keeping the recurrence's state, and is trained on stored sequences with Double-DQN targets (Eq.9) and Huber's
loss, in bf16 with fp32 master weights, by AdamW, MatrixQ's matrices by Muon.  Dense products of training are torch's; the rest is
the library's.
"""
import torch

from . import seq

K, NOISE = 4, 10          # symbols, noise channels
D = K + 2 + NOISE         # an observation: symbol, start, signal, noise


class Recall:
    """E copies of the task, `length` steps each."""

    def __init__(self, E, length, seed, device="cuda"):
        self.E, self.length, self.device = E, length, device
        self.g = torch.Generator(device=device).manual_seed(seed)
        self.t = 0

    def observe(self):
        """-> (observations [E][D], whether an episode starts [E])"""
        if self.t == 0:
            self.symbol = torch.randint(0, K, (self.E,), generator=self.g, device=self.device)
        o = torch.zeros(self.E, D, device=self.device)
        if self.t == 0:
            o[torch.arange(self.E, device=self.device), self.symbol] = 1
            o[:, K] = 1
        if self.t == self.length - 1:
            o[:, K + 1] = 1
        o[:, K + 2:] = 0.5 * torch.randn(self.E, NOISE, generator=self.g, device=self.device)
        return o.to(torch.bfloat16), torch.full((self.E, 1), self.t == 0, device=self.device)

    def step(self, actions):
        """-> (rewards [E], whether the episode is over)"""
        self.t += 1
        if self.t < self.length:
            return torch.zeros(self.E, device=self.device), False
        self.t = 0
        return torch.where(actions == self.symbol, 1.0, -1.0), True


class RecurrentQ:
    """Parameters, gradients and bf16 copies of the block; C channels."""

    def __init__(self, C, seed, device="cuda", bits=8, lr=2e-3):
        g = torch.Generator().manual_seed(seed)

        def he(n, m):
            return torch.randn(n, m, generator=g) * (1.0 / m) ** 0.5

        gate_bias = torch.zeros(2 * C)
        gate_bias[:C] = 3.0      # a memory of some twenty steps to begin with
        p = dict(enc=he(C, D), enc_b=torch.zeros(C), n1=torch.ones(C), z=he(2 * C, C), z_b=gate_bias, o=he(C, C), n2=torch.ones(C),
                 q=0.1 * he(K, C), q_b=torch.zeros(K))
        self.C = C
        self.p = {k: v.to(device) for k, v in p.items()}
        self.grad = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.half = {k: v.to(torch.bfloat16) for k, v in self.p.items()}
        names = list(self.p)
        self.opt = seq.AdamW([self.p[k] for k in names], [self.grad[k] for k in names], bits=bits, lr=lr,
                             weight_decay=[0.01 if self.p[k].ndim == 2 else 0.0 for k in names], copies=[self.half[k] for k in names])
        self.steps = 0

    # ---- training: whole sequences
    def forward(self, obs, reset, half=None):
        """obs [B][T][D] bf16, reset [B][T] -> Q [B][T][K] float32 and what backward() needs"""
        w, C, (B, T, _) = half or self.half, self.C, obs.shape
        x0 = torch.addmm(w["enc_b"], obs.reshape(B * T, D), w["enc"].t())
        y1, _, s1 = seq.norm(x0, w["n1"].float())
        z = torch.addmm(w["z_b"], y1, w["z"].t()).view(B, T, 2 * C)
        h, _, carry = seq.scan(z[..., :C], z[..., C:], reset=reset, save=True)
        o = h.view(B * T, C) @ w["o"].t()
        y2, r, s2 = seq.norm(o, w["n2"].float(), residual=x0)
        q = (y2 @ w["q"].t()).float() + w["q_b"].float()
        return q.view(B, T, K), (obs, reset, x0, y1, s1, z, h, carry, y2, r, s2)

    def backward(self, dq, saved):
        """Gradients of all parameters from dq [B][T][K]."""
        obs, reset, x0, y1, s1, z, h, carry, y2, r, s2 = saved
        w, g, C, (B, T, _) = self.half, self.grad, self.C, obs.shape
        dq = dq.reshape(B * T, K).to(torch.bfloat16)
        g["q"].copy_(dq.t() @ y2)
        g["q_b"].copy_(dq.float().sum(0))
        do, dn2 = seq.norm_backward(dq @ w["q"], r, s2, w["n2"].float())     # of o and, through the residual, of x0
        g["n2"].copy_(dn2)
        g["o"].copy_(do.t() @ h.view(B * T, C))
        dz = torch.empty_like(z)
        seq.scan_backward((do @ w["o"]).view(B, T, C), z[..., :C], z[..., C:], carry, reset=reset, out=(dz[..., :C], dz[..., C:]))
        dz = dz.view(B * T, 2 * C)
        g["z"].copy_(dz.t() @ y1)
        g["z_b"].copy_(dz.float().sum(0))
        dx0, dn1 = seq.norm_backward(dz @ w["z"], x0, s1, w["n1"].float(), dr=do)
        g["n1"].copy_(dn1)
        g["enc"].copy_(dx0.t() @ obs.reshape(B * T, D))
        g["enc_b"].copy_(dx0.float().sum(0))

    def train(self, target, obs, reset, a, r, done, gamma=0.97):
        """One step on sequences: obs [B][T][D], reset, done [B][T] bool, actions a [B][T], rewards r [B][T]."""
        q, saved = self.forward(obs, reset)
        q_target, _ = self.forward(obs, reset, half=target)
        best = q.argmax(2)
        bootstrap = q_target.gather(2, best[..., None])[..., 0]
        y = r[:, :-1] + gamma * (~done[:, :-1]) * bootstrap[:, 1:]
        td = y - q.gather(2, a[..., None])[..., 0][:, :-1]
        dq = torch.zeros_like(q)
        dq[:, :-1].scatter_(2, a[:, :-1, None], -(td.clamp(-1, 1) / td.numel())[..., None])     # Huber, mean over the steps
        self.backward(dq, saved)
        self.steps += 1
        self.update()
        return td

    def update(self):
        self.opt.step(self.steps, seed=self.steps)

    def copy(self):
        return {k: v.clone() for k, v in self.half.items()}

    # ---- acting: one step at a time in 8 bits
    def acting_weights(self):
        """The weights in 8 bits, laid out once for as many acting steps as they last."""
        return {k: seq.rows(self.half[k]) for k in ("z", "o", "q")}

    def state(self, E):
        """The memory of E agents before their first step."""
        return torch.zeros(E, self.C, device="cuda")

    def act(self, obs, start, state, w8):
        """obs [E][D], start [E][1], state [E][C] float32 (updated in place) -> Q [E][K]"""
        C, p = self.C, self.p
        x0 = torch.addmm(self.half["enc_b"], obs, self.half["enc"].t())
        q1, scale1, _ = seq.norm_rows(x0, p["n1"])
        z = seq.product((q1, scale1), w8["z"], bias=p["z_b"]).view(-1, 1, 2 * C)
        h, _ = seq.scan(z[..., :C], z[..., C:], h0=state, reset=start, last=state)
        o = seq.product(seq.rows(h.view(-1, C)), w8["o"])
        q2, scale2, _ = seq.norm_rows(o, p["n2"], residual=x0)
        return seq.product((q2, scale2), w8["q"], bias=p["q_b"], dtype=torch.float32)


class MatrixQ(RecurrentQ):
    """The same block with a memory of one matrix per head: queries and keys normalised per head and turned by their step in the episode,
    the gated delta rule over time."""

    def __init__(self, C, seed, H=4, device="cuda", lr=2e-3, muon_lr=0.02):
        g = torch.Generator().manual_seed(seed)

        def he(n, m):
            return torch.randn(n, m, generator=g) * (1.0 / m) ** 0.5

        self.C, self.H, self.width = C, H, C // H
        bias = torch.zeros(3 * C + 2 * H)
        bias[3 * C:3 * C + H] = 3.0      # a memory of some twenty steps to begin with
        p = dict(enc=he(C, D), enc_b=torch.zeros(C), n1=torch.ones(C), z=he(3 * C + 2 * H, C), z_b=bias, qn=torch.ones(self.width),
                 kn=torch.full((self.width,), self.width ** -0.5), o=he(C, C), n2=torch.ones(C), q=0.1 * he(K, C), q_b=torch.zeros(K))
        self.p = {k: v.to(device) for k, v in p.items()}
        self.grad = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.half = {k: v.to(torch.bfloat16) for k, v in self.p.items()}
        self.turns, self.scale = seq.rotation(self.width), self.width ** -0.5
        matrices = ["enc", "z", "o"]
        others = [k for k in self.p if k not in matrices]
        self.muon = seq.Muon([self.p[k] for k in matrices], [self.grad[k] for k in matrices], lr=muon_lr, copies=[self.half[k] for k in matrices])
        self.opt = seq.AdamW([self.p[k] for k in others], [self.grad[k] for k in others], lr=lr, weight_decay=0.0, copies=[self.half[k] for k in others])
        self.steps = 0

    def update(self):
        self.muon.step()
        self.opt.step(self.steps)

    def parts(self, z, B, T):
        """Queries and keys [B T][H][width], values [B][T][H][width], gates and rates [B][T][H]: views of rows [B T][3 C + 2 H]."""
        C, H = self.C, self.H
        z3 = z.view(B, T, -1)
        return (z[:, :C].view(B * T, H, self.width), z[:, C:2 * C].view(B * T, H, self.width), z3[..., 2 * C:3 * C].view(B, T, H, self.width),
                z3[..., 3 * C:3 * C + H], z3[..., 3 * C + H:])

    def forward(self, obs, reset, half=None):
        w, C, (B, T, _) = half or self.half, self.C, obs.shape
        step = torch.arange(T, device=obs.device, dtype=torch.int32)
        position = (step - torch.where(reset, step, torch.zeros_like(step)).cummax(1)[0]).reshape(-1).to(torch.int32)      # in the episode
        x0 = torch.addmm(w["enc_b"], obs.reshape(B * T, D), w["enc"].t())
        y1, _, s1 = seq.norm(x0, w["n1"].float())
        z = torch.addmm(w["z_b"], y1, w["z"].t())
        q, k, v, f, b = self.parts(z, B, T)
        yq, yk, rstd = seq.norm_heads(q, k, w["qn"].float(), w["kn"].float(), position=position, turns=self.turns)
        yq, yk = yq.view(v.shape), yk.view(v.shape)
        h, _, carry = seq.delta(yq, yk, v, f, b, reset=reset, scale=self.scale, save=True)
        o = h.view(B * T, C) @ w["o"].t()
        y2, r, s2 = seq.norm(o, w["n2"].float(), residual=x0)
        out = (y2 @ w["q"].t()).float() + w["q_b"].float()
        return out.view(B, T, K), (obs, reset, position, x0, y1, s1, z, yq, yk, rstd, h, carry, y2, r, s2)

    def backward(self, dq, saved):
        obs, reset, position, x0, y1, s1, z, yq, yk, rstd, h, carry, y2, r, s2 = saved
        w, g, C, (B, T, _) = self.half, self.grad, self.C, obs.shape
        dq = dq.reshape(B * T, K).to(torch.bfloat16)
        g["q"].copy_(dq.t() @ y2)
        g["q_b"].copy_(dq.float().sum(0))
        do, dn2 = seq.norm_backward(dq @ w["q"], r, s2, w["n2"].float())
        g["n2"].copy_(dn2)
        g["o"].copy_(do.t() @ h.view(B * T, C))
        dz = torch.empty_like(z)
        (q, k, v, f, b), (zq, zk, zv, zf, zb) = self.parts(z, B, T), self.parts(dz, B, T)
        dyq, dyk = seq.delta_backward((do @ w["o"]).view(v.shape), yq, yk, v, f, b, carry, reset=reset, scale=self.scale, out=(None, None, zv, zf, zb))[:2]
        _, _, dqn, dkn = seq.norm_heads_backward(dyq.view(q.shape), dyk.view(k.shape), q, k, rstd, w["qn"].float(), w["kn"].float(), position=position,
                                                 turns=self.turns, out=(zq, zk))
        g["qn"].copy_(dqn)
        g["kn"].copy_(dkn)
        g["z"].copy_(dz.t() @ y1)
        g["z_b"].copy_(dz.float().sum(0))
        dx0, dn1 = seq.norm_backward(dz @ w["z"], x0, s1, w["n1"].float(), dr=do)
        g["n1"].copy_(dn1)
        g["enc"].copy_(dx0.t() @ obs.reshape(B * T, D))
        g["enc_b"].copy_(dx0.float().sum(0))

    def state(self, E):
        """The heads' matrices and the step in the episode."""
        return torch.zeros(E, self.H, self.width, self.width, device="cuda"), torch.zeros(E, dtype=torch.int32, device="cuda")

    def act(self, obs, start, state, w8):
        p, C, E, (S, position) = self.p, self.C, obs.shape[0], state
        position.masked_fill_(start[:, 0], 0)
        x0 = torch.addmm(self.half["enc_b"], obs, self.half["enc"].t())
        q1, scale1, _ = seq.norm_rows(x0, p["n1"])
        q, k, v, f, b = self.parts(seq.product((q1, scale1), w8["z"], bias=p["z_b"]), E, 1)
        yq, yk, _ = seq.norm_heads(q, k, p["qn"], p["kn"], position=position, turns=self.turns)
        h, _ = seq.delta(yq.view(v.shape), yk.view(v.shape), v, f, b, s0=S, reset=start, scale=self.scale, last=S)
        position.add_(1)
        o = seq.product(seq.rows(h.view(E, C)), w8["o"])
        q2, scale2, _ = seq.norm_rows(o, p["n2"], residual=x0)
        return seq.product((q2, scale2), w8["q"], bias=p["q_b"], dtype=torch.float32)


def run(iterations, seed=0, E=64, length=12, C=64, bits=8, episodes=4, batch=32, target_period=20, log=None, lr=2e-3, memory="scan"):
    """Collects `episodes` episodes of E environments per iteration and trains eight steps on batches of what the last ten
    iterations stored.  memory: "scan" or "matrix".  -> mean reward of 20 near-greedy rounds of E episodes at the end."""
    net = RecurrentQ(C, 1804 + seed, bits=bits, lr=lr) if memory == "scan" else MatrixQ(C, 1804 + seed, lr=lr)
    env = Recall(E, length, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 7)
    target, store = net.copy(), []

    def play(env, rounds, eps):
        w8, state = net.acting_weights(), net.state(env.E)
        obs, start, acts, rew, over = [], [], [], [], []
        for _ in range(rounds * length):
            o, s = env.observe()
            a = net.act(o, s, state, w8).argmax(1)
            a = torch.where(torch.rand(env.E, generator=g, device="cuda") < eps, torch.randint(0, K, (env.E,), generator=g, device="cuda"), a)
            r, done = env.step(a)
            for to, v in zip((obs, start, acts, rew, over), (o, s[:, 0], a, r, torch.full((env.E,), done, device="cuda"))):
                to.append(v)
        return [torch.stack(v, 1) for v in (obs, start, acts, rew, over)]

    for it in range(1, iterations + 1):
        store.append(play(env, episodes, max(0.05, 1.0 - it / (0.4 * iterations))))
        del store[:-10]
        for _ in range(8):
            s = store[int(torch.randint(0, len(store), (1,), generator=g, device="cuda"))]
            pick = torch.randint(0, E, (batch,), generator=g, device="cuda")
            net.train(target, *(v[pick] for v in s))
        if it % target_period == 0:
            target = net.copy()
        if log and it % 20 == 0:
            r = store[-1][3]
            log("iteration %d: mean reward per episode while exploring %.2f" % (it, float(r.sum() / (E * episodes))))
    r = play(Recall(E, length, seed + 1000), 20, 0.001)[3]
    return float(r.sum() / (E * 20))


if __name__ == "__main__":
    import sys
    n = int(sys.argv[1]) if len(sys.argv) > 1 else 200
    for bits in (8, 32):
        print("moments in %d bits" % bits, flush=True)
        print("mean reward per episode: %.2f (without a memory: %.2f)" % (run(n, bits=bits, log=lambda s: print(s, flush=True)), -1 + 2 / K), flush=True)
    print("a matrix per head", flush=True)
    print("mean reward per episode: %.2f" % run(n, memory="matrix", log=lambda s: print(s, flush=True)), flush=True)
