"""The recurrent Q-network with a matrix memory of toy_recall.py: its gradients against torch's autograd, its 8-bit acting path against
its training pass, and that its training runs."""
import pytest
import torch

pytestmark = pytest.mark.gpu
C = 64


@pytest.fixture(scope="module")
def toy():
    from paper_1804_05834_amd import toy_recall
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return toy_recall


def sequences(toy, B, T, seed):
    g = torch.Generator().manual_seed(seed)
    obs = torch.randn(B, T, toy.D, generator=g).to(torch.bfloat16)
    reset = torch.rand(B, T, generator=g) < 0.1
    reset[:, 0] = True
    return obs.cuda(), reset.cuda()


def plain(net, p, obs, reset):
    """The network in fp32 with torch on the CPU, step by step."""
    B, T, _ = obs.shape
    H, W = net.H, net.width
    turns = torch.tensor(list(net.turns._turns), dtype=torch.float64)

    def norm(x, w):
        return w * x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)

    def turned(x, position):
        t = 2 * torch.pi * position[:, None, None].double() * turns
        c, s = torch.cos(t).float(), torch.sin(t).float()
        lo, hi = x[..., :W // 2], x[..., W // 2:]
        return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)

    x0 = obs @ p["enc"].t() + p["enc_b"]
    z = norm(x0, p["n1"]) @ p["z"].t() + p["z_b"]
    q, k, v = (z[..., i * C:(i + 1) * C].view(B, T, H, W) for i in range(3))
    a, beta = torch.sigmoid(z[..., 3 * C:3 * C + H]), torch.sigmoid(z[..., 3 * C + H:])
    S, position, out = torch.zeros(B, H, W, W), torch.zeros(B, dtype=torch.long), []
    for t in range(T):
        S = torch.where(reset[:, t, None, None, None], torch.zeros_like(S), S)
        position = torch.where(reset[:, t], torch.zeros_like(position), position)
        kt, qt = turned(norm(k[:, t], p["kn"]), position), turned(norm(q[:, t], p["qn"]), position)
        held = a[:, t, :, None, None] * S
        gap = v[:, t] - (held * kt[..., None]).sum(2)
        S = held + (beta[:, t, :, None] * kt)[..., None] * gap[:, :, None]
        out.append(net.scale * (S * qt[..., None]).sum(2).reshape(B, C))
        position = position + 1
    o = torch.stack(out, 1) @ p["o"].t()
    return norm(x0 + o, p["n2"]) @ p["q"].t() + p["q_b"]


def off(x, y):
    return float((x.double().cpu() - y.double().cpu()).norm() / y.double().cpu().norm())


@pytest.mark.parametrize("B,T", [(3, 50), (100, 24)])
def test_gradients_of_the_network(toy, B, T):
    """About a dozen numbers between an input and a gradient are rounded to bf16, each 2^-9 off on average: one part in a
    hundred, and 5 % is allowed."""
    net = toy.MatrixQ(C, 5)
    obs, reset = sequences(toy, B, T, 6)
    q, saved = net.forward(obs, reset)
    dq = torch.randn(B, T, toy.K, generator=torch.Generator().manual_seed(7)) / (B * T)
    net.backward(dq.cuda(), saved)
    p = {k: v.float().cpu().requires_grad_() for k, v in net.half.items()}
    want = plain(net, p, obs.float().cpu(), reset.cpu())
    assert off(q, want.detach()) < 0.03
    want.backward(dq)
    for k, v in p.items():
        assert off(net.grad[k], v.grad) < 0.05, k


def test_acting_in_eight_bits_is_the_training_pass(toy):
    """The same sequences one step at a time with 8-bit rows and weights: an e4m3 number is 2.6 % off on average, so a product is about 4 %,
    and what is read, a product of a query, a key and a value of that, 7 %; with the two products behind it 10 %, and 25 % is allowed."""
    B, T = 33, 20
    net = toy.MatrixQ(C, 8)
    obs, reset = sequences(toy, B, T, 9)
    q, _ = net.forward(obs, reset)
    w8, state = net.acting_weights(), net.state(B)
    state[0].fill_(9.0)
    steps = torch.stack([net.act(obs[:, t].contiguous(), reset[:, t:t + 1], state, w8) for t in range(T)], 1)
    assert off(steps, q) < 0.25
    assert float(state[0].abs().max()) < 9.0


def test_training_runs(toy):
    reward = toy.run(3, seed=1, memory="matrix")
    assert -1.0 <= reward <= 1.0
