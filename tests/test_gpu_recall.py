"""The recurrent Q-network of toy_recall.py: its gradients against torch's autograd, its 8-bit acting path against its
training pass, and that it learns what takes a memory."""
import pytest
import torch

pytestmark = pytest.mark.gpu


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


def plain(toy, p, obs, reset, C):
    """The network in fp32 with torch on the CPU, step by step."""
    B, T, _ = obs.shape

    def norm(x, w):
        return w * x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)

    x0 = obs @ p["enc"].t() + p["enc_b"]
    z = norm(x0, p["n1"]) @ p["z"].t() + p["z_b"]
    a, x = torch.sigmoid(z[..., :C]), z[..., C:]
    s, hs = torch.zeros(B, C), []
    for t in range(T):
        s = torch.where(reset[:, t, None], torch.zeros_like(s), s)
        s = a[:, t] * s + (1 - a[:, t]) * x[:, t]
        hs.append(s)
    o = torch.stack(hs, 1) @ p["o"].t()
    return norm(x0 + o, p["n2"]) @ p["q"].t() + p["q_b"]


def off(x, y):
    return float((x.double().cpu() - y.double().cpu()).norm() / y.double().cpu().norm())


@pytest.mark.parametrize("B,T", [(3, 50), (300, 24)])
def test_gradients_of_the_network(toy, B, T):
    """About ten numbers between an input and a gradient are rounded to bf16, each 2^-9 off on average: one part in a
    hundred, and 5 % is allowed."""
    C = 64
    net = toy.RecurrentQ(C, 5)
    obs, reset = sequences(toy, B, T, 6)
    q, saved = net.forward(obs, reset)
    dq = torch.randn(B, T, toy.K, generator=torch.Generator().manual_seed(7)) / (B * T)
    net.backward(dq.cuda(), saved)
    p = {k: v.float().cpu().requires_grad_() for k, v in net.half.items()}
    want = plain(toy, p, obs.float().cpu(), reset.cpu(), C)
    assert off(q, want.detach()) < 0.03
    want.backward(dq)
    for k, v in p.items():
        assert off(net.grad[k], v.grad) < 0.05, k


def test_acting_in_eight_bits_is_the_training_pass(toy):
    """The same sequences one step at a time with 8-bit rows and weights: an e4m3 number is 2.6 % off on average, so a product is
    about 4 % and the three in a chain 7 %; 20 % is allowed.  The state is kept in place, new episodes start from nothing."""
    C, B, T = 128, 33, 20
    net = toy.RecurrentQ(C, 8)
    obs, reset = sequences(toy, B, T, 9)
    q, _ = net.forward(obs, reset)
    w8, state = net.acting_weights(), torch.full((B, C), 9.0, device="cuda")
    steps = torch.stack([net.act(obs[:, t].contiguous(), reset[:, t:t + 1], state, w8) for t in range(T)], 1)
    assert off(steps, q) < 0.2
    assert float(state.abs().max()) < 9.0


@pytest.mark.parametrize("bits", [8, 32])
def test_it_learns_to_remember(toy, bits):
    print("case recall", bits, flush=True)
    reward = toy.run(120, seed=1, bits=bits)
    assert reward > 0.8, reward      # -0.5 without a memory
