"""The operators run together: Hier-AVG with AdamW local steps on ragged batches."""
import torch
import pytest

from paper_1903_05133_gb300 import configs
from paper_1903_05133_gb300.inputs import initial_layers, learner_data, perturbed_layers
from paper_1903_05133_gb300.local_adamw import LocalAdamW, ragged_batches

pytestmark = pytest.mark.gpu

W = configs.Workload("tiny_mlp_bf16", P=6, S=3, K1=2, K2=2, rounds=1, dims=(200, 136, 10), precision="bf16",
                     N=96, B=24, lr=0.01, sigma_mu=0.3, init="he")


@pytest.fixture(scope="module", autouse=True)
def _cuda(lib):
    assert torch.cuda.is_available(), "GPU tests need CUDA"


@pytest.mark.parametrize("bits", [32, 8])
def test_step_matches_autograd(bits):
    # The first step of Adam is lr * g / (|g| + eps'): its direction is the gradient's sign, so the
    # gradients are compared through the first moments, which are 0.1 g.
    X, y = learner_data(W, device="cuda")
    m = LocalAdamW(W.P, W.S, W.K1, W.K2, W.lr, W.dims, bits=bits)
    layers = perturbed_layers(W, 0.01, seed=3)
    m.load(layers)
    before = [(w.clone(), b.clone()) for w, b in m.layers]
    x, t, off = next(ragged_batches(X, y, W.B, 5))
    logp = m.step(x, t, off)
    at = off.tolist()
    state = m.opt_w.state_dict()
    flat = state["m"] if bits == 32 else (state["m"].float().view(-1, 256) * state["m_scale"][:, None]).view(-1)
    pos = 0
    for l, (w, b) in enumerate(before):
        n = w[0].numel()
        pad = -(-n // 256) * 256
        for j in range(W.P):
            got = flat[pos:pos + n].view(w[j].shape) * 10
            pos += pad
            ws = [v[j].bfloat16().double().requires_grad_() for v, _ in before]
            bs = [v[j].double().requires_grad_() for _, v in before]
            h = x[at[j]:at[j + 1]].double()
            for k in range(len(ws)):
                h = h @ ws[k].T + bs[k]
                if k + 1 < len(ws):
                    h = torch.relu(h)
            lp = torch.log_softmax(h, 1).gather(1, t[at[j]:at[j + 1]].long()[:, None])[:, 0]
            (-lp.mean()).backward()
            assert (logp[at[j]:at[j + 1]].double() - lp).abs().max() < 0.05        # logits of 8 bits' precision
            ref = ws[l].grad
            # activations, logits and gradients pass through bf16 (2^-8 each), 8-bit moments add 2^-4
            assert (got.double() - ref).norm() <= (0.02 if bits == 32 else 0.06) * ref.norm()
    for w, c in zip(m.layers, m.weights):
        assert torch.equal(c, w[0].to(torch.bfloat16))


@pytest.mark.parametrize("bits", [32, 8])
def test_rounds_learn_and_agree(bits):
    X, y = learner_data(W, device="cuda")
    m = LocalAdamW(W.P, W.S, W.K1, W.K2, W.lr, W.dims, bits=bits)
    m.load(initial_layers(W, device="cuda"))
    batches = ragged_batches(X, y, W.B, 1)
    first = -m.step(*next(batches)).mean().item()
    for _ in range(6):
        last = m.round(batches)
        bits_of = m.params.view(torch.int32)
        assert (bits_of == bits_of[0]).all()                # after the global average
    assert -last.mean().item() < 0.5 * first
    assert torch.equal(m.copy, m.params.to(torch.bfloat16)) and m.t == 1 + 6 * W.K1 * W.K2


def test_round_reports_a_wait_that_ran_out(monkeypatch):
    from paper_1903_05133_gb300 import local_adamw
    from paper_1903_05133_gb300._lib import HierAvgError
    X, y = learner_data(W, device="cuda")
    m = LocalAdamW(W.P, W.S, W.K1, W.K2, W.lr, W.dims)
    m.load(initial_layers(W, device="cuda"))
    batches = ragged_batches(X, y, W.B, 1)
    m.round(batches)

    def ran_out():
        raise HierAvgError(-5, "operator_check")
    monkeypatch.setattr(local_adamw, "operator_check", ran_out)
    with pytest.raises(HierAvgError):
        m.round(batches)
