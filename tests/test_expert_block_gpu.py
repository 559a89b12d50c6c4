"""The operators of a mixture of experts together: the example's block against the same block in 64 bits."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("expert_block", os.path.join(ROOT, "examples", "expert_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _bf16(x):
    import torch
    return x.to(torch.bfloat16).double()


def _codes(z):
    import torch
    top = z.abs().amax(1, keepdim=True)
    return torch.round(127 * z / top), top / 127


def _rms(x, weight):
    import torch
    return x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6) * weight.double()


def _block(B, x):
    """(logits, then for given ids: the stream and the next norm's values) in float64, with the program's roundings between its calls"""
    import torch
    q, s = _codes(x * B.norm.double())
    s = s / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6)
    logits = (q @ B.router.double().T) * s * B.router_scales.double()

    def rest(ids):
        score = torch.sigmoid(logits)
        w = torch.gather(score, 1, ids)
        w = w / w.sum(1, keepdim=True)
        y = torch.zeros_like(x)
        for e in range(B.experts):
            t, j = torch.nonzero(ids == e, as_tuple=True)
            if not len(t):
                continue
            u = (q[t] @ B.up[e].double().T) * s[t] * B.up_scales[e].double()
            g, u = u[:, :B.hidden], u[:, B.hidden:]
            mq, ms = _codes(_bf16(g * torch.sigmoid(g) * u))
            y.index_add_(0, t, _bf16((mq @ B.down[e].double().T) * ms * B.down_scales[e].double()) * w[t, j][:, None])
        h = _bf16(x + _rms(y, B.post))
        return h, _rms(h, B.next_norm)
    return logits, rest


def _choice(logits, balance, top, groups, top_groups):
    c = 1 / (1 + np.exp(-logits)) + balance
    part = -np.sort(-c.reshape(len(c), groups, -1), 2)[:, :, :2].sum(2)
    order = np.argsort(-part, 1, kind="stable")[:, :top_groups]
    kept = np.zeros((len(c), groups), bool)
    np.put_along_axis(kept, order, True, 1)
    return np.argsort(-np.where(np.repeat(kept, c.shape[1] // groups, 1), c, -np.inf), 1, kind="stable")[:, :top]


@pytest.mark.parametrize("tokens", [1, 7, 33, 200, 512])
def test_a_block(example, tokens):
    import torch
    B = example.ExpertBlock()
    x = torch.randn((tokens, B.width), generator=torch.Generator().manual_seed(tokens)).to(torch.bfloat16).cuda()
    codes, scales = torch.empty((tokens, B.width), dtype=torch.int8, device="cuda"), torch.empty(tokens, device="cuda")
    before = x.double()
    B.step(x, codes, scales)
    torch.cuda.synchronize()
    logits, rest = _block(B, before)
    got = B.logits[:tokens].double()
    # a handful of roundings of float32, of which the square root's and the sums' are the most
    assert float((got - logits).abs().max()) <= 2.0 ** -16 * float(logits.abs().max())
    ids = B.ids[:tokens].long()
    assert np.array_equal(ids.cpu().numpy(), _choice(got.cpu().numpy(), B.balance.double().cpu().numpy(), B.top, B.groups, B.top_groups))
    h, z = rest(ids)
    # roundings to bfloat16 of 2^-9 each, of the middle, the rows and the stream, and where one falls the other way, a code of 1 / 127 of a row's
    # largest beside it among hundreds of terms: below 2^-6 of the result together
    assert float((x.double() - h).norm() / h.norm()) <= 2.0 ** -6
    back = codes.double() * scales.double()[:, None]
    # the codes themselves: half a step, of a 127th of a row's largest of some four times its root mean square, evenly spread
    assert float((back - z).norm() / z.norm()) <= 2.0 ** -6 + 4.5 / 127 / 12 ** 0.5


def test_a_token_that_is_no_number_stays_by_itself(example):
    import torch
    B = example.ExpertBlock(width=256, hidden=128, experts=8, top=2, groups=2, top_groups=1)
    x = torch.randn((40, 256), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()
    codes, scales = torch.empty((40, 256), dtype=torch.int8, device="cuda"), torch.empty(40, device="cuda")
    clean = x.clone()
    B.step(clean, codes, scales)
    y, c, s = x.clone(), codes.clone(), scales.clone()
    y[17, 3] = float("nan")
    B.step(y, c, s)
    torch.cuda.synchronize()
    others = torch.arange(40, device="cuda") != 17
    assert torch.equal(y[others], clean[others]) and torch.equal(c[others], codes[others]) and torch.equal(s[others], scales[others])
    assert torch.isnan(y[17]).all() and torch.isnan(s[17]) and (c[17] == 0).all() and (B.ids[17] == -1).all()


def test_a_captured_block(example):
    import torch
    B = example.ExpertBlock(width=512, hidden=256, experts=16, top=3)
    x = torch.zeros((50, 512), dtype=torch.bfloat16, device="cuda")
    codes, scales = torch.empty((50, 512), dtype=torch.int8, device="cuda"), torch.empty(50, device="cuda")
    source = torch.zeros_like(x)

    def step():
        x.copy_(source)
        B.step(x, codes, scales)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    g = torch.Generator().manual_seed(7)
    for i in range(4):
        source.copy_(torch.randn((50, 512), generator=g))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (x, codes, scales)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (x, codes, scales))), i


def test_the_example_runs(example, capsys):
    example.main()
    assert capsys.readouterr().out.count("root mean square") == 3
