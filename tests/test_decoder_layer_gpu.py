"""The operators together: the example's layer over prompts and single tokens, against the same layer in 64 bits."""
import importlib.util
import os

import pytest

import layer_reference as R

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("decoder_layer", os.path.join(ROOT, "examples", "decoder_layer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _bf16(x):
    import torch
    return x.to(torch.bfloat16).double()


def _linear(x, w, norm=None, act=0, residual=None):
    import torch
    z = x * norm.double() if norm is not None else x
    top = z.abs().amax(1, keepdim=True)
    scales = top / 127
    if norm is not None:
        scales = scales / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6)
    y = torch.round(127 * z / top) @ w.codes.double().T.contiguous() * scales * w.scales.double()
    if w.bias is not None:
        y = y + w.bias.double()
    y = R.act(y, act)
    return _bf16(y if residual is None else y + residual)


def _layer(L, x, counts, history):
    """The layer in float64 with the program's roundings between its calls; history: keys and values of each request."""
    import torch
    d, q, kv = L.d, L.q_heads, L.kv_heads
    wide = _linear(x, L.qkv, L.norm1)
    heads = wide.reshape(-1, q + 2 * kv, d)
    at = torch.cat([torch.arange(len(h[0]), len(h[0]) + n) for h, n in zip(history, counts)]).cuda()
    y = heads[:, :q + kv]
    y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * torch.cat((L.q_norm.expand(q, d), L.k_norm.expand(kv, d))).double()
    c, s = L.cos.double()[at][:, None], L.sin.double()[at][:, None]
    a, b = y[..., :d // 2], y[..., d // 2:]
    y = torch.cat((a * c - b * s, b * c + a * s), -1)
    queries, keys, values = _bf16(y[:, :q]), R.held(y[:, q:]), R.held(heads[:, q + kv:])
    out, first = torch.empty_like(queries), 0
    for r, n in enumerate(counts):
        here = slice(first, first + n)
        history[r] = [torch.cat((history[r][0], keys[here])), torch.cat((history[r][1], values[here]))]
        for h in range(q):
            g = h // (q // kv)
            out[here, h] = R.attention(queries[here, h], history[r][0][:, g], history[r][1][:, g], d ** -0.5)
        first += n
    x = _linear(_bf16(out.reshape(-1, q * d)), L.out, residual=x)
    return _linear(_linear(x, L.up, L.norm2, act=2), L.down, residual=x)


def test_prompts_and_single_tokens(example):
    import torch
    layer = example.Layer(width=512, q_heads=8, kv_heads=2, hidden=1024, pages=40, page=16, most_tokens=256)
    requests, history = example.Requests(layer, 3), [[torch.zeros((0, 2, 64), dtype=torch.float64, device="cuda")] * 2 for _ in range(3)]
    g = torch.Generator().manual_seed(2)
    for counts in ((100, 7, 33), (1, 1, 1), (2, 60, 1), (1, 1, 1)):
        x = torch.randn((sum(counts), 512), generator=g).to(torch.bfloat16).cuda()
        got = requests.step(x, counts).double()
        want = _layer(layer, x.double(), counts, history)
        # six roundings to bfloat16, of 2^-9 each, and where one falls the other way, a code of 1 / 127 of a row's
        # largest beside it in four products of hundreds of terms: below 2^-5 of the result together
        assert float((got - want).norm() / want.norm()) <= 2.0 ** -5, counts


def test_a_prompt_at_once_and_token_by_token(example):
    import torch
    x = torch.randn((40, 1024), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    layer = example.Layer()
    whole = example.Requests(layer, 1).step(x, (40,)).double()
    layer = example.Layer()
    one = example.Requests(layer, 1)
    each = torch.cat([one.step(x[i:i + 1], (1,)) for i in range(40)]).double()
    assert float((whole - each).norm() / whole.norm()) <= 2.0 ** -5


def test_the_example_runs(example, capsys):
    example.main()
    assert capsys.readouterr().out.count("root mean square") == 5
