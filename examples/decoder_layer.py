"""A transformer layer in 8-bit weights and activations over a 4-bit cache, as a serving program runs it.

    python examples/decoder_layer.py          # a prompt of each of three requests, then tokens one by one

One step takes the tokens of any mix of requests, prompts and single tokens alike:

    8-bit rows through the first norm  ->  queries, keys and values (one product, bias)
    heads normed and rotated, keys and values into the cache  ->  attention over it
    8-bit rows  ->  output projection, residual added in its write-back
    8-bit rows through the second norm  ->  first feed-forward product, bias and GELU
    8-bit rows  ->  second feed-forward product, residual

ten kernels (one more where attention joins ranges of keys) and no other traffic of activations than these.  Weights
are random: the sizes are those of an encoder block with 1024 channels, with four key heads for its sixteen query
heads.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2506_11728_amd as M  # noqa: E402

EPS = 1e-6


class Weights:
    """A linear layer's weights: int8 codes, n x k, a float32 scale for each of the n outputs, and a bias."""

    def __init__(self, n, k, seed, bias=True):
        g = torch.Generator().manual_seed(seed)
        w = torch.randn((n, k), generator=g) / math.sqrt(k)
        self.scales = (w.abs().amax(1) / 127).cuda()
        self.codes = (w / w.abs().amax(1, keepdim=True) * 127).round().to(torch.int8).cuda()
        self.bias = (torch.randn(n, generator=g) * 0.1).cuda() if bias else None
        self.n, self.k = n, k


class Layer:
    def __init__(self, width=1024, q_heads=16, kv_heads=4, hidden=4096, pages=64, page=32, positions=4096, most_tokens=512, seed=0):
        self.width, self.q_heads, self.kv_heads, self.d = width, q_heads, kv_heads, width // q_heads
        self.page, self.pages, self.positions = page, pages, positions
        self.qkv = Weights((q_heads + 2 * kv_heads) * self.d, width, seed)
        self.out = Weights(width, width, seed + 1, bias=False)
        self.up, self.down = Weights(hidden, width, seed + 2), Weights(width, hidden, seed + 3, bias=False)
        g = torch.Generator().manual_seed(seed + 4)
        self.norm1, self.norm2 = (torch.randn(width, generator=g) * 0.1 + 1).cuda(), (torch.randn(width, generator=g) * 0.1 + 1).cuda()
        self.q_norm, self.k_norm = (torch.randn(self.d, generator=g) * 0.1 + 1).cuda(), (torch.randn(self.d, generator=g) * 0.1 + 1).cuda()
        angle = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, self.d, 2, dtype=torch.float64) / self.d)
        self.cos, self.sin = angle.cos().float().cuda(), angle.sin().float().cuda()
        self.cache = torch.empty(M.mipgemm_kv4_bytes(pages, page, kv_heads, self.d), dtype=torch.uint8, device="cuda")
        # what a step needs, for as many tokens as a step may have
        widest = max(hidden, self.qkv.n)
        self.codes = torch.empty((most_tokens, widest), dtype=torch.int8, device="cuda")
        self.scales = torch.empty(most_tokens, device="cuda")
        self.wide = torch.empty((most_tokens, widest), dtype=torch.bfloat16, device="cuda")
        self.heads = torch.empty((most_tokens, width), dtype=torch.bfloat16, device="cuda")
        self.workspace = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    def linear(self, x, w, to, norm=None, act=M.NONE, residual=None):
        """to = act(x w + bias) + residual for the rows of x, in 8 bits, through an RMS norm where one is given."""
        rows = x.shape[0]
        M.mipgemm_quantize_rows(rows, w.k, x, x.stride(0), M.BF16, norm, EPS, self.codes, w.k, self.scales)
        M.mipgemm_s8s8_linear(rows, w.n, w.k, self.codes, w.k, self.scales, w.codes, w.k, M.COL_MAJOR, w.scales, w.bias, act,
                              residual, w.n, to, w.n, M.BF16, workspace=self.workspace, workspace_bytes=self.workspace.numel())

    def step(self, x, at, slots, starts, lengths, table, most_q, most_kv):
        """x: tokens x width, of every request in turn; at: their positions; slots: where their keys and values go;
        starts, lengths, table: the requests' rows, tokens and pages (as mipgemm_attention_kv4 takes them).  Returns x after
        the layer."""
        rows, d, q, kv = x.shape[0], self.d, self.q_heads, self.kv_heads
        wide = self.wide.view(-1)[:rows * self.qkv.n].view(rows, self.qkv.n)
        self.linear(x, self.qkv, wide, norm=self.norm1)
        heads = self.heads[:rows]
        M.mipgemm_qk_norm_rope(rows, q, kv, d, M.BF16, wide, self.qkv.n, wide[:, q * d:], self.qkv.n, wide[:, (q + kv) * d:], self.qkv.n,
                               self.q_norm, self.k_norm, EPS, self.cos, self.sin, self.positions, d, M.ROTATE_HALVES, at, wide, self.qkv.n,
                               None, kv * d, self.cache, self.cache.numel(), self.pages, self.page, slots)
        M.mipgemm_attention_kv4(lengths.numel(), q, kv, d, M.BF16, wide, self.qkv.n, rows, starts, most_q, lengths, most_kv, self.cache,
                                self.cache.numel(), self.pages, self.page, table, table.shape[1], 1 / math.sqrt(d), heads, self.width,
                                workspace=self.workspace, workspace_bytes=self.workspace.numel())
        y = torch.empty_like(x)
        self.linear(heads, self.out, y, residual=x)
        wide = self.wide.view(-1)[:rows * self.up.n].view(rows, self.up.n)
        self.linear(y, self.up, wide, norm=self.norm2, act=M.GELU)
        self.linear(wide, self.down, y, residual=y)  # the residual is added in place
        return y


class Requests:
    """Pages of the cache handed out to requests as they grow."""

    def __init__(self, layer, count):
        self.layer, self.lengths = layer, [0] * count
        self.free = list(range(layer.pages - 1, -1, -1))
        self.table = torch.full((count, layer.pages), -1, dtype=torch.int32)

    def step(self, x, counts):
        """x: the new tokens of every request in turn, counts of them."""
        page, slots, at = self.layer.page, [], []
        for r, n in enumerate(counts):
            for t in range(self.lengths[r], self.lengths[r] + n):
                if t % page == 0:
                    self.table[r, t // page] = self.free.pop()
                slots.append(int(self.table[r, t // page]) * page + t % page)
                at.append(t)
            self.lengths[r] += n
        starts = torch.tensor([0] + list(counts)).cumsum(0).to(torch.int32)
        return self.layer.step(x, torch.tensor(at, dtype=torch.int32).cuda(), torch.tensor(slots).cuda(), starts.cuda(),
                               torch.tensor(self.lengths, dtype=torch.int32).cuda(), self.table.cuda(), max(counts), max(self.lengths))


def main():
    layer = Layer()
    requests = Requests(layer, 3)
    g = torch.Generator().manual_seed(1)
    prompts = (130, 7, 64)
    x = torch.randn((sum(prompts), layer.width), generator=g).to(torch.bfloat16).cuda()
    y = requests.step(x, prompts)
    print("prompts of %s tokens: root mean square %.3f" % (prompts, y.float().square().mean().sqrt()))
    for i in range(4):
        y = requests.step(torch.randn((3, layer.width), generator=g).to(torch.bfloat16).cuda(), (1, 1, 1))
        print("token %d of each: root mean square %.3f" % (i + 1, y.float().square().mean().sqrt()))


if __name__ == "__main__":
    main()
