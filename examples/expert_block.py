"""The feed-forward block of a mixture of experts in 8-bit weights and activations, as a serving program runs it.

    python examples/expert_block.py          # a prompt, then single tokens of a few requests

A step takes the tokens of any mix of requests:

    8-bit rows through the block's norm   ->  the router's product, its logits in float32
    each token's experts and weights, the tokens' rows sorted by expert
    first products of the experts (gated, SiLU), the tokens' codes read where they are
    8-bit rows   ->  second products
    a token's rows summed by weight, normed, added to the stream; the next block's norm, in 8 bits

Nothing is read back by the host, so that a step of given sizes can be captured in a graph.  Weights are random.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2506_11728_amd as M  # noqa: E402

EPS = 1e-6


def _weights(shape, seed):
    """int8 codes and a float32 scale for each row, of random numbers of size 1 / sqrt(k)"""
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(shape, generator=g) / math.sqrt(shape[-1])
    top = w.abs().amax(-1, keepdim=True)
    return (w / top * 127).round().to(torch.int8).cuda(), (top[..., 0] / 127).contiguous().cuda()


class ExpertBlock:
    def __init__(self, width=1024, hidden=512, experts=32, top=4, groups=4, top_groups=2, most_tokens=512, seed=0):
        self.width, self.hidden, self.experts, self.top, self.groups, self.top_groups = width, hidden, experts, top, groups, top_groups
        self.router, self.router_scales = _weights((experts, width), seed)
        self.up, self.up_scales = _weights((experts, 2 * hidden, width), seed + 1)    # the gate's rows, then the others
        self.down, self.down_scales = _weights((experts, width, hidden), seed + 2)
        g = torch.Generator().manual_seed(seed + 3)
        self.balance = (torch.randn(experts, generator=g) * 0.05).cuda()
        gain = lambda: (torch.randn(width, generator=g) * 0.1 + 1).cuda()  # noqa: E731
        self.norm, self.post, self.next_norm = gain(), gain(), gain()
        rows = most_tokens * top
        self.codes, self.scales = torch.empty((most_tokens, width), dtype=torch.int8, device="cuda"), torch.empty(most_tokens, device="cuda")
        self.logits = torch.empty((most_tokens, experts), device="cuda")
        self.ids, self.weights = torch.empty((most_tokens, top), dtype=torch.int32, device="cuda"), torch.empty((most_tokens, top), device="cuda")
        self.starts = torch.empty(experts + 1, dtype=torch.int32, device="cuda")
        self.order, self.places = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda")
        self.middle = torch.empty((rows, hidden), dtype=torch.bfloat16, device="cuda")
        self.middle_codes, self.middle_scales = torch.empty((rows, hidden), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
        self.out = torch.empty((rows, width), dtype=torch.bfloat16, device="cuda")
        self.workspace = torch.empty(max(16, M.mipgemm_route_workspace_size(most_tokens, experts, top)), dtype=torch.uint8, device="cuda")

    def step(self, x, next_codes, next_scales):
        """x (tokens x width, bfloat16): the stream, the block's result added in place; next_codes and next_scales: the next
        block's norm of it in 8 bits."""
        t, w, f, e, top = x.shape[0], self.width, self.hidden, self.experts, self.top
        M.mipgemm_quantize_rows(t, w, x, w, M.BF16, self.norm, EPS, self.codes, w, self.scales)
        M.mipgemm_s8s8_linear(t, e, w, self.codes, w, self.scales, self.router, w, M.COL_MAJOR, self.router_scales, None, M.NONE, None, e,
                              self.logits, e, M.F32)
        M.mipgemm_route(t, e, top, self.logits, e, M.F32, self.balance, M.SIGMOID, self.groups, self.top_groups, 2, 1, 1.0, self.ids,
                        self.weights, self.starts, self.order, self.places, workspace=self.workspace, workspace_bytes=self.workspace.numel())
        rows = t * top
        M.mipgemm_s8s8_experts(rows, e, f, w, self.codes, w, t, self.scales, self.starts, self.order, top, self.up, w, 2 * f * w,
                               self.up_scales, None, M.SILU, 1, self.middle, f, M.BF16)
        M.mipgemm_quantize_rows(rows, f, self.middle, f, M.BF16, None, 0.0, self.middle_codes, f, self.middle_scales)
        M.mipgemm_s8s8_experts(rows, e, w, f, self.middle_codes, f, rows, self.middle_scales, self.starts, None, 1, self.down, f, w * f,
                               self.down_scales, None, M.NONE, 0, self.out, w, M.BF16)
        M.mipgemm_join_rows(t, w, top, M.BF16, self.out, w, rows, self.places, self.weights, M.RMS_NORM, self.post, None, None, w, 1, 1.0,
                            x, w, x, w, M.RMS_NORM, self.next_norm, None, EPS, None, w, next_codes, w, next_scales)


def main():
    block = ExpertBlock()
    g = torch.Generator().manual_seed(1)
    codes, scales = torch.empty((512, block.width), dtype=torch.int8, device="cuda"), torch.empty(512, device="cuda")
    for tokens in (300, 5, 1):
        x = torch.randn((tokens, block.width), generator=g).to(torch.bfloat16).cuda()
        block.step(x, codes, scales)
        most = int((block.starts[1:] - block.starts[:-1]).max())
        print("%d tokens: root mean square %.3f, at most %d rows of an expert" % (tokens, x.float().square().mean().sqrt(), most))


if __name__ == "__main__":
    main()
