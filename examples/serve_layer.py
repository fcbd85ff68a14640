#!/usr/bin/env python3
"""The attention half of a repaired decoder layer, served in 8 bits on one GPU.

Repairs the layer's q, k, v and o projections (backbone, seed search, ranking,
dense reconstruction), turns the repaired weights into int8 codes with one
scale per output channel, and runs prompts and then single tokens through

    q, k, v = linear_i8(x)              awsrc_linear_i8
    rotate q and k, append k and v      awsrc_kv_append
    attention over the cache            awsrc_kv_attention
    y = linear_i8(o)                    awsrc_linear_i8

with a paged int8 cache.  The decode step is captured as a graph and replayed.
At the end the last tokens' outputs are compared with the same layer in fp32 on
the repaired weights, without any 8-bit rounding.

    python examples/serve_layer.py [--seeds 16] [--prompts 700,65,1] [--steps 8]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_23144_amd as awsrc  # noqa: E402
from synth import gen_module_inputs, workload  # noqa: E402

HEAD_DIM, PAGE = 128, 64


def repaired_weights(seeds: int, device: str):
    """Dense bf16 weights of the 3B layer's q, k, v and o projections after repair at 0.32 bits per weight."""
    wl = workload("block3b", S=seeds)
    mods = wl.modules[:4]
    inputs = [gen_module_inputs(wl, m, device) for m in mods]
    backbones = [awsrc.awsrc_backbone_rtn(i["W"]) for i in inputs]
    p = awsrc.make_params(wl.C, wl.P, wl.b, wl.S, ridge_lambda=wl.ridge_lambda)
    enc = awsrc.awsrc_encode_modules(p, [i["W"] for i in inputs], [b[3] for b in backbones], [i["d"] for i in inputs])
    stream, _, _ = awsrc.awsrc_rank_prefix(p, [(m.rows, m.cols) for m in mods], awsrc.AWSRC_MODE_GLOBAL, 0.32, enc["seed"],
                                           enc["codes"], enc["scale"], enc["gain"])
    dense = [torch.empty(m.rows, m.cols, dtype=torch.bfloat16, device=device) for m in mods]
    plan, keep = awsrc.awsrc_decode_prepare(stream, dense)
    awsrc.awsrc_reconstruct_bf16(plan, [b[:3] for b in backbones])
    torch.cuda.synchronize()
    del keep
    return dense


class Attention:
    """The served half layer: int8 weights, a paged int8 cache, a batch of sequences."""

    def __init__(self, weights, n_seq: int, max_tokens: int, device: str):
        wq, wk, wv, wo = weights
        self.hq, self.hk = wq.shape[0] // HEAD_DIM, wk.shape[0] // HEAD_DIM
        self.qkv, self.qkv_scale = awsrc.awsrc_quantize_rows_i8(torch.cat([wq, wk, wv]))
        self.o, self.o_scale = awsrc.awsrc_quantize_rows_i8(wo)
        pages = -(-max_tokens // PAGE)
        self.max_tokens = max_tokens
        self.cache = awsrc.make_kv_cache(n_seq * pages, self.hk, HEAD_DIM, PAGE, device)
        self.table = torch.randperm(n_seq * pages, device=device).int().view(n_seq, pages)
        angle = torch.arange(max_tokens, device=device).double()[:, None] * 1e6 ** (
            -torch.arange(0, HEAD_DIM, 2, device=device).double() / HEAD_DIM)
        self.cos, self.sin = torch.cos(angle).float(), torch.sin(angle).float()

    def forward(self, x, cu, kv_len, max_new: int, max_kv: int):
        """Rows of x are the sequences' newest tokens (cu as in awsrc_kv_append); kv_len counts them."""
        n, hq, hk = x.shape[0], self.hq, self.hk
        heads = awsrc.awsrc_linear_i8(x, self.qkv, self.qkv_scale).view(n, hq + 2 * hk, HEAD_DIM)
        q = awsrc.awsrc_kv_append(self.cache, heads[:, hq:hq + hk], heads[:, hq + hk:], cu, kv_len, self.table, max_new,
                                  cos=self.cos, sin=self.sin, q=heads[:, :hq])
        a = awsrc.awsrc_kv_attention(self.cache, q, cu, kv_len, self.table, max_new, max_kv)
        return awsrc.awsrc_linear_i8(a.view(n, hq * HEAD_DIM), self.o, self.o_scale)


def reference(weights, x, cos, sin):
    """The same half layer over one whole sequence x [tokens, hidden] in fp32."""
    wq, wk, wv, wo = (w.float() for w in weights)
    n, hk, half = x.shape[0], wk.shape[0] // HEAD_DIM, HEAD_DIM // 2
    c, s = cos[:n, None], sin[:n, None]

    def turn(t):
        a, b = t[..., :half], t[..., half:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    q, k = turn((x @ wq.T).view(n, -1, HEAD_DIM)), turn((x @ wk.T).view(n, hk, HEAD_DIM))
    v = (x @ wv.T).view(n, hk, HEAD_DIM)
    q = q.view(n, hk, -1, HEAD_DIM).permute(1, 2, 0, 3).reshape(hk, -1, HEAD_DIM)
    score = torch.bmm(q, k.permute(1, 2, 0).contiguous()).view(hk, -1, n, n) * HEAD_DIM ** -0.5
    score = score.masked_fill(torch.ones(n, n, dtype=torch.bool, device=x.device).triu(1), -float("inf"))
    o = torch.bmm(torch.softmax(score, -1).view(hk, -1, n), v.permute(1, 0, 2).contiguous())
    return o.view(hk, -1, n, HEAD_DIM).permute(2, 0, 1, 3).reshape(n, -1) @ wo.T


def main(argv=None) -> float:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--seeds", type=int, default=16, help="seeds of the repair's search")
    ap.add_argument("--prompts", default="700,65,1", help="tokens of each sequence's prompt")
    ap.add_argument("--steps", type=int, default=8, help="single tokens after the prompts")
    args = ap.parse_args(argv)
    dev = "cuda"
    prompts = [int(n) for n in args.prompts.split(",")]
    n_seq, longest = len(prompts), max(prompts) + args.steps
    weights = repaired_weights(args.seeds, dev)
    layer = Attention(weights, n_seq, longest, dev)
    g = torch.Generator(device=dev)
    g.manual_seed(1)
    hidden = weights[0].shape[1]
    tokens = [torch.randn(n + args.steps, hidden, generator=g, device=dev).bfloat16() for n in prompts]

    cu = torch.tensor([0] + prompts, device=dev).cumsum(0).int()
    kv_len = torch.tensor(prompts, dtype=torch.int32, device=dev)
    y = layer.forward(torch.cat([t[:n] for t, n in zip(tokens, prompts)]), cu, kv_len, max(prompts), max(prompts))

    # one token a sequence from here on: the same graph every step, lengths and inputs in place
    cu1 = torch.arange(n_seq + 1, dtype=torch.int32, device=dev)
    x1 = torch.empty(n_seq, hidden, dtype=torch.bfloat16, device=dev)
    graph = torch.cuda.CUDAGraph()
    last = y[(cu[1:] - 1).long()]
    for i in range(args.steps):
        x1.copy_(torch.stack([t[n + i] for t, n in zip(tokens, prompts)]))
        kv_len += 1
        if i == 0:  # once as it is, then captured
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                last = layer.forward(x1, cu1, kv_len, 1, longest)
            torch.cuda.current_stream().wait_stream(side)
            with torch.cuda.graph(graph):
                captured = layer.forward(x1, cu1, kv_len, 1, longest)
        else:
            graph.replay()
            last = captured
    torch.cuda.synchronize()

    worst = 0.0
    for s, t in enumerate(tokens):
        want = reference(weights, t.float(), layer.cos, layer.sin)[-1]
        worst = max(worst, float((last[s].float() - want).norm() / want.norm()))
    print(f"{n_seq} sequences, prompts {args.prompts}, {args.steps} steps: 8-bit outputs within {worst:.3%} of fp32")
    return worst


if __name__ == "__main__":
    main()
