#!/usr/bin/env python3
"""A repaired attention layer that generates text with drafted tokens, on one GPU.

Repairs the q, k, v and o projections of a 3B layer, turns them and a random output head into
e4m3 codes with a scale per block of 128, and runs sequences through turns of

    pages and rows of the step            awsrc_kv_plan
    q, k, v = linear_f8(x)                awsrc_linear_f8
    rotate q and k, append k and v        awsrc_kv_append
    attention over the cache              awsrc_kv_attention
    logits = linear_f8(x + linear_f8(o))  awsrc_linear_f8
    accept drafts, draw the next token    awsrc_verify_drafts

A turn appends each sequence's last token and its drafts; what is refused leaves the cache with the next plan.
Drafts come from the head alone, without attention.  Lengths, page tables and counts stay on the device, no turn waits
for the host.  Half way the first sequence ends and another prompt takes its slot.  At the end the logits of the last
turn are compared with the same model in fp32 on the repaired weights, without any 8-bit rounding.

    python examples/serve_drafts.py [--seeds 16] [--prompts 300,65,1] [--turns 12] [--drafts 4]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import paper_2608_23144_amd as awsrc  # noqa: E402
from serve_layer import HEAD_DIM, PAGE, reference, repaired_weights  # noqa: E402

VOCAB = 4096


class Model:
    """Embedding, one attention layer, head; the layer and the head in e4m3, a paged int8 cache for `slots` sequences."""

    def __init__(self, weights, slots: int, max_tokens: int, n_pages: int, device: str):
        wq, wk, wv, wo = weights
        self.hq, self.hk = wq.shape[0] // HEAD_DIM, wk.shape[0] // HEAD_DIM
        g = torch.Generator(device=device)
        g.manual_seed(1)
        hidden = wq.shape[1]
        self.embed = torch.randn(VOCAB, hidden, generator=g, device=device).bfloat16()
        self.head = (0.05 * torch.randn(VOCAB, hidden, generator=g, device=device)).bfloat16()
        self.qkv8 = awsrc.awsrc_quantize_blocks_f8(torch.cat([wq, wk, wv]), awsrc.BLOCK_F8)
        self.o8 = awsrc.awsrc_quantize_blocks_f8(wo, awsrc.BLOCK_F8)
        self.head8 = awsrc.awsrc_quantize_blocks_f8(self.head, awsrc.BLOCK_F8)
        self.cache = awsrc.make_kv_cache(n_pages, self.hk, HEAD_DIM, PAGE, device)
        self.pool = awsrc.make_page_pool(n_pages, device)
        self.table = torch.zeros(slots, -(-max_tokens // PAGE), dtype=torch.int32, device=device)
        self.kv_len = torch.zeros(slots, dtype=torch.int32, device=device)
        self.max_tokens = max_tokens
        angle = torch.arange(max_tokens, device=device).double()[:, None] * 1e6 ** (
            -torch.arange(0, HEAD_DIM, 2, device=device).double() / HEAD_DIM)
        self.cos, self.sin = torch.cos(angle).float(), torch.sin(angle).float()

    def logits_of(self, x):
        return awsrc.awsrc_linear_f8(x, *self.head8, out_dtype=torch.float32)

    def turn(self, keep, new, tokens, rows: int, max_new: int):
        """Slot s keeps keep[s] cached tokens and appends the first new[s] of tokens[s] ([slots, max_new]).
        Returns the step's row starts, its tokens packed in rows, and the rows' logits."""
        cu, slot, pos, _ = awsrc.awsrc_kv_plan(self.pool, self.kv_len, keep, new, self.table, PAGE, rows)
        at = (pos - keep[slot.clamp_min(0)]).clamp_min(0)
        packed = torch.where(slot >= 0, tokens[slot.clamp_min(0), at], 0).int()
        x = self.embed[packed]
        heads = awsrc.awsrc_linear_f8(x, *self.qkv8).view(rows, self.hq + 2 * self.hk, HEAD_DIM)
        hq, hk = self.hq, self.hk
        q = awsrc.awsrc_kv_append(self.cache, heads[:, hq:hq + hk], heads[:, hq + hk:], cu, self.kv_len, self.table, max_new,
                                  cos=self.cos, sin=self.sin, q=heads[:, :hq])
        a = awsrc.awsrc_kv_attention(self.cache, q, cu, self.kv_len, self.table, max_new, self.max_tokens)
        return cu, packed, self.logits_of(x + awsrc.awsrc_linear_f8(a.view(rows, hq * HEAD_DIM), *self.o8))

    def draft(self, last, n: int, g):
        """n drafts a sequence after its last token, and the distributions that they were drawn from."""
        tokens, probs = [last.long()], []
        for _ in range(n):
            probs.append(torch.softmax(self.logits_of(self.embed[tokens[-1]]), -1))
            tokens.append(torch.multinomial(probs[-1], 1, generator=g)[:, 0])
        return torch.stack(tokens, 1), torch.stack(probs + probs[-1:], 1) if n else None


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--seeds", type=int, default=16, help="seeds of the repair's search")
    ap.add_argument("--prompts", default="300,65,1", help="tokens of each sequence's prompt")
    ap.add_argument("--turns", type=int, default=12, help="turns after the prompts")
    ap.add_argument("--drafts", type=int, default=4, help="drafted tokens of a sequence and turn")
    args = ap.parse_args(argv)
    dev = "cuda"
    prompts = [int(n) for n in args.prompts.split(",")]
    slots, D = len(prompts), args.drafts
    later = prompts[-1] + 7  # tokens of the prompt that takes the first slot half way
    longest = max(prompts + [later]) + args.turns * (D + 1) + D + 1
    weights = repaired_weights(args.seeds, dev)
    n_pages = slots * -(-longest // PAGE)
    model = Model(weights, slots, longest, n_pages, dev)
    g = torch.Generator(device=dev)
    g.manual_seed(2)
    texts = [torch.randint(0, VOCAB, (n,), generator=g, device=dev) for n in prompts]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731

    def prompt(keep, lengths, into):
        """Runs prompts of these lengths (0: the slot waits, its cached tokens stay) and draws each one's next token."""
        padded = torch.zeros(slots, max(lengths), dtype=torch.long, device=dev)
        for s, n in enumerate(lengths):
            if n:
                padded[s, :n] = texts[s][-n:]
        rows = sum(lengths)
        cu, _, logits = model.turn(keep, ints(lengths), padded, rows, max(lengths))
        ran = (cu[1:] > cu[:-1])
        p = torch.softmax(logits[(cu[1:] - 1).clamp_min(0).long()], -1)
        one = torch.arange(slots + 1, dtype=torch.int32, device=dev)
        drawn, _, _ = awsrc.awsrc_verify_drafts(p, torch.zeros(slots, dtype=torch.int32, device=dev),
                                                torch.rand(slots, generator=g, device=dev), one)
        return torch.where(ran, drawn, into)

    last = prompt(torch.zeros(slots, dtype=torch.int32, device=dev), prompts, torch.zeros(slots, dtype=torch.int32, device=dev))
    keep = model.kv_len.clone()
    new = ints([1 + (D if s % 2 == 0 else D // 2) for s in range(slots)])
    rows = int(new.sum())
    out, accepted, offered = [], [], []
    for t in range(args.turns):
        if t == args.turns // 2 and slots > 1:  # the first sequence ends, another prompt takes its slot
            texts[0], out = torch.randint(0, VOCAB, (later,), generator=g, device=dev), out + [None]
            keep = keep * (torch.arange(slots, device=dev) > 0)
            last = prompt(keep, [later] + [0] * (slots - 1), last)
            keep = model.kv_len.clone()
        drafts, q = model.draft(last, D, g)
        cu, packed, logits = model.turn(keep, new, drafts, rows, D + 1)
        p = torch.softmax(logits, -1)
        row_slot = torch.repeat_interleave(torch.arange(slots, device=dev), new.long(), output_size=rows)
        place = torch.arange(rows, device=dev) - cu[row_slot].long()
        tokens, n, keep = awsrc.awsrc_verify_drafts(p, packed, torch.rand(rows, generator=g, device=dev), cu,
                                                    q=None if q is None else q[row_slot, place], kv_len=model.kv_len)
        out.append((cu, last, tokens, n))
        last = tokens[(cu[:-1] + n - 1).long()]
        accepted.append(n - 1)
        offered.append(new - 1)

    torch.cuda.synchronize()
    # the texts as they came out, and the model in fp32 on them
    full = [t.tolist() for t in texts]
    # (what the first slot gave before its sequence ended is not part of its text)
    since = max((i for i, turn in enumerate(out) if turn is None), default=-1)
    for i, turn in enumerate(out):
        if turn is None:
            continue
        cu, before, tokens, n = (x.tolist() for x in turn)
        for s in range(slots):
            if s or i > since:
                full[s] += [before[s]] + tokens[cu[s]:cu[s] + n[s] - 1]
    worst = 0.0
    for s in range(slots):
        ids = torch.tensor(full[s], device=dev)
        # the cache keeps what this turn accepted: the text up to the last accepted token, whose row's logits are the ones to look at
        assert len(ids) == int(keep[s]), (s, len(ids), int(keep[s]))
        x = model.embed[ids].float()
        want = ((x + reference(weights, x, model.cos, model.sin))[-1] @ model.head.float().T)
        got = logits[int(cu[s]) + int(n[s]) - 1]
        worst = max(worst, float((got - want).norm() / want.norm()))
    free = int(model.pool[1])
    held = sum(-(-int(k) // PAGE) for k in model.kv_len.tolist())
    took, gave = int(torch.stack(accepted).sum()), int(torch.stack(offered).sum())
    print(f"{slots} sequences, {args.turns} turns: {took} of {gave} drafts accepted, {held} pages held and {free} free of {n_pages}; "
          f"8-bit logits within {worst:.3%} of fp32")
    return {"worst": worst, "accepted": took, "offered": gave, "pages": (held, free, n_pages)}


if __name__ == "__main__":
    main()
