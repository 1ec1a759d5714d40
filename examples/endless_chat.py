"""Endless conversations on a bounded pool: decode steps of a small stack of
layers whose paged cache is held in 4 bits (or bf16), under a sliding window
with pinned first tokens.

    python examples/endless_chat.py [--cache kv4|bf16] [--steps N] [--forks F] ...

What a serving loop does around its layers, all of it on the device:

1. prompts arrive and are quantised into their pages (``kv4_append``);
2. every conversation is forked into several continuations that share its
   pages (``pages_update`` with parents, ``pages_copy`` for the pages that a
   continuation will write into);
3. every step the table of the next one gives each sequence room for its token
   and releases the pages that window and sinks have left behind
   (``pages_update``), and each layer runs prelude, append, attention and
   output projection;
4. the first continuation of each conversation is kept, the others are freed,
   and the pages left are moved to the front of the pool (``pages_compact``,
   ``pages_copy``), which changes no output.

Weights, prompts and the first hidden states are random; the sizes are those
of a small layer with 32:8 heads.
"""
from __future__ import annotations

import argparse
import sys
import time
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))
from paper_2606_07665_amd import binding as pda  # noqa: E402

HQ, HKV, D, HIDDEN = 32, 8, 128, 512
THETA = 5e5


class Layer:
    """One layer's weights, and its K and V pools in either form."""

    def __init__(self, kv4, num_pages, page, gen):
        def bf16(*shape, std):
            return (torch.randn(shape, device="cuda", generator=gen) * std).bfloat16()

        self.w_qkv = pda.pack_weights(bf16((HQ + 2 * HKV) * D, HIDDEN, std=HIDDEN ** -0.5))
        self.w_o = pda.pack_weights(bf16(HIDDEN, HQ * D, std=(HQ * D) ** -0.5))
        self.norm = torch.ones(HIDDEN, dtype=torch.bfloat16, device="cuda")
        self.kv4 = kv4
        if kv4:
            self.pools = [*pda.kv4_cache(num_pages, page, HKV, D), *pda.kv4_cache(num_pages, page, HKV, D)]
        else:
            self.pools = [torch.zeros((num_pages, page, HKV, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def append(self, k, v, table, lens):
        (pda.kv4_append if self.kv4 else pda.kv_append_n)(k, v, *self.pools, table, lens)

    def attend(self, q, table, lens, window, sinks):
        out = torch.empty_like(q)
        call = pda.paged_decode_attention_kv4 if self.kv4 else pda.paged_decode_attention_sink
        return call(q, *self.pools, table, lens, out, D ** -0.5, window, sinks)

    def step(self, x, residual, table, lens, window, sinks):
        """One token of every sequence: (its queries, the attention, the next layer's input); residual is updated."""
        b = x.shape[0]
        dims = dict(num_q_heads=HQ, num_kv_heads=HKV, head_dim=D, rope_theta=THETA)
        q = torch.empty((b, HQ, D), dtype=torch.bfloat16, device="cuda")
        if self.kv4:
            k, v = (torch.empty((b, HKV, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            pda.attention_prelude(x, self.w_qkv, lens, q, k, v, **dims)
            self.append(k[:, None], v[:, None], table, lens)
        else:
            pda.attention_prelude_append(x, self.w_qkv, lens, q, *self.pools, table, **dims)
        q = q[:, None]
        out = self.attend(q, table, lens, window, sinks)
        pda.o_proj_residual_norm(out.reshape(b, HQ * D), self.w_o, residual, self.norm, residual, h := torch.empty_like(x))
        return q, out, h


class Pages:
    """The block table, lengths and page counts of a pool, and the pools that go with them."""

    def __init__(self, num_pages, page, max_pages, window, sinks, pools):
        self.page, self.window, self.sinks, self.pools = page, window, sinks, pools
        self.refcount = torch.zeros(num_pages, dtype=torch.int32, device="cuda")
        self.table = torch.full((1, max_pages), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.lacking = torch.zeros(1, dtype=torch.int32, device="cuda")

    def update(self, new_lens, parents=None):
        """Rows of ``new_lens`` tokens that continue ``parents`` (None: row by row)."""
        rows, dev = new_lens.shape[0], dict(dtype=torch.int32, device="cuda")
        table, ref = torch.empty((rows, self.table.shape[1]), **dev), torch.empty_like(self.refcount)
        src, dst, info = torch.empty(rows, **dev), torch.empty(rows, **dev), torch.empty(2, **dev)
        pda.pages_update(self.table, self.lens, parents, new_lens, self.refcount, table, ref, src, dst, info, self.page,
                         self.window, self.sinks)
        pda.pages_copy(self.pools, src, dst)
        self.table, self.refcount, self.lens = table, ref, new_lens
        self.lacking += info[1:]

    def compact(self):
        """Every live page to the front of the pools; (live pages, pages moved) on the device."""
        dev = dict(dtype=torch.int32, device="cuda")
        table, ref, page_map = (torch.empty_like(t) for t in (self.table, self.refcount, self.refcount))
        src, dst, info = torch.empty_like(ref), torch.empty_like(ref), torch.empty(2, **dev)
        pda.pages_compact(self.table, self.lens, self.refcount, table, ref, page_map, src, dst, info, self.page)
        pda.pages_copy(self.pools, src, dst, count=info[1:])
        self.table, self.refcount = table, ref
        return info

    def live(self):
        return int((self.refcount > 0).sum())


def run(cache="kv4", conversations=4, prompt=300, forks=3, steps=400, window=256, sinks=4, page=16, layers=2, seed=0,
        log=print):
    """The loop above; returns the last step's tensors and what compaction left unchanged."""
    for name, n in (("conversations", conversations), ("prompt", prompt), ("forks", forks), ("steps", steps), ("layers", layers)):
        if n < 1:
            raise ValueError(f"{name} must be at least 1, got {n}")
    pda.load()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows = conversations * forks
    max_pages = -(-(prompt + steps) // page)
    # Pages of a row at most: all of them, or its window and its sinks, wherever they start in their pages.
    held = max_pages if window <= 0 else min(max_pages, -(-window // page) + 1 + -(-sinks // page))
    num_pages = conversations * -(-prompt // page) + rows * held
    stack = [Layer(cache == "kv4", num_pages, page, gen) for _ in range(layers)]
    pages = Pages(num_pages, page, max_pages, window, sinks, [p for layer in stack for p in layer.pools])

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    # 1. The prompts.
    pages.update(ints([prompt] * conversations), ints([-1] * conversations))
    for layer in stack:
        k, v = (torch.randn((conversations, prompt, HKV, D), device="cuda", generator=gen).bfloat16() for _ in range(2))
        layer.append(k, v, pages.table, pages.lens)
    # 2. The forks, each with room for its first token.
    pages.update(ints([prompt + 1] * rows), ints([r // forks for r in range(rows)]))
    log(f"{conversations} prompts of {prompt} tokens, forked {forks} ways: {pages.live()} of {num_pages} pages live")
    # 3. The steps.
    x = torch.randn((rows, HIDDEN), device="cuda", generator=gen).bfloat16()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for step in range(steps):
        if step:
            pages.update(pages.lens + 1)
        residual, h = x.clone(), x
        for layer in stack:
            q, out, h = layer.step(h, residual, pages.table, pages.lens, window, sinks)
        x = h
    torch.cuda.synchronize()
    us = (time.perf_counter() - t0) / max(steps, 1) * 1e6
    if int(pages.lacking):
        raise RuntimeError(f"the pool lacked {int(pages.lacking)} pages")
    log(f"{steps} steps of {rows} sequences, {layers} layers: {us:.0f} us a step, {pages.live()} pages live at "
        f"{prompt + steps} tokens")
    # 4. One continuation of each conversation, at the front of the pool.
    first = torch.arange(0, rows, forks, device="cuda", dtype=torch.int32)
    pages.update(pages.lens[first.long()].contiguous(), first)
    keep = q[first.long()].contiguous()
    before = stack[-1].attend(keep, pages.table, pages.lens, window, sinks)
    scattered = int(pages.table.max()) + 1
    info = pages.compact()
    after = stack[-1].attend(keep, pages.table, pages.lens, window, sinks)
    n, moved = info.tolist()
    log(f"kept {conversations}: {n} live pages of the first {scattered}, {moved} moved to the front; same output: "
        f"{torch.equal(before, after)}")
    return dict(q=keep, out=out[first.long()], before=before, after=after, layer=stack[-1], pages=pages, live=n, x=x)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--cache", choices=("kv4", "bf16"), default="kv4")
    for name, default in (("conversations", 4), ("prompt", 300), ("forks", 3), ("steps", 400), ("window", 256),
                          ("sinks", 4), ("page", 16), ("layers", 2), ("seed", 0)):
        ap.add_argument(f"--{name}", type=int, default=default)
    run(**vars(ap.parse_args(argv)))


if __name__ == "__main__":
    main()
