"""The operators of a long-lived, small KV cache, as measurable cases.

Four kinds of pass, each what a serving program does between or inside decode
steps:

* ``append4``: the new tokens' keys and values are quantised to 4 bits (E2M1
  elements, one E8M0 power of two per 32) into their pages, and read back as
  the bf16 values they now stand for, as a chunk of prefill attends to them;
* ``attn4``: paged decode attention over such a 4-bit cache, one or several
  query tokens, with or without a sliding window and sinks;
* ``sink``: paged decode attention over a bf16 cache with a sliding window and
  a few first tokens that stay visible;
* ``fork`` and ``compact``: sequences are continued by one or several rows with
  their pages shared, or the live pages are moved to the front of the pool;
  then the pages that this moves are copied in every layer's pools.

A case fixes the set of context lengths; the seed decides which sequence has
which, where the pages lie in the pool, and every value.
"""
from __future__ import annotations

import math

import numpy as np
import torch

#: False: ``run`` computes the operators with elementary torch operations; True: with the library.
own = False

#: The values of the 16 E2M1 codes: sign, two exponent bits, one mantissa bit.
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)
GROUP = 32  # elements that share a scale


def _append4(**kw):
    return dict(dict(kind="append4", batch=1, tokens=1, hkv=8, d=128, page=16, lengths="fixed:4096"), **kw)


def _attn(kind, **kw):
    return dict(dict(kind=kind, batch=1, hq=32, hkv=8, d=128, page=16, lengths="fixed:4096", capacity=0,
                     queries=1, window=0, sinks=0, empty=0), **kw)


def _fork(**kw):
    return dict(dict(kind="fork", batch=8, ended=0, children=4, grow=1, hkv=8, d=128, page=16, lengths="uniform:128:8192",
                     bits=4, layers=2), **kw)


def _compact(**kw):
    return dict(dict(kind="compact", batch=64, moved=1000, hkv=8, d=128, page=16, lengths="uniform:128:8192",
                     bits=16, layers=1), **kw)


def listed():
    return [
        # the newest token of a serving batch goes into the cache: latency
        _append4(name="append4_decode_b64", batch=64, lengths="uniform:128:8192"),
        # two prompts of odd length are written as they arrive: bandwidth
        _append4(name="append4_prompt_2x4095", batch=2, tokens=4095, lengths="fixed:4095"),
        # one interactive request on an 8B model, half-way through its 8192-token table: latency
        _attn("attn4", name="attn4_single_8b", capacity=8192),
        # continuous batching on an 8B model: ordinary serving
        _attn("attn4", name="attn4_batched_8b", batch=64, lengths="uniform:128:8192"),
        # a few very long documents on a 70B model: the largest
        _attn("attn4", name="attn4_long_70b", batch=4, hq=64, lengths="fixed:131072"),
        # three drafted tokens to verify at 40:8 heads, an odd batch with a heavy tail and an idle slot
        _attn("attn4", name="attn4_draft3_ragged", batch=101, hq=40, page=32, lengths="zipf:1.2:16:32768", queries=3,
              empty=1),
        # head size 256 under a sliding window with sinks
        _attn("attn4", name="attn4_d256_sink", batch=16, hq=12, hkv=4, d=256, lengths="uniform:16:32768", window=4096,
              sinks=4),
        # one endless chat in a bf16 cache: a short window and four sinks, latency
        _attn("sink", name="sink_single", lengths="fixed:20001", window=1024, sinks=4),
        # a batch of long conversations under a 4096-token window and four sinks
        _attn("sink", name="sink_batched", batch=64, lengths="uniform:1024:16384", window=4096, sinks=4),
        # drafted tokens under a window with a whole system prompt pinned
        _attn("sink", name="sink_draft4_pinned", batch=33, lengths="uniform:300:32768", queries=4, window=2000, sinks=77),
        # eight of ten sequences go on four ways each, two have ended, in a 4-bit cache of four layers
        _fork(name="fork_8x4", batch=10, ended=2, layers=4),
        # a batch's bf16 pages moved to the front of a fragmented pool
        _compact(name="compact_b64", batch=64, moved=4000),
    ]


# (query heads, kv heads, head size): the head layouts of the repository's workloads
_HEADS = ((32, 8, 128), (32, 8, 128), (64, 8, 128), (40, 8, 128), (32, 2, 128), (12, 4, 256), (8, 2, 64))


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _draw_lengths(rng, batch, mean):
    mean = max(1, min(131072, int(mean)))
    form = rng.choice(("fixed", "uniform", "uniform", "zipf"))
    if batch == 1 or form == "fixed" or mean < 32:
        return "fixed:%d" % mean
    if form == "zipf" and batch >= 16:
        return "zipf:1.2:16:%d" % min(32768, 2 * mean + 16)
    return "uniform:%d:%d" % (max(1, mean // 8), 2 * mean - max(1, mean // 8))


def draw(rng):
    kind = rng.choice(("append4",) * 2 + ("attn4",) * 5 + ("sink",) * 3 + ("fork", "compact"))
    hq, hkv, d = rng.choice(_HEADS)
    page = rng.choice((16, 16, 32, 64))
    if kind == "append4":
        total = _log_int(rng, 1, 16384)  # new tokens of the call
        tokens = _log_int(rng, 1, total) if rng.random() < 0.6 else 1
        batch = max(1, min(256, total // tokens))
        return _append4(batch=batch, tokens=tokens, hkv=hkv, d=d, page=page,
                        lengths="fixed:%d" % (tokens + rng.randint(0, 2000)))
    batch = _log_int(rng, 1, 256)
    if kind in ("attn4", "sink"):
        c = _attn(kind, batch=batch, hq=hq, hkv=hkv, d=d, page=page)
        if rng.random() < 0.4:
            c["queries"] = rng.randint(1, max(1, min(8, 16 // (hq // hkv))))
        if kind == "sink" or rng.random() < 0.3:
            c["window"] = rng.choice((100, 512, 1024, 2048, 4096))
            c["sinks"] = rng.choice((1, 4, 4, 16, 77))
        if batch > 4 and rng.random() < 0.2:
            c["empty"] = 1
        token = 4 * hkv * d if kind == "sink" else hkv * d * 17 // 16  # bytes of K and V per token
        seen = math.exp(rng.uniform(math.log(2e5), math.log(5e8))) / (batch * token)
        if c["window"]:
            seen = min(131072, rng.uniform(1, 6) * min(seen, c["window"]))
        c["lengths"] = _draw_lengths(rng, batch, seen)
        if batch <= 8:
            c["capacity"] = int(max(_lens(c))) * rng.choice((1, 1, 2))
        return c
    if kind == "fork":
        batch = _log_int(rng, 1, 32)
        return _fork(batch=batch, ended=rng.randint(0, batch // 3), children=rng.randint(1, max(1, min(8, 128 // batch))), grow=rng.choice((1, 1, 1, 5, 40)),
                     hkv=hkv, d=d, page=page, lengths=_draw_lengths(rng, batch, _log_int(rng, 32, 4096)),
                     bits=rng.choice((4, 16)), layers=rng.randint(1, 4))
    c = _compact(batch=batch, hkv=hkv, d=d, page=page, bits=rng.choice((4, 16)),
                 lengths=_draw_lengths(rng, batch, _log_int(rng, 32, 200000) / batch))
    c["moved"] = _log_int(rng, 1, max(1, min(3000, _live_pages(c) // 2)))
    return c


# ------------------------------------------------------------------ inputs
def _lens(case):
    """The case's context lengths, the new tokens included."""
    b = case["batch"]
    kind, *args = case["lengths"].split(":")
    if kind == "fixed":
        lens = np.full(b, int(args[0]), dtype=np.int64)
    elif kind == "uniform":
        lo, hi = int(args[0]), int(args[1])
        lens = (lo + (hi - lo) * (np.arange(b) + 0.5) / b).astype(np.int64)
    else:
        s, lo, hi = float(args[0]), int(args[1]), int(args[2])
        lens = np.clip(np.random.default_rng([b, hi]).zipf(s, size=b).astype(np.int64), lo, hi)
    lens = np.maximum(lens, case.get("queries", case.get("tokens", 1)))
    if case.get("empty"):
        lens[:case["empty"]] = 0
    return lens


def _live_pages(case):
    return int((-(-_lens(case) // case["page"])).sum())


def _visible(case, length):
    """The tokens that some query of a sequence sees: [0, pinned) and [first, length)."""
    if not case["window"]:
        return 0, 0
    first = max(0, length - case["queries"] + 1 - case["window"])
    return min(case["sinks"], first), first


def _table(case, seed):
    """(block table, lengths, pages in the pool): pages of a shuffled pool with a tenth of it unused; pages
    that a window and its sinks leave invisible have been released (-1)."""
    rng = np.random.default_rng([seed, 7])
    lens = rng.permutation(_lens(case))
    page = case["page"]
    held = []
    for n in lens:
        j = np.arange(-(-int(n) // page))
        if case.get("window"):
            pinned, first = _visible(case, int(n))
            j = j[(j * page < pinned) | ((j + 1) * page > first)]
        held.append(j)
    used = int(sum(len(j) for j in held))
    pool = used + used // 10 + 1
    width = max(1, -(-int(lens.max()) // page), -(-case.get("capacity", 0) // page))
    ids = rng.permutation(pool)
    table = np.full((case["batch"], width), -1, dtype=np.int32)
    at = 0
    for i, j in enumerate(held):
        table[i, j] = ids[at:at + len(j)]
        at += len(j)
    return table, lens.astype(np.int32), pool


class _Values:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(1_000_003 * (seed + 1))
        u = (torch.arange(256, dtype=torch.float64) + 0.5) / 256
        code = _round_e2m1((2.0 * torch.special.ndtri(u)).float())  # normal values in units of half their deviation
        self.pairs = (code[None, :] | (code[:, None] << 4)).reshape(-1).cuda()

    def normal(self, *shape, std=1.0):
        return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=self.gen)

    def _ints(self, n, hi):
        return torch.randint(hi, (n,), dtype=torch.int32, device="cuda", generator=self.gen)

    def cache4(self, pool, hkv, d, page):
        """Codes and scales of a cache of normal keys or values, as quantising them leaves it."""
        shape = (pool, hkv, d // GROUP, page, GROUP // 2)
        codes = torch.empty(math.prod(shape), dtype=torch.uint8, device="cuda")
        for part in codes.split(1 << 27):
            part.copy_(self.pairs[self._ints(part.numel(), 65536)])
        spread = torch.tensor([125, 126, 126, 126, 126, 126, 126, 127], dtype=torch.uint8, device="cuda")
        return codes.view(shape), spread[self._ints(math.prod(shape) // 16, 8)].view(shape[:-1])

    def bytes(self, *shape):
        return self._ints(math.prod(shape), 256).to(torch.uint8).view(shape)


def _gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _pools(case, pool, v):
    """Every layer's K and V pools (their codes and scales with 4 bits)."""
    n, h, d, p = pool, case["hkv"], case["d"], case["page"]
    if case["bits"] == 16:
        return [v.normal(n, p, h, d) for _ in range(2 * case["layers"])]
    out = []
    for _ in range(2 * case["layers"]):
        out += [v.bytes(n, h, d // GROUP, p, GROUP // 2), v.bytes(n, h, d // GROUP, p)]
    return out


def _fork_pages(case):
    """Pages of each parent, pages with the new tokens, and pages in the pool."""
    lens, page = _lens(case), case["page"]
    pages, grown = -(-lens // page), -(-(lens + case["grow"]) // page)
    return pages, grown, int(pages.sum()) + case["children"] * int((grown - pages + 1).sum()) + 8


def _fork_inputs(case, seed):
    """Parents in shuffled pages of a pool, one page of each shared with a cache of prompts; all but the
    ``ended`` ones continue as ``children`` rows in a shuffled order, each with ``grow`` tokens more."""
    rng = np.random.default_rng([seed, 8])
    page, b = case["page"], case["batch"]
    order = rng.permutation(b)
    lens = _lens(case)[order].astype(np.int32)
    pages, grown, pool = _fork_pages(case)
    pages, grown = pages[order], grown[order]
    table = np.full((b, int(grown.max())), -1, dtype=np.int32)
    ids = rng.permutation(pool)
    refcount = np.zeros(pool, dtype=np.int32)
    at = 0
    for i, n in enumerate(pages):
        table[i, :n] = ids[at:at + n]
        at += int(n)
    refcount[ids[:at]] = 1
    for i in range(b):
        if lens[i] >= 2 * page:
            refcount[table[i, 0]] += 1
    parents = rng.permutation(np.repeat(np.flatnonzero(order >= case["ended"]).astype(np.int32), case["children"]))
    return table, lens, refcount, parents, (lens[parents] + case["grow"]).astype(np.int32), pool


def _compact_inputs(case, seed):
    """``moved`` of the live pages lie past the place where the live ones would end."""
    rng = np.random.default_rng([seed, 9])
    page = case["page"]
    lens = rng.permutation(_lens(case)).astype(np.int32)
    pages = -(-lens.astype(np.int64) // page)
    live = int(pages.sum())
    moved = min(case["moved"], live)
    pool = live + 2 * moved
    low = rng.permutation(live)[moved:]
    high = live + rng.permutation(pool - live)[:moved]
    ids = rng.permutation(np.concatenate([low, high]))
    table = np.full((case["batch"], int(pages.max())), -1, dtype=np.int32)
    at = 0
    for i, n in enumerate(pages):
        table[i, :n] = ids[at:at + n]
        at += int(n)
    refcount = np.zeros(pool, dtype=np.int32)
    refcount[ids] = 1 + (rng.random(live) < 0.2)  # some held by others too
    return table, lens, refcount, pool


def _inputs(case, seed):
    """Everything the seed decides."""
    v = _Values(seed)
    kind, b = case["kind"], case["batch"]
    s = dict(case=case)
    if kind == "fork":
        table, lens, refcount, parents, new_lens, pool = _fork_inputs(case, seed)
        s.update(parents=_gpu(parents), new_lens=_gpu(new_lens), refcount=_gpu(refcount), pools=_pools(case, pool, v))
    elif kind == "compact":
        table, lens, refcount, pool = _compact_inputs(case, seed)
        s.update(refcount=_gpu(refcount), pools=_pools(case, pool, v))
    else:
        table, lens, pool = _table(case, seed)
        if kind == "append4":
            shape = (b, case["tokens"], case["hkv"], case["d"])
            s.update(k_new=v.normal(*shape), v_new=v.normal(*shape))
            for t in (s["k_new"], s["v_new"]):  # a few channels much larger than the rest, as keys have them
                t[..., 3::61] *= 8
        else:
            s["q"] = v.normal(b, case["queries"], case["hq"], case["d"])
        if kind == "sink":
            shape = (pool, case["page"], case["hkv"], case["d"])
            s.update(k=v.normal(*shape), v=v.normal(*shape))
        else:
            s["k"], s["k_scales"] = v.cache4(pool, case["hkv"], case["d"], case["page"])
            s["v"], s["v_scales"] = v.cache4(pool, case["hkv"], case["d"], case["page"])
    s.update(table=_gpu(table), lens=_gpu(lens), host_lens=[int(n) for n in lens])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind in ("attn4", "sink"):
        s["out"] = torch.empty_like(s["q"])
        s["scale"] = case["d"] ** -0.5
    if kind == "append4":
        s["k_back"], s["v_back"] = torch.empty_like(s["k_new"]), torch.empty_like(s["v_new"])
    if kind in ("fork", "compact"):
        rows = s["parents"].numel() if kind == "fork" else case["batch"]
        moves = rows if kind == "fork" else s["refcount"].numel()
        s["table_out"] = torch.empty((rows, s["table"].shape[1]), dtype=torch.int32, device="cuda")
        s["refcount_out"] = torch.empty_like(s["refcount"])
        s["src"], s["dst"] = (torch.empty(moves, dtype=torch.int32, device="cuda") for _ in range(2))
        s["info"] = torch.empty(2, dtype=torch.int32, device="cuda")
        if kind == "compact":
            s["page_map"] = torch.empty_like(s["refcount"])
    return s


# -------------------------------------------------------------------- pass
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2606_07665_amd import binding as pda
    case = s["case"]
    kind = case["kind"]
    if kind == "append4":
        cache = (s["k"], s["k_scales"], s["v"], s["v_scales"], s["table"], s["lens"])
        pda.kv4_append(s["k_new"], s["v_new"], *cache)
        pda.kv4_read(s["k_back"], s["v_back"], *cache)
        return s["k_back"], s["v_back"]
    if kind == "attn4":
        return pda.paged_decode_attention_kv4(s["q"], s["k"], s["k_scales"], s["v"], s["v_scales"], s["table"], s["lens"],
                                              s["out"], s["scale"], window=case["window"], sinks=case["sinks"])
    if kind == "sink":
        return pda.paged_decode_attention_sink(s["q"], s["k"], s["v"], s["table"], s["lens"], s["out"], s["scale"],
                                               window=case["window"], sinks=case["sinks"])
    if kind == "fork":
        pda.pages_update(s["table"], s["lens"], s["parents"], s["new_lens"], s["refcount"], s["table_out"],
                         s["refcount_out"], s["src"], s["dst"], s["info"], page_size=case["page"])
        pda.pages_copy(s["pools"], s["src"], s["dst"])
        return s["table_out"], s["refcount_out"], s["src"], s["dst"], s["info"], s["pools"]
    pda.pages_compact(s["table"], s["lens"], s["refcount"], s["table_out"], s["refcount_out"], s["page_map"], s["src"],
                      s["dst"], s["info"], page_size=case["page"])
    pda.pages_copy(s["pools"], s["src"], s["dst"], count=s["info"][1:])
    return s["table_out"], s["refcount_out"], s["page_map"], s["src"], s["dst"], s["info"], s["pools"]


# The plain forms: elementary torch operations in 32 bits.
def _round_e2m1(x):
    """The E2M1 codes of x, to the nearest value, ties to the even code, 6 where it is past 6."""
    m = x.abs()
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0))
    return code.to(torch.uint8) | (torch.signbit(x).to(torch.uint8) << 3)


def _plain_quantise(x):
    """bf16 [..., D] -> codes [..., D / 32, 16] and scales [..., D / 32]."""
    g = x.unflatten(-1, (-1, GROUP))
    exponent = (g.view(torch.int16).to(torch.int32) >> 7) & 255
    scale = (exponent.amax(-1) - 2).clamp_min(0)  # the largest element lies in [4, 8) units
    code = _round_e2m1(g.float() * torch.exp2((127 - scale).float()).unsqueeze(-1))
    return code[..., 0::2] | (code[..., 1::2] << 4), scale.to(torch.uint8)


def _plain_values(codes, scales, values):
    """Codes [..., 16] and scales [...] -> fp32 [..., 32]."""
    both = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2)
    return values[both.int()] * torch.exp2(scales.float() - 127.0).unsqueeze(-1)


def _slots(case, table, lens, count):
    """Page and slot of each sequence's last ``count`` tokens, [B, count]."""
    t = lens.long()[:, None] - count + torch.arange(count, device="cuda")
    return torch.gather(table.long(), 1, t // case["page"]), t % case["page"]


def _plain_append4(s, values):
    pages, slots = _slots(s["case"], s["table"], s["lens"], s["case"]["tokens"])
    out = []
    for new, codes, scales in ((s["k_new"], s["k"], s["k_scales"]), (s["v_new"], s["v"], s["v_scales"])):
        q, e = _plain_quantise(new)  # [B, T, Hkv, D / 32, ...]
        codes.permute(0, 3, 1, 2, 4)[pages, slots] = q
        scales.permute(0, 3, 1, 2)[pages, slots] = e
        back = _plain_values(codes.permute(0, 3, 1, 2, 4)[pages, slots], scales.permute(0, 3, 1, 2)[pages, slots], values)
        out.append(back.flatten(-2).to(torch.bfloat16))
    return tuple(out)


def _plain_rows(s, ids, which, values):
    """fp32 [B, Hkv, tokens, D] of each sequence's listed pages [B, pages]."""
    if s["case"]["kind"] == "sink":
        return s[which][ids].flatten(1, 2).transpose(1, 2).float()
    x = _plain_values(s[which][ids], s[which + "_scales"][ids], values)  # [B, pages, Hkv, D / 32, P, 32]
    return x.permute(0, 2, 1, 4, 3, 5).flatten(4).flatten(2, 3)


def _plain_attention(s, values):
    case = s["case"]
    page, nq, w, hkv = case["page"], case["queries"], case["window"], case["hkv"]
    group = case["hq"] // hkv
    lens, table = s["lens"].long(), s["table"].long()
    width = table.shape[1]
    if w:  # the pages of the sinks, then those of the window; a page that is in both counts among the first
        pinned = min(width, -(-case["sinks"] // page))
        first = (lens - nq + 1 - w).clamp_min(0) // page
        tail = first[:, None] + torch.arange(min(width, (w + nq) // page + 2), device="cuda")
        j = torch.cat((torch.arange(pinned, device="cuda").expand(lens.numel(), -1), tail), dim=1)
        here = torch.cat((torch.ones_like(j[:, :pinned], dtype=torch.bool), (tail >= pinned) & (tail < width)), dim=1)
    else:
        j = torch.arange(width, device="cuda").expand(lens.numel(), -1)
        here = torch.ones_like(j, dtype=torch.bool)
    ids = torch.gather(table, 1, j.clamp_max(width - 1)).clamp_min(0)
    t = (j[:, :, None] * page + torch.arange(page, device="cuda")).flatten(1)[:, None, None, :]
    here = here.repeat_interleave(page, 1)[:, None, None, :]
    q = s["q"].float().unflatten(2, (hkv, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [B, Hkv, nq * G, D]
    at = lens[:, None] - nq + torch.arange(nq, device="cuda").repeat_interleave(group)
    at = at[:, None, :, None]
    sees = here & (t <= at)
    if w:
        sees = sees & ((t > at - w) | (t < case["sinks"]))
    score = torch.matmul(q, _plain_rows(s, ids, "k", values).transpose(2, 3)) * s["scale"]
    score = torch.where(sees, score, torch.full_like(score, -math.inf))
    top = score.amax(-1, keepdim=True).clamp_min(-1e30)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, _plain_rows(s, ids, "v", values)) / torch.where(total > 0, total, torch.ones_like(total))
    return o.unflatten(2, (nq, group)).transpose(1, 2).flatten(2, 3).to(torch.bfloat16)


def _plain_fork(s):
    case = s["case"]
    page, table, lens = case["page"], s["table"].long(), s["lens"].long()
    n, m = s["refcount"].numel(), table.shape[1]
    parents, new = s["parents"].long(), s["new_lens"].long()
    j = torch.arange(m, device="cuda")
    used = table[j[None, :] < -(-lens[:, None] // page)]
    outside = s["refcount"].long() - torch.bincount(used, minlength=n)  # held by others than this table
    kept = torch.minimum(lens[parents], new)
    rows = table[parents]
    full = j[None, :] < (kept // page)[:, None]
    last = kept // page
    part = kept % page != 0
    writes = part & (new > kept)
    shared = full | ((j[None, :] == last[:, None]) & (part & ~writes)[:, None])
    holders = outside + torch.bincount(rows[shared], minlength=n)
    tail = torch.gather(rows, 1, last.clamp_max(m - 1)[:, None])[:, 0]  # the page each writer would write into
    r = torch.arange(parents.numel(), device="cuda")
    lowest = torch.full((n,), parents.numel(), device="cuda").scatter_reduce(0, tail[writes], r[writes], "amin")
    keeps = writes & (holders[tail] == 0) & (lowest[tail] == r)
    copies = writes & ~keeps
    holders[tail[keeps]] += 1
    first_new = -(-kept // page)
    count = copies.long() + -(-new // page) - first_new
    fresh = torch.nonzero(holders == 0)[:, 0]
    want = int(count.sum())
    given = torch.full((max(1, want),), -1, dtype=torch.long, device="cuda")
    given[:min(want, fresh.numel())] = fresh[:want]
    start = torch.cumsum(count, 0) - count
    index = start[:, None] + copies[:, None].long() + j[None, :] - first_new[:, None]
    grown = (j[None, :] >= first_new[:, None]) & (j[None, :] < -(-new // page)[:, None])
    out = torch.full_like(rows, -1)
    out = torch.where(shared | ((j[None, :] == last[:, None]) & keeps[:, None]), rows, out)
    out = torch.where(grown, given[index.clamp(0, given.numel() - 1)], out)
    dst = torch.where(copies, given[start.clamp_max(given.numel() - 1)], torch.full_like(tail, -1))
    out = torch.where((j[None, :] == last[:, None]) & copies[:, None], dst[:, None], out)
    src = torch.where(dst >= 0, tail, torch.full_like(tail, -1))
    holders[fresh[:want]] = 1
    info = torch.tensor([min(want, fresh.numel()), want - min(want, fresh.numel())], dtype=torch.int32, device="cuda")
    take = dst >= 0
    for pool in s["pools"]:
        pool[dst[take]] = pool[src[take]]
    return out.int(), holders.int(), src.int(), dst.int(), info, s["pools"]


def _plain_compact(s):
    refcount, page, table = s["refcount"], s["case"]["page"], s["table"].long()
    n = refcount.numel()
    ids = torch.arange(n, device="cuda")
    live = refcount > 0
    total = int(live.sum())
    src, dst = ids[live & (ids >= total)], ids[~live & (ids < total)]
    page_map = torch.where(live, ids, torch.full_like(ids, -1))
    page_map[src] = dst
    counts = torch.zeros_like(refcount)
    counts[page_map[live]] = refcount[live]
    used = torch.arange(table.shape[1], device="cuda")[None, :] < -(-s["lens"].long()[:, None] // page)
    out = torch.where(used, page_map[table.clamp_min(0)], torch.full_like(table, -1))
    pairs = torch.full((2, n), -1, dtype=torch.int32, device="cuda")
    pairs[0, :src.numel()], pairs[1, :src.numel()] = src.int(), dst.int()
    info = torch.tensor([total, src.numel()], dtype=torch.int32, device="cuda")
    for pool in s["pools"]:
        pool[dst] = pool[src]
    return out.int(), counts, page_map.int(), pairs[0], pairs[1], info, s["pools"]


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "fork":
        return _plain_fork(s)
    if kind == "compact":
        return _plain_compact(s)
    values = torch.tensor(E2M1, dtype=torch.float32, device="cuda")
    return _plain_append4(s, values) if kind == "append4" else _plain_attention(s, values)


# ---------------------------------------------------------- what it cannot do without
def work(case):
    kind, b = case["kind"], case["batch"]
    heads = case["hkv"] * case["d"]
    cached = heads * 17 // 16  # bytes of a token's K and V in 4 bits
    if kind == "append4":
        n = b * case["tokens"]
        # K and V in, their cached form written and read, the values out
        return {"bytes": n * (8 * heads + 2 * cached) + 8 * b + 8 * (n // case["page"] + b), "flops": 4 * n * heads}
    if kind in ("attn4", "sink"):
        tokens = 0
        for n in _lens(case):
            pinned, first = _visible(case, int(n))
            tokens += int(n) - first + pinned
        q = 2 * b * case["queries"] * case["hq"] * case["d"]
        token = 4 * heads if kind == "sink" else cached
        return {"bytes": tokens * token + 2 * q + 4 * (tokens // case["page"] + b) + 4 * b,
                "flops": 4 * case["queries"] * case["hq"] * case["d"] * tokens}
    lens, page = _lens(case), case["page"]
    pages = -(-lens // page)
    one = page * heads * (2 if case["bits"] == 16 else 17 / 32) * 2 * case["layers"]  # K and V of a page, all layers
    if kind == "fork":
        pages, grown, pool = _fork_pages(case)
        on = slice(case["ended"], None)
        copies = int((lens[on] % page != 0).sum()) * (case["children"] - 1)
        entries = int(pages.sum()) + case["children"] * int(grown[on].sum())
        return {"bytes": int(2 * copies * one) + 4 * entries + 8 * pool, "flops": 0}
    live = int(pages.sum())
    moved = min(case["moved"], live)
    return {"bytes": int(2 * moved * one) + 8 * live + 12 * (live + 2 * moved), "flops": 0}


# ------------------------------------------------------------------ in 64 bits
def _exact_e2m1(x):
    """x to the nearest E2M1 value, of two as near the one with the even code (64 bits)."""
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    out = torch.empty_like(x)
    for a, o in zip(x.reshape(-1).split(1 << 24), out.view(-1).split(1 << 24)):
        d = (a.abs()[:, None] - grid).abs()
        best = d.amin(1, keepdim=True)
        order = torch.tensor([0, 4, 1, 5, 2, 6, 3, 7], device=x.device)  # even codes first
        pick = torch.where(d == best, order, torch.full_like(order, 99)).argmin(1)
        o.copy_(torch.copysign(grid[pick], a))
    return out


def _exact_append4(s):
    out = []
    for new in (s["k_new"], s["v_new"]):
        g = new.double().unflatten(-1, (-1, GROUP))
        top = g.abs().amax(-1, keepdim=True)
        _, exponent = torch.frexp(top.clamp_min(2.0 ** -125))  # top = m 2^exponent, 0.5 <= m < 1
        unit = torch.ldexp(torch.ones_like(top), exponent - 3)
        out.append((_exact_e2m1(g / unit) * unit).flatten(-2))
    return tuple(out)


def _exact_token_values(s, which, ids):
    """fp64 [tokens, Hkv, D] of pages in order."""
    if s["case"]["kind"] == "sink":
        x = s[which][ids].double()
        return x.reshape(-1, *x.shape[2:])
    c = s[which][ids].long()
    sign = lambda v: 1.0 - 2.0 * (v >> 3).double()
    def magnitude(v):
        e, m = (v >> 1) & 3, (v & 1).double()
        return torch.where(e == 0, 0.5 * m, torch.ldexp(1.0 + 0.5 * m, (e - 1).double()))
    x = torch.empty(*c.shape[:-1], GROUP, dtype=torch.float64, device=c.device)
    for half, v in ((0, c % 16), (1, c // 16)):
        x[..., half::2] = sign(v) * magnitude(v)
    x = x * torch.pow(2.0, s[which + "_scales"][ids].double() - 127)[..., None]
    n, h, g, p, e = x.shape
    return x.permute(0, 3, 1, 2, 4).reshape(n * p, h, g * e)


def _exact_attention(s):
    """The definition per sequence, with the weights from log-sum-exp, the keys a position at a time in blocks."""
    case = s["case"]
    nq, hq, hkv, page = case["queries"], case["hq"], case["hkv"], case["page"]
    q = s["q"].double()
    out = torch.zeros_like(q)
    for b, n in enumerate(s["host_lens"]):
        if not n:
            continue
        pos = torch.arange(n, device="cuda")
        allowed = []
        for i in range(nq):
            p = n - nq + i
            ok = pos <= p
            if case["window"]:
                ok &= (p - pos < case["window"]) | (pos < case["sinks"])
            allowed.append(ok)
        allowed = torch.stack(allowed)
        keep = allowed.any(0)
        pos = pos[keep]
        allowed = allowed[:, keep]
        first = torch.unique(pos // page)
        where = torch.zeros(s["table"].shape[1], dtype=torch.long, device="cuda")
        where[first] = torch.arange(first.numel(), device="cuda")
        rows = where[pos // page] * page + pos % page
        ids = s["table"][b].long()[first]
        k = _exact_token_values(s, "k", ids)[rows].transpose(0, 1).contiguous()
        v = _exact_token_values(s, "v", ids)[rows].transpose(0, 1).contiguous()
        for i in range(nq):
            qi = q[b, i].view(hkv, hq // hkv, -1)
            logit = torch.bmm(qi, k.transpose(1, 2).contiguous()) * float(np.float32(case["d"] ** -0.5))
            logit = logit.masked_fill(~allowed[i], -math.inf)
            weight = torch.exp(logit - torch.logsumexp(logit, -1, keepdim=True))
            out[b, i] = torch.bmm(weight, v).view(hq, -1)
    return out


def _exact_fork(s):
    """Row by row on the host, from the definition."""
    case = s["case"]
    page = case["page"]
    table, lens = s["table"].cpu().numpy().astype(np.int64), s["host_lens"]
    parents, new = s["parents"].tolist(), s["new_lens"].tolist()
    count = s["refcount"].cpu().numpy().astype(np.int64)
    for b, n in enumerate(lens):
        for j in range(-(-n // page)):
            count[table[b, j]] -= 1
    out = np.full((len(parents), table.shape[1]), -1, dtype=np.int64)
    writers = []
    for r, (b, n) in enumerate(zip(parents, new)):
        kept = min(lens[b], n)
        for j in range(-(-kept // page)):
            if j == kept // page and n > kept:
                writers.append((r, j, table[b, j]))
            else:
                out[r, j] = table[b, j]
                count[table[b, j]] += 1
    src, dst = [-1] * len(parents), [-1] * len(parents)
    copied = {}
    for r, j, p in writers:
        if count[p] == 0:
            out[r, j] = p
            count[p] = 1
        else:
            copied[r] = (j, p)
    free = iter(np.flatnonzero(count == 0).tolist())
    taken = 0
    for r, (b, n) in enumerate(zip(parents, new)):
        if r in copied:
            j, src[r] = copied[r]
            out[r, j] = dst[r] = next(free)
            count[dst[r]] = 1
            taken += 1
        for j in range(-(-min(lens[b], n) // page), -(-n // page)):
            out[r, j] = next(free)
            count[out[r, j]] = 1
            taken += 1
    return out, count, src, dst, [taken, 0]


def _exact_compact(s):
    page = s["case"]["page"]
    refcount = s["refcount"].tolist()
    total = sum(c > 0 for c in refcount)
    holes = [p for p in range(total) if refcount[p] == 0]
    page_map = [p if c > 0 else -1 for p, c in enumerate(refcount)]
    src, dst = [-1] * len(refcount), [-1] * len(refcount)
    at = 0
    for p in range(total, len(refcount)):
        if refcount[p] > 0:
            page_map[p] = holes[at]
            src[at], dst[at] = p, holes[at]
            at += 1
    counts = [0] * len(refcount)
    for p, c in enumerate(refcount):
        if c > 0:
            counts[page_map[p]] = c
    out = np.full(tuple(s["table"].shape), -1, dtype=np.int64)
    table = s["table"].tolist()
    for b, n in enumerate(s["host_lens"]):
        for j in range(-(-n // page)):
            out[b, j] = page_map[table[b][j]]
    return out, counts, page_map, src, dst, [total, at]


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "append4":
        return _exact_append4(s)
    if kind in ("attn4", "sink"):
        return _exact_attention(s)
    got = _exact_fork(s) if kind == "fork" else _exact_compact(s)
    src, dst = got[-3], got[-2]
    pools = []
    for pool in s["pools"]:
        moved = pool.clone()
        pairs = [(a, b) for a, b in zip(src, dst) if b >= 0]
        for i in range(0, len(pairs), 64):
            a, b = zip(*pairs[i:i + 64])
            moved.index_copy_(0, torch.tensor(b, device="cuda"), pool.index_select(0, torch.tensor(a, device="cuda")))
        pools.append(moved)
    return tuple(torch.as_tensor(np.asarray(x, dtype=np.int64)).to(torch.int32).cuda() for x in got) + (pools,)
