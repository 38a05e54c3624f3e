"""The end of a generation step over a bounded cache, measured against elementary torch operations.

Three operators, each in the library's form (`own`) and in plain form:
  weigh   what attention each cached token has received: the softmax weights of new rows (one per sequence in a decode
          step, many in a chunk) over the 8-bit paged cache, added up per token and kv head
  evict   a sequence's cache cut down to a number of tokens: the first, the last, and those of the largest weight, moved into
          other blocks and encoded anew where a block's scale changes
  sample  the next token: temperature, top-k, top-p, min-p, and a given random number

A case is a dict of plain values.  Lengths and per-row settings follow from the case alone (`layout`), so that `work` knows
them; tensor contents follow from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E4M3 = torch.float8_e4m3fn


# ------------------------------------------------------------------ cases
def _weigh(dtype, heads, kv_heads, dim, seqs, tokens, block, rows=1, window=0, softcap=0.0, slopes=False, layout=0):
    return dict(op="weigh", dtype=dtype, heads=heads, kv_heads=kv_heads, dim=dim, seqs=seqs, tokens=tokens, block=block,
                rows=rows, window=window, softcap=softcap, slopes=slopes, layout=layout)


def _evict(kv_heads, dim, seqs, tokens, block, keep, first, recent, layout=0):
    return dict(op="evict", kv_heads=kv_heads, dim=dim, seqs=seqs, tokens=tokens, block=block, keep=keep, first=first,
                recent=recent, layout=layout)


def _sample(dtype, rows, vocab, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False, banned=0.0, layout=0):
    return dict(op="sample", dtype=dtype, rows=rows, vocab=vocab, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p,
                mixed=mixed, banned=banned, layout=layout)


def listed():
    return [
        # a single short sequence in the fp32 path: the call's latency
        dict(_weigh("f32", 4, 2, 64, 1, 37, 16), name="weigh_short"),
        # a decode step of 16 sequences of uneven lengths, the 70B block's grouped heads, capped scores
        dict(_weigh("bf16", 64, 8, 128, 16, 4096, 64, softcap=50.0), name="weigh_batch"),
        # a decode step of one long text: a hundred thousand tokens behind the 7B block's 32 heads
        dict(_weigh("bf16", 32, 32, 128, 1, 100003, 64), name="weigh_long"),
        # a chunk of the 7B block behind its context: what the prompt's tokens receive
        dict(_weigh("bf16", 32, 32, 128, 1, 4096, 64, rows=1024), name="weigh_chunk"),
        # ragged rows of three sequences in fp32, odd head size, distance slopes under a window
        dict(_weigh("f32", 16, 4, 80, 3, 1501, 32, rows=61, window=700, slopes=True), name="weigh_rows_f32"),
        # a short cache cut down: the call's latency
        dict(_evict(2, 64, 1, 90, 16, 48, 4, 16), name="evict_small"),
        # 16 sequences of the 70B block brought back to 2048 tokens, a block over
        dict(_evict(8, 128, 16, 2112, 64, 2048, 4, 512), name="evict_step"),
        # the context of a long text cut down to 4096 tokens before generation, the 7B block's 32 heads
        dict(_evict(32, 128, 1, 50011, 64, 4096, 16, 1024), name="evict_context"),
        # one row of a 32000-token vocabulary, top-k and top-p: a single text's step
        dict(_sample("bf16", 1, 32000, 0.7, 50, 0.9), name="sample_one"),
        # a batch with its own settings in every row, padded vocabulary entries banned
        dict(_sample("f32", 64, 32000, 0.8, 40, 0.95, 0.05, mixed=True, banned=0.02), name="sample_mixed"),
        # a wide vocabulary of odd size under top-p alone: rows off the vectors' alignment
        dict(_sample("f32", 24, 128251, 1.0, 0, 0.9), name="sample_wide_top_p"),
        # many rows in bf16 (ties), min-p alone
        dict(_sample("bf16", 192, 64000, 1.2, 0, 1.0, 0.02), name="sample_rows_min_p"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["weigh", "weigh", "evict", "sample", "sample"])
    seed = rng.randrange(1 << 20)
    if op == "sample":
        rows, vocab = _log_int(rng, 1, 256), _log_int(rng, 500, 200000)
        while rows * vocab > 192 * 64000:
            rows = (rows + 1) // 2
        return _sample(rng.choice(["bf16", "f32"]), rows, vocab, rng.choice([0.0, 1.0, 1.0, round(rng.uniform(0.3, 1.7), 3), round(rng.uniform(0.3, 1.7), 3)]),
                       rng.choice([0, 0, 1, _log_int(rng, 2, 2000), _log_int(rng, 2, 2000)]), rng.choice([1.0, round(rng.uniform(0.05, 0.999), 4)]),
                       rng.choice([0.0, 0.0, round(rng.uniform(0.001, 0.3), 4)]), rng.random() < 0.5, rng.choice([0.0, 0.0, 0.1]), seed)
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32])
    dim = rng.choice([64, 80, 96, 128, 128, 128])
    block = rng.choice([16, 32, 64, 128])
    seqs, tokens = _log_int(rng, 1, 48), _log_int(rng, 8, 100000)
    if op == "evict":
        while seqs * tokens * kv_heads > 32 * 50000:
            seqs, tokens = (seqs + 1) // 2, max(1, tokens * 2 // 3)
        keep = max(1, min(6000, int(tokens * rng.uniform(0.05, 1.05))))
        while seqs * keep * kv_heads > 16 * 2048 * 8:
            keep = (keep + 1) // 2
        first = rng.choice([0, min(keep, 4), rng.randint(0, keep // 4)])
        return _evict(kv_heads, dim, seqs, tokens, block, keep, first, rng.randint(0, keep - first), seed)
    group = rng.choice([g for g in (1, 2, 4, 8, 16) if g * kv_heads <= 64])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    rows = rng.choice([1, 1, _log_int(rng, 2, 1500)])
    while seqs * tokens * kv_heads > 32 * 100000 or seqs * tokens * kv_heads * group * rows > 32 << 20:
        seqs, tokens, rows = (seqs + 1) // 2, max(1, tokens * 2 // 3), (rows + 1) // 2
    return _weigh(dtype, kv_heads * group, kv_heads, dim, seqs, tokens, block, min(rows, tokens), rng.choice([0, 0, rng.randint(1, 2000)]),
                  rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.3, seed)


def layout(case):
    """What follows from the case alone: tokens and new rows per sequence, or the settings of every row."""
    rng = random.Random(case["layout"] * 7919 + 29)
    if case["op"] == "sample":
        keys = ("temperature", "top_k", "top_p", "min_p")
        off = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
        rows = []
        for _ in range(case["rows"]):
            row = {k: case[k] for k in keys}
            if case["mixed"]:
                row.update({k: off[k] for k in keys if rng.random() < 0.3})
                row["temperature"] = rng.choice([row["temperature"], 0.0, round(rng.uniform(0.3, 1.5), 2)])
            rows.append(row)
        return {k: [row[k] for row in rows] for k in keys}
    many = case["seqs"] > 1
    lens = [max(1, int(case["tokens"] * rng.uniform(0.25, 1.0))) if many else case["tokens"] for _ in range(case["seqs"])]
    if case["op"] == "evict":
        # most sequences are over the budget when a program evicts; one in five is still below
        lens = [case["tokens"] if rng.random() < 0.8 else n for n in lens]
        return dict(lens=lens, kept=[min(n, case["keep"]) for n in lens])
    if case["rows"] == 1:
        return dict(lens=lens, rows=[1] * case["seqs"])
    return dict(lens=lens, rows=[min(n, rng.randint(0 if i else 1, case["rows"]) if many else case["rows"]) for i, n in enumerate(lens)])


def work(case):
    lay = layout(case)
    if case["op"] == "sample":
        size = 2 if case["dtype"] == "bf16" else 4
        n = case["rows"] * case["vocab"]
        return dict(bytes=n * size + 28 * case["rows"], flops=4 * n)
    g, d = case["kv_heads"], case["dim"]
    if case["op"] == "evict":
        # weights of all places, then codes, weights and scales of the kept ones from one place to another
        return dict(bytes=g * (4 * sum(lay["lens"]) + (4 * d + 12) * sum(lay["kept"])), flops=0)
    size, h = 2 if case["dtype"] == "bf16" else 4, case["heads"]
    reach = lambda p: min(p + 1, case["window"] or p + 1)  # noqa: E731
    pairs = sum(reach(n - r + i) for n, r in zip(lay["lens"], lay["rows"]) for i in range(r)) * h
    seen = sum(min(n, (case["window"] or n) + r - 1) for n, r in zip(lay["lens"], lay["rows"]) if r)
    return dict(bytes=seen * g * (d + 8) + sum(lay["rows"]) * h * (d * size + 4), flops=(2 * d + 4) * pairs)


# ------------------------------------------------------------------ inputs
def _power(e):
    """2^e in 64 bits, from the bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed * 1000003 + case["layout"])
    normal = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    uniform = lambda *shape: torch.rand(shape, generator=gen, device=dev)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    floats = lambda v: torch.tensor(v, dtype=torch.float32, device=dev)  # noqa: E731
    lay, st = layout(case), dict(case=case, plan=None)
    if case["op"] == "sample":
        n, v = case["rows"], case["vocab"]
        # a bulk of unlikely tokens and a few likely ones, the more peaked the surer the model is of its next token
        x = 2.0 * normal(n, v) + 12.0 * uniform(n, v) ** 40 * uniform(n, 1)
        if case["banned"]:
            x[uniform(n, v) < case["banned"]] = -math.inf
        st.update(logits=x.to(DTYPES[case["dtype"]]), u=uniform(n), temperature=floats(lay["temperature"]), top_k=ints(lay["top_k"]),
                  top_p=floats(lay["top_p"]), min_p=floats(lay["min_p"]), tokens=torch.empty((n,), dtype=torch.int32, device=dev),
                  logprobs=torch.empty((n,), dtype=torch.float32, device=dev))
        if own:
            st["plan"] = _plan(st)
        return st
    g, d, bt, lens = case["kv_heads"], case["dim"], case["block"], lay["lens"]
    need = [-(-n // bt) for n in lens]
    more = [-(-n // bt) for n in lay["kept"]] if case["op"] == "evict" else [0] * len(lens)
    blocks = sum(need) + sum(more) + 3
    order = torch.randperm(blocks, generator=gen, device=dev).cpu().tolist()

    def table(counts):
        t = np.full((len(counts), max(counts) + 1), -1, dtype=np.int32)
        for i, n in enumerate(counts):
            t[i, :n] = [order.pop() for _ in range(n)]
        return torch.from_numpy(t).to(dev)

    # a few channels of the keys are several times larger than the rest, as in trained models
    channel = torch.exp(0.5 * normal(g, d))
    channel /= channel.amax()
    pool = lambda spread: (normal(blocks, g, bt, d) * spread).clamp_(-448.0, 448.0).to(E4M3)  # noqa: E731
    exps = lambda: _power(torch.randint(-8, -5, (blocks, g), generator=gen, device=dev)).float()  # noqa: E731
    st.update(k_cache=pool(100.0 * channel[None, :, None, :]), k_scale=exps(), table=table(need), lens=ints(lens),
              weights=torch.exp(2.0 * normal(blocks, g, bt) - 2.0))
    if case["op"] == "evict":
        st.update(v_cache=pool(80.0), v_scale=exps(), to_table=table(more), longest=max(lens),
                  new_lens=torch.empty((len(lens),), dtype=torch.int32, device=dev),
                  kept=torch.full((len(lens), g, case["keep"]), -1, dtype=torch.int32, device=dev))
    else:
        h, total = case["heads"], sum(lay["rows"])
        slopes = floats([2.0 ** (-8.0 * (i + 1) / h) for i in range(h)]) if case["slopes"] else None
        offsets = np.concatenate([[0], np.cumsum(lay["rows"])]).tolist()
        st.update(v_cache=torch.zeros((blocks, g, bt, d), dtype=torch.uint8, device=dev), v_scale=torch.zeros((blocks, g), device=dev),
                  q=normal(total, h, d).to(DTYPES[case["dtype"]]), scale=d ** -0.5, slopes=slopes, offsets=ints(offsets), plain_rows=lay["rows"],
                  plain_lens=lens)
        # what the step's attention has left behind: one row after another, or, of a chunk, one head after another
        lse = torch.empty((total, h), dtype=torch.float32, device=dev)
        st["lse"] = lse if case["rows"] == 1 else torch.empty((h, total), dtype=torch.float32, device=dev).T
        for seqs in _together(st):
            _lse_of(st, seqs).permute(0, 2, 3, 1, 4).copy_(torch.logsumexp(_scores(st, seqs), -1, keepdim=True))
    if own:
        st["plan"] = _plan(st)
    return st


# ------------------------------------------------------------------ plain forms
def _scores(st, seqs):
    """Scores [sequences, kv heads, heads, rows, tokens] in fp32, masked ones -inf, of sequences that have equally many new rows."""
    case, bt, dev = st["case"], st["case"]["block"], st["q"].device
    g, r = case["kv_heads"], st["plain_rows"][seqs[0]]
    width = max(-(-st["plain_lens"][s] // bt) for s in seqs)
    at = sum(st["plain_rows"][:seqs[0]])
    ids = st["table"][seqs[0]:seqs[-1] + 1, :width].long().clamp(min=0)
    k = st["k_cache"].view(torch.uint8)[ids].view(E4M3).float() * st["k_scale"][ids][..., None, None]
    k = k.transpose(1, 2).flatten(2, 3)
    q = st["q"][at:at + r * len(seqs)].float().view(len(seqs), r, g, -1, case["dim"]).permute(0, 2, 3, 1, 4)
    z = torch.matmul(q.flatten(2, 3), k.transpose(2, 3)).view(*q.shape[:4], -1) * st["scale"]
    if case["softcap"]:
        z = torch.tanh(z / case["softcap"]) * case["softcap"]
    row = st["lens"][seqs[0]:seqs[-1] + 1].long()[:, None] - r + torch.arange(r, device=dev)
    back = row[:, :, None] - torch.arange(width * bt, device=dev)
    if st["slopes"] is not None:
        z = z - st["slopes"].view(1, g, -1, 1, 1) * back[:, None, None].abs().float()
    ok = back >= 0
    if case["window"]:
        ok &= back < case["window"]
    return z.masked_fill(~ok[:, None, None], -math.inf)


def _together(st):
    """Runs of sequences whose scores are formed at once: all of them in a decode step, one by one in a chunk."""
    n = len(st["plain_rows"])
    return [list(range(n))] if st["case"]["rows"] == 1 else [[s] for s in range(n) if st["plain_rows"][s]]


def _lse_of(st, seqs):
    """View [sequences, kv heads, heads, rows, 1] of the rows' log-sums."""
    r, at = st["plain_rows"][seqs[0]], sum(st["plain_rows"][:seqs[0]])
    rows = st["lse"][at:at + r * len(seqs)]
    return rows.view(len(seqs), r, st["case"]["kv_heads"], -1, 1) if rows.is_contiguous() else rows.unflatten(1, (st["case"]["kv_heads"], -1))[None, ..., None]


def _plain_weigh(st):
    bt, dev = st["case"]["block"], st["q"].device
    for seqs in _together(st):
        z = _scores(st, seqs)
        w = torch.exp(z - _lse_of(st, seqs).permute(0, 2, 3, 1, 4)).sum((2, 3))
        w = w.unflatten(2, (-1, bt)).transpose(1, 2)
        lens = st["lens"][seqs[0]:seqs[-1] + 1].long()[:, None, None]
        j = torch.arange(w.shape[1] * bt, device=dev).view(1, -1, bt)
        there, blocks = j[..., 0] < lens[:, 0], st["table"][seqs[0]:seqs[-1] + 1, :w.shape[1]].long()
        held = st["weights"][blocks[there]]
        fresh = ((j >= lens - z.shape[3]) & (j < lens))[there][:, None]
        held = torch.where(fresh, 0.0, held) + torch.where((j < lens)[there][:, None], w[there], 0.0)
        st["weights"][blocks[there]] = held
    return st["weights"]


def _plain_evict(st):
    case = st["case"]
    g, d, bt, keep = case["kv_heads"], case["dim"], case["block"], case["keep"]
    n, lens = st["lens"].numel(), st["lens"].long()
    width = -(-st["longest"] // bt)
    table = st["table"][:, :width].long().clamp(min=0)
    lines = lambda x: x[table].transpose(1, 2).reshape(n, g, width * bt, *x.shape[3:])  # noqa: E731
    j = torch.arange(width * bt, device=lens.device)
    w = lines(st["weights"])
    new = lens.clamp(max=keep)
    # the order in which tokens are kept: first and last ones, then by weight, what is behind the end last of all
    rank = torch.where(torch.isnan(w), -math.inf, w)
    sure = (j < case["first"]) | (j >= lens[:, None] - case["recent"])
    rank = torch.where((sure & (j < lens[:, None]))[:, None], math.inf, rank)
    rank = torch.where((j < lens[:, None])[:, None], rank, -math.inf)
    behind = (j >= lens[:, None]).long()[:, None].expand(n, g, -1)
    order = torch.argsort(rank, dim=-1, descending=True, stable=True)
    order = order.gather(-1, torch.argsort(behind.gather(-1, order), dim=-1, stable=True))[..., :keep]
    order = torch.where(torch.arange(order.shape[-1], device=lens.device) < new[:, None, None], order, width * bt)
    order = order.sort(-1).values
    there = order < width * bt
    cells = -(-order.shape[-1] // bt) * bt
    src = torch.nn.functional.pad(order, (0, cells - order.shape[-1]), value=width * bt).clamp(max=width * bt - 1)
    full = torch.nn.functional.pad(there, (0, cells - order.shape[-1]))
    to = st["to_table"][:, :cells // bt].long()
    seqs, blks = torch.nonzero(full[:, 0].view(n, -1, bt)[..., 0], as_tuple=True)
    ids = to[seqs, blks]
    live = full.view(n, g, -1, bt)[seqs, :, blks]
    pick = lambda x: x.view(n, g, -1, bt, *x.shape[3:])[seqs, :, blks]  # noqa: E731
    for pool, scale in ((st["k_cache"], st["k_scale"]), (st["v_cache"], st["v_scale"])):
        code = lines(pool.view(torch.uint8)).gather(2, src[..., None].expand(-1, -1, -1, d)).view(E4M3).float()
        unit = scale[table].transpose(1, 2).gather(2, src // bt)
        code, unit = pick(code), pick(unit)
        size = torch.where(torch.isfinite(code), code.abs(), 0.0) * unit[..., None]
        top = _scale_for(torch.where(live, size.amax(-1), 0.0).amax(-1))
        got = (code * (unit / top[..., None])[..., None]).to(E4M3).view(torch.uint8)
        codes = pool.view(torch.uint8)
        codes[ids] = torch.where(live[..., None], got, codes[ids])
        scale[ids] = top
    st["weights"][ids] = torch.where(live, pick(w.gather(2, src)), st["weights"][ids])
    st["new_lens"].copy_(new)
    at = st["kept"][..., :order.shape[-1]]
    at.copy_(torch.where(there, order, at.long()))


def _scale_for(amax):
    """Smallest power of two 2^e, e >= -126, with amax <= 448 2^e."""
    m, e = torch.frexp(amax)                     # amax = m 2^e, m in [0.5, 1)
    e = torch.where(m > 0.875, e - 8, e - 9)     # 448 = 0.875 2^9
    e = torch.where(amax > 0, e, -126).clamp(min=-126)
    return ((e + 127) << 23).int().view(torch.float32)


def _plain_sample(st):
    x, n = st["logits"].double(), st["logits"].shape[0]
    x = torch.where(torch.isnan(x), -math.inf, x)
    top = x.amax(-1, keepdim=True)
    greedy = st["temperature"] <= 0
    t = torch.where(greedy, 1.0, st["temperature"]).double()[:, None]
    # in 64 bits: the borders of top-p and of the random number fall between sums of many weights
    w = torch.where(x == -math.inf, 0.0, torch.exp((x - top) / t))
    by_size = torch.argsort(x, dim=-1, descending=True, stable=True)
    place = torch.arange(x.shape[1], device=x.device)
    k = torch.where(greedy, 1, torch.where(st["top_k"] > 0, st["top_k"], x.shape[1])).long()[:, None]
    sorted_w = torch.where(place < k, w.gather(-1, by_size), 0.0)
    sums = torch.cumsum(sorted_w, -1)
    p = torch.where(st["top_p"] < 1, st["top_p"].double(), 2.0)[:, None]
    stay = (place < k) & ((sums - sorted_w < p * sums[:, -1:]) | (place == 0)) & (sorted_w >= st["min_p"].double()[:, None])
    mine = torch.where(torch.zeros_like(stay).scatter(-1, by_size, stay), w, 0.0)
    sums = torch.cumsum(mine, -1)
    total = sums[:, -1:]
    token = (sums <= st["u"].double()[:, None] * total).sum(-1)
    last = x.shape[1] - 1 - (mine.flip(-1) > 0).long().argmax(-1)
    token = torch.minimum(token, last)
    st["tokens"].copy_(token)
    st["logprobs"].copy_(torch.log(mine.gather(-1, token[:, None]) / total).view(n))


# ------------------------------------------------------------------ the library's calls
def _plan(st):
    from paper_2401_11504_b200 import binding as b
    case = st["case"]
    if case["op"] == "sample":
        args = b.SampleArgs(st["logits"], st["u"], st["tokens"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
                            min_p=st["min_p"], logprobs=st["logprobs"])
        return (b, args, None)
    cache = b.kv_cache_desc(st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"], st["table"])
    if case["op"] == "evict":
        to = b.kv_cache_desc(st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"], st["to_table"])
        args = b.KvCacheEvictArgs(cache, st["weights"], st["lens"], to, st["weights"], st["new_lens"], case["keep"], n_first=case["first"],
                                  n_recent=case["recent"], kept=st["kept"])
        return (b, args, b.alloc_workspace(b.templora_kv_cache_evict_workspace_bytes(cache, case["keep"])))
    code = {"bf16": b.BF16, "f32": b.F32}[case["dtype"]]
    attn = b.attention_desc(case["heads"], case["kv_heads"], case["dim"], code, scale=st["scale"], softcap=case["softcap"],
                            window=case["window"], slopes=st["slopes"])
    args = b.KvCacheWeighArgs(attn, cache, st["lens"], st["q"], st["lse"], st["weights"],
                              row_offsets=None if case["rows"] == 1 else st["offsets"])
    return (b, args, b.alloc_workspace(b.templora_kv_cache_weigh_workspace_bytes(attn, cache, st["q"].shape[0])))


def run(st):
    op = st["case"]["op"]
    if own:
        if st["plan"] is None:
            st["plan"] = _plan(st)
        b, args, ws = st["plan"]
        if op == "sample":
            b.templora_sample(args)
        elif op == "evict":
            b.templora_kv_cache_evict(args, ws)
        else:
            b.templora_kv_cache_weigh(args, ws)
    else:
        {"sample": _plain_sample, "evict": _plain_evict, "weigh": _plain_weigh}[op](st)
    if op == "sample":
        return st["tokens"], st["logprobs"]
    if op == "evict":
        return st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"], st["weights"], st["new_lens"], st["kept"]
    return st["weights"]


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"sample": _exact_sample, "evict": _exact_evict, "weigh": _exact_weigh}[case["op"]](case, st)


def _exact_weigh(case, st):
    lay, bt, out, at = layout(case), case["block"], st["weights"].double(), 0
    group, table = case["heads"] // case["kv_heads"], st["table"].cpu().numpy()
    for s, (n, r) in enumerate(zip(lay["lens"], lay["rows"])):
        if r == 0:
            continue
        ids = torch.from_numpy(table[s, :(n + bt - 1) // bt].astype(np.int64)).to(out.device)
        key = torch.arange(n, device=out.device)
        row = torch.arange(n - r, n, device=out.device)
        far = (row.unsqueeze(1) - key.unsqueeze(0)).double()
        hidden = (far < 0) | (far >= (case["window"] if case["window"] else math.inf))
        for h in range(case["heads"]):
            hk = h // group
            k = st["k_cache"].view(torch.uint8)[ids, hk].view(E4M3).double() * st["k_scale"][ids, hk].double().view(-1, 1, 1)
            z = st["q"][at:at + r, h].double() @ k.reshape(-1, case["dim"])[:n].t() * st["scale"]
            if case["softcap"]:
                z = case["softcap"] * torch.tanh(z / case["softcap"])
            if st["slopes"] is not None:
                z = z - float(st["slopes"][h]) * far
            got = torch.exp(z - st["lse"][at:at + r, h].double().unsqueeze(1)).masked_fill(hidden, 0.0).sum(0)
            block, place = ids[key // bt], key % bt
            if h % group == 0:      # places that this call's rows have brought hold nothing yet
                out[block[n - r:], hk, place[n - r:]] = 0.0
            out[block, hk, place] += got
        at += r
    return out


def _exact_evict(case, st):
    lay, bt, g = layout(case), case["block"], case["kv_heads"]
    dev = st["weights"].device
    out = {n: st[n].double() for n in ("k_cache", "v_cache", "k_scale", "v_scale", "weights")}
    before = {n: t.clone() for n, t in out.items()}
    kept = st["kept"].cpu().numpy().copy()
    w, src, dst = st["weights"].cpu().numpy(), st["table"].cpu().numpy(), st["to_table"].cpu().numpy()
    for s, (n, m) in enumerate(zip(lay["lens"], lay["kept"])):
        ids = src[s, :(n + bt - 1) // bt]
        for hk in range(g):
            line = w[ids, hk].reshape(-1)[:n]
            a, z = (case["first"], n - case["recent"]) if n > m else (n, n)
            best = a + np.lexsort((np.arange(a, z), -line[a:z].astype(np.float64)))[:m - a - (n - z)]
            places = np.concatenate([np.arange(a), np.sort(best), np.arange(z, n)]).astype(np.int64)
            assert len(places) == m
            kept[s, hk, :m] = places
            for b0 in range(0, m, bt):
                one = places[b0:b0 + bt]
                frm = torch.from_numpy(ids[one // bt].astype(np.int64)).to(dev)
                at = torch.from_numpy(one % bt).to(dev)
                blk = int(dst[s, b0 // bt])
                out["weights"][blk, hk, :len(one)] = before["weights"][frm, hk, at]
                for pool in "kv":
                    x = before[pool + "_cache"][frm, hk, at] * before[pool + "_scale"][frm, hk].unsqueeze(1)
                    m2, e2 = torch.frexp(x.abs().amax().clamp(min=2.0 ** -140) / 448.0)
                    unit = _power(torch.where(m2 > 0.5, e2, e2 - 1)).clamp(min=2.0 ** -126)
                    out[pool + "_scale"][blk, hk] = unit
                    out[pool + "_cache"][blk, hk, :len(one)] = _nearest_e4m3(x / unit)
    new = torch.tensor(lay["kept"], dtype=torch.int32, device=dev)
    return out["k_cache"], out["v_cache"], out["k_scale"], out["v_scale"], out["weights"], new, torch.from_numpy(kept).to(dev)


def _nearest_e4m3(x):
    """Nearest value with 4 significant bits and exponents from -6 on (below: multiples of 2^-9), ties to even."""
    step = _power(torch.frexp(x.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(x / step) * step


def _exact_sample(case, st):
    lay = layout(case)
    logits, u = st["logits"].double().cpu().numpy(), st["u"].double().cpu().numpy()
    f32 = lambda v: float(np.float32(v))  # noqa: E731
    tokens, logprobs = np.zeros(case["rows"], dtype=np.int32), np.zeros(case["rows"])
    for i, x in enumerate(logits):
        temperature, k = f32(lay["temperature"][i]), lay["top_k"][i]
        if temperature <= 0:
            tokens[i] = int(np.argmax(x))
            continue
        order = np.argsort(-x, kind="stable")
        order = order[:k] if k > 0 else order
        w = np.exp((x[order] - x.max()) / temperature)
        if lay["top_p"][i] < 1:
            reach = np.cumsum(w)
            count = 1 + int(np.searchsorted(reach, f32(lay["top_p"][i]) * reach[-1]))
            order, w = order[:count], w[:count]
        stay = w >= f32(lay["min_p"][i])
        order, w = order[stay], w[stay]
        by_token = np.argsort(order)
        order, w = order[by_token], w[by_token]
        reach = np.cumsum(w)
        at = min(int(np.searchsorted(reach, u[i] * reach[-1], side="right")), len(w) - 1)
        tokens[i], logprobs[i] = order[at], np.log(w[at] / reach[-1])
    return torch.from_numpy(tokens), torch.from_numpy(logprobs)
