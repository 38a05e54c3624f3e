"""Attention between a decoder block's projections, measured against elementary torch operations.

Three operators, each in the library's form (`own`) and in plain form:
  attn_fwd, attn_bwd  attention of a chunk and its gradients: grouped heads, tanh-capped scores, a bias that grows
                      with the distance, causal / prefix / document / window masks
  append              new keys and values encoded into a paged 8-bit cache, one scale per block of tokens and head
  decode              attention of one new token per sequence over that cache

A case is a dict of plain values.  Documents and sequence lengths follow from the case alone (`layout`), so
that `work` knows them; tensor contents follow from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E4M3_MAX = 448.0


# ------------------------------------------------------------------ cases
def _attn(op, dtype, heads, kv_heads, dim, tq, context=0, causal=True, window=0, softcap=0.0, slopes=False, docs=0,
          prefix=False, fused=False, layout=0):
    return dict(op=op, dtype=dtype, heads=heads, kv_heads=kv_heads, dim=dim, tq=tq, context=context, causal=causal,
                window=window, softcap=softcap, slopes=slopes, docs=docs, prefix=prefix, fused=fused, layout=layout)


def _cache(op, dtype, heads, kv_heads, dim, seqs, tokens, block, new=1, window=0, softcap=0.0, slopes=False, layout=0):
    return dict(op=op, dtype=dtype, heads=heads, kv_heads=kv_heads, dim=dim, seqs=seqs, tokens=tokens, block=block,
                new=new, window=window, softcap=softcap, slopes=slopes, layout=layout)


def listed():
    return [
        # a handful of new tokens behind a short context in the fp32 path: the call's latency
        dict(_attn("attn_fwd", "f32", 4, 2, 64, 17, context=79), name="fwd_f32_tail"),
        # one chunk of the Llama-2-7B block, the update's forward
        dict(_attn("attn_fwd", "bf16", 32, 32, 128, 1024), name="fwd_7b_chunk"),
        # one chunk of the Llama-2-70B block with capped scores, the largest chunk
        dict(_attn("attn_fwd", "bf16", 64, 8, 128, 4096, softcap=50.0), name="fwd_70b_capped"),
        # packed documents of uneven lengths, each with a prefix that sees itself whole, and distance slopes;
        # q, k and v are slices of one buffer
        dict(_attn("attn_fwd", "bf16", 32, 8, 128, 4099, slopes=True, docs=7, prefix=True, fused=True), name="fwd_docs_prefix"),
        # the backward of the 7B chunk
        dict(_attn("attn_bwd", "bf16", 32, 32, 128, 1024), name="bwd_7b_chunk"),
        # the backward of packed documents with grouped heads, prefixes and capped scores
        dict(_attn("attn_bwd", "bf16", 32, 8, 128, 4099, softcap=30.0, docs=5, prefix=True), name="bwd_docs_prefix"),
        # a small fp32 backward under a sliding window
        dict(_attn("attn_bwd", "f32", 4, 2, 64, 251, window=64), name="bwd_f32_window"),
        # one new token for each of 16 sequences of the 70B block: a decode step's cache write
        dict(_cache("append", "bf16", 64, 8, 128, 16, 2000, 64), name="append_step"),
        # the context of a 7B block written in one go, behind partly filled blocks
        dict(_cache("append", "bf16", 32, 32, 128, 3, 100, 64, new=1365), name="append_context"),
        # a single short sequence: the decode call's latency
        dict(_cache("decode", "bf16", 32, 32, 128, 1, 37, 16), name="decode_short"),
        # 16 sequences of uneven lengths, the 70B block's grouped heads, capped scores
        dict(_cache("decode", "bf16", 64, 8, 128, 16, 4096, 64, softcap=50.0), name="decode_batch"),
        # one long text: a hundred thousand tokens behind the 7B block's 32 heads
        dict(_cache("decode", "bf16", 32, 32, 128, 1, 100003, 64), name="decode_long"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attn_fwd", "attn_fwd", "attn_bwd", "attn_bwd", "append", "decode", "decode"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32])
    group = rng.choice([g for g in (1, 2, 4, 8) if g * kv_heads <= 64])
    dim = rng.choice([64, 80, 96, 128, 128, 128])
    softcap = rng.choice([0.0, 0.0, 20.0, 50.0])
    slopes = rng.random() < 0.3
    window = rng.choice([0, 0, 0, rng.randint(1, 2000)])
    layout = rng.randrange(1 << 20)
    if op.startswith("attn"):
        causal = rng.random() < 0.8
        # scores in all: a backward has five products to a forward's two, and fp32 runs on the plain pipes
        budget = (64 << 24) >> ((0 if causal else 1) + (2 if op == "attn_bwd" else 0) + (3 if dtype == "f32" else 0))
        tq = _log_int(rng, 1, 4500)
        context = rng.choice([0, 0, _log_int(rng, 1, 4000)])
        while kv_heads * group * tq * (tq + context) > budget:
            tq, context = (tq + 1) // 2, context // 2
        docs = rng.choice([0, 0, 1, rng.randint(2, 12)])
        prefix = causal and not window and rng.random() < 0.4
        return _attn(op, dtype, kv_heads * group, kv_heads, dim, tq, context, causal, window, softcap, slopes, docs,
                     prefix, rng.random() < 0.4, layout)
    block = rng.choice([16, 32, 64, 128])
    seqs = _log_int(rng, 1, 48)
    if op == "append":
        new = rng.choice([1, _log_int(rng, 1, 2000)])
        while seqs * new * kv_heads > 32 * 4096:
            new = (new + 1) // 2
            seqs = (seqs + 1) // 2
        return _cache(op, dtype, kv_heads * group, kv_heads, dim, seqs, _log_int(rng, 1, 3000), block, new, layout=layout)
    tokens = _log_int(rng, 1, 100000)
    while seqs * tokens * kv_heads > 32 * 100000:
        seqs, tokens = (seqs + 1) // 2, max(1, tokens * 2 // 3)
    return _cache(op, dtype, kv_heads * group, kv_heads, dim, seqs, tokens, block, 1, window, softcap, slopes, layout)


def layout(case):
    """What follows from the case alone: document offsets and prefixes, or tokens held and new per sequence."""
    rng = random.Random(case["layout"] * 7919 + 17)
    if case["op"].startswith("attn"):
        tk = case["context"] + case["tq"]
        if not case["docs"]:
            return dict(tk=tk, offsets=None, prefix=[rng.randint(0, tk // 2)] if case["prefix"] else None)
        # a few rows may lie behind the last document: padding, which attends to nothing
        end = tk - rng.choice([0, 0, rng.randint(0, tk // 16)])
        cuts = sorted(rng.randint(0, end) for _ in range(case["docs"] - 1))
        offsets = [0] + cuts + [end]
        lens = [b - a for a, b in zip(offsets, offsets[1:])]
        return dict(tk=tk, offsets=offsets, prefix=[rng.randint(0, n // 2) for n in lens] if case["prefix"] else None)
    uneven = lambda n: max(1, int(n * rng.uniform(0.25, 1.0)))  # noqa: E731
    n, many = case["seqs"], case["seqs"] > 1
    held = [uneven(case["tokens"]) if many else case["tokens"] for _ in range(n)]
    if case["op"] == "decode":
        return dict(held=held, new=[0] * n)
    new = [uneven(case["new"]) if many and case["new"] > 1 else case["new"] for _ in range(n)]
    return dict(held=held, new=new)


def _intervals_np(case, lay):
    """Allowed keys [lo, hi) of every query row."""
    tk, p = lay["tk"], case["context"] + np.arange(case["tq"], dtype=np.int64)
    off = np.array(lay["offsets"] if lay["offsets"] is not None else [0, tk], dtype=np.int64)
    d = np.searchsorted(off, p, side="right") - 1
    inside = (d >= 0) & (d < len(off) - 1)
    d = np.clip(d, 0, len(off) - 2)
    s, e = off[d], off[d + 1]
    lo, hi = s.copy(), e.copy()
    if case["causal"]:
        hi = np.minimum(e, np.maximum(p + 1, s + (np.array(lay["prefix"])[d] if lay["prefix"] is not None else 0)))
    if case["window"]:
        lo = np.maximum(s, p - case["window"] + 1)
        if not case["causal"]:
            hi = np.minimum(e, p + case["window"])
    return np.where(inside, lo, 0), np.where(inside, np.maximum(hi, lo), 0)


def work(case):
    lay, size = layout(case), 2 if case["dtype"] == "bf16" else 4
    h, g, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"].startswith("attn"):
        lo, hi = _intervals_np(case, lay)
        pairs = int((hi - lo).sum()) * h
        rows_q, rows_k = case["tq"] * h * d * size, lay["tk"] * g * d * size
        if case["op"] == "attn_fwd":
            return dict(bytes=2 * rows_q + 2 * rows_k + 4 * case["tq"] * h, flops=4 * d * pairs)
        return dict(bytes=4 * rows_q + 4 * rows_k + 4 * case["tq"] * h, flops=10 * d * pairs)
    if case["op"] == "append":
        rows = sum(lay["new"]) * g * d
        return dict(bytes=2 * rows * (size + 1), flops=4 * rows)
    seen = sum(min(n, case["window"] or n) for n in lay["held"])
    return dict(bytes=2 * seen * g * d + 2 * case["seqs"] * h * d * size, flops=4 * seen * h * d)


# ------------------------------------------------------------------ inputs
def _slopes(case, dev):
    # the geometric series that distance biases use
    h = case["heads"]
    return torch.tensor([2.0 ** (-8.0 * (i + 1) / h) for i in range(h)], dtype=torch.float32, device=dev) if case["slopes"] else None


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed * 1000003 + case["layout"])
    dt, lay = DTYPES[case["dtype"]], layout(case)
    h, g, d = case["heads"], case["kv_heads"], case["dim"]
    normal = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    st = dict(case=case, scale=d ** -0.5, slopes=_slopes(case, dev), plan=None)
    ints = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    # a few channels of the keys are several times larger than the rest, as in trained models
    channel = torch.exp(0.5 * normal(g, d))
    if case["op"].startswith("attn"):
        tq, tk = case["tq"], lay["tk"]
        st.update(offsets=ints(lay["offsets"]), prefix=ints(lay["prefix"]))
        if case["fused"]:
            buf = torch.empty((tk, h + 2 * g, d), dtype=dt, device=dev)
            q, k, v = buf[case["context"]:, :h], buf[:, h:h + g], buf[:, h + g:]
        else:
            q, k, v = (torch.empty((n, m, d), dtype=dt, device=dev) for n, m in ((tq, h), (tk, g), (tk, g)))
        q.copy_(normal(tq, h, d)); k.copy_(normal(tk, g, d) * channel); v.copy_(normal(tk, g, d))
        st.update(q=q, k=k, v=v, o=torch.empty((tq, h, d), dtype=dt, device=dev),
                  lse=torch.empty((h, tq), dtype=torch.float32, device=dev))
        if case["op"] == "attn_bwd":
            o, lse = _plain_fwd(st)
            st["o"].copy_(o); st["lse"].copy_(lse)
            st["do"] = normal(tq, h, d).to(dt)
            st.update(dq=torch.empty((tq, h, d), dtype=dt, device=dev), dk=torch.empty((tk, g, d), dtype=dt, device=dev),
                      dv=torch.empty((tk, g, d), dtype=dt, device=dev))
        return st
    bt, held, new = case["block"], lay["held"], lay["new"]
    need = [-(-(a + b) // bt) for a, b in zip(held, new)]
    blocks = sum(need) + 3
    order = torch.randperm(blocks, generator=gen, device=dev).cpu().tolist()
    width = max(need) + 1
    table, at = np.full((len(held), width), -1, dtype=np.int32), 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    code = lambda x: (x.clamp_(-E4M3_MAX, E4M3_MAX)).to(torch.float8_e4m3fn)  # noqa: E731
    pool = lambda spread: code(torch.randn((blocks, g, bt, d), generator=gen, device=dev) * spread)  # noqa: E731
    exps = lambda: _power(torch.randint(-8, -5, (blocks, g), generator=gen, device=dev)).float()  # noqa: E731
    st.update(k_cache=pool(100.0 * channel[None, :, None, :] / channel.amax()), v_cache=pool(80.0), k_scale=exps(),
              v_scale=exps(), table=torch.from_numpy(table).to(dev), block=bt)
    if case["op"] == "append":
        total = sum(new)
        st.update(held=ints(held), offsets=ints(np.concatenate([[0], np.cumsum(new)]).tolist()),
                  k_new=(normal(total, g, d) * channel).to(dt), v_new=normal(total, g, d).to(dt))
        return st
    st.update(held=ints(held), q=normal(len(held), h, d).to(dt), o=torch.empty((len(held), h, d), dtype=dt, device=dev),
              longest=max(held))
    return st


# ------------------------------------------------------------------ plain forms
def _bounds(st, device):
    case = st["case"]
    p = case["context"] + torch.arange(case["tq"], device=device)
    tk = case["context"] + case["tq"]
    off = st["offsets"].long() if st["offsets"] is not None else torch.tensor([0, tk], device=device)
    d = torch.searchsorted(off, p, right=True) - 1
    inside = d < off.numel() - 1
    d = d.clamp(0, off.numel() - 2)
    lo, hi = off[d], off[d + 1]
    if case["causal"]:
        reach = p + 1
        if st["prefix"] is not None:
            reach = torch.maximum(reach, lo + st["prefix"].long()[d])
        hi = torch.minimum(hi, reach)
    if case["window"]:
        lo = torch.maximum(lo, p - case["window"] + 1)
        if not case["causal"]:
            hi = torch.minimum(hi, p + case["window"])
    return torch.where(inside, lo, 0), torch.where(inside, hi, 0), p


def _plain_scores(st):
    """Scores [kv_heads, group, tq, tk] in fp32, masked ones -inf, and the tanh of the capped ones."""
    case = st["case"]
    q, k = st["q"].float(), st["k"].float()
    tq, tk, g = q.shape[0], k.shape[0], case["kv_heads"]
    rows = q.transpose(0, 1).reshape(g, -1, case["dim"])
    z = torch.matmul(rows, k.permute(1, 2, 0)).view(g, -1, tq, tk) * st["scale"]
    t = None
    if case["softcap"]:
        t = torch.tanh(z / case["softcap"])
        z = t * case["softcap"]
    lo, hi, p = _bounds(st, q.device)
    j = torch.arange(tk, device=q.device)
    if st["slopes"] is not None:
        z = z - st["slopes"].view(g, -1, 1, 1) * (p[:, None] - j[None, :]).abs().float()
    ok = (j[None, :] >= lo[:, None]) & (j[None, :] < hi[:, None])
    return z.masked_fill(~ok, -math.inf), t


def _plain_fwd(st):
    case = st["case"]
    z, _ = _plain_scores(st)
    g, n, tq, tk = z.shape
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(g, n * tq, tk), st["v"].float().transpose(0, 1)).view(g * n, tq, -1)
    o = torch.where(total.view(g * n, tq, 1) > 0, o / total.view(g * n, tq, 1), 0.0)
    return o.transpose(0, 1).to(DTYPES[case["dtype"]]), (top + torch.log(total)).view(g * n, tq)


def _plain_bwd(st):
    case = st["case"]
    z, t = _plain_scores(st)
    g, n, tq, tk = z.shape
    lse = st["lse"].view(g, n, tq, 1)
    p = torch.where(lse == -math.inf, 0.0, torch.exp(z - lse))
    do = st["do"].float().transpose(0, 1).reshape(g, n * tq, -1)
    dp = torch.matmul(do, st["v"].float().permute(1, 2, 0)).view(g, n, tq, tk)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * st["scale"]
    if t is not None:
        ds = ds * (1.0 - t * t)
    ds, p = ds.view(g, n * tq, tk), p.view(g, n * tq, tk)
    rows = st["q"].float().transpose(0, 1).reshape(g, n * tq, -1)
    dq = torch.matmul(ds, st["k"].float().transpose(0, 1)).view(g * n, tq, -1).transpose(0, 1)
    dk = torch.matmul(ds.transpose(1, 2), rows).transpose(0, 1)
    dv = torch.matmul(p.transpose(1, 2), do).transpose(0, 1)
    dt = DTYPES[case["dtype"]]
    return dq.to(dt), dk.to(dt), dv.to(dt)


def _scale_for(amax):
    """Smallest power of two 2^e, e >= -126, with amax <= 448 2^e."""
    m, e = torch.frexp(amax)                     # amax = m 2^e, m in [0.5, 1)
    e = torch.where(m > 0.875, e - 8, e - 9)     # 448 = 0.875 2^9
    e = torch.where(amax > 0, e, -126).clamp(min=-126)
    return ((e + 127) << 23).int().view(torch.float32)


def _plain_encode(pool, scale, rows, slot, at, blocks, held):
    """Rows [n, heads, dim] go to position `at` of the block blocks[slot], which held so many tokens before."""
    x = rows.float()
    codes = pool.view(torch.uint8)
    fine = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    top = torch.zeros((blocks.numel(), x.shape[1]), device=x.device)
    top = top.scatter_reduce(0, slot[:, None].expand_as(fine), fine, "amax")
    before = scale[blocks]
    after = torch.where(held[:, None] > 0, torch.maximum(before, _scale_for(top)), _scale_for(top))
    ratio = torch.where(held[:, None] > 0, before / after, 1.0)
    kept = codes[blocks].view(pool.dtype).float() * ratio[:, :, None, None]
    old = torch.arange(pool.shape[2], device=x.device)[None, :] < held[:, None]
    codes[blocks] = torch.where(old[:, None, :, None], kept.to(pool.dtype).view(torch.uint8), codes[blocks])
    scale[blocks] = after
    codes[blocks[slot], :, at] = (x / after[slot][:, :, None]).to(pool.dtype).view(torch.uint8)


def _plain_append(st):
    bt, held, offsets, table = st["block"], st["held"].long(), st["offsets"].long(), st["table"].long()
    rows = torch.arange(st["k_new"].shape[0], device=table.device)
    seq = torch.searchsorted(offsets, rows, right=True) - 1
    pos = held[seq] + rows - offsets[seq]
    key = seq * table.shape[1] + pos // bt
    keys, slot = torch.unique(key, return_inverse=True)
    blocks = table.reshape(-1)[keys]
    in_block = (held[keys // table.shape[1]] - keys % table.shape[1] * bt).clamp(0, bt)
    for pool, scale, new in ((st["k_cache"], st["k_scale"], st["k_new"]), (st["v_cache"], st["v_scale"], st["v_new"])):
        _plain_encode(pool, scale, new, slot, pos % bt, blocks, in_block)


def _plain_decode(st):
    case = st["case"]
    g, d, bt = case["kv_heads"], case["dim"], st["block"]
    n, width = st["table"].shape[0], -(-st["longest"] // bt)
    table = st["table"][:, :width].long().clamp(min=0)
    values = lambda pool: pool.view(torch.uint8)[table].view(pool.dtype).float()  # noqa: E731
    wide = lambda pool, scale: (values(pool) * scale[table][..., None, None]).transpose(1, 2).reshape(n, g, -1, d)  # noqa: E731
    q = st["q"].float().view(n, g, -1, d)
    z = torch.matmul(q, wide(st["k_cache"], st["k_scale"]).transpose(2, 3)) * st["scale"]
    if case["softcap"]:
        z = torch.tanh(z / case["softcap"]) * case["softcap"]
    j = torch.arange(width * bt, device=q.device)
    back = st["held"].long()[:, None] - 1 - j[None, :]
    if st["slopes"] is not None:
        z = z - st["slopes"].view(1, g, -1, 1) * back[:, None, None, :].abs().float()
    ok = back >= 0
    if case["window"]:
        ok &= back < case["window"]
    z = z.masked_fill(~ok[:, None, None, :], -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True))
    # what lies behind a sequence's last token in its last block is not part of it
    v = torch.where(ok[:, None, :, None], wide(st["v_cache"], st["v_scale"]), 0.0)
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    return o.view(n, g * q.shape[2], d).to(DTYPES[case["dtype"]])


# ------------------------------------------------------------------ the library's calls
def _plan(st):
    from paper_2401_11504_b200 import binding as b
    case = st["case"]
    code = {"bf16": b.BF16, "f32": b.F32}[case["dtype"]]
    desc = lambda **kw: b.attention_desc(case["heads"], case["kv_heads"], case["dim"], code, scale=st["scale"],  # noqa: E731
                                         softcap=case["softcap"], window=case["window"], slopes=st["slopes"], **kw)
    if case["op"].startswith("attn"):
        a = desc(causal=case["causal"], doc_offsets=st["offsets"], prefix_lens=st["prefix"])
        ws = b.alloc_workspace(b.templora_attention_workspace_bytes(a, case["tq"], case["context"] + case["tq"]))
        grads = {n: st[n] for n in ("do", "dq", "dk", "dv") if n in st}
        args = b.AttentionArgs(a, st["q"], st["k"], st["v"], st["o"], st["lse"], q_start=case["context"], **grads)
        return (b, args, ws)
    cache = b.kv_cache_desc(st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"], st["table"])
    if case["op"] == "append":
        ws = b.alloc_workspace(b.templora_kv_cache_append_workspace_bytes(cache))
        return (b, b.KvCacheAppendArgs(cache, st["held"], st["k_new"], st["v_new"], new_offsets=st["offsets"]), ws)
    a = desc()
    ws = b.alloc_workspace(b.templora_attention_decode_workspace_bytes(a, cache))
    return (b, b.AttentionDecodeArgs(a, cache, st["held"], st["q"], st["o"]), ws)


def run(st):
    op = st["case"]["op"]
    if own:
        if st["plan"] is None:
            st["plan"] = _plan(st)
        b, args, ws = st["plan"]
        {"attn_fwd": b.templora_attention_fwd, "attn_bwd": b.templora_attention_bwd, "append": b.templora_kv_cache_append,
         "decode": b.templora_attention_decode_fwd}[op](args, ws)
        if op == "attn_fwd":
            return st["o"], st["lse"]
        if op == "attn_bwd":
            return st["dq"], st["dk"], st["dv"]
        if op == "decode":
            return st["o"]
    elif op == "attn_fwd":
        return _plain_fwd(st)
    elif op == "attn_bwd":
        return _plain_bwd(st)
    elif op == "decode":
        return _plain_decode(st)
    else:
        _plain_append(st)
    return st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"]


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"].startswith("attn"):
        return _exact_attention(case, st)
    if case["op"] == "decode":
        return _exact_decode(case, st)
    return _exact_append(case, st)


def _exact_attention(case, st):
    dev, h = st["q"].device, case["heads"]
    group = h // case["kv_heads"]
    q, k, v = (st[n].double() for n in ("q", "k", "v"))
    lo, hi = (torch.from_numpy(x).to(dev) for x in _intervals_np(case, layout(case)))
    pos = case["context"] + torch.arange(case["tq"], device=dev)
    j = torch.arange(k.shape[0], device=dev)
    ok = (lo[:, None] <= j) & (j < hi[:, None])
    far = (pos[:, None] - j).abs().double()
    empty = ~ok.any(1)
    o, lse = torch.zeros_like(q), torch.empty((h, q.shape[0]), dtype=torch.float64, device=dev)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for i in range(h):
        kk, vv = k[:, i // group], v[:, i // group]
        z = q[:, i] @ kk.T * st["scale"]
        slope = 1.0
        if case["softcap"]:
            c = torch.tanh(z / case["softcap"])
            z, slope = case["softcap"] * c, 1.0 - c * c
        if st["slopes"] is not None:
            z = z - st["slopes"][i].double() * far
        z = torch.where(ok, z, -math.inf)
        lse[i] = torch.logsumexp(z, 1)
        p = torch.where(empty[:, None], 0.0, torch.exp(z - lse[i][:, None]))
        o[:, i] = p @ vv
        if case["op"] == "attn_bwd":
            do = st["do"][:, i].double()
            dp = do @ vv.T
            ds = p * (dp - (do * o[:, i]).sum(1, keepdim=True)) * slope * st["scale"]
            dq[:, i] = ds @ kk
            dk[:, i // group] += ds.T @ q[:, i]
            dv[:, i // group] += p.T @ do
    return (o, lse) if case["op"] == "attn_fwd" else (dq, dk, dv)


def _exact_decode(case, st):
    group, bt = case["heads"] // case["kv_heads"], st["block"]
    o = torch.zeros(st["q"].shape, dtype=torch.float64, device=st["q"].device)
    for b, n in enumerate(st["held"].tolist()):
        ids = st["table"][b, :-(-n // bt)].long()
        k, v = ((c.view(torch.uint8)[ids].view(c.dtype).double() * s[ids].double()[:, :, None, None]).transpose(0, 1).flatten(1, 2)[:, :n]
                for c, s in ((st["k_cache"], st["k_scale"]), (st["v_cache"], st["v_scale"])))
        first = max(0, n - case["window"]) if case["window"] else 0
        k, v = k[:, first:].repeat_interleave(group, 0), v[:, first:].repeat_interleave(group, 0)
        z = torch.einsum("hd,htd->ht", st["q"][b].double(), k) * st["scale"]
        if case["softcap"]:
            z = case["softcap"] * torch.tanh(z / case["softcap"])
        if st["slopes"] is not None:
            back = torch.arange(n - 1 - first, -1, -1, device=z.device).double()
            z = z - st["slopes"].double()[:, None] * back
        o[b] = torch.einsum("ht,htd->hd", torch.softmax(z, 1), v)
    return o


def _exact_append(case, st):
    bt, lay = st["block"], layout(case)
    out, at = [], 0
    pools = [[st[n + "_cache"].double(), st[n + "_scale"].double(), st[n + "_new"].double()] for n in "kv"]
    table = st["table"].tolist()
    for b, (held, new) in enumerate(zip(lay["held"], lay["new"])):
        done = 0
        while done < new:
            pos = held + done
            block, first = table[b][pos // bt], pos % bt
            count = min(bt - first, new - done)
            for pool, scale, rows in pools:
                x = rows[at + done:at + done + count].transpose(0, 1)          # [heads, count, dim]
                top = x.abs().amax((1, 2)).clamp(min=2.0 ** -140)
                m, e = torch.frexp(top / E4M3_MAX)
                need = _power(torch.where(m > 0.5, e, e - 1)).clamp(min=2.0 ** -126)
                if first:
                    need = torch.maximum(need, scale[block])
                    pool[block, :, :first] = _nearest_e4m3(pool[block, :, :first] * (scale[block] / need)[:, None, None])
                scale[block] = need
                pool[block, :, first:first + count] = _nearest_e4m3(x / need[:, None, None])
            done += count
        at += new
    for pool, scale, _ in pools:
        out.append(pool)
    return (*out, pools[0][1], pools[1][1])


def _power(e):
    """2^e in 64 bits, from the bits: exp2 may be off by a unit in the last place, which moves ties."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _nearest_e4m3(x):
    """Nearest value with 4 significant bits and exponents from -6 on (below: multiples of 2^-9), ties to even."""
    step = _power(torch.frexp(x.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(x / step) * step
