"""The 8-bit key/value cache: encoding against the oracle code by code, decode attention against the fp64 oracle, and a
run of update, append and decode as a generation loop makes them.

Bounds of the decode attention: probabilities are held in fp16 (2^-11 of each term) on the bf16 path, the result is
rounded once; scores, sums and everything on the fp32 path are fp32 (SLACK, as for the chunk's attention)."""
import numpy as np
import pytest
import torch

from oracle import templora_oracle as orc
from parity_utils import Guarded

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ROUND = {"bf16": 2.0 ** -8, "f32": 2.0 ** -23}
SLACK = 4e-5


@pytest.fixture(scope="module")
def b():
    from paper_2401_11504_b200 import build
    build.build_library()
    from paper_2401_11504_b200 import binding
    return binding


class Cache:
    """A pool with a random block order, every place a NaN code at first, guarded."""

    def __init__(self, b, heads, dim, bt, lens, seed=0, spare=2, scale=float("nan")):
        g = np.random.default_rng(seed)
        need = [-(-n // bt) for n in lens]
        self.blocks, self.width, self.bt = sum(need) + spare, max(need) + 1, bt
        ids = list(g.permutation(self.blocks))
        self.tables = [[int(ids.pop()) for _ in range(n)] for n in need]
        host = np.full((len(lens), self.width), -7, dtype=np.int32)
        for i, t in enumerate(self.tables):
            host[i, :len(t)] = t
        self.guard = Guarded()
        self.k, self.v = (self.guard.empty((self.blocks, heads, bt, dim), torch.uint8, 0x7f) for _ in range(2))
        self.ks, self.vs = (self.guard.empty((self.blocks, heads), torch.float32, scale) for _ in range(2))
        self.table = torch.from_numpy(host).cuda()
        self.desc = b.kv_cache_desc(self.k, self.v, self.ks, self.vs, self.table)
        self.ws = self.guard.workspace(b.templora_kv_cache_append_workspace_bytes(self.desc))

    def host(self):
        return [t.cpu().numpy().copy() for t in (self.k, self.ks, self.v, self.vs)]

    def status(self, b):
        return b.templora_read_device_status(self.ws)[0]


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def rows(seed, n, heads, dim, dtype, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((n, heads, dim), generator=g) * spread).to(DT[dtype])


def f(t):
    return t.double().cpu().numpy()


def same_codes(cache, want):
    for got, ref in zip(cache.host(), want):
        if got.dtype == np.float32:
            assert np.array_equal(got.astype(np.float64), ref.astype(np.float64), equal_nan=True)
        else:
            assert np.array_equal(got, ref)


APPEND = [
    # dtype, heads, dim, block, held, new
    ("bf16", 2, 128, 64, [0], [1]),
    ("bf16", 2, 64, 16, [5, 0, 31], [1, 40, 17]),
    ("bf16", 3, 80, 32, [0, 33, 63, 7], [0, 1, 1, 70]),
    ("bf16", 1, 16, 128, [127, 100, 3], [2, 28, 300]),
    ("f32", 2, 128, 128, [12, 256], [130, 1]),
    ("f32", 2, 96, 16, [3, 16], [1, 1]),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: f"{c[0]}-{c[1]}x{c[2]}-b{c[3]}-{len(c[4])}")
def test_append_matches_oracle_code_by_code(b, case):
    """In two calls: the tokens held first, then, ten times as large in some blocks, the new ones."""
    dtype, heads, dim, bt, held, new = case
    cache = Cache(b, heads, dim, bt, [a + n for a, n in zip(held, new)])
    want = cache.host()
    for step, (before, counts, spread) in enumerate((([0] * len(held), held, 1.0), (held, new, 10.0))):
        total = sum(counts)
        if total == 0:
            continue
        k, v = rows(10 + step, total, heads, dim, dtype, spread), rows(20 + step, total, heads, dim, dtype, 0.3)
        if step == 1:
            k[0, 0, :5] = torch.tensor([float("nan"), float("inf"), float("-inf"), 0.0, 3e38])
        offs = np.concatenate([[0], np.cumsum(counts)]).tolist()
        args = b.KvCacheAppendArgs(cache.desc, i32(before), k.cuda(), v.cuda(), new_offsets=i32(offs))
        b.templora_kv_cache_append(args, cache.ws)
        for x, codes, scales in ((k, want[0], want[1]), (v, want[2], want[3])):
            for s, n in enumerate(counts):
                orc.kv_append(codes, scales, f(x)[offs[s]:offs[s] + n], before[s], cache.tables[s])
        torch.cuda.synchronize()
        cache.guard.check()
        assert cache.status(b) == 0
        same_codes(cache, want)


def test_append_one_token_each_without_offsets_and_strided_rows(b):
    held, heads, dim, bt = [0, 15, 16, 40], 2, 48, 16
    cache = Cache(b, heads, dim, bt, [n + 1 for n in held])
    want = cache.host()
    cache.ks.fill_(1.0), cache.vs.fill_(1.0)
    want[1][:], want[3][:] = 1.0, 1.0
    buf = torch.randn((4, 3 * heads, dim)).to(torch.bfloat16).cuda()
    k, v = buf[:, heads:2 * heads], buf[:, 2 * heads:]
    b.templora_kv_cache_append(b.KvCacheAppendArgs(cache.desc, i32(held), k, v), cache.ws)
    for x, codes, scales in ((k, want[0], want[1]), (v, want[2], want[3])):
        for s in range(4):
            orc.kv_append(codes, scales, f(x)[s:s + 1], held[s], cache.tables[s])
    torch.cuda.synchronize()
    cache.guard.check()
    same_codes(cache, want)


def test_append_rows_outside_the_offsets_are_ignored(b):
    cache = Cache(b, 1, 16, 16, [3, 2])
    want = cache.host()
    k = rows(3, 9, 1, 16, "bf16")
    b.templora_kv_cache_append(b.KvCacheAppendArgs(cache.desc, i32([0, 0]), k.cuda(), k.cuda(), new_offsets=i32([2, 5, 7])), cache.ws)
    for codes, scales in ((want[0], want[1]), (want[2], want[3])):
        orc.kv_append(codes, scales, f(k)[2:5], 0, cache.tables[0])
        orc.kv_append(codes, scales, f(k)[5:7], 0, cache.tables[1])
    torch.cuda.synchronize()
    same_codes(cache, want)


def test_bad_tables_and_lengths_are_recorded_and_left_out(b):
    for table, lens in (([[99], [1]], [0, 0]), ([[-1], [1]], [0, 0]), ([[0], [1]], [16, 0]), ([[0], [1]], [-4, 0]),
                        ([[0], [1]], [2 ** 31 - 1, 0])):
        cache = Cache(b, 1, 16, 16, [1, 1], spare=0)
        cache.table = i32(table)
        desc = b.kv_cache_desc(cache.k, cache.v, cache.ks, cache.vs, cache.table)
        want = cache.host()
        k = rows(4, 2, 1, 16, "bf16")
        b.templora_kv_cache_append(b.KvCacheAppendArgs(desc, i32(lens), k.cuda(), k.cuda()), cache.ws)
        for codes, scales in ((want[0], want[1]), (want[2], want[3])):
            orc.kv_append(codes, scales, f(k)[1:], 0, [1])
        torch.cuda.synchronize()
        cache.guard.check()
        assert cache.status(b) == b.ERR_INVALID_ARG
        same_codes(cache, want)
        # decode: the sequence reads nothing through a bad entry, the other one is answered
        attn = b.attention_desc(1, 1, 16, b.BF16)
        ws = cache.guard.workspace(b.templora_attention_decode_workspace_bytes(attn, desc))
        q = rows(5, 2, 1, 16, "bf16").cuda()
        o = cache.guard.empty((2, 1, 16), torch.bfloat16)
        b.templora_attention_decode_fwd(b.AttentionDecodeArgs(attn, desc, i32([max(1, min(lens[0] + 1, 40)), 1]), q, o), ws)
        torch.cuda.synchronize()
        cache.guard.check()
        val = orc.kv_read(want[2], want[3], [1], 1)[0, 0]
        assert np.allclose(f(o)[1, 0], val, rtol=2.0 ** -7, atol=0)
        if table[0][0] in (99, -1):
            assert (o[0] == 0).all() and b.templora_read_device_status(ws)[0] == b.ERR_INVALID_ARG


def filled(b, dtype, heads, dim, bt, lens, seed=0, outliers=True):
    """A cache with random codes in every held place, NaN codes everywhere else, and uneven scales."""
    cache = Cache(b, heads, dim, bt, lens, seed=seed)
    g = np.random.default_rng(seed + 1)
    for codes, scales in ((cache.k, cache.ks), (cache.v, cache.vs)):
        hc, hs = codes.cpu().numpy(), scales.cpu().numpy()
        for t, n in zip(cache.tables, lens):
            for i, blk in enumerate(t):
                fill = min(bt, n - i * bt)
                hs[blk] = 2.0 ** g.integers(-9, -3 if outliers else -7, size=heads)
                vals = g.standard_normal((heads, fill, dim)) * 100.0
                hc[blk, :, :fill] = orc.e4m3_encode(np.clip(vals, -448, 448))
        codes.copy_(torch.from_numpy(hc)), scales.copy_(torch.from_numpy(hs))
    return cache


def check_decode(b, cache, dtype, H, Hkv, dim, lens, window=0, softcap=0.0, slopes=None, q=None, wide=False, stream=None):
    attn = b.attention_desc(H, Hkv, dim, {"bf16": b.BF16, "f32": b.F32}[dtype], softcap=softcap, window=window,
                            slopes=None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device="cuda"))
    n = len(lens)
    q = rows(77, n, H, dim, dtype, 0.3) if q is None else q
    ws = cache.guard.workspace(b.templora_attention_decode_workspace_bytes(attn, cache.desc))
    if wide:
        qd = torch.full((n, H + 3, dim), float("nan"), dtype=DT[dtype], device="cuda")[:, :H]
        qd.copy_(q)
        whole = cache.guard.empty((n, H + 1, dim), DT[dtype], 7.0)
        o = whole[:, :H]
    else:
        qd, o = q.cuda(), cache.guard.empty((n, H, dim), DT[dtype])
    lse = cache.guard.empty((n, H), torch.float32)
    args = b.AttentionDecodeArgs(attn, cache.desc, i32(lens), qd, o, lse=lse)
    for _ in range(2):                       # the second call finds the counters as the first left them
        b.templora_attention_decode_fwd(args, ws)
    torch.cuda.synchronize()
    cache.guard.check()
    assert b.templora_read_device_status(ws)[0] == 0
    if wide:
        assert (whole[:, H] == 7.0).all()
    kc, ks, vc, vs = cache.host()
    scale = float(np.float32(dim ** -0.5))
    for s, m in enumerate(lens):
        k, v = orc.kv_read(kc, ks, cache.tables[s], m), orc.kv_read(vc, vs, cache.tables[s], m)
        ref, ref_lse = orc.attention_decode(f(q)[s], k, v, scale, softcap=softcap, slopes=slopes, window=window)
        size = orc.attention_decode(f(q)[s], k, np.abs(v), scale, softcap=softcap, slopes=slopes, window=window)[0]
        bound = ((2.0 ** -11 if dtype == "bf16" else 0.0) + SLACK) * size + ROUND[dtype] * np.abs(ref)
        err = np.abs(f(o)[s] - ref)
        assert np.isfinite(f(o)[s]).all() and (err <= bound).all(), (s, m, (err - bound).max())
        fin = np.isfinite(ref_lse)
        assert np.array_equal(np.isfinite(f(lse)[s]), fin)
        assert (np.abs(f(lse)[s] - ref_lse)[fin] <= SLACK * (1 + np.abs(ref_lse[fin]))).all()
    return o


DECODE = [
    # dtype, H, Hkv, dim, block, lens, modifications
    ("bf16", 1, 1, 128, 64, [1], {}),
    ("bf16", 4, 4, 128, 16, [37], {}),
    ("bf16", 8, 1, 128, 64, [700, 1, 64], {}),
    ("bf16", 16, 1, 64, 32, [333, 0, 65], {}),                       # two groups of heads per kv head, an empty sequence
    ("bf16", 12, 1, 64, 128, [513], dict(softcap=10.0)),             # groups of 8 and 4
    ("bf16", 6, 2, 80, 16, [100, 259], dict(slopes=[0.5, 0.25, 0.125, 0.06, 0.03, 0.01])),
    ("bf16", 4, 2, 96, 64, [1000, 30], dict(window=100)),
    ("bf16", 4, 2, 48, 64, [500, 129, 16], dict(window=1)),
    ("bf16", 2, 1, 16, 16, [90], dict(softcap=5.0, window=33)),
    ("bf16", 8, 8, 128, 128, [6001, 17], {}),                        # pairs cut over many CTAs
    ("f32", 4, 2, 128, 64, [300, 1], {}),
    ("f32", 3, 1, 64, 16, [70, 0, 16], dict(softcap=8.0)),
    ("f32", 2, 2, 80, 32, [2000, 31], dict(window=700, slopes=[0.01, 0.02])),
    ("f32", 2, 1, 32, 128, [129], {}),
]


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("case", DECODE, ids=lambda c: "-".join(str(x) for x in c[:5]) + f"-{max(c[5])}" + "".join(sorted(c[6])))
def test_decode_matches_oracle(b, case, wide):
    dtype, H, Hkv, dim, bt, lens, mods = case
    cache = filled(b, dtype, Hkv, dim, bt, lens, seed=3)
    check_decode(b, cache, dtype, H, Hkv, dim, lens, wide=wide, **mods)


def test_decode_of_many_ragged_sequences(b):
    lens = [int(x) for x in np.random.default_rng(5).integers(0, 150, size=300)]
    cache = filled(b, "bf16", 2, 64, 16, lens, seed=5)
    check_decode(b, cache, "bf16", 4, 2, 64, lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("spread", [1e-30, 1e30])
def test_decode_queries_of_extreme_size(b, dtype, spread):
    """Queries at the ends of bf16's range: the scores are ~0 or one key wins; scales of 2^-100 keep them finite."""
    lens = [50, 3]
    cache = filled(b, dtype, 1, 128, 16, lens, seed=6, outliers=False)
    if spread > 1:
        cache.ks.mul_(2.0 ** -100)
    check_decode(b, cache, dtype, 2, 1, 128, lens, q=rows(8, 2, 2, 128, dtype, spread))


def test_decode_weighs_blocks_of_very_different_scale(b):
    """A block whose values are 2^40 times another's, with next to no weight: the small ones must not be lost."""
    lens = [32]
    cache = filled(b, "bf16", 1, 64, 16, lens, seed=9)
    t = cache.tables[0]
    cache.vs[t[0]] = 2.0 ** -40
    cache.vs[t[1]] = 2.0 ** -1
    k = cache.k.cpu().numpy()
    k[t[0], 0] = orc.e4m3_encode(np.full((16, 64), 64.0))
    k[t[1], 0] = orc.e4m3_encode(np.full((16, 64), -64.0))
    cache.k.copy_(torch.from_numpy(k))
    cache.ks[t[0]] = cache.ks[t[1]] = 2.0 ** -4
    q = torch.ones((1, 2, 64)).to(torch.bfloat16)              # scores +-32: weights e^-64 apart
    check_decode(b, cache, "bf16", 2, 1, 64, lens, q=q)


def test_decode_bad_values_stay_with_who_sees_them(b):
    lens = [40, 40]
    cache = filled(b, "bf16", 1, 64, 16, lens, seed=11)
    cache.v[cache.tables[0][1], 0, 3, 7] = 0x7f                # a NaN among the first sequence's values
    attn = b.attention_desc(2, 1, 64, b.BF16)
    ws = b.alloc_workspace(b.templora_attention_decode_workspace_bytes(attn, cache.desc))
    o = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    b.templora_attention_decode_fwd(b.AttentionDecodeArgs(attn, cache.desc, i32(lens), rows(1, 2, 2, 64, "bf16").cuda(), o), ws)
    bad = torch.isnan(o)
    assert bad[0, :, 7].all() and bad.sum() == 2


def test_generation_loop_recorded_once(b):
    """Append and decode of one step recorded into a graph, replayed while the lengths grow; every step against the
    oracle, which encodes the same tokens in the same order."""
    H, Hkv, dim, bt, held, steps = 4, 2, 64, 16, [14, 0, 30], 5
    n = len(held)
    cache = Cache(b, Hkv, dim, bt, [x + steps for x in held], seed=13)
    attn = b.attention_desc(H, Hkv, dim, b.BF16)
    want = cache.host()
    ctx = rows(30, sum(held), Hkv, dim, "bf16")
    offs = np.concatenate([[0], np.cumsum(held)]).tolist()
    b.templora_kv_cache_append(b.KvCacheAppendArgs(cache.desc, i32([0] * n), ctx.cuda(), ctx.cuda(), new_offsets=i32(offs)), cache.ws)
    for codes, scales in ((want[0], want[1]), (want[2], want[3])):
        for s in range(n):
            orc.kv_append(codes, scales, f(ctx)[offs[s]:offs[s + 1]], 0, cache.tables[s])
    before, after = i32(held), i32([x + 1 for x in held])
    k, v, q = (torch.zeros((n, m, dim), dtype=torch.bfloat16, device="cuda") for m in (Hkv, Hkv, H))
    o = torch.zeros_like(q)
    ws = b.alloc_workspace(b.templora_attention_decode_workspace_bytes(attn, cache.desc))
    put, get = b.KvCacheAppendArgs(cache.desc, before, k, v), b.AttentionDecodeArgs(attn, cache.desc, after, q, o)
    b.templora_attention_decode_fwd(get, ws)                   # one call outside a capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.templora_kv_cache_append(put, cache.ws)
        b.templora_attention_decode_fwd(get, ws)
        before.add_(1)
        after.add_(1)
    for t in range(steps):
        new = [rows(100 + t + 50 * i, n, m, dim, "bf16", 1.0 + t) for i, m in enumerate((Hkv, Hkv, H))]
        for dst, src in zip((k, v, q), new):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        for x, codes, scales in ((new[0], want[0], want[1]), (new[1], want[2], want[3])):
            for s in range(n):
                orc.kv_append(codes, scales, f(x)[s:s + 1], held[s] + t, cache.tables[s])
        same_codes(cache, want)
        for s in range(n):
            m = held[s] + t + 1
            kk, vv = orc.kv_read(want[0], want[1], cache.tables[s], m), orc.kv_read(want[2], want[3], cache.tables[s], m)
            ref = orc.attention_decode(f(new[2])[s], kk, vv, float(np.float32(dim ** -0.5)))[0]
            size = orc.attention_decode(f(new[2])[s], kk, np.abs(vv), float(np.float32(dim ** -0.5)))[0]
            assert (np.abs(f(o)[s] - ref) <= (2.0 ** -11 + SLACK) * size + 2.0 ** -8 * np.abs(ref)).all()
    cache.guard.check()


def test_block_update_and_generation_step_together(b):
    """As a block uses them: q, k, v from the norm and projections, attention, its backward into the projections' update;
    then a decode step whose new key and value go through the cache, compared with the chunk's last row."""
    from paper_2401_11504_b200 import inputs
    T, H, Hkv, dim, d, r, s = 96, 4, 2, 64, 256, 16, 2.0
    norm_w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    x = inputs.make_tensor(5, "attn", "x", (T, d), "normal", 1.0, "bf16", "cuda")
    lins, A, B = [], [], []
    for n, out in (("q", H * dim), ("k", Hkv * dim), ("v", Hkv * dim)):
        h = {k: t.cuda() for k, t in inputs.make_linear(5, f"attn-{n}", T, d, out, r, dtype="bf16").items()}
        st = []
        for m in ("A", "B"):
            master = h[m].float()
            st.append((master, torch.zeros_like(master), torch.zeros_like(master), torch.zeros_like(master), h[m].contiguous()))
        lins.append(b.linear_desc(h["W0"], st[0][4], st[1][4], s))
        A.append(b.param_desc(*st[0][:4], st[0][4])), B.append(b.param_desc(*st[1][:4], st[1][4]))
    bf = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    xn, y = bf(T, d), [bf(T, H * dim), bf(T, Hkv * dim), bf(T, Hkv * dim)]
    b.templora_rmsnorm_fwd(x, norm_w, 1e-5, xn)
    ws_p = b.alloc_workspace(b.templora_update_block_workspace_bytes(lins, T))
    for lin, out in zip(lins, y):
        b.templora_linear_fwd(lin, xn, out, ws_p)
    heads = lambda t, n: t.view(T, n, dim)  # noqa: E731
    q, k, v = heads(y[0], H), heads(y[1], Hkv), heads(y[2], Hkv)
    attn = b.attention_desc(H, Hkv, dim, b.BF16)
    o, lse = bf(T, H, dim), torch.empty((H, T), dtype=torch.float32, device="cuda")
    do = inputs.make_tensor(6, "attn", "do", (T, H * dim), "normal", 1.0, "bf16", "cuda").view(T, H, dim)
    grads = [torch.empty_like(t) for t in (q, k, v)]
    ws = b.alloc_workspace(b.templora_attention_workspace_bytes(attn, T, T))
    args = b.AttentionArgs(attn, q, k, v, o, lse, do=do, dq=grads[0], dk=grads[1], dv=grads[2])
    b.templora_attention_fwd(args, ws)
    b.templora_attention_bwd(args, ws)
    dYs = [g.view(T, -1) for g in grads]
    keep = [t.clone() for t in y]
    dXn, dX = bf(T, d), bf(T, d)
    b.templora_update_attn_in(lins, A, B, x, norm_w, 1e-5, dYs, xn, y, dXn, dX, 1, 5e-5, 0.9, 0.999, 1e-8, 0.0, 0, ws_p)
    torch.cuda.synchronize()
    scale = dim ** -0.5
    ref, _, _ = orc.attention_fwd(f(heads(keep[0], H)), f(heads(keep[1], Hkv)), f(heads(keep[2], Hkv)), scale)
    assert np.abs(f(o) - ref).max() <= 2.0 ** -7 * np.abs(ref).max()
    assert torch.isfinite(dX).all() and float(dX.abs().max()) > 0
    # generation: the chunk's keys and values into the cache in two goes, then the last row's query
    cache = Cache(b, Hkv, dim, 16, [T], seed=21)
    kk, vv = heads(keep[1], Hkv), heads(keep[2], Hkv)
    for a, e in ((0, T - 1), (T - 1, T)):
        b.templora_kv_cache_append(b.KvCacheAppendArgs(cache.desc, i32([a]), kk[a:e], vv[a:e], new_offsets=i32([0, e - a])), cache.ws)
    out = check_decode(b, cache, "bf16", H, Hkv, dim, [T], q=heads(keep[0], H)[T - 1:].cpu())
    # e4m3 rounds every key and value by 2^-4 at most; over 96 tokens the output moves far less than that
    assert np.abs(f(out)[0] - ref[T - 1]).max() <= 2.0 ** -3 * np.abs(ref[T - 1]).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_of_pairs_cut_evenly(b, dtype):
    """More than 32 sequences, and few long ones among many short: shares that hold several pairs and parts of them."""
    lens = [int(x) for x in np.random.default_rng(9).integers(0, 900, size=45)] + [4000, 0, 1]
    cache = filled(b, dtype, 2, 80, 32, lens, seed=9)
    check_decode(b, cache, dtype, 6, 2, 80, lens, window=3500, softcap=20.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("limit", [1, 3])
def test_decode_on_few_sms(b, dtype, limit):
    """Long shares: a warp takes hundreds of steps of a pair, and blocks are looked up in many turns."""
    lens = [17000, 5000]
    cache = filled(b, dtype, 1, 64, 16, lens, seed=10, outliers=False)
    stream = torch.cuda.Stream()
    b.templora_set_stream_sm_limit(stream, limit)
    try:
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            check_decode(b, cache, dtype, 3, 1, 64, lens)
    finally:
        b.templora_set_stream_sm_limit(stream, 0)


def test_decode_scales_far_apart_and_of_other_kinds(b):
    """Neighbouring blocks whose scales are 2^70 apart, in both orders, and a caller's own scales that are no powers of two."""
    lens = [200, 200, 130]
    cache = filled(b, "bf16", 2, 128, 16, lens, seed=12, outliers=False)
    vs = cache.vs.cpu().numpy()
    for i, blk in enumerate(cache.tables[0]):
        vs[blk] = 2.0 ** (-35 if i % 2 else 35)
    for i, blk in enumerate(cache.tables[1]):
        vs[blk] = 2.0 ** (-20 * i)
    for i, blk in enumerate(cache.tables[2]):
        vs[blk] = (1.5, 1.0, 0.75)[i % 3]
    cache.vs.copy_(torch.from_numpy(vs))
    check_decode(b, cache, "bf16", 4, 2, 128, lens)


def test_decode_and_append_beyond_4_gb(b):
    """Blocks at the end of a cache whose codes take more than 2^32 bytes each."""
    heads, dim, bt, n = 2, 128, 128, 140000
    k, v = (torch.empty((n, heads, bt, dim), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((n, heads), float("nan"), device="cuda") for _ in range(2))
    tables, lens = [[n - 1, 5], [131072, n - 2]], [150, 256]
    desc = b.kv_cache_desc(k, v, ks, vs, i32(tables))
    kn, vn = rows(41, sum(lens), heads, dim, "bf16"), rows(42, sum(lens), heads, dim, "bf16", 0.3)
    ws = b.alloc_workspace(b.templora_kv_cache_append_workspace_bytes(desc))
    b.templora_kv_cache_append(b.KvCacheAppendArgs(desc, i32([0, 0]), kn.cuda(), vn.cuda(), new_offsets=i32([0, 150, 406])), ws)
    attn = b.attention_desc(4, heads, dim, b.BF16)
    q = rows(43, 2, 4, dim, "bf16")
    o = torch.empty((2, 4, dim), dtype=torch.bfloat16, device="cuda")
    wd = b.alloc_workspace(b.templora_attention_decode_workspace_bytes(attn, desc))
    b.templora_attention_decode_fwd(b.AttentionDecodeArgs(attn, desc, i32(lens), q.cuda(), o), wd)
    torch.cuda.synchronize()
    assert b.templora_read_device_status(ws)[0] == 0 and b.templora_read_device_status(wd)[0] == 0
    small = [[0, 1], [2, 3]]
    ids = [x for t in tables for x in t]
    for x, codes, scales in ((kn, k, ks), (vn, v, vs)):
        want, ws_ = np.full((4, heads, bt, dim), 0x7f, dtype=np.uint8), np.full((4, heads), np.nan, dtype=np.float32)
        for s, at in enumerate((0, 150)):
            orc.kv_append(want, ws_, f(x)[at:at + lens[s]], 0, small[s])
        got, got_s = codes[ids].cpu().numpy(), scales[ids].cpu().numpy()
        assert np.array_equal(got_s, ws_)
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1, :, :22], want[1, :, :22]) and np.array_equal(got[2:], want[2:])
        if x is kn:
            kw, kws = want, ws_
        else:
            vw, vws = want, ws_
    scale = float(np.float32(dim ** -0.5))
    for s in range(2):
        kk, vv = orc.kv_read(kw, kws, small[s], lens[s]), orc.kv_read(vw, vws, small[s], lens[s])
        ref = orc.attention_decode(f(q)[s], kk, vv, scale)[0]
        size = orc.attention_decode(f(q)[s], kk, np.abs(vv), scale)[0]
        assert (np.abs(f(o)[s] - ref) <= (2.0 ** -11 + SLACK) * size + 2.0 ** -8 * np.abs(ref)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_with_the_smallest_cap(b, dtype):
    """A subnormal cap makes every score 0 (zero queries among them): the mean of the values."""
    lens = [70, 3]
    cache = filled(b, dtype, 1, 64, 16, lens, seed=14)
    q = rows(77, 2, 2, 64, dtype, 0.3)
    q[0, 1] = 0
    attn = b.attention_desc(2, 1, 64, {"bf16": b.BF16, "f32": b.F32}[dtype], softcap=1e-39)
    ws = b.alloc_workspace(b.templora_attention_decode_workspace_bytes(attn, cache.desc))
    o = torch.empty((2, 2, 64), dtype=DT[dtype], device="cuda")
    b.templora_attention_decode_fwd(b.AttentionDecodeArgs(attn, cache.desc, i32(lens), q.cuda(), o), ws)
    torch.cuda.synchronize()
    _, _, vc, vs = cache.host()
    for s, m in enumerate(lens):
        v = orc.kv_read(vc, vs, cache.tables[s], m)[:, 0]
        bound = ((2.0 ** -11 if dtype == "bf16" else 0.0) + SLACK) * np.abs(v).mean(axis=0) + ROUND[dtype] * np.abs(v.mean(axis=0))
        for h in range(2):
            assert (np.abs(f(o)[s, h] - v.mean(axis=0)) <= bound).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("softcap", [2e5, 3e38])
def test_decode_with_large_caps(b, dtype, softcap):
    lens = [70, 300]
    cache = filled(b, dtype, 1, 64, 16, lens, seed=15, outliers=False)
    check_decode(b, cache, dtype, 2, 1, 64, lens, softcap=float(np.float32(softcap)))


def odd_rows(t, extra, guard=None, fill=float("nan")):
    """The same rows `extra` elements further apart, so that most of them begin off a 16-byte boundary."""
    n, heads, dim = t.shape
    pitch = heads * dim + extra
    buf = torch.full((n * pitch,), fill, dtype=t.dtype, device="cuda") if guard is None else guard.empty((n * pitch,), t.dtype, fill)
    view = buf.as_strided((n, heads, dim), (pitch, dim, 1))
    view.copy_(t)
    return view, buf


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("extra", [1, 3])
def test_rows_at_odd_distances(b, dtype, extra):
    """New rows, queries and outputs whose stride is no multiple of 16 bytes, against the same rows one after the other."""
    held, new, heads, dim, bt, H = [5, 0, 31], [1, 40, 17], 2, 80, 16, 6
    offs = np.concatenate([[0], np.cumsum(new)]).tolist()
    k, v = rows(50, offs[-1], heads, dim, dtype), rows(51, offs[-1], heads, dim, dtype, 0.3)
    first = rows(52, sum(held), heads, dim, dtype)
    at = np.concatenate([[0], np.cumsum(held)]).tolist()
    cache = Cache(b, heads, dim, bt, [a + n for a, n in zip(held, new)])
    want = cache.host()
    b.templora_kv_cache_append(b.KvCacheAppendArgs(cache.desc, i32([0] * 3), first.cuda(), first.cuda(), new_offsets=i32(at)), cache.ws)
    kd, vd = odd_rows(k, extra)[0], odd_rows(v, extra + 2)[0]
    b.templora_kv_cache_append(b.KvCacheAppendArgs(cache.desc, i32(held), kd, vd, new_offsets=i32(offs)), cache.ws)
    for x, codes, scales in ((k, want[0], want[1]), (v, want[2], want[3])):
        for s in range(3):
            orc.kv_append(codes, scales, f(first)[at[s]:at[s + 1]], 0, cache.tables[s])
            orc.kv_append(codes, scales, f(x)[offs[s]:offs[s + 1]], held[s], cache.tables[s])
    torch.cuda.synchronize()
    cache.guard.check()
    assert cache.status(b) == 0
    same_codes(cache, want)

    lens = [a + n for a, n in zip(held, new)]
    q = rows(53, 3, H, dim, dtype, 0.3)
    plain = check_decode(b, cache, dtype, H, heads, dim, lens, q=q)
    attn = b.attention_desc(H, heads, dim, {"bf16": b.BF16, "f32": b.F32}[dtype])
    ws = cache.guard.workspace(b.templora_attention_decode_workspace_bytes(attn, cache.desc))
    o, buf = odd_rows(torch.zeros((3, H, dim), dtype=DT[dtype]), extra, cache.guard, 7.0)
    b.templora_attention_decode_fwd(b.AttentionDecodeArgs(attn, cache.desc, i32(lens), odd_rows(q, extra)[0], o), ws)
    torch.cuda.synchronize()
    cache.guard.check()
    assert torch.equal(o, plain)
    assert (buf.view(3, -1)[:, H * dim:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_of_one_long_sequence_among_short_ones(b, dtype):
    """Nearly all CTAs work on one pair, whole CTAs to each pair and cut evenly (more than 32 sequences)."""
    for lens in ([17000, 64], [17000] + [1] * 33):
        cache = filled(b, dtype, 1, 64, 64, lens, seed=16, outliers=False)
        check_decode(b, cache, dtype, 4, 1, 64, lens)
