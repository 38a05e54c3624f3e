"""Cache weights, cache eviction and sampling against the fp64 oracle, and a run of append, decode, weigh, evict and sample as a
generation loop makes them.

Bounds.  Weights: a product of D terms added up in fp32 is off by at most (D + 8) 2^-23 of the sum of its terms' magnitudes
(products are exact; the tensor cores cut each addition off at 2^-23), the cap's tanh by 2^-21, lse and slope terms by a rounding each;
exp turns that into a relative error of the weight, and its own error and the sum's are 2^-20 in all for the sums here.  Eviction is
exact.  Sampling: tokens are equal; the log-probability is rounded once to fp32 from a value that is off by 1e-10."""
import numpy as np
import pytest
import torch

from oracle import templora_oracle as orc
from parity_utils import Guarded

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def b():
    from paper_2401_11504_b200 import build
    build.build_library()
    from paper_2401_11504_b200 import binding
    return binding


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def f(t):
    return t.double().cpu().numpy()


class Pool:
    """A guarded pool of blocks in random order: random codes and power-of-two scales everywhere, tables for the lengths."""

    def __init__(self, b, heads, dim, bt, lens, seed=0, spare=2, more=(), spread=3, width=None):
        g = np.random.default_rng(seed)
        need = [-(-n // bt) for n in lens]
        extra = [-(-n // bt) for n in more]
        self.bt, self.heads, self.dim = bt, heads, dim
        self.blocks = sum(need) + sum(extra) + spare
        ids = [int(x) for x in g.permutation(self.blocks)]
        self.guard = Guarded()
        codes = g.integers(0, 256, size=(2, self.blocks, heads, bt, dim)).astype(np.uint8)
        codes[(codes & 0x7f) == 0x7f] = 0x30                      # NaN only where a test puts it
        codes[0] = np.where((codes[0] & 0x78) > 0x40, codes[0] & 0xbf, codes[0])      # keys of moderate size
        self.codes = codes
        self.scales = 2.0 ** g.integers(-spread, spread + 1, size=(2, self.blocks, heads)).astype(np.float32)
        self.w = (g.random((self.blocks, heads, bt)) * 4).astype(np.float32)
        self.k, self.v = (self.guard.empty(codes[0].shape, torch.uint8, 0) for _ in range(2))
        self.ks, self.vs = (self.guard.empty((self.blocks, heads), torch.float32) for _ in range(2))
        self.weights = self.guard.empty(self.w.shape, torch.float32)
        self.table_of = lambda counts: [[ids.pop() for _ in range(n)] for n in counts]  # noqa: E731
        self.tables = self.table_of(need)
        self.desc = self.describe(b, self.tables, width)
        if len(more):
            self.to_tables = self.table_of(extra)
            self.to = self.describe(b, self.to_tables)
        self.upload()

    def describe(self, b, tables, width=None):
        host = np.full((len(tables), width or max(len(t) for t in tables) + 1), -5, dtype=np.int32)
        for i, t in enumerate(tables):
            host[i, :len(t)] = t
        return b.kv_cache_desc(self.k, self.v, self.ks, self.vs, torch.from_numpy(host).cuda())

    def upload(self):
        for t, x in ((self.k, self.codes[0]), (self.v, self.codes[1]), (self.ks, self.scales[0]), (self.vs, self.scales[1]), (self.weights, self.w)):
            t.copy_(torch.from_numpy(np.ascontiguousarray(x)))

    def same(self, k, ks, v, vs, w):
        for name, got, want in (("k", self.k, k), ("v", self.v, v), ("k_scale", self.ks, ks), ("v_scale", self.vs, vs), ("weights", self.weights, w)):
            got = got.cpu().numpy()
            want = np.asarray(want).astype(got.dtype)
            same = (got == want) | (np.isnan(got) & np.isnan(want))
            assert same.all(), (name, [(int(x), got[tuple(at)], want[tuple(at)]) for x, at in zip(range(4), np.argwhere(~same))])


# ------------------------------------------------------------------ weights
def weigh_reference(pool, q, lse, lens, counts, scale, softcap=0.0, slopes=None, window=0):
    """The weights afterwards and how far each may be off."""
    want, slack = pool.w.astype(np.float64), np.zeros(pool.w.shape)
    at = 0
    for s, (n, r) in enumerate(zip(lens, counts)):
        rows, e = f(q)[at:at + r], lse[at:at + r]
        at += r
        if r == 0 or n == 0:
            continue
        k = orc.kv_read(pool.codes[0], pool.scales[0].astype(np.float64), pool.tables[s], n)
        kw = dict(softcap=softcap, slopes=slopes, window=window)
        a = orc.attention_received(rows, e, k, scale, **kw)
        # the scores' error, largest over the rows and heads
        size = np.abs(scale) * np.einsum("ihd,jhd->jhi", np.abs(rows).reshape(r, pool.heads, -1, pool.dim).transpose(0, 2, 1, 3).reshape(-1, pool.heads, pool.dim),
                                         np.abs(k)).max(-1).T
        far = max(n, 1) * (max(slopes) if slopes is not None else 0.0)
        finite = np.abs(e[np.isfinite(e)])
        d = (pool.dim + 8) * 2.0 ** -23 * size + 2.0 ** -21 * softcap + 2.0 ** -22 * (far + (finite.max() if finite.size else 0.0))
        err = a * (np.expm1(d) + 2.0 ** -20)
        orc.kv_weigh(want, a, r, pool.tables[s])
        for j in range(n):
            slack[pool.tables[s][j // pool.bt], :, j % pool.bt] = err[:, j]
    return want, slack + 2.0 ** -23 * np.abs(want) + 1e-37


def softmax_rows(pool, q, lens, counts, H, scale, softcap=0.0, slopes=None, window=0):
    """lse [rows, H] that the step's attention leaves."""
    out, at = [], 0
    for s, (n, r) in enumerate(zip(lens, counts)):
        if r == 0:
            continue
        k = orc.kv_read(pool.codes[0], pool.scales[0].astype(np.float64), pool.tables[s], n) if n else np.zeros((0, pool.heads, pool.dim))
        e = np.full((r, H), -np.inf)
        if n:
            z, _ = orc.attention_scores(f(q)[at:at + r], k, scale, softcap=softcap, slopes=slopes, q_start=n - r, causal=True, window=window)
            with np.errstate(divide="ignore"):
                top = z.max(-1, keepdims=True)
                top = np.where(np.isneginf(top), 0.0, top)
                e = (top[..., 0] + np.log(np.exp(z - top).sum(-1))).T
        out.append(e)
        at += r
    return np.concatenate(out)


def check_weigh(b, pool, dtype, H, lens, counts, seed=0, by_heads=False, offsets=None, lse=None, q=None, stream=None, twice=False, **kw):
    """counts None: one row per sequence."""
    rows = [1] * len(lens) if counts is None else counts
    g = torch.Generator().manual_seed(seed)
    if q is None:
        q = (torch.randn((sum(rows), H, pool.dim), generator=g) * 0.5).to(DT[dtype])
    scale = float(np.float32(pool.dim ** -0.5))
    slopes = kw.get("slopes")
    if lse is None:
        lse = softmax_rows(pool, q, lens, rows, H, scale, **kw)
    lse = lse.astype(np.float32)
    attn = b.attention_desc(H, pool.heads, pool.dim, {"bf16": b.BF16, "f32": b.F32}[dtype], scale=scale, softcap=kw.get("softcap", 0.0),
                            window=kw.get("window", 0), slopes=None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device="cuda"))
    dev = torch.from_numpy(lse).cuda()
    if by_heads:
        dev = dev.T.contiguous().T
    if counts is not None and offsets is None:
        offsets = np.concatenate([[0], np.cumsum(rows)]).tolist()
    ws = pool.guard.workspace(b.templora_kv_cache_weigh_workspace_bytes(attn, pool.desc, q.shape[0]))
    args = b.KvCacheWeighArgs(attn, pool.desc, i32(lens), q.cuda(), dev, pool.weights, row_offsets=None if counts is None else i32(offsets))
    b.templora_kv_cache_weigh(args, ws, stream=stream)
    torch.cuda.synchronize()
    pool.guard.check()
    assert b.templora_read_device_status(ws)[0] == 0
    want, slack = weigh_reference(pool, q, lse.astype(np.float64), lens, rows, scale, **kw)
    got = f(pool.weights)
    assert (np.isnan(got) == np.isnan(want)).all()
    fine = ~np.isnan(want)
    off = np.abs(got - want)[fine] - slack[fine]
    assert (off <= 0).all(), (off.max(), np.abs(got - want)[fine].max())
    if twice:
        first = pool.weights.clone()
        pool.upload()
        b.templora_kv_cache_weigh(args, ws, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(first, pool.weights)
    return got


SLOPES = [0.5, 0.25, 0.125, 0.0625, 0.03125, 0.25, 0.5, 0.125]
STEPS = [
    # dtype, query heads, kv heads, dim, block, lens, masks
    ("bf16", 2, 2, 128, 64, [1], {}),
    ("bf16", 8, 1, 128, 64, [37, 0, 64, 300], {}),
    ("bf16", 3, 1, 64, 16, [15, 16, 17, 1, 250], dict(softcap=5.0)),
    ("bf16", 8, 2, 80, 32, [100, 3, 65], dict(slopes=SLOPES, window=20)),
    ("bf16", 16, 1, 96, 16, [90, 1, 33], dict(window=33)),            # more heads of a kv head than a product has columns
    ("bf16", 24, 2, 16, 128, [200, 129], dict(slopes=SLOPES * 3)),
    ("bf16", 17, 1, 128, 64, [70, 300], dict(softcap=4.0)),
    ("bf16", 11, 1, 64, 32, [900], dict(slopes=SLOPES + SLOPES[:3])),
    ("f32", 4, 4, 128, 128, [130, 7], {}),
    ("f32", 5, 1, 48, 16, [77, 16, 1], dict(softcap=2.0, window=30)),
    ("f32", 20, 2, 64, 32, [40, 95], {}),
    ("bf16", 4, 2, 128, 64, [5000, 13, 1200], {}),
]


@pytest.mark.parametrize("case", STEPS, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}x{c[3]}-b{c[4]}-{sum(c[5])}")
def test_weigh_of_one_row_per_sequence(b, case):
    dtype, H, heads, dim, bt, lens, kw = case
    pool = Pool(b, heads, dim, bt, lens, seed=1)
    for s, n in enumerate(lens):       # what a new token's place holds does not count
        if n:
            pool.w[pool.tables[s][(n - 1) // bt], :, (n - 1) % bt] = np.nan
    pool.upload()
    got = check_weigh(b, pool, dtype, H, lens, None, twice=True, **kw)
    assert np.isfinite(got).all()


CHUNKS = [
    # dtype, query heads, kv heads, dim, block, lens, rows, masks
    ("bf16", 2, 1, 128, 64, [200], [200], {}),
    ("bf16", 8, 2, 64, 16, [50, 333, 0, 7], [50, 1, 0, 9], {}),          # more rows than tokens
    ("bf16", 6, 2, 80, 32, [300, 100], [130, 0], dict(window=40, softcap=4.0)),
    ("bf16", 8, 1, 96, 128, [520, 1], [100, 1], dict(slopes=SLOPES)),
    ("f32", 4, 2, 128, 64, [140, 65], [70, 3], {}),
    ("f32", 3, 3, 64, 16, [90], [33], dict(window=1)),
    ("f32", 8, 4, 112, 32, [257, 20], [19, 20], dict(slopes=SLOPES, window=100, softcap=3.0)),
]


@pytest.mark.parametrize("case", CHUNKS, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}x{c[3]}-{sum(c[5])}-{sum(c[6])}")
@pytest.mark.parametrize("path", [0, 1])
def test_weigh_of_chunks(b, case, path):
    """On the tensor cores where they apply, and on the generic kernel."""
    dtype, H, heads, dim, bt, lens, counts, kw = case
    pool = Pool(b, heads, dim, bt, lens, seed=2)
    for s, (n, r) in enumerate(zip(lens, counts)):
        for j in range(max(n - r, 0), n):
            pool.w[pool.tables[s][j // bt], :, j % bt] = np.nan
    pool.upload()
    before = b.templora_set_kernel_path(path)
    try:
        got = check_weigh(b, pool, dtype, H, lens, counts, by_heads=path == 0, twice=True, **kw)
    finally:
        b.templora_set_kernel_path(before)
    assert np.isfinite(got).all()


@pytest.mark.parametrize("group,dim", [(1, 128), (5, 80), (16, 64), (40, 16), (128, 48)])
def test_weigh_of_long_chunks_of_any_group(b, group, dim):
    """Several tiles of pairs and of places, several items to a CTA on one SM, groups that do not divide 128."""
    lens, counts, heads = [700, 300], [260 // group + 3, 300 // group + 1], 2
    pool = Pool(b, heads, dim, 32, lens, seed=14)
    check_weigh(b, pool, "bf16", heads * group, lens, counts, twice=True)
    pool = Pool(b, heads, dim, 32, lens, seed=15)
    stream = torch.cuda.Stream()
    b.templora_set_stream_sm_limit(stream, 1)
    try:
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            check_weigh(b, pool, "bf16", heads * group, lens, counts, stream=stream, window=150)
    finally:
        b.templora_set_stream_sm_limit(stream, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [None, [1, 1], [40, 3]])
def test_weigh_hidden_places_and_rows_that_count_for_nothing(b, dtype, counts):
    """NaN codes behind the end and before the window, NaN in rows of others, infinite lse."""
    lens, H, heads, dim, bt = [100, 41], 4, 2, 64, 32
    pool = Pool(b, heads, dim, bt, lens, seed=3)
    window = 30
    first = [n - (1 if counts is None else r) - window + 1 for n, r in zip(lens, counts or [1, 1])]
    for s, n in enumerate(lens):
        for j in list(range(max(first[s], 0))) + list(range(n, len(pool.tables[s]) * bt)):
            pool.codes[0][pool.tables[s][j // bt], :, j % bt] = 0x7f
    # a token that only sequence 0's later rows see
    rows = [1, 1] if counts is None else counts
    q = (torch.randn((sum(rows), H, dim), generator=torch.Generator().manual_seed(4)) * 0.5).to(DT[dtype])
    pool.upload()
    clean = pool.codes.copy()
    pool.codes[0][pool.codes[0] == 0x7f] = 0      # the oracle reads hidden keys too
    lse = softmax_rows(pool, q, lens, rows, H, float(np.float32(dim ** -0.5)), window=window)
    lse[-1, 1], lse[-1, 2] = -np.inf, np.inf
    host = pool.codes
    pool.codes = clean
    pool.upload()
    pool.codes = host
    got = check_weigh(b, pool, dtype, H, lens, counts, q=q, lse=lse, window=window)
    assert np.isfinite(got).all()
    # a NaN key makes its own place NaN and no other
    j = lens[0] - 2
    pool.codes[0][pool.tables[0][j // bt], 1, j % bt, 5] = 0x7f
    pool.upload()
    got = check_weigh(b, pool, dtype, H, lens, counts, q=q, lse=lse, window=window)
    assert np.isnan(got).sum() == 1 and np.isnan(got[pool.tables[0][j // bt], 1, j % bt])


def test_weigh_rows_at_odd_distances_and_offsets_with_gaps(b):
    lens, H, heads, dim, bt = [70, 30], 4, 2, 80, 16
    for dtype in ("bf16", "f32"):
        for counts, offsets in ((None, None), ([5, 9], [0, 5, 14])):
            pool = Pool(b, heads, dim, bt, lens, seed=5)
            n = 2 if counts is None else 14
            buf = torch.zeros(n * (H * dim + 3), dtype=DT[dtype], device="cuda")
            q = (torch.randn((n, H, dim), generator=torch.Generator().manual_seed(6)) * 0.5).to(DT[dtype])
            view = buf.as_strided((n, H, dim), (H * dim + 3, dim, 1))
            view.copy_(q)
            plain = check_weigh(b, pool, dtype, H, lens, counts, q=q, offsets=offsets)
            pool.upload()
            scale = float(np.float32(dim ** -0.5))
            lse = torch.from_numpy(softmax_rows(pool, q, lens, counts or [1, 1], H, scale).astype(np.float32)).cuda()
            attn = b.attention_desc(H, heads, dim, {"bf16": b.BF16, "f32": b.F32}[dtype], scale=scale)
            ws = b.alloc_workspace(b.templora_kv_cache_weigh_workspace_bytes(attn, pool.desc, n))
            b.templora_kv_cache_weigh(b.KvCacheWeighArgs(attn, pool.desc, i32(lens), view, lse, pool.weights,
                                                         row_offsets=None if offsets is None else i32(offsets)), ws)
            torch.cuda.synchronize()
            assert np.array_equal(f(pool.weights), plain)
    # rows in front of and behind all sequences' are ignored, offsets beyond the rows are clamped
    pool = Pool(b, heads, dim, bt, lens, seed=5)
    wide = torch.full((n + 5, H, dim), float("nan"), dtype=torch.float32)
    wide[3:3 + n] = q
    wide_lse = torch.full((n + 5, H), float("nan"))
    wide_lse[3:3 + n] = lse.cpu()
    attn = b.attention_desc(H, heads, dim, b.F32, scale=scale)
    b.templora_kv_cache_weigh(b.KvCacheWeighArgs(attn, pool.desc, i32(lens), wide.cuda(), wide_lse.cuda(), pool.weights, row_offsets=i32([3, 8, 17])), ws)
    torch.cuda.synchronize()
    assert np.array_equal(f(pool.weights), plain)
    pool.upload()
    cut, cut_lse = wide[3:17].cuda(), lse
    b.templora_kv_cache_weigh(b.KvCacheWeighArgs(attn, pool.desc, i32(lens), cut, cut_lse, pool.weights, row_offsets=i32([-4, 5, 99])), ws)
    torch.cuda.synchronize()
    assert np.array_equal(f(pool.weights), plain)


# few places and many rows: a cluster of CTAs shares out an item's pairs, more of them than some sequences have
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,heads,dim,lens,counts,masks", [
    (8, 1, 64, [300], [290], {}),
    (8, 1, 80, [300, 41, 0, 17], [200, 1, 0, 17], {}),
    (16, 2, 128, [150, 500], [150, 90], dict(softcap=0.5)),
    (8, 2, 48, [260, 33], [130, 33], dict(slopes=SLOPES, window=30)),
    (8, 1, 128, [700], [64], dict(slopes=SLOPES, softcap=2.0, window=129)),
    (5, 5, 32, [129], [129], dict(window=1)),
])
def test_weigh_of_few_places_by_many_rows(b, dtype, H, heads, dim, lens, counts, masks):
    check_weigh(b, Pool(b, heads, dim, 32, lens, seed=21), dtype, H, lens, counts, twice=True, **masks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,masks", [(40, {}), (40, dict(softcap=3.0)), (200, dict(window=90))])
def test_weigh_rows_beside_those_of_the_sequences_do_not_matter(b, dtype, n, masks):
    lens, H, heads, dim, bt = [70 + n, 30 + n], 4, 2, 64, 16
    q = (torch.randn((2 * n, H, dim), generator=torch.Generator().manual_seed(31)) * 0.5).to(DT[dtype])
    pool = Pool(b, heads, dim, bt, lens, seed=32)
    plain = check_weigh(b, pool, dtype, H, lens, [n, n], q=q, **masks)
    scale = float(np.float32(dim ** -0.5))
    # the wider call may be another kernel's, which adds up in another order: both are within the formula's bound, not equal
    exact, slack = weigh_reference(pool, q, softmax_rows(pool, q, lens, [n, n], H, scale, **masks).astype(np.float32).astype(np.float64), lens, [n, n],
                                   scale, **masks)
    wide = torch.full((2 * n + 30, H, dim), float("nan"), dtype=DT[dtype])
    lse = torch.full((2 * n + 30, H), float("nan"))
    rows = list(range(10, 10 + n)) + list(range(20 + n, 20 + 2 * n))
    wide[rows] = q
    lse[rows] = torch.from_numpy(softmax_rows(pool, q, lens, [n, n], H, scale, **masks).astype(np.float32))
    attn = b.attention_desc(H, heads, dim, {"bf16": b.BF16, "f32": b.F32}[dtype], scale=scale, softcap=masks.get("softcap", 0.0),
                            window=masks.get("window", 0))
    for part, (first, last) in enumerate(((10, 10 + n), (20 + n, 20 + 2 * n))):      # a sequence's rows, and none of the other's
        pool.upload()
        offsets = [first, last, last] if part == 0 else [first, first, last]
        ws = b.alloc_workspace(b.templora_kv_cache_weigh_workspace_bytes(attn, pool.desc, 2 * n + 30))
        before = f(pool.weights)
        b.templora_kv_cache_weigh(b.KvCacheWeighArgs(attn, pool.desc, i32(lens), wide.cuda(), lse.cuda(), pool.weights, row_offsets=i32(offsets)), ws)
        torch.cuda.synchronize()
        assert b.templora_read_device_status(ws)[0] == 0
        got, changed = f(pool.weights), plain != before
        mine = got != before
        assert mine.any() and (changed | ~mine).all()
        assert (np.abs(got - exact)[mine] <= slack[mine]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,masks", [(3, {}), (40, {}), (40, dict(softcap=3.0)), (200, dict(window=90))])
@pytest.mark.parametrize("beside", [0, 30, 700])
def test_weigh_of_one_sequence_among_rows_of_none_reaches_all_its_places_and_no_others(b, dtype, n, masks, beside):
    """The whole array of weights: within the bound at every place of the sequence whose rows are given, untouched elsewhere."""
    lens, H, heads, dim, bt = [270 + n, 130 + n], 8, 2, 64, 16
    q = (torch.randn((2 * n, H, dim), generator=torch.Generator().manual_seed(33)) * 0.5).to(DT[dtype])
    pool = Pool(b, heads, dim, bt, lens, seed=34)
    scale = float(np.float32(dim ** -0.5))
    lse = softmax_rows(pool, q, lens, [n, n], H, scale, **masks).astype(np.float32)
    exact, slack = weigh_reference(pool, q, lse.astype(np.float64), lens, [n, n], scale, **masks)
    wide, wide_lse = torch.full((2 * n + beside, H, dim), float("nan"), dtype=DT[dtype]), torch.full((2 * n + beside, H), float("nan"))
    first = beside // 3
    wide[first:first + 2 * n], wide_lse[first:first + 2 * n] = q, torch.from_numpy(lse)
    attn = b.attention_desc(H, heads, dim, {"bf16": b.BF16, "f32": b.F32}[dtype], scale=scale, softcap=masks.get("softcap", 0.0),
                            window=masks.get("window", 0))
    ws = pool.guard.workspace(b.templora_kv_cache_weigh_workspace_bytes(attn, pool.desc, len(wide)))
    for s, offsets in enumerate(([first, first + n, first + n], [first + n, first + n, first + 2 * n])):
        pool.upload()
        b.templora_kv_cache_weigh(b.KvCacheWeighArgs(attn, pool.desc, i32(lens), wide.cuda(), wide_lse.cuda(), pool.weights, row_offsets=i32(offsets)), ws)
        torch.cuda.synchronize()
        pool.guard.check()
        assert b.templora_read_device_status(ws)[0] == 0
        want, off = pool.w.astype(np.float64), np.zeros(pool.w.shape)
        seen = max(lens[s] - n - masks["window"] + 1, 0) if masks.get("window") else 0
        for j in range(seen, lens[s]):
            at = (pool.tables[s][j // bt], slice(None), j % bt)
            want[at], off[at] = exact[at], slack[at]
        got = f(pool.weights)
        assert (np.abs(got - want) <= off).all(), np.argwhere(np.abs(got - want) > off)[:4]
        assert (want[off > 0] != pool.w[off > 0]).all()


@pytest.mark.parametrize("pitch", [0, 3, 8])
def test_weigh_many_fp32_rows_at_any_distance(b, pitch):
    lens, counts, H, heads, dim, bt = [260, 190], [150, 101], 4, 1, 80, 32
    pool = Pool(b, heads, dim, bt, lens, seed=41)
    n = sum(counts)
    q = torch.randn((n, H, dim), generator=torch.Generator().manual_seed(42)) * torch.logspace(-3, 0.2, n)[:, None, None]
    buf = torch.zeros(n * (H * dim + pitch), device="cuda")
    view = buf.as_strided((n, H, dim), (H * dim + pitch, dim, 1))
    view.copy_(q)
    plain = check_weigh(b, pool, "f32", H, lens, counts, q=q, twice=True)
    pool.upload()
    scale = float(np.float32(dim ** -0.5))
    lse = torch.from_numpy(softmax_rows(pool, q, lens, counts, H, scale).astype(np.float32)).cuda()
    attn = b.attention_desc(H, heads, dim, b.F32, scale=scale)
    need = b.templora_kv_cache_weigh_workspace_bytes(attn, pool.desc, n)
    args = b.KvCacheWeighArgs(attn, pool.desc, i32(lens), view, lse, pool.weights, row_offsets=i32([0, counts[0], n]))
    with pytest.raises(b.TemploraError):
        b.templora_kv_cache_weigh(args, b.alloc_workspace(need - 1024))
    b.templora_kv_cache_weigh(args, b.alloc_workspace(need))
    torch.cuda.synchronize()
    assert np.array_equal(f(pool.weights), plain)
    # a row of NaN or infinities reaches the places that it sees, and no others
    bad = q.clone()
    bad[30] = float("nan")
    bad[60, 1] = float("inf")
    pool.upload()
    b.templora_kv_cache_weigh(b.KvCacheWeighArgs(attn, pool.desc, i32(lens), bad.cuda(), lse, pool.weights, row_offsets=i32([0, counts[0], n])),
                              b.alloc_workspace(need))
    torch.cuda.synchronize()
    got = f(pool.weights)
    first = lens[0] - counts[0]
    at = np.array([[pool.tables[0][j // bt], 0, j % bt] for j in range(lens[0])])
    seen = got[tuple(at.T)]
    assert np.isnan(seen[:first + 31]).all() and not np.isnan(seen[first + 61:]).any()
    other = np.ones(got.shape, dtype=bool)
    other[tuple(at.T)] = False
    assert np.array_equal(got[other], plain[other])


@pytest.mark.parametrize("rows", [1, 4])
def test_weigh_bad_lengths_and_tables_are_recorded_and_left_out(b, rows):
    lens, H, heads, dim, bt = [40, 60, 33, 20], 2, 1, 64, 16
    pool = Pool(b, heads, dim, bt, lens, seed=7)
    table = pool.desc._keep[4]
    table[1, 2] = pool.blocks
    want_lens = [40, 60, -1, 16 * table.shape[1] + 1]
    q = (torch.randn((4 * rows, H, dim), generator=torch.Generator().manual_seed(8)) * 0.5).to(torch.bfloat16)
    scale = float(np.float32(dim ** -0.5))
    lse = softmax_rows(pool, q, lens, [rows] * 4, H, scale).astype(np.float32)
    attn = b.attention_desc(H, heads, dim, b.BF16, scale=scale)
    ws = pool.guard.workspace(b.templora_kv_cache_weigh_workspace_bytes(attn, pool.desc, 4 * rows))
    args = b.KvCacheWeighArgs(attn, pool.desc, i32(want_lens), q.cuda(), torch.from_numpy(lse).cuda(), pool.weights,
                              row_offsets=None if rows == 1 else i32([rows * s for s in range(5)]))
    b.templora_kv_cache_weigh(args, ws)
    torch.cuda.synchronize()
    pool.guard.check()
    assert b.templora_read_device_status(ws)[0] == b.ERR_INVALID_ARG
    want, slack = weigh_reference(pool, q, lse.astype(np.float64), lens, [rows] * 4, scale)
    for blk in (*pool.tables[2], *pool.tables[3], pool.tables[1][2]):
        want[blk], slack[blk] = pool.w[blk], 0.0
    assert (np.abs(f(pool.weights) - want) <= slack).all()


def test_weigh_many_sequences_few_sms_and_other_streams(b):
    lens = [int(x) for x in np.random.default_rng(11).integers(0, 60, size=300)]
    pool = Pool(b, 2, 64, 16, lens, seed=12)
    stream = torch.cuda.Stream()
    for limit in (0, 1, 3):
        b.templora_set_stream_sm_limit(stream, limit)
        try:
            for counts in (None, [i % 3 for i in range(300)]):
                pool.upload()
                torch.cuda.synchronize()
                with torch.cuda.stream(stream):
                    check_weigh(b, pool, "bf16", 4, lens, counts, stream=stream)
        finally:
            b.templora_set_stream_sm_limit(stream, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weigh_extreme_scales_and_caps(b, dtype):
    """Zero queries under any scale: every place gets exp(-lse), not NaN; a large cap is none."""
    lens, H, heads, dim, bt = [33, 5], 2, 1, 64, 16
    for counts in (None, [2, 2]):
        for scale, softcap in ((3e38, 0.0), (-3e38, 0.0), (0.125, 3e38), (0.125, 1e-39)):
            pool = Pool(b, heads, dim, bt, lens, seed=13, spread=30)
            n = 2 if counts is None else 4
            attn = b.attention_desc(H, heads, dim, {"bf16": b.BF16, "f32": b.F32}[dtype], scale=scale, softcap=softcap)
            ws = b.alloc_workspace(b.templora_kv_cache_weigh_workspace_bytes(attn, pool.desc, n))
            q = torch.zeros((n, H, dim), dtype=DT[dtype], device="cuda")
            b.templora_kv_cache_weigh(b.KvCacheWeighArgs(attn, pool.desc, i32(lens), q, torch.zeros((n, H), device="cuda"), pool.weights,
                                                         row_offsets=None if counts is None else i32([0, 2, 4])), ws)
            torch.cuda.synchronize()
            r = 1 if counts is None else 2
            want = pool.w.astype(np.float64)
            for s, m in enumerate(lens):
                a = np.array([[H * min(r, m - j) for j in range(m)]], dtype=np.float64)
                orc.kv_weigh(want, a, r, pool.tables[s])
            assert np.abs(f(pool.weights) - want).max() <= 1e-5


# ------------------------------------------------------------------ eviction
def check_evict(b, pool, lens, keep, first=0, recent=0, with_kept=True, alias=False, to=None, stream=None):
    """`to`: another pool; else the same under its second tables."""
    n, heads = len(lens), pool.heads
    dst = to or pool
    out = [x.copy() for x in (dst.codes[0], dst.scales[0], dst.codes[1], dst.scales[1], dst.w)]
    kept = torch.full((n, heads, keep), -9, dtype=torch.int32, device="cuda")
    lens_d = i32(lens)
    new = lens_d if alias else torch.full((n,), -1, dtype=torch.int32, device="cuda")
    ws = pool.guard.workspace(b.templora_kv_cache_evict_workspace_bytes(pool.desc, keep))
    desc = to.desc if to else pool.to
    args = b.KvCacheEvictArgs(pool.desc, pool.weights, lens_d, desc, dst.weights, new, keep, n_first=first, n_recent=recent,
                              kept=kept if with_kept else None)
    b.templora_kv_cache_evict(args, ws, stream=stream)
    torch.cuda.synchronize()
    pool.guard.check(), dst.guard.check()
    assert b.templora_read_device_status(ws)[0] == 0
    want_kept = np.full(kept.shape, -9, dtype=np.int32)
    for s, m in enumerate(lens):
        places = orc.kv_evict(pool.codes[0], pool.scales[0].astype(np.float64), pool.codes[1], pool.scales[1].astype(np.float64), pool.w,
                              pool.tables[s], m, out, (to.tables if to else pool.to_tables)[s], keep, first, recent)
        for h, p in enumerate(places):
            want_kept[s, h, :len(p)] = p
    assert new.cpu().tolist() == [min(m, keep) for m in lens]
    if with_kept:
        assert np.array_equal(kept.cpu().numpy(), want_kept)
    dst.same(*out)
    if to:
        pool.same(pool.codes[0], pool.scales[0], pool.codes[1], pool.scales[1], pool.w)


EVICTIONS = [
    # heads, dim, block, lens, keep, first, recent
    (1, 16, 16, [1], 1, 0, 0),
    (2, 64, 16, [90, 0, 48, 49, 200], 48, 4, 16),
    (3, 80, 32, [100, 33, 1], 33, 0, 0),
    (2, 128, 64, [700, 640, 65], 65, 65, 0),
    (1, 128, 128, [500, 129], 200, 0, 200),
    (2, 96, 16, [40, 41, 42], 41, 20, 20),
    (1, 48, 64, [333], 1, 0, 0),
    (4, 128, 128, [900], 899, 1, 1),
]


@pytest.mark.parametrize("case", EVICTIONS, ids=lambda c: f"{c[0]}x{c[1]}-b{c[2]}-{sum(c[3])}-keep{c[4]}")
@pytest.mark.parametrize("ties", [False, True])
def test_evict_matches_oracle_code_by_code(b, case, ties):
    heads, dim, bt, lens, keep, first, recent = case
    pool = Pool(b, heads, dim, bt, lens, seed=20, more=[min(n, keep) for n in lens], spread=12)
    if ties:
        pool.w = np.floor(pool.w).astype(np.float32)
        g = np.random.default_rng(21)
        for bad in (np.nan, -np.inf, np.inf, -0.0, 1e-42):
            pool.w[g.random(pool.w.shape) < 0.05] = bad
        pool.codes[g.random(pool.codes.shape) < 0.01] = 0x7f
        pool.codes[g.random(pool.codes.shape) < 0.01] = 0xff
        pool.codes[:, :, :, :, :] = np.where(g.random((2, pool.blocks, heads, bt, 1)) < 0.2, 0x80, pool.codes)      # tokens of zeros
        pool.upload()
    check_evict(b, pool, lens, keep, first, recent)


def test_evict_into_another_pool_aliased_lengths_no_list(b):
    lens, keep = [70, 12, 33], 32
    pool = Pool(b, 2, 64, 16, lens, seed=22)
    to = Pool(b, 2, 64, 16, [keep] * 3, seed=23, width=2)
    check_evict(b, pool, lens, keep, 2, 5, to=to, with_kept=False, alias=True)
    pool = Pool(b, 2, 64, 16, lens, seed=24, more=[min(n, keep) for n in lens])
    check_evict(b, pool, lens, keep, 2, 5, with_kept=False, alias=True)


def test_evict_many_short_sequences_with_new_lengths_in_place_of_the_old(b):
    lens, keep = [90 + i % 20 for i in range(60)], 30
    for alias in (True, False):
        pool = Pool(b, 32, 16, 16, lens, seed=51, more=[keep] * len(lens))
        check_evict(b, pool, lens, keep, 3, 4, alias=alias)


def test_evict_from_blocks_that_sequences_share(b):
    """A common beginning is read by both and left as it is."""
    lens, keep = [64, 64], 20
    pool = Pool(b, 1, 32, 16, lens, seed=25, more=[keep] * 2)
    pool.tables[1][:2] = pool.tables[0][:2]
    pool.desc = pool.describe(b, pool.tables)
    check_evict(b, pool, lens, keep, 1, 4)


@pytest.mark.parametrize("n,keep", [(30000, 4000), (230000, 1000), (230000, 150001)])
def test_evict_long_sequences(b, n, keep):
    """Several CTAs to a pair; beyond 8 x 24576 places keys are read again in every count."""
    pool = Pool(b, 1, 16, 128, [n], seed=26, more=[keep])
    pool.w = np.exp(np.random.default_rng(27).normal(size=pool.w.shape) * 3).astype(np.float32)
    pool.w[np.random.default_rng(28).random(pool.w.shape) < 0.5] = 0.25
    pool.upload()
    check_evict(b, pool, [n], keep, 3, 100)


def test_evict_many_sequences_on_few_sms(b):
    lens = [int(x) for x in np.random.default_rng(29).integers(0, 200, size=120)]
    pool = Pool(b, 2, 16, 16, lens, seed=30, more=[min(n, 50) for n in lens])
    stream = torch.cuda.Stream()
    b.templora_set_stream_sm_limit(stream, 3)
    try:
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            check_evict(b, pool, lens, 50, 4, 10, stream=stream)
    finally:
        b.templora_set_stream_sm_limit(stream, 0)


def test_evict_extreme_scales(b):
    """Blocks whose scales are the largest and the smallest there are; tokens of zeros and NaN alone from a block of a huge scale."""
    pool = Pool(b, 1, 16, 16, [64], seed=31, more=[20])
    t = pool.tables[0]
    for kv in range(2):
        pool.scales[kv][t[0]], pool.scales[kv][t[1]], pool.scales[kv][t[2]], pool.scales[kv][t[3]] = 2.0 ** 119, 2.0 ** -126, 2.0 ** 100, 1.0
        pool.codes[kv][t[2]] = np.where(np.arange(16)[None, None] % 2 == 0, 0x80, 0x7f)
        pool.codes[kv][t[1], :, 3:] = 1
    for hot in ([0, 1], [2], [1], [1, 2], [0, 3]):
        pool.w[t] = 0.0
        for i in hot:
            pool.w[t[i]] = 1.0
        pool.upload()
        check_evict(b, pool, [64], 20)


@pytest.mark.parametrize("keep", [30, 150])
def test_evict_scales_of_any_value(b, keep):
    """Scales that are no powers of two, as of a cache that another program has filled: negative, zero, subnormal ones too.  Codes are
    rounded once; what a scale that is not finite stands for is NaN and asks for no scale."""
    lens = [300, 33, 260]
    pool = Pool(b, 2, 64, 16, lens, seed=33, more=[min(n, keep) for n in lens], spread=4)
    g = np.random.default_rng(34)
    shape = pool.scales.shape
    pool.scales *= (1 + g.random(shape)).astype(np.float32) * np.where(g.random(shape) < 0.3, -1, 1).astype(np.float32)
    for odd in (0.0, -0.0, 1e-42, -3e-39, np.nan, np.inf, -np.inf):
        pool.scales[g.random(shape) < 0.02] = odd
    pool.scales[g.random(shape) < 0.03] = np.float32(1.7 * 2.0 ** 118)
    pool.codes[g.random(pool.codes.shape) < 0.02] = 0x7f
    pool.upload()
    with np.errstate(invalid="ignore"):
        check_evict(b, pool, lens, keep, 2, 5)


def test_evict_codes_are_rounded_once(b):
    """Scales that bring codes next to the middle between two others: rounded to fp32 on the way, some would end up on the other side."""
    odd = [(np.float32(m / c), c) for c in (9, 11, 13, 15) for m in range(17, 32, 2)]
    values = orc.e4m3_decode(np.arange(127))
    twice = sum((orc.e4m3_encode((values * float(s)).astype(np.float32)) != orc.e4m3_encode(values * float(s))).sum() for s, _ in odd)
    assert twice > 20
    n = 16 * len(odd)
    pool = Pool(b, 1, 128, 16, [n], seed=35, more=[n - 8], spread=0)
    for blk, (s, _) in zip(pool.tables[0], odd):
        for kv in range(2):
            pool.scales[kv][blk] = s
            pool.codes[kv][blk] = np.arange(16 * 128).reshape(16, 128) % 127
    pool.upload()
    check_evict(b, pool, [n], n - 8, 2, 5)


def test_evict_bad_lengths_and_tables_leave_the_sequence_out(b):
    lens, keep = [40, 60, 33, 20, 50, 60], 32
    pool = Pool(b, 2, 32, 16, lens, seed=32, more=[min(n, keep) for n in lens])
    src, dst = pool.desc._keep[4], pool.to._keep[4]
    src[1, 3] = -1
    dst[4, 1] = pool.blocks
    given = [40, 60, -7, 16 * src.shape[1] + 1, 50, 60]
    out = [x.copy() for x in (pool.codes[0], pool.scales[0], pool.codes[1], pool.scales[1], pool.w)]
    new = torch.full((6,), -1, dtype=torch.int32, device="cuda")
    kept = torch.full((6, 2, keep), -9, dtype=torch.int32, device="cuda")
    ws = pool.guard.workspace(b.templora_kv_cache_evict_workspace_bytes(pool.desc, keep))
    b.templora_kv_cache_evict(b.KvCacheEvictArgs(pool.desc, pool.weights, i32(given), pool.to, pool.weights, new, keep, 1, 2, kept), ws)
    torch.cuda.synchronize()
    pool.guard.check()
    assert b.templora_read_device_status(ws)[0] == b.ERR_INVALID_ARG
    assert new.cpu().tolist() == [32, 0, 0, 0, 0, 32]
    for s in (0, 5):
        orc.kv_evict(pool.codes[0], pool.scales[0].astype(np.float64), pool.codes[1], pool.scales[1].astype(np.float64), pool.w, pool.tables[s], lens[s],
                     out, pool.to_tables[s], keep, 1, 2)
    pool.same(*out)
    assert (kept[[1, 2, 3, 4]] == -9).all()


# ------------------------------------------------------------------ sampling
def check_sample(b, x, u, temperature=None, top_k=None, top_p=None, min_p=None, stride=0, logprobs=True, stream=None, at=0):
    """x: logits [rows, vocab]; settings: a number for all rows, a list, or None."""
    rows, vocab = x.shape
    guard = Guarded()
    pitch = vocab + stride
    buf = guard.empty((at + rows * pitch,), x.dtype, float("nan"))
    logits = buf[at:].as_strided((rows, vocab), (pitch, 1))
    logits.copy_(x)
    tokens, lp = guard.empty((rows,), torch.int32, -77), guard.empty((rows,), torch.float32, float("nan"))
    spread = lambda v, dt: None if v is None else torch.tensor(v if isinstance(v, list) else [v] * rows, dtype=dt, device="cuda")  # noqa: E731
    u = spread(u, torch.float32)
    dev = dict(temperature=spread(temperature, torch.float32), top_k=spread(top_k, torch.int32), top_p=spread(top_p, torch.float32),
               min_p=spread(min_p, torch.float32))
    args = b.SampleArgs(logits, u, tokens, logprobs=lp if logprobs else None, **dev)
    b.templora_sample(args, stream=stream)
    torch.cuda.synchronize()
    guard.check()
    host = {k: None if v is None else v.cpu().numpy() for k, v in dev.items()}
    got, got_lp, us = tokens.cpu().numpy(), f(lp), u.cpu().numpy()
    for i in range(rows):
        kw = {k: v[i] if k == "top_k" else float(v[i]) for k, v in host.items() if v is not None}
        want, want_lp = orc.sample(f(x[i]), float(us[i]), **kw)
        assert got[i] == want, (i, got[i], want, kw, us[i])
        if logprobs:
            assert got_lp[i] == want_lp or abs(got_lp[i] - want_lp) <= 2.0 ** -24 * abs(want_lp) + 1e-9, (i, got_lp[i], want_lp)
    return got


def logits(seed, rows, vocab, dtype="f32", spread=3.0):
    return (torch.randn((rows, vocab), generator=torch.Generator().manual_seed(seed)) * spread).to(DT[dtype])


US = [0.0, 1e-7, 0.1, 0.25, 0.5, 0.75, 0.9, 0.99999, 1.0 - 2.0 ** -24]
SETTINGS = [
    {}, dict(temperature=0.0), dict(temperature=0.3), dict(temperature=2.5), dict(top_k=1), dict(top_k=2), dict(top_k=40), dict(top_p=0.9),
    dict(top_p=0.05), dict(top_p=0.9999), dict(min_p=0.05), dict(min_p=1.0), dict(temperature=0.7, top_k=50, top_p=0.9),
    dict(temperature=1.3, top_k=500, top_p=0.97, min_p=0.01), dict(top_k=3000, top_p=0.5),
]


@pytest.mark.parametrize("kw", SETTINGS, ids=lambda kw: "-".join(f"{k}{v}" for k, v in kw.items()) or "plain")
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 37, 1000, 4099])
def test_sample_matches_oracle(b, kw, dtype, vocab):
    check_sample(b, logits(vocab, len(US), vocab, dtype), US, stride=3, **kw)


@pytest.mark.parametrize("rows,vocab,dtype", [(1, 32000, "bf16"), (3, 32003, "f32"), (40, 50021, "bf16"), (2, 128251, "f32"), (1, 262144, "f32"),
                                              (300, 300, "f32"), (170, 9001, "bf16")])
def test_sample_sizes(b, rows, vocab, dtype):
    """Rows and vocabularies that take one to eight CTAs to a row."""
    g = np.random.default_rng(vocab)
    pick = lambda v: [v[int(i)] for i in g.integers(0, len(v), size=rows)]  # noqa: E731
    check_sample(b, logits(1, rows, vocab, dtype, 2.0), [float(x) for x in g.random(rows)], temperature=pick([0.0, 0.6, 1.0, 1.4]),
                 top_k=pick([0, 1, 50, 700, vocab]), top_p=pick([1.0, 0.95, 0.6, 0.2]), min_p=pick([0.0, 0.0, 0.02, 0.3]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(2, 262144), (3, 262143), (2, 139265), (2, 139264)])
def test_sample_of_the_largest_vocabularies(b, dtype, rows, vocab):
    """On both sides of the size at which fp32 rows take all of an SM; bf16 rows never do."""
    x = logits(9, rows, vocab, dtype, 2.0)
    for kw in ({}, dict(temperature=0.0), dict(top_k=50, top_p=0.9), dict(top_k=3000), dict(top_p=0.95), dict(min_p=0.01)):
        check_sample(b, x, [0.07, 0.6, 0.99][:rows], **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample_ties(b, dtype):
    """Equal logits: the lower tokens first, whether one bin, several CTAs or all of a row hold them."""
    for vocab in (64, 5000, 33000):
        x = torch.zeros((9, vocab)).to(DT[dtype])
        for kw in ({}, dict(top_k=5), dict(top_k=vocab - 1), dict(top_p=0.5), dict(top_k=vocab // 2, top_p=0.25), dict(min_p=1.0)):
            check_sample(b, x, US, **kw)
        x = torch.round(logits(2, 9, vocab) * 0.7).to(DT[dtype])          # a dozen values
        for kw in ({}, dict(top_k=7), dict(top_k=vocab // 3), dict(top_p=0.8), dict(top_k=vocab // 3, top_p=0.6, min_p=0.1)):
            check_sample(b, x, US, **kw)


def test_sample_values_close_together_and_far_apart(b):
    """Borders inside a bin that holds many different values, and logits that span the whole range of fp32."""
    g = torch.Generator().manual_seed(3)
    x = 20.0 + torch.randint(0, 4000, (9, 8000), generator=g) * 2.0 ** -18           # all within a 64th
    x[:, 17] = -1e30
    for kw in (dict(top_k=3000), dict(top_p=0.37), dict(top_k=2999, top_p=0.77), dict(temperature=1e-3, top_p=0.9), dict(temperature=1e30, top_p=0.4)):
        check_sample(b, x, US, **kw)
    x = torch.sign(logits(4, 9, 3000)) * torch.exp(logits(5, 9, 3000, spread=25.0)).clamp(max=3e38)
    for kw in ({}, dict(top_k=100), dict(top_k=2500), dict(top_p=0.5), dict(temperature=1e38, top_p=0.9), dict(temperature=1e-38),
               dict(temperature=1e-45, top_p=0.5), dict(temperature=float("inf"), top_p=0.3)):
        check_sample(b, x, US, **kw)


def test_sample_masked_and_infinite_rows(b):
    inf, nan = float("inf"), float("nan")
    for dtype in ("f32", "bf16"):
        x = logits(6, 9, 700, dtype)
        x[0] = -inf
        x[1] = nan
        x[2, :699] = -inf
        x[3, ::2], x[3, 1::4] = -inf, nan
        x[4, 5], x[4, 600], x[4, 7] = inf, inf, nan
        x[5] = inf
        x[6] = torch.finfo(DT[dtype]).min                                    # a mask of the type's lowest value, one token left
        x[6, 300] = 1.0
        x[7] = torch.finfo(DT[dtype]).min
        x[8, 3], x[8, 9] = 0.0, -0.0
        x[8, 10:] = -1.0
        for kw in ({}, dict(top_k=2), dict(top_k=600), dict(top_p=0.5), dict(min_p=0.5), dict(temperature=0.0), dict(top_k=3, top_p=0.9, min_p=0.2)):
            for u in (0.0, 0.6, 0.999):
                check_sample(b, x, u, **kw)


def test_sample_settings_out_of_range(b):
    nan, inf = float("nan"), float("inf")
    x = logits(7, 12, 500)
    check_sample(b, x, [nan, -3.0, 1.0, 7.0, inf, -inf, 0.3, 0.3, 0.3, 0.3, 0.3, 0.3],
                 temperature=[1.0, 1.0, 1.0, 1.0, 1.0, 1.0, nan, -1.0, -inf, inf, 1e-45, 1.0],
                 top_k=[0, -5, 501, 500, 2 ** 31 - 1, -2 ** 31, 3, 3, 3, 3, 3, 3],
                 top_p=[nan, -1.0, 2.0, inf, -inf, 0.0, 0.5, 0.5, 0.5, 0.5, 0.5, 1e-40],
                 min_p=[nan, -1.0, 2.0, inf, -inf, 0.0, 0.1, 0.1, 0.1, 0.1, 0.1, 1e-40])
    check_sample(b, x, 0.4, logprobs=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample_rows_anywhere(b, dtype):
    """Rows that begin at every place within 16 bytes, also the first."""
    for vocab in (5, 1003):
        for at in range(9):
            check_sample(b, logits(at, 9, vocab, dtype), US, stride=at % 4, at=at, top_k=20, top_p=0.9)


def test_sample_on_partitioned_sms_and_few_sms(b):
    x, wide = logits(8, 2, 32000), logits(8, 2, 140001)
    stream = torch.cuda.Stream()
    b.templora_set_stream_sm_limit(stream, 1)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        check_sample(b, x, 0.7, top_k=50, top_p=0.9, stream=stream)
    b.templora_set_stream_sm_limit(stream, 0)
    try:
        part = b.templora_sm_partition_create(32)
    except b.TemploraError as e:
        assert e.code == b.ERR_UNSUPPORTED
        return
    try:
        for s in (part.stream_first, part.stream_rest):
            stream = torch.cuda.ExternalStream(s)
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                check_sample(b, x, 0.7, top_k=50, top_p=0.9, stream=stream)
                check_sample(b, wide, 0.7, top_p=0.95, stream=stream)
                for n in (30000, 100000):
                    pool = Pool(b, 1, 16, 128, [n], seed=33, more=[500])
                    torch.cuda.synchronize()
                    check_evict(b, pool, [n], 500, 3, 100, stream=stream)
    finally:
        torch.cuda.synchronize()
        b.templora_sm_partition_destroy(part)


def test_weigh_on_partitioned_sms_and_few_sms(b):
    lens, counts, H, heads, dim = [300, 41], [260, 9], 8, 1, 64
    stream = torch.cuda.Stream()
    b.templora_set_stream_sm_limit(stream, 3)
    for dtype in ("bf16", "f32"):
        pool = Pool(b, heads, dim, 32, lens, seed=61)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            check_weigh(b, pool, dtype, H, lens, counts, stream=stream)
    b.templora_set_stream_sm_limit(stream, 0)
    try:
        part = b.templora_sm_partition_create(32)
    except b.TemploraError as e:
        assert e.code == b.ERR_UNSUPPORTED
        return
    try:
        for s in (part.stream_first, part.stream_rest):
            stream = torch.cuda.ExternalStream(s)
            for dtype in ("bf16", "f32"):
                for n in ([260, 9], [12, 3]):
                    pool = Pool(b, heads, dim, 32, lens, seed=62)
                    torch.cuda.synchronize()
                    with torch.cuda.stream(stream):
                        check_weigh(b, pool, dtype, H, lens, n, stream=stream)
    finally:
        torch.cuda.synchronize()
        b.templora_sm_partition_destroy(part)


# ------------------------------------------------------------------ recorded calls, large caches
def test_evict_and_chunk_weights_recorded_and_replayed(b):
    """Lengths, rows, weights and queries change between replays; two graphs have workspaces of their own."""
    lens, counts, H, heads, dim, bt, keep = [150, 64], [64, 20], 4, 2, 64, 16, 40
    pool = Pool(b, heads, dim, bt, [200, 120], seed=50, more=[keep] * 2)
    scale = float(np.float32(dim ** -0.5))
    attn = b.attention_desc(H, heads, dim, b.BF16, scale=scale)
    q = torch.zeros((84, H, dim), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((84, H), device="cuda")
    lens_d, offsets, new = i32(lens), i32([0, 64, 84]), i32([0, 0])
    kept = torch.full((2, heads, keep), -9, dtype=torch.int32, device="cuda")
    graphs = []
    weigh = b.KvCacheWeighArgs(attn, pool.desc, lens_d, q, lse, pool.weights, row_offsets=offsets)
    evict = b.KvCacheEvictArgs(pool.desc, pool.weights, lens_d, pool.to, pool.weights, new, keep, 2, 8, kept)
    for args, call, size in ((weigh, b.templora_kv_cache_weigh, b.templora_kv_cache_weigh_workspace_bytes(attn, pool.desc, 84)),
                             (evict, b.templora_kv_cache_evict, b.templora_kv_cache_evict_workspace_bytes(pool.desc, keep))):
        ws = pool.guard.workspace(size)
        call(args, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(args, ws)
        graphs.append((graph, ws))
    for step, (now, rows) in enumerate((([150, 64], [64, 20]), ([200, 120], [1, 83]), ([41, 7], [41, 7]))):
        g = np.random.default_rng(60 + step)
        pool.w = (g.random(pool.w.shape) * 4).astype(np.float32)
        pool.upload()
        kept.fill_(-9)
        lens_d.copy_(i32(now)), offsets.copy_(i32([0, rows[0], sum(rows)]))
        host_q = torch.zeros((84, H, dim))
        host_q[:sum(rows)] = torch.randn((sum(rows), H, dim), generator=torch.Generator().manual_seed(step)) * 0.5
        q.copy_(host_q)
        host_lse = softmax_rows(pool, q[:sum(rows)], now, rows, H, scale).astype(np.float32)
        lse[:sum(rows)].copy_(torch.from_numpy(host_lse))
        graphs[0][0].replay()
        torch.cuda.synchronize()
        want, slack = weigh_reference(pool, q[:sum(rows)], host_lse.astype(np.float64), now, rows, scale)
        assert (np.abs(f(pool.weights) - want) <= slack).all()
        pool.w = pool.weights.cpu().numpy()
        out = [x.copy() for x in (pool.codes[0], pool.scales[0], pool.codes[1], pool.scales[1], pool.w)]
        graphs[1][0].replay()
        torch.cuda.synchronize()
        for s, m in enumerate(now):
            places = orc.kv_evict(pool.codes[0], pool.scales[0].astype(np.float64), pool.codes[1], pool.scales[1].astype(np.float64), pool.w, pool.tables[s], m,
                                  out, pool.to_tables[s], keep, 2, 8)
            assert [kept[s, h, :len(p)].cpu().tolist() for h, p in enumerate(places)] == places
        pool.same(*out)
        assert new.cpu().tolist() == [min(m, keep) for m in now]
        assert all(b.templora_read_device_status(ws)[0] == 0 for _, ws in graphs)
    pool.guard.check()


def test_two_chunks_weighed_at_once_on_two_streams(b):
    """Both want tensor memory; each has a workspace of its own."""
    lens, H, heads, dim = [600], 8, 2, 128
    pools = [Pool(b, heads, dim, 64, lens, seed=70 + i) for i in range(2)]
    scale = float(np.float32(dim ** -0.5))
    attn = b.attention_desc(H, heads, dim, b.BF16, scale=scale)
    q = (torch.randn((300, H, dim), generator=torch.Generator().manual_seed(71)) * 0.5).to(torch.bfloat16)
    streams = [torch.cuda.Stream() for _ in range(2)]
    sides = []
    for pool in pools:
        lse = softmax_rows(pool, q, lens, [300], H, scale).astype(np.float32)
        args = b.KvCacheWeighArgs(attn, pool.desc, i32(lens), q.cuda(), torch.from_numpy(lse).cuda(), pool.weights, row_offsets=i32([0, 300]))
        sides.append((args, pool.guard.workspace(b.templora_kv_cache_weigh_workspace_bytes(attn, pool.desc, 300)), lse))
    torch.cuda.synchronize()
    for _ in range(4):
        for (args, ws, _), stream in zip(sides, streams):
            b.templora_kv_cache_weigh(args, ws, stream=stream)
    torch.cuda.synchronize()
    for pool, (_, ws, lse) in zip(pools, sides):
        pool.guard.check()
        assert b.templora_read_device_status(ws)[0] == 0
        for _ in range(4):
            want, slack = weigh_reference(pool, q, lse.astype(np.float64), lens, [300], scale)
            pool.w = want.astype(np.float32)
        assert (np.abs(f(pool.weights) - want) <= 4 * slack).all()


@pytest.mark.parametrize("rows", [1, 40])
def test_weigh_and_evict_beyond_4_gb(b, rows):
    """Blocks at the end of a pool whose codes take more than 2^32 bytes each, and weights more than 2^31."""
    heads, dim, bt, n, H, keep = 2, 128, 128, 140000, 4, 100
    k, v = (torch.zeros((n, heads, bt, dim), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.ones((n, heads), device="cuda") for _ in range(2))
    w = torch.zeros((n, heads, bt), device="cuda")
    small = Pool(b, heads, dim, bt, [150, 256], seed=80, more=[keep] * 2, spare=0)
    at = [n - 1, 5, 131072, n - 2, n - 3, 139000]                       # where the small pool's blocks lie in the large one
    for big, x in ((k, small.codes[0]), (v, small.codes[1]), (ks, small.scales[0]), (vs, small.scales[1]), (w, small.w)):
        big[at] = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    table = lambda ts: i32([[at[x] for x in t] + [-1] * (2 - len(t)) for t in ts])  # noqa: E731
    cache, to = (b.kv_cache_desc(k, v, ks, vs, table(t)) for t in (small.tables, small.to_tables))
    scale = float(np.float32(dim ** -0.5))
    attn = b.attention_desc(H, heads, dim, b.BF16, scale=scale)
    lens, counts = [150, 256], [rows] * 2
    q = (torch.randn((2 * rows, H, dim), generator=torch.Generator().manual_seed(81)) * 0.5).to(torch.bfloat16)
    lse = softmax_rows(small, q, lens, counts, H, scale).astype(np.float32)
    ws = b.alloc_workspace(b.templora_kv_cache_weigh_workspace_bytes(attn, cache, 2 * rows))
    b.templora_kv_cache_weigh(b.KvCacheWeighArgs(attn, cache, i32(lens), q.cuda(), torch.from_numpy(lse).cuda(), w,
                                                 row_offsets=None if rows == 1 else i32([0, rows, 2 * rows])), ws)
    torch.cuda.synchronize()
    want, slack = weigh_reference(small, q, lse.astype(np.float64), lens, counts, scale)
    assert (np.abs(f(w[at]) - want) <= slack).all() and int((w != 0).sum()) == int((w[at] != 0).sum())
    small.w = w[at].cpu().numpy()
    out = [x.copy() for x in (small.codes[0], small.scales[0], small.codes[1], small.scales[1], small.w)]
    new = i32([0, 0])
    ws = b.alloc_workspace(b.templora_kv_cache_evict_workspace_bytes(cache, keep))
    b.templora_kv_cache_evict(b.KvCacheEvictArgs(cache, w, i32(lens), to, w, new, keep, 3, 20), ws)
    torch.cuda.synchronize()
    for s, m in enumerate(lens):
        orc.kv_evict(small.codes[0], small.scales[0].astype(np.float64), small.codes[1], small.scales[1].astype(np.float64), small.w, small.tables[s], m, out,
                     small.to_tables[s], keep, 3, 20)
    for big, ref in zip((k, ks, v, vs, w), out):
        assert np.array_equal(big[at].cpu().numpy(), np.asarray(ref).astype(big[:1].cpu().numpy().dtype))
    assert new.cpu().tolist() == [keep, keep]


# ------------------------------------------------------------------ the ends of what the calls take
@pytest.mark.parametrize("dtype,H,counts", [("bf16", 4, False), ("bf16", 20, False), ("f32", 4, False), ("f32", 12, False), ("bf16", 8, True), ("f32", 2, True)])
def test_weigh_of_the_most_sequences(b, dtype, H, counts):
    g = np.random.default_rng(90)
    lens = [int(x) for x in g.integers(0, 21, size=4096)]
    rows = [int(x) for x in g.integers(0, 12, size=4096)] if counts else None      # some more than the sequence has tokens
    check_weigh(b, Pool(b, 1, 16, 16, lens, seed=91), dtype, H, lens, rows)


def test_weigh_without_rows_changes_nothing(b):
    for dtype in ("bf16", "f32"):
        pool = Pool(b, 2, 64, 16, [90, 40], seed=92)
        q = torch.zeros((200, 4, 64), dtype=DT[dtype])
        check_weigh(b, pool, dtype, 4, [90, 40], [0, 0], q=q, lse=np.zeros((200, 4)), offsets=[7, 7, 7])
        check_weigh(b, pool, dtype, 4, [0, 0], None)


@pytest.mark.parametrize("counts", [None, [3, 3], [60, 33]])
def test_weigh_under_the_largest_window(b, counts):
    pool = Pool(b, 2, 64, 16, [90, 40], seed=93)
    check_weigh(b, pool, "bf16", 4, [90, 40], counts, window=2 ** 31 - 1)


@pytest.mark.parametrize("alias", [False, True])
def test_evict_of_the_most_sequences(b, alias):
    lens = [int(x) for x in np.random.default_rng(94).integers(0, 40, size=4096)]
    check_evict(b, Pool(b, 1, 16, 16, lens, seed=95, more=[min(n, 17) for n in lens]), lens, 17, 2, 3, alias=alias)


@pytest.mark.parametrize("n", [150, 5000])
def test_evict_that_keeps_all(b, n):
    """Sequences within the budget are moved whole; a budget of the table's very size."""
    lens = [n, 0, n // 3]
    pool = Pool(b, 2, 32, 32, lens, seed=96, more=lens)
    check_evict(b, pool, lens, n, n // 2, n - n // 2)
    pool.upload()
    check_evict(b, pool, lens, pool.to._keep[4].shape[1] * 32)


def test_evict_by_choice_and_move_recorded_and_replayed(b):
    """As two launches, on clusters; lengths and weights change between replays, new lengths in a buffer of their own and in place."""
    heads, dim, bt, keep, n = 2, 32, 64, 700, [9000, 4000]
    for alias in (False, True):
        pool = Pool(b, heads, dim, bt, n, seed=97, more=[keep] * 2)
        lens = i32(n)
        new = lens if alias else i32([0, 0])
        ws = pool.guard.workspace(b.templora_kv_cache_evict_workspace_bytes(pool.desc, keep))
        args = b.KvCacheEvictArgs(pool.desc, pool.weights, lens, pool.to, pool.weights, new, keep, 3, 50)
        b.templora_kv_cache_evict(args, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.templora_kv_cache_evict(args, ws)
        for step, now in enumerate((n, [701, 8], [8999, 0])):
            pool.w = (np.random.default_rng(98 + step).random(pool.w.shape) * 4).astype(np.float32)
            pool.upload()
            lens.copy_(i32(now))
            out = [x.copy() for x in (pool.codes[0], pool.scales[0], pool.codes[1], pool.scales[1], pool.w)]
            graph.replay()
            torch.cuda.synchronize()
            for s, m in enumerate(now):
                orc.kv_evict(pool.codes[0], pool.scales[0].astype(np.float64), pool.codes[1], pool.scales[1].astype(np.float64), pool.w, pool.tables[s], m, out,
                             pool.to_tables[s], keep, 3, 50)
            pool.same(*out)
            assert new.cpu().tolist() == [min(m, keep) for m in now]
            assert b.templora_read_device_status(ws)[0] == 0
        pool.guard.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample_of_many_rows(b, dtype):
    rows = 70000
    x = logits(10, rows, 9, dtype)
    u = torch.rand(rows, generator=torch.Generator().manual_seed(11))
    tokens, lp = torch.full((rows,), -7, dtype=torch.int32, device="cuda"), torch.zeros(rows, device="cuda")
    at = torch.arange(rows)
    k, p = (at % 5).int(), torch.tensor([1.0, 0.7, 0.3])[at % 3]
    b.templora_sample(b.SampleArgs(x.cuda(), u.cuda(), tokens, top_k=k.cuda(), top_p=p.cuda(), logprobs=lp))
    torch.cuda.synchronize()
    got, got_lp = tokens.cpu().numpy(), f(lp)
    for i in list(range(0, rows, 97)) + [65535, 65536, rows - 1]:
        want, want_lp = orc.sample(f(x[i]), float(u[i]), 1.0, int(k[i]), float(p[i]))
        assert got[i] == want and abs(got_lp[i] - want_lp) <= 2.0 ** -24 * abs(want_lp) + 1e-9, (i, got[i], want)
    assert ((got >= 0) & (got < 9)).all()


# ------------------------------------------------------------------ together
def test_generation_over_a_bounded_cache(b):
    """A prompt's keys and values and the weights its rows give, then steps of append, decode, weigh and sample recorded into a
    graph and replayed while the lengths grow; whenever the cache is a block over its budget it is cut down into fresh blocks.
    Every call's inputs and outputs are compared with the oracle's."""
    n, H, heads, dim, bt, vocab, budget = 2, 4, 2, 64, 16, 1000, 48
    prompt, steps = [40, 29], 28
    scale = float(np.float32(dim ** -0.5))
    g = torch.Generator(device="cuda").manual_seed(1)
    pool = Pool(b, heads, dim, bt, [budget + bt] * n, seed=40, more=[budget + bt] * n, spread=0)
    pool.w[:] = np.nan
    pool.upload()
    width = (budget + 2 * bt - 1) // bt
    table = pool.desc._keep[4]                       # the cache's table, in place; the second half's blocks take turns
    spare = [list(t) for t in pool.to_tables]
    held = [list(t) for t in pool.tables]
    table[:, width:] = -5
    attn = b.attention_desc(H, heads, dim, b.BF16, scale=scale)
    ws = [pool.guard.workspace(x) for x in (b.templora_kv_cache_append_workspace_bytes(pool.desc), b.templora_attention_decode_workspace_bytes(attn, pool.desc),
                                            b.templora_kv_cache_weigh_workspace_bytes(attn, pool.desc, n), b.templora_kv_cache_evict_workspace_bytes(pool.desc, budget))]
    bf = lambda *s: (torch.randn(s, generator=g, device="cuda")).to(torch.bfloat16)  # noqa: E731
    # the prompt
    rows = sum(prompt)
    q, k, v = bf(rows, H, dim), bf(rows, heads, dim), bf(rows, heads, dim)
    off = i32([0, prompt[0], rows])
    b.templora_kv_cache_append(b.KvCacheAppendArgs(pool.desc, i32([0] * n), k, v, new_offsets=off), ws[0])
    o, lse = torch.empty_like(q), torch.empty((H, rows), device="cuda")
    chunk = b.attention_desc(H, heads, dim, b.BF16, scale=scale, doc_offsets=off)
    wa = b.alloc_workspace(b.templora_attention_workspace_bytes(chunk, rows, rows))
    b.templora_attention_fwd(b.AttentionArgs(chunk, q, k, v, o, lse), wa)
    lens = i32(prompt)
    b.templora_kv_cache_weigh(b.KvCacheWeighArgs(attn, pool.desc, lens, q, lse.T, pool.weights, row_offsets=off), ws[2])
    torch.cuda.synchronize()

    def snapshot():
        pool.codes = np.stack([pool.k.cpu().numpy(), pool.v.cpu().numpy()])
        pool.scales = np.stack([pool.ks.cpu().numpy(), pool.vs.cpu().numpy()])
        pool.w = pool.weights.cpu().numpy()

    before = pool.w.copy()
    snapshot()
    pool.tables, seen, pool.w = held, pool.w, before
    want, slack = weigh_reference(pool, q, f(lse).T, prompt, prompt, scale)
    fine = np.isfinite(want)
    assert np.isfinite(seen).sum() == fine.sum() == heads * rows and (np.abs(seen - want)[fine] <= slack[fine]).all()

    # a step
    q1, k1, v1, o1 = (torch.zeros((n, m, dim), dtype=torch.bfloat16, device="cuda") for m in (H, heads, heads, H))
    lse1, u = torch.zeros((n, H), device="cuda"), torch.zeros(n, device="cuda")
    lin = b.linear_desc(bf(vocab, H * dim) * 0.3, bf(8, H * dim) * 0.1, bf(vocab, 8) * 0.1, 1.0)
    wl = b.alloc_workspace(b.templora_workspace_bytes(lin, 16))
    scores = torch.zeros((n, vocab), dtype=torch.bfloat16, device="cuda")
    tokens, logprobs = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
    one = lambda x, dt=torch.float32: torch.full((n,), x, dtype=dt, device="cuda")  # noqa: E731
    after = lens + 1
    calls = [lambda: b.templora_kv_cache_append(put, ws[0]), lambda: b.templora_attention_decode_fwd(get, ws[1]), lambda: b.templora_kv_cache_weigh(weigh, ws[2]),
             lambda: b.templora_decode_fwd(lin, o1.view(n, -1), scores, wl), lambda: b.templora_sample(draw)]
    put, get = b.KvCacheAppendArgs(pool.desc, lens, k1, v1), b.AttentionDecodeArgs(attn, pool.desc, after, q1, o1, lse1)
    weigh = b.KvCacheWeighArgs(attn, pool.desc, after, q1, lse1, pool.weights)
    draw = b.SampleArgs(scores, u, tokens, temperature=one(0.8), top_k=one(60, torch.int32), top_p=one(0.9), min_p=one(0.02), logprobs=logprobs)
    state = [t.clone() for t in (pool.k, pool.v, pool.ks, pool.vs, pool.weights)]
    for c in calls:                                  # one call of each kind outside a capture, undone
        c()
    for t, was in zip((pool.k, pool.v, pool.ks, pool.vs, pool.weights), state):
        t.copy_(was)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for c in calls:
            c()
        lens.add_(1), after.add_(1)
    now = list(prompt)
    evictions = 0
    for t in range(steps):
        for x in (q1, k1, v1):
            x.copy_(bf(*x.shape))
        u.copy_(torch.rand(n, generator=g, device="cuda"))
        before = pool.weights.cpu().numpy()
        graph.replay()
        torch.cuda.synchronize()
        now = [m + 1 for m in now]
        snapshot()
        seen, pool.w = pool.w, before
        want, slack = weigh_reference(pool, q1, f(lse1), now, [1] * n, scale)
        fine = np.isfinite(want)
        assert (np.isfinite(seen) == fine).all() and (np.abs(seen - want)[fine] <= slack[fine]).all()
        for s in range(n):
            kk, vv = (orc.kv_read(pool.codes[i], pool.scales[i].astype(np.float64), held[s], now[s]) for i in range(2))
            ref, ref_lse = orc.attention_decode(f(q1)[s], kk, vv, scale)
            assert np.abs(f(o1)[s] - ref).max() <= 2.0 ** -7 * np.abs(vv).max() and np.abs(f(lse1)[s] - ref_lse).max() <= 1e-4
            token, lp = orc.sample(f(scores)[s], float(u[s]), float(np.float32(0.8)), 60, float(np.float32(0.9)), float(np.float32(0.02)))
            assert int(tokens[s]) == token and abs(float(logprobs[s]) - lp) <= 1e-6
        if max(now) > budget:
            evictions += 1
            pool.w = seen
            out = [x.copy() for x in (pool.codes[0], pool.scales[0], pool.codes[1], pool.scales[1], pool.w)]
            to = pool.describe(b, spare, table.shape[1])
            b.templora_kv_cache_evict(b.KvCacheEvictArgs(pool.desc, pool.weights, lens, to, pool.weights, lens, budget - bt, 2, 8), ws[3])
            torch.cuda.synchronize()
            for s in range(n):
                orc.kv_evict(pool.codes[0], pool.scales[0].astype(np.float64), pool.codes[1], pool.scales[1].astype(np.float64), seen, held[s], now[s], out,
                             spare[s], budget - bt, 2, 8)
            pool.same(*out)
            now = [min(m, budget - bt) for m in now]
            assert lens.cpu().tolist() == now
            after.copy_(lens + 1)
            table.copy_(to._keep[4])                 # the graph reads the table in place
            held, spare = spare, held
            pool.tables = held
    assert evictions >= 2
    pool.guard.check()
    for w in (*ws, wl):
        assert b.templora_read_device_status(w)[0] == 0
