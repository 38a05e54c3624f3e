"""Pins of the oracle's attention and 8-bit cache functions, and the refusals of their entry points.  No GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import templora_oracle as orc

RNG = np.random.default_rng(7)


def _rand(*shape):
    return RNG.standard_normal(shape)


MASKS = [
    dict(causal=True),
    dict(causal=False),
    dict(causal=True, window=3),
    dict(causal=False, window=2),
    dict(causal=True, doc_offsets=[0, 4, 4, 9], prefix_lens=[2, 0, 3]),
    dict(causal=True, softcap=1.5, slopes=[0.25, 0.5, 0.125, 1.0]),
    dict(causal=True, q_start=2, prefix_lens=[5]),
]


@pytest.mark.parametrize("masks", MASKS)
def test_forward_is_the_definition_place_by_place(masks):
    Tq, Tk, H, Hkv, D, scale = 7, 9, 4, 2, 3, 0.6
    q, k, v = _rand(Tq, H, D), _rand(Tk, Hkv, D), _rand(Tk, Hkv, D)
    o, lse, _ = orc.attention_fwd(q, k, v, scale, **masks)
    off, pre = masks.get("doc_offsets"), masks.get("prefix_lens")
    for h in range(H):
        for i in range(Tq):
            p, w = masks.get("q_start", 0) + i, masks.get("window", 0)
            num, den = np.zeros(D), 0.0
            for j in range(Tk):
                same = off is None or any(a <= p < b and a <= j < b for a, b in zip(off, off[1:]))
                d = 0 if off is None else max(n for n in range(len(off) - 1) if off[n] <= p)
                in_prefix = pre is not None and j < (0 if off is None else off[d]) + pre[d]
                seen = same and (not masks["causal"] or j <= p or in_prefix) and (not w or abs(p - j) < w)
                if not seen:
                    continue
                s = scale * float(q[i, h] @ k[j, h // 2])
                if masks.get("softcap"):
                    s = masks["softcap"] * np.tanh(s / masks["softcap"])
                if masks.get("slopes"):
                    s -= masks["slopes"][h] * abs(p - j)
                num, den = num + np.exp(s) * v[j, h // 2], den + np.exp(s)
            want = num / den if den else num
            assert np.allclose(o[i, h], want, rtol=1e-12, atol=1e-13)
            assert lse[h, i] == -np.inf if den == 0 else abs(lse[h, i] - np.log(den)) < 1e-12


def test_special_cases_of_the_forward():
    q, k, v = _rand(5, 2, 4), _rand(5, 2, 4), _rand(5, 2, 4)
    o, lse, P = orc.attention_fwd(q, k, v, 0.5, causal=True)
    assert np.allclose(o[0], v[0]) and np.allclose(P.sum(-1), 1.0)            # the first row sees itself alone
    o, _, _ = orc.attention_fwd(q, np.zeros_like(k), v, 0.5, causal=False)
    assert np.allclose(o, v.mean(axis=0, keepdims=True))                       # equal scores: the mean
    o, lse, _ = orc.attention_fwd(q, k, v, 0.5, causal=True, doc_offsets=[0, 3])
    assert (o[3:] == 0).all() and np.isneginf(lse[:, 3:]).all()                # rows behind the last document
    a = orc.attention_fwd(q, k, v, 0.5, causal=True, softcap=1e9)[0]
    assert np.allclose(a, orc.attention_fwd(q, k, v, 0.5, causal=True)[0])     # a cap far away does nothing
    two = orc.attention_fwd(q, k, v, 0.5, causal=True, doc_offsets=[0, 2, 5])[0]
    parts = [orc.attention_fwd(q[a:b], k[a:b], v[a:b], 0.5, causal=True)[0] for a, b in ((0, 2), (2, 5))]
    assert np.allclose(two, np.concatenate(parts))                             # documents are calls of their own
    ref = torch.nn.functional.scaled_dot_product_attention(
        *(torch.from_numpy(x).transpose(0, 1) for x in (q, k, v)), is_causal=True, scale=0.5)
    assert np.allclose(orc.attention_fwd(q, k, v, 0.5, causal=True)[0], ref.transpose(0, 1).numpy())


@pytest.mark.parametrize("masks", MASKS)
def test_backward_against_central_differences(masks):
    Tq, Tk, H, Hkv, D, scale = 7, 9, 4, 2, 3, 0.6
    q, k, v, dO = _rand(Tq, H, D), _rand(Tk, Hkv, D), _rand(Tk, Hkv, D), _rand(Tq, H, D)
    o, _, _ = orc.attention_fwd(q, k, v, scale, **masks)
    grads = orc.attention_bwd(q, k, v, o, dO, scale, **masks)
    h = 1e-6
    for x, g in zip((q, k, v), grads):
        for at in [tuple(RNG.integers(0, n) for n in x.shape) for _ in range(12)]:
            keep = x[at]
            x[at] = keep + h
            up = (orc.attention_fwd(q, k, v, scale, **masks)[0] * dO).sum()
            x[at] = keep - h
            down = (orc.attention_fwd(q, k, v, scale, **masks)[0] * dO).sum()
            x[at] = keep
            assert abs((up - down) / (2 * h) - g[at]) < 1e-7 * (1 + abs(g[at]))


def test_e4m3_codes_against_torch():
    grid = orc.e4m3_values()
    assert grid[0] == 0 and grid[1] == 2.0 ** -9 and grid[-1] == 448.0
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(orc.e4m3_decode(codes), want.astype(np.float64), equal_nan=True)
    mids = (grid[1:] + grid[:-1]) / 2                                          # exact ties
    x = np.concatenate([grid, -grid, mids, -mids, mids * (1 + 1e-6), mids * (1 - 1e-6), RNG.uniform(-448, 448, 4096),
                        RNG.standard_normal(4096) * 0.01])
    want = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(orc.e4m3_encode(x.astype(np.float32)), want)
    assert list(orc.e4m3_encode([np.nan, np.inf, -np.inf, 1e9, -1e9])) == [0x7f, 0x7f, 0x7f, 0x7e, 0xfe]


def test_block_scale_and_append():
    for amax, e in ((448.0, 0), (448.0000001, 1), (1.75, -8), (1.7500001, -7), (0.0, -126), (3.3e38, 120)):
        assert orc.kv_block_scale(amax) == 2.0 ** e
    bt, D = 4, 2
    codes, scales = np.full((3, 1, bt, D), 0x7f, dtype=np.uint8), np.full((3, 1), np.nan)
    rows = np.array([[[1.0, 2.0]], [[3.0, 448.0]], [[0.5, 0.25]], [[900.0, 1.0]], [[7.0, 8.0]]])
    orc.kv_append(codes, scales, rows[:1], 0, [2, 0])
    assert scales[2, 0] == 2.0 ** -7
    orc.kv_append(codes, scales, rows[1:3], 1, [2, 0])                          # the block's scale rises to 1
    orc.kv_append(codes, scales, rows[3:], 3, [2, 0])                           # to 4, and a second block begins
    assert scales[2, 0] == 4.0 and scales[0, 0] == 2.0 ** -5
    got = orc.kv_read(codes, scales, [2, 0], 5)
    assert np.allclose(got, rows, rtol=2.0 ** -4, atol=4 * 2.0 ** -10)
    assert (codes[0, 0, 1:] == 0x7f).all() and (codes[1] == 0x7f).all()         # untouched places
    one = orc.attention_decode(np.ones((2, 2)), got, got, 0.1, window=1)[0]
    assert np.allclose(one, got[-1])                                            # a window of one: its own value


# ------------------------------------------------------------------ refusals (host side)
@pytest.fixture(scope="module")
def b():
    from paper_2401_11504_b200 import build
    build.build_library()
    from paper_2401_11504_b200 import binding
    return binding


P = 0x10000


def _desc(b, **kw):
    f = dict(n_heads=8, n_kv_heads=2, head_dim=64, dtype=b.BF16, scale=0.125, softcap=0.0, causal=1, window=0, slopes=None,
             n_docs=0, doc_offsets=None, prefix_lens=None)
    f.update(kw)
    return b.AttentionDesc(*f.values())


def _io(b, **kw):
    io = b.AttentionIo()
    for n in ("q", "k", "v", "o", "lse", "dO", "dq", "dk", "dv"):
        setattr(io, n, P)
    for n, v in kw.items():
        setattr(io, n, v)
    return io


def test_attention_refusals(b):
    lib, vp = b.lib, C.c_void_p

    def call(desc, io, Tq=16, Tk=16, start=0, ws=P, n=1 << 26, fn=lib.templora_attention_bwd):
        return fn(C.byref(desc), C.byref(io), Tq, Tk, start, vp(ws), n, None)

    I, U, W = b.ERR_INVALID_ARG, b.ERR_UNSUPPORTED, b.ERR_WORKSPACE
    for kw, want in ((dict(n_heads=0), I), (dict(n_kv_heads=3), I), (dict(head_dim=0), I), (dict(head_dim=129), U),
                     (dict(dtype=5), U), (dict(scale=float("nan")), I), (dict(scale=float("inf")), I),
                     (dict(softcap=-1.0), I), (dict(softcap=float("nan")), I), (dict(softcap=float("inf")), I),
                     (dict(window=-1), I), (dict(causal=2), I), (dict(n_docs=-1), I), (dict(n_docs=2), I),
                     (dict(causal=0, prefix_lens=P), I), (dict(window=4, prefix_lens=P), U), (dict(n_heads=65537 * 2), U)):
        assert call(_desc(b, **kw), _io(b)) == want, kw
        assert b.templora_attention_workspace_bytes(_desc(b, **kw), 16, 16) == 0, kw
    ok = _desc(b)
    for kw in (dict(q=None), dict(lse=None), dict(dO=None), dict(dv=None), dict(k=P + 8), dict(dq=P + 2), dict(ld_q=511),
               dict(ld_k=64), dict(ld_dv=-1)):
        assert call(ok, _io(b, **kw)) == I, kw
    assert call(ok, _io(b), Tq=0) == I and call(ok, _io(b), Tk=-3) == I and call(ok, _io(b), start=-1) == I
    assert call(ok, _io(b), start=1 << 30) == U and call(ok, _io(b), Tk=(1 << 30) + 1) == U
    need = b.templora_attention_workspace_bytes(ok, 16, 16)
    assert need > 1024
    assert call(ok, _io(b), n=need - 1) == W and call(ok, _io(b), ws=0) == W and call(ok, _io(b), ws=P + 16) == W
    assert call(ok, _io(b), n=need - 1, fn=lib.templora_attention_fwd) == W
    assert lib.templora_attention_fwd(None, None, 16, 16, 0, vp(P), 1 << 20, None) == I
    assert lib.templora_attention_fwd(C.byref(ok), None, 16, 16, 0, vp(P), 1 << 20, None) == I


def _cache(b, **kw):
    f = dict(n_kv_heads=2, head_dim=64, block_tokens=16, n_blocks=8, k=P, v=P, k_scale=P, v_scale=P, n_seqs=3, max_blocks=4,
             block_table=P)
    f.update(kw)
    return b.KvCacheDesc(*f.values())


def test_kv_cache_refusals(b):
    lib, vp = b.lib, C.c_void_p
    I, U, W = b.ERR_INVALID_ARG, b.ERR_UNSUPPORTED, b.ERR_WORKSPACE

    def append(c, lens=P, off=P, n=3, dt=None, k=P, v=P, lk=0, lv=0, ws=P, nb=1 << 20):
        return lib.templora_kv_cache_append(C.byref(c), vp(lens), vp(off), n, b.BF16 if dt is None else dt, vp(k), vp(v), lk, lv,
                                            vp(ws), nb, None)

    def decode(c, a=None, lens=P, q=P, o=P, lq=0, lo=0, ws=P, nb=1 << 26):
        return lib.templora_attention_decode_fwd(C.byref(a or _desc(b)), C.byref(c), vp(lens), vp(q), lq, vp(o), lo, None,
                                                 vp(ws), nb, None)

    for kw, want in ((dict(n_kv_heads=0), I), (dict(head_dim=24), U), (dict(head_dim=144), U), (dict(block_tokens=8), U),
                     (dict(block_tokens=48), U), (dict(n_blocks=0), I), (dict(n_seqs=0), I), (dict(n_seqs=4097), U),
                     (dict(max_blocks=0), I), (dict(max_blocks=1 << 27), U)):
        assert append(_cache(b, **kw)) == want and decode(_cache(b, **kw)) == want, kw
        assert b.templora_kv_cache_append_workspace_bytes(_cache(b, **kw)) == 0, kw
    for kw in (dict(k=None), dict(v_scale=None), dict(block_table=None), dict(v=P + 4)):
        assert append(_cache(b, **kw)) == I and decode(_cache(b, **kw)) == I, kw
    ok = _cache(b)
    assert append(ok, lens=0) == I and append(ok, k=0) == I and append(ok, n=0) == I and append(ok, v=P + 2) == I
    assert append(ok, off=0, n=4) == I                        # without offsets: one row per sequence
    assert append(ok, dt=9) == U and append(ok, lk=127) == I and append(ok, lv=-5) == I
    assert append(ok, nb=1023) == W and append(ok, ws=0) == W
    assert decode(ok, lens=0) == I and decode(ok, q=0) == I and decode(ok, o=P + 8) == I and decode(ok, lq=511) == I
    assert decode(ok, a=_desc(b, n_kv_heads=4)) == I and decode(ok, a=_desc(b, head_dim=48)) == I
    assert decode(ok, a=_desc(b, n_docs=1, doc_offsets=P)) == U and decode(ok, a=_desc(b, prefix_lens=P)) == U
    need = b.templora_attention_decode_workspace_bytes(_desc(b), ok)
    assert need > 1024 and decode(ok, nb=need - 1) == W and decode(ok, ws=P + 128) == W
    assert b.templora_attention_decode_workspace_bytes(_desc(b, head_dim=48), ok) == 0


def test_binding_checks_shapes_before_the_call(b):
    t = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    a = b.attention_desc(4, 2, 16, b.BF16)
    args = lambda **kw: b.AttentionArgs(a, **{**dict(q=t(5, 4, 16), k=t(7, 2, 16), v=t(7, 2, 16), o=t(5, 4, 16),  # noqa: E731
                                                     lse=t(4, 5, dt=torch.float32)), **kw})
    for kw in (dict(q=t(5, 3, 16)), dict(k=t(7, 2, 8)), dict(v=t(6, 2, 16)), dict(o=t(5, 4, 16, dt=torch.float32)),
               dict(lse=t(5, 4, dt=torch.float32)), dict(q=t(5, 16, 4).transpose(1, 2)), dict(do=t(4, 4, 16))):
        with pytest.raises(ValueError):
            args(**kw)
    with pytest.raises(ValueError):
        args()                                                # tensors on the host
    with pytest.raises(ValueError):
        b.attention_desc(4, 2, 16, b.BF16, slopes=t(3, dt=torch.float32))
    with pytest.raises(ValueError):
        b.attention_desc(4, 2, 16, b.BF16, doc_offsets=torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        b.attention_desc(4, 2, 16, b.BF16, doc_offsets=torch.zeros(3, dtype=torch.int32), prefix_lens=torch.zeros(3, dtype=torch.int32))
    u8 = torch.zeros((4, 2, 16, 16), dtype=torch.uint8)
    with pytest.raises(ValueError):
        b.kv_cache_desc(u8, u8, t(4, 3, dt=torch.float32), t(4, 2, dt=torch.float32), torch.zeros((2, 2), dtype=torch.int32))
    with pytest.raises(ValueError):
        b.kv_cache_desc(u8, u8.float(), t(4, 2, dt=torch.float32), t(4, 2, dt=torch.float32), torch.zeros((2, 2), dtype=torch.int32))


def test_cache_with_too_many_blocks_is_refused(b):
    """A block's head is a 31-bit coordinate."""
    for kw in (dict(n_blocks=1 << 30), dict(n_blocks=(1 << 31) - 1)):
        c = _cache(b, **kw)
        assert b.lib.templora_kv_cache_append(C.byref(c), C.c_void_p(P), C.c_void_p(P), 3, b.BF16, C.c_void_p(P), C.c_void_p(P), 0, 0,
                                              C.c_void_p(P), 1 << 20, None) == b.ERR_UNSUPPORTED
        assert b.templora_attention_decode_workspace_bytes(_desc(b), c) == 0
    assert b.templora_attention_decode_workspace_bytes(_desc(b), _cache(b, n_blocks=(1 << 30) - 1)) > 0


@pytest.mark.parametrize("name", ["q", "k", "v", "o", "do", "dq", "dk", "dv"])
def test_rows_that_share_memory_are_refused_by_attention(b, name):
    """A tensor broadcast along its rows has a row stride of 0, the library's word for contiguous rows: they would be read, or
    written, behind its one row.  Rows that overlap in part are refused too."""
    shape = lambda n: (5, 4, 16) if n in ("q", "o", "do", "dq") else (7, 2, 16)  # noqa: E731
    t = lambda n: torch.zeros(shape(n), dtype=torch.bfloat16)  # noqa: E731
    a = b.attention_desc(4, 2, 16, b.BF16)
    rows, heads, dim = shape(name)
    one = torch.zeros((1, heads, dim), dtype=torch.bfloat16)
    part = torch.zeros(rows * heads * dim, dtype=torch.bfloat16).as_strided((rows, heads, dim), (dim, dim, 1))
    for bad in (one.expand(rows, heads, dim), part):
        given = {n: t(n) for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv")}
        given[name] = bad
        with pytest.raises(ValueError, match="rows"):
            b.AttentionArgs(a, given.pop("q"), given.pop("k"), given.pop("v"), given.pop("o"), torch.zeros((4, 5)), **given)


def test_rows_that_share_memory_are_refused_by_the_cache(b):
    one = lambda h: torch.zeros((1, h, 16), dtype=torch.bfloat16)  # noqa: E731
    t = lambda h: torch.zeros((3, h, 16), dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    c = _cache(b, head_dim=16)
    c._keep = (t(2),)
    for k, v in ((one(2).expand(3, 2, 16), t(2)), (t(2), one(2).expand(3, 2, 16))):
        with pytest.raises(ValueError, match="rows"):
            b.KvCacheAppendArgs(c, i32(3), k, v)
    a = b.attention_desc(4, 2, 16, b.BF16)
    for q, o in ((one(4).expand(3, 4, 16), t(4)), (t(4), one(4).expand(3, 4, 16))):
        with pytest.raises(ValueError, match="rows"):
            b.AttentionDecodeArgs(a, c, i32(3), q, o)
    assert b._rows("q", one(4), 1, 4, 16, b.BF16) == 64                          # one row has no stride to speak of
    with pytest.raises(ValueError, match="contiguous"):
        b._call_on(torch.device("cpu"), None, torch.zeros(1, dtype=torch.uint8).expand(4096), lambda *a: b.OK, "call")


@pytest.mark.parametrize("kw", [dict(n_heads=32, n_kv_heads=32, head_dim=128), dict(n_heads=64, n_kv_heads=8, head_dim=128),
                                dict(n_heads=1, n_kv_heads=1, head_dim=36), dict(n_heads=8, n_kv_heads=1, dtype=0),
                                dict(n_heads=6, n_kv_heads=2, window=700), dict(n_heads=40, n_kv_heads=40, causal=0, window=300)],
                         ids=lambda kw: "-".join(f"{n}{v}" for n, v in kw.items()))
def test_a_workspace_for_long_chunks_serves_shorter_ones(b, kw):
    """The last chunk of a text is shorter than the others: the query never falls as a length grows."""
    d = _desc(b, **kw)
    lengths = sorted({1, 2, 31, 32, 33, 64, 65, 127, 128, 129, 500, 511, 512, 513, 1000, 1024, 1025, 1500, 2047, 2048, 2049, 3000, 4096,
                      4097, 6000, 8192, 20000, 37888, 40000, 100000, *range(64, 2400, 160)})
    size = np.array([[b.templora_attention_workspace_bytes(d, q, k) for k in lengths] for q in lengths], dtype=np.int64)
    assert (size > 1024).all()
    assert (np.diff(size, axis=0) >= 0).all() and (np.diff(size, axis=1) >= 0).all()


def test_arrays_off_their_elements_boundary_are_refused(b):
    """Slopes, offsets, prefix lengths, sequence lengths and statistics are read as 4-byte words."""
    lib, vp, I = b.lib, C.c_void_p, b.ERR_INVALID_ARG
    for kw in (dict(slopes=P + 2), dict(n_docs=1, doc_offsets=P + 1), dict(prefix_lens=P + 3)):
        d = _desc(b, **kw)
        assert b.templora_attention_workspace_bytes(d, 16, 16) == 0, kw
        for fn in (lib.templora_attention_fwd, lib.templora_attention_bwd):
            assert fn(C.byref(d), C.byref(_io(b)), 16, 16, 0, vp(P), 1 << 26, None) == I, kw
    c = _cache(b)
    assert lib.templora_kv_cache_append(C.byref(c), vp(P + 2), vp(P), 3, b.BF16, vp(P), vp(P), 0, 0, vp(P), 1 << 20, None) == I
    assert lib.templora_kv_cache_append(C.byref(c), vp(P), vp(P + 1), 3, b.BF16, vp(P), vp(P), 0, 0, vp(P), 1 << 20, None) == I
    for lens, lse, kw in ((P + 1, P, {}), (P, P + 2, {}), (P, P, dict(slopes=P + 2))):
        assert lib.templora_attention_decode_fwd(C.byref(_desc(b, **kw)), C.byref(c), vp(lens), vp(P), 0, vp(P), 0, vp(lse), vp(P), 1 << 26,
                                                 None) == I
