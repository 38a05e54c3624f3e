"""Pins of the oracle's cache weights, cache eviction and sampling, and the refusals of their entry points.  No GPU."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import templora_oracle as orc

RNG = np.random.default_rng(23)


# ------------------------------------------------------------------ weights
@pytest.mark.parametrize("kw", [{}, dict(window=3), dict(softcap=1.5, slopes=[0.25, 0.5, 0.125, 1.0]), dict(window=1)])
def test_received_weights_are_the_columns_of_the_attention_matrix(kw):
    n, r, H, Hkv, D = 9, 4, 4, 2, 3
    q, k = RNG.standard_normal((r, H, D)), RNG.standard_normal((n, Hkv, D))
    _, lse, P = orc.attention_fwd(q, k, np.zeros_like(k), 0.6, q_start=n - r, causal=True, **kw)
    a = orc.attention_received(q, lse.T, k, 0.6, **kw)
    for hk in range(Hkv):
        for j in range(n):
            assert abs(a[hk, j] - sum(P[h, i, j] for h in (2 * hk, 2 * hk + 1) for i in range(r))) < 1e-12
    assert np.allclose(a.sum(), r * H)                                   # every row pays 1 per head


def test_received_weights_by_hand():
    # one head of one dim, keys 0 and log 3 at a query of 1: weights 1/4 and 3/4
    k = np.array([0.0, math.log(3.0)]).reshape(2, 1, 1)
    a = orc.attention_received(np.ones((1, 1, 1)), np.array([[math.log(4.0)]]), k, 1.0)
    assert np.allclose(a, [[0.25, 0.75]])
    assert np.array_equal(orc.attention_received(np.ones((1, 1, 1)), np.array([[-np.inf]]), k, 1.0), [[0.0, 0.0]])
    # more rows than tokens: the first stand before the text and see nothing
    a = orc.attention_received(np.ones((4, 1, 1)), np.zeros((4, 1)), np.zeros((2, 1, 1)), 1.0)
    assert np.allclose(a, [[2.0, 1.0]])


def test_weights_of_new_tokens_are_set_and_of_old_ones_added():
    w = np.full((3, 1, 4), 10.0)
    orc.kv_weigh(w, np.arange(1.0, 7.0)[None], 2, [2, 0])
    assert w[2, 0].tolist() == [11, 12, 13, 14] and w[0, 0].tolist() == [5, 6, 10, 10] and w[1, 0].tolist() == [10] * 4
    before = w.copy()
    orc.kv_weigh(w, np.ones((1, 6)), 0, [2, 0])                          # no rows: nothing is written
    assert np.array_equal(w, before)


# ------------------------------------------------------------------ eviction
def test_kept_places_by_hand():
    w = [9.0, 1.0, 5.0, 5.0, np.nan, 5.0, 7.0, -np.inf, 0.0, 3.0]
    assert orc.kv_keep(w, 5, 1, 2) == [0, 2, 6, 8, 9]                    # 7, then the first of the three fives
    assert orc.kv_keep(w, 6, 0, 0) == [0, 2, 3, 5, 6, 9]
    assert orc.kv_keep(w, 9, 0, 0) == [0, 1, 2, 3, 4, 5, 6, 8, 9]        # NaN as -infinity: the earlier of the two stays
    assert orc.kv_keep(w, 10, 3, 3) == list(range(10)) and orc.kv_keep(w, 99, 0, 0) == list(range(10))
    assert orc.kv_keep(w, 4, 2, 2) == [0, 1, 8, 9]
    assert orc.kv_keep([], 4, 0, 0) == []


def test_eviction_is_the_kept_tokens_one_by_one():
    """Every kept token's value is its old value rounded once to its new block's scale; what is read stays."""
    heads, bt, dim, n = 2, 4, 3, 11
    k, v = (RNG.integers(0, 256, size=(9, heads, bt, dim)).astype(np.uint8) for _ in range(2))
    ks, vs = (2.0 ** RNG.integers(-6, 6, size=(9, heads)) for _ in range(2))
    w = RNG.standard_normal((9, heads, bt))
    table, to_table = [4, 0, 7], [1, 8]
    was = [x.copy() for x in (k, ks, v, vs, w)]
    kept = orc.kv_evict(k, ks, v, vs, w, table, n, (k, ks, v, vs, w), to_table, 6, 1, 2)
    for now, old in zip((k, ks, v, vs, w), was):
        assert all(np.array_equal(now[b], old[b], equal_nan=True) for b in (0, 2, 3, 4, 5, 6, 7))
    for h in range(heads):
        assert len(kept[h]) == 6 and kept[h] == sorted(kept[h]) and kept[h][0] == 0 and kept[h][-2:] == [9, 10]
        for codes, scales, c0, s0 in ((k, ks, was[0], was[1]), (v, vs, was[2], was[3])):
            for b in range(2):
                top = 0.0
                for i, j in enumerate(kept[h][4 * b:4 * b + 4]):
                    old = orc.e4m3_decode(c0[table[j // bt], h, j % bt]) * s0[table[j // bt], h]
                    new = orc.e4m3_decode(codes[to_table[b], h, i]) * scales[to_table[b], h]
                    step = np.maximum(np.abs(old), 2.0 ** -6 * scales[to_table[b], h]) * 2.0 ** -4
                    assert (np.isnan(old) == np.isnan(new)).all()
                    assert (np.abs(new - old)[~np.isnan(old)] <= step[~np.isnan(old)]).all()
                    assert w[to_table[b], h, i] == was[4][table[j // bt], h, j % bt]
                    top = max(top, np.nanmax(np.abs(np.append(old, 0.0))))
                assert 224 * scales[to_table[b], h] < top <= 448 * scales[to_table[b], h]
    assert np.array_equal(w[8, :, 2:], was[4][8, :, 2:])                 # behind the last kept token


# ------------------------------------------------------------------ sampling
def _dist(x, **kw):
    """Probability of every token, from the definition: draws at the middles of very many equal steps of u."""
    n = 4000
    return np.bincount([orc.sample(x, (i + 0.5) / n, **kw)[0] for i in range(n)], minlength=len(x)) / n


def test_sampling_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    assert [orc.sample(x, u)[0] for u in (0.0, 0.099, 0.101, 0.499, 0.501, 0.699, 0.701, 0.9999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert np.allclose(_dist(x), [0.1, 0.4, 0.2, 0.3], atol=1e-3)
    assert np.allclose(_dist(x, top_k=2), [0, 4 / 7, 0, 3 / 7], atol=1e-3)
    assert np.allclose(_dist(x, top_p=0.69), [0, 4 / 7, 0, 3 / 7], atol=1e-3)
    assert np.allclose(_dist(x, top_p=0.71), [0, 4 / 9, 2 / 9, 3 / 9], atol=1e-3)
    assert np.allclose(_dist(x, top_k=2, top_p=0.57), [0, 1, 0, 0], atol=1e-3)       # 4/7 of what top-k leaves
    assert np.allclose(_dist(x, min_p=0.6), [0, 4 / 7, 0, 3 / 7], atol=1e-3)
    assert np.allclose(_dist(x, temperature=0.5), np.array([1, 16, 4, 9]) / 30, atol=1e-3)
    assert abs(orc.sample(x, 0.6, top_k=2)[1] - math.log(3 / 7)) < 1e-12
    assert orc.sample(x, 0.9, temperature=0.0) == (1, 0.0) and orc.sample(x, 0.9, temperature=float("nan")) == (1, 0.0)
    assert orc.sample(x, 0.9, top_p=0.0)[0] == 1 and orc.sample(x, 0.9, min_p=7.0)[0] == 1 and orc.sample(x, 0.9, top_k=1)[0] == 1


def test_sampling_at_the_edges():
    inf, nan = np.inf, np.nan
    assert orc.sample(np.array([-inf, nan, -inf]), 0.5) == (-1, -inf)
    assert orc.sample(np.array([nan, 1.0, -inf]), 0.99)[0] == 1
    assert [orc.sample(np.array([3.0, inf, 0.0, inf]), u)[0] for u in (0.0, 0.49, 0.5, 1.0)] == [1, 1, 3, 3]
    assert [orc.sample(np.zeros(4), u, top_k=3)[0] for u in (0.0, 0.34, 0.99)] == [0, 1, 2]        # ties: the lower tokens
    assert [orc.sample(np.zeros(4), u, top_p=0.5)[0] for u in (0.0, 0.49, 0.5, 0.99)] == [0, 0, 1, 1]
    assert orc.sample(np.zeros(4), 1.0)[0] == 3 and orc.sample(np.zeros(4), -1.0)[0] == 0 and orc.sample(np.zeros(4), nan)[0] == 0
    assert orc.sample(np.array([0.0, -1000.0]), 1.0)[0] == 0                                       # no weight, never drawn
    assert orc.sample(np.array([2.0]), 0.3) == (0, 0.0)
    assert [orc.sample(np.array([d, 0.0]), 0.0)[0] for d in (-31.1, -31.3)] == [0, 1]              # half of 2^-44 is exp(-31.19)


# ------------------------------------------------------------------ refusals
@pytest.fixture(scope="module")
def b():
    from paper_2401_11504_b200 import build
    build.build_library()
    from paper_2401_11504_b200 import binding
    return binding


P = 0x10000
vp = C.c_void_p


def _attn(b, **kw):
    f = dict(n_heads=8, n_kv_heads=2, head_dim=64, dtype=b.BF16, scale=0.125, softcap=0.0, causal=1, window=0, slopes=None,
             n_docs=0, doc_offsets=None, prefix_lens=None)
    f.update(kw)
    return b.AttentionDesc(*f.values())


def _cache(b, **kw):
    f = dict(n_kv_heads=2, head_dim=64, block_tokens=16, n_blocks=8, k=P, v=P, k_scale=P, v_scale=P, n_seqs=3, max_blocks=4,
             block_table=P)
    f.update(kw)
    return b.KvCacheDesc(*f.values())


BAD_CACHES = [(dict(n_kv_heads=0), "I"), (dict(head_dim=24), "U"), (dict(head_dim=144), "U"), (dict(block_tokens=48), "U"),
              (dict(n_seqs=4097), "U"), (dict(max_blocks=0), "I"), (dict(n_blocks=0), "I")]
BAD_POINTERS = [dict(k=None), dict(v=P + 8), dict(k_scale=P + 4), dict(block_table=None)]


def test_weigh_refusals(b):
    I, U, W = b.ERR_INVALID_ARG, b.ERR_UNSUPPORTED, b.ERR_WORKSPACE

    def call(a=None, c=None, lens=P, off=None, n=3, q=P, lq=0, lse=P, lr=8, lh=1, w=P, ws=P, nb=1 << 20):
        return b.lib.templora_kv_cache_weigh(C.byref(a or _attn(b)), C.byref(c or _cache(b)), vp(lens), vp(off), n, vp(q), lq, vp(lse), lr,
                                             lh, vp(w), vp(ws), nb, None)

    size = lambda a, c, n=3: b.templora_kv_cache_weigh_workspace_bytes(a, c, n)  # noqa: E731
    for kw, want in BAD_CACHES:
        assert call(c=_cache(b, **kw)) == {"I": I, "U": U}[want], kw
        assert size(_attn(b), _cache(b, **kw)) == 0
    for kw in BAD_POINTERS:
        assert call(c=_cache(b, **kw)) == I, kw
    for kw, want in ((dict(n_kv_heads=4), I), (dict(head_dim=32), I), (dict(n_docs=1, doc_offsets=P), U), (dict(prefix_lens=P), U),
                     (dict(dtype=9), U), (dict(scale=float("nan")), I), (dict(slopes=P + 2), I), (dict(window=-1), I)):
        assert call(a=_attn(b, **kw)) == want, kw
        assert size(_attn(b, **kw), _cache(b)) == 0
    for kw in (dict(lens=None), dict(q=None), dict(lse=None), dict(w=None), dict(q=P + 8), dict(lens=P + 1), dict(off=P + 2), dict(lse=P + 2),
               dict(w=P + 3), dict(n=0), dict(n=4), dict(n=2), dict(n=-1, off=P), dict(lq=511), dict(lq=-512), dict(lr=-1), dict(lh=-8)):
        assert call(**kw) == I, kw
    assert call(n=(1 << 30) + 1, off=P) == U
    need = size(_attn(b), _cache(b))
    assert need >= 1024 and size(_attn(b), _cache(b), 0) == 0
    for kw in (dict(ws=None), dict(ws=P + 16), dict(nb=need - 1)):
        assert call(**kw) == W, kw
    assert b.lib.templora_kv_cache_weigh(None, None, None, None, 0, None, 0, None, 0, 0, None, None, 0, None) == I


def test_evict_refusals(b):
    I, U, W = b.ERR_INVALID_ARG, b.ERR_UNSUPPORTED, b.ERR_WORKSPACE

    def call(c=None, w=P, lens=P, to=None, tw=P, nl=P, keep=20, first=0, recent=0, kept=None, ws=P, nb=1 << 20):
        return b.lib.templora_kv_cache_evict(C.byref(c or _cache(b)), vp(w), vp(lens), C.byref(to or _cache(b, block_table=2 * P)), vp(tw), vp(nl), keep, first, recent,
                                             vp(kept), vp(ws), nb, None)

    for kw, want in BAD_CACHES:
        assert call(c=_cache(b, **kw)) == {"I": I, "U": U}[want], kw
        assert call(to=_cache(b, **kw)) == {"I": I, "U": U}[want], kw
        assert b.templora_kv_cache_evict_workspace_bytes(_cache(b, **kw), 20) == 0
    for kw in BAD_POINTERS:
        assert call(c=_cache(b, **kw)) == I and call(to=_cache(b, **kw)) == I, kw
    for kw in (dict(n_kv_heads=4), dict(head_dim=32), dict(block_tokens=32), dict(n_seqs=2), dict(max_blocks=1), {}):
        assert call(to=_cache(b, **kw)) == I, kw                         # the last: the pool under the table that is read
    for kw in (dict(w=None), dict(lens=None), dict(tw=None), dict(nl=None), dict(w=P + 1), dict(lens=P + 2), dict(tw=P + 2), dict(nl=P + 3),
               dict(kept=P + 2), dict(keep=0), dict(keep=-1), dict(first=-1), dict(recent=-1), dict(first=11, recent=10),
               dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), dict(keep=65)):
        assert call(**kw) == I, kw
    need = b.templora_kv_cache_evict_workspace_bytes(_cache(b), 20)
    assert need >= 1024 + 6 * 20 * 4 and b.templora_kv_cache_evict_workspace_bytes(_cache(b), 0) == 0
    for kw in (dict(ws=None), dict(ws=P + 16), dict(nb=need - 1)):
        assert call(**kw) == W, kw
    assert b.lib.templora_kv_cache_evict(None, None, None, None, None, None, 1, 0, 0, None, None, 0, None) == I


def test_sample_refusals(b):
    I, U = b.ERR_INVALID_ARG, b.ERR_UNSUPPORTED

    def call(rows=2, **kw):
        f = dict(vocab=100, dtype=b.F32, logits=P, ld=0, temperature=P, top_k=P, top_p=P, min_p=P, u=P, tokens=P, logprobs=P)
        f.update(kw)
        return b.lib.templora_sample(C.byref(b.SampleDesc(*f.values())), rows, None)

    for kw, want in ((dict(rows=0), I), (dict(rows=-3), I), (dict(vocab=0), I), (dict(vocab=(1 << 18) + 1), U), (dict(dtype=4), U), (dict(logits=None), I),
                     (dict(logits=P + 2), I), (dict(logits=P + 1, dtype=1), I), (dict(u=None), I), (dict(tokens=None), I), (dict(ld=99), I), (dict(ld=-100), I), (dict(ld=1 << 40), I),
                     (dict(temperature=P + 2), I), (dict(top_k=P + 1), I), (dict(top_p=P + 2), I), (dict(min_p=P + 3), I), (dict(u=P + 2), I),
                     (dict(tokens=P + 2), I), (dict(logprobs=P + 1), I), (dict(rows=(1 << 24) + 1), U)):
        assert call(**kw) == want, kw
    assert b.lib.templora_sample(None, 1, None) == I


def test_binding_refusals(b):
    z = torch.zeros
    i32 = lambda *n: z(n, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="rows"):
        b.SampleArgs(z(1, 8).expand(3, 8), z(3), i32(3))
    with pytest.raises(ValueError, match="contiguous rows"):
        b.SampleArgs(z(8, 3).T, z(3), i32(3))
    for kw in (dict(u=z(2)), dict(tokens=z(3)), dict(top_k=z(3)), dict(top_p=i32(3)), dict(min_p=z(6)[::2]), dict(logprobs=z(3, 1)),
               dict(temperature=z(3).double())):
        with pytest.raises(ValueError, match=list(kw)[0]):
            b.SampleArgs(**{**dict(logits=z(3, 8), u=z(3), tokens=i32(3)), **kw})
    with pytest.raises(ValueError, match="one CUDA device"):
        b.SampleArgs(z(3, 8), z(3), i32(3))
    c = _cache(b)
    c._keep = (z(1),)
    a = b.attention_desc(8, 2, 64, b.BF16)
    q, lse, w = z(3, 8, 64, dtype=torch.bfloat16), z(3, 8), z(8, 2, 16)
    for kw, what in ((dict(q=q.float()), "q"), (dict(lse=z(8, 3)), "lse"), (dict(weights=z(8, 2, 17)), "weights"), (dict(weights=z(8, 2, 32)[..., ::2]), "weights"),
                     (dict(seq_lens=i32(2)), "seq_lens"), (dict(row_offsets=i32(3)), "row_offsets"), (dict(q=z(1, 8, 64, dtype=torch.bfloat16).expand(3, 8, 64)), "rows")):
        with pytest.raises(ValueError, match=what):
            b.KvCacheWeighArgs(**{**dict(attn=a, cache=c, seq_lens=i32(3), q=q, lse=lse, weights=w), **kw})
    for kw, what in ((dict(weights=z(7, 2, 16)), "weights"), (dict(to_weights=w.double()), "to_weights"), (dict(new_lens=z(3)), "new_lens"), (dict(seq_lens=i32(4)), "seq_lens"),
                     (dict(kept=i32(3, 2, 19)), "kept"), (dict(kept=z(3, 2, 20)), "kept")):
        with pytest.raises(ValueError, match=what):
            b.KvCacheEvictArgs(**{**dict(cache=c, weights=w, seq_lens=i32(3), to=c, to_weights=w, new_lens=i32(3), n_keep=20), **kw})
