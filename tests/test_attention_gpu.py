"""Attention of a chunk, forward and backward, against the fp64 oracle, element by element.

The bound of an element is what its roundings can make of it.  bf16 path: probabilities and score gradients are rounded
to bf16 before the second product (2^-8 of each term), the result once more (2^-8 of the value).  Everything else is
fp32: products of up to 128 terms, exp and tanh, and sums stay within SLACK of the terms' magnitudes, where a term's
relative error is the absolute error of its score: 2^-24 * sum |q k| * scale * sqrt(128) < 1e-5 for the inputs here, and
about 1e-7 * softcap for the capped ones.
"""
import numpy as np
import pytest
import torch

from oracle import templora_oracle as orc
from parity_utils import Guarded

pytestmark = pytest.mark.gpu

ROUND = {"bf16": 2.0 ** -8, "f32": 2.0 ** -23}
SLACK = 4e-5
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def b():
    from paper_2401_11504_b200 import build
    build.build_library()
    from paper_2401_11504_b200 import binding
    binding.templora_set_kernel_path(0)
    yield binding
    binding.templora_set_kernel_path(0)


def make(case, seed=1):
    """Host tensors and masks of a case: (dtype, H, Hkv, D, Tq, context, masks)."""
    dtype, H, Hkv, D, Tq, ctx, masks = case
    g = torch.Generator().manual_seed(seed)
    Tk = Tq + ctx
    r = lambda *s: torch.randn(s, generator=g).to(DT[dtype])  # noqa: E731
    return dict(q=r(Tq, H, D) * 1.5, k=r(Tk, Hkv, D), v=r(Tk, Hkv, D), do=r(Tq, H, D))


def oracle_masks(masks, ctx):
    m = dict(masks)
    m["q_start"] = m.get("q_start", ctx)
    m.setdefault("causal", True)
    return m


class Call:
    """One case on the device: guarded outputs, optionally q, k, v and their gradients as slices of wider buffers."""

    def __init__(self, b, case, host, wide=False):
        dtype, H, Hkv, D, Tq, ctx, masks = case
        self.b, self.guard, dt, Tk = b, Guarded(), DT[dtype], Tq + ctx
        dev = {n: t.cuda() for n, t in host.items()}
        i32 = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        sl = masks.get("slopes")
        self.desc = b.attention_desc(H, Hkv, D, {"bf16": b.BF16, "f32": b.F32}[dtype], softcap=masks.get("softcap", 0.0),
                                     causal=masks.get("causal", True), window=masks.get("window", 0),
                                     slopes=None if sl is None else torch.tensor(sl, dtype=torch.float32, device="cuda"),
                                     doc_offsets=i32(masks.get("doc_offsets")), prefix_lens=i32(masks.get("prefix_lens")))
        if wide:
            buf = torch.full((Tk, H + 2 * Hkv, D), float("nan"), dtype=dt, device="cuda")
            q, k, v = buf[ctx:, :H], buf[:, H:H + Hkv], buf[:, H + Hkv:]
            q.copy_(dev["q"]); k.copy_(dev["k"]); v.copy_(dev["v"])
            dev.update(q=q, k=k, v=v)
            gb = self.guard.empty((Tk, H + 2 * Hkv, D), dt)
            self.rest = gb[:ctx, :H]
            dq, dk, dv = gb[ctx:, :H], gb[:, H:H + Hkv], gb[:, H + Hkv:]
        else:
            dq, dk, dv = (self.guard.empty((n, m, D), dt) for n, m in ((Tq, H), (Tk, Hkv), (Tk, Hkv)))
        self.o, self.lse = self.guard.empty((Tq, H, D), dt), self.guard.empty((H, Tq), torch.float32)
        self.dq, self.dk, self.dv, self.dev = dq, dk, dv, dev
        self.ws = self.guard.workspace(b.templora_attention_workspace_bytes(self.desc, Tq, Tk))
        self.args = b.AttentionArgs(self.desc, dev["q"], dev["k"], dev["v"], self.o, self.lse,
                                    q_start=masks.get("q_start", ctx), do=dev["do"], dq=dq, dk=dk, dv=dv)

    def forward(self):
        self.b.templora_attention_fwd(self.args, self.ws)

    def backward(self):
        self.b.templora_attention_bwd(self.args, self.ws)

    def check(self):
        torch.cuda.synchronize()
        self.guard.check()
        code, where = self.b.templora_read_device_status(self.ws)
        assert code == 0, (code, where)


def f(t):
    return t.double().cpu().numpy()


def near(name, got, want, bound):
    assert got.shape == want.shape and np.isfinite(got).all(), f"{name}: not finite"
    over = np.abs(got - want) - bound
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, f"{name}{at}: {got[at]} against {want[at]}, bound {bound[at]:.3e}"


def check_forward(case, host, o, lse, rows=None):
    dtype, H, Hkv, D, Tq, ctx, masks = case
    v = f(host["v"])
    ref, ref_lse, P = orc.attention_fwd(f(host["q"]), f(host["k"]), v, np.float32(D ** -0.5), **oracle_masks(masks, ctx))
    w = np.stack([P[h] @ np.abs(v[:, h // (H // Hkv)]) for h in range(H)], axis=1)
    rows = slice(None) if rows is None else rows
    round_p = ROUND[dtype] if dtype == "bf16" else 0.0
    near("o", f(o)[rows], ref[rows], ((round_p + SLACK) * w + ROUND[dtype] * np.abs(ref))[rows])
    got, want = f(lse)[:, rows], ref_lse[:, rows]
    assert np.array_equal(np.isneginf(got), np.isneginf(want))
    fin = np.isfinite(want)
    near("lse", got[fin], want[fin], SLACK * (1 + np.abs(want[fin])))
    return ref


def check_backward(case, host, o, dq, dk, dv, q_rows=None, k_rows=None):
    dtype, H, Hkv, D, Tq, ctx, masks = case
    q, k, v, do = (f(host[n]) for n in ("q", "k", "v", "do"))
    scale, group = float(np.float32(D ** -0.5)), H // Hkv
    m = oracle_masks(masks, ctx)
    refs = orc.attention_bwd(q, k, v, f(o), do, scale, **m)
    z, t = orc.attention_scores(q, k, scale, **m)
    P, _ = orc._softmax_rows(z)
    bounds = [np.zeros_like(x) for x in refs]
    r = ROUND[dtype] if dtype == "bf16" else 0.0
    for h in range(H):
        hk = h // group
        dP = do[:, h] @ v[:, hk].T
        delta = (do[:, h] * f(o)[:, h]).sum(axis=1, keepdims=True)
        size = np.abs(do[:, h]) @ np.abs(v[:, hk]).T + (np.abs(do[:, h]) * np.abs(f(o)[:, h])).sum(axis=1, keepdims=True)
        err = scale * (r * np.abs(P[h] * (dP - delta)) + SLACK * P[h] * size)
        bounds[0][:, h] += err @ np.abs(k[:, hk])
        bounds[1][:, hk] += err.T @ np.abs(q[:, h])
        bounds[2][:, hk] += ((r + SLACK) * P[h]).T @ np.abs(do[:, h])
    for name, got, ref, bound, rows in zip(("dq", "dk", "dv"), (dq, dk, dv), refs, bounds, (q_rows, k_rows, k_rows)):
        rows = slice(None) if rows is None else rows
        near(name, f(got)[rows], ref[rows], (bound + ROUND[dtype] * np.abs(ref) + 1e-30)[rows])


CASES = [
    # dtype, heads, kv heads, head_dim, Tq, context, masks
    ("bf16", 2, 2, 128, 1, 0, {}),
    ("bf16", 4, 1, 64, 1, 300, {}),
    ("bf16", 2, 1, 128, 127, 0, {}),
    ("bf16", 2, 2, 128, 128, 0, dict(causal=False)),
    ("bf16", 2, 2, 128, 129, 0, {}),
    ("bf16", 4, 2, 64, 257, 0, {}),
    ("bf16", 2, 1, 128, 300, 213, {}),
    ("bf16", 2, 2, 80, 190, 0, dict(softcap=5.0)),
    ("bf16", 3, 3, 96, 200, 0, dict(slopes=[0.5, 0.03, 0.0])),
    ("bf16", 4, 2, 128, 200, 0, dict(softcap=20.0, slopes=[0.25, 0.125, 0.06, 0.03], causal=False)),
    ("bf16", 2, 1, 128, 500, 0, dict(window=1)),
    ("bf16", 2, 1, 128, 400, 70, dict(window=100)),
    ("bf16", 2, 1, 64, 400, 0, dict(window=37, causal=False)),
    ("bf16", 2, 1, 128, 500, 0, dict(doc_offsets=[0, 1, 1, 130, 385, 470])),                     # an empty one, padding behind
    ("bf16", 2, 1, 128, 500, 0, dict(doc_offsets=[0, 100, 300, 500], prefix_lens=[50, 0, 190])),
    ("bf16", 2, 1, 64, 300, 100, dict(doc_offsets=[0, 120, 390], causal=False)),
    ("bf16", 2, 1, 128, 260, 0, dict(prefix_lens=[140])),
    ("bf16", 2, 1, 128, 200, 0, dict(doc_offsets=[50, 60, 150])),                                # rows ahead of the first
    ("bf16", 2, 1, 128, 64, 0, dict(q_start=1000)),                                              # queries far behind all keys
    ("bf16", 2, 2, 40, 100, 0, {}),
    ("bf16", 2, 2, 8, 100, 0, {}),
    ("bf16", 2, 1, 36, 90, 0, dict(softcap=5.0)),                                                # not a multiple of 8
    ("f32", 4, 2, 64, 65, 0, {}),
    ("f32", 2, 2, 128, 130, 70, dict(softcap=20.0)),
    ("f32", 2, 1, 128, 1, 0, {}),
    ("f32", 2, 1, 33, 70, 0, dict(causal=False)),
    ("f32", 2, 1, 80, 150, 0, dict(doc_offsets=[0, 40, 110], prefix_lens=[13, 60], slopes=[0.1, 0.2])),
    ("f32", 2, 1, 64, 251, 0, dict(window=64)),
    ("f32", 2, 1, 64, 100, 0, dict(window=20, causal=False)),
]


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:6]) + "".join(sorted(c[6])))
def test_attention_matches_oracle(b, case, wide):
    host = make(case)
    c = Call(b, case, host, wide)
    if any(t.data_ptr() % 16 for t in (c.dev["k"], c.dev["v"], c.dk, c.dv)):
        with pytest.raises(b.TemploraError):     # slices that begin off a 16-byte boundary are refused
            c.forward() or c.backward()
        return
    c.forward()
    c.check()
    check_forward(case, host, c.o, c.lse)
    c.backward()
    c.check()
    check_backward(case, host, c.o.cpu(), c.dq, c.dk, c.dv)


@pytest.mark.parametrize("path", [1, 2])
def test_other_kernel_paths(b, path):
    case = ("bf16", 4, 2, 128, 200, 57, dict(softcap=10.0))
    host = make(case)
    prev = b.templora_set_kernel_path(path)
    try:
        c = Call(b, case, host)
        c.forward()
        c.backward()
        c.check()
    finally:
        b.templora_set_kernel_path(prev)
    check_forward(case, host, c.o, c.lse)
    check_backward(case, host, c.o.cpu(), c.dq, c.dk, c.dv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_masked_places_reach_nothing(b, dtype, bad):
    """One document's rows, and the rows behind the last document, hold non-finite values; the others do not notice."""
    offs = [0, 150, 161, 330]
    case = (dtype, 2, 1, 128, 400, 0, dict(doc_offsets=offs))
    host = make(case)
    clean = {n: t.clone() for n, t in host.items()}
    for n in ("q", "k", "v", "do"):
        host[n][150:161] = bad
        host[n][330:] = bad
        clean[n][150:161] = 0
        clean[n][330:] = 0
    c = Call(b, case, host)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    c.guard.check()
    rows = np.r_[0:150, 161:400]                 # the rows behind the last document come out as zeros
    check_forward(case, clean, c.o, c.lse, rows)
    o = c.o.cpu().clone()
    o[150:161] = 0
    check_backward(case, clean, o, c.dq, c.dk, c.dv, rows, rows)
    assert (c.o[330:] == 0).all() and torch.isneginf(c.lse[:, 330:]).all() and (c.dk[330:] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_bad_value_reaches_the_rows_that_see_it(b, dtype):
    case = (dtype, 2, 2, 64, 300, 0, {})
    host = make(case)
    clean = host["v"].clone()
    host["v"][200, 0, 5] = float("nan")
    c = Call(b, case, host)
    c.forward()
    torch.cuda.synchronize()
    o = f(c.o)
    assert np.isnan(o[200:, 0, 5]).all() and np.isfinite(o[:200]).all() and np.isfinite(o[:, 1]).all()
    assert np.isfinite(np.delete(o[:, 0], 5, axis=1)).all()
    check_forward(case, {**host, "v": clean}, c.o, c.lse, np.r_[0:200])


def test_large_scores_do_not_overflow(b):
    case = ("bf16", 2, 2, 128, 150, 0, {})
    host = make(case)
    host["q"] *= 64.0
    host["k"] *= 64.0
    c = Call(b, case, host)
    c.forward()
    c.check()
    o = f(c.o)
    assert np.isfinite(o).all() and np.abs(o).max() <= np.abs(f(host["v"])).max() * (1 + 2.0 ** -8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_call_same_bits_and_replay(b, dtype):
    """Twice the same bits; recorded into a CUDA graph on a stream of its own and replayed with new contents."""
    case = (dtype, 4, 2, 128, 333, 0, dict(doc_offsets=[0, 200, 333], softcap=10.0))
    host, other = make(case, 1), make(case, 2)
    c = Call(b, case, host)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    first = [t.clone() for t in (c.o, c.lse, c.dq, c.dk, c.dv)]
    for t in (c.o, c.lse, c.dq, c.dk, c.dv):
        t.fill_(float("nan"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.forward()
        c.backward()
    graph.replay()
    torch.cuda.synchronize()
    for x, y in zip(first, (c.o, c.lse, c.dq, c.dk, c.dv)):
        assert torch.equal(x, y)
    for n in ("q", "k", "v", "do"):
        c.dev[n].copy_(other[n])
    graph.replay()
    c.check()
    check_forward(case, other, c.o, c.lse)
    check_backward(case, other, c.o.cpu(), c.dq, c.dk, c.dv)


def test_untrusted_offsets_stay_inside(b):
    """Document offsets and prefix lengths that make no sense are clamped; nothing outside is read or written."""
    for offs, pre in (([-5, 7, 100000, 3], [10 ** 9, -4, 2 ** 31 - 1]), ([2 ** 31 - 1, 0, -2 ** 31, 5], [0, 0, 0])):
        case = ("bf16", 2, 1, 128, 200, 0, dict(doc_offsets=offs, prefix_lens=pre))
        host = make(case)
        c = Call(b, case, host)
        c.forward()
        c.backward()
        c.check()
        assert all(torch.isfinite(t).all() for t in (c.o, c.dq, c.dk, c.dv))


def test_long_rows_in_pieces(b):
    """A few queries over a long context, against the oracle row by row (checked on one head)."""
    case = ("bf16", 2, 1, 128, 5, 9000, dict(window=8500))
    host = make(case)
    c = Call(b, case, host)
    c.forward()
    c.backward()
    c.check()
    check_forward(case, host, c.o, c.lse)
    check_backward(case, host, c.o.cpu(), c.dq, c.dk, c.dv)


@pytest.mark.parametrize("case", [
    ("f32", 2, 1, 128, 1100, 0, {}),                                                             # heads and stretches of queries
    ("f32", 3, 1, 64, 700, 40, dict(window=90)),                                                 # stretches that reach no key of a tile
    ("f32", 6, 2, 36, 520, 0, dict(doc_offsets=[5, 200, 515], prefix_lens=[20, 300], softcap=10.0)),
    ("bf16", 2, 1, 36, 600, 0, dict(causal=False)),
    ("bf16", 8, 1, 128, 300, 0, {}),                                                             # tensor cores: a part to each head
    ("bf16", 2, 1, 64, 1100, 33, dict(window=200, softcap=10.0)),                                # and stretches that reach no key of a tile
    ("bf16", 3, 1, 80, 700, 0, dict(doc_offsets=[3, 100, 650], prefix_lens=[20, 200])),
    ("f32", 20, 1, 16, 30, 0, {}),                                                               # a part to each head
], ids=lambda c: "-".join(str(x) for x in c[:6]) + "".join(sorted(c[6])))
def test_key_gradients_added_from_parts(b, case):
    host = make(case)
    c = Call(b, case, host)
    c.forward()
    c.backward()
    c.check()
    check_backward(case, host, c.o.cpu(), c.dq, c.dk, c.dv)
    dk, dv = c.dk.clone(), c.dv.clone()
    c.backward()
    c.check()
    assert torch.equal(dk, c.dk) and torch.equal(dv, c.dv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale, softcap, slopes", [(-0.2, 0.0, None), (0.0, 0.0, None), (0.0, 3.0, None), (0.1, 1e-39, None),
                                                    (-0.05, 2.0, [0.03, -0.01]), (0.3, 2e5, None), (0.3, 3e38, [0.03, 0.0])])
def test_unusual_scales_and_caps(b, dtype, scale, softcap, slopes):
    """Negative and zero scales, a subnormal cap (every score becomes 0), slopes of either sign."""
    case = (dtype, 2, 1, 64, 200, 30, {})
    host = make(case)
    c = Call(b, case, host)
    c.desc = b.attention_desc(2, 1, 64, {"bf16": b.BF16, "f32": b.F32}[dtype], scale=scale, softcap=softcap,
                              slopes=None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device="cuda"))
    c.args = b.AttentionArgs(c.desc, c.dev["q"], c.dev["k"], c.dev["v"], c.o, c.lse, q_start=30, do=c.dev["do"], dq=c.dq, dk=c.dk, dv=c.dv)
    c.forward()
    c.check()
    s32 = float(np.float32(scale))
    kw = dict(q_start=30, causal=True, softcap=float(np.float32(softcap)), slopes=slopes)
    v = f(host["v"])
    ref, ref_lse, P = orc.attention_fwd(f(host["q"]), f(host["k"]), v, s32, **kw)
    w = np.stack([P[h] @ np.abs(v[:, 0]) for h in range(2)], axis=1)
    round_p = ROUND[dtype] if dtype == "bf16" else 0.0
    near("o", f(c.o), ref, (round_p + SLACK) * w + ROUND[dtype] * np.abs(ref))
    near("lse", f(c.lse), ref_lse, SLACK * (1 + np.abs(ref_lse)))
    if softcap != 1e-39:                     # there the gradient of tanh is a jump
        c.backward()
        c.check()
        for got, want in zip((c.dq, c.dk, c.dv), orc.attention_bwd(f(host["q"]), f(host["k"]), v, f(c.o), f(host["do"]), s32, **kw)):
            if scale == 0.0 and got is not c.dv:
                assert (got == 0).all()
            else:
                assert np.isfinite(f(got)).all()
                assert np.abs(f(got) - want).max() <= (2.0 ** -6 if dtype == "bf16" else 1e-4) * np.abs(want).max()


@pytest.mark.parametrize("case", [
    ("bf16", 2, 1, 128, 60, 2400, {}),
    ("bf16", 3, 3, 64, 300, 1700, dict(causal=False)),
    ("bf16", 4, 2, 80, 200, 3000, dict(softcap=10.0, slopes=[0.1, 0.05, 0.02, 0.01])),
    ("bf16", 2, 1, 128, 1800, 0, dict(doc_offsets=[0, 600, 601, 1500], prefix_lens=[50, 0, 700])),    # rows without keys behind
    ("bf16", 1, 1, 96, 1700, 100, dict(window=1500)),
    ("bf16", 2, 2, 40, 1, 5000, {}),
], ids=lambda c: "-".join(str(x) for x in c[:6]) + "".join(sorted(c[6])))
def test_rows_whose_keys_are_shared_out(b, case):
    host = make(case)
    c = Call(b, case, host)
    c.forward()
    c.check()
    check_forward(case, host, c.o, c.lse)
    o, lse = c.o.clone(), c.lse.clone()
    c.backward()                             # the workspace again, for something else
    c.forward()
    c.check()
    assert torch.equal(o, c.o) and torch.equal(lse, c.lse)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_bad_values_in_shared_out_keys(b, bad):
    """Values that a row's mask hides never reach it, through the parts' sums either; one that it sees does."""
    case = ("bf16", 2, 1, 64, 1600, 400, dict(window=1200))
    host = make(case)
    c = Call(b, case, host)
    c.dev["v"][1000] = bad                   # seen by positions 1000 .. 2199
    c.dev["k"][1990] = bad
    c.forward()
    c.check()
    # rows up to position 999 as without them, within the bound of the clean call: rows that share a tile with such a value are
    # formed again with fp32 weights, where the others' are rounded to bf16, 2^-8 of each
    check_forward(case, host, c.o, c.lse, rows=slice(0, 600))
    assert not torch.isfinite(c.o[600:700]).all()


@pytest.mark.parametrize("case", [
    ("f32", 2, 1, 64, 1100, 0, {}),
    ("f32", 1, 1, 96, 40, 1500, dict(slopes=[0.02], softcap=15.0)),
    ("f32", 2, 2, 80, 1300, 0, dict(doc_offsets=[0, 100, 1200], prefix_lens=[30, 700])),             # rows without keys behind
    ("f32", 1, 1, 128, 1, 2100, dict(causal=False)),
    ("bf16", 2, 1, 36, 600, 900, dict(window=800)),
], ids=lambda c: "-".join(str(x) for x in c[:6]) + "".join(sorted(c[6])))
def test_generic_kernels_with_shared_out_keys(b, case):
    host = make(case)
    c = Call(b, case, host)
    c.forward()
    c.check()
    check_forward(case, host, c.o, c.lse)
    c.backward()
    c.check()
    check_backward(case, host, c.o.cpu(), c.dq, c.dk, c.dv)
    dq = c.dq.clone()
    c.backward()
    c.check()
    assert torch.equal(dq, c.dq)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_longest_chunks_workspace_serves_the_last_one(b, dtype):
    """A workspace asked for at 4096 tokens, a chunk of 1000 tokens: the bits of a call with a workspace of its own."""
    case = (dtype, 32, 32, 64, 1000, 0, {})
    host = make(case)
    c = Call(b, case, host)
    c.forward()
    c.backward()
    c.check()
    first = [t.clone() for t in (c.o, c.lse, c.dq, c.dk, c.dv)]
    for t in (c.o, c.lse, c.dq, c.dk, c.dv):
        t.fill_(float("nan"))
    c.ws = c.guard.workspace(b.templora_attention_workspace_bytes(c.desc, 4096, 4096))
    c.forward()
    c.backward()
    c.check()
    for x, y in zip(first, (c.o, c.lse, c.dq, c.dk, c.dv)):
        assert torch.equal(x, y)


BAD_CASES = [
    ("bf16", 4, 2, 64, 700, 0, {}),
    ("bf16", 4, 2, 128, 700, 0, dict(doc_offsets=[0, 300, 690], prefix_lens=[20, 200])),
    ("bf16", 2, 2, 80, 500, 0, dict(window=130, softcap=10.0)),
    ("bf16", 2, 1, 64, 300, 1700, {}),                           # keys shared out, dk and dv in parts
    ("f32", 4, 2, 64, 700, 0, {}),
    ("f32", 2, 1, 96, 40, 1500, dict(causal=False)),             # parts on the generic path
    ("bf16", 2, 1, 36, 500, 0, dict(doc_offsets=[0, 300, 490])),
]


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("where", ["v", "do"])
@pytest.mark.parametrize("case", BAD_CASES, ids=lambda c: "-".join(str(x) for x in c[:6]) + "".join(sorted(c[6])))
def test_bad_values_show_where_they_are_seen_and_nowhere_else(b, case, where, bad):
    """Single bad values among v or dO: the places of o, dq, dk, dv that see one are not finite, all others are the clean call's."""
    dtype, H, Hkv, D, Tq, ctx, masks = case
    Tk, group, m = Tq + ctx, H // Hkv, oracle_masks(masks, ctx)
    host = make(case)
    clean = {n: t.clone() for n, t in host.items()}
    at = [(3 * Tk // 5, 0, 5), (3 * Tk // 5, Hkv - 1, D - 1), (Tk // 7, Hkv - 1, 1)] if where == "v" else \
         [(3 * Tq // 5, 0, 5), (3 * Tq // 5, H - 1, D - 1), (Tq // 7, H - 1, 1)]
    for a in at:
        host[where][a] = bad
        clean[where][a] = 0
    c = Call(b, case, host)
    c.forward()
    c.backward()
    c.check()
    seen = np.zeros((Tq, Tk), dtype=bool)
    for i in range(Tq):
        seen[i, slice(*orc.attention_interval(m["q_start"] + i, Tk, m["causal"], m.get("window", 0), m.get("doc_offsets"),
                                              m.get("prefix_lens")))] = True
    bad_v, bad_do = ~np.isfinite(f(host["v"])), ~np.isfinite(f(host["do"]))
    sums = lambda a, x: np.einsum("ij,jd->id", a.astype(np.int64), x.astype(np.int64)) > 0  # noqa: E731
    bad_o = np.stack([sums(seen, bad_v[:, h // group]) for h in range(H)], axis=1)
    bad_row = (bad_o | bad_do).any(axis=2) & seen.any(axis=1)[:, None]                        # delta is not finite
    bad_dq = np.broadcast_to(bad_row[:, :, None], bad_o.shape)
    bad_dk, bad_dv = np.zeros((Tk, Hkv, D), dtype=bool), np.zeros((Tk, Hkv, D), dtype=bool)
    for h in range(H):
        bad_dk[:, h // group] |= sums(seen.T, bad_row[:, h:h + 1])
        bad_dv[:, h // group] |= sums(seen.T, bad_do[:, h])
    for name, got, want in (("o", c.o, bad_o), ("dq", c.dq, bad_dq), ("dk", c.dk, bad_dk), ("dv", c.dv, bad_dv)):
        assert np.array_equal(~np.isfinite(f(got)), want), name
    assert not bad_o.all() and (bad_o.any() or where == "do")
    scale = float(np.float32(D ** -0.5))
    fill = lambda got, mask, ref: torch.from_numpy(np.where(mask, ref, f(got)))  # noqa: E731
    o = fill(c.o, bad_o, orc.attention_fwd(f(clean["q"]), f(clean["k"]), f(clean["v"]), scale, **m)[0])
    check_forward(case, clean, o, c.lse)
    refs = orc.attention_bwd(f(clean["q"]), f(clean["k"]), f(clean["v"]), f(o), f(clean["do"]), scale, **m)
    grads = [fill(got, mask, ref) for got, mask, ref in zip((c.dq, c.dk, c.dv), (bad_dq, bad_dk, bad_dv), refs)]
    check_backward(case, clean, o, *grads)


def device_ms(fn):
    fn()
    times = []
    for _ in range(4):
        a, e = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        fn()
        e.record()
        e.synchronize()
        times.append(a.elapsed_time(e))
    return min(times)


@pytest.mark.parametrize("token", [0, 900])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_step_gone_wrong_takes_about_as_long_as_any(b, dtype, token):
    """One bad value that all later rows see: rows that it explains are not formed again, key by key.  (Formed again, they took
    hundreds of times the call.)"""
    case = (dtype, 8, 1, 128, 1800, 0, {})
    host = make(case)
    c = Call(b, case, host)
    clean = device_ms(c.forward), device_ms(c.backward)
    c.dev["v"][token, 0, 5] = float("nan")
    wrong = device_ms(c.forward), device_ms(c.backward)
    print(f"{dtype} {token}: forward {1e3 * clean[0]:.0f} -> {1e3 * wrong[0]:.0f} us, backward {1e3 * clean[1]:.0f} -> {1e3 * wrong[1]:.0f} us")
    assert wrong[0] < 40 * clean[0] and wrong[1] < 40 * clean[1]


class few_sms:
    """A stream whose kernels are planned for `limit` SMs, current inside the block."""

    def __init__(self, b, limit):
        self.b, self.stream, self.limit = b, torch.cuda.Stream(), limit

    def __enter__(self):
        self.b.templora_set_stream_sm_limit(self.stream, self.limit)
        torch.cuda.synchronize()
        self.ctx = torch.cuda.stream(self.stream)
        self.ctx.__enter__()

    def __exit__(self, *exc):
        torch.cuda.synchronize()
        self.ctx.__exit__(*exc)
        self.b.templora_set_stream_sm_limit(self.stream, 0)


@pytest.mark.parametrize("limit", [1, 3])
@pytest.mark.parametrize("case", [
    ("bf16", 3, 3, 128, 700, 0, {}),                             # neighbouring row tiles of a head, six of them
    ("bf16", 2, 2, 64, 600, 70, dict(window=300)),               # five: the last tile of a pair is missing
    ("bf16", 4, 2, 128, 800, 0, dict(doc_offsets=[0, 90, 500, 510, 790], prefix_lens=[10, 200, 0, 100])),   # key tiles taken by their work
    ("bf16", 6, 3, 80, 500, 0, dict(doc_offsets=[0, 260, 500], softcap=10.0, causal=False)),
    ("f32", 2, 1, 64, 300, 0, {}),
], ids=lambda c: "-".join(str(x) for x in c[:6]) + "".join(sorted(c[6])))
def test_plans_for_more_ctas_than_sms(b, case, limit):
    host = make(case)
    c = Call(b, case, host)
    with few_sms(b, limit):
        c.forward()
        c.backward()
    c.check()
    check_forward(case, host, c.o, c.lse)
    check_backward(case, host, c.o.cpu(), c.dq, c.dk, c.dv)


@pytest.mark.parametrize("case", [
    ("bf16", 40, 40, 64, 1024, 0, {}),                           # the 13B block's heads: 160 forward, 320 backward CTAs
    ("bf16", 48, 24, 64, 900, 0, dict(doc_offsets=[0, 300, 310, 880], prefix_lens=[100, 0, 50])),           # 192 key tiles by their work
    ("f32", 16, 16, 64, 1000, 0, {}),
], ids=lambda c: "-".join(str(x) for x in c[:6]) + "".join(sorted(c[6])))
def test_several_waves_of_ctas(b, case):
    host = make(case)
    c = Call(b, case, host)
    c.forward()
    c.backward()
    c.check()
    check_forward(case, host, c.o, c.lse)
    check_backward(case, host, c.o.cpu(), c.dq, c.dk, c.dv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_query_tiles_than_have_a_bit(b, dtype):
    """Half a million rows and some: the rows around the last tile with a bit, the first and the last, as calls of their own."""
    T, D, w = 524288 + 300, 16, 64
    case = (dtype, 1, 1, D, T, 0, dict(window=w))
    host = make(case)
    c = Call(b, case, host)
    c.forward()
    c.backward()
    c.check()
    for t in (c.o, c.lse, c.dq, c.dk, c.dv):
        assert torch.isfinite(t).all()
    for first, end in ((w - 1, 300), (262144 - 100, 262144 + 200), (524288 - 200, 524288 + 180), (T - 200, T)):
        ctx = w - 1                                              # the rows' keys begin that much ahead of them
        rows, keys = slice(first, end), slice(first - ctx, end)
        part = dict(q=host["q"][rows], k=host["k"][keys], v=host["v"][keys], do=host["do"][rows])
        sub = (dtype, 1, 1, D, end - first, ctx, dict(window=w))
        o = c.o[rows].cpu()
        check_forward(sub, part, o, c.lse[:, rows])
        # keys whose rows are all among these
        whole = slice(ctx, end - first + ctx - (0 if end == T else ctx))
        check_backward(sub, part, o, c.dq[rows], c.dk[keys], c.dv[keys], k_rows=whole)


@pytest.mark.parametrize("case", [("bf16", 4, 2, 64, 200, 30, {}), ("f32", 4, 2, 64, 70, 30, dict(softcap=10.0)), ("bf16", 2, 1, 128, 300, 1000, {})],
                         ids=lambda c: "-".join(str(x) for x in c[:6]) + "".join(sorted(c[6])))
def test_rows_at_odd_distances(b, case):
    """Row strides that are no multiple of 16 bytes, another one for each tensor."""
    dtype, H, Hkv, D, Tq, ctx, masks = case
    host = make(case)
    c = Call(b, case, host)

    def odd(n, heads, extra, data=None):
        pitch = heads * D + extra
        buf = c.guard.empty((n * pitch,), DT[dtype], 7.0)
        view = buf.as_strided((n, heads, D), (pitch, D, 1))
        if data is not None:
            view.copy_(data)
        return view, buf.view(n, pitch)[:, heads * D:]

    Tk = Tq + ctx
    made = {n: odd(*spec) for n, spec in dict(q=(Tq, H, 1, host["q"]), k=(Tk, Hkv, 3, host["k"]), v=(Tk, Hkv, 5, host["v"]), o=(Tq, H, 7),
                                              do=(Tq, H, 9, host["do"]), dq=(Tq, H, 11), dk=(Tk, Hkv, 13), dv=(Tk, Hkv, 1)).items()}
    t = {n: view for n, (view, _) in made.items()}
    c.args = b.AttentionArgs(c.desc, t["q"], t["k"], t["v"], t["o"], c.lse, q_start=ctx, do=t["do"], dq=t["dq"], dk=t["dk"], dv=t["dv"])
    c.forward()
    c.backward()
    c.check()
    check_forward(case, host, t["o"], c.lse)
    check_backward(case, host, t["o"].cpu(), t["dq"], t["dk"], t["dv"])
    assert all((rest == 7.0).all() for _, rest in made.values())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale, softcap", [(0.3, 1e-39), (-0.5, 1e-39), (2.0, 2e-38), (0.3, 1e-45)])
def test_zero_scores_under_the_smallest_caps(b, dtype, scale, softcap):
    """scale / softcap near and beyond the largest fp32 number: every score becomes 0, those of zero queries too."""
    case = (dtype, 2, 1, 64, 200, 30, {})
    host = make(case)
    host["q"][::3] = 0
    c = Call(b, case, host)
    c.desc = b.attention_desc(2, 1, 64, {"bf16": b.BF16, "f32": b.F32}[dtype], scale=scale, softcap=softcap)
    c.args = b.AttentionArgs(c.desc, c.dev["q"], c.dev["k"], c.dev["v"], c.o, c.lse, q_start=30)
    c.forward()
    c.check()
    v = f(host["v"])
    ref, ref_lse, P = orc.attention_fwd(f(host["q"]), f(host["k"]), v, float(np.float32(scale)), q_start=30, softcap=float(np.float32(softcap)))
    w = np.stack([P[h] @ np.abs(v[:, 0]) for h in range(2)], axis=1)
    near("o", f(c.o), ref, ((ROUND[dtype] if dtype == "bf16" else 0.0) + SLACK) * w + ROUND[dtype] * np.abs(ref))
    near("lse", f(c.lse), ref_lse, SLACK * (1 + np.abs(ref_lse)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [3e38, -3e38])
def test_zero_scores_under_the_largest_scales(b, dtype, scale):
    """Zero queries score 0 whatever the scale: the mean of the values they see."""
    case = (dtype, 2, 1, 64, 200, 30, {})
    host = make(case)
    host["q"][:] = 0
    c = Call(b, case, host)
    c.desc = b.attention_desc(2, 1, 64, {"bf16": b.BF16, "f32": b.F32}[dtype], scale=scale)
    c.args = b.AttentionArgs(c.desc, c.dev["q"], c.dev["k"], c.dev["v"], c.o, c.lse, q_start=30)
    c.forward()
    c.check()
    check_forward(case, host, c.o, c.lse)
