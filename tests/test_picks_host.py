"""Host side of tokens from logits and of clipping, no GPU needed: the definition that the GPU tests compare with against closed forms, workspace sizes, and refusals, which come before
anything is enqueued."""
import ctypes as C
import math

import numpy as np
import pytest

import picks

AT = 1 << 40       # an address that nothing is behind: whatever is refused does not touch it


@pytest.fixture(scope="module")
def tr():
    from paper_2504_07878_amd import tokroute
    tokroute.load_library()
    return tokroute


def test_the_definition_in_closed_forms():
    z = np.array([0.0, math.log(4.0), -np.inf, math.log(2.0), np.nan, math.log(2.0)])      # weights 1, 4, -, 2, -, 2: order 1, 3, 5, 0
    kept = lambda **how: picks.kept_of(z, *[(dict(t=1.0, k=0, p=1.0, m=0.0) | how)[x] for x in "tkpm"])[0].tolist()   # noqa: E731
    assert kept() == [1, 3, 5, 0] and kept(k=2) == [1, 3] and kept(k=9) == [1, 3, 5, 0] and kept(t=0.0) == [1]
    assert kept(p=0.4) == [1] and kept(p=0.5) == [1, 3] and kept(p=0.8) == [1, 3, 5] and kept(p=0.95) == [1, 3, 5, 0] and kept(p=0.0) == [1]
    assert kept(k=3, p=0.6) == [1, 3]                       # of 8: 4 are 0.5, 6 are 0.75
    assert kept(m=0.49) == [1, 3, 5] and kept(m=0.6) == [1] and kept(m=2.0) == [1]
    assert picks.kept_of(np.array([np.inf, 1.0, np.inf]), 1.0, 0, 1.0, 0.0)[1].tolist() == [1.0, 1.0, 0.0]
    for u, token in ((0.0, 0), (0.11, 0), (0.12, 1), (0.55, 1), (0.56, 3), (0.77, 3), (0.78, 5), (1.0, 5)):
        p = {0: 1, 1: 4, 3: 2, 5: 2}[token] / 9
        assert picks.check_draw(z, u, 1.0, 0, 1.0, 0.0, token, np.float32(math.log(p)))
        assert not picks.check_draw(z, u, 1.0, 0, 1.0, 0.0, token, math.log(p) * (1 + 1e-6))
        for other in {0, 1, 2, 3, 4, 5} - {token}:
            assert not picks.check_draw(z, u, 1.0, 0, 1.0, 0.0, other, math.log(p))
    assert picks.check_draw(np.full(3, -np.inf), 0.5, 1.0, 0, 1.0, 0.0, -1, 0.0)


def test_workspace_sizes(tr):
    size = lambda *c: tr.load_library().tr_pick_workspace_bytes(C.byref(tr.tr_pick_config(*c)))   # noqa: E731
    assert 0 < size(1, 1, tr.F32) <= size(64, 151936, tr.F32) < 64 << 20 and 0 < size(1 << 20, 1 << 20, tr.BF16) < 1 << 30
    for bad in ((0, 10, 0), (10, 0, 0), ((1 << 20) + 1, 10, 0), (10, (1 << 20) + 1, 0), (10, 10, 2), (10, 10, -1)):
        assert size(*bad) == 0
    assert tr.load_library().tr_pick_workspace_bytes(None) == 0 and 0 < tr.load_library().tr_grad_workspace_bytes() < 1 << 20


def test_draws_are_refused_before_anything_is_enqueued(tr):
    lib, cfg = tr.load_library(), tr.tr_pick_config(64, 1000, tr.F32)
    nbytes = lib.tr_pick_workspace_bytes(C.byref(cfg))
    good = dict(cfg=cfg, ws=AT, nbytes=nbytes, logits=AT, stride=1000, rows=8, u=AT, ts=None, ks=None, ps=None, ms=None, t=1.0, k=0, p=1.0, m=0.0, token=AT, logprob=AT, entries=4, ids=AT, values=AT)

    def call(name, **kw):
        d = good | kw
        rows = tr.tr_pick_rows(d["logits"], d["stride"], d["rows"])
        cfg = None if d["cfg"] is None else C.byref(d["cfg"])
        if name == "tr_top":
            return lib.tr_top(cfg, d["ws"], d["nbytes"], None, None if kw.get("no_rows") else C.byref(rows), d["entries"], d["ids"], d["values"])
        how = tr.tr_sample_how(d["u"], d["ts"], d["ks"], d["ps"], d["ms"], d["t"], d["k"], d["p"], d["m"])
        return lib.tr_sample(cfg, d["ws"], d["nbytes"], None, None if kw.get("no_rows") else C.byref(rows), None if kw.get("no_how") else C.byref(how), d["token"], d["logprob"])

    inf, nan = float("inf"), float("nan")
    for f in ("tr_sample", "tr_top"):
        for bad in (dict(cfg=None), dict(no_rows=True), dict(ws=None), dict(ws=AT + 16), dict(logits=None), dict(logits=AT + 2), dict(stride=999), dict(rows=-1)):
            assert call(f, **bad) == tr.ERR_INVALID_ARG, (f, bad)
        assert call(f, nbytes=nbytes - 1) == tr.ERR_CAPACITY and call(f, rows=65) == tr.ERR_CAPACITY
        assert call(f, cfg=tr.tr_pick_config(64, 1000, 5)) == tr.ERR_SHAPE
        assert call(f, rows=0) == tr.OK
    for bad in (dict(no_how=True), dict(u=None), dict(u=AT + 1), dict(token=None), dict(logprob=None), dict(token=AT + 2), dict(logprob=AT + 1), dict(ts=AT + 1), dict(ks=AT + 2), dict(ps=AT + 3), dict(ms=AT + 1),
                dict(t=-1.0), dict(t=nan), dict(k=-1), dict(p=1.01), dict(p=-0.1), dict(p=nan), dict(m=1.01), dict(m=-0.1), dict(m=nan)):
        assert call("tr_sample", **bad) == tr.ERR_INVALID_ARG, bad
    assert call("tr_sample", rows=0, t=inf) == tr.OK
    for bad in (dict(ids=None), dict(values=None), dict(ids=AT + 2), dict(values=AT + 2), dict(entries=0), dict(entries=-1)):
        assert call("tr_top", **bad) == tr.ERR_INVALID_ARG, bad
    assert call("tr_top", entries=1025) == tr.ERR_CAPACITY


def test_clipping_is_refused_before_anything_is_enqueued(tr):
    lib = tr.load_library()
    nbytes = lib.tr_grad_workspace_bytes()

    def call(grads, out, counts, dtypes, ws=AT, size=nbytes, max_norm=1.0, norm=AT, n=None):
        n = len(grads) if n is None else n
        arr = lambda t, x: None if x is None else (t * len(x))(*x)   # noqa: E731
        g, o, c, d = arr(C.c_void_p, grads), arr(C.c_void_p, out), arr(C.c_int64, counts), arr(C.c_int32, dtypes)
        clip = lib.tr_grad_clip(ws, size, None, n, g, o, c, d, max_norm, norm)
        return clip, None if out != grads else lib.tr_grad_norm(ws, size, None, n, g, c, d, norm)

    a, b = AT + (1 << 30), AT + (2 << 30)
    bad = tr.ERR_INVALID_ARG
    assert call([a], [a], [10], [0], ws=None) == call([a], [a], [10], [0], ws=AT + 8) == call([a], [a], [10], [0], norm=None) == call([a], [a], [10], [0], norm=AT + 2) == (bad, bad)
    assert call([a], [a], [10], [0], n=-1) == call([a + 2], [a + 2], [10], [0]) == call([a + 1], [a + 1], [10], [1]) == call([None], [None], [10], [0]) == (bad, bad)
    assert call([a], [a], [10], [0], size=nbytes - 1) == (tr.ERR_CAPACITY,) * 2
    assert call([a], [a], [-1], [0]) == call([a], [a], [(1 << 40) + 1], [0]) == call([a], [a], [1], [2]) == (tr.ERR_SHAPE,) * 2
    assert call([a], None, [10], [0])[0] == call([a], [None], [10], [0])[0] == call([a], [b + 2], [10], [0])[0] == bad
    for m in (-1.0, float("nan")):
        assert call([a], [a], [10], [0], max_norm=m)[0] == bad
    # what is written lies across something else of the call
    for grads, out, counts in (([a, a], [a, a], [10, 10]), ([a, a + 36], [a, a + 36], [10, 10]), ([a], [a + 4], [10]), ([a, b], [b, a], [10, 10]), ([a, b], [b + 4000, b], [10, 1001]),
                               ([a, b], [a + 4096, a + 4100], [2, 2]), ([a, a + 400, b], [a, a + 400, a + 396], [100, 100, 1])):
        assert call(grads, out, counts, [0] * len(grads))[0] == bad, (grads, out, counts)


@pytest.mark.parametrize("top_k, passed", [(7, 7), (np.int64(7), 7), (2**31, 2**31 - 1), (2**32 + 1, 2**31 - 1), (-2**32 + 1, -2**31)])
def test_numbers_beyond_32_bits_are_not_cut_off(tr, top_k, passed):
    import torch
    from paper_2504_07878_amd import sampling
    s = object.__new__(sampling.Sampler)                  # (without a GPU)
    s.dtype, s.device, s.cfg, s.lib, got = torch.float32, torch.device("cpu"), tr.tr_pick_config(4, 10, tr.F32), tr.load_library(), []
    s._call = lambda fn, what, rows, how, *out: got.append(how._obj.top_k)
    s.sample(torch.zeros(4, 10), torch.zeros(4), top_k=top_k)
    assert got == [passed]
    for entries in (1025, 2**32 + 1):
        with pytest.raises(tr.TokrouteError) as e:
            s.top(torch.zeros(0, 10), entries)
        assert e.value.code == tr.ERR_CAPACITY
    assert s._rows(torch.zeros(1, 10).expand(2**32 + 1, 10)).rows == 2**31 - 1       # more than any Sampler is for


def test_autograd_sees_what_is_written_over(tr):
    """A tensor that a graph has kept, and that a call has written over since, is no gradient of it any more: the backward pass says so, as after PyTorch's own calls."""
    import torch
    from types import SimpleNamespace
    from paper_2504_07878_amd import clipping, sampling
    cpu, noted = torch.device("cpu"), []                  # (without a GPU)
    c, s = object.__new__(clipping.Clipper), object.__new__(sampling.Sampler)
    c.device, c.lib = cpu, SimpleNamespace(tr_grad_clip=None)
    s.dtype, s.device, s.cfg, s.lib = torch.float32, cpu, tr.tr_pick_config(4, 10, tr.F32), SimpleNamespace(tr_sample=None, tr_top=None)
    c._call = s._call = lambda *a: noted.append(a)
    w, z, u = torch.ones(4, requires_grad=True), torch.zeros(4, 10), torch.zeros(4)
    wide = torch.ones(4, 3, requires_grad=True)
    calls = [(w, lambda t: c.clip([t], 1.0)), (w, lambda t: c.clip([torch.zeros(4)], 1.0, out=[t])), (w, lambda t: c.clip([None, t], 1.0)), (w, lambda t: s.sample(z, u, logprob=t)), (wide, lambda t: s.top(z, 3, values=t))]
    for x, write in calls:
        kept = torch.ones_like(x).detach()
        y = (x * kept).sum()
        write(kept)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    assert len(noted) == len(calls)
    with torch.inference_mode():
        c.clip([torch.ones(3)], 1.0)                      # (keeps no count)
    same = torch.ones(4)
    y = (w * same).sum()
    c.clip([same], 1.0, out=[torch.zeros(4)])             # what is only read is still what it was
    y.backward()
