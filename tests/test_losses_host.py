"""Host side of the losses over the vocabulary, no GPU needed: workspace sizes, and refusals, which come before anything is enqueued."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def tr():
    from paper_2504_07878_amd import tokroute
    tokroute.load_library()
    return tokroute


def cfg(tr, **kw):
    d = dict(max_rows=64, dim=896, vocab=151936, hidden_dtype=tr.BF16, weight_dtype=tr.BF16, max_entries=16) | kw
    return tr.tr_loss_config(*[d[k] for k in ("max_rows", "dim", "vocab", "hidden_dtype", "weight_dtype", "max_entries")])


def size(tr, **kw):
    return tr.load_library().tr_loss_workspace_bytes(C.byref(cfg(tr, **kw)))


def test_workspace_holds_pieces_and_not_the_logits(tr):
    """8192 rows of 151936 logits would be 2.5 GB in bf16 and 5 GB in fp32; the pieces stay at half a gigabyte."""
    assert 0 < size(tr) < 400 << 20
    assert size(tr, max_rows=8192) < 1200 << 20
    assert size(tr, max_rows=8192) > size(tr, max_rows=1024) > 0
    assert size(tr, hidden_dtype=tr.F32) > 0 and size(tr, hidden_dtype=tr.F32, weight_dtype=tr.F32) > 0
    assert size(tr, max_rows=1, dim=1, vocab=1, max_entries=1) > 0
    for rows, dim, vocab in ((1 << 20, 64, 1000), (256, 65536, 300), (1, 8, 1 << 24)):
        assert size(tr, max_rows=rows, dim=dim, vocab=vocab) > 0


def test_configurations_that_are_not_supported(tr):
    for bad in (dict(max_rows=0), dict(max_rows=(1 << 20) + 1), dict(dim=0), dict(dim=65537), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(hidden_dtype=7), dict(weight_dtype=-1),
                dict(weight_dtype=tr.F32), dict(max_entries=0), dict(max_entries=1025)):
        assert size(tr, **bad) == 0, bad
    assert tr.load_library().tr_loss_workspace_bytes(None) == 0


def test_calls_are_refused_before_anything_is_enqueued(tr):
    """Addresses that nothing is behind: whatever is refused does not touch them."""
    lib, c = tr.load_library(), cfg(tr)
    at, n = 1 << 40, size(tr)
    good = dict(hidden=at, weight=at, hidden_stride=896, weight_stride=896, ids=at, teacher=at, rows=8, entries=4, temperature=1.0)

    def call(name, config=c, ws=at, nbytes=n, out=at, **kw):
        d = good | kw
        rows = tr.tr_loss_rows(*[d[k] for k in ("hidden", "weight", "hidden_stride", "weight_stride", "ids", "teacher", "rows", "entries", "temperature")])
        if name.endswith("_grad"):
            g = tr.tr_loss_grads(kw.get("dh", at), kw.get("dw", at), kw.get("dhs", 896), kw.get("dws", 896))
            return getattr(lib, name)(C.byref(config), ws, nbytes, None, C.byref(rows), kw.get("lse", at), kw.get("grad", at), C.byref(g) if not kw.get("no_out") else None)
        return getattr(lib, name)(C.byref(config), ws, nbytes, None, C.byref(rows), out, kw.get("lse", at))

    every = ("tr_cross_entropy", "tr_distill", "tr_cross_entropy_grad", "tr_distill_grad")
    for f in every:
        for bad in (dict(ws=None), dict(ws=at + 16), dict(hidden=None), dict(weight=None), dict(ids=None), dict(hidden_stride=895), dict(weight_stride=1), dict(rows=-1), dict(hidden=at + 1),
                    dict(weight=at + 1), dict(lse=None)):
            assert call(f, **bad) == tr.ERR_INVALID_ARG, (f, bad)
        assert call(f, nbytes=n - 1) == tr.ERR_CAPACITY and call(f, rows=65) == tr.ERR_CAPACITY
        assert call(f, config=cfg(tr, dim=0)) == tr.ERR_SHAPE
    for f in ("tr_distill", "tr_distill_grad"):
        for bad in (dict(teacher=None), dict(entries=0), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf"))):
            assert call(f, **bad) == tr.ERR_INVALID_ARG, (f, bad)
        assert call(f, entries=17) == tr.ERR_CAPACITY
    for f in ("tr_cross_entropy", "tr_distill"):
        assert call(f, out=None) == tr.ERR_INVALID_ARG
        assert call(f, rows=0) == tr.OK                      # nothing to do
    for f in ("tr_cross_entropy_grad", "tr_distill_grad"):
        for bad in (dict(grad=None), dict(no_out=True), dict(dhs=895), dict(dws=895), dict(dh=at + 1), dict(dw=at + 1)):
            assert call(f, **bad) == tr.ERR_INVALID_ARG, (f, bad)
        assert call(f, dh=None, dw=None) == tr.OK            # nothing asked for


@pytest.mark.skipif(torch.cuda.is_available(), reason="needs a machine without a GPU")
def test_binding_raises_without_a_gpu():
    from paper_2504_07878_amd import losses
    with pytest.raises(RuntimeError, match="no CPU path"):
        losses.VocabLoss(8, 64, 100)


def test_calls_run_with_the_workspaces_device_current(tr, monkeypatch):
    """A default stream is the current device's: every call makes the workspace's current, and only for its time. (Tensors of this machine's memory, and calls that only look at the device.)"""
    from contextlib import contextmanager

    from paper_2504_07878_amd import losses
    now, seen = ["another"], []

    @contextmanager
    def device(d):
        before, now[0] = now[0], d
        yield
        now[0] = before

    def look(*args):
        seen.append(now[0])
        return tr.OK

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(losses.VocabLoss, "_matrix", lambda self, t, *_: t.stride(0))
    monkeypatch.setattr(losses.VocabLoss, "_flat", lambda self, t, *_: t)
    monkeypatch.setattr(losses.VocabLoss, "_stream", lambda self: seen.append(now[0]))
    plan = object.__new__(losses.VocabLoss)
    plan.cfg, plan.workspace, plan.hidden_dtype, plan.weight_dtype = cfg(tr, dim=4, vocab=6), torch.empty(64, dtype=torch.uint8), torch.float32, torch.float32
    plan.lib = type("Calls", (), {n: staticmethod(look) for n in ("tr_cross_entropy", "tr_cross_entropy_grad", "tr_distill", "tr_distill_grad")})
    h, w, ids, x, row = torch.zeros(3, 4), torch.zeros(6, 4), torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, 2), torch.zeros(3)
    plan.cross_entropy(h, w, ids[:, 0])
    plan.cross_entropy_grad(h, w, ids[:, 0], row, row)
    plan.distill(h, w, ids, x)
    plan.distill_grad(h, w, ids, x, 1.0, row, row)
    assert seen == [plan.workspace.device] * 8 and now == ["another"]
