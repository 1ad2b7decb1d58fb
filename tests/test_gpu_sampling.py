"""Tokens drawn from logits and a row's largest logits, against their definition in 64 bits (picks.py): sizes, types, ties, masks, settings, streams, graphs, refusals."""
import numpy as np
import pytest
import torch

import picks

pytestmark = pytest.mark.gpu
SIZES = (1, 2, 7, 63, 65, 255, 1000, 2049, 4096, 5003, 16384, 16385, 40001, 151936, 152064)
SETTINGS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=5), dict(top_k=50, temperature=0.8), dict(top_p=0.9), dict(top_p=0.5, temperature=1.3), dict(min_p=0.05),
            dict(top_k=40, top_p=0.95, min_p=0.02, temperature=0.6), dict(temperature=0.0), dict(top_p=0.0), dict(min_p=1.0), dict(top_k=1000, top_p=0.999),
            dict(top_p=0.95, min_p=0.02), dict(top_p=0.999, min_p=0.2), dict(top_p=0.9999, min_p=0.001), dict(top_k=700, min_p=0.05), dict(top_k=3000, min_p=0.02), dict(top_k=700, top_p=0.99, min_p=0.01)]
NAMES = ("temperature", "top_k", "top_p", "min_p")
NONE = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)


@pytest.fixture(scope="module")
def sampling():
    from paper_2504_07878_amd import sampling
    return sampling


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def logits_of(kind, n, v, seed, dtype=torch.float32):
    """peaked: a body and a few tokens far above it; flat: a body alone; ties: whole numbers; equal: one value; steep: falling by id, so that the largest lie together."""
    g = rng(seed)
    z = torch.randn((n, v), device="cuda", generator=g)
    if kind == "peaked":
        z = z * 2.2
        z.scatter_add_(1, torch.randint(0, v, (n, 40), device="cuda", generator=g), 6 + 14 * torch.rand((n, 40), device="cuda", generator=g))
    elif kind == "ties":
        z = (z * 2).round()
    elif kind == "equal":
        z = torch.full_like(z, -3.25)
    elif kind == "steep":
        z = z * 0.01 - torch.arange(v, device="cuda") * (20.0 / v)
    return z.to(dtype)


def as_row(value, n, i):
    return value[i].item() if isinstance(value, torch.Tensor) else value


def check(z, u, how, token, logprob):
    z, u, token, logprob = z.float().cpu().numpy(), u.cpu().numpy(), token.cpu().numpy(), logprob.cpu().numpy()
    how = NONE | how
    for i in range(len(z)):
        t, k, p, m = (as_row(how[x], len(z), i) for x in NAMES)
        t, p, m = (float(np.float32(x)) for x in (t, p, m))
        assert picks.check_draw(z[i], u[i], t, k, p, m, token[i], logprob[i]), (i, t, k, p, m, u[i], token[i], logprob[i])


@pytest.mark.parametrize("how", SETTINGS, ids=[",".join(f"{k}{v}" for k, v in h.items()) or "none" for h in SETTINGS])
@pytest.mark.parametrize("kind", ["peaked", "flat", "ties", "equal", "steep"])
def test_draws_of_a_small_and_a_large_vocabulary(sampling, kind, how):
    for n, v in ((9, 1003), (5, 40001)):
        z, u = logits_of(kind, n, v, 11), torch.rand(n, device="cuda", generator=rng(12))
        check(z, u, how, *sampling.Sampler(n, v).sample(z, u, **how))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", SIZES)
def test_every_size(sampling, v, dtype):
    n = 4
    s = sampling.Sampler(n, v, dtype)
    for kind, how in (("peaked", dict(top_k=20, top_p=0.9)), ("flat", dict(top_p=0.9)), ("ties", dict(min_p=0.02)), ("flat", {}), ("steep", dict(top_p=0.8, temperature=0.5))):
        z, u = logits_of(kind, n, v, v, dtype), torch.rand(n, device="cuda", generator=rng(v + 1))
        check(z, u, how, *s.sample(z, u, **how))
        for k in {1, min(v, 17), min(v, 300)}:
            check_top(z, k, *s.top(z, k))


def check_top(z, k, ids, values):
    z = z.float().cpu().numpy()
    for i, (row, got) in enumerate(zip(ids.cpu().numpy(), values.cpu().numpy())):
        want = picks.order_of(z[i])[:k]
        assert np.array_equal(row, np.concatenate([want, np.full(k - len(want), -1)])), i
        assert np.array_equal(got, np.concatenate([z[i][want], np.full(k - len(want), -np.inf, np.float32)])), i


@pytest.mark.parametrize("k", [1, 2, 16, 63, 64, 65, 200, 777, 1024])
@pytest.mark.parametrize("kind", ["peaked", "flat", "ties", "equal", "steep"])
def test_the_largest_logits_in_order(sampling, kind, k):
    for n, v in ((3, 500), (3, 30011), (2, 151936)):
        z = logits_of(kind, n, v, 21)
        check_top(z, k, *sampling.Sampler(n, v).top(z, k))


def masked(v):
    """Rows that a mask leaves little or nothing of, and what must not be in the way of the rest."""
    inf, nan = float("inf"), float("nan")
    z = logits_of("peaked", 12, v, 31)
    z[0] = -inf                                   # nothing
    z[1] = nan
    z[2] = torch.finfo(torch.float32).min         # the type's lowest value is a logit like any other
    z[3] = -inf
    z[3, v - 1] = -70.0                           # one
    z[4, ::2] = -inf
    z[5, 1::2] = nan
    z[6] = torch.finfo(torch.float32).min         # a mask with the lowest value
    z[6, v // 2:v // 2 + 3] = torch.tensor([1.0, 2.0, 3.0], device="cuda")[:z[6, v // 2:v // 2 + 3].numel()]
    z[7, v // 3] = inf
    z[7, v // 2] = inf
    z[8] = inf
    z[9] = torch.finfo(torch.float32).max
    z[9, v // 2:] = torch.finfo(torch.float32).min
    z[10] = 0.0
    z[10, ::3] = -0.0                             # the same logit
    z[11] *= 1e-38                                # subnormal ones among them
    return z


@pytest.mark.parametrize("v", [5, 3001, 40001])
@pytest.mark.parametrize("how", SETTINGS, ids=[",".join(f"{k}{v}" for k, v in h.items()) or "none" for h in SETTINGS])
def test_masks_infinities_and_nan(sampling, v, how):
    z = masked(v)
    u = torch.rand(len(z), device="cuda", generator=rng(32))
    s = sampling.Sampler(len(z), v)
    check(z, u, how, *s.sample(z, u, **how))
    for k in (1, 4, 100):
        check_top(z, k, *s.top(z, k))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v, pad", [(8193, 1), (30011, 0), (151936, 3)])
def test_large_logits_that_lie_together(sampling, v, pad, dtype):
    """Runs of neighbouring ids that are far above the rest, one run or several, longer and shorter than top-k, at the row's ends too; in one row at equal logits."""
    z = logits_of("flat", 8, v + pad, 41)[:, :v]
    for row, (begin, length) in enumerate(((0, 30), (v - 40, 40), (v // 2, 300), (77, 1500), (v // 3, 4000), (0, v), (v // 2, 700), (v // 4, 256))):
        z[row, begin:begin + length] += 9
    z[6, v // 2:v // 2 + 700] = 9.5
    z[7, v // 2:v // 2 + 256] += 20
    z[7, v - 300:] += 7
    z, u = z.to(dtype), torch.rand(8, device="cuda", generator=rng(42))
    s = sampling.Sampler(8, v, dtype)
    for k in (5, 50, 400, 1000):
        for how in (dict(top_k=k), dict(top_k=k, top_p=0.9, temperature=2.0), dict(top_k=torch.full((8,), k, dtype=torch.int32, device="cuda"), top_p=0.95, min_p=0.01)):
            check(z, u, how, *s.sample(z, u, **how))
        check_top(z, k, *s.top(z, k))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v, left", [(2153, 0.3), (30843, 0.01), (30092, 0.02), (151936, 0.005)])
def test_few_tokens_among_masked_ones(sampling, v, left, dtype):
    """Most of a row is -inf, some of the rest the type's lowest value: the tokens that are left lie in a vanishing part of the row's range, on both sides of 0."""
    n, s = 6, sampling.Sampler(6, v, dtype)
    for kind in ("flat", "peaked", "ties"):
        z, g = logits_of(kind, n, v, 35, dtype), rng(36)
        z = z.masked_fill(torch.rand((n, v), device="cuda", generator=g) > left, float("-inf"))
        z[:, ::3] = torch.finfo(dtype).min
        u = torch.rand(n, device="cuda", generator=g)
        for how in (dict(top_p=0.9), dict(top_p=0.9, temperature=5.0), dict(top_k=50), dict(top_k=300, top_p=0.99), dict(min_p=0.01), dict()):
            check(z, u, how, *s.sample(z, u, **how))
        for k in (50, 300):
            check_top(z, k, *s.top(z, k))


@pytest.mark.parametrize("v", [1003, 40001])
def test_settings_of_their_own_for_every_row(sampling, v):
    t = torch.tensor([0.0, 1e-30, 0.5, 1.0, 1.5, float("inf"), -1.0, float("nan"), 1.0, 1.0, 1.0, 1.0, 1.0, 1.0], device="cuda")
    k = torch.tensor([0, 0, 3, 0, 40, 0, 0, 0, -5, 1 << 30, v, 0, 0, 0], dtype=torch.int32, device="cuda")
    p = torch.tensor([1.0, 1.0, 0.9, 0.3, 1.0, 1.0, 1.0, 1.0, float("nan"), 2.0, 1.0, -1.0, 1.0, 1.0], device="cuda")
    m = torch.tensor([0.0, 0.0, 0.0, 0.0, 0.1, 0.0, 0.0, 0.0, 0.0, 0.0, float("nan"), 0.0, 2.0, -1.0], device="cuda")
    n = len(t)
    how = dict(temperature=t, top_k=k, top_p=p, min_p=m)
    s = sampling.Sampler(n, v)
    for kind in ("peaked", "flat", "ties"):
        z, u = logits_of(kind, n, v, 41), torch.rand(n, device="cuda", generator=rng(42))
        check(z, u, how, *s.sample(z, u, **how))


@pytest.mark.parametrize("v", [1, 6, 1000, 40001])
@pytest.mark.parametrize("how", [dict(), dict(top_k=3), dict(top_p=0.9)])
def test_random_numbers_at_the_ends(sampling, v, how):
    u = torch.tensor([0.0, 2.0 ** -24, 1 - 2.0 ** -24, 1.0, 7.0, -1.0, float("nan"), -0.0], device="cuda")
    for kind in ("flat", "equal"):
        z = logits_of(kind, len(u), v, 51)
        check(z, u, how, *sampling.Sampler(len(u), v).sample(z, u, **how))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", [1000, 40001, 151936])
def test_numbers_at_the_ends_draw_nothing_without_weight(sampling, v, dtype):
    """0 and numbers that 32 bits round to 1: at low temperatures nearly all tokens have no weight that 64 bits hold beside the largest, the first and the last ids too."""
    u = torch.tensor([0.0, 1e-20, 2.0 ** -24, 1 - 2.0 ** -24, 1.0, 5.0], device="cuda")
    z, s = (2 * logits_of("flat", 1, v, 52)).to(dtype).expand(len(u), v), sampling.Sampler(len(u), v, dtype)
    for t in (1.0, 0.1, 0.01, 1e-3, 1e-30):
        check(z, u, dict(temperature=t), *s.sample(z.contiguous(), u, temperature=t))


def test_equal_logits_are_drawn_by_place(sampling):
    """All weights are 1: u takes the token at floor(u V), and filters keep the lowest ids."""
    v = 40000
    z = torch.full((5, v), 2.5, device="cuda")
    u = torch.tensor([0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24], device="cuda")
    s = sampling.Sampler(5, v)
    at = (u.double() * v).long().cpu()
    assert torch.equal(s.sample(z, u)[0].cpu().long(), at)
    assert torch.equal(s.sample(z, u, top_p=0.5)[0].cpu().long(), (u.double() * (v // 2)).long().cpu())
    assert torch.equal(s.sample(z, u, top_k=100)[0].cpu().long(), (u.double() * 100).long().cpu())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", [1001, 33333])
def test_strides_alignment_and_what_lies_beside_the_rows(sampling, v, dtype):
    """Rows that begin at any element, NaN between them; nothing but the outputs is written."""
    n = 5
    for pad, skip in ((0, 1), (1, 3), (7, 0), (13, 5)):
        buf = torch.full((n * (v + pad) + skip + 16,), float("nan"), device="cuda", dtype=dtype)
        z = buf[skip:skip + n * (v + pad)].view(n, v + pad)[:, :v]
        z.copy_(logits_of("peaked", n, v, 61, dtype))
        before = buf.clone()
        u = torch.rand(n, device="cuda", generator=rng(62))
        out, lp = torch.full((n + 2,), 77, dtype=torch.int32, device="cuda"), torch.full((n + 2,), 77.0, device="cuda")
        s = sampling.Sampler(n, v, dtype)
        s.sample(z, u, top_p=0.9, token=out[1:-1], logprob=lp[1:-1])
        check(z, u, dict(top_p=0.9), out[1:-1], lp[1:-1])
        assert out[0] == out[-1] == 77 and lp[0] == lp[-1] == 77
        check_top(z, 9, *s.top(z, 9))
        assert torch.equal(buf.view(torch.int16 if dtype == torch.bfloat16 else torch.int32), before.view(torch.int16 if dtype == torch.bfloat16 else torch.int32))


def test_the_same_row_every_time(sampling):
    """A row's token does not depend on which rows are beside it, on how often it is asked for, or on the sampler."""
    v, n = 40001, 33
    z, u = torch.cat([logits_of("peaked", 17, v, 71), logits_of("flat", 16, v, 72)]), torch.rand(33, device="cuda", generator=rng(73))
    for how in (dict(), dict(top_p=0.9), dict(top_k=30), dict(min_p=0.1, temperature=1.4)):
        s = sampling.Sampler(n, v)
        token, lp = s.sample(z, u, **how)
        for _ in range(3):
            again, lp2 = s.sample(z, u, **how)
            assert torch.equal(token, again) and torch.equal(lp, lp2)
        back, lp3 = sampling.Sampler(n + 7, v).sample(z.flip(0), u.flip(0), **how)
        assert torch.equal(token, back.flip(0)) and torch.equal(lp, lp3.flip(0))
        one = torch.cat([s.sample(z[i:i + 1], u[i:i + 1], **how)[0] for i in range(0, n, 8)])
        assert torch.equal(one, token[::8])


def test_draws_are_distributed_as_the_weights_are(sampling):
    """Numbers in steps of 1 / N draw each token as often as its share of N, give or take one at either end of its stretch."""
    v, n = 50, 4096
    z = logits_of("peaked", 1, v, 81).expand(n, v).contiguous()
    u = (torch.arange(n, device="cuda") + 0.5) / n
    token, _ = sampling.Sampler(n, v).sample(z, u, temperature=2.0, top_p=0.95)
    kept, w = picks.kept_of(z[0].cpu().numpy(), 2.0, 0, float(np.float32(0.95)), 0.0)
    count = np.bincount(token.cpu().numpy(), minlength=v)
    assert set(np.flatnonzero(count)) <= set(kept.tolist())
    assert (np.abs(count[kept] - w / w.sum() * n) <= 1.0).all()


def test_other_streams_and_graphs(sampling):
    """Captured once, replayed on other logits between eager calls of another sampler; two graphs of one sampler, one after the other."""
    n, v = 6, 40001
    s, other = sampling.Sampler(n, v), sampling.Sampler(n, v)
    z, u = logits_of("peaked", n, v, 91), torch.rand(n, device="cuda", generator=rng(92))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        token, lp = s.sample(z, u, top_p=0.9)
    torch.cuda.current_stream().wait_stream(side)
    check(z, u, dict(top_p=0.9), token, lp)
    graphs, outs = [], []
    for how in (dict(top_p=0.9), dict()):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(s.sample(z, u, **how) + s.top(z, 7))
        graphs.append(g)
    for step in range(4):
        z.copy_(logits_of(("peaked", "flat", "ties", "steep")[step], n, v, 93 + step))
        u.copy_(torch.rand(n, device="cuda", generator=rng(97 + step)))
        for g, how, (token, lp, ids, values) in zip(graphs, (dict(top_p=0.9), dict()), outs):
            g.replay()
            eager = other.sample(z, u, **how)
            torch.cuda.synchronize()
            assert torch.equal(token, eager[0]) and torch.equal(lp, eager[1])
            check(z, u, how, token, lp)
            check_top(z, 7, ids, values)


def test_no_rows(sampling):
    s = sampling.Sampler(4, 77)
    z, u = torch.zeros((0, 77), device="cuda"), torch.zeros(0, device="cuda")
    assert s.sample(z, u)[0].shape == (0,) and s.top(z, 3)[0].shape == (0, 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n, v", [(3000, 77), (1030, 9000), (600, 20001), (300, 40003)])
def test_many_rows(sampling, n, v, dtype):
    """More than one launch takes, and more than one wavefront of 1024 tokens each for all of them."""
    s, some = sampling.Sampler(n, v, dtype), slice(n % 7, None, 41)
    for kind, how in (("peaked", dict(top_k=9, top_p=0.8)), ("flat", dict(top_p=0.9)), ("flat", {}), ("ties", dict(min_p=0.05)), ("peaked", dict(top_p=0.95, temperature=1.2))):
        z, u = logits_of(kind, n, v, 101, dtype), torch.rand(n, device="cuda", generator=rng(102))
        token, lp = s.sample(z, u, **how)
        check(z[some], u[some], how, token[some], lp[some])
    ids, values = s.top(z, 33)
    check_top(z[some], 33, ids[some], values[some])


def test_a_long_row(sampling):
    v = 1 << 20
    z, u = torch.cat([logits_of("flat", 1, v, 111), logits_of("peaked", 1, v, 112)]), torch.tensor([0.37, 0.81], device="cuda")
    s = sampling.Sampler(2, v)
    for how in (dict(), dict(top_p=0.9), dict(top_k=500, min_p=0.01)):
        check(z, u, how, *s.sample(z, u, **how))
    check_top(z, 1000, *s.top(z, 1000))


def test_offsets_past_32_bits(sampling):
    """Rows 2^30 elements apart: the third begins past 2^31 elements and 2^32 bytes."""
    v, far = 1500, 1 << 30
    buf = torch.empty(2 * far + v, dtype=torch.bfloat16, device="cuda")
    z = buf.as_strided((3, v), (far, 1))
    z.copy_(logits_of("peaked", 3, v, 121, torch.bfloat16))
    u = torch.rand(3, device="cuda", generator=rng(122))
    s = sampling.Sampler(3, v, torch.bfloat16)
    check(z, u, dict(top_p=0.9), *s.sample(z, u, top_p=0.9))
    check_top(z, 5, *s.top(z, 5))


def test_refusals(sampling):
    from paper_2504_07878_amd import tokroute
    s = sampling.Sampler(4, 100)
    z, u = torch.zeros((4, 100), device="cuda"), torch.zeros(4, device="cuda")
    for bad in (z.bfloat16(), z[:, :99], z.cpu(), z[0], z.t().contiguous().t()):
        with pytest.raises(ValueError):
            s.sample(bad, u)
        with pytest.raises(ValueError):
            s.top(bad, 3)
    for bad in (u[:3], u.double(), u.cpu(), torch.zeros(8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            s.sample(z, bad)
    for how in (dict(top_k=torch.zeros(4, device="cuda")), dict(temperature=torch.ones(3, device="cuda")), dict(token=torch.zeros(4, device="cuda")), dict(logprob=torch.zeros(5, device="cuda"))):
        with pytest.raises(ValueError):
            s.sample(z, u, **how)
    for how in (dict(temperature=-1.0), dict(temperature=float("nan")), dict(top_k=-1), dict(top_p=1.5), dict(top_p=-0.1), dict(top_p=float("nan")), dict(min_p=2.0), dict(min_p=-1.0)):
        with pytest.raises(tokroute.TokrouteError) as e:
            s.sample(z, u, **how)
        assert e.value.code == tokroute.ERR_INVALID_ARG
    with pytest.raises(tokroute.TokrouteError) as e:
        s.sample(torch.zeros((5, 100), device="cuda"), torch.zeros(5, device="cuda"))
    assert e.value.code == tokroute.ERR_CAPACITY
    for k, code in ((0, tokroute.ERR_INVALID_ARG), (1025, tokroute.ERR_CAPACITY)):
        with pytest.raises(tokroute.TokrouteError) as e:
            s.top(z, k)
        assert e.value.code == code
    for rows, v, dtype in ((0, 10, torch.float32), (1, 0, torch.float32), (1, (1 << 20) + 1, torch.float32), ((1 << 20) + 1, 8, torch.float32)):
        with pytest.raises(tokroute.TokrouteError):
            sampling.Sampler(rows, v, dtype)
    with pytest.raises(ValueError):
        sampling.Sampler(1, 10, torch.float16)
