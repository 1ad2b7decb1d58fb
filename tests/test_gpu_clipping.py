"""The length of many gradients together and its clipping, against their definition in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}    # half a step of a rounding


@pytest.fixture(scope="module")
def clipping():
    from paper_2504_07878_amd import clipping
    return clipping


def some(sizes, dtypes, seed=1, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(s, device="cuda", generator=g) * scale * 10.0 ** (i % 5 - 2)).to(dtypes[i % len(dtypes)]) for i, s in enumerate(sizes)]


def length(grads):
    return float(np.sqrt(sum((t.double().cpu().numpy() ** 2).sum() for t in grads)))


def check(grads, before, norm, max_norm):
    """The norm is a 64-bit sum, rounded to fp32; max_norm is handed over in fp32, the scale is rounded to it, and each product, which is then rounded to its type."""
    want = length(before)
    assert norm.shape == () and abs(float(norm) - want) <= 2.0 ** -23 * want
    by = min(1.0, max_norm / want) if want else 1.0
    for a, b in zip(grads, before):
        x = b.double() * by
        off = (a.double() - x).abs()
        tiny = torch.finfo(a.dtype).tiny * EPS[a.dtype] * 2
        assert (off <= x.abs() * ((EPS[a.dtype] if a.dtype != torch.float32 else 0) + 3.1 * EPS[torch.float32]) + tiny).all()
        if by == 1.0:
            assert torch.equal(a, b)


SETS = {"one": [1], "empty": [0, 5, 0], "few": [(3, 5), 7, 8, 9], "tile": [8191, 8192, 8193, 1], "odd": [(1001, 77), 33, (5, 5, 5), 100003], "many": [(i % 37 + 1,) for i in range(500)],
        "large": [(4096, 896), 896, (151936, 64)]}


@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.bfloat16,), (torch.bfloat16, torch.float32)], ids=["f32", "bf16", "both"])
@pytest.mark.parametrize("name", SETS)
def test_norm_and_clipping(clipping, name, dtypes):
    grads = some(SETS[name], dtypes)
    c = clipping.Clipper()
    check(grads, grads, c.norm(grads), float("inf"))
    for max_norm in (0.0, 0.37, length(grads) * 0.999, length(grads) * 1.001, float("inf")):
        mine, out = [t.clone() for t in grads], [torch.full_like(t, 7) for t in grads]
        check(mine, grads, c.clip(mine, max_norm), max_norm)
        norm = c.clip(grads, max_norm, out=out)
        check(out, grads, norm, max_norm)
        assert all(torch.equal(a, b) for a, b in zip(mine, out))


def test_no_gradients(clipping):
    c = clipping.Clipper()
    assert float(c.norm([])) == 0 and float(c.norm([None])) == 0 and float(c.clip([None, torch.zeros(0, device="cuda")], 1.0)) == 0
    zeros = [torch.zeros(100, device="cuda")]
    assert float(c.clip(zeros, 0.0)) == 0 and not zeros[0].any()


@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e18, 1e30])
def test_lengths_whose_squares_leave_the_range_of_32_bits(clipping, scale):
    grads = some([(300, 70), 11], (torch.float32, torch.bfloat16), scale=scale)
    mine = [t.clone() for t in grads]
    check(mine, grads, clipping.Clipper().clip(mine, length(grads) / 3), length(grads) / 3)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_gradients_that_are_not_finite_stay_as_they_are(clipping, bad):
    grads = some([(300, 70), 11], (torch.float32, torch.bfloat16))
    grads[1][3] = bad
    mine = [t.clone() for t in grads]
    norm = clipping.Clipper().clip(mine, 0.5)
    assert torch.equal(norm.cpu(), torch.tensor(float("inf"))) if bad == bad else norm.isnan()
    assert all(torch.equal(a.nan_to_num(5.0), b.nan_to_num(5.0)) for a, b in zip(mine, grads))


def test_gradients_whose_norm_is_beyond_32_bits_stay_as_they_are(clipping):
    """100 elements of 2^127 are 2^130 long: the norm that the call reports is infinite."""
    grads = [torch.full((100,), 2.0 ** 127, device="cuda"), torch.ones(33, device="cuda", dtype=torch.bfloat16)]
    mine, out, c = [t.clone() for t in grads], [torch.full_like(t, 7) for t in grads], clipping.Clipper()
    assert float(c.clip(mine, 1.0)) == float(c.clip(grads, 1.0, out=out)) == float("inf")
    assert all(torch.equal(a, b) and torch.equal(a, x) for a, b, x in zip(mine, out, grads))


@pytest.mark.parametrize("max_norm, size", [(1e-8, 1e37), (1e-30, 1e15), (3e-38, 2e30), (1e-44, 1e36)])
def test_scales_below_what_32_bits_hold(clipping, max_norm, size):
    """max_norm / norm is subnormal in 32 bits, or zero, where the products are not. Results below 2^-126 are off by half of 2^-149 (bfloat16: 2^-133) twice at most: `tiny` of check. max_norm
    is the float32 that it is handed over as."""
    grads, max_norm = [x * size for x in some([(300, 70), 11], (torch.float32, torch.bfloat16), scale=0.01)], float(np.float32(max_norm))
    mine = [t.clone() for t in grads]
    check(mine, grads, clipping.Clipper().clip(mine, max_norm), max_norm)


def test_alignment_order_of_dimensions_and_what_lies_beside(clipping):
    c = clipping.Clipper()
    for dtype in (torch.float32, torch.bfloat16):
        for skip in (1, 3, 5):
            for n in (1, 100, 8193, 30001):
                buf = torch.full((n + skip + 9,), 3.0, device="cuda", dtype=dtype)
                mine = buf[skip:skip + n]
                mine.copy_(some([n], (dtype,))[0])
                before = mine.clone()
                check([mine], [before], c.clip([mine], 0.25), 0.25)
                assert (buf[:skip] == 3).all() and (buf[skip + n:] == 3).all()
        turned = some([(40, 3, 50)], (dtype,))[0].permute(2, 0, 1)
        before = turned.clone()
        check([turned], [before], c.clip([turned], 0.25), 0.25)
        # out that begins elsewhere than its gradient does
        src, to = some([1003], (dtype,))[0][2:], torch.zeros(1006, device="cuda", dtype=dtype)
        check([to[5:]], [src], c.clip([src], 0.25, out=[to[5:]]), 0.25)
        assert not to[:5].any()


def test_into_tensors_of_other_shapes(clipping):
    """Contiguous ones of as many elements: a bucket's rows. Types are one by one the same, and orders of dimensions are not mixed."""
    c, grads = clipping.Clipper(), some([(33, 70), 9, (3, 4, 5)], (torch.float32, torch.bfloat16, torch.float32))
    out = [torch.zeros(t.numel(), device="cuda", dtype=t.dtype) for t in grads]
    check([a.view(b.shape) for a, b in zip(out, grads)], grads, c.clip(grads, 0.5, out=out), 0.5)
    turned = [t.clone() for t in grads]
    turned[0] = torch.zeros((70, 33), device="cuda").t()
    for bad in ([out[1], out[0], out[2]], [out[0], out[1].float(), out[2].bfloat16()], turned, [out[0][:-1], out[1], out[2]]):
        before = [t.clone() for t in bad]
        with pytest.raises(ValueError):
            c.clip(grads, 0.5, out=bad)
        assert all(torch.equal(a, b) for a, b in zip(bad, before))


def test_the_same_gradient_twice(clipping):
    t = some([1000], (torch.float32,))[0]
    c = clipping.Clipper()
    check([t, t], [t, t], c.norm([t, t]), float("inf"))
    from paper_2504_07878_amd import tokroute
    other = torch.zeros(1000, device="cuda")
    for grads, out in (([t, t], None), ([t[:600], t[500:]], None), ([t, other], [other, torch.zeros(1000, device="cuda")]), ([t[1:]], [t[:-1]])):
        with pytest.raises(tokroute.TokrouteError) as e:
            c.clip(grads, 1.0, out=out)
        assert e.value.code == tokroute.ERR_INVALID_ARG
    c.clip([t, t], 1.0, out=[other, torch.zeros(1000, device="cuda")])      # read twice, written to different places


def test_the_same_bits_every_time(clipping):
    grads = some([(1500, 896), 896, 77, (300, 300)] * 40, (torch.bfloat16, torch.float32))
    c = clipping.Clipper()
    first = c.norm(grads)
    assert all(torch.equal(first, c.norm(grads)) for _ in range(5)) and torch.equal(first, clipping.Clipper().norm(grads))


def test_other_streams_and_graphs(clipping):
    grads = some([(1500, 96), 896, 77] * 50, (torch.bfloat16, torch.float32))
    c, out = clipping.Clipper(), [torch.empty_like(t) for t in grads]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        norm = c.clip(grads, 1.0, out=out)
    torch.cuda.current_stream().wait_stream(side)
    check(out, grads, norm, 1.0)
    g, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        norm = c.clip(grads, 1.0, out=out)
    with torch.cuda.graph(g2):
        norm2 = c.norm(grads)
    for step in range(4):
        for t, x in zip(grads, some([t.shape for t in grads], (torch.bfloat16, torch.float32), seed=step + 5)):
            t.copy_(x * 2.0 ** -step)
        g.replay()
        eager = clipping.Clipper().norm(grads)
        g2.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, eager) and torch.equal(norm2, eager)
        check(out, grads, norm, 1.0)


def test_gradients_of_autograd(clipping):
    """As after a backward pass: clipped in place, so that a step uses them."""
    torch.manual_seed(3)
    model = torch.nn.Sequential(torch.nn.Linear(33, 65), torch.nn.Linear(65, 9)).cuda()
    model[1].bias.requires_grad_(False)
    model(torch.randn(20, 33, device="cuda")).square().sum().backward()
    grads = [p.grad for p in model.parameters()]
    before = [g.clone() for g in grads if g is not None]
    norm = clipping.Clipper().clip(grads, 0.5)
    check([g for g in grads if g is not None], before, norm, 0.5)


def test_refusals(clipping):
    from paper_2504_07878_amd import tokroute
    c = clipping.Clipper()
    t = torch.ones(10, device="cuda")
    for bad in (t.cpu(), t.double(), t.half(), t[::2], 3.0):
        with pytest.raises(ValueError):
            c.norm([t, bad])
        with pytest.raises(ValueError):
            c.clip([bad], 1.0)
    for out in ([], [t, t], [None], [torch.ones(11, device="cuda")], [torch.ones(10, device="cuda", dtype=torch.bfloat16)], [torch.ones(10)]):
        with pytest.raises(ValueError):
            c.clip([t], 1.0, out=out)
    for bad in (-1.0, float("nan")):
        with pytest.raises(tokroute.TokrouteError) as e:
            c.clip([t], bad)
        assert e.value.code == tokroute.ERR_INVALID_ARG
    assert (t == 1).all()


LARGE = [(500 + i % 7, 901) if i % 5 else (i % 31 + 1,) for i in range(490)] + [(151936, 11), 7]
LARGE[40:40] = [(0,), (20000, 1003)]


@pytest.mark.parametrize("by", [0.37, 1.5])
@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.bfloat16,), (torch.bfloat16, torch.float32, torch.bfloat16)], ids=["f32", "bf16", "both"])
def test_more_sums_than_one_join_and_more_bytes_than_the_cache(clipping, dtypes, by):
    """A large model's gradients: four lists that fill all workgroups of a launch (8192 sums, joined on the way twice, and before the scaling) and a fifth, 390 MB in bf16 and 770 MB in fp32, of which the
    last 192 MB are read through the caches, from a gradient's middle on; sizes that are no whole number of tiles, some small ones between them. Element by element."""
    grads, c = some(LARGE, dtypes, seed=9), clipping.Clipper()
    want = float(np.sqrt(sum(float(t.double().square().sum()) for t in grads)))
    max_norm = float(np.float32(by * want))
    scale = min(1.0, max_norm / want)
    out = [torch.full_like(t, 7) for t in grads]
    norms = [c.norm(grads), c.clip(grads, max_norm, out=out)]
    for t, x in zip(out, grads):
        y = x.double() * scale
        assert ((t.double() - y).abs() <= y.abs() * ((EPS[t.dtype] if t.dtype != torch.float32 else 0) + 3.1 * EPS[torch.float32]) + torch.finfo(t.dtype).tiny * EPS[t.dtype] * 2).all()
        assert by < 1 or torch.equal(t, x)
    norms.append(c.clip(grads, max_norm))
    assert all(torch.equal(a, b) for a, b in zip(grads, out))
    assert abs(float(norms[0]) / want - 1) <= 2.0 ** -23 and torch.equal(norms[0], norms[1]) and torch.equal(norms[0], norms[2])


@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.bfloat16, torch.float32)], ids=["f32", "both"])
def test_the_norm_of_many_lists(clipping, dtypes):
    """As those of test_the_same_bits_every_time, some 3200 sums, against 64 bits."""
    grads = some([(1500, 896), 896, 77, (300, 300)] * 40, dtypes)
    norm, want = clipping.Clipper().norm(grads), float(np.sqrt(sum(float(t.double().square().sum()) for t in grads)))
    assert abs(float(norm) / want - 1) <= 2.0 ** -23
