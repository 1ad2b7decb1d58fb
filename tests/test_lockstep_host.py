"""The kernels of draws, largest logits, gradient norm and clipping on the CPU (lockstep.py), no GPU needed: wavefronts that get ahead of each other, and ends of the ranges that are the same on either."""
import numpy as np
import pytest

import lockstep
import picks


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    return lockstep.build(str(tmp_path_factory.mktemp("lanes")))


def rows_of(kind, n, v, seed, half=False):
    """peaked: a body and a few tokens far above it; flat: a body alone; ties: a body in steps of 1/8; together: the largest are neighbours; equal: one value; masked: most is -inf. half: bits of bfloat16."""
    g = np.random.Generator(np.random.Philox(seed))
    z = g.standard_normal((n, v), dtype=np.float32)
    if kind == "peaked":
        z = z * 2 + np.where(g.random((n, v)) < 20 / v, g.uniform(6, 14, (n, v)), 0)
    elif kind == "ties":
        z = np.round(z * 8) / 8
    elif kind == "together":
        z[:, v // 3:v // 3 + 700] += 9
    elif kind == "equal":
        z[:] = 1.5
    elif kind == "masked":
        z[g.random((n, v)) < 0.97] = -np.inf
        z[0] = -np.inf
    z = np.ascontiguousarray(z, dtype=np.float32)
    return (z.view(np.uint32) >> 16).astype(np.uint16) if half else z


def values(z):
    return (z.astype(np.uint32) << 16).view(np.float32) if z.dtype == np.uint16 else z


def check(z, u, how, token, logprob):
    how = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0) | how
    t, p, m = (float(np.float32(how[x])) for x in ("temperature", "top_p", "min_p"))
    for i, row in enumerate(values(z)):
        assert picks.check_draw(row, u[i], t, how["top_k"], p, m, token[i], logprob[i]), (i, how, u[i], token[i], logprob[i])


# what each reaches: filters that end among few tokens, among more than are compared all with all (top-p 0.9, top-k 100 of neighbours), among equal ones (ties at top-k's border, a few or many), below
# what the parts of a row have listed (flat rows, through the queue), and nothing cut
SETTINGS = [dict(), dict(top_k=20), dict(top_p=0.9), dict(top_k=200, top_p=0.95), dict(top_k=700), dict(min_p=0.05), dict(top_k=700, min_p=0.01), dict(top_p=0.99, min_p=0.02, temperature=1.5), dict(top_p=0.999),
            dict(temperature=0.0)]


@pytest.mark.parametrize("order", lockstep.ORDERS)
@pytest.mark.parametrize("kind", ["peaked", "flat", "ties", "together", "equal", "masked"])
@pytest.mark.parametrize("v", [257, 3001, 9001, 20001])
def test_a_wavefront_that_is_ahead_of_the_others_changes_no_draw(host, v, kind, order):
    for i, how in enumerate(SETTINGS):
        z, u = rows_of(kind, 3, v, 100 * v + i, half=i % 3 == 2), np.random.Generator(np.random.Philox(i)).random(3, dtype=np.float32)
        check(z, u, how, *host.sample(z, u, order, **how))


@pytest.mark.parametrize("order", lockstep.ORDERS)
@pytest.mark.parametrize("kind", ["peaked", "flat", "ties", "together", "equal", "masked"])
@pytest.mark.parametrize("v", [257, 3001, 20001])
def test_a_wavefront_that_is_ahead_of_the_others_changes_no_list(host, v, kind, order):
    for k in (5, 60, 300, 1000):
        z = rows_of(kind, 2, v, v + k, half=k == 60)
        ids, got = host.top(z, k, order)
        for row, i, x in zip(values(z), ids, got):
            want = picks.order_of(row)[:k]
            assert np.array_equal(i, np.concatenate([want, np.full(k - len(want), -1)]))
            assert np.array_equal(x, np.concatenate([row[want], np.full(k - len(want), -np.inf, np.float32)]))


def halved(x):
    """Bits of bfloat16, of values that have them."""
    return (np.ascontiguousarray(x, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)


@pytest.mark.parametrize("inside", [False, True])
def test_gradients_whose_norm_is_beyond_32_bits_stay_as_they_are(host, inside):
    """The norm that the call reports says which case it is: infinite (100 elements of 2^127 are 2^130 long), and nothing is scaled."""
    grads = [np.full(100, 2.0 ** 127, np.float32), halved(np.full(33, -1.5)), np.ones(7, np.float32)]
    before, out = [x.copy() for x in grads], None if inside else [np.full_like(x, 7) for x in grads]
    assert host.clip(grads, 1.0, out) == np.inf
    assert all(np.array_equal(a, b) for a, b in zip(grads if inside else out, before))
    # at the last length that 32 bits hold they are
    grads = [np.full(2, 2.0 ** 127, np.float32)]
    assert host.clip(grads, 1.0) == np.float32(2.0 ** 127.5) and np.allclose(grads[0], 0.5 ** 0.5, rtol=2 ** -22, atol=0)


@pytest.mark.parametrize("max_norm, size", [(1e-8, 1e37), (1e-3, 3e37), (1e-30, 1e15), (3e-38, 2e30), (1e-44, 1e38), (0.25, 2e37)])
def test_scales_below_what_32_bits_hold(host, max_norm, size):
    """max_norm / norm is subnormal in 32 bits, or zero, where the products are not. The scale and the product are rounded to 24 bits, bfloat16 to 8 then; results below 2^-126 are off by half
    of 2^-149 (bfloat16: 2^-133) twice. max_norm is the float32 that it is handed over as."""
    g = np.random.Generator(np.random.Philox(5))
    grads = [(g.uniform(-1, 1, 300) * size).astype(np.float32), halved(g.uniform(-1, 1, 77) * size), np.array([0.0, -0.0, 1e-30, size], np.float32)]
    wide = [values(x).astype(np.float64) for x in grads]
    length, max_norm = np.sqrt(sum((x * x).sum() for x in wide)), float(np.float32(max_norm))
    out = [np.full_like(x, 7) for x in grads]
    held = length <= np.finfo(np.float32).max          # (two of the lengths are beyond 32 bits)
    norm = host.clip(grads, max_norm, out)
    assert abs(norm / length - 1) <= 2.0 ** -23 if held else norm == np.inf
    for got, x in zip(out, wide):
        want, half = x * (max_norm / length if held else 1.0), got.dtype == np.uint16
        off = np.abs(values(got).astype(np.float64) - want)
        assert (off <= np.abs(want) * ((2.0 ** -8 if half else 0) + 3.1 * 2.0 ** -24) + (2.0 ** -133 if half else 0) + 2.0 ** -149).all()


@pytest.mark.parametrize("how", [dict(top_p=0.9), dict(min_p=0.01), dict(top_p=0.95, min_p=0.001)])
@pytest.mark.parametrize("more", [0, 1, 2**31 - 1 - 9001])
def test_a_top_k_of_all_tokens_is_none(host, how, more):
    """Flat rows go the way that they go without top-k, read by all workgroups rather than by one."""
    z, u = rows_of("flat", 3, 9001, 3), np.float32([0.1, 0.5, 0.9])
    without = host.sample(z, u, **how)
    assert host.launches("steps_kernel") == 1
    got = host.sample(z, u, **how, top_k=9001 + more)
    assert host.launches("steps_kernel") == 1 and all(np.array_equal(a, b) for a, b in zip(got, without))
    check(z, u, how, *got)


ENDS = np.float32([0.0, 1e-20, 2.0 ** -24, 1 - 2.0 ** -24, 1.0, 5.0])


@pytest.mark.parametrize("temperature", [1.0, 0.1, 0.01, 1e-3, 1e-30])
@pytest.mark.parametrize("v", [3001, 9001, 20001])
def test_numbers_at_the_ends_draw_nothing_without_weight(host, v, temperature):
    """0 and numbers that 32 bits round to 1: at low temperatures nearly all tokens have no weight that 64 bits hold beside the largest, the first and the last ids too."""
    z = np.repeat(2 * rows_of("flat", 1, v, 7), len(ENDS), 0)
    check(z, ENDS, dict(temperature=temperature), *host.sample(z, ENDS, temperature=temperature))


@pytest.mark.parametrize("order", lockstep.ORDERS)
def test_clipping_of_several_lists(host, order):
    """Two lists and a half, one of the gradients of several tiles: in place as into others, and the norm alone."""
    g = np.random.Generator(np.random.Philox(9))
    grads = [(g.standard_normal(30011 if i == 130 else i % 37, dtype=np.float32)) for i in range(290)]
    grads = [halved(x) if i % 3 == 1 else x for i, x in enumerate(grads)]
    wide = [values(x).astype(np.float64) for x in grads]
    length = np.sqrt(sum((x * x).sum() for x in wide))
    max_norm, out = float(np.float32(0.37 * length)), [np.full_like(x, 7) for x in grads]
    norms = [host.clip(grads, None, order=order), host.clip(grads, max_norm, out, order), host.clip(grads, max_norm, order=order)]
    assert norms[0] == norms[1] == norms[2] and abs(norms[0] / length - 1) <= 2.0 ** -23
    for a, b, x in zip(grads, out, wide):
        want = x * (max_norm / length)
        assert np.array_equal(a, b) and (np.abs(values(b) - want) <= np.abs(want) * ((2.0 ** -8 if b.dtype == np.uint16 else 0) + 3.1 * 2.0 ** -24)).all()
