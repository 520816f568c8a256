"""How far a cached element may be from what was appended, and when a page that fills up token by token holds the codes of one that is filled at once.

A code is off by half a step: 2^-4 of a normal element, 2^-10 of the scale below 2^-6 of it.  Where a scale s grows to s' >= 2 s, an element that stays a
normal code does not change; one that falls below 2^-6 s' is rounded again, to a multiple of 2^-9 s': by 2^-10 s' at most.  It was off by less
than 2^-9 s <= 2^-10 s' before if it was subnormal already, and by half a step of the binades below 2^-6 s', 2^-11 s' at most, if it was normal.  So it stays
within 2^-9 of the scale that the page has."""
import numpy as np
import pytest

from tests import paged_oracle as po


def _bf16(x):
    return (x.astype(np.float32).view(np.uint32) & 0xffff0000).view(np.float32).astype(np.float64)


def _pages(seed, n_pages=100):
    """Tokens [n, Hkv, 64] of a page: bf16 values (eight significant bits), magnitudes that rise, fall or jump over up to 2^24."""
    rng = np.random.default_rng(seed)
    for i in range(n_pages):
        n = int(rng.integers(2, 17))
        mag = rng.uniform(-14, 10, n)
        mag = np.sort(mag) if i % 3 == 0 else np.sort(mag)[::-1] if i % 3 == 1 else mag
        yield _bf16(rng.uniform(-1, 1, (n, 1, 64)) * 2.0 ** mag[:, None, None])


def _empty():
    return po.Pool(*[np.zeros((1, 1, 16, 64), np.uint8)] * 2, *[np.zeros((1, 1), np.uint8)] * 2)


@pytest.mark.parametrize("seed", range(3))
def test_pages_filled_token_by_token(seed):
    for x in _pages(seed):
        n = len(x)
        one, many = _empty(), _empty()
        one.append(0, 0, x, x)
        for t in range(n):
            many.append(0, t, x[t:t + 1], x[t:t + 1])
        scale = float(po.scale_value(many.ks)[0, 0])
        assert np.array_equal(one.ks, many.ks)
        # from what was appended
        assert np.all(np.abs(many.tokens([0], n)[0] - x) <= np.maximum(np.abs(x) * 2.0 ** -4, scale * 2.0 ** -9))
        assert np.all(np.abs(one.tokens([0], n)[0] - x) <= np.maximum(np.abs(x) * 2.0 ** -4, scale * 2.0 ** -10))
        # from the page filled at once
        normal = np.abs(x[:, 0]) >= scale * 2.0 ** -6
        assert np.array_equal(one.k[0, 0, :n][normal], many.k[0, 0, :n][normal])
        assert np.all(np.abs(po.VALUES[one.k] - po.VALUES[many.k]) <= 2.0 ** -9)


def test_an_element_rounded_twice():
    """0.02844 under a scale of 1, which another token then doubles: further off than half a step of either scale."""
    x = 233 * 2.0 ** -13
    p = _empty()
    first = np.zeros((1, 1, 64))
    first[0, 0, :2] = x, 448.0
    p.append(0, 0, first, first)
    p.append(0, 1, np.full((1, 1, 64), 896.0), np.full((1, 1, 64), 896.0))
    off = abs(p.tokens([0], 1)[0][0, 0, 0] - x)
    assert po.scale_value(p.ks)[0, 0] == 2 and 2 * 2.0 ** -10 < off <= 2 * 2.0 ** -9


def test_the_same_codes_reach_down_to_2_to_the_minus_6_of_the_scale_only():
    """The largest element of a page may be just above 224 scales: an element of more than 2^-14 of it can be rounded twice."""
    x = float(_bf16(np.array([0.01428]))[0])
    top = 225.0
    assert x > 2.0 ** -14 * top and x < 2.0 ** -6
    one, many = _empty(), _empty()
    tokens = np.zeros((4, 1, 64))
    tokens[:, 0, 0] = x, 0.25 * top, 0.5 * top, top
    one.append(0, 0, tokens, tokens)
    for t in range(4):
        many.append(0, t, tokens[t:t + 1], tokens[t:t + 1])
    assert one.ks[0, 0] == many.ks[0, 0] == 127 and one.k[0, 0, 0, 0] != many.k[0, 0, 0, 0]


def test_infinities_keep_the_largest_code_of_the_scale_that_they_met():
    x = np.full((2, 1, 64), np.inf)
    x[0, 0, 1:], x[1] = 100.0, 4000.0
    p = _empty()
    p.append(0, 0, x[:1], x[:1])
    assert p.tokens([0], 1)[0][0, 0, 0] == 448 * 2.0 ** -2
    p.append(0, 1, x[1:], x[1:])
    assert po.scale_value(p.ks)[0, 0] == 16 and p.tokens([0], 1)[0][0, 0, 0] == 448 * 2.0 ** -2


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["step", "tokens"])
@pytest.mark.parametrize("heads", [(4, 1, 64), (8, 2, 128)])
def test_grown_pages_hold_what_was_appended(form, heads):
    """Calls of one token each (and chunks in between, tokens form) into pages whose scales grow: every element against what was appended."""
    import torch
    from tests.test_gpu_paged_append import geom, i32
    from paper_2604_26209_b200 import binding as B
    g, P, n = geom(heads, cap=16), 16, 40
    rng = np.random.default_rng(heads[2])
    mag = rng.uniform(-14, 10, (n, P))
    mag[::3] = np.sort(mag[::3], axis=1)
    cache = B.PagedCache.alloc(g, n, 1, P)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    k, v = (torch.from_numpy(_bf16(rng.uniform(-1, 1, (n, P, g.Hkv, g.D)) * 2.0 ** mag[:, :, None, None])).cuda().to(torch.bfloat16) for _ in range(2))
    t = 0
    while t < P:
        m = min(1 if form == "step" or t % 3 else 2, P - t)
        rows = n * m
        rs, start = (None, None) if form == "step" else (i32(np.repeat(np.arange(n), m)), i32(np.arange(n + 1) * m))
        B.hpd_append_paged(g, n, rows, i32([rows]), rs, start, None, i32(np.full(n, t)), cache, None, None, None, k[:, t:t + m].reshape(rows, g.Hkv, g.D).contiguous(),
                           v[:, t:t + m].reshape(rows, g.Hkv, g.D).contiguous(), status)
        t += m
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for codes, scales, x in ((cache.k, cache.k_scale, k), (cache.v, cache.v_scale, v)):
        scale = po.scale_value(scales.view(torch.uint8).cpu().numpy())[:, :, None, None]
        got = po.VALUES[codes.view(torch.uint8).cpu().numpy()] * scale                    # [n, Hkv, P, D]
        want = x.double().cpu().numpy().transpose(0, 2, 1, 3)
        assert np.all(np.abs(got - want) <= np.maximum(np.abs(want) * 2.0 ** -4, scale * 2.0 ** -9))
