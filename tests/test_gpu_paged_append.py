"""hpd_append_paged against the plain implementation: codes, scales, status and what must stay as it was, byte for byte."""
import numpy as np
import pytest
import torch

from paper_2604_26209_b200 import synth
from tests import paged_oracle as po

pytestmark = pytest.mark.gpu

HEADS = [(4, 1, 64), (8, 2, 128), (2, 2, 64), (8, 1, 128)]


def geom(heads, cap=16, theta=500000.0):
    Hq, Hkv, D = heads
    return synth.Geom(Hq=Hq, Hkv=Hkv, D=D, rope_theta=theta, sm_scale=D ** -0.5, suffix_cap=cap)


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def wide(t):
    return t.float().cpu().numpy().astype(np.float64)


class Case:
    """A pool with random bytes everywhere (scales within the numbers of real data), tables, and random rows."""

    def __init__(self, g, n_pages, P, table, rows, seed=0, spread=0):
        from paper_2604_26209_b200 import binding as B
        self.B, self.g = B, g
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        codes = lambda: torch.from_numpy(rng.integers(0, 256, (n_pages, g.Hkv, P, g.D), dtype=np.uint8)).cuda()        # noqa: E731
        scales = lambda: torch.from_numpy(rng.integers(115, 125, (n_pages, g.Hkv), dtype=np.uint8)).cuda()             # noqa: E731
        e4, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
        self.cache = B.PagedCache(codes().view(e4), codes().view(e4), scales().view(e8), scales().view(e8), i32(table))
        rnd = lambda h: (torch.randn(rows, h, g.D, device="cuda", generator=gen) *                                     # noqa: E731
                         torch.exp2(torch.randint(-spread, spread + 1, (rows, 1, 1), device="cuda", generator=gen).float())).to(torch.bfloat16)
        self.q, self.k, self.v = rnd(g.Hq), rnd(g.Hkv), rnd(g.Hkv)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.table = np.asarray(table)
        self.before = self.host()

    def host(self):
        c = self.cache
        return po.Pool(*[x.view(torch.uint8).cpu().numpy() for x in (c.k, c.v, c.k_scale, c.v_scale)])

    def rotated(self, n, pos):
        """The bits of hpd_rope for the first n rows (None: as they are)."""
        q, k = self.q.clone(), self.k.clone()
        if pos is not None and n:
            self.B.hpd_rope(self.g, n, i32([n]), i32(pos), q, k)
        return q, k

    def check(self, row_seq, row_index, pos, q_rot=None, want_status=0):
        n = len(row_seq)
        q, k = self.rotated(n, pos)
        want = self.before
        status = po.append(want, self.table, wide(k)[:n], wide(self.v)[:n], row_seq, row_index)
        got = self.host()
        for name in ("k", "v"):
            assert po.same_codes(getattr(got, name), getattr(want, name)), name
        assert np.array_equal(got.ks, want.ks) and np.array_equal(got.vs, want.vs)
        assert int(self.status.item()) == status | want_status
        if q_rot is not None:
            assert torch.equal(q_rot[:n].view(torch.int16), q[:n].view(torch.int16))


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("P,rows,n", [(1, 3, 3), (5, 1, 1), (16, 40, 33), (30, 700, 641), (80, 9, 9)])
def test_step_form(heads, P, rows, n):
    g = geom(heads, cap=P)
    rng = np.random.default_rng(P + rows)
    slots = rows + 4
    c = Case(g, slots + 3, P, rng.permutation(slots + 3)[:slots, None], rows, seed=P, spread=3)
    seq_id = rng.permutation(slots)[:rows]
    held = rng.integers(0, P, rows)
    pos = rng.integers(0, 5000, rows)
    q_rot = torch.full_like(c.q, 7.0)
    k0, q0, v0 = c.k.clone(), c.q.clone(), c.v.clone()
    c.B.hpd_append_paged(g, rows, rows, i32([n]), None, None, i32(seq_id), i32(held), c.cache, i32(pos), c.q, q_rot, c.k, c.v, c.status)
    c.check(seq_id[:n], held[:n], pos[:n], q_rot)
    assert bool((q_rot[n:] == 7).all())                                        # rows behind the last one
    assert torch.equal(c.k, k0) and torch.equal(c.q, q0) and torch.equal(c.v, v0)
    # in place, and without the queries: the same
    c.B.hpd_append_paged(g, rows, rows, i32([n]), None, None, i32(seq_id), i32(held), c.cache, i32(pos), c.q, c.q, c.k, c.v, c.status)
    assert torch.equal(c.q[:n].view(torch.int16), q_rot[:n].view(torch.int16)) and torch.equal(c.q[n:], q0[n:])


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("P", [16, 32, 64, 24, 1])
@pytest.mark.parametrize("rotate", [False, True])
def test_token_form(heads, P, rotate):
    """Ragged chunks, empty ones among them, behind nothing, part of a page, or several pages; sequences named out of order."""
    g = geom(heads)
    rng = np.random.default_rng(P)
    new = np.array([0, 1, P, P - 1, 2 * P + 3, 0, 150, 17, 1, 0])
    held = np.array([3, 0, 0, 1, P // 2, 5, 2 * P - 1, P, 3 * P + P // 3, 0])
    per = int((-(-(new + held) // P)).max()) + 1
    n_seqs, T = len(new), int(new.sum())
    order = rng.permutation(n_seqs * per + 2)
    table = order[:n_seqs * per].reshape(n_seqs, per)
    c = Case(g, n_seqs * per + 2, P, table, T + 5, seed=P + 1, spread=2)
    seq_id = rng.permutation(n_seqs)
    start = np.concatenate([[0], np.cumsum(new)])
    row_seq = np.repeat(np.arange(n_seqs), new)
    index = held[row_seq] + np.arange(T) - start[row_seq]
    pos = rng.integers(0, 9000, T + 5) if rotate else None
    q_rot = torch.full_like(c.q, 7.0)
    c.B.hpd_append_paged(g, n_seqs, T + 5, i32([T]), i32(np.concatenate([row_seq, [-1] * 5])), i32(start), i32(seq_id), i32(held), c.cache,
                         i32(pos) if rotate else None, c.q if rotate else None, q_rot if rotate else None, c.k, c.v, c.status)
    c.check(seq_id[row_seq], index, pos[:T] if rotate else None, q_rot if rotate else None)
    assert bool((q_rot[T if rotate else 0:] == 7).all())


@pytest.mark.parametrize("P", [64, 50, 33, 32, 16, 7])
def test_token_form_of_many_rows(P):
    """More windows of rows than are on the GPU at a time; pages that end anywhere in them; one row, whole pages and long chunks side by side."""
    g = geom((16, 8, 64))
    rng = np.random.default_rng(100 + P)
    new = np.concatenate([rng.integers(1, 900, 10), [1, 1, 1, P, 2 * P, 64, 65, 63], rng.integers(0, 3, 30)])
    new = np.concatenate([new, [5400 - new.sum()]]) if new.sum() < 5400 else new
    rng.shuffle(new)
    held = rng.integers(0, 2 * P, len(new))
    per = int((-(-(new + held) // P)).max())
    n_seqs, T = len(new), int(new.sum())
    table = np.full((n_seqs, per), -1)
    need = -(-(new + held) // P)
    pages = rng.permutation(int(need.sum()))
    for s, a in enumerate(np.cumsum(need) - need):
        table[s, :need[s]] = pages[a:a + need[s]]
    c = Case(g, len(pages), P, table, T, seed=P + 5, spread=2)
    start = np.concatenate([[0], np.cumsum(new)])
    row_seq = np.repeat(np.arange(n_seqs), new)
    index = held[row_seq] + np.arange(T) - start[row_seq]
    pos = rng.integers(0, 9000, T)
    q_rot = torch.full_like(c.q, 7.0)
    c.B.hpd_append_paged(g, n_seqs, T, i32([T]), i32(row_seq), i32(start), None, i32(held), c.cache, i32(pos), c.q, q_rot, c.k, c.v, c.status)
    c.check(row_seq, index, pos, q_rot)


def test_keys_only_with_rotation():
    g = geom((8, 2, 128))
    c = Case(g, 8, 16, np.arange(8)[:, None], 8, seed=3)
    pos = np.arange(8) * 511
    for form in ("step", "tokens"):
        rs, start = (None, None) if form == "step" else (i32(np.arange(8)), i32(np.arange(9)))
        c.B.hpd_append_paged(g, 8, 8, i32([8]), rs, start, None, i32(np.zeros(8)), c.cache, i32(pos), None, None, c.k, c.v, c.status)
        c.check(np.arange(8), np.zeros(8, int), pos)
        c.before = c.host()


@pytest.mark.parametrize("form", ["step", "tokens"])
def test_extreme_values(form):
    """Zeros, subnormals, the largest numbers, infinities and NaN: in new pages, and behind tokens of another magnitude."""
    g = geom((2, 1, 64), cap=4)
    rows = [0.0, -0.0, 1e-40, 9.2e-41, 3.38e38, np.inf, -np.inf, np.nan, 448.0, 449.0, 1.75, 1.7578125, 2.0 ** -126, 1e-30, 1e30]
    n = len(rows)
    c = Case(g, 2 * n, 4, np.arange(2 * n)[:, None], 2 * n, seed=5)
    for x in (c.k, c.v):
        x[:, :, ::3] = torch.tensor(rows * 2, device="cuda", dtype=torch.float32).to(torch.bfloat16)[:, None, None]
    x = torch.tensor(rows * 2, device="cuda", dtype=torch.float32).to(torch.bfloat16)
    c.k[n:] = x[n:, None, None]
    c.v[n:] = x[n:, None, None]
    held = np.array([0, 3] * n)[:2 * n]
    rs, start = (None, None) if form == "step" else (i32(np.arange(2 * n)), i32(np.arange(2 * n + 1)))
    c.B.hpd_append_paged(g, 2 * n, 2 * n, i32([2 * n]), rs, start, None, i32(held), c.cache, None, None, None, c.k, c.v, c.status)
    c.check(np.arange(2 * n), held, None)


@pytest.mark.parametrize("was", [0, 1, 60, 126, 200, 253, 254, 255])
def test_scales_of_before(was):
    """Every kind of scale byte a page may hold, below and above what the new token needs."""
    g = geom((2, 2, 64), cap=8)
    c = Case(g, 3, 8, np.arange(3)[:, None], 3, seed=6)
    for s in (c.cache.k_scale, c.cache.v_scale):
        s.view(torch.uint8).fill_(was)
    c.before = c.host()
    c.B.hpd_append_paged(g, 3, 3, i32([3]), None, None, None, i32([1, 4, 7]), c.cache, None, None, None, c.k, c.v, c.status)
    if was < 255:
        c.check(np.arange(3), [1, 4, 7], None)
    else:
        assert bool((c.cache.k_scale.view(torch.uint8) == 255).all()) and int(c.status.item()) == 0


@pytest.mark.parametrize("form", ["step", "tokens"])
def test_bad_tables_are_reported_and_harm_nobody(form):
    """Pages out of range, sequences out of range, full sequences: a status bit, nothing stored, the queries rotated all the same."""
    g = geom((4, 2, 64), cap=4)
    table = np.array([[0], [9], [-1], [2], [2147483647], [3]])
    for seq_id, held, bits in (([0, 1, 5], [0, 1, 2], 2), ([2, 0, 4], [1, 3, 0], 2), ([0, 6, 3], [1, 0, 0], 2), ([-5, 0, 3], [1, 0, 0], 2),
                               ([0, 3, 5], [4, 2, 1], 1), ([0, 3, 5], [1, 2, 2147483647], 1), ([0, 3, 1], [5, 2, 0], 3)):
        c = Case(g, 9, 4, table, 3, seed=7)
        rs, start = (None, None) if form == "step" else (i32(np.arange(3)), i32(np.arange(4)))
        pos, q_rot = np.array([1, 77, 4000]), torch.zeros_like(c.q)
        c.B.hpd_append_paged(g, 3, 3, i32([3]), rs, start, i32(seq_id), i32(held), c.cache, i32(pos), c.q, q_rot, c.k, c.v, c.status)
        c.check(seq_id, held, pos, q_rot)
        assert int(c.status.item()) == bits


def test_rows_of_no_sequence_are_reported():
    """Token form: a row whose sequence is out of range, or that lies outside its sequence's rows."""
    g = geom((4, 2, 64), cap=16)
    c = Case(g, 4, 16, np.arange(4)[:, None], 12, seed=8)
    seq = np.array([0, 0, 0, 1, 1, 9, -3, 2, 2, 0, 3, 3])
    start = np.array([0, 3, 7, 10, 12])                                        # row 5, 6: no sequence; row 9: not one of sequence 0's
    q_rot, pos = torch.zeros_like(c.q), np.arange(12) * 3
    c.B.hpd_append_paged(g, 4, 12, i32([12]), i32(seq), i32(start), None, i32([2, 0, 0, 5]), c.cache, i32(pos), c.q, q_rot, c.k, c.v, c.status)
    index = np.array([2, 3, 4, 0, 1, 0, 0, 0, 1, 0, 5, 6])
    kept = np.array([0, 1, 2, 3, 4, 7, 8, 10, 11])
    q, k = c.rotated(12, pos)
    po.append(c.before, c.table, wide(k)[kept], wide(c.v)[kept], seq[kept], index[kept])
    got = c.host()
    assert po.same_codes(got.k, c.before.k) and po.same_codes(got.v, c.before.v) and np.array_equal(got.ks, c.before.ks)
    assert int(c.status.item()) == 2
    assert torch.equal(q_rot.view(torch.int16), q.view(torch.int16))


def test_negative_lengths_are_bad_tables():
    g = geom((4, 2, 64), cap=16)
    for form in ("step", "tokens"):
        c = Case(g, 2, 16, np.arange(2)[:, None], 2, seed=9)
        rs, start = (None, None) if form == "step" else (i32([0, 1]), i32([0, 1, 2]))
        c.B.hpd_append_paged(g, 2, 2, i32([2]), rs, start, None, i32([-1, 3]), c.cache, None, None, None, c.k, c.v, c.status)
        po.append(c.before, c.table, wide(c.k)[1:], wide(c.v)[1:], [1], [3])
        got = c.host()
        assert po.same_codes(got.k, c.before.k) and np.array_equal(got.ks, c.before.ks) and int(c.status.item()) == 2


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 bytes of codes: its last page."""
    g = geom((8, 8, 128))
    P = 64
    n_pages = 2 ** 32 // (8 * P * 128) + 2
    from paper_2604_26209_b200 import binding as B
    codes = [torch.zeros(n_pages, 8, P, 128, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(n_pages, 8, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = B.PagedCache(*[x.view(torch.float8_e4m3fn) for x in codes], *[x.view(torch.float8_e8m0fnu) for x in scales], i32([[n_pages - 1], [0]]))
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(20, 8, 128, device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.hpd_append_paged(g, 1, 20, i32([20]), i32(np.zeros(20)), i32([0, 20]), None, i32([0]), cache, None, None, None, k, v, status)
    B.hpd_append_paged(g, 1, 1, i32([1]), None, None, None, i32([20]), cache, None, None, None, k, v, status)
    want = po.Pool(*[np.zeros((1, 8, P, 128), np.uint8)] * 2, *[np.zeros((1, 8), np.uint8)] * 2)
    want.append(0, 0, wide(k), wide(v))
    want.append(0, 20, wide(k)[:1], wide(v)[:1])
    assert np.array_equal(codes[0][-1].cpu().numpy(), want.k[0]) and np.array_equal(codes[1][-1].cpu().numpy(), want.v[0])
    assert np.array_equal(scales[0][-1].cpu().numpy(), want.ks[0]) and int(status.item()) == 0
    for x in codes + scales:                             # nothing else was touched (piece by piece: a sum over 4 GB takes memory)
        assert not any(bool(x[lo:min(lo + 4096, n_pages - 1)].any()) for lo in range(0, n_pages - 1, 4096))


def test_rotation_is_that_of_64_bits():
    g = geom((2, 1, 128))
    c = Case(g, 200, 4, np.arange(200)[:, None], 200, seed=11)
    pos = np.arange(200) * 641
    q_rot = torch.zeros_like(c.q)
    c.B.hpd_append_paged(g, 200, 200, i32([200]), None, None, None, i32(np.zeros(200)), c.cache, i32(pos), c.q, q_rot, c.k, c.v, c.status)
    ang = pos[:, None, None] * 500000.0 ** (-np.arange(64) / 64)

    def turn(x):
        a, b = x[..., :64], x[..., 64:]
        return np.concatenate([a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)], axis=-1)
    # bf16: half a step, 2^-8; the fp32 sine of an angle of up to pi, rounded, and two products: 2^-21 of the pair's length
    want, q = turn(wide(c.q)), wide(c.q)
    length = np.tile(np.hypot(q[..., :64], q[..., 64:]), (1, 1, 2))
    assert np.all(np.abs(wide(q_rot) - want) <= np.abs(want) * 2.0 ** -8 + length * 2.0 ** -21)
    want = turn(wide(c.k))
    got = c.host().tokens(np.arange(200), 200 * 4)[0][::4]
    # codes: half a step of e4m3, 2^-4 of the value or half of the smallest step, 2^-10 of the scale (rounded to bf16 before)
    scale = po.scale_value(c.host().ks)[:, 0][:, None, None]
    assert np.all(np.abs(got - want) <= np.abs(want) * (2.0 ** -4 + 2.0 ** -7) + scale * 2.0 ** -10)


def test_captured_and_on_another_stream():
    """The call in a graph, replayed with other data in the same buffers, on a stream of its own."""
    g = geom((8, 2, 128))
    c = Case(g, 64, 16, np.arange(64)[:, None], 64, seed=12)
    held, pos = np.arange(64) % 16, np.arange(64) * 9
    args = (g, 64, 64, i32([64]), None, None, None, i32(held), c.cache, i32(pos), c.q, torch.zeros_like(c.q), c.k, c.v, c.status)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            c.B.hpd_append_paged(*args)
        c.k.mul_(-2)
        c.v.mul_(4)
        graph.replay()
    s.synchronize()
    c.check(np.arange(64), held, pos, args[11])
