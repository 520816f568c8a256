"""hpd_append_paged at the grids of large prompts: several heads to a CTA, one CTA to a window's heads; queries rotated in place.  Every code and every
scale against the definition in 64 bits, a sample of pages against the plain implementation on the host too."""
import numpy as np
import pytest
import torch

from tests import paged_oracle as po
from tests.test_gpu_paged_append import geom, i32

pytestmark = pytest.mark.gpu

E4, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _sequences(rng, rows, P):
    """Ragged sequences of `rows` tokens in all, single tokens and empty ones among them, behind nothing or behind up to two pages."""
    new = [0, 1, 1, P, P + 1, 64, 63]
    while sum(new) < rows:
        new.append(int(min(rng.integers(1, 3000), rows - sum(new))))
    new = rng.permutation(new)
    return new, rng.integers(0, 2 * P, len(new)) * (rng.random(len(new)) < 0.6)


class Tokens:
    def __init__(self, g, rows, P, seed):
        from paper_2604_26209_b200 import binding as B
        self.B, self.g, self.P, self.n = B, g, P, rows
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.new, self.held = _sequences(rng, rows, P)
        need = -(-(self.new + self.held) // P)
        self.table = np.full((len(need), int(need.max())), -1)
        order = rng.permutation(int(need.sum()) + 2)
        for s, at in enumerate(np.cumsum(need) - need):
            self.table[s, :need[s]] = order[at:at + need[s]]
        self.start = np.concatenate([[0], np.cumsum(self.new)])
        self.seq = np.repeat(np.arange(len(need)), self.new)
        self.index = self.held[self.seq] + np.arange(rows) - self.start[self.seq]
        self.page, self.slot = self.table[self.seq, self.index // P], self.index % P
        self.pos = rng.integers(0, 9000, rows)
        rnd = lambda h: (torch.randn(rows, h, g.D, device="cuda", generator=gen) *                                    # noqa: E731
                         torch.exp2(torch.randint(-2, 3, (rows, 1, 1), device="cuda", generator=gen).float())).to(torch.bfloat16)
        self.q, self.k, self.v = rnd(g.Hq), rnd(g.Hkv), rnd(g.Hkv)
        code = lambda: torch.randint(0, 256, (len(order), g.Hkv, P, g.D), dtype=torch.uint8, device="cuda", generator=gen)  # noqa: E731
        scale = lambda: torch.randint(115, 125, (len(order), g.Hkv), dtype=torch.uint8, device="cuda", generator=gen)      # noqa: E731
        self.before = [code(), code(), scale(), scale()]
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def append(self, q=None, q_rot=None, rotate=True):
        """The call on a copy of the pools; what they hold then."""
        pools = [x.clone() for x in self.before]
        cache = self.B.PagedCache(pools[0].view(E4), pools[1].view(E4), pools[2].view(E8), pools[3].view(E8), i32(self.table))
        self.B.hpd_append_paged(self.g, len(self.new), self.n, i32([self.n]), i32(self.seq), i32(self.start), None, i32(self.held), cache,
                                i32(self.pos) if rotate else None, q, q_rot, self.k, self.v, self.status)
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0
        return pools

    def rotated(self):
        """The bits of hpd_rope."""
        q, k = self.q.clone(), self.k.clone()
        self.B.hpd_rope(self.g, self.n, i32([self.n]), i32(self.pos), q, k)
        return q, k

    def check(self, got, k):
        """Every code and scale, page by page, 64 bits throughout."""
        page, slot = (torch.from_numpy(x).cuda() for x in (self.page, self.slot))
        first = torch.zeros(len(self.before[0]), dtype=torch.int64, device="cuda")           # tokens that each page held
        seqs = np.flatnonzero(self.new)
        first[torch.from_numpy(self.table[seqs, self.held[seqs] // self.P]).cuda()] = torch.from_numpy(self.held[seqs] % self.P).cuda()
        touched = torch.zeros_like(first, dtype=torch.bool)
        touched[page] = True
        for codes, scales, was_codes, was, x in ((got[0], got[2], self.before[0], self.before[2], k), (got[1], got[3], self.before[1], self.before[3], self.v)):
            top = torch.zeros(len(codes), self.g.Hkv, dtype=torch.float64, device="cuda")
            top.index_reduce_(0, page, x.double().abs().amax(dim=2), "amax")
            e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448)).clamp(min=-126)
            e = torch.where(top > 448 * torch.exp2(e), e + 1, e)
            e = torch.where((top <= 448 * torch.exp2(e - 1)) & (e > -126), e - 1, e)
            old = was.double() - 127
            now = torch.where(touched[:, None], torch.where(first[:, None] > 0, torch.maximum(e, old), e), old)
            assert torch.equal(scales, (now + 127).to(torch.uint8))
            want = was_codes.clone()
            grown = (now > old) & (first > 0)[:, None]
            for p, h in grown.nonzero().tolist():
                n = int(first[p])
                f = float(2.0 ** (old[p, h] - now[p, h]))
                want[p, h, :n] = (was_codes[p, h, :n].view(E4).double() * f).to(torch.float32).to(E4).view(torch.uint8)
            for lo in range(0, self.n, 16384):
                part = slice(lo, min(lo + 16384, self.n))
                y = (x[part].double() * torch.exp2(-now[page[part]])[:, :, None]).to(torch.float32).to(E4)      # exact in 32 bits: a bf16 times a power of two
                want.view(torch.uint8)[page[part], :, slot[part]] = y.view(torch.uint8)
            nan = ((codes & 0x7f) == 0x7f) & ((want & 0x7f) == 0x7f)
            assert bool((nan | (codes == want)).all())

    def check_on_the_host(self, got, k, some=40):
        rng = np.random.default_rng(self.n)
        for s in rng.choice(np.flatnonzero(self.new), min(some, int((self.new > 0).sum())), replace=False):
            j = int(rng.integers(self.held[s] // self.P, (self.held[s] + self.new[s] - 1) // self.P + 1))
            rows = np.arange(self.start[s], self.start[s + 1])
            rows = rows[self.index[rows] // self.P == j]
            p = int(self.table[s, j])
            pool = po.Pool(*[x[p:p + 1].cpu().numpy() for x in (self.before[0], self.before[1], self.before[2], self.before[3])])
            f = lambda x: x[rows[0]:rows[-1] + 1].double().cpu().numpy()                                             # noqa: E731
            pool.append(0, int(self.slot[rows[0]]), f(k), f(self.v))
            assert po.same_codes(got[0][p].cpu().numpy(), pool.k[0]) and po.same_codes(got[1][p].cpu().numpy(), pool.v[0])
            assert np.array_equal(got[2][p].cpu().numpy(), pool.ks[0]) and np.array_equal(got[3][p].cpu().numpy(), pool.vs[0])


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("heads,rows,P", [((8, 8, 128), 12000, 64), ((8, 8, 128), 12000, 16), ((16, 8, 128), 25000, 32), ((4, 4, 128), 12000, 64),
                                          ((16, 8, 64), 16000, 33)])
def test_several_heads_to_a_cta(heads, rows, P):
    """More windows than half of what the GPU holds at once: a third of the heads' CTAs to a window, so that a CTA takes three heads (or two of four)."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    resident = (3 if heads[2] == 128 else 4) * sms
    assert resident // 2 < -(-rows // 48) < 6 * resident
    t = Tokens(geom(heads), rows, P, seed=rows + P)
    q, k = t.rotated()
    q_rot = torch.full_like(t.q, 7.0)
    got = t.append(t.q, q_rot)
    assert torch.equal(q_rot.view(torch.int16), q.view(torch.int16))
    t.check(got, k)
    t.check_on_the_host(got, k)
    assert _same(t.append(), got)                                     # without the queries: the same pages
    plain = t.append(rotate=False)
    t.check(plain, t.k)
    k0, v0 = t.k.clone(), t.v.clone()
    assert _same(t.append(t.q, t.q), got)                             # in place
    assert torch.equal(t.q.view(torch.int16), q.view(torch.int16)) and torch.equal(t.k, k0) and torch.equal(t.v, v0)


def test_one_cta_to_a_windows_heads():
    """The grid of the largest prompts: six rounds of windows and more, every CTA takes all eight heads."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    rows = 6 * 3 * sms * 48 + 1000
    t = Tokens(geom((8, 8, 128)), rows, 16, seed=9)
    q, k = t.rotated()
    q_rot = torch.full_like(t.q, 7.0)
    got = t.append(t.q, q_rot)
    assert torch.equal(q_rot.view(torch.int16), q.view(torch.int16))
    t.check(got, k)
    t.check_on_the_host(got, k)


@pytest.mark.parametrize("heads", [(4, 1, 64), (8, 2, 128)])
def test_few_rows_in_place_and_without_queries(heads):
    t = Tokens(geom(heads), 500, 16, seed=4)
    q, k = t.rotated()
    got = t.append()
    t.check(got, k)
    assert _same(t.append(t.q, t.q), got)
    assert torch.equal(t.q.view(torch.int16), q.view(torch.int16))


@pytest.mark.parametrize("heads", [(4, 1, 64), (8, 2, 128)])
def test_step_form_without_queries(heads):
    """The same pages and scales as with the queries, in place or not."""
    from paper_2604_26209_b200 import binding as B
    g, n, P = geom(heads, cap=16), 300, 16
    gen = torch.Generator(device="cuda").manual_seed(6)
    rng = np.random.default_rng(6)
    rnd = lambda h: torch.randn(n, h, g.D, device="cuda", generator=gen).to(torch.bfloat16)                           # noqa: E731
    q, k, v = rnd(g.Hq), rnd(g.Hkv), rnd(g.Hkv)
    code = lambda: torch.randint(0, 256, (n, g.Hkv, P, g.D), dtype=torch.uint8, device="cuda", generator=gen)           # noqa: E731
    before = [code(), code()] + [torch.randint(115, 125, (n, g.Hkv), dtype=torch.uint8, device="cuda", generator=gen) for _ in range(2)]
    held, pos, table = rng.integers(0, P, n), rng.integers(0, 9000, n), rng.permutation(n)[:, None]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    results = []
    for a, b in ((q, torch.zeros_like(q)), (None, None), (q, q)):
        pools = [x.clone() for x in before]
        cache = B.PagedCache(pools[0].view(E4), pools[1].view(E4), pools[2].view(E8), pools[3].view(E8), i32(table))
        B.hpd_append_paged(g, n, n, i32([n]), None, None, None, i32(held), cache, i32(pos), a, b, k, v, status)
        results.append(pools)
    torch.cuda.synchronize()
    assert _same(results[0], results[1]) and _same(results[0], results[2]) and int(status.item()) == 0
