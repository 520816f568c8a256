"""hpd_attn_decode_paged against the plain implementation in 64 bits, with the bounds that its roundings allow."""
import numpy as np
import pytest
import torch

from paper_2604_26209_b200 import synth
from tests import paged_oracle as po

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


class Case:
    """Documents and branches over pools of pages in random order.  Every byte that no live token owns is random, NaN codes and all scales among them.

    k_exp / v_exp: the pages' scale bytes are drawn from that range."""

    def __init__(self, heads, P, lengths, branches, cap, depth=None, alive=None, seed=0, k_exp=(118, 122), v_exp=(118, 122), spare=3, q_scale=1.0):
        from paper_2604_26209_b200 import binding as B
        self.B = B
        Hq, Hkv, D = heads
        rng = np.random.default_rng(seed)
        self.rng = rng
        self.g = g = synth.Geom(Hq=Hq, Hkv=Hkv, D=D, rope_theta=10000.0, sm_scale=D ** -0.5, suffix_cap=cap)
        self.L, self.cnt = np.asarray(lengths), np.asarray(branches)
        n_docs, n_slots = len(self.L), int(self.cnt.sum())
        self.n_docs, self.n_slots = n_docs, n_slots
        self.depth = rng.integers(0, cap, n_slots) if depth is None else np.broadcast_to(np.asarray(depth), n_slots).copy()
        self.alive = np.ones(n_slots, bool) if alive is None else rng.random(n_slots) < alive
        need = -(-self.L // P)
        self.table = np.full((n_docs, max(1, int(need.max(initial=0)))), -1)
        order = rng.permutation(int(need.sum()) + spare)
        at = 0
        for d in range(n_docs):
            self.table[d, :need[d]] = order[at:at + need[d]]
            at += need[d]
        self.slot_page = rng.permutation(n_slots + spare)[:n_slots]

        def pool(pages, tokens):
            live = (rng.standard_normal((pages, Hkv, tokens, D)) * 100).clip(-448, 448)
            mk = lambda lo, hi: rng.integers(lo, hi, (pages, Hkv), dtype=np.uint8)                                     # noqa: E731
            k = po.encode(live)
            v = po.encode(live[::-1].transpose(0, 1, 2, 3) * rng.choice([-1, 1], (1, 1, 1, D)))
            return po.Pool(k, v, mk(*k_exp), mk(*v_exp))
        self.docs, self.branches = pool(len(order), P), pool(n_slots + spare, cap)
        # what nobody owns: any byte
        used = np.zeros((len(order), P), bool)
        for d in range(n_docs):
            for t in range(self.L[d]):
                used[self.table[d, t // P], t % P] = True
        mine = np.zeros((n_slots + spare, cap), bool)
        for s in range(n_slots):
            mine[self.slot_page[s], : min(cap, self.depth[s] + 1)] = True
        self.junk((self.docs, used), (self.branches, mine))
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.q = (torch.randn(max(n_slots, 1), Hq, D, device="cuda", generator=gen) * q_scale).to(torch.bfloat16)
        self.o = torch.full((max(n_slots, 1), Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((max(n_slots, 1), Hq), 7.0, device="cuda")

    def junk(self, *pools):
        for p, used in pools:
            for codes, scales in ((p.k, p.ks), (p.v, p.vs)):
                free = ~used
                rows = codes.transpose(0, 2, 1, 3)
                rows[free] = self.rng.integers(0, 256, (int(free.sum()), *rows.shape[2:]), dtype=np.uint8)
                empty = free.all(axis=1)
                scales[empty] = self.rng.integers(0, 256, (int(empty.sum()), scales.shape[1]), dtype=np.uint8)

    def upload(self):
        e4, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
        g = self.g
        up = lambda p, table: self.B.PagedCache(*[torch.from_numpy(x).cuda().view(e4) for x in (p.k, p.v)],            # noqa: E731
                                                *[torch.from_numpy(x).cuda().view(e8) for x in (p.ks, p.vs)], i32(table))
        self.dc, self.bc = up(self.docs, self.table), up(self.branches, self.slot_page.reshape(self.n_slots, 1))
        self.tL, self.tcnt, self.tdepth = i32(self.L), i32(self.cnt), i32(self.depth)
        self.talive = torch.from_numpy(self.alive.astype(np.uint8)).cuda()
        self.m = self.B.MetaTables.alloc(g, self.n_docs, self.n_slots, int(self.L.sum()))
        self.B.hpd_build_meta(g, self.n_docs, self.n_slots, self.tL, self.tcnt, self.tdepth, self.talive, 0, self.m)

    def attend(self, new=True, lse=True):
        self.B.hpd_attn_decode_paged(self.g, self.n_docs, self.n_slots, self.n_slots, self.q, self.dc, self.bc, self.tL, self.m, new, self.o,
                                     self.lse if lse else None)

    def rows(self):
        return np.flatnonzero(self.alive)

    def seen(self, slot, new=True):
        """Keys and values that a slot's row sees."""
        d = int(np.searchsorted(np.cumsum(self.cnt), slot, side="right"))
        n = min(int(self.depth[slot]) + int(new), self.g.suffix_cap)
        P = self.docs.k.shape[2]
        a = self.docs.tokens(self.table[d, : -(-self.L[d] // P)], int(self.L[d]))
        b = self.branches.tokens(self.slot_page[slot:slot + 1], n)
        return [np.concatenate(x) for x in zip(a, b)]

    def check(self, new=True, lse=True, some=None, status=0):
        torch.cuda.synchronize()
        rows = self.rows()
        q = self.q.float().cpu().numpy().astype(np.float64)
        got, gl = self.o.float().cpu().numpy(), self.lse.cpu().numpy()
        assert int(self.m.dev_status.item()) == status
        pick = range(len(rows)) if some is None or len(rows) <= some else self.rng.choice(len(rows), some, replace=False)
        for r in pick:
            K, V = self.seen(rows[r], new)
            o, l = po.attend(q[r], self.g.sm_scale, K, V)
            bo, bl = po.attention_bounds(q[r], self.g.sm_scale, K, V, o, l)
            err = np.abs(got[r] - o)
            assert np.all(err <= bo), (r, float((err - bo).max()), float((err / np.maximum(bo, 1e-30)).max()))
            if lse:
                if np.isneginf(l).all():
                    assert np.isneginf(gl[r]).all()
                else:
                    assert np.all(np.abs(gl[r] - l) <= bl), (r, float(np.abs(gl[r] - l).max()), float(bl.min()))
        assert (got[len(rows):] == 7).all() and (gl[len(rows) if lse else 0:] == 7).all()          # rows behind the last one


HEADS = [(4, 1, 64), (8, 2, 128), (2, 2, 128), (16, 2, 64), (8, 1, 128), (4, 2, 128)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("P", [16, 32, 64])
def test_ragged_documents(heads, P):
    """Lengths of 0, 1 and around pages and tiles, 0 to 40 branches, branches of 0 to cap tokens, half of them retired."""
    c = Case(heads, P, [0, 1, P - 1, P, P + 1, 63, 64, 65, 127, 130, 300, 511], [3, 1, 5, 0, 40, 7, 2, 1, 33, 4, 20, 9], 9, alive=0.6, seed=P)
    c.upload()
    c.attend()
    c.check(some=80)


@pytest.mark.parametrize("heads", [(4, 1, 64), (8, 2, 128)])
@pytest.mark.parametrize("cap,depth", [(1, 0), (16, 15), (16, 0), (30, None), (70, None), (200, 199)])
def test_branch_pages(heads, cap, depth):
    """Branches of one token, full ones, pages of more than a tile; the whole tile of rows."""
    c = Case(heads, 64, [40, 200], [33, 20], cap, depth=depth, seed=cap)
    c.upload()
    c.attend()
    c.check(some=50)
    for new, lse in ((False, True), (True, False)):
        c.o.fill_(7)
        c.lse.fill_(7)
        c.attend(new=new, lse=lse)
        c.check(new=new, lse=lse, some=20)


@pytest.mark.parametrize("heads", [(4, 1, 64), (8, 2, 128), (2, 2, 128)])
def test_rows_that_see_nothing(heads):
    """Empty documents whose branches hold nothing: zeros and -inf, next to rows that see something."""
    c = Case(heads, 32, [0, 5, 0, 0], [3, 2, 4, 1], 4, depth=[0, 1, 0, 0, 2, 0, 0, 3, 0, 0], seed=1)
    c.upload()
    c.attend(new=False)
    c.check(new=False)
    assert bool((c.o[0] == 0).all()) and bool(torch.isneginf(c.lse[0]).all())


@pytest.mark.parametrize("lengths,branches,P", [([9000], [5], 64), ([5000, 3100], [24, 3], 16), ([2049, 700, 4096], [2, 1, 40], 32)])
def test_few_long_documents_are_split(lengths, branches, P):
    c = Case((8, 2, 128), P, lengths, branches, 8, seed=len(lengths))
    c.upload()
    c.attend()
    c.check(some=12)
    c.o.fill_(7)
    c.attend()                                            # again on the same tables
    c.check(some=4)


@pytest.mark.parametrize("heads", [(4, 1, 64), (8, 2, 128)])
def test_many_units(heads):
    """More units than pipelines: fixed rounds and the ticket counter."""
    c = Case(heads, 16, np.random.default_rng(2).integers(1, 90, 2100), np.random.default_rng(3).integers(0, 4, 2100), 5, seed=4)
    c.upload()
    c.attend()
    c.check(some=60)


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 1, 64), (2, 2, 128), (8, 1, 64)])
@pytest.mark.parametrize("P", [16, 64])
def test_rows_in_two_ways(heads, P):
    """Enough units that none is halved, few rows on average: units of up to 64 rows and eight tiles or more have their rows twice in the tile, the others
    once, in the same launch; 64 and 65 rows, 7 and 8 tiles, branches of several tiles and none."""
    G = heads[0] // heads[1]
    rng = np.random.default_rng(P)
    docs = 170 // heads[1]
    L = rng.integers(440, 700, docs)
    L[:8] = [448, 449, 512, 511, 1100, 64, 0, 1]
    n = rng.integers(0, 64 // G // 2, docs)
    n[:8] = [64 // G, 64 // G + 1, 64 // G, 1, 128 // G, 3, 2, 64 // G]
    c = Case(heads, P, L, n, 7, seed=P + heads[0], alive=0.9)
    c.upload()
    c.attend()
    c.check(some=60)
    for d in range(8):                                    # the first documents' first and last row
        rows = np.flatnonzero(np.repeat(np.arange(docs), n)[c.rows()] == d)
        q = c.q.float().cpu().numpy().astype(np.float64)
        for r in rows[[0, -1]] if len(rows) else []:
            K, V = c.seen(c.rows()[r])
            o, l = po.attend(q[r], c.g.sm_scale, K, V)
            bo, bl = po.attention_bounds(q[r], c.g.sm_scale, K, V, o, l)
            assert np.all(np.abs(c.o[r].float().cpu().numpy() - o) <= bo) and np.all(np.abs(c.lse[r].cpu().numpy() - l) <= bl), (d, r)


def test_two_ways_with_scales_of_all_sizes_and_one_visible_half():
    """Two ways whose references differ by hundreds: pages of very different scales, scores that leave one token, branches in one half of a tile."""
    for seed, k_exp, v_exp, q_scale in ((31, (118, 122), (60, 190), 1.0), (32, (122, 126), (118, 122), 8.0), (33, (60, 61), (1, 40), 30.0)):
        c = Case((8, 2, 128), 16, [520 + 7 * (i % 9) for i in range(90)], [1 + i % 5 for i in range(90)], 70, depth=[(13 * i) % 69 for i in range(270)],
                 seed=seed, k_exp=k_exp, v_exp=v_exp, q_scale=q_scale)
        c.upload()
        c.attend()
        c.check(some=50)


@pytest.mark.parametrize("k_exp,v_exp,q_scale", [((60, 61), (100, 160), 1.0), ((105, 122), (60, 190), 1.0), ((120, 121), (1, 40), 30.0),
                                                 ((1, 3), (230, 240), 1e3), ((200, 210), (119, 121), 1e-25)])
def test_scales_of_all_sizes(k_exp, v_exp, q_scale):
    """Pages whose scales differ by many powers of two, in keys and in values; tiny and large queries."""
    c = Case((8, 2, 128), 16, [200, 77, 1000], [9, 5, 3], 12, seed=5, k_exp=k_exp, v_exp=v_exp, q_scale=q_scale)
    c.upload()
    c.attend()
    c.check()


def test_scores_that_leave_one_token():
    """Scores of hundreds: the softmax is one token's, whichever tile it stands in; the maximum grows from tile to tile."""
    c = Case((8, 2, 128), 64, [640, 100], [6, 6], 12, seed=6, k_exp=(122, 126), q_scale=8.0)
    c.upload()
    c.attend()
    c.check()


def test_documents_may_share_pages():
    c = Case((8, 2, 128), 32, [100, 200, 64], [5, 6, 7], 6, seed=7)
    c.table[1, :3] = c.table[0, :3]
    c.table[2] = -1
    c.table[2, :2] = c.table[0, :2]
    c.upload()
    c.attend()
    c.check()


def _bits(t):
    return t.view(torch.int16) if t.dtype == torch.bfloat16 else t.view(torch.int32)


def test_nan_reaches_its_own_rows_only():
    """A NaN code in a document's key or value: its document's rows; in a branch's key or value: that branch's row; the others keep their bits."""
    def outputs(change=None, heads=(8, 2, 128)):
        c = Case(heads, 32, [100, 70, 130], [5, 40, 7], 6, depth=3, seed=8)
        if change:
            change(c)
        c.upload()
        c.attend()
        torch.cuda.synchronize()
        assert int(c.m.dev_status.item()) == 0
        return c, c.o.clone(), c.lse.clone()
    doc = np.repeat([0, 1, 2], [5, 40, 7])
    for heads in ((8, 2, 128), (4, 1, 64)):
        _, o0, l0 = outputs(heads=heads)
        for what, hit in (("k doc", doc == 1), ("v doc", doc == 1), ("k branch", np.arange(52) == 7), ("v branch", np.arange(52) == 7), ("q", np.arange(52) == 7)):
            def change(c):
                which, _, where = what.partition(" ")
                if which == "q":
                    c.q[7, 0, 5] = float("inf")
                elif where == "doc":
                    getattr(c.docs, which)[c.table[1, 2], 0, 5, 9] = 0xff
                else:
                    getattr(c.branches, which)[c.slot_page[7], 0, 1, 9] = 0x7f
            c, o, l = outputs(change, heads)
            G = heads[0] // heads[1]
            mine = torch.from_numpy(np.flatnonzero(hit)).cuda()
            rest = torch.from_numpy(np.flatnonzero(~hit)).cuda()
            head = slice(0, 1) if what == "q" else slice(0, G)
            bad = torch.isnan(o[mine][:, head])
            assert bool((bad[..., 9] if what == "v doc" else bad).all()), what
            if what == "v doc":
                assert int(bad.sum()) == bad[..., 9].numel()                   # the others of its elements are numbers
            assert torch.equal(_bits(o[rest]), _bits(o0[rest])) and torch.equal(_bits(l[rest]), _bits(l0[rest])), what
            assert torch.equal(_bits(o[mine][:, G:]), _bits(o0[mine][:, G:])), what            # other kv heads


def test_bad_pages():
    """Pages out of range: a status bit; a document's rows are NaN, a branch without its page sees the document only; the others are right."""
    for value in (-1, 10 ** 6, -2 ** 31, 2 ** 31 - 1):
        c = Case((8, 2, 128), 32, [100, 70, 130], [5, 4, 7], 6, seed=9)
        c.table[1, 2] = value
        c.slot_page[11] = value
        c.upload()
        c.attend()
        torch.cuda.synchronize()
        assert int(c.m.dev_status.item()) == po.S_BAD_TABLE
        assert bool(torch.isnan(c.o[5:9]).all()) and bool(torch.isnan(c.lse[5:9]).all())
        q = c.q.float().cpu().numpy().astype(np.float64)
        for r in (0, 4, 9, 10, 11, 15):
            if r == 11:
                K, V = c.docs.tokens(c.table[2, :5], 130)
            else:
                K, V = c.seen(r)
            o, l = po.attend(q[r], c.g.sm_scale, K, V)
            bo, bl = po.attention_bounds(q[r], c.g.sm_scale, K, V, o, l)
            assert np.all(np.abs(c.o[r].float().cpu().numpy() - o) <= bo) and np.all(np.abs(c.lse[r].cpu().numpy() - l) <= bl), r


def test_documents_longer_than_their_table():
    c = Case((8, 2, 128), 32, [64, 70], [5, 4], 6, seed=10)
    c.upload()
    c.tL = i32([64, 97])                                  # three pages in the table, four needed
    c.B.hpd_build_meta(c.g, 2, 9, c.tL, c.tcnt, c.tdepth, c.talive, 0, c.m)
    c.attend()
    torch.cuda.synchronize()
    assert int(c.m.dev_status.item()) == po.S_BAD_TABLE
    assert bool(torch.isnan(c.o[5:9]).all()) and not bool(torch.isnan(c.o[:5]).any())


def test_no_documents_pages_at_all():
    """Empty documents over a pool without pages: the branches alone."""
    c = Case((8, 2, 128), 64, [0, 0], [3, 4], 6, seed=11, spare=1)
    c.docs = po.Pool(*[x[:1] for x in (c.docs.k, c.docs.v, c.docs.ks, c.docs.vs)])
    c.upload()
    c.attend()
    c.check()


def test_pools_beyond_32_bits():
    """Codes beyond 2^32 bytes into a pool."""
    from paper_2604_26209_b200 import binding as B
    c = Case((8, 8, 128), 64, [130, 64], [3, 2], 8, seed=12)
    c.upload()
    n = 2 ** 32 // (8 * 64 * 128) + 8
    far = n - 1 - np.arange(len(c.docs.k))
    big = [torch.full((n, 8, 64, 128), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(2)]
    sc = [torch.full((n, 8), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    at = torch.from_numpy(far).cuda()
    for x, y in zip(big + sc, (c.docs.k, c.docs.v, c.docs.ks, c.docs.vs)):
        x[at] = torch.from_numpy(y).cuda()
    table = np.where(c.table >= 0, far[np.clip(c.table, 0, None)], -1)
    c.dc = B.PagedCache(*[x.view(torch.float8_e4m3fn) for x in big], *[x.view(torch.float8_e8m0fnu) for x in sc], i32(table))
    c.attend()
    c.check()


def test_captured_on_another_stream_and_repeatable():
    """A graph on a stream of its own gives the bits of the direct call, every time."""
    c = Case((8, 2, 128), 32, [700, 90, 333], [20, 24, 9], 10, seed=13)
    c.upload()
    c.attend()
    torch.cuda.synchronize()
    o, l = c.o.clone(), c.lse.clone()
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            c.attend()
        for _ in range(3):
            c.o.fill_(7)
            c.lse.fill_(7)
            graph.replay()
            assert torch.equal(_bits(c.o), _bits(o)) and torch.equal(_bits(c.lse), _bits(l))
    s.synchronize()
    c.check(some=10)
