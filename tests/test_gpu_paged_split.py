"""hpd_attn_decode_paged where a row's result comes from several places: documents split over work items and merged, units whose rows stand twice
in the tile.  NaN and pages out of range there, and values at the top of the range."""
import copy
import functools

import numpy as np
import pytest
import torch

from tests import paged_oracle as po
from tests.test_gpu_paged_attn import Case, _bits

pytestmark = pytest.mark.gpu

# name: heads, page size, documents' tokens, branches, whether the plan splits documents.  The document that is changed is number 1.
SHAPES = {
    # few documents: chunks of 512 tokens, units halved, rows twice in the tile
    "split": ((8, 2, 128), 16, [700, 3000, 130], [9, 5, 3], True),
    # units of more than 64 rows
    "split_full_units": ((8, 2, 64), 32, [700] * 40, [20] * 40, True),
    # whole documents of eight tiles and more, up to 64 rows: the two halves of every tile apart
    "two_ways": ((8, 2, 128), 16, [600, 577, 520] * 30, [3, 9, 14] * 30, False),
    "two_ways_d64": ((4, 1, 64), 16, [600, 577, 520] * 55, [3, 9, 14] * 55, False),
}


@functools.lru_cache(maxsize=1)
def _made(name):
    heads, P, lengths, branches, _ = SHAPES[name]
    return Case(heads, P, lengths, branches, 6, depth=3, seed=len(lengths))


def _case(name, change=None):
    """A call over a copy of the case's pools, changed."""
    split, made = SHAPES[name][4], _made(name)
    c = copy.copy(made)
    c.docs, c.branches = (po.Pool(p.k, p.v, p.ks, p.vs) for p in (made.docs, made.branches))
    c.table, c.q, c.o, c.lse = made.table.copy(), made.q.clone(), made.o.clone(), made.lse.clone()
    if change:
        change(c)
    c.upload()
    c.attend()
    torch.cuda.synchronize()
    header = c.m.workspace.cpu().numpy()[:32].view(np.int32)
    assert bool(header[3]) == split and (not split or (header[1] == 512 and header[2] > 0)), header
    return c


def _places(length):
    """Tokens of a document: both halves of a tile in its first chunk, one in the middle, its last whole tile's halves, and its last token."""
    last = length // 64 * 64
    return [5, 40, length // 2, last - 60, last - 3, length - 1]


@pytest.mark.parametrize("name", list(SHAPES))
def test_right_without_a_change(name):
    _case(name).check(some=30)


@pytest.mark.parametrize("name", list(SHAPES))
def test_nan_reaches_its_own_rows_only(name):
    base = _case(name)
    heads, P, lengths, branches, _ = SHAPES[name]
    G, n = heads[0] // heads[1], sum(branches)
    doc = np.repeat(np.arange(len(branches)), branches)
    row = branches[0] + 2                                 # a branch of document 1
    kinds = [(which, "doc", t) for which in "kv" for t in _places(lengths[1])] + [(which, "branch", 1) for which in "kv"] + [("q", "", 0)]
    for which, where, t in kinds:
        def change(c):
            if where == "doc":
                getattr(c.docs, which)[c.table[1, t // P], 0, t % P, 9] = 0xff
            elif where == "branch":
                getattr(c.branches, which)[c.slot_page[row], 0, t, 9] = 0x7f
            else:
                c.q[row, 0, 5] = float("inf")
        c = _case(name, change)
        assert int(c.m.dev_status.item()) == 0
        hit = doc == 1 if where == "doc" else np.arange(n) == row
        mine, rest = (torch.from_numpy(np.flatnonzero(x)).cuda() for x in (hit, ~hit))
        head = slice(0, G) if where else slice(0, 1)
        bad = torch.isnan(c.o[mine][:, head])
        if (which, where) == ("v", "doc"):
            assert bool(bad[..., 9].all()) and int(bad.sum()) == bad[..., 9].numel(), (which, where, t)       # the others of its elements are numbers
            assert torch.equal(_bits(c.lse[mine]), _bits(base.lse[mine])), (which, where, t)
        else:
            assert bool(bad.all()) and bool(torch.isnan(c.lse[mine][:, head]).all()), (which, where, t)
        assert torch.equal(_bits(c.o[rest]), _bits(base.o[rest])) and torch.equal(_bits(c.lse[rest]), _bits(base.lse[rest])), (which, where, t)
        assert torch.equal(_bits(c.o[mine][:, G:]), _bits(base.o[mine][:, G:])), (which, where, t)            # other kv heads


@pytest.mark.parametrize("name", list(SHAPES))
def test_bad_pages(name):
    """A page out of range anywhere in a document: a status bit, the document's rows are NaN, the others keep their bits."""
    base = _case(name)
    _, P, lengths, branches, _ = SHAPES[name]
    doc = np.repeat(np.arange(len(branches)), branches)
    mine, rest = (torch.from_numpy(np.flatnonzero(x)).cuda() for x in (doc == 1, doc != 1))
    for t, value in zip(_places(lengths[1]), (-1, 10 ** 6, -2 ** 31, 2 ** 31 - 1, -1, 10 ** 6)):
        c = _case(name, lambda c: c.table.__setitem__((1, t // P), value))
        assert int(c.m.dev_status.item()) == po.S_BAD_TABLE, t
        assert bool(torch.isnan(c.o[mine]).all()) and bool(torch.isnan(c.lse[mine]).all()), t
        assert torch.equal(_bits(c.o[rest]), _bits(base.o[rest])) and torch.equal(_bits(c.lse[rest]), _bits(base.lse[rest])), t


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("v_exp", [(240, 241), (243, 246)])
def test_values_at_the_top_of_the_range(name, v_exp):
    """Values of one sign of up to 2^122 and 2^127 (a bf16 holds them): their weighted mean is a number, however many tokens it is of."""
    def change(c):
        for p in (c.docs, c.branches):
            p.v &= 0x7f
            p.v[p.v == 0x7f] = 0x7e
            p.vs[:] = c.rng.integers(*v_exp, p.vs.shape)
    c = _case(name, change)
    assert bool(torch.isfinite(c.o.float()).all())
    c.check(some=30)


@pytest.mark.parametrize("heads", [(4, 1, 64), (8, 2, 128)])
def test_rows_that_see_nothing_whatever_their_queries(heads):
    """Zeros and -inf for a row without a token, an infinity or NaN in its q or not; a row with tokens is NaN."""
    c = Case(heads, 32, [0, 5], [3, 2], 4, depth=[0, 0, 1, 0, 0], seed=2)
    c.q[0, 0, 3], c.q[1, 0, 3], c.q[2, 0, 3], c.q[3, 0, 3] = float("inf"), float("nan"), float("nan"), float("inf")
    c.upload()
    c.attend(new=False)
    torch.cuda.synchronize()
    assert bool((c.o[:2] == 0).all()) and bool(torch.isneginf(c.lse[:2]).all())
    assert bool(torch.isnan(c.o[2:4, 0]).all()) and bool(torch.isnan(c.lse[2:4, 0]).all())
    assert bool(torch.isfinite(c.o[2:, 1:].float()).all()) and int(c.m.dev_status.item()) == 0
