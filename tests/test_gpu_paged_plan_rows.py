"""hpd_attn_decode_paged whose row tables were moved after the work list was made: the tables passed decide, as with hpd_attn_decode."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from tests.test_gpu_paged_attn import Case

pytestmark = pytest.mark.gpu

MOVED = 37
# name: (Hq, Hkv, D), documents' tokens, branches (both repeated over the documents), documents, split or not
CALLS = {"own": ((8, 2, 128), [200, 3, 90], [9, 70, 1], 60, False), "own_d64": ((4, 4, 64), [60, 0, 130], [50, 2, 33], 50, False),
         "two_ways": ((8, 2, 128), [520, 700, 64], [9, 3, 12], 90, False), "halves": ((4, 1, 64), [300], [50], 1, False),
         "split": ((8, 2, 128), [3000, 2000], [4, 30], 2, True), "split_full_units": ((8, 2, 64), [700], [20], 40, True)}


@pytest.mark.parametrize("name", list(CALLS))
def test_tables_moved_after_the_list_was_made(name):
    """The same rows 37 places further in every row table, with the list of the tables as they were: the same output, 37 places further."""
    heads, lens, cnts, docs, split = CALLS[name]
    L, cnt = np.resize(lens, docs + 1), np.resize(cnts, docs + 1)
    cnt[-1] = 0                                                       # no rows: the merge passes over the rows in front, which are given to it
    c = Case(heads, 32, L, cnt, 5, seed=docs)
    c.upload()
    n, rows = c.n_slots, c.n_slots + MOVED
    torch.cuda.synchronize()
    assert bool(c.m.workspace.cpu().numpy()[:32].view(np.int32)[3]) == split

    def attend(m, q):
        o, lse = torch.full((rows, *q.shape[1:]), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((rows, heads[0]), 7.0, device="cuda")
        c.B.hpd_attn_decode_paged(c.g, docs + 1, rows, n, q, c.dc, c.bc, c.tL, m, True, o, lse)
        torch.cuda.synchronize()
        return o, lse

    def later(t, fill):
        return torch.cat([torch.full((MOVED,), fill, dtype=t.dtype, device="cuda"), t])
    other = torch.randn(MOVED, *c.q.shape[1:], device="cuda").to(torch.bfloat16)
    want, want_lse = attend(c.m, torch.cat([c.q, other]))
    c.o, c.lse = want[:n], want_lse[:n]
    c.check(some=20)
    moved = replace(c.m, doc_active_start=c.m.doc_active_start + MOVED, n_active=c.m.n_active + MOVED, doc_id=later(c.m.doc_id, docs),
                    active_slot=later(c.m.active_slot, 0), suffix_len=later(c.m.suffix_len, 0))
    got, got_lse = attend(moved, torch.cat([other, c.q]))
    assert int(c.m.dev_status.item()) == 0
    assert torch.equal(got[MOVED:], want[:n]) and torch.equal(got_lse[MOVED:], want_lse[:n])
    assert bool((got[:MOVED] == 7).all()) and bool((got_lse[:MOVED] == 7).all())
