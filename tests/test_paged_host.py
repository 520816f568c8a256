"""The paged operators before anything reaches a GPU: what they refuse, and the plain implementation that the GPU tests go by."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2604_26209_b200 import binding, synth
from tests import paged_oracle as po

GEOM = binding.HpdGeom(8, 2, 128, 10000.0, 0.1, 16)
FAKE = 0x1000                                            # an address that no refused call looks at


def _append(geom=GEOM, n_seqs=1, max_rows=1, n_rows=FAKE, row_seq=None, seq_row_start=None, seq_id=None, seq_len=FAKE, table=FAKE, table_rows=1,
            pages_per_seq=1, n_pages=1, page_size=16, pos=None, q=None, q_rot=None, k=FAKE, v=FAKE, pk=FAKE, pv=FAKE, sk=FAKE, sv=FAKE):
    return binding.load().hpd_append_paged(C.byref(geom), n_seqs, max_rows, n_rows, row_seq, seq_row_start, seq_id, seq_len, table, table_rows,
                                           pages_per_seq, n_pages, page_size, pos, q, q_rot, k, v, pk, pv, sk, sv, None, None)


@pytest.mark.parametrize("change,code", [
    (dict(geom=binding.HpdGeom(8, 2, 96, 10000.0, 0.1, 16)), -2), (dict(geom=binding.HpdGeom(6, 2, 128, 10000.0, 0.1, 16)), -2),
    (dict(max_rows=-1), -1), (dict(n_seqs=-1), -1), (dict(page_size=0), -1), (dict(n_pages=-1), -1), (dict(table_rows=-1), -1), (dict(pages_per_seq=-1), -1),
    (dict(row_seq=FAKE), -1), (dict(seq_row_start=FAKE), -1),               # half of the token form
    (dict(q=FAKE, pos=FAKE), -1), (dict(q_rot=FAKE, pos=FAKE), -1),         # queries with nowhere to go, and the other way round
    (dict(q=FAKE, q_rot=FAKE), -1),                                         # queries without positions
    (dict(n_rows=None), -1), (dict(seq_len=None), -1), (dict(table=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(pk=None), -1),
    (dict(pv=None), -1), (dict(sk=None), -1), (dict(sv=None), -1),
    (dict(k=FAKE + 2), -1), (dict(v=FAKE + 8), -1), (dict(pk=FAKE + 1), -1), (dict(pv=FAKE + 4), -1), (dict(pos=FAKE, q=FAKE + 2, q_rot=FAKE), -1),
    (dict(row_seq=FAKE, seq_row_start=FAKE, page_size=65), -4), (dict(page_size=65536), -4),
    (dict(max_rows=0, k=None), 0), (dict(n_seqs=0, table=None), 0)])        # nothing to do
def test_append_refuses(change, code):
    assert _append(**change) == code


def _attend(geom=GEOM, n_docs=1, max_rows=1, n_slots=1, q=FAKE, pk=FAKE, pv=FAKE, sk=FAKE, sv=FAKE, doc_page=FAKE, pages_per_doc=1, n_pages=1,
            page_size=64, bk=FAKE, bv=FAKE, bsk=FAKE, bsv=FAKE, slot_page=FAKE, n_branch_pages=1, L=FAKE, das=FAKE, doc_id=FAKE, active=FAKE, slen=FAKE,
            n_active=FAKE, o=FAKE, ws=FAKE, wsb=1 << 40):
    return binding.load().hpd_attn_decode_paged(C.byref(geom), n_docs, max_rows, n_slots, q, pk, pv, sk, sv, doc_page, pages_per_doc, n_pages,
                                                page_size, bk, bv, bsk, bsv, slot_page, n_branch_pages, L, das, doc_id, active, slen, n_active, 1, o, None,
                                                ws, wsb, None, None)


@pytest.mark.parametrize("change,code", [
    (dict(geom=binding.HpdGeom(8, 2, 32, 10000.0, 0.1, 16)), -2), (dict(geom=binding.HpdGeom(8, 2, 128, 10000.0, 0.0, 16)), -2),
    (dict(geom=binding.HpdGeom(8, 2, 128, 10000.0, float("nan"), 16)), -2),
    (dict(n_docs=-1), -1), (dict(max_rows=-1), -1), (dict(n_slots=-1), -1), (dict(pages_per_doc=-1), -1), (dict(n_pages=-1), -1), (dict(n_branch_pages=-1), -1),
    (dict(page_size=0), -1), (dict(page_size=8), -1), (dict(page_size=48), -1), (dict(page_size=128), -1),
    (dict(geom=binding.HpdGeom(8, 2, 128, 10000.0, 0.1, 4093)), -4),                              # packed columns beyond 16 bits
    (dict(n_pages=1 << 24, page_size=64), -4), (dict(n_branch_pages=1 << 26), -4),                # 2^31 rows of codes
    *[(dict([(name, None)]), -1) for name in ("q", "pk", "pv", "sk", "sv", "doc_page", "bk", "bv", "bsk", "bsv", "slot_page", "L", "das", "doc_id", "active",
                                              "slen", "n_active", "o", "ws")],
    *[(dict([(name, FAKE + 8)]), -1) for name in ("q", "pk", "pv", "bk", "bv", "o", "ws")],
    (dict(wsb=16), -3), (dict(max_rows=0, q=None), 0), (dict(n_docs=0, o=None), 0)])
def test_attention_refuses(change, code):
    assert _attend(**change) == code


def _cache(n=3, H=2, P=16, D=64, rows=2, per=1):
    z = lambda *s: torch.zeros(*s, dtype=torch.uint8)                                              # noqa: E731
    return dict(k=z(n, H, P, D).view(torch.float8_e4m3fn), v=z(n, H, P, D).view(torch.float8_e4m3fn), k_scale=z(n, H).view(torch.float8_e8m0fnu),
                v_scale=z(n, H).view(torch.float8_e8m0fnu), table=torch.zeros(rows, per, dtype=torch.int32))


def test_cache_objects_are_checked():
    good = _cache()
    binding.PagedCache(**good)
    for change in (dict(k=torch.zeros(3, 2, 16, 64)), dict(v=_cache(n=4)["v"]), dict(k_scale=torch.zeros(3, 2)), dict(v_scale=_cache(H=1)["v_scale"]),
                   dict(table=torch.zeros(2, 1)), dict(table=torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(binding.HpdError):
            binding.PagedCache(**{**good, **change})
    own = binding.PagedCache.alloc(synth.Geom(4, 2, 64, 1e4, 0.1, 8), 3, 2, 32, device="cpu")
    assert own.table.tolist() == [[0, 1], [2, 3], [4, 5]] and tuple(own.k.shape) == (6, 2, 32, 64) and own.page_size == 32 and own.n_pages == 6
    left = binding.PagedCache.alloc(synth.Geom(4, 2, 64, 1e4, 0.1, 8), 3, 2, 32, n_pages=5, device="cpu")
    assert left.table.tolist() == [[-1, -1]] * 3 and left.n_pages == 5


def test_cache_and_geometry_have_to_agree():
    g = synth.Geom(Hq=4, Hkv=2, D=64, rope_theta=1e4, sm_scale=0.1, suffix_cap=16)
    c, wrong = binding.PagedCache(**_cache()), binding.PagedCache(**_cache(H=1))
    with pytest.raises(binding.HpdError, match="heads"):
        binding.hpd_append_paged(g, 1, 1, None, None, None, None, None, wrong, None, None, None, None, None, None)
    for docs, branches, n_docs, n_slots in ((wrong, c, 1, 2), (c, wrong, 1, 2), (c, binding.PagedCache(**_cache(P=8)), 1, 2), (c, c, 1, 3), (c, c, 3, 2),
                                            (c, binding.PagedCache(**_cache(per=2)), 1, 2)):
        with pytest.raises(binding.HpdError):
            binding.hpd_attn_decode_paged(g, n_docs, 1, n_slots, None, docs, branches, None, None, True, None)


# ------------------------------------------------ the plain implementation itself ------------------------------------------------
def test_codes_are_torchs():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(po.VALUES, want, equal_nan=True)
    x = np.concatenate([np.linspace(-450, 450, 20001), 2.0 ** np.linspace(-12, 8.8, 5000), (po.GRID[:-1] + po.GRID[1:]) / 2])
    x = x[np.abs(x) <= 448]
    assert np.array_equal(po.encode(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert po.encode(np.array([np.inf, -np.inf, np.nan, 1e9])).tolist() == [0x7e, 0xfe, 0x7f, 0x7e]


def test_scales_are_the_smallest_that_reach():
    for a in (448.0, 449.0, 1.75, 1.7578125, 2.0, 1e-39, 3.3e38, 0.0, 448.0 * 2.0 ** -126):
        b = po.needed(np.array([[a, -a / 3, np.nan, np.inf]]))
        assert a <= 448 * po.scale_value(b) and (b == 1 or a > 224 * po.scale_value(b))


def test_a_page_filled_token_by_token_has_the_codes_of_one_filled_at_once():
    """Powers of two as scales: growth is exact for elements above 2^-14 of the page's largest, which these all are."""
    rng = np.random.default_rng(0)
    x = rng.choice([-1, 1], (16, 1, 64)) * rng.integers(8, 16, (16, 1, 64)) * 2.0 ** rng.integers(-6, 6, (16, 1, 64))
    empty = lambda: po.Pool(*[np.zeros((1, 1, 16, 64), np.uint8)] * 2, *[np.zeros((1, 1), np.uint8)] * 2)             # noqa: E731
    one, many = empty(), empty()
    one.append(0, 0, x, x)
    for t in range(16):
        many.append(0, t, x[t:t + 1], x[t:t + 1])
    assert np.array_equal(one.k, many.k) and np.array_equal(one.ks, many.ks)
