"""Rows that hold a NaN under hpd_attn_decode: the same answer whether their document was split or not."""
import numpy as np
import pytest
import torch

from paper_2604_26209_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 1, 64)])
@pytest.mark.parametrize("lengths,split", [([3000, 700], True), ([200, 100], False)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_log_sum_of_a_row_of_nan(heads, lengths, split, value):
    """The row's output is NaN and its log-sum-exp -inf (the sum is not above zero); the other rows keep their bits."""
    from paper_2604_26209_b200 import binding as B
    Hq, Hkv, D = heads
    cnt, cap = [5, 3], 4
    n, T = sum(cnt), sum(lengths)
    g = synth.Geom(Hq=Hq, Hkv=Hkv, D=D, rope_theta=10000.0, sm_scale=D ** -0.5, suffix_cap=cap)
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()                  # noqa: E731
    gen = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen).to(torch.bfloat16)                 # noqa: E731
    q, pk, pv, sk, sv = rnd(n, Hq, D), rnd(T, Hkv, D), rnd(T, Hkv, D), rnd(n * cap, Hkv, D), rnd(n * cap, Hkv, D)
    L, m = i32(lengths), B.MetaTables.alloc(g, 2, n, T)
    B.hpd_build_meta(g, 2, n, L, i32(cnt), i32(np.full(n, 2)), torch.ones(n, dtype=torch.uint8, device="cuda"), 0, m)

    def attend(q):
        o, lse = torch.zeros(n, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, Hq, device="cuda")
        B.hpd_attn_decode(g, 2, n, n, T, q, pk, pv, sk, sv, L, m, True, o, lse)
        torch.cuda.synchronize()
        return o, lse
    o0, l0 = attend(q)
    assert bool(m.workspace.cpu().numpy()[:32].view(np.int32)[3]) == split
    q[2, 0, 5] = value
    o, lse = attend(q)
    assert bool(torch.isnan(o[2, 0]).all()) and bool(torch.isneginf(lse[2, 0]))
    o[2, 0], lse[2, 0] = o0[2, 0], l0[2, 0]
    assert torch.equal(o, o0) and torch.equal(lse, l0)
