"""Tensors of another device than the current one are refused on the host: a kernel of the current device's stream would fault at their addresses."""
import pytest
import torch

from paper_2604_26209_b200 import binding as B, runtime, synth

pytestmark = pytest.mark.gpu


def _args(g, device, table_device=None):
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=device)                               # noqa: E731
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=device)                                # noqa: E731
    cache = B.PagedCache.alloc(g, 2, 1, 16, device=device)
    if table_device is not None:
        cache.table = cache.table.to(table_device)
    return g, 2, 2, i32(2), None, None, None, i32(0, 0), cache, None, None, None, z(2, g.Hkv, g.D), z(2, g.Hkv, g.D), i32(0)


def test_the_current_device_is_accepted():
    g = synth.Geom(Hq=4, Hkv=1, D=64, rope_theta=1e4, sm_scale=0.125, suffix_cap=16)
    B.hpd_append_paged(*_args(g, "cuda:0"))
    torch.cuda.synchronize()


@pytest.mark.skipif(not torch.cuda.is_available() or torch.cuda.device_count() < 2, reason="two devices")
def test_another_device_is_refused():
    g = synth.Geom(Hq=4, Hkv=1, D=64, rope_theta=1e4, sm_scale=0.125, suffix_cap=16)
    for args in (_args(g, "cuda:1"), _args(g, "cuda:0", "cuda:1"), _args(g, "cuda:1", "cuda:0")):
        with pytest.raises(AssertionError, match="current device"):
            B.hpd_append_paged(*args)
    s = synth.config_tiny()
    with pytest.raises(AssertionError, match="current device"):
        runtime.PagedBatch(s, synth.make_tensors(s), 16, device="cuda:1")
    with torch.cuda.device(1):
        B.hpd_append_paged(*_args(g, "cuda:1"))
        torch.cuda.synchronize(1)
