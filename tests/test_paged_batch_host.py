"""PagedBatch: structures that run under the position-order mask elsewhere are not given another mask in silence."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from paper_2604_26209_b200 import binding, runtime, synth


def _anchored():
    s = synth.config_tiny()
    return s, replace(s, slot_vis=s.doc_prefix_len[s.slot_doc()].astype(np.int32))


def test_position_order_is_refused():
    s, anchored = _anchored()
    t = synth.make_tensors(s)
    for structure, kw in ((anchored, {}), (anchored, dict(posorder=True)), (s, dict(posorder=True))):
        with pytest.raises(binding.HpdError, match="position-order"):
            runtime.PagedBatch(structure, t, 16, device="cpu", **kw)


@pytest.mark.gpu
def test_anchors_only():
    """Anchors at the documents' ends say what the structure without them says: the same bits."""
    s, anchored = _anchored()
    t = synth.make_tensors(s)
    made = []
    for structure, kw in ((s, {}), (anchored, dict(posorder=False))):
        pb = runtime.PagedBatch(structure, t, 16, **kw)
        pb.build_meta()
        act = pb.tables()["active_slot"][:pb.tables()["n_active"]]
        pb.set_step_inputs(t["q"][act], t["k_new"][act], t["v_new"][act])
        pb.step()
        torch.cuda.synchronize()
        assert pb.status() == 0
        made.append(pb)
    assert torch.equal(made[0].o, made[1].o) and torch.equal(made[0].lse, made[1].lse) and torch.equal(made[0].q_rot, made[1].q_rot)
