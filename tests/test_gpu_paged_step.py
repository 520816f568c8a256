"""The paged operators as a decode loop uses them: first step, tables, append, attention and end of step, one after another."""
import numpy as np
import pytest
import torch

from paper_2604_26209_b200 import synth
from tests import paged_oracle as po

pytestmark = pytest.mark.gpu


def _pool(c):
    return po.Pool(*[x.view(torch.uint8).cpu().numpy() for x in (c.k, c.v, c.k_scale, c.v_scale)])


def _wide(t):
    return t.float().cpu().numpy().astype(np.float64)


def _check_rows(g, q, o, lse, docs, doc_table, L, branches, slot_page, doc, slots, tokens, some):
    rng = np.random.default_rng(len(slots))
    for r in (range(len(slots)) if len(slots) <= some else rng.choice(len(slots), some, replace=False)):
        d, s, P = int(doc[r]), int(slots[r]), docs.k.shape[2]
        a = docs.tokens(doc_table[d, : -(-int(L[d]) // P)], int(L[d]))
        b = branches.tokens(slot_page[s:s + 1], int(tokens[r]))
        K, V = (np.concatenate(x) for x in zip(a, b))
        want, want_l = po.attend(q[r], g.sm_scale, K, V)
        bo, bl = po.attention_bounds(q[r], g.sm_scale, K, V, want, want_l)
        assert np.all(np.abs(o[r] - want) <= bo) and np.all(np.abs(lse[r] - want_l) <= bl), r


@pytest.mark.parametrize("cfg,page_size", [
    (lambda: synth.config_tiny(), 16), (lambda: synth.config_main(n_prompts=1), 64),
    (lambda: synth.config_custom("ragged", 16, 4, 128, 1e4, 12, [0, 1, 70, 300, 129], [3, 1, 20, 33, 0], 12, alive_frac=0.7), 32),
    (lambda: synth.config_custom("g1", 4, 4, 64, 1e4, 5, [33, 200], [6, 9], 5, pos_gap=5), 16)])
def test_a_step_of_a_batch(cfg, page_size):
    """PagedBatch: filled from bf16 caches, one step; every cached token of every slot and the attention against 64 bits."""
    from paper_2604_26209_b200 import binding as B, runtime
    s = cfg()
    g, t = s.geom, synth.make_tensors(s)
    pb = runtime.PagedBatch(s, t, page_size)
    # what the pages hold: codes of the batch's bf16 values, pages filled as the calls fill them
    docs, branches = _pool(pb.docs), _pool(pb.branches)
    doc_table = pb.docs.table.cpu().numpy()
    want = po.Pool(*[np.zeros_like(x) for x in (docs.k, docs.v, docs.ks, docs.vs)])
    k, v = (synth.bf16_bits_to_f32(t[x]).astype(np.float64) for x in ("prefix_k", "prefix_v"))
    seq = np.repeat(np.arange(s.n_docs), s.doc_prefix_len)
    index = np.concatenate([np.arange(n) for n in s.doc_prefix_len])
    assert po.append(want, doc_table, k, v, seq, index) == 0
    assert po.same_codes(docs.k, want.k) and po.same_codes(docs.v, want.v) and np.array_equal(docs.ks, want.ks)
    pb.build_meta()
    tabs = pb.tables()
    n = tabs["n_active"]
    act, depth = tabs["active_slot"][:n], tabs["suffix_len"][:n]
    pb.set_step_inputs(t["q"][act], t["k_new"][act], t["v_new"][act])
    q, k_new = pb.db.q.clone(), pb.db.k_new.clone()
    B.hpd_rope(g, s.n_slots, pb.db.meta.n_active, pb.db.meta.pos_id, q, k_new)
    assert po.append(branches, np.arange(s.n_slots)[:, None], _wide(k_new)[:n], _wide(pb.db.v_new)[:n], act, depth) == 0
    pb.step(with_meta=False)
    torch.cuda.synchronize()
    got = _pool(pb.branches)
    assert po.same_codes(got.k, branches.k) and po.same_codes(got.v, branches.v) and np.array_equal(got.ks, branches.ks) and np.array_equal(got.vs, branches.vs)
    assert torch.equal(pb.q_rot[:n].view(torch.int16), q[:n].view(torch.int16)) and pb.status() == 0
    _check_rows(g, _wide(q), _wide(pb.o), pb.lse.cpu().numpy(), docs, doc_table, s.doc_prefix_len, got, np.arange(s.n_slots), tabs["doc_id"], act, depth + 1, 40)
    # again as a graph: the tokens are appended to the same places, the bits are the same
    o, lse = pb.o.clone(), pb.lse.clone()
    graph = pb.capture_step()
    pb.o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(pb.o.view(torch.int16), o.view(torch.int16)) and torch.equal(pb.lse, lse)


def test_the_same_values_in_bf16_caches():
    """A code times a power of two is a bf16: hpd_attn_decode over caches of those values agrees, to both kernels' roundings."""
    from paper_2604_26209_b200 import runtime
    s = synth.config_main(n_prompts=1, seed=5)
    g, t = s.geom, synth.make_tensors(s)
    pb = runtime.PagedBatch(s, t)
    pb.build_meta()
    n = pb.tables()["n_active"]
    act = pb.tables()["active_slot"][:n]
    pb.set_step_inputs(t["q"][act], t["k_new"][act], t["v_new"][act])
    pb.step(with_meta=False)
    db = runtime.DeviceBatch(s, t)
    docs, branches, table = _pool(pb.docs), _pool(pb.branches), pb.docs.table.cpu().numpy()
    f = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()                  # noqa: E731
    cat = [docs.tokens(table[d], int(L)) for d, L in enumerate(s.doc_prefix_len)]
    db.prefix_k, db.prefix_v = (f(np.concatenate([c[i] for c in cat])).to(torch.bfloat16) for i in (0, 1))
    own = [branches.tokens(np.array([i]), g.suffix_cap) for i in range(s.n_slots)]
    db.suffix_k, db.suffix_v = (f(np.concatenate([c[i] for c in own])).to(torch.bfloat16) for i in (0, 1))
    db.build_meta()
    db.q.copy_(pb.q_rot)
    db.attn(True)
    torch.cuda.synchronize()
    # P in bf16 (2^-8 of each probability) there, in fp16 here, both outputs rounded to bf16; |v| is at most the page's 448 scales
    top = float(max(x.float().abs().max() for x in (db.prefix_v, db.suffix_v)))
    assert float((db.o.float() - pb.o.float()).abs().max()) <= top * (2.0 ** -8 + 2.0 ** -11) + 2 * 2.0 ** -8 * float(db.o.float().abs().max())
    assert float((db.lse - pb.lse).abs().max()) <= 2.0 ** -12


@pytest.mark.parametrize("mode", ["direct", "graph", "stream"])
def test_decode_loop(mode):
    """Prompt and decode loop with retirement: the first step's keys go into the pages, then tables, append, attention, end of step, several
    times without a host wait; every step's rows against 64 bits over the pages of that moment."""
    from paper_2604_26209_b200 import binding as B
    g = synth.Geom(Hq=8, Hkv=2, D=128, rope_theta=500000.0, sm_scale=128 ** -0.5, suffix_cap=5)
    rng = np.random.default_rng(3)
    L, cnt, steps = np.array([90, 33, 200]), np.array([7, 40, 4]), 5
    n_docs, n, T = len(L), int(cnt.sum()), int(L.sum())
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()                   # noqa: E731
    gen = torch.Generator(device="cuda").manual_seed(4)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen).to(torch.bfloat16)                  # noqa: E731
    tL, tcnt = i32(L), i32(cnt)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    # the first step: tables of the prompt, rotation and append in one call (chunked: the first 70 tokens of each document, then the rest)
    pt = B.PrefillTables.alloc(g, n_docs, T)
    B.hpd_prefill_meta(g, n_docs, 0, T, tL, i32(np.zeros(n_docs)), i32([0]), 0, pt)
    docs = B.PagedCache.alloc(g, n_docs, 4, 64)
    pq, pk, pv = rnd(T, g.Hq, g.D), rnd(T, g.Hkv, g.D), rnd(T, g.Hkv, g.D)
    whole = B.PagedCache.alloc(g, n_docs, 4, 64)
    pq_rot = torch.zeros_like(pq)
    B.hpd_append_paged(g, n_docs, T, pt.n_tokens, pt.tok_doc, pt.doc_kv_start, None, i32(np.zeros(n_docs)), whole, pt.tok_pos, pq, pq_rot, pk, pv, status)
    start = np.concatenate([[0], np.cumsum(L)])
    parts = [np.concatenate([np.arange(start[d], start[d] + min(70, L[d])) for d in range(n_docs)]),
             np.concatenate([np.arange(start[d] + min(70, L[d]), start[d + 1]) for d in range(n_docs)])]
    held = np.zeros(n_docs, np.int64)
    pos = np.concatenate([np.arange(x) for x in L])
    for rows in parts:
        doc = np.searchsorted(start, rows, side="right") - 1
        m = len(rows)
        at = torch.from_numpy(rows).cuda()
        B.hpd_append_paged(g, n_docs, m, i32([m]), i32(doc), i32(np.searchsorted(doc, np.arange(n_docs + 1))), None, i32(held), docs, i32(pos[rows]), None,
                           None, pk[at].contiguous(), pv[at].contiguous(), status)
        held += np.bincount(doc, minlength=n_docs)
    torch.cuda.synchronize()
    one, two = _pool(whole), _pool(docs)
    q0, k0 = pq.clone(), pk.clone()
    B.hpd_rope(g, T, pt.n_tokens, pt.tok_pos, q0, k0)
    assert torch.equal(pq_rot.view(torch.int16), q0.view(torch.int16))
    for d in range(n_docs):                                                                            # a page that grew in two calls: the values, but for faint ones
        for x, y in zip(one.tokens(np.arange(4 * d, 4 * d + 4), int(L[d])), two.tokens(np.arange(4 * d, 4 * d + 4), int(L[d]))):
            assert np.all(np.abs(x - y) <= np.abs(x).max() * 2.0 ** -17)
    # the loop
    branches = B.PagedCache.alloc(g, n, 1, g.suffix_cap, n_pages=n + 4)
    slot_page = rng.permutation(n + 4)[:n]
    branches.table.copy_(i32(slot_page[:, None]))
    m = B.MetaTables.alloc(g, n_docs, n, T)
    depth, alive = i32(np.zeros(n)), torch.ones(n, dtype=torch.uint8, device="cuda")
    token = i32(rng.integers(0, 5, (steps, n)))                                                        # 0 ends the value
    q, k, v = (rnd(steps, n, h, g.D) for h in (g.Hq, g.Hkv, g.Hkv))
    now = [torch.zeros_like(x[0]) for x in (q, k, v)] + [torch.zeros_like(token[0])]
    q_rot, o, lse = torch.zeros_like(q[0]), torch.zeros_like(q[0]), torch.zeros(n, g.Hq, device="cuda")
    n_alive = i32([0])

    def step():
        B.hpd_build_meta(g, n_docs, n, tL, tcnt, depth, alive, 0, m)
        B.hpd_append_paged(g, n, n, m.n_active, None, None, m.active_slot, m.suffix_len, branches, m.pos_id, now[0], q_rot, now[1], now[2], m.dev_status)
        B.hpd_attn_decode_paged(g, n_docs, n, n, q_rot, docs, branches, tL, m, True, o, lse)
        B.hpd_advance(g, n, m.n_active, m.active_slot, now[3], 0, depth, alive, n_alive)
    stream = torch.cuda.Stream() if mode == "stream" else torch.cuda.current_stream()
    stream.wait_stream(torch.cuda.current_stream())
    seen = []
    with torch.cuda.stream(stream):
        if mode == "graph":
            before = [x.clone() for x in (depth, alive, branches.k.view(torch.uint8), branches.v.view(torch.uint8), branches.k_scale.view(torch.uint8),
                                          branches.v_scale.view(torch.uint8))]
            step()
            for x, y in zip((depth, alive, branches.k.view(torch.uint8), branches.v.view(torch.uint8), branches.k_scale.view(torch.uint8),
                             branches.v_scale.view(torch.uint8)), before):
                x.copy_(y)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        for t in range(steps):
            for x, y in zip(now, (q, k, v, token)):
                x.copy_(y[t])
            graph.replay() if mode == "graph" else step()
            seen.append([x.clone() for x in (m.n_active, m.active_slot, m.doc_id, m.suffix_len, q_rot, o, lse, branches.k.view(torch.uint8),
                                             branches.v.view(torch.uint8), branches.k_scale.view(torch.uint8), branches.v_scale.view(torch.uint8))])
    torch.cuda.synchronize()
    assert int(m.dev_status.item()) == 0 and int(status.item()) == 0
    live = np.ones(n, bool)
    for t, (na, act, doc, slen, qr, ot, lt, *pages) in enumerate(seen):
        na = int(na.item())
        act = act.cpu().numpy()[:na]
        assert np.array_equal(act, np.flatnonzero(live))
        pool = po.Pool(*[x.cpu().numpy() for x in pages])
        _check_rows(g, _wide(qr), _wide(ot), lt.cpu().numpy(), two, docs.table.cpu().numpy(), L, pool, slot_page, doc.cpu().numpy(), act, slen.cpu().numpy()[:na] + 1, 25)
        live[act[token[t].cpu().numpy()[:na] == 0]] = False
        if t + 1 == g.suffix_cap:
            live[:] = False


def test_two_layers_share_tables_and_workspace():
    """Layers one after another on the tables and the workspace of one step: the bits of each alone."""
    from paper_2604_26209_b200 import binding as B
    from tests.test_gpu_paged_attn import Case
    a, b = (Case((8, 2, 128), 32, [700, 2600], [20, 6], 10, seed=21, depth=4) for _ in range(2))
    for c in (a, b):
        c.upload()
    b.q = a.q * -0.5
    alone = []
    for c in (a, b):
        c.attend()
        torch.cuda.synchronize()
        alone.append((c.o.clone(), c.lse.clone()))
        c.o.zero_()
    for _ in range(3):
        for c in (a, b):
            B.hpd_attn_decode_paged(c.g, 2, 26, 26, c.q, c.dc, c.bc, c.tL, a.m, True, c.o, c.lse)
    torch.cuda.synchronize()
    for c, (o, l) in zip((a, b), alone):
        assert torch.equal(c.o.view(torch.int16), o.view(torch.int16)) and torch.equal(c.lse, l)


def test_two_batches_at_once():
    """Batches with caches and workspaces of their own, their steps as graphs on two streams at the same time: the bits of each alone."""
    from paper_2604_26209_b200 import runtime
    made = []
    for i, cfg in enumerate((synth.config_main(n_prompts=4, seed=8), synth.config_custom("ragged", 8, 2, 64, 1e4, 12, [0, 1, 70, 3000, 129], [3, 1, 20, 33, 0], 12, alive_frac=0.7))):
        t = synth.make_tensors(cfg)
        pb = runtime.PagedBatch(cfg, t, (64, 16)[i])
        pb.build_meta()
        n = pb.tables()["n_active"]
        act = pb.tables()["active_slot"][:n]
        pb.set_step_inputs(t["q"][act], t["k_new"][act], t["v_new"][act])
        pb.step()
        torch.cuda.synchronize()
        made.append((pb, pb.capture_step(), torch.cuda.Stream(), pb.o.clone(), pb.lse.clone()))
        pb.o.zero_()
        pb.lse.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for pb, graph, stream, _, _ in made:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for pb, _, _, o, lse in made:
        assert torch.equal(pb.o.view(torch.int16), o.view(torch.int16)) and torch.equal(pb.lse, lse) and pb.status() == 0


def test_bf16_and_paged_calls_take_turns_on_one_workspace():
    """The two attentions on the tables, the plan and the ticket counter of one step, one after the other: the bits of each alone."""
    from paper_2604_26209_b200 import runtime
    s = synth.config_main(n_prompts=1, seed=9)
    t = synth.make_tensors(s)
    pb, db = runtime.PagedBatch(s, t), runtime.DeviceBatch(s, t)
    db.meta = pb.db.meta
    pb.build_meta()
    n = pb.tables()["n_active"]
    act = pb.tables()["active_slot"][:n]
    for b in (pb, db):
        b.set_step_inputs(t["q"][act], t["k_new"][act], t["v_new"][act])
    db.rope()
    db.kv_append()
    db.attn(True)
    pb.append()
    pb.attn()
    torch.cuda.synchronize()
    want = [x.clone() for x in (db.o, pb.o, pb.lse)]
    for _ in range(10):
        pb.attn()
        db.attn(True)
    pb.attn()
    torch.cuda.synchronize()
    for x, y in zip((db.o, pb.o, pb.lse), want):
        assert torch.equal(x, y)
    assert pb.status() == 0
