"""The paged cache in 8 bits as cases that can be timed: appending the new tokens of a step, a prompt or a chunk to it, and the
decode attention that reads it.

A cache is a pool of pages.  A page holds `page` tokens: for each kv head the e4m3 codes of its keys and of its values
([Hkv, page, D]) and one scale each, a power of two in e8m0.  Sequences (documents, branches) own the pages that their row of a
table names.

    own                 False: the operators in elementary torch operations; True: the framework's calls
    listed()            the cases by name
    draw(rng)           one more case of the same ranges
    prepare(case, seed) a user's state: activations, pools of pages, tables
    run(state)          one call of one operator
    work(case)          bytes and operations that the call cannot do without
    exact(case, seed)   the call's outputs in 64 bits

`kind` names the operator and its form:
    step     hpd_append_paged, one token for each live branch: prompts x docs x branches slots, a share `alive` of them live, a page of
             `page` tokens (= the slab) for each, 0 .. depth_hi - 1 tokens in it
    tokens   hpd_append_paged, the new tokens of `seqs` sequences, new_lo..new_hi each, behind old_lo..old_hi cached ones; rotate: whether
             keys and queries are rotated on the way
    attn     hpd_attn_decode_paged: documents of len_lo..len_hi tokens in pages of `page`, branches of 0 .. depth_hi - 1 tokens and the
             step's own, a page of `cap` tokens each
"""
import numpy as np
import torch

own = False

THETA = 500000.0
TOP = 448.0                                  # largest e4m3 value
LLAMA = dict(Hq=32, Hkv=8, D=128)            # the benchmark's attention geometry (Llama-3-8B)
MAIN = dict(docs=4, branches=24, alive=1.0, **LLAMA)


def listed():
    return [
        # the decode step of a tiny model: four branches, nothing but latency
        dict(name="append_step_tiny", kind="step", prompts=1, docs=1, branches=4, alive=1.0, page=8, depth_hi=8, Hq=4, Hkv=1, D=64),
        # the paper's prompt (6 documents x 16 attributes, K_max = 30) some way into decoding: half of the branches retired
        dict(name="append_step_paper_shape", kind="step", prompts=11, docs=6, branches=16, alive=0.5, page=30, depth_hi=30, Hq=32, Hkv=4, D=128),
        # the decode step of the benchmark's full batch
        dict(MAIN, name="append_step_64_prompts", kind="step", prompts=64, page=16, depth_hi=16),
        # the first step of one stacked prompt; keys come rotated from the prompt's attention
        dict(name="append_prompt_1", kind="tokens", seqs=1, new_lo=2288, new_hi=2288, old_lo=0, old_hi=0, page=64, rotate=False, **LLAMA),
        # ragged chunks behind what is cached already, in small pages, rotated on the way
        dict(name="append_chunks_ragged", kind="tokens", seqs=37, new_lo=1, new_hi=701, old_lo=0, old_hi=900, page=16, rotate=True, Hq=8, Hkv=4, D=64),
        # the first step of a full batch of stacked prompts, rotated on the way
        dict(name="append_prompt_64", kind="tokens", seqs=64, new_lo=2144, new_hi=2432, old_lo=0, old_hi=0, page=64, rotate=True, **LLAMA),
        # one short document, four attributes, a small head geometry
        dict(name="attn_tiny", kind="attn", prompts=1, docs=1, len_lo=256, len_hi=256, branches=4, alive=1.0, page=64, cap=8, depth_hi=8, lse=True,
             Hq=4, Hkv=1, D=64),
        # one product page answered interactively
        dict(MAIN, name="attn_1_prompt", kind="attn", prompts=1, len_lo=512, len_hi=512, page=64, cap=16, depth_hi=16, lse=True),
        # a small batch
        dict(MAIN, name="attn_8_prompts", kind="attn", prompts=8, len_lo=512, len_hi=512, page=64, cap=16, depth_hi=16, lse=True),
        # the benchmark's full batch
        dict(MAIN, name="attn_64_prompts", kind="attn", prompts=64, len_lo=512, len_hi=512, page=64, cap=16, depth_hi=16, lse=True),
        # long documents of ragged length, few branches each, pages of 32
        dict(MAIN, name="attn_long", kind="attn", prompts=24, docs=8, len_lo=1024, len_hi=4096, branches=12, page=32, cap=32, depth_hi=32, lse=True),
        # the paper's prompt some way into decoding: odd lengths, small pages, half of the branches retired, 8 query heads per kv head
        dict(name="attn_paper_shape", kind="attn", prompts=11, docs=6, len_lo=83, len_hi=1277, branches=16, alive=0.5, page=16, cap=30, depth_hi=30,
             lse=False, Hq=32, Hkv=4, D=128),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["step", "tokens", "tokens", "attn", "attn", "attn", "attn"])
    Hq, Hkv, D = rng.choice([(32, 8, 128)] * 4 + [(32, 4, 128), (16, 8, 128), (8, 8, 128), (4, 1, 64), (8, 4, 64), (8, 1, 64)])
    c = dict(kind=kind, Hq=Hq, Hkv=Hkv, D=D)
    if kind == "tokens":
        lo = _log_int(rng, 1, 2400)
        c.update(seqs=_log_int(rng, 1, 64), new_lo=lo, new_hi=lo + int(lo * rng.choice([0, 0.1, 1, 3])), page=rng.choice([16, 32, 64]),
                 rotate=rng.random() < 0.6)
        c["old_lo"] = rng.choice([0, 0, 5, 64, 500])
        c["old_hi"] = c["old_lo"] * rng.choice([1, 2])
    else:
        cap = rng.choice([5, 8, 16, 16, 30, 32])
        c.update(prompts=_log_int(rng, 1, 64), docs=rng.randint(1, 8), branches=_log_int(rng, 1, 48), alive=rng.choice([1.0, 1.0, 0.7, 0.3]),
                 depth_hi=rng.randint(1, cap))
        if kind == "step":
            c["page"] = cap
        else:
            lo = _log_int(rng, 1, 3000)
            c.update(cap=cap, page=rng.choice([16, 32, 64, 64]), len_lo=lo, len_hi=min(4096, lo + int(lo * rng.choice([0, 0.3, 1, 3]))),
                     lse=rng.random() < 0.5)
    # no drawn case costs more than the largest listed one
    most = {"step": (0.15e9, 1e12), "tokens": (3.4e9, 1e12), "attn": (1.05e9, 0.1e12)}[kind]
    size = "seqs" if kind == "tokens" else "prompts"
    while c[size] > 1:
        w = work(c)
        if w["bytes"] <= most[0] and w["flops"] <= most[1]:
            break
        c[size] = max(1, c[size] * 3 // 4)
    return c


# ---------------------------------------------------------------------------------------------------------------------
def _sizes(c):
    """The lengths of a case's documents or sequences; they belong to the case, their order to the seed."""
    if c["kind"] == "tokens":
        own_rng = np.random.default_rng([c["seqs"], c["new_lo"], c["new_hi"], c["old_hi"]])
        return own_rng.integers(c["new_lo"], c["new_hi"] + 1, c["seqs"]), own_rng.integers(c["old_lo"], c["old_hi"] + 1, c["seqs"])
    own_rng = np.random.default_rng([c["prompts"], c["docs"], c["branches"]])
    docs = c["prompts"] * c["docs"]
    live = own_rng.random(docs * c["branches"]) < c["alive"]
    live[0] = True
    depth = own_rng.integers(0, c["depth_hi"], docs * c["branches"])
    length = own_rng.integers(c["len_lo"], c["len_hi"] + 1, docs) if c["kind"] == "attn" else np.zeros(docs, np.int64)
    return length, live, depth


def _quantised(x):
    """Pages of codes and their scales for x [pages, Hkv, tokens, D] (one scale per page and head)."""
    e = _exponent(x.float().abs().amax(dim=(2, 3)))
    codes = (x.float() * torch.exp2(-e.float())[:, :, None, None]).clamp(-TOP, TOP).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8)


def prepare(case, seed):
    c = case
    rng = np.random.default_rng([seed & 0x7FFFFFFF, 0x50414745])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed & 0x7FFFFFFFFFFF)
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    gpu = lambda a, t=np.int32: torch.from_numpy(np.ascontiguousarray(a, dtype=t)).cuda()                              # noqa: E731
    rnd = lambda *shape: torch.randn(*shape, device="cuda", dtype=torch.bfloat16, generator=gen)                        # noqa: E731

    def pool(pages, tokens, filled):
        """A pool of pages; `filled`: with tokens from earlier calls (codes of normal numbers), else empty."""
        p = {}
        for name in ("k", "v"):
            if filled:
                p[name] = torch.empty(pages, Hkv, tokens, D, dtype=torch.float8_e4m3fn, device="cuda")
                scale = torch.empty(pages, Hkv, dtype=torch.uint8, device="cuda")
                for lo in range(0, pages, 4096):
                    part = p[name][lo:lo + 4096]
                    part[:], scale[lo:lo + 4096] = _quantised(rnd(*part.shape))
            else:
                p[name] = torch.zeros(pages, Hkv, tokens, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
                scale = torch.zeros(pages, Hkv, dtype=torch.uint8, device="cuda")
            p[name + "_scale"] = scale.view(torch.float8_e8m0fnu)
        return p

    if c["kind"] == "tokens":
        turn = rng.permutation(c["seqs"])
        new, old = (x[turn] for x in _sizes(c))
        P, T = c["page"], int(new.sum())
        need = -(-(old + new) // P)
        table = np.full((c["seqs"], int(need.max())), -1, np.int64)
        order = rng.permutation(int(need.sum()) + 3)
        for s, at in enumerate(np.concatenate([[0], np.cumsum(need)])[:-1]):
            table[s, :need[s]] = order[at:at + need[s]]
        start = np.concatenate([[0], np.cumsum(new)])
        seq = np.repeat(np.arange(c["seqs"]), new)
        index = old[seq] + np.arange(T) - start[seq]
        s = dict(c=c, n_seqs=c["seqs"], n=T, n_rows=gpu([T]), row_seq=gpu(seq), seq_row_start=gpu(start), seq_id=None, seq_len=gpu(old),
                 table=gpu(table), pos=gpu(index + 30 * (index // 100)) if c["rotate"] else None, k=rnd(T, Hkv, D), v=rnd(T, Hkv, D),
                 q=rnd(T, Hq, D) if c["rotate"] else None, cache=pool(len(order), P, bool(old.max() > 0)))
        s["q_rot"] = torch.zeros_like(s["q"]) if c["rotate"] else None
        return _planned(s)
    length, live, depth = _sizes(c)
    docs, slots = len(length), len(live)
    length = length[rng.permutation(docs)]
    depth = depth[rng.permutation(slots)]
    live = live[rng.permutation(slots)]
    rows = np.flatnonzero(live)
    cap = c["page"] if c["kind"] == "step" else c["cap"]
    slot_page = rng.permutation(slots + 2)[:slots]
    active = np.full(slots, -1, np.int64)
    active[:len(rows)] = rows
    seq_len = np.full(slots, -1, np.int64)
    seq_len[:len(rows)] = depth[rows]
    s = dict(c=c, n_seqs=slots, n=slots, live_rows=len(rows), n_rows=gpu([len(rows)]), row_seq=None, seq_row_start=None, seq_id=gpu(active), seq_len=gpu(seq_len),
             table=gpu(slot_page[:, None]), q=rnd(slots, Hq, D), cache=pool(slots + 2, cap, True))
    if c["kind"] == "step":
        s.update(pos=gpu(np.concatenate([rng.integers(100, 4500, len(rows)), np.full(slots - len(rows), -1)])), k=rnd(slots, Hkv, D), v=rnd(slots, Hkv, D),
                 q_rot=torch.zeros(slots, Hq, D, dtype=torch.bfloat16, device="cuda"))
        return _planned(s)
    P = c["page"]
    need = -(-length // P)
    table = np.full((docs, int(need.max())), -1, np.int64)
    order = rng.permutation(int(need.sum()) + 3)
    for d, at in enumerate(np.concatenate([[0], np.cumsum(need)])[:-1]):
        table[d, :need[d]] = order[at:at + need[d]]
    s.update(n_docs=docs, L=gpu(length), doc_table=gpu(table), doc_cache=pool(len(order), P, True), depth=gpu(depth), alive=gpu(live, np.uint8),
             cnt=gpu(np.full(docs, c["branches"])), doc_of_row=gpu(rows // c["branches"], np.int64), rank_of_row=gpu(_ranks(rows // c["branches"]), np.int64),
             rows_of_doc=int(np.bincount(rows // c["branches"]).max()), longest=int(length.max()),
             o=torch.zeros(slots, Hq, D, dtype=torch.bfloat16, device="cuda"), lse=torch.zeros(slots, Hq, device="cuda") if c["lse"] else None)
    return _planned(s)


def _ranks(doc):
    """The number of each row within its document (rows come grouped by document)."""
    first = np.searchsorted(doc, doc, side="left")
    return np.arange(len(doc)) - first


def _planned(s):
    """What a program that uses the framework keeps besides: its cache objects and, for the attention, the step's tables."""
    if own:
        from paper_2604_26209_b200 import binding as B
        from paper_2604_26209_b200.synth import Geom
        c = s["c"]
        cap = c["cap"] if c["kind"] == "attn" else 16
        s["g"] = g = Geom(Hq=c["Hq"], Hkv=c["Hkv"], D=c["D"], rope_theta=THETA, sm_scale=float(c["D"]) ** -0.5, suffix_cap=cap)
        s["pages"] = B.PagedCache(s["cache"]["k"], s["cache"]["v"], s["cache"]["k_scale"], s["cache"]["v_scale"], s["table"])
        s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        if c["kind"] == "attn":
            d = s["doc_cache"]
            s["doc_pages"] = B.PagedCache(d["k"], d["v"], d["k_scale"], d["v_scale"], s["doc_table"])
            s["m"] = B.MetaTables.alloc(g, s["n_docs"], s["n"], int(s["L"].sum()))
            B.hpd_build_meta(g, s["n_docs"], s["n"], s["L"], s["cnt"], s["depth"], s["alive"], 0, s["m"])
    return s


def run(state):
    s = state
    if s["c"]["kind"] == "attn":
        if own:
            from paper_2604_26209_b200 import binding as B
            B.hpd_attn_decode_paged(s["g"], s["n_docs"], s["n"], s["n"], s["q"], s["doc_pages"], s["pages"], s["L"], s["m"], True, s["o"], s["lse"])
        else:
            _attend(s)
        return [s["o"], s["lse"]] if s["lse"] is not None else s["o"]
    if own:
        from paper_2604_26209_b200 import binding as B
        B.hpd_append_paged(s["g"], s["n_seqs"], s["n"], s["n_rows"], s["row_seq"], s["seq_row_start"], s["seq_id"], s["seq_len"], s["pages"], s["pos"],
                           s["q"], s["q_rot"], s["k"], s["v"], s["status"])
    else:
        _append(s)
    return [s["cache"][k] for k in ("k", "v", "k_scale", "v_scale")] + ([s["q_rot"]] if s["q_rot"] is not None else [])


# --------------------------------------------- the operators in elementary operations ---------------------------------------------
def _exponent(a):
    """The smallest n >= -126 with a <= 448 * 2^n."""
    m, e = torch.frexp(a)
    return torch.where(a > 0, e - 9 + (m > 0.875), torch.full_like(e, -126)).clamp(min=-126)


def _rotated(x, pos):
    """x [rows, heads, D] rotated at its rows' positions; element i goes with i + D/2."""
    half = x.shape[-1] // 2
    inv = torch.pow(torch.tensor(THETA, dtype=torch.float64, device=x.device), -2.0 * torch.arange(half, device=x.device, dtype=torch.float64) / (2 * half))
    ang = pos.double()[:, None, None] * inv
    c, s = torch.cos(ang).float(), torch.sin(ang).float()
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1).to(torch.bfloat16)


def _append(s):
    c, cache = s["c"], s["cache"]
    P = cache["k"].shape[2]
    n = s["n"] if s["row_seq"] is not None else s["live_rows"]
    if s["row_seq"] is not None:
        seq = s["row_seq"][:n].long()
        index = s["seq_len"][seq] + torch.arange(n, device=seq.device) - s["seq_row_start"][seq]
        before = s["seq_len"][seq]
        entry = seq
    else:
        index = before = s["seq_len"][:n].long()
        entry = s["seq_id"][:n].long()
    page, slot = s["table"][entry, index // P].long(), index % P
    k, v = s["k"][:n], s["v"][:n]
    if s["pos"] is not None:
        k = _rotated(k, s["pos"][:n])
        s["q_rot"][:n] = _rotated(s["q"][:n], s["pos"][:n])
    # tokens that each page held before, and the exponents that the new ones need
    pages = cache["k"].shape[0]
    held = torch.zeros(pages, dtype=torch.int64, device=k.device)
    held.index_put_((page,), (before - index // P * P).clamp(0, P))
    touched = torch.zeros(pages, dtype=torch.bool, device=k.device)
    touched.index_fill_(0, page, True)
    for name, x in (("k", k), ("v", v)):
        top = x.float().abs().amax(dim=2)
        need = _exponent(torch.zeros(pages, top.shape[1], device=k.device).index_reduce_(0, page, top, "amax"))
        was = cache[name + "_scale"].view(torch.uint8).int() - 127
        now = torch.where(touched[:, None], torch.where(held[:, None] > 0, torch.maximum(was, need), need), was)
        change = torch.where((held > 0)[:, None], torch.exp2((was - now).float()), torch.ones_like(top[:1]))
        old = torch.arange(P, device=k.device)[None, :] < held[:, None]
        codes = cache[name]
        again = (codes.float() * torch.where(old[:, None, :, None], change[:, :, None, None], torch.ones(1, device=k.device))).to(torch.float8_e4m3fn)
        codes.view(torch.uint8).copy_(again.view(torch.uint8))
        code = (x.float() * torch.exp2(-now[page].float())[:, :, None]).clamp(-TOP, TOP).to(torch.float8_e4m3fn)
        codes.view(torch.uint8)[page, :, slot] = code.view(torch.uint8)
        cache[name + "_scale"].view(torch.uint8).copy_((now + 127).to(torch.uint8))


def _attend(s):
    c = s["c"]
    G, D, Hkv = c["Hq"] // c["Hkv"], c["D"], c["Hkv"]
    n, doc, rank = s["live_rows"], s["doc_of_row"], s["rank_of_row"]
    scale = float(D) ** -0.5

    def values(cache, pages, name):
        return cache[name][pages].float() * cache[name + "_scale"][pages].float()[..., None, None]

    pages = s["doc_table"].long().clamp(min=0)
    span = pages.shape[1] * c["page"]
    K, V = (values(s["doc_cache"], pages, x).transpose(1, 2).reshape(s["n_docs"], Hkv, span, D) for x in ("k", "v"))
    seen = torch.arange(span, device=doc.device)[None, :] < s["L"][:, None]
    own_page = s["table"][s["seq_id"][:n].long(), 0].long()
    k, v = (values(s["cache"], own_page, x) for x in ("k", "v"))                                 # [rows, Hkv, cap, D]
    mine = torch.arange(c["cap"], device=doc.device)[None, :] < (s["seq_len"][:n] + 1)[:, None]
    q = s["q"][:n].float().view(n, Hkv, G, D)
    tiles = torch.zeros(s["n_docs"], s["rows_of_doc"], Hkv, G, D, device=doc.device)
    tiles[doc, rank] = q
    tiles = tiles.permute(0, 2, 1, 3, 4).reshape(s["n_docs"], Hkv, -1, D)
    low = float("-inf")
    a = torch.matmul(tiles, K.transpose(2, 3)).mul_(scale).masked_fill_(~seen[:, None, None, :], low)
    b = torch.matmul(q, k.transpose(2, 3)).mul_(scale).masked_fill_(~mine[:, None, None, :], low)
    top_a = a.amax(dim=3).view(s["n_docs"], Hkv, s["rows_of_doc"], G).permute(0, 2, 1, 3)[doc, rank]
    top = torch.maximum(top_a, b.amax(dim=3))                                                    # [rows, Hkv, G]; every row sees its own token
    spread = torch.zeros(s["n_docs"], s["rows_of_doc"], Hkv, G, device=doc.device)
    spread[doc, rank] = top
    a = a.sub_(spread.permute(0, 2, 1, 3).reshape(s["n_docs"], Hkv, -1, 1)).exp_()
    b = torch.exp(b - top[..., None])
    V = V.mul_(seen[:, None, :, None])
    v = v * mine[:, None, :, None]
    back = lambda x: x.view(s["n_docs"], Hkv, s["rows_of_doc"], G, -1).permute(0, 2, 1, 3, 4)[doc, rank]              # noqa: E731
    total = back(a.sum(dim=3, keepdim=True))[..., 0] + b.sum(dim=3)
    o = (back(torch.matmul(a, V)) + torch.matmul(b, v)) / total[..., None]
    s["o"][:n] = o.view(n, c["Hq"], D).to(torch.bfloat16)
    if s["lse"] is not None:
        s["lse"][:n] = (top + torch.log(total)).view(n, c["Hq"])


# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    c = case
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    token, row = 2 * Hkv * D, Hq * D * 2                         # a cached token's codes; one row's q or o in bf16
    if c["kind"] == "attn":
        length, live, depth = _sizes(c)
        P = c["page"]
        per_doc = np.bincount(np.flatnonzero(live) // c["branches"], minlength=len(length))
        n, cached = int(live.sum()), int((depth[live] + 1).sum())
        prefix, pages = int(length[per_doc > 0].sum()), int((-(-length[per_doc > 0] // P)).sum())
        keys = float((per_doc * length).sum()) + cached
        return {"bytes": (prefix + cached) * token + (pages + n) * (2 * Hkv + 4) + n * (2 * row + (Hq * 4 if c["lse"] else 0) + 12),
                "flops": 4.0 * D * Hq * keys}
    if c["kind"] == "step":
        _, live, _ = _sizes(c)
        n = int(live.sum())
        return {"bytes": n * (2 * row + 2 * token + token + 4 * Hkv + 16), "flops": 3.0 * n * (Hq + Hkv) * D + 2.0 * n * Hkv * D}
    new, old = _sizes(c)
    n = int(new.sum())
    return {"bytes": n * ((2 * row if c["rotate"] else 0) + 2 * token + token + 12) + int((-(-new // c["page"])).sum()) * (2 * Hkv + 4),
            "flops": (3.0 * n * (Hq + Hkv) * D if c["rotate"] else 0.0) + 2.0 * n * Hkv * D}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_attention(s) if case["kind"] == "attn" else _exact_append(s)


def _exact_attention(s):
    """Document by document: softmax over [the document's tokens; the branch's], everything in 64 bits."""
    c = s["c"]
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    G, n = Hq // Hkv, s["live_rows"]
    table, length = s["doc_table"].cpu().numpy(), s["L"].cpu().numpy()
    doc, tokens = s["doc_of_row"].cpu().numpy(), s["seq_len"].cpu().numpy()[:n] + 1
    pages = s["table"].cpu().numpy()[s["seq_id"].cpu().numpy()[:n], 0]
    out = torch.zeros(s["n"], Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["n"], Hq, dtype=torch.float64, device="cuda")

    def take(cache, name, ids):
        two = 2.0 ** (cache[name + "_scale"].view(torch.uint8)[ids].double() - 127)
        return (cache[name][ids].double() * two[:, :, None, None]).permute(0, 2, 1, 3)           # [pages, tokens, Hkv, D]
    for d in range(s["n_docs"]):
        rows = np.flatnonzero(doc == d)
        if not len(rows):
            continue
        ids = torch.from_numpy(table[d, :-(-length[d] // c["page"])]).long().cuda()
        K, V = (take(s["doc_cache"], x, ids).reshape(-1, Hkv, D)[:int(length[d])] for x in ("k", "v"))
        mine = torch.from_numpy(pages[rows]).long().cuda()
        k, v = (take(s["cache"], x, mine) for x in ("k", "v"))
        at = torch.from_numpy(rows).cuda()
        q = s["q"][at].double().view(len(rows), Hkv, G, D) * D ** -0.5
        x = torch.einsum("rhgd,thd->rhgt", q, K)
        y = torch.einsum("rhgd,rthd->rhgt", q, k)
        hidden = torch.arange(c["cap"], device="cuda")[None, :] >= torch.from_numpy(tokens[rows]).cuda()[:, None]
        y[hidden[:, None, None, :].expand_as(y)] = -torch.inf
        z = torch.cat([x, y], dim=3)
        norm = torch.logsumexp(z, dim=3)
        p = torch.exp(z - norm[..., None])
        v = torch.where(hidden[:, :, None, None], 0.0, v)
        o = torch.einsum("rhgt,thd->rhgd", p[..., :int(length[d])], V) + torch.einsum("rhgt,rthd->rhgd", p[..., int(length[d]):], v)
        out[at], lse[at] = o.reshape(len(rows), Hq, D), norm.reshape(len(rows), Hq)
    return [out, lse] if s["lse"] is not None else out


def _exact_append(s):
    """Token by token of the definition on the host, vectorised over pages: rotation in 64 bits, rounded to bf16; codes by nearest value."""
    c = s["c"]
    grid = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()           # the non-negative codes' values, ascending

    def to_code(x):
        """Nearest e4m3 value, ties to the even code."""
        a = np.minimum(np.abs(x), grid[-1])
        hi = np.clip(np.searchsorted(grid, a), 1, len(grid) - 1)
        lo = hi - 1
        below, above = a - grid[lo], grid[hi] - a
        up = (above < below) | ((above == below) & (hi % 2 == 0))
        return np.copysign(np.where(up, grid[hi], grid[lo]), x)

    def needed(a):
        n = -126
        if a > 0:
            n = max(n, int(np.ceil(np.log2(a / TOP))) - 1)
            while a > TOP * 2.0 ** n:
                n += 1
        return n

    n = s["live_rows"] if s["row_seq"] is None else s["n"]
    if n * c["Hkv"] * c["D"] > 2 ** 23:
        return None                                                # too long on the host
    rot = None
    k, v = s["k"][:n].double().cpu(), s["v"][:n].double().cpu()
    if s["pos"] is not None:
        half = c["D"] // 2
        ang = s["pos"][:n].cpu().double()[:, None, None] * THETA ** (-torch.arange(half, dtype=torch.float64) / half)

        def turn(x):
            a, b = x[..., :half], x[..., half:]
            return torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()], dim=-1)
        k = turn(k).to(torch.float32).to(torch.bfloat16).double()
        rot = s["q_rot"].double().cpu()
        rot[:n] = turn(s["q"][:n].double().cpu())
    P = s["cache"]["k"].shape[2]
    if s["row_seq"] is None:
        entry, index = s["seq_id"].cpu().numpy()[:n], s["seq_len"].cpu().numpy()[:n]
        before = index
    else:
        entry = s["row_seq"].cpu().numpy()
        before = s["seq_len"].cpu().numpy()[entry]
        index = before + np.arange(n) - s["seq_row_start"].cpu().numpy()[entry]
    page = s["table"].cpu().numpy()[entry, index // P]
    result = []
    for name, x in (("k", k.numpy()), ("v", v.numpy())):
        codes = s["cache"][name].double().cpu().numpy()
        exps = s["cache"][name + "_scale"].view(torch.uint8).cpu().numpy().astype(np.int64) - 127
        order = np.argsort(page, kind="stable")
        cuts = np.flatnonzero(np.diff(page[order])) + 1
        for rows in np.split(order, cuts):
            p, held = page[rows[0]], int(np.clip(before[rows[0]] - index[rows[0]] // P * P, 0, P))
            for h in range(c["Hkv"]):
                e = needed(np.abs(x[rows, h]).max())
                if held:
                    e = max(e, exps[p, h])
                    codes[p, h, :held] = to_code(codes[p, h, :held] * 2.0 ** (exps[p, h] - e))
                exps[p, h] = e
                codes[p, h, index[rows] % P] = to_code(x[rows, h] * 2.0 ** -e)
        result += [torch.from_numpy(codes), torch.from_numpy(2.0 ** exps.astype(np.float64))]
    return [result[0], result[2], result[1], result[3]] + ([rot] if rot is not None else [])
