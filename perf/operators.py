"""Serving operators around the cached denoising step, as cases that can be timed and compared.

Four groups, in the order in which a serving loop calls them:

  rope    norms of queries and keys for each head and the position rotation in one pass; the paged form also writes the
          new K and V rows into the pages of the cache
  attend  attention of a ragged chunk of new tokens over a paged cache
  sample  one token per row of logits from temperature, top-k, top-p, min-p and a given uniform number
  pages   the cache's pages: fork, reserve with copy on write, compaction, and the copies that follow from them

`own = False`: plain torch forms.  `own = True`: the library's entry points.
"""
import math
import random

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases -----------------------------------------------------------------------------------------------------------
def _rope(name, dtype, *, batch, rows, q_heads, kv_heads, head_dim, rot_dim, norm, interleaved, paged, page, base, lens_seed):
    """`rows`: most rows of a sequence (ragged where there are several sequences); `base`: positions start below this."""
    return dict(name=name, kind="rope", dtype=dtype, batch=batch, rows=rows, q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, rot_dim=rot_dim, norm=norm, interleaved=interleaved, paged=paged, page=page, base=base,
                lens_seed=lens_seed)


def _attend(name, dtype, *, batch, rows, ctx, q_heads, kv_heads, head_dim, page, mask_block, lens_seed, ragged=True):
    """`rows`, `ctx`: most new rows and keys of a sequence.  `mask_block`: 0 every row sees all keys, 1 causal, n rows of
    a block of n positions see all of it and what stands before it."""
    return dict(name=name, kind="attend", dtype=dtype, batch=batch, rows=rows, ctx=ctx, q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, page=page, mask_block=mask_block, lens_seed=lens_seed, ragged=ragged)


def _sample(name, dtype, *, rows, vocab, pad, filters):
    """`pad`: columns behind the vocabulary in every row.  `filters`: which of the arrays a caller passes."""
    return dict(name=name, kind="sample", dtype=dtype, rows=rows, vocab=vocab, pad=pad, filters=filters)


def _pages(name, what, *, batch, ctx, layers, kv_heads, head_dim, page, lens_seed):
    return dict(name=name, kind="pages", what=what, batch=batch, ctx=ctx, layers=layers, kv_heads=kv_heads,
                head_dim=head_dim, page=page, lens_seed=lens_seed)


def listed():
    return [
        # one partial step of the smallest configuration in fp32: rotation only, for the dense cache; a few kilobytes
        _rope("rope_f32_34", "f32", batch=1, rows=34, q_heads=4, kv_heads=4, head_dim=64, rot_dim=64, norm=False,
              interleaved=False, paged=False, page=16, base=256, lens_seed=1),
        # eight sequences of ragged chunks, grouped queries, norms, rows taken out of the packed projection's output
        _rope("rope_paged_8x1531", "bf16", batch=8, rows=1531, q_heads=28, kv_heads=4, head_dim=128, rot_dim=128, norm=True,
              interleaved=False, paged=True, page=16, base=4096, lens_seed=2),
        # prefill of long prompts with many heads
        _rope("rope_paged_4x4096", "bf16", batch=4, rows=4096, q_heads=32, kv_heads=32, head_dim=128, rot_dim=128, norm=True,
              interleaved=False, paged=True, page=64, base=2048, lens_seed=3),
        # one sequence, one token: the latency of a decode step
        _attend("attend_1x1_768", "bf16", batch=1, rows=1, ctx=768, q_heads=28, kv_heads=4, head_dim=128, page=16, mask_block=1,
                lens_seed=4, ragged=False),
        # a served batch, one token each, ragged contexts
        _attend("attend_32x1_8192", "bf16", batch=32, rows=1, ctx=8192, q_heads=32, kv_heads=8, head_dim=128, page=16,
                mask_block=1, lens_seed=5),
        # partial denoising steps: a block of mask tokens and the recent ones over everything, full heads
        _attend("attend_8x34_4096", "bf16", batch=8, rows=34, ctx=4096, q_heads=32, kv_heads=32, head_dim=128, page=64,
                mask_block=0, lens_seed=6),
        # chunked prefill, block-causal, long ragged contexts
        _attend("attend_4x2048_8192", "bf16", batch=4, rows=2048, ctx=8192, q_heads=32, kv_heads=8, head_dim=128, page=64,
                mask_block=32, lens_seed=7),
        # the small fp32 configuration
        _attend("attend_f32_2x34_256", "f32", batch=2, rows=34, ctx=256, q_heads=4, kv_heads=4, head_dim=64, page=32,
                mask_block=0, lens_seed=8),
        # a block of mask tokens of one sequence, all filters
        _sample("sample_32x126464", "f32", rows=32, vocab=126464, pad=0, filters="all"),
        # eight sequences served together
        _sample("sample_256x152064", "bf16", rows=256, vocab=152064, pad=0, filters="all"),
        # a step of branching: half of the slots forked from the others, every sequence about to write its next tokens
        _pages("pages_branch_16", "branch", batch=16, ctx=1024, layers=4, kv_heads=4, head_dim=128, page=16, lens_seed=9),
        # a fragmented pool is moved together
        _pages("pages_compact_64", "compact", batch=64, ctx=4096, layers=4, kv_heads=4, head_dim=128, page=32, lens_seed=10),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("rope", "attend", "attend", "sample", "pages"))
    seed = rng.randrange(1 << 30)
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    kv = rng.choice((1, 2, 4, 8, 12, 32))
    group = rng.choice([g for g in (1, 2, 3, 4, 7, 8) if g * kv <= 40])
    head_dim = rng.choice((64, 128, 128))
    page = rng.choice((16, 32, 64, 128))
    if kind == "rope":
        batch = _log(rng, 1, 16)
        rows = _log(rng, 1, 16384 // batch)
        rot = rng.choice((head_dim, head_dim, head_dim // 2))
        c = _rope("", dtype, batch=batch, rows=min(rows, 4096), q_heads=kv * group, kv_heads=kv, head_dim=head_dim, rot_dim=rot,
                  norm=rng.random() < 0.6, interleaved=rng.random() < 0.3, paged=rng.random() < 0.6, page=page,
                  base=_log(rng, 1, 100000), lens_seed=seed)
        limit, cost = _cost(listed()[2]), _cost(c)
        if cost > limit:
            c["rows"] = max(1, int(c["rows"] * limit / cost))
    elif kind == "attend":
        mask = rng.choice((0, 1, 1, 4, 32))
        batch = _log(rng, 1, 48)
        ctx = _log(rng, 1, 12000)
        rows = _log(rng, 1, 2500)
        if dtype == "f32":
            ctx, rows, batch = min(ctx, 2048), min(rows, 300), min(batch, 8)
        c = _attend("", dtype, batch=batch, rows=rows, ctx=ctx, q_heads=kv * group, kv_heads=kv, head_dim=head_dim, page=page,
                    mask_block=mask, lens_seed=seed, ragged=rng.random() < 0.8)
        limit = _cost(listed()[6]) * (0.05 if dtype == "f32" else 1.0)
        while _cost(c) > limit:
            longest = max(("batch", "rows", "ctx"), key=lambda n: c[n])
            c[longest] = max(1, c[longest] * 2 // 3)
    elif kind == "sample":
        vocab = rng.choice((rng.randint(1, 1000), rng.randint(1000, 60000), rng.randint(60000, 152064), 126464, 152064))
        rows = _log(rng, 1, 256)
        if dtype == "f32":
            rows = max(1, rows // 2)
        step = 8 if dtype == "bf16" else 4
        pad = -vocab % step + rng.choice((0, 0, step * 5))
        c = _sample("", dtype, rows=rows, vocab=vocab, pad=pad,
                    filters=rng.choice(("all", "all", "none", "temperature", "top_k", "top_p", "min_p")))
    else:
        c = _pages("", rng.choice(("branch", "compact")), batch=2 * _log(rng, 1, 32), ctx=_log(rng, 16, 4096),
                   layers=rng.randint(1, 4), kv_heads=rng.choice((1, 2, 4)), head_dim=head_dim, page=page, lens_seed=seed)
        limit = _cost(listed()[11])
        while _cost(c) > limit:
            c["batch"] = max(2, c["batch"] // 4 * 2)
    c.pop("name")
    return c


def _cost(case):
    w = work(case)
    return w["bytes"] / 6.5e12 + w["flops"] / 1.6e15


# ---- what a case's shape fixes ---------------------------------------------------------------------------------------
def _chunks(case):
    """New rows and total keys of every sequence, from the case alone."""
    r = random.Random(case["lens_seed"])
    rows, lens = [], []
    for _ in range(case["batch"]):
        if case["kind"] == "rope":
            n = case["rows"] if case["batch"] == 1 else r.randint((case["rows"] + 1) // 2, case["rows"])
            rows.append(n)
            lens.append(r.randint(0, case["base"]) + n)
        elif not case["ragged"]:
            rows.append(min(case["rows"], case["ctx"]))
            lens.append(case["ctx"])
        else:
            lens.append(r.randint((case["ctx"] + 15) // 16, case["ctx"]))
            rows.append(min(lens[-1], r.randint((case["rows"] + 1) // 2, case["rows"])))
    return rows, lens


def _visible(n, kv, mask_block):
    """Keys that each of the last n of kv positions sees."""
    if mask_block == 0:
        return [kv] * n
    return [min(kv, (p // mask_block + 1) * mask_block) for p in range(kv - n, kv)]


def _page_state(case):
    """Page table, lengths and reference counts of a pool in use, from the case alone."""
    r = np.random.default_rng(case["lens_seed"])
    b, ps = case["batch"], case["page"]
    max_pages = -(-case["ctx"] // ps) + 2
    n_pages = b * max_pages
    lens = r.integers(1, case["ctx"] + 1, b)
    if case["what"] == "branch":
        lens[b // 2:] = 0        # empty slots, the children of the fork
    else:
        lens[r.random(b) < 0.4] = 0   # sequences that have ended
    table = np.full((b, max_pages), -1, np.int32)
    ids = r.permutation(n_pages)
    at = 0
    for i in range(b):
        n = -(-int(lens[i]) // ps)
        table[i, :n] = ids[at:at + n]
        at += n
    refs = np.zeros(n_pages, np.int32)
    refs[table[table >= 0]] = 1
    grow = r.integers(1, 2 * ps - 1, b)
    return table, lens.astype(np.int32), refs, grow.astype(np.int32), n_pages, max_pages


def _moved(case):
    """Pages that the case's copies move."""
    table, lens, refs, _, _, _ = _page_state(case)
    if case["what"] == "branch":
        half = case["batch"] // 2
        return int(2 * (lens[:half] % case["page"] != 0).sum())
    used = refs > 0
    return int(used[int(used.sum()):].sum())


def work(case):
    if case["kind"] == "rope":
        rows, _ = _chunks(case)
        e = 2 if case["dtype"] == "bf16" else 4
        heads = case["q_heads"] + case["kv_heads"] * (2 if case["paged"] else 1)
        values = sum(rows) * heads * case["head_dim"]
        return {"bytes": 2 * values * e + 8 * sum(rows), "flops": 8 * values}
    if case["kind"] == "attend":
        rows, lens = _chunks(case)
        e = 2 if case["dtype"] == "bf16" else 4
        pairs = keys = 0
        for n, kv in zip(rows, lens):
            vis = _visible(n, kv, case["mask_block"])
            pairs += sum(vis)
            keys += max(vis, default=0)
        d = case["head_dim"]
        return {"bytes": 2 * sum(rows) * case["q_heads"] * d * e + 2 * keys * case["kv_heads"] * d * e,
                "flops": 4 * d * case["q_heads"] * pairs}
    if case["kind"] == "sample":
        e = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": case["rows"] * (case["vocab"] * e + 32), "flops": 4 * case["rows"] * case["vocab"]}
    page_bytes = case["page"] * case["kv_heads"] * case["head_dim"] * 2
    table, _, refs, _, n_pages, max_pages = _page_state(case)
    book = 2 * 4 * (case["batch"] * (max_pages + 1) + n_pages)
    return {"bytes": 4 * _moved(case) * page_bytes * case["layers"] + book, "flops": case["batch"] * max_pages + n_pages}


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _randn(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["kind"] in ("rope", "attend"):
        rows, lens = _chunks(case)
        b, ps, d, hq, hkv = case["batch"], case["page"], case["head_dim"], case["q_heads"], case["kv_heads"]
        dt, total = _DT[case["dtype"]], sum(rows)
        offsets = [0]
        for n in rows:
            offsets.append(offsets[-1] + n)
        per = [-(-kv // ps) for kv in lens]
        max_pages, n_pages = max(per), sum(per) + 3
        ids = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        table = torch.full((b, max_pages), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(per):
            table[i, :n] = ids[at:at + n]
            at += n
        s.update(rows=rows, lens=lens, offsets=offsets, row_offsets=_int(offsets), kv_lens=_int(lens), table=table)
    if case["kind"] == "rope":
        # the rows as the packed projection leaves them: q, k and v of a token side by side
        qkv = _randn(gen, (total, (hq + 2 * hkv) * d), dt)
        s["q"], s["k"], s["v"] = (qkv[:, o * d:(o + h) * d].unflatten(1, (h, d)) for o, h in
                                  ((0, hq), (hq, hkv), (hq + hkv, hkv)))
        pos = [kv - n + i for n, kv in zip(rows, lens) for i in range(n)]
        s["positions"] = _int(pos)
        half = case["rot_dim"] // 2
        s["inv_freq"] = (500000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)).to(torch.float32)
        s["wq"] = s["wk"] = None
        if case["norm"]:
            s["wq"], s["wk"] = ((1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt) for _ in range(2))
        s["q_out"] = torch.empty(total, hq, d, dtype=dt, device="cuda")
        if case["paged"]:
            s["k_pages"], s["v_pages"] = (_randn(gen, (n_pages, hkv, ps, d), dt) for _ in range(2))
        else:
            s["k_out"] = torch.empty(total, hkv, d, dtype=dt, device="cuda")
        if own:
            import paper_2603_18489_b200 as ec
            s["rope"] = ec.make_rope_desc(hq, hkv, d, dt, case["rot_dim"], eps=1e-6, interleaved=case["interleaved"])
            if case["paged"]:
                s["desc"] = ec.make_paged_desc(b, hq, hkv, d, dt, ps, n_pages, max_pages)
    elif case["kind"] == "attend":
        s["q"] = _randn(gen, (total, hq, d), dt)
        s["k_pages"], s["v_pages"] = (_randn(gen, (n_pages, hkv, ps, d), dt) for _ in range(2))
        s["out"] = torch.empty_like(s["q"])
        if own:
            import paper_2603_18489_b200 as ec
            s["desc"] = ec.make_paged_desc(b, hq, hkv, d, dt, ps, n_pages, max_pages, mask_block=case["mask_block"])
            s["max_rows"] = max(rows)
            s["workspace"] = ec.new_workspace(ec.ec_attend_paged_workspace_bytes(s["desc"], s["max_rows"]))
    elif case["kind"] == "sample":
        n, vocab, dt = case["rows"], case["vocab"], _DT[case["dtype"]]
        sigma = torch.rand(n, 1, generator=gen, device="cuda") * 7.5 + 0.5
        logits = torch.randn(n, vocab + case["pad"], generator=gen, device="cuda")
        logits *= sigma
        # some tokens may not be sampled (the mask token among them)
        if vocab > 1:
            banned = torch.randint(0, vocab, (max(1, vocab // 500),), generator=gen, device="cuda")
            keep_one = torch.randint(0, vocab, (1,), generator=gen, device="cuda")
            logits.index_fill_(1, banned[banned != keep_one], float("-inf"))
        s["logits"] = logits.to(dt)
        u = torch.rand(n, 6, generator=gen, device="cuda")
        s["u"] = torch.rand(n, generator=gen, device="cuda")
        f = case["filters"]
        s["temperature"] = torch.where(u[:, 0] < 0.1, 0.0, 0.2 + 1.3 * u[:, 1]) if f in ("all", "temperature") else None
        s["top_k"] = torch.where(u[:, 2] < 0.3, 0.0, 1 + 1000 * u[:, 3] ** 3).to(torch.int32) if f in ("all", "top_k") else None
        s["top_p"] = torch.where(u[:, 4] < 0.3, 1.0, 0.5 + 0.49 * u[:, 5]) if f in ("all", "top_p") else None
        s["min_p"] = torch.where(u[:, 1] < 0.5, 0.0, 0.2 * u[:, 0]) if f in ("all", "min_p") else None
        if own:
            import paper_2603_18489_b200 as ec
            s["workspace"] = ec.new_workspace(ec.ec_sample_workspace_bytes(n, vocab))
    else:
        table, lens, refs, grow, n_pages, max_pages = _page_state(case)
        b = case["batch"]
        book = np.concatenate([table.ravel(), lens, refs])
        s["book0"] = torch.from_numpy(book).cuda()   # the state as the step finds it, and the copy that it works on
        s["book"] = s["book0"].clone()
        t = b * max_pages
        s["table"], s["kv_lens"], s["refs"] = s["book"][:t].view(b, max_pages), s["book"][t:t + b], s["book"][t + b:]
        shape = (case["layers"], n_pages, case["kv_heads"], case["page"], case["head_dim"])
        s["k_pages"], s["v_pages"] = (torch.randint(-2 ** 30, 2 ** 30, shape[:-1] + (shape[-1] // 2,), generator=gen,
                                                    device="cuda", dtype=torch.int32).view(torch.int16) for _ in range(2))
        s["src"], s["dst"] = _int(list(range(b // 2))), _int(list(range(b // 2, b)))
        full = np.concatenate([lens[:b // 2], lens[:b // 2]])
        s["write_from"], s["new_lens"] = _int(full.tolist()), _int((full + grow).tolist())
        cap = 2 * b if case["what"] == "branch" else n_pages
        s["copy_src"], s["copy_dst"] = _int([-1] * cap), _int([-1] * cap)
        s["n_copies"] = _int([0])
        if own:
            import paper_2603_18489_b200 as ec
            s["workspace"] = ec.new_workspace(ec.ec_pages_workspace_bytes(n_pages))
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if kind == "rope":
        return _own_rope(s) if own else _plain_rope(s)
    if kind == "attend":
        return _own_attend(s) if own else _plain_attend(s)
    if kind == "sample":
        return _own_sample(s) if own else _plain_sample(s)
    s["book"].copy_(s["book0"])
    return _own_pages(s) if own else _plain_pages(s)


def _own_rope(s):
    import paper_2603_18489_b200 as ec
    if s["case"]["paged"]:
        ec.ec_qk_norm_rope_paged(s["rope"], s["desc"], s["q"], s["k"], s["v"], s["row_offsets"], s["positions"], s["inv_freq"],
                                 s["table"], s["k_pages"], s["v_pages"], q_weight=s["wq"], k_weight=s["wk"], q_out=s["q_out"])
        return s["q_out"], s["k_pages"], s["v_pages"]
    ec.ec_qk_norm_rope(s["rope"], s["q"], s["k"], s["positions"], s["inv_freq"], q_weight=s["wq"], k_weight=s["wk"],
                       q_out=s["q_out"], k_out=s["k_out"])
    return s["q_out"], s["k_out"]


def _own_attend(s):
    import paper_2603_18489_b200 as ec
    return ec.ec_attend_paged(s["desc"], s["q"], s["row_offsets"], s["kv_lens"], s["max_rows"], s["table"], s["k_pages"],
                              s["v_pages"], out=s["out"], workspace=s["workspace"])


def _own_sample(s):
    import paper_2603_18489_b200 as ec
    o = ec.ec_sample(s["logits"], s["case"]["vocab"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                     min_p=s["min_p"], workspace=s["workspace"])
    return o["token"], o["prob"], o["kept"]


def _own_pages(s):
    import paper_2603_18489_b200 as ec
    ps = s["case"]["page"]
    if s["case"]["what"] == "branch":
        ec.ec_pages_fork(s["table"], s["kv_lens"], s["refs"], s["src"], s["dst"], ps)
        ec.ec_pages_reserve(s["table"], s["kv_lens"], s["refs"], s["write_from"], s["new_lens"], ps, s["copy_src"],
                            s["copy_dst"], s["n_copies"], workspace=s["workspace"])
    else:
        ec.ec_pages_compact(s["table"], s["kv_lens"], s["refs"], ps, s["copy_src"], s["copy_dst"], s["n_copies"],
                            workspace=s["workspace"])
    ec.ec_pages_copy(s["k_pages"], s["v_pages"], s["copy_src"], s["copy_dst"], s["n_copies"])
    return s["table"], s["kv_lens"], s["refs"], s["copy_src"], s["copy_dst"], s["n_copies"], s["k_pages"], s["v_pages"]


def _plain_rope(s):
    c = s["case"]
    half = c["rot_dim"] // 2
    angle = s["positions"].double()[:, None, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def turned(x, w):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * w.float()
        r = y[..., :c["rot_dim"]]
        if c["interleaved"]:
            a, b = r[..., 0::2], r[..., 1::2]
            r = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = r[..., :half], r[..., half:]
            r = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        return torch.cat((r, y[..., c["rot_dim"]:]), -1).to(x.dtype)

    s["q_out"].copy_(turned(s["q"], s["wq"]))
    k = turned(s["k"], s["wk"])
    if not c["paged"]:
        s["k_out"].copy_(k)
        return s["q_out"], s["k_out"]
    seq = torch.repeat_interleave(torch.arange(c["batch"], device="cuda"), s["row_offsets"].diff(), output_size=k.shape[0])
    pos = s["positions"].long()
    page, slot = s["table"][seq, pos // c["page"]].long(), pos % c["page"]
    s["k_pages"][page, :, slot] = k
    s["v_pages"][page, :, slot] = s["v"]
    return s["q_out"], s["k_pages"], s["v_pages"]


def _plain_attend(s):
    c = s["case"]
    d, hkv, group = c["head_dim"], c["kv_heads"], c["q_heads"] // c["kv_heads"]
    for i, (n, kv) in enumerate(zip(s["rows"], s["lens"])):
        lo = s["offsets"][i]
        pages = s["table"][i, :-(-kv // c["page"])].long()
        k = s["k_pages"][pages].transpose(0, 1).reshape(hkv, -1, d)[:, :kv].float()
        v = s["v_pages"][pages].transpose(0, 1).reshape(hkv, -1, d)[:, :kv].float()
        q = s["q"][lo:lo + n].view(n, hkv, group, d).permute(1, 2, 0, 3).reshape(hkv, group * n, d).float()
        scores = (q @ k.transpose(1, 2) * d ** -0.5).view(hkv, group, n, kv)
        if c["mask_block"]:
            pos = torch.arange(kv - n, kv, device="cuda")
            limit = (pos // c["mask_block"] + 1) * c["mask_block"]
            scores.masked_fill_(torch.arange(kv, device="cuda") >= limit[:, None], float("-inf"))
        p = torch.exp(scores - scores.amax(-1, keepdim=True))
        o = p.view(hkv, group * n, kv) @ v / p.sum(-1).view(hkv, group * n, 1)
        s["out"][lo:lo + n] = o.view(hkv, group, n, d).permute(2, 0, 1, 3).reshape(n, c["q_heads"], d).to(s["out"].dtype)
    return s["out"]


def _plain_sample(s):
    vocab = s["case"]["vocab"]
    x, order = torch.sort(s["logits"][:, :vocab].float(), dim=1, descending=True, stable=True)
    n = x.shape[0]
    greedy = torch.zeros(n, dtype=torch.bool, device="cuda") if s["temperature"] is None else s["temperature"] <= 0
    t = torch.ones(n, device="cuda") if s["temperature"] is None else torch.where(greedy, 1.0, s["temperature"])
    w = torch.exp((x.double() - x[:, :1].double()) / t.double()[:, None])
    cum = w.cumsum(1)
    live = (x > float("-inf")).sum(1)
    kept = live
    if s["top_k"] is not None:
        kept = torch.where(s["top_k"] > 0, torch.minimum(live, s["top_k"].long()), live)
    if s["top_p"] is not None:
        need = s["top_p"].double() * cum.gather(1, kept[:, None] - 1)[:, 0]
        in_p = (cum < need[:, None]).sum(1) + 1
        kept_p = torch.where(s["top_p"] < 1, torch.minimum(kept, in_p), kept)
    else:
        kept_p = kept
    if s["min_p"] is not None:
        kept_p = torch.minimum(kept_p, (w >= s["min_p"].double()[:, None]).sum(1).clamp(min=1))
    kept = torch.where(greedy, 1, kept_p)
    total = cum.gather(1, kept[:, None] - 1)
    rank = torch.minimum((cum <= s["u"].double()[:, None] * total).sum(1), kept - 1)[:, None]
    return (order.gather(1, rank)[:, 0].to(torch.int32), (w.gather(1, rank) / total)[:, 0].float(), kept.to(torch.int32))


def _plain_pages(s):
    ps, table, lens, refs = s["case"]["page"], s["table"], s["kv_lens"], s["refs"]
    s["copy_src"].fill_(-1)
    s["copy_dst"].fill_(-1)
    slots = torch.arange(table.shape[1], device="cuda")
    if s["case"]["what"] == "branch":
        # fork: the children take the parents' entries, every shared page counts once more
        src, dst = s["src"].long(), s["dst"].long()
        table[dst], lens[dst] = table[src], lens[src]
        shared = table[src][slots < (lens[src, None] + ps - 1) // ps].long()
        refs.index_add_(0, shared, torch.ones_like(shared, dtype=torch.int32))
        # reserve: what will be written belongs to one sequence alone
        have, want = (lens + ps - 1) // ps, (s["new_lens"] + ps - 1) // ps
        before = refs[table.clamp(min=0).long()]
        copied = (slots >= (s["write_from"] // ps)[:, None]) & (slots < have[:, None]) & (before > 1)
        fresh = (slots >= have[:, None]) & (slots < want[:, None])
        old = table[copied].long()
        refs_before = refs.clone()
        refs.index_add_(0, old, torch.full_like(old, -1, dtype=torch.int32))
        ids = torch.nonzero(refs_before == 0)[:, 0]
        need = copied | fresh
        table[need] = ids[:int(need.sum())].to(torch.int32)
        refs[table[need].long()] = 1
        n = old.numel()
        s["copy_src"][:n], s["copy_dst"][:n] = old.to(torch.int32), table[copied]
        lens.copy_(s["new_lens"])
    else:
        used = refs > 0
        count = int(used.sum())
        src, dst = torch.nonzero(used[count:])[:, 0] + count, torch.nonzero(~used[:count])[:, 0]
        n = src.numel()
        to = torch.arange(refs.numel(), device="cuda", dtype=torch.int32)
        to[src] = dst.to(torch.int32)
        live = slots < ((lens + ps - 1) // ps)[:, None]
        table[live] = to[table[live].long()]
        refs[dst] = refs[src]
        refs[src] = 0
        s["copy_src"][:n], s["copy_dst"][:n] = src.to(torch.int32), dst.to(torch.int32)
    s["n_copies"].fill_(n)
    a, b = s["copy_src"][:n].long(), s["copy_dst"][:n].long()
    s["k_pages"][:, b] = s["k_pages"][:, a]
    s["v_pages"][:, b] = s["v_pages"][:, a]
    return table, lens, refs, s["copy_src"], s["copy_dst"], s["n_copies"], s["k_pages"], s["v_pages"]


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "attend": _exact_attend, "sample": _exact_sample, "pages": _exact_pages}[case["kind"]](s)


def _exact_rope(s):
    c = s["case"]
    pos, freq, r = s["positions"].double(), s["inv_freq"].double(), c["rot_dim"]

    def turned(x, w):
        y = x.double().clone()
        if w is not None:
            y /= (y.pow(2).sum(-1, keepdim=True) / c["head_dim"] + 1e-6).sqrt()
            y *= w.double()
        # the pairs as complex numbers, turned by e^(i angle)
        lo = slice(0, r, 2) if c["interleaved"] else slice(0, r // 2)
        hi = slice(1, r, 2) if c["interleaved"] else slice(r // 2, r)
        spin = torch.polar(torch.ones_like(pos)[:, None] * torch.ones_like(freq), torch.outer(pos, freq))
        z = torch.complex(y[..., lo].contiguous(), y[..., hi].contiguous()) * spin[:, None, :]
        y[..., lo], y[..., hi] = z.real, z.imag
        return y

    q, k = turned(s["q"], s["wq"]), turned(s["k"], s["wk"])
    if not c["paged"]:
        return q, k
    kp, vp = s["k_pages"].double(), s["v_pages"].double()
    table = s["table"].cpu().tolist()
    where = []
    for i, (n, kv) in enumerate(zip(s["rows"], s["lens"])):
        where += [table[i][p // c["page"]] * c["page"] + p % c["page"] for p in range(kv - n, kv)]
    where = torch.tensor(where, device="cuda")
    for pool, new in ((kp, k), (vp, s["v"].double())):
        flat = pool.transpose(1, 2).reshape(-1, c["kv_heads"], c["head_dim"])
        flat[where] = new
        pool.copy_(flat.view(pool.shape[0], c["page"], c["kv_heads"], c["head_dim"]).transpose(1, 2))
    return q, kp, vp


def _exact_attend(s):
    c = s["case"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    group = c["q_heads"] // c["kv_heads"]
    for i, (n, kv) in enumerate(zip(s["rows"], s["lens"])):
        limit = torch.tensor(_visible(n, kv, c["mask_block"]), device="cuda")
        hidden = torch.arange(kv, device="cuda")[None, :] >= limit[:, None]
        table = s["table"][i].long()
        at = torch.arange(kv, device="cuda")
        page, slot = table[at // c["page"]], at % c["page"]
        for h in range(c["kv_heads"]):
            k, v = s["k_pages"][page, h, slot].double(), s["v_pages"][page, h, slot].double()
            for g in range(group):
                lo = s["offsets"][i]
                x = s["q"][lo:lo + n, h * group + g].double() @ k.T / math.sqrt(c["head_dim"])
                x[hidden] = float("-inf")
                out[lo:lo + n, h * group + g] = torch.softmax(x, 1) @ v
    return out


def _exact_sample(s):
    vocab = s["case"]["vocab"]
    rows = s["logits"][:, :vocab].double().cpu().numpy()

    def host(name, default):
        return np.full(len(rows), default, np.float64) if s[name] is None else s[name].double().cpu().numpy()

    temperature, top_k, top_p, min_p = host("temperature", 1), host("top_k", 0), host("top_p", 1), host("min_p", 0)
    u = host("u", 0)
    token, prob, kept = [], [], []
    for i, x in enumerate(rows):
        order = np.argsort(-x, kind="stable")
        if temperature[i] <= 0:
            token.append(order[0]), prob.append(1.0), kept.append(1)
            continue
        z = x[order]
        z = z[z > -np.inf]
        w = np.exp((z - z[0]) / temperature[i])
        n = len(w) if top_k[i] <= 0 else min(len(w), int(top_k[i]))
        run = np.cumsum(w)
        k = n
        if top_p[i] < 1:
            k = min(k, int(np.searchsorted(run[:n], top_p[i] * run[n - 1])) + 1)
        if min_p[i] > 0:
            k = min(k, max(1, int((w >= min_p[i]).sum())))
        j = min(int(np.searchsorted(run[:k], u[i] * run[k - 1], side="right")), k - 1)
        token.append(order[j]), prob.append(w[j] / run[k - 1]), kept.append(k)
    return (torch.tensor(np.array(token), dtype=torch.int32), torch.tensor(prob, dtype=torch.float64),
            torch.tensor(kept, dtype=torch.int32))


def _exact_pages(s):
    c, ps = s["case"], s["case"]["page"]
    table, lens, refs = (s[n].cpu().numpy().copy() for n in ("table", "kv_lens", "refs"))
    src, dst = [], []
    if c["what"] == "branch":
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            table[b], lens[b] = table[a], lens[a]
            for page in table[a, :-(-int(lens[a]) // ps)]:
                refs[page] += 1
        shared, free = refs > 1, iter(np.flatnonzero(refs == 0))
        for b in range(c["batch"]):
            new, have = int(s["new_lens"][b]), -(-int(lens[b]) // ps)
            for slot in range(-(-new // ps)):
                page = table[b, slot]
                if slot >= have:
                    table[b, slot] = next(free)
                elif slot >= int(s["write_from"][b]) // ps and shared[page]:
                    table[b, slot] = next(free)
                    refs[page] -= 1
                    src.append(page), dst.append(table[b, slot])
                else:
                    continue
                refs[table[b, slot]] = 1
            lens[b] = new
    else:
        total = int((refs > 0).sum())
        dst = [p for p in range(total) if refs[p] == 0]
        src = [p for p in range(total, len(refs)) if refs[p] > 0]
        to = dict(zip(src, dst))
        for b in range(c["batch"]):
            for slot in range(-(-int(lens[b]) // ps)):
                table[b, slot] = to.get(table[b, slot], table[b, slot])
        for a, b in zip(src, dst):
            refs[b], refs[a] = refs[a], 0
    cs, cd = s["copy_src"].cpu().numpy().copy(), s["copy_dst"].cpu().numpy().copy()
    cs[:len(src)], cd[:len(dst)] = src, dst
    for pool in (s["k_pages"], s["v_pages"]):
        for a, b in zip(src, dst):
            pool[:, int(b)] = pool[:, int(a)]
    return tuple(torch.from_numpy(x) for x in (table, lens, refs, cs, cd)) + (
        torch.tensor([len(src)], dtype=torch.int32), s["k_pages"], s["v_pages"])
