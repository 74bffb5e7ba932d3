"""The serving operators in the order in which a program calls them, against histories kept on the host; and the paged path
against the dense one."""
import numpy as np
import pytest
import torch

import _serving as ref

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def f64(t):
    return t.detach().cpu().double().numpy()


def dev(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()


class Program:
    """Two layers' pools, slots for sequences, one step after another; K and V of every sequence are kept as 64-bit arrays too."""

    def __init__(self, slots=5, hq=6, hkv=2, d=64, ps=16, max_pages=12, n_pages=40, mask=4, seed=0):
        import paper_2603_18489_b200 as ec

        self.ec, self.g = ec, np.random.default_rng(seed)
        self.hq, self.hkv, self.d, self.ps, self.mask, self.slots = hq, hkv, d, ps, mask, slots
        self.table, self.lens, self.refs = ec.new_pages(slots, max_pages, n_pages)
        self.k, self.v = (torch.full((2, n_pages, hkv, ps, d), float("nan"), dtype=BF, device="cuda") for _ in range(2))
        self.paged = ec.make_paged_desc(slots, hq, hkv, d, BF, ps, n_pages, max_pages, mask_block=mask)
        self.rope = ec.make_rope_desc(hq, hkv, d, BF, d)
        self.freq = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).float().cuda()
        self.w = [(1 + 0.2 * torch.randn(d)).to(BF).cuda() for _ in range(2)]
        self.lists = [torch.empty(n_pages, dtype=torch.int32, device="cuda") for _ in range(2)] + [dev([0])]
        self.status = dev([0])
        self.hist = [[np.zeros((0, hkv, d)) for _ in range(2)] for _ in range(slots)]   # layer 0: K, V

    def copies(self):
        self.ec.ec_pages_copy(self.k, self.v, *self.lists, dev_status=self.status)

    def reserve(self, write_from, new_lens):
        self.ec.ec_pages_reserve(self.table, self.lens, self.refs, dev(write_from), dev(new_lens), self.ps, *self.lists, dev_status=self.status)
        self.copies()

    def step(self, rows, write_from):
        """`rows[b]` rows of sequence b at positions write_from[b] .. (its end)."""
        n = sum(rows)
        end = [w + r if r else len(h[0]) for w, r, h in zip(write_from, rows, self.hist)]
        self.reserve(write_from, end)
        qkv = torch.randn(n, (self.hq + 2 * self.hkv) * self.d).to(BF).cuda()
        q, k, v = (qkv[:, o * self.d:(o + h) * self.d].unflatten(1, (h, self.d)) for o, h in
                   ((0, self.hq), (self.hq, self.hkv), (self.hq + self.hkv, self.hkv)))
        offsets = dev([0] + list(np.cumsum(rows)))
        pos = np.concatenate([np.arange(w, w + r) for w, r in zip(write_from, rows)]).astype(np.int64)
        args = (self.rope, self.paged, q, k, v, offsets, dev(pos), self.freq, self.table)
        qo = self.ec.ec_qk_norm_rope_paged(*args, self.k[0], self.v[0], *self.w, dev_status=self.status)
        self.ec.ec_qk_norm_rope_paged(*args, self.k[1], self.v[1], *self.w)
        out = self.ec.ec_attend_paged(self.paged, qo, offsets, self.lens, max(rows), self.table, self.k[0], self.v[0],
                                      dev_status=self.status)
        assert int(self.status) == 0
        # the host's side
        kr, size = ref.norm_rope(f64(k), f64(self.w[1]), 1e-6, pos, f64(self.freq), self.d, False)
        tol = ref.rope_tolerance(kr, size, True)
        at = 0
        table, lens = self.table.cpu().numpy(), self.lens.cpu().numpy()
        for b, r in enumerate(rows):
            if r == 0:
                continue
            for i, new in enumerate((kr, f64(v))):
                self.hist[b][i] = np.concatenate([self.hist[b][i][:write_from[b]], new[at:at + r]])
            kv = end[b]
            assert lens[b] == kv
            kc, vc = (ref.gather(f64(p[0]), table[b], kv, self.ps) for p in (self.k, self.v))
            # what stands in the pages is the history: V to the bit, K to one rounding
            assert np.array_equal(vc, self.hist[b][1].transpose(1, 0, 2))
            new_k = kc[:, write_from[b]:].transpose(1, 0, 2)
            assert (np.abs(new_k - kr[at:at + r]) <= tol[at:at + r]).all()
            old = self.hist[b][0][:write_from[b]].transpose(1, 0, 2)
            assert (np.abs(kc[:, :write_from[b]] - old) <= np.abs(old) * 2.0 ** -7 + 1e-4).all()
            want, mass, sz = ref.attend(f64(qo)[at:at + r], kc, vc, ref.visible(r, kv, self.mask), self.d ** -0.5)
            assert (np.abs(f64(out)[at:at + r] - want) <= ref.attend_tolerance(want, mass, sz, self.d, kv, True)).all()
            at += r
        assert torch.equal(self.v[0][self.refs > 0].isnan(), self.v[1][self.refs > 0].isnan())   # the layers move together
        return out

    def invariants(self):
        table, lens, refs = self.table.cpu().numpy(), self.lens.cpu().numpy(), self.refs.cpu().numpy()
        count = np.zeros_like(refs)
        for b, n in enumerate(lens):
            np.add.at(count, table[b, :-(-int(n) // self.ps)], 1)
        assert np.array_equal(count, refs)


def test_prompts_branches_sampled_steps_and_compaction():
    torch.manual_seed(0)
    p = Program()
    ec = p.ec
    p.step([37, 0, 50, 0, 0], [0, 0, 0, 0, 0])                       # two prompts
    ec.ec_pages_fork(p.table, p.lens, p.refs, dev([0, 2, 0]), dev([1, 3, 4]), p.ps, dev_status=p.status)
    for a, b in ((0, 1), (2, 3), (0, 4)):
        p.hist[b] = [h.copy() for h in p.hist[a]]
    p.invariants()
    assert int((p.refs > 1).sum()) > 0
    before = f64(p.v[0])[p.table.cpu().numpy()[0, :3]]
    p.step([0, 4, 4, 1, 4], [37, 37, 50, 50, 37])                    # the branches write; the parents' pages stay
    assert np.array_equal(f64(p.v[0])[p.table.cpu().numpy()[0, :3]], before, equal_nan=True)
    p.invariants()
    p.step([4, 4, 4, 3, 4], [36, 40, 52, 50, 37])                    # some positions are written again (a block denoised once more)
    p.invariants()
    # tokens of the step's last rows: the logits of a projection, and the same numbers against the 64-bit form
    out = p.step([1, 1, 1, 1, 1], [40, 44, 56, 53, 41])
    logits = (out.flatten(1).float() @ torch.randn(p.hq * p.d, 1008, device="cuda") * 0.3).to(BF)
    u = torch.rand(5, device="cuda")
    top_p, top_k = torch.full((5,), 0.9, device="cuda"), dev([0, 50, 5, 1, 0])
    got = ec.ec_sample(logits, 1003, u, top_p=top_p, top_k=top_k)
    for b in range(5):
        want = ref.sample(logits[b, :1003].float().cpu().numpy(), u[b].item(), top_p=top_p[b].item(), top_k=int(top_k[b]))
        assert (int(got["token"][b]), int(got["kept"][b])) == (want[0], want[2])
    # a branch ends, another is cut back, the pool is moved together, and the rest goes on
    ec.ec_pages_release(p.table, p.lens, p.refs, dev([0, 20, 1000, 1000, 1000]), p.ps)
    p.hist[0] = [h[:0] for h in p.hist[0]]
    p.hist[1] = [h[:20] for h in p.hist[1]]
    p.invariants()
    ec.ec_pages_compact(p.table, p.lens, p.refs, p.ps, *p.lists)
    p.copies()
    p.invariants()
    used = int((p.refs > 0).sum())
    assert (p.refs[:used] > 0).all() and (p.refs[used:] == 0).all()
    p.step([20, 3, 2, 70, 1], [0, 20, 57, 54, 42])
    p.invariants()


@pytest.mark.parametrize("dtype,hq,hkv,d,n,L", [(BF, 8, 8, 128, 34, 300), (BF, 14, 2, 128, 34, 768), (torch.float32, 4, 4, 64, 34, 256)])
def test_paged_equals_dense(dtype, hq, hkv, d, n, L):
    """The same rows through ec_qk_norm_rope and ec_attend over a dense cache, and through the pages."""
    import paper_2603_18489_b200 as ec

    g = torch.Generator().manual_seed(4)
    ps = 16
    pages = -(-L // ps)
    kc, vc = (torch.randn(1, hkv, L, d, generator=g).to(dtype).cuda() for _ in range(2))
    q, k, v = (torch.randn(1, n, h, d, generator=g).to(dtype).cuda() for h in (hq, hkv, hkv))
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(dtype).cuda() for _ in range(2)]
    idx = torch.randperm(L, generator=g)[:n].to(torch.int32).cuda()          # active rows anywhere in the sequence
    freq = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).float().cuda()
    table = torch.randperm(pages, generator=g).to(torch.int32).cuda()[None]
    kp, vp = (torch.zeros(pages, hkv, ps, d, dtype=dtype, device="cuda") for _ in range(2))
    for e in range(pages):
        m = min(ps, L - e * ps)
        kp[table[0, e], :, :m], vp[table[0, e], :, :m] = kc[0, :, e * ps:e * ps + m], vc[0, :, e * ps:e * ps + m]
    rope = ec.make_rope_desc(hq, hkv, d, dtype, d)
    qo, ko = ec.ec_qk_norm_rope(rope, q, k, idx, freq, *w)
    dense = ec.ec_attend(ec.make_desc(1, L, hq, hkv, d, dtype), qo, ko, v, kc, vc, idx[None])
    desc = ec.make_paged_desc(1, hq, hkv, d, dtype, ps, pages, pages)
    offsets = dev([0, n])
    q2 = ec.ec_qk_norm_rope_paged(rope, desc, q[0], k[0], v[0], offsets, idx, freq, table, kp, vp, *w)
    assert torch.equal(q2, qo[0])
    out = ec.ec_attend_paged(desc, q2, offsets, dev([L]), n, table, kp, vp)
    for e in range(pages):
        m = min(ps, L - e * ps)
        assert torch.equal(kp[table[0, e], :, :m], kc[0, :, e * ps:e * ps + m])
    k64, v64 = f64(kc)[0], f64(vc)[0]
    want, mass, size = ref.attend(f64(q2), k64, v64, np.full(n, L), d ** -0.5)
    tol = ref.attend_tolerance(want, mass, size, d, L, dtype == BF)
    assert (np.abs(f64(out) - want) <= tol).all()
    assert (np.abs(f64(out) - f64(dense)[0]) <= 2 * tol).all()


def test_a_whole_step_captured():
    """Rotation, attention, projection, sampling and the pages' growth in one graph, replayed: every step as when called."""
    import paper_2603_18489_b200 as ec

    torch.manual_seed(3)
    hq, hkv, d, ps, slots = 4, 2, 64, 16, 3
    lens0 = [20, 33, 7]

    def fresh():
        table, lens, refs = ec.new_pages(slots, 8, 24)
        k, v = (torch.zeros(24, hkv, ps, d, dtype=BF, device="cuda") for _ in range(2))
        return dict(table=table, lens=lens, refs=refs, k=k, v=v, new=dev(lens0), grow=torch.ones(slots, dtype=torch.int32, device="cuda"),
                    cs=torch.empty(24, dtype=torch.int32, device="cuda"), cd=torch.empty(24, dtype=torch.int32, device="cuda"), n=dev([0]),
                    token=torch.zeros(slots, dtype=torch.int32, device="cuda"), ws1=ec.new_workspace(ec.ec_pages_workspace_bytes(24)),
                    status=dev([0]), prob=torch.zeros(slots, device="cuda"), kept=torch.zeros(slots, dtype=torch.int32, device="cuda"))

    desc = ec.make_paged_desc(slots, hq, hkv, d, BF, ps, 24, 8, mask_block=1)
    rope = ec.make_rope_desc(hq, hkv, d, BF, d)
    freq = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).float().cuda()
    embed = torch.randn(512, (hq + 2 * hkv) * d, device="cuda").to(BF)
    proj = (torch.randn(hq * d, 512, device="cuda") * 0.3).to(BF)
    offsets, u = dev(np.arange(slots + 1)), torch.rand(slots, device="cuda")
    top_p = torch.full((slots,), 0.9, device="cuda")
    ws2 = ec.new_workspace(ec.ec_attend_paged_workspace_bytes(desc, 1))
    ws3 = ec.new_workspace(ec.ec_sample_workspace_bytes(slots, 512))

    def step(s):
        s["pos"] = s["new"].clone()
        s["new"].add_(s["grow"])
        ec.ec_pages_reserve(s["table"], s["lens"], s["refs"], s["pos"], s["new"], ps, s["cs"], s["cd"], s["n"], workspace=s["ws1"], dev_status=s["status"])
        ec.ec_pages_copy(s["k"], s["v"], s["cs"], s["cd"], s["n"], dev_status=s["status"])
        qkv = embed[s["token"].long()]
        q, k, v = (qkv[:, o * d:(o + h) * d].unflatten(1, (h, d)) for o, h in ((0, hq), (hq, hkv), (hq + hkv, hkv)))
        qo = ec.ec_qk_norm_rope_paged(rope, desc, q, k, v, offsets, s["pos"], freq, s["table"], s["k"], s["v"], dev_status=s["status"])
        out = ec.ec_attend_paged(desc, qo, offsets, s["lens"], 1, s["table"], s["k"], s["v"], workspace=ws2, dev_status=s["status"])
        ec.ec_sample(out.flatten(1) @ proj, 512, u, top_p=top_p, token_out=s["token"], prob_out=s["prob"], kept_out=s["kept"], workspace=ws3)

    a = fresh()
    called = []
    for _ in range(40):
        step(a)
        called.append(a["token"].tolist())
    assert int(a["status"]) == 0 and len({tuple(t) for t in called}) > 5
    b = fresh()
    start = {n: t.clone() for n, t in b.items() if torch.is_tensor(t)}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(b)
    for n, t in start.items():
        b[n].copy_(t)
    for i in range(40):
        graph.replay()
        assert b["token"].tolist() == called[i], i
    assert int(b["status"]) == 0 and torch.equal(a["k"], b["k"]) and torch.equal(a["table"], b["table"])


def test_what_a_call_makes_belongs_to_its_stream(monkeypatch):
    """Outputs and workspaces that are not given are made on the stream that is: a fill on another one, or another's use of the
    memory once the call has returned, would run beside its kernels."""
    import paper_2603_18489_b200 as ec

    p = Program()
    q = torch.randn(3, p.hq, p.d, dtype=BF, device="cuda")
    k, v = (torch.randn(3, p.hkv, p.d, dtype=BF, device="cuda") for _ in range(2))
    ro, pos, none, lens = dev([0, 2, 2, 3, 3, 3]), dev([0, 1, 0]), dev([0] * 5), dev([2, 0, 1, 0, 0])
    x, u = torch.randn(4, 512, device="cuda"), torch.rand(4, device="cuda")
    p.k.zero_(), p.v.zero_()

    def step(stream):
        ec.ec_pages_reserve(p.table, p.lens, p.refs, none, lens, p.ps, *p.lists, stream=stream)
        a, b = ec.ec_qk_norm_rope(p.rope, q, k, pos, p.freq, stream=stream)
        c = ec.ec_qk_norm_rope_paged(p.rope, p.paged, q, k, v, ro, pos, p.freq, p.table, p.k[0], p.v[0], stream=stream)
        o = ec.ec_attend_paged(p.paged, c, ro, p.lens, 2, p.table, p.k[0], p.v[0], stream=stream)
        s = ec.ec_sample(x, 512, u, stream=stream)
        ec.ec_pages_compact(p.table, p.lens, p.refs, p.ps, *p.lists, stream=stream)
        return a, b, c, o, s["token"], s["prob"], s["kept"]

    want = step(None)
    torch.cuda.synchronize()
    side, made = torch.cuda.Stream(), []
    for name in ("empty", "empty_like", "zeros"):
        was = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, was=was, **kw: (made.append(torch.cuda.current_stream()), was(*a, **kw))[1])
    got = step(side)
    monkeypatch.undo()
    side.synchronize()
    assert len(made) == 11 and all(s == side for s in made)     # 7 outputs, workspaces of four calls
    assert all(torch.equal(g, w) for g, w in zip(got, want))
