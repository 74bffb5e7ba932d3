"""GPU parity: ec_qk_norm_rope and ec_qk_norm_rope_paged against the 64-bit form."""
import numpy as np
import pytest
import torch

import _serving as ref

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def f64(t):
    return t.detach().cpu().double().numpy()


def inputs(dtype, n, hq, hkv, d, norm, rot, seed=0, top=100000, pad=0):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(n, (hq + 2 * hkv) * d + pad, generator=g).to(dtype).cuda()
    q, k, v = (qkv[:, o * d:(o + h) * d].unflatten(1, (h, d)) for o, h in ((0, hq), (hq, hkv), (hq + hkv, hkv)))
    pos = torch.randint(0, top, (n,), generator=g, dtype=torch.int32).cuda()
    freq = (10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) / max(rot // 2, 1))).float().cuda()
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(dtype).cuda() if norm else None for _ in range(2)]
    return q, k, v, pos, freq, w


def close(got, x, w, pos, freq, rot, inter, eps=1e-6):
    y, size = ref.norm_rope(f64(x), None if w is None else f64(w), eps, pos.cpu().numpy(), f64(freq), rot, inter)
    tol = ref.rope_tolerance(y, size, got.dtype == BF)
    err = np.abs(f64(got) - y)
    assert (err <= tol).all(), float((err - tol).max())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 64), (64, 16), (128, 0), (128, 112)])
@pytest.mark.parametrize("norm,inter", [(True, False), (False, True), (True, True), (False, False)])
def test_dense(dtype, d, rot, norm, inter):
    import paper_2603_18489_b200 as ec

    q, k, _, pos, freq, w = inputs(dtype, 37, 5, 2, d, norm, rot)
    desc = ec.make_rope_desc(5, 2, d, dtype, rot, interleaved=inter)
    qo, ko = ec.ec_qk_norm_rope(desc, q, k, pos, freq if rot else None, *w)
    close(qo, q, w[0], pos, freq, rot, inter)
    close(ko, k, w[1], pos, freq, rot, inter)


@pytest.mark.parametrize("n", [1, 2, 1200, 5000])
def test_row_counts(n):
    import paper_2603_18489_b200 as ec

    q, k, _, pos, freq, w = inputs(BF, n, 7, 1, 128, True, 128, pad=8)
    qo, ko = ec.ec_qk_norm_rope(ec.make_rope_desc(7, 1, 128, BF, 128), q, k, pos, freq, *w)
    close(qo, q, w[0], pos, freq, 128, False)
    close(ko, k, w[1], pos, freq, 128, False)


def test_far_positions_and_small_values():
    import paper_2603_18489_b200 as ec

    q, k, _, pos, freq, w = inputs(F32, 16, 2, 2, 64, True, 64, top=2 ** 31 - 1)
    q, k = q * 1e-4, k * 1e3
    desc = ec.make_rope_desc(2, 2, 64, F32, 64, eps=1e-5)
    qo, ko = ec.ec_qk_norm_rope(desc, q, k, pos, freq, *w)
    close(qo, q, w[0], pos, freq, 64, False, 1e-5)
    close(ko, k, w[1], pos, freq, 64, False, 1e-5)
    z = torch.zeros_like(q)
    zo, _ = ec.ec_qk_norm_rope(ec.make_rope_desc(2, 2, 64, F32, 64, eps=1e-6), z, k, pos, freq, *w)
    assert (zo == 0).all()


def test_in_place_padding_rows_and_four_dimensions():
    import paper_2603_18489_b200 as ec

    q, k, _, pos, freq, w = inputs(BF, 24, 4, 2, 64, True, 64)
    q, k = q.contiguous(), k.contiguous()
    pos[5] = -1
    pos[23] = -7
    desc = ec.make_rope_desc(4, 2, 64, BF, 64)
    want_q, want_k = torch.full_like(q, 3.0), torch.full_like(k, 3.0)
    ec.ec_qk_norm_rope(desc, q, k, pos, freq, *w, q_out=want_q, k_out=want_k)
    live = pos >= 0
    close(want_q[live], q[live], w[0], pos[live], freq, 64, False)
    assert (want_q[~live] == 3.0).all() and (want_k[~live] == 3.0).all()
    q4, k4 = q.clone().view(2, 12, 4, 64), k.clone().view(2, 12, 2, 64)
    ec.ec_qk_norm_rope(desc, q4, k4, pos.view(2, 12), freq, *w, q_out=q4, k_out=k4)
    assert torch.equal(q4.view(24, 4, 64)[live], want_q[live]) and torch.equal(k4.view(24, 2, 64)[live], want_k[live])
    assert torch.equal(q4.view(24, 4, 64)[~live], q[~live])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("ps,d,rot,inter,norm", [(16, 128, 128, False, True), (64, 64, 32, True, False), (32, 128, 64, False, True)])
def test_paged(dtype, ps, d, rot, inter, norm):
    import paper_2603_18489_b200 as ec

    hq, hkv, rows, lens = 6, 3, [7, 0, 1, 30], [50, 0, ps + 1, 30]
    n = sum(rows)
    q, k, v, _, freq, w = inputs(dtype, n + 5, hq, hkv, d, norm, rot)
    per = [-(-x // ps) for x in lens]
    n_pages, max_pages = sum(per) + 2, max(per) + 1
    ids = torch.randperm(n_pages, generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    table = torch.full((4, max_pages), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, m in enumerate(per):
        table[b, :m] = ids[at:at + m]
        at += m
    offsets = torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32, device="cuda")
    pos = torch.tensor([kv - r + i for r, kv in zip(rows, lens) for i in range(r)] + [0] * 5, dtype=torch.int32, device="cuda")
    pos[3] = -1                                                     # a padding row inside a sequence
    kp, vp = (torch.randn(n_pages, hkv, ps, d, device="cuda").to(dtype) for _ in range(2))
    k0, v0 = kp.clone(), vp.clone()
    desc = ec.make_rope_desc(hq, hkv, d, dtype, rot, interleaved=inter)
    paged = ec.make_paged_desc(4, hq, hkv, d, dtype, ps, n_pages, max_pages)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    qo = torch.full((n + 5, hq, d), 3.0, dtype=dtype, device="cuda")
    ec.ec_qk_norm_rope_paged(desc, paged, q, k, v, offsets, pos, freq, table, kp, vp, *w, q_out=qo, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    assert (qo[n:] == 3.0).all() and (qo[3] == 3.0).all()
    row = 0
    for b, r in enumerate(rows):
        for i in range(r):
            if row + i == 3:
                continue
            p = int(pos[row + i])
            page, slot = int(table[b, p // ps]), p % ps
            sl = slice(row + i, row + i + 1)
            close(kp[page, :, slot][None], k[sl], w[1], pos[sl], freq, rot, inter)
            close(qo[sl], q[sl], w[0], pos[sl], freq, rot, inter)
            assert torch.equal(vp[page, :, slot], v[row + i])
            k0[page, :, slot], v0[page, :, slot] = kp[page, :, slot], vp[page, :, slot]
        row += r
    assert torch.equal(kp, k0) and torch.equal(vp, v0)              # nothing else was written
    # a page outside the pool, a position outside the table: refused row by row
    for bad_table, bad_pos, code in ((n_pages, None, 9), (-1, None, 9), (None, max_pages * ps, 2)):
        t2, p2 = table.clone(), pos.clone()
        if bad_table is not None:
            t2[3, 0] = bad_table
        else:
            p2[n - 1] = bad_pos
        status.zero_()
        ec.ec_qk_norm_rope_paged(desc, paged, q, k, v, offsets, p2, freq, t2, kp, vp, *w, q_out=qo, dev_status=status)
        assert int(status) == code
    assert torch.equal(kp, k0) and torch.equal(vp, v0)
