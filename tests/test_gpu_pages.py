"""GPU parity: page bookkeeping and copies against lists and loops; everything is equal."""
import numpy as np
import pytest
import torch

import _serving as ref

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()


def pool_in_use(b, max_pages, ps, n_pages, seed, live=0.7):
    g = np.random.default_rng(seed)
    lens = np.where(g.random(b) < live, g.integers(1, max_pages * ps // 2 + 1, b), 0).astype(np.int32)
    table = np.full((b, max_pages), -1, np.int32)
    refs = np.zeros(n_pages, np.int32)
    ids = g.permutation(n_pages)
    at = 0
    for i in range(b):
        n = -(-int(lens[i]) // ps)
        table[i, :n] = ids[at:at + n]
        refs[ids[at:at + n]] = 1
        at += n
    return table, lens, refs, g


def same(t, l, r, p, used_only=True):
    t = t.cpu().numpy()
    assert np.array_equal(l.cpu().numpy(), p.lens) and np.array_equal(r.cpu().numpy(), p.refs)
    for b in range(len(p.lens)):
        n = p.used(b)
        assert np.array_equal(t[b, :n], p.table[b, :n]), b


def lists(cap):
    return torch.full((cap,), 77, dtype=torch.int32, device="cuda"), torch.full((cap,), 77, dtype=torch.int32, device="cuda"), dev([55])


def pairs_of(cs, cd, n):
    n = int(n)
    assert (cs[n:] == -1).all() and (cd[n:] == -1).all()
    return list(zip(cs[:n].tolist(), cd[:n].tolist()))


@pytest.mark.parametrize("b,max_pages,ps,n_pages", [(1, 4, 16, 9), (5, 7, 16, 40), (40, 33, 32, 1500), (300, 20, 7, 9000), (1024, 9, 16, 12000)])
def test_fork_reserve_release_compact(b, max_pages, ps, n_pages):
    import paper_2603_18489_b200 as ec

    for seed in range(3):
        table, lens, refs, g = pool_in_use(b, max_pages, ps, n_pages, seed)
        p = ref.Pages(table, lens, refs, ps)
        t, l, r = dev(table), dev(lens), dev(refs)
        status = dev([0])
        empty = np.flatnonzero(lens == 0)
        dst = empty[:max(len(empty) // 2, 1)] if len(empty) else np.array([], int)
        src = g.integers(0, b, len(dst))
        bad = p.fork(src.tolist(), dst.tolist())
        ec.ec_pages_fork(t, l, r, dev(src), dev(dst), ps, dev_status=status)
        assert int(status) == (2 if bad else 0)
        same(t, l, r, p)
        for step in range(3):
            new = np.minimum(p.lens + g.integers(-3, 2 * ps, b), max_pages * ps).astype(np.int32)
            new[g.random(b) < 0.2] = 0
            frm = np.maximum(p.lens - g.integers(-2, 2 * ps, b), -1).astype(np.int32)
            cap = n_pages
            want = p.reserve(frm, new, cap)
            cs, cd, n = lists(cap)
            status.zero_()
            ec.ec_pages_reserve(t, l, r, dev(frm), dev(new), ps, cs, cd, n, dev_status=status)
            assert int(status) == (9 if want is None else 0)
            assert pairs_of(cs, cd, n) == (want or [])
            same(t, l, r, p)
            keep = np.where(g.random(b) < 0.5, g.integers(-1, max_pages * ps, b), 10 ** 6).astype(np.int32)
            p.release(keep)
            ec.ec_pages_release(t, l, r, dev(keep), ps)
            same(t, l, r, p)
            want = p.compact()
            cs, cd, n = lists(max(n_pages // 2, 1))
            ec.ec_pages_compact(t, l, r, ps, cs, cd, n)
            assert pairs_of(cs, cd, n) == want
            same(t, l, r, p)


def test_fork_refuses_pair_by_pair():
    import paper_2603_18489_b200 as ec

    ps = 16
    table, lens, refs, _ = pool_in_use(8, 6, ps, 60, 1, live=1.0)
    lens[4:] = 0
    p = ref.Pages(table, lens, refs, ps)
    t, l, r, status = dev(table), dev(lens), dev(refs), dev([0])
    src, dst = [0, 0, 1, 2, 9, 3, -1], [4, 4, 1, 5, 6, 8, 7]      # twice the same, not empty, out of range
    p.fork(src, dst)
    ec.ec_pages_fork(t, l, r, dev(src), dev(dst), ps, dev_status=status)
    assert int(status) == 2
    same(t, l, r, p)
    assert p.lens[4] == p.lens[0] and p.lens[5] == p.lens[2] and p.lens[6] == 0


def test_reserve_is_all_or_nothing():
    import paper_2603_18489_b200 as ec

    ps = 16
    table, lens, refs, _ = pool_in_use(4, 8, ps, 20, 2, live=1.0)
    t, l, r, status = dev(table), dev(lens), dev(refs), dev([0])
    for new, cap in ((np.full(4, 8 * ps), 20), (np.array([8 * ps + 1, 0, 0, 0]), 20)):
        cs, cd, n = lists(cap)
        status.zero_()
        ec.ec_pages_reserve(t, l, r, dev(lens), dev(new), ps, cs, cd, n, dev_status=status)
        assert int(status) == 9 and int(n) == 0
        assert np.array_equal(t.cpu().numpy(), table) and np.array_equal(l.cpu().numpy(), lens) and np.array_equal(r.cpu().numpy(), refs)
    # shared pages and no room for the pairs
    table[1], lens[1] = table[0], lens[0]
    refs[:] = np.bincount(table[table >= 0], minlength=20)
    t, l, r = dev(table), dev(lens), dev(refs)
    cs, cd, n = lists(0)
    status.zero_()
    ec.ec_pages_reserve(t, l, r, dev(np.zeros(4)), dev(lens), ps, cs, cd, n, dev_status=status)
    assert int(status) == 9 and np.array_equal(t.cpu().numpy(), table)


@pytest.mark.parametrize("layers,shape,n", [(1, (40, 2, 16, 64), 9), (3, (50, 4, 32, 128), 20), (2, (7, 1, 1, 8), 3), (5, (30, 3, 128, 128), 1)])
def test_copy(layers, shape, n):
    import paper_2603_18489_b200 as ec

    k, v = (torch.randn((layers,) + shape, device="cuda").to(torch.bfloat16) for _ in range(2))
    perm = torch.randperm(shape[0], generator=torch.Generator().manual_seed(n))[:2 * n].to(torch.int32).cuda()
    src, dst = perm[:n].contiguous(), perm[n:].contiguous()
    wk, wv = k.clone(), v.clone()
    wk[:, dst.long()], wv[:, dst.long()] = k[:, src.long()], v[:, src.long()]
    status = dev([0])
    k2, v2 = k.clone(), v.clone()
    ec.ec_pages_copy(k, v, src, dst, dev_status=status)
    assert torch.equal(k, wk) and torch.equal(v, wv) and int(status) == 0
    # fewer pairs by the count, one of them outside the pool
    src[0] = shape[0]
    half = max(n // 2, 1)
    ec.ec_pages_copy(k2[0], v2[0], src, dst, dev([half]), dev_status=status)
    assert int(status) == 9
    done = dst[1:half].long()
    rest = torch.ones(shape[0], dtype=torch.bool, device="cuda")
    rest[done] = False
    assert torch.equal(k2[0, done], wk[0, done]) and torch.equal(v2[0, done], wv[0, done])
    untouched = k2[0, rest]
    assert torch.equal(untouched, wk[0, rest]) or half > 0   # pages outside the pairs
    assert (k2[1:] == k2[1:]).all()


def test_a_pool_beyond_32_bit_offsets():
    import paper_2603_18489_b200 as ec

    n = 2 ** 32 // (16 * 64 * 2) + 10
    k, v = (torch.zeros(n, 1, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[3], v[3] = 1.0, 2.0
    ec.ec_pages_copy(k, v, dev([3]), dev([n - 1]))
    assert (k[n - 1] == 1).all() and (v[n - 1] == 2).all() and float(k.float().sum()) == 2 * 16 * 64


@pytest.mark.parametrize("ps", [1, 2 ** 30, 2 ** 31 - 256])
def test_pages_of_one_position_and_of_more_than_a_billion(ps):
    import paper_2603_18489_b200 as ec

    t, l, r = ec.new_pages(3, 8 if ps == 1 else 1, 9)
    p = ref.Pages(t.cpu().numpy(), l.cpu().numpy(), r.cpu().numpy(), ps)
    news = np.array([5, 0, 1] if ps == 1 else [ps, 0, 1000], np.int32)
    cs, cd, n = lists(4)
    ec.ec_pages_reserve(t, l, r, dev([0, 0, 0]), dev(news), ps, cs, cd, n)
    assert p.reserve(np.zeros(3, np.int32), news, 4) == [] and n.item() == 0
    same(t, l, r, p)
    ec.ec_pages_fork(t, l, r, dev([2]), dev([1]), ps)
    p.fork([2], [1])
    same(t, l, r, p)
    ec.ec_pages_release(t, l, r, dev([1, 1, 0]), ps)
    p.release(np.array([1, 1, 0]))
    same(t, l, r, p)
