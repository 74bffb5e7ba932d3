"""Page bookkeeping entry by entry: after every call the WHOLE table is what lists and loops give, entries that are not in use
among them (left as they were, -1 behind a cut), and a copy changes the pages of its pairs and nothing else."""
import numpy as np
import pytest
import torch

import _serving as ref

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()


def whole(t, l, r, p, what):
    for have, want, name in ((t, p.table, "table"), (l, p.lens, "lengths"), (r, p.refs, "counts")):
        bad = np.argwhere(have.cpu().numpy() != want)
        assert bad.size == 0, (what, name, bad[:4].tolist())


def pool_in_use(b, max_pages, ps, n_pages, seed):
    """Some sequences empty; what stands behind a sequence's pages is anything at all, ids of the pool among it."""
    g = np.random.default_rng(seed)
    lens = np.where(g.random(b) < 0.7, g.integers(1, max_pages * ps // 2 + 1, b), 0).astype(np.int32)
    table = g.choice([-1, -77, 0, 1, n_pages - 1, n_pages, 2 ** 31 - 1], (b, max_pages)).astype(np.int32)
    refs = np.zeros(n_pages, np.int32)
    ids, at = g.permutation(n_pages), 0
    for i in range(b):
        n = -(-int(lens[i]) // ps)
        table[i, :n] = ids[at:at + n]
        refs[ids[at:at + n]] = 1
        at += n
    return table, lens, refs, g


@pytest.mark.parametrize("b,max_pages,ps,n_pages", [(1, 4, 16, 9), (6, 7, 16, 44), (33, 40, 1, 1400), (40, 33, 32, 1500), (1024, 9, 7, 12000)])
def test_every_entry_after_every_call(b, max_pages, ps, n_pages):
    import paper_2603_18489_b200 as ec

    for seed in range(3):
        table, lens, refs, g = pool_in_use(b, max_pages, ps, n_pages, seed)
        p = ref.Pages(table, lens, refs, ps)
        t, l, r, status = dev(table), dev(lens), dev(refs), dev([0])
        empty = np.flatnonzero(lens == 0)
        dst = empty[:max(len(empty) // 2, 1)] if len(empty) else np.array([], int)
        src = g.integers(0, b, len(dst))
        p.fork(src.tolist(), dst.tolist())
        ec.ec_pages_fork(t, l, r, dev(src), dev(dst), ps, dev_status=status)
        whole(t, l, r, p, "fork")
        for step in range(3):
            new = np.minimum(p.lens + g.integers(-3, 2 * ps + 1, b), max_pages * ps).astype(np.int32)
            new[g.random(b) < 0.2] = 0
            frm = np.maximum(p.lens - g.integers(-2, 2 * ps + 1, b), -1).astype(np.int32)
            p.reserve(frm, new, n_pages)
            cs, cd, n = dev(np.full(n_pages, 77)), dev(np.full(n_pages, 77)), dev([55])
            ec.ec_pages_reserve(t, l, r, dev(frm), dev(new), ps, cs, cd, n, dev_status=status)
            whole(t, l, r, p, "reserve")
            keep = np.where(g.random(b) < 0.5, g.integers(-1, max_pages * ps, b), 10 ** 6).astype(np.int32)
            before = p.lens.copy()
            p.release(keep)
            ec.ec_pages_release(t, l, r, dev(keep), ps)
            whole(t, l, r, p, "release")
            for i in range(b):                      # (what the interface says of them, apart from the lists)
                k = max(int(keep[i]), 0)
                if k < before[i]:
                    assert (t[i, -(-k // ps):-(-int(before[i]) // ps)] == -1).all()
                if b > 64 and i > 64:
                    break
            p.compact()
            cs, cd = dev(np.full(max(n_pages // 2, 1), 77)), dev(np.full(max(n_pages // 2, 1), 77))
            ec.ec_pages_compact(t, l, r, ps, cs, cd, n)
            whole(t, l, r, p, "compact")


@pytest.mark.parametrize("layers,shape,n", [(1, (40, 2, 16, 64), 9), (3, (50, 4, 32, 128), 20), (2, (7, 1, 1, 8), 3), (5, (30, 3, 128, 128), 2)])
def test_copy_changes_the_pages_of_its_pairs_alone(layers, shape, n):
    import paper_2603_18489_b200 as ec

    g = torch.Generator().manual_seed(n)
    k0, v0 = (torch.randn((layers,) + shape, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    perm = torch.randperm(shape[0], generator=g)[:2 * n].tolist()
    src, dst = perm[:n], perm[n:]
    src[0] = shape[0]                                     # outside the pool: skipped
    for layer, count in ((None, n - 1), (0, n - 1), (layers - 1, 1), (0, 0), (None, -3), (None, 10 ** 6)):
        k, v, want_k, want_v, status = k0.clone(), v0.clone(), k0.clone(), v0.clone(), dev([0])
        at = slice(None) if layer is None else slice(layer, layer + 1)
        pairs = list(zip(src, dst))[:max(count, 0)]
        for a, b in pairs:
            if a < shape[0]:
                want_k[at, b], want_v[at, b] = k0[at, a], v0[at, a]
        ec.ec_pages_copy(k if layer is None else k[layer], v if layer is None else v[layer], dev(src), dev(dst), dev([count]),
                         dev_status=status)
        assert torch.equal(k, want_k) and torch.equal(v, want_v), (layer, count)
        assert int(status) == (9 if pairs else 0)
