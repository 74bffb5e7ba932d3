"""GPU parity: ec_sample against the 64-bit form; tokens and counts equal, probabilities to fp32's rounding."""
import numpy as np
import pytest
import torch

import _serving as ref

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def run(x, u, temperature=None, top_k=None, top_p=None, min_p=None, vocab=None):
    import paper_2603_18489_b200 as ec

    n, vocab = x.shape[0], vocab or x.shape[1]

    def vec(a, dt):
        return None if a is None else torch.as_tensor(np.broadcast_to(np.asarray(a), (n,)).copy(), dtype=dt).cuda()

    args = dict(temperature=vec(temperature, F32), top_k=vec(top_k, torch.int32), top_p=vec(top_p, F32), min_p=vec(min_p, F32))
    uu = vec(u, F32)
    got = ec.ec_sample(x, vocab, uu, **args)
    torch.cuda.synchronize()
    host = x.float().cpu().numpy()[:, :vocab]
    default = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    cols = {k: (np.full(n, default[k]) if a is None else a.cpu().numpy()) for k, a in args.items()}
    for i in range(n):
        want = ref.sample(host[i], uu[i].item(), **{k: a[i] for k, a in cols.items()})
        have = (int(got["token"][i]), float(got["prob"][i]), int(got["kept"][i]))
        assert have[0] == want[0] and have[2] == want[2], (i, have, want, {k: a[i] for k, a in cols.items()})
        # one rounding to fp32; the weights' own 1e-13 and the units' 2^-42 of 1 over up to 2^17 tokens stay below 2^-25
        assert abs(have[1] - want[1]) <= want[1] * (2.0 ** -24 + 2.0 ** -25), (i, have, want)
    return got


def logits(n, v, dtype, seed=0, sigma=None, pad=0):
    g = torch.Generator().manual_seed(seed)
    s = torch.rand(n, 1, generator=g) * 7.5 + 0.5 if sigma is None else torch.full((n, 1), float(sigma))
    x = torch.randn(n, v + pad, generator=g) * s
    return x.to(dtype).cuda(), torch.rand(n, generator=g).numpy().astype(np.float32)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("v,pad", [(1, 7), (2, 6), (7, 1), (64, 0), (1000, 0), (4097, 7), (50001, 7), (126464, 0)])
def test_vocabularies_without_filters(dtype, v, pad):
    x, u = logits(6, v, dtype, pad=pad)
    run(x, u, vocab=v)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [1, 3, 40, 300])
def test_all_filters_mixed(dtype, n):
    x, u = logits(n, 32008, dtype, seed=n)
    g = np.random.default_rng(n)
    t = np.where(g.random(n) < 0.1, 0.0, g.uniform(0.1, 2.0, n)).astype(np.float32)
    k = np.where(g.random(n) < 0.3, 0, g.integers(1, 2000, n)).astype(np.int32)
    p = np.where(g.random(n) < 0.3, 1.0, g.uniform(0.05, 0.999, n)).astype(np.float32)
    m = np.where(g.random(n) < 0.3, 0.0, g.uniform(0.0, 0.3, n)).astype(np.float32)
    run(x, u, t, k, p, m)


@pytest.mark.parametrize("kw", [dict(top_k=1), dict(top_k=50), dict(top_k=9000), dict(top_k=10 ** 6), dict(top_k=-3), dict(top_p=0.9),
                                dict(top_p=0.0), dict(top_p=-1.0), dict(top_p=1e-9), dict(top_p=0.9999999), dict(top_p=2.0),
                                dict(min_p=0.05), dict(min_p=1.0), dict(min_p=1.5), dict(min_p=1e-20), dict(temperature=0.0),
                                dict(temperature=1e-6), dict(temperature=50.0), dict(temperature=1e-30), dict(temperature=1e20),
                                dict(top_k=20000, top_p=0.95), dict(top_k=30, top_p=0.5, min_p=0.01, temperature=3.0)])
def test_single_filters(kw):
    for dtype, sigma in ((BF, 0.5), (F32, 0.5), (F32, 6.0), (BF, 3.0)):
        x, u = logits(4, 20008, dtype, seed=5, sigma=sigma)
        run(x, u, **kw)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_ties_constant_rows_and_masked_tokens(dtype):
    v = 40000
    x = torch.zeros(8, v, dtype=dtype, device="cuda")
    x[1] = -3.5
    x[2, ::2] = 1.0
    x[3] = float("-inf")
    x[4] = float("-inf")
    x[4, 777] = -1e30
    x[5] = torch.finfo(dtype).min
    x[5, 3:9] = 2.0
    x[6, ::3] = -0.0
    x[7] = float("-inf")
    x[7, 100:200] = torch.finfo(dtype).min
    for u in (0.0, 0.25, 0.5, 0.75, float(np.float32(1 - 2 ** -24))):
        run(x, u)
        run(x, u, top_p=0.5)
        run(x, u, top_k=12345)
        run(x, u, top_k=300, top_p=0.5, min_p=0.5)
    run(x, 0.3, temperature=0.0)


def test_prefix_views_other_rows_and_outputs_left_out():
    import paper_2603_18489_b200 as ec

    x, u = logits(9, 4096, BF, pad=512)
    got = run(x, u, vocab=4096, top_p=0.8)
    # rows of a larger buffer
    big = torch.full((9, 8192), 100.0, dtype=BF, device="cuda")
    big[:, :4608] = x
    t = torch.as_tensor(u).cuda()
    two = ec.ec_sample(big[:, :4608], 4096, t, top_p=torch.full((9,), 0.8, device="cuda"))
    assert all(torch.equal(got[k], two[k]) for k in got)


def test_deterministic_whatever_the_split():
    """One row alone (a cluster of CTAs) and among many (one CTA each) give the same bits; so does a replayed graph."""
    import paper_2603_18489_b200 as ec

    x, u = logits(200, 60000, F32, seed=3)
    t = torch.as_tensor(u).cuda()
    p = torch.full((200,), 0.95, device="cuda")
    many = ec.ec_sample(x, 60000, t, top_p=p)
    for i in range(0, 200, 37):
        one = ec.ec_sample(x[i:i + 1], 60000, t[i:i + 1], top_p=p[i:i + 1])
        few = ec.ec_sample(x[i:i + 3], 60000, t[i:i + 3], top_p=p[i:i + 3])
        assert all(torch.equal(many[k][i:i + 1], one[k]) and torch.equal(many[k][i:i + 3], few[k]) for k in many)
    out = {k: torch.empty_like(v) for k, v in many.items()}
    ws = ec.new_workspace(ec.ec_sample_workspace_bytes(200, 60000))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ec.ec_sample(x, 60000, t, top_p=p, token_out=out["token"], prob_out=out["prob"], kept_out=out["kept"], workspace=ws)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(many[k], out[k]) for k in many)


def test_frequencies():
    """20000 equally spaced numbers draw every token in proportion."""
    import paper_2603_18489_b200 as ec

    n = 20000
    row = torch.tensor([0.0, 1.0, 2.0, float("-inf"), 1.0, -1.0, 0.5, 0.25], device="cuda")
    u = (torch.arange(n, device="cuda") + 0.5) / n
    got = ec.ec_sample(row.repeat(n, 1), 8, u)["token"]
    share = torch.bincount(got.long(), minlength=8).double() / n
    assert (share - torch.softmax(row.double(), 0)).abs().max() <= 1.0 / n


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_largest_vocabulary(dtype):
    v = 1 << 20
    x, u = logits(3, v, dtype, seed=9, sigma=2.0)
    x[2] = 0.25                     # equal logits: found by the index
    run(x, u)
    run(x, u, top_k=70000, top_p=0.7, min_p=1e-4)
    run(x, u, top_p=0.3, temperature=0.5)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("v", [5, 1001, 20001])
def test_what_stands_behind_the_vocabulary_is_not_read(dtype, v):
    x, u = logits(5, v, dtype, pad=-v % 8 + 16)
    x[:, v:] = float("nan")
    run(x, u, vocab=v, top_p=0.9)
    x[:, v:] = float("inf")
    run(x, u, vocab=v, top_k=3)


def test_clusters_of_equal_and_scattered_logits():
    """Rows that the estimates cannot settle, and rows that they can, next to one another."""
    g = torch.Generator().manual_seed(2)
    x = torch.randn(12, 60000, generator=g)
    x[0] = torch.where(torch.rand(60000, generator=g) < 0.5, 1.0, 0.0)            # two values
    x[1] = (torch.randint(0, 5, (60000,), generator=g) * 0.01).float()            # five close ones
    x[2, :50000] = 3.0
    x[3] = torch.linspace(0, 1e-4, 60000)                                          # all but equal
    x[4] = torch.linspace(-80, 0, 60000)
    x[5] *= 1e-6
    x[6] *= 1e4
    x[7, 100:] = -1e30
    u = torch.rand(12, generator=g).numpy().astype(np.float32)
    for dtype in (F32, BF):
        y = x.to(dtype).cuda()
        run(y, u)
        run(y, u, top_p=0.6)
        run(y, u, top_k=30000, top_p=0.9)
        run(y, u, top_k=30000, min_p=0.3, temperature=0.7)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("v", [24, 20008, 200000])
def test_rows_with_nan_and_infinities(dtype, v):
    """NaN counts as -inf; a row with +inf gives the first such token, for certain."""
    import paper_2603_18489_b200 as ec

    x, u = logits(6, v, dtype, seed=4, sigma=2.0)
    x[0, ::3] = float("nan")
    x[1] = float("nan")
    x[2, 1:] = float("nan")
    x[3, 5::7] = float("inf")
    x[4, ::2] = float("nan")
    x[4, 9] = float("inf")
    x[5] = float("-inf")
    plain = torch.where(torch.isnan(x), torch.full_like(x, float("-inf")), x)
    ut = torch.tensor(u, device="cuda")
    for kw in ({}, dict(top_p=0.7), dict(top_k=7), dict(top_k=v // 2, top_p=0.9, min_p=0.01), dict(min_p=0.3), dict(temperature=0.0)):
        t = {k: torch.full((6,), z, device="cuda", dtype=torch.int32 if k == "top_k" else F32) for k, z in kw.items()}
        got, same = ec.ec_sample(x, v, ut, **t), ec.ec_sample(plain, v, ut, **t)
        assert all(torch.equal(got[k], same[k]) for k in got), kw
        assert got["token"].tolist()[1:] == [-1, 0, 5, 9, -1] and got["kept"].tolist()[1:] == [0, 1, 1, 1, 0], kw
        assert got["prob"].tolist()[1:] == [0, 1, 1, 1, 0] and got["token"][0].item() % 3 != 0, kw
