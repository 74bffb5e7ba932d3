"""ec_sample's results do not depend on how many CTAs share a row: vocabularies for which few rows have clusters of eight CTAs each and
many rows one CTA each."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
ROWS = 400      # one CTA a row; 100 of them still (with the row in shared memory); 1 and 3: clusters


def rows(v, dtype):
    g = torch.Generator().manual_seed(v)
    x = torch.randn(ROWS, v, generator=g) * (0.2 + 6 * torch.rand(ROWS, 1, generator=g))
    x[0] = 1.5                                                                  # equal logits
    x[1] = torch.where(torch.rand(v, generator=g) < 0.5, 1.0, 0.0)              # two values
    x[2] = torch.linspace(0, 1e-4, v)                                           # all but equal
    x[3] = float("-inf")
    x[4, 5:] = torch.finfo(dtype).min
    x[5] = torch.randint(0, 4, (v,), generator=g) * 0.01
    x[6, ::3] = float("nan")
    x[7] = torch.linspace(-60, 0, v)
    return x.to(dtype).cuda(), torch.rand(ROWS, generator=g).cuda()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("v", [8200, 12000, 16376])
def test_few_and_many_rows_give_the_same_bits(v, dtype):
    import paper_2603_18489_b200 as ec

    x, u = rows(v, dtype)
    g = np.random.default_rng(v)
    cols = [dict(), dict(top_p=np.full(ROWS, 0.9)), dict(top_k=g.integers(0, v, ROWS), min_p=g.uniform(0, 0.1, ROWS)),
            dict(temperature=g.uniform(0, 2, ROWS), top_k=g.integers(0, 300, ROWS), top_p=g.uniform(0.3, 1.1, ROWS))]
    for kw in cols:
        t = {k: torch.as_tensor(c, dtype=torch.int32 if k == "top_k" else F32).cuda() for k, c in kw.items()}
        many = ec.ec_sample(x, v, u, **t)
        for lo, n in ((0, 1), (0, 3), (1, 3), (2, 1), (4, 4), (5, 1), (6, 3), (7, 1), (200, 1), (300, 100), (399, 1)):
            part = slice(lo, lo + n)
            got = ec.ec_sample(x[part], v, u[part], **{k: c[part].contiguous() for k, c in t.items()})
            assert all(torch.equal(many[k][part], got[k]) for k in many), (kw.keys(), lo, n)
