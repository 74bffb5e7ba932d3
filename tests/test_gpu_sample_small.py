"""ec_sample at temperatures at and below the end of fp32's normal range: those below 2^-126 count as 2^-126."""
import numpy as np
import pytest
import torch

import _serving as ref

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
LEAST = 2.0 ** -126


def rows(v, dtype):
    """Ordinary logits, ties for the first place, and rows whose logits differ by a few temperatures: by 1e-39 (below the normal range),
    by 1e-38 and by 1e-36, near 0 and near 1e-30 where that is a few last bits."""
    g = torch.Generator().manual_seed(v)
    x = torch.randn(7, v, generator=g, dtype=torch.float64) * 3
    x[1, ::5] = 9.0
    j = torch.randperm(v, generator=g).double()
    x[2], x[3], x[4] = -1.5e-39 * j, -2e-38 * (j % 50), -1e-36 * (j % 90)
    x[5] = 1e-30 + 1e-36 * (j % 7)
    x[6] = 0.0
    x[6, 3:] = -1e-37
    return x.to(dtype).cuda()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("v", [40, 2000, 20008])
@pytest.mark.parametrize("t", [1.4e-45, 1e-41, 1e-39, LEAST, 4e-38, 1.4e-37, 3e-36])
def test_small_temperatures(dtype, v, t):
    import paper_2603_18489_b200 as ec

    x = rows(v, dtype)
    host = x.float().cpu().numpy()
    n = x.shape[0]
    temp = torch.full((n,), t, dtype=F32, device="cuda")
    counts_as = max(float(temp[0]), LEAST)
    for u in (0.0, 0.37, 0.93):
        for kw in ({}, dict(top_p=0.8), dict(top_k=7), dict(top_k=v // 2, min_p=0.05), dict(min_p=1e-3, top_p=0.9)):
            cols = {k: torch.full((n,), z, dtype=torch.int32 if k == "top_k" else F32, device="cuda") for k, z in kw.items()}
            at = {k: float(c[0]) for k, c in cols.items()}
            got = ec.ec_sample(x, v, torch.full((n,), u, dtype=F32, device="cuda"), temp, **cols)
            for i in range(n):
                want = ref.sample(host[i], float(np.float32(u)), counts_as, **at)
                have = (int(got["token"][i]), float(got["prob"][i]), int(got["kept"][i]))
                assert have[0] == want[0] and have[2] == want[2], (i, u, kw, have, want)
                # one rounding to fp32; the weights' own 1e-13 and the units' 2^-42 of 1 stay below 2^-25
                assert abs(have[1] - want[1]) <= want[1] * (2.0 ** -24 + 2.0 ** -25), (i, u, kw, have, want)
