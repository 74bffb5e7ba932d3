"""ec_sample: which tokens a small min_p keeps is decided in 64 bits, not in the units that weights are summed in."""
import numpy as np
import pytest
import torch

import _serving as ref

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("v", [548, 4672, 33000, 131072, 400000])
def test_counts_at_small_min_p(v, dtype):
    """Logits all over the range that weighs anything: some tokens stand within every percent of every bound."""
    import paper_2603_18489_b200 as ec

    g = torch.Generator().manual_seed(v)
    x = torch.rand(4, v, generator=g) * torch.tensor([[-34.0], [-60.0], [-20.0], [-34.0]])
    x[3] = torch.round(x[3] * 50) / 50                     # ties
    host = x.to(dtype).float().numpy()
    x = torch.nn.functional.pad(x, (0, -v % 8)).to(dtype).cuda()   # rows are 16-byte aligned
    u = np.float32([0.1, 0.5, 0.7, 0.99])
    for m in (1e-25, 1e-14, 1e-13, 1.0000001e-12, 3e-11, 1e-9, 1e-6, 1e-3, 0.5, 1.0):
        m = float(np.float32(m))
        for t in (0.25, 1.0, 3.0):
            for k in (0, 200, v // 3):
                cols = dict(temperature=torch.full((4,), t), min_p=torch.full((4,), m), top_k=torch.full((4,), k, dtype=torch.int32))
                got = ec.ec_sample(x, v, torch.as_tensor(u).cuda(), **{n: c.cuda() for n, c in cols.items()})
                for i in range(4):
                    want = ref.sample(host[i], float(u[i]), t, k, 1.0, m)
                    have = (int(got["token"][i]), float(got["prob"][i]), int(got["kept"][i]))
                    assert have[0] == want[0] and have[2] == want[2], (i, m, t, k, have, want)
                    assert abs(have[1] - want[1]) <= want[1] * (2.0 ** -24 + 2.0 ** -25), (i, m, t, k, have, want)
