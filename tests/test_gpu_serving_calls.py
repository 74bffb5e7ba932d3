"""Calls of the serving entry points that the binding has to sort out before it launches anything."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def ints(*v):
    return torch.tensor(v, dtype=I32, device="cuda")


@pytest.mark.parametrize("workspace", [16, "workspace", b"0123456789abcdef", [1, 2], object()])
def test_a_workspace_that_is_no_tensor_is_refused(workspace):
    import paper_2603_18489_b200 as ec

    logits = torch.zeros(2, 64, device="cuda")
    out = dict(token_out=ints(7, 7), prob_out=torch.zeros(2, device="cuda"), kept_out=ints(7, 7))
    state, one = ec.new_pages(2, 4, 16), ints(0)
    lists = ints(*[5] * 8), ints(*[5] * 8)
    q = torch.zeros(3, 4, 64, device="cuda")
    pool = torch.zeros(16, 2, 16, 64, device="cuda")
    desc = ec.make_paged_desc(2, 4, 2, 64, F32, 16, 16, 4)
    calls = [lambda: ec.ec_sample(logits, 64, torch.zeros(2, device="cuda"), workspace=workspace, **out),
             lambda: ec.ec_pages_reserve(*state, ints(0, 0), ints(3, 3), 16, *lists, one, workspace=workspace),
             lambda: ec.ec_pages_compact(*state, 16, *lists, one, workspace=workspace),
             lambda: ec.ec_attend_paged(desc, q, ints(0, 1, 3), ints(1, 2), 2, torch.zeros(2, 4, dtype=I32, device="cuda"), pool, pool,
                                        workspace=workspace)]
    for call in calls:
        with pytest.raises(TypeError, match="workspace must be a torch.Tensor"):
            call()
    torch.cuda.synchronize()
    assert out["token_out"].tolist() == [7, 7] and lists[0].tolist() == [5] * 8 and state[1].tolist() == [0, 0]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lead", [(2, 12), (1, 24), (24, 1), (2, 3, 4), (1, 1, 1), (0, 5)])
def test_rotation_of_slices_with_several_leading_dimensions(dtype, lead):
    """q, k and v of [batch, sequence, packed columns] as they come out of a projection: the same as dense copies."""
    import paper_2603_18489_b200 as ec

    hq, hkv, d, ps = 4, 2, 64, 16
    n = int(torch.tensor(lead).prod())
    packed = torch.randn(*lead, (hq + 2 * hkv) * d + 16, device="cuda").to(dtype)
    q, k, v = (packed[..., o * d:(o + h) * d].unflatten(-1, (h, d)) for o, h in ((0, hq), (hq, hkv), (hq + hkv, hkv)))
    pos = torch.arange(n, dtype=I32, device="cuda").view(lead)
    freq = torch.rand(d // 2, device="cuda")
    desc = ec.make_rope_desc(hq, hkv, d, dtype, d)
    got = ec.ec_qk_norm_rope(desc, q, k, pos, freq)
    flat = [x.reshape(n, x.shape[-2], d).contiguous() for x in (q, k, v)]
    want = ec.ec_qk_norm_rope(desc, *flat[:2], pos.view(n), freq)
    assert got[0].shape == q.shape and got[1].shape == k.shape
    assert all(torch.equal(g.view(w.shape), w) for g, w in zip(got, want))
    paged = ec.make_paged_desc(1, hq, hkv, d, dtype, ps, 3, 2)
    args = ints(0, n), pos.view(n), freq, ints(2, 0)
    pools = [torch.zeros(3, hkv, ps, d, dtype=dtype, device="cuda") for _ in range(4)]
    a = ec.ec_qk_norm_rope_paged(desc, paged, q, k, v, *args, *pools[:2])
    b = ec.ec_qk_norm_rope_paged(desc, paged, *flat, *args, *pools[2:])
    assert torch.equal(a.view(b.shape), b) and torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])
    assert n == 0 or (pools[1] != 0).any()


def test_rotation_refuses_rows_at_no_single_stride():
    import paper_2603_18489_b200 as ec

    desc = ec.make_rope_desc(4, 2, 64, F32, 64)
    pos, freq = torch.zeros(24, dtype=I32, device="cuda"), torch.rand(32, device="cuda")
    q, k = torch.randn(2, 12, 4, 64, device="cuda"), torch.randn(2, 12, 2, 64, device="cuda")
    bad = [q.transpose(0, 1), torch.randn(2, 20, 4, 64, device="cuda")[:, :12], torch.randn(1, 12, 4, 64, device="cuda").expand(2, 12, 4, 64)]
    for x in bad:
        with pytest.raises(ValueError, match="the rows of q must be one stride apart"):
            ec.ec_qk_norm_rope(desc, x, k, pos, freq)
    with pytest.raises(ValueError, match="heads of a row of q must be contiguous"):
        ec.ec_qk_norm_rope(desc, torch.randn(2, 12, 64, 4, device="cuda").transpose(2, 3), k, pos, freq)
    with pytest.raises(ec.EcError):                     # one row for all: the library takes no rows that overlap
        ec.ec_qk_norm_rope(desc, torch.randn(1, 4, 64, device="cuda").expand(24, 4, 64), k.view(24, 2, 64), pos, freq)
