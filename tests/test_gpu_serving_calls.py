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
