"""GPU parity: ec_attend_paged against the 64-bit form."""
import numpy as np
import pytest
import torch

import _serving as ref

pytestmark = pytest.mark.gpu


def setup(dtype, lens, rows, hq, hkv, d, ps, seed=0, spare=3, garbage=True, pad_rows=0, scale_q=1.0, room=0):
    """Random pages in a random order; everything that no position of a sequence uses is NaN."""
    g = torch.Generator().manual_seed(seed)
    b = len(lens)
    per = [-(-n // ps) for n in lens]
    n_pages, max_pages = sum(per) + spare, max(max(max(per), 1) + 1, -(-room // ps))   # room: positions of the table
    ids = torch.randperm(n_pages, generator=g)
    table = torch.full((b, max_pages), -1, dtype=torch.int32)
    k, v = (torch.full((n_pages, hkv, ps, d), float("nan") if garbage else 0.0) for _ in range(2))
    at = 0
    for i, n in enumerate(per):
        table[i, :n] = ids[at:at + n].to(torch.int32)
        at += n
        for e in range(n):
            m = min(ps, lens[i] - e * ps)
            k[table[i, e], :, :m], v[table[i, e], :, :m] = torch.randn(2, hkv, m, d, generator=g)
    offsets = torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32)
    q = torch.randn(sum(rows) + pad_rows, hq, d, generator=g) * scale_q
    return dict(q=q.to(dtype).cuda(), k=k.to(dtype).cuda(), v=v.to(dtype).cuda(), table=table.cuda(), offsets=offsets.cuda(),
                lens=torch.tensor(lens, dtype=torch.int32).cuda(), n_pages=n_pages, max_pages=max_pages)


def f64(t):
    return t.detach().cpu().double().numpy()


def check(s, got, lens, rows, ps, mask, d, bf16, scale=None):
    q, k, v, table = f64(s["q"]), f64(s["k"]), f64(s["v"]), s["table"].cpu().numpy()
    out = f64(got)
    at = 0
    for b, (n, kv) in enumerate(zip(rows, lens)):
        want, mass, size = ref.attend(q[at:at + n], ref.gather(k, table[b], kv, ps), ref.gather(v, table[b], kv, ps),
                                      ref.visible(n, kv, mask), scale or d ** -0.5)
        tol = ref.attend_tolerance(want, mass, size, d, kv, bf16)
        err = np.abs(out[at:at + n] - want)
        assert (err <= tol).all(), (b, n, kv, float((err - tol).max()), np.unravel_index((err - tol).argmax(), err.shape))
        at += n


def run(dtype, lens, rows, hq, hkv, d, ps, mask, kernel=None, **kw):
    import paper_2603_18489_b200 as ec

    s = setup(dtype, lens, rows, hq, hkv, d, ps, **kw)
    desc = ec.make_paged_desc(len(lens), hq, hkv, d, dtype, ps, s["n_pages"], s["max_pages"], mask_block=mask)
    if kernel:
        assert ec.ec_attend_paged_kernel_name(desc, max(rows)) == kernel
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full_like(s["q"], 7.0)
    ec.ec_attend_paged(desc, s["q"], s["offsets"], s["lens"], max(max(rows), 1), s["table"], s["k"], s["v"], out=out,
                       dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    check(s, out, lens, rows, ps, mask, d, dtype == torch.bfloat16)
    assert (out[sum(rows):] == 7.0).all(), "rows behind the last sequence"
    return s, out


BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mask", [0, 1, 5])
def test_ragged_chunks(dtype, d, mask):
    run(dtype, [1, 70, 257, 0, 33, 128], [1, 5, 40, 3, 33, 2], 6, 2, d, 16, mask, pad_rows=4)


@pytest.mark.parametrize("ps", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_page_sizes_and_ends_inside_a_tile(dtype, ps):
    run(dtype, [ps - 1, ps, ps + 1, 3 * ps + 7, 200], [1, 1, 2, 7, 19], 4, 4, 64, ps, 1)


@pytest.mark.parametrize("dtype,hq,hkv,d", [(BF, 28, 4, 128), (BF, 8, 8, 64), (BF, 33, 1, 128), (F32, 12, 3, 64), (BF, 128, 1, 64)])
def test_single_tokens(dtype, hq, hkv, d):
    run(dtype, [1, 2, 15, 16, 17, 63, 64, 65, 500, 1023], [1] * 10, hq, hkv, d, 16, 1)


@pytest.mark.parametrize("dtype,kv,rows", [(BF, 5000, 1), (BF, 3001, 34), (F32, 2000, 3), (BF, 1500, 300)])
def test_one_sequence_split_over_the_gpu(dtype, kv, rows):
    run(dtype, [kv], [rows], 4, 2, 128, 32, 0)


@pytest.mark.parametrize("mask", [0, 1, 32])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (3, 3, 64), (14, 2, 128), (5, 1, 128)])
def test_chunked_prefill(mask, hq, hkv, d):
    run(BF, [700, 129, 512, 300], [300, 129, 256, 1], hq, hkv, d, 64, mask, pad_rows=130)


def test_rows_in_front_of_the_sequence_see_nothing():
    s, out = run(BF, [3, 5], [10, 5], 4, 2, 64, 16, 1)
    assert (out[:7] == 0).all()
    s, out = run(BF, [0, 0, 40], [2, 0, 3], 4, 2, 128, 16, 0)
    assert (out[:2] == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 40, 150])
def test_scores_of_every_size(dtype, rows):
    """Scores of a hundred and more: one key rules a row, and the maximum moves along the keys."""
    run(dtype, [600], [rows], 4, 2, 64, 16, 1, scale_q=30.0)
    run(dtype, [600], [rows], 4, 2, 128, 16, 0, scale_q=8.0)


def test_scale_and_many_empty_sequences():
    import paper_2603_18489_b200 as ec

    lens, rows = [0] * 40 + [90] + [0] * 20 + [17], [0] * 40 + [4] + [0] * 20 + [1]
    s = setup(BF, lens, rows, 4, 2, 64, 16)
    desc = ec.make_paged_desc(len(lens), 4, 2, 64, BF, 16, s["n_pages"], s["max_pages"], mask_block=1, scale=0.3)
    out = ec.ec_attend_paged(desc, s["q"], s["offsets"], s["lens"], 4, s["table"], s["k"], s["v"])
    check(s, out, lens, rows, 16, 1, 64, True, scale=0.3)


@pytest.mark.parametrize("rows", [2, 200])
def test_what_the_device_refuses(rows):
    import paper_2603_18489_b200 as ec

    lens = [300, 280]
    s = setup(BF, lens, [rows, rows], 4, 2, 128, 16)
    desc = ec.make_paged_desc(2, 4, 2, 128, BF, 16, s["n_pages"], s["max_pages"], mask_block=1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call(table, kv, max_rows):
        status.zero_()
        out = torch.full_like(s["q"], 7.0)
        ec.ec_attend_paged(desc, s["q"], s["offsets"], kv, max_rows, table, s["k"], s["v"], out=out, dev_status=status)
        return int(status), out

    good = call(s["table"], s["lens"], rows)
    assert good[0] == 0
    for bad in (-1, s["n_pages"], 2 ** 31 - 1, -2 ** 31):
        table = s["table"].clone()
        table[1, 3] = bad
        code, out = call(table, s["lens"], rows)
        assert code == 9
        assert torch.equal(out[:rows], good[1][:rows])   # the other sequence
    assert call(s["table"], torch.tensor([300, 10 ** 6], dtype=torch.int32, device="cuda"), rows)[0] in (2, 9)
    assert call(s["table"], torch.tensor([300, -5], dtype=torch.int32, device="cuda"), rows)[0] == 2
    code, out = call(s["table"], s["lens"], rows - 1)
    assert code == 2 and (out[rows - 1] == 7.0).all()


def test_deterministic_and_captured():
    """The same bits from every call, from a replayed graph with other lengths too, with one workspace in use again and again."""
    import paper_2603_18489_b200 as ec

    for rows in (1, 60):
        lens = [900, 300, 77]
        s = setup(BF, lens, [rows] * 3, 8, 2, 128, 32, garbage=False)
        desc = ec.make_paged_desc(3, 8, 2, 128, BF, 32, s["n_pages"], s["max_pages"], mask_block=1)
        ws = ec.new_workspace(ec.ec_attend_paged_workspace_bytes(desc, rows))
        ws.fill_(0xff)
        out = torch.empty_like(s["q"])

        def call():
            return ec.ec_attend_paged(desc, s["q"], s["offsets"], s["lens"], rows, s["table"], s["k"], s["v"], out=out, workspace=ws)

        first = call().clone()
        check(s, first, lens, [rows] * 3, 32, 1, 128, True)
        for _ in range(5):
            assert torch.equal(call(), first)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)
        lens = [100, 299, 64]
        s["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        check(s, out, lens, [rows] * 3, 32, 1, 128, True)


def test_two_streams_with_workspaces_of_their_own():
    import paper_2603_18489_b200 as ec

    lens = [2000, 1500]
    s = setup(BF, lens, [1, 1], 8, 2, 128, 16)
    desc = ec.make_paged_desc(2, 8, 2, 128, BF, 16, s["n_pages"], s["max_pages"], mask_block=1)
    args = (desc, s["q"], s["offsets"], s["lens"], 1, s["table"], s["k"], s["v"])
    want = ec.ec_attend_paged(*args)
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [ec.new_workspace(ec.ec_attend_paged_workspace_bytes(desc, 1)) for _ in range(2)]
    outs = [torch.empty_like(s["q"]) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            ec.ec_attend_paged(*args, out=outs[i], workspace=ws[i], stream=streams[i])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


@pytest.mark.parametrize("rows", [1, 200])
def test_a_pool_beyond_32_bit_offsets(rows):
    """Pages whose offset in elements passes 2^32."""
    import paper_2603_18489_b200 as ec

    hkv, ps, d = 2, 128, 128
    n_pages = 2 ** 32 // (hkv * ps * d) + 40
    k, v = (torch.zeros(n_pages, hkv, ps, d, dtype=BF, device="cuda") for _ in range(2))
    ids = [n_pages - 1, 5, n_pages - 17, n_pages // 2 + 3]
    s = setup(BF, [450], [rows], 4, hkv, d, ps, spare=0)
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    for e, p in enumerate(ids):
        k[p], v[p] = s["k"][s["table"][0, e]], s["v"][s["table"][0, e]]
    desc = ec.make_paged_desc(1, 4, hkv, d, BF, ps, n_pages, 4, mask_block=1)
    out = ec.ec_attend_paged(desc, s["q"], s["offsets"], s["lens"], rows, table, k, v)
    check(s, out, [450], [rows], ps, 1, d, True)


TILES, ROWS = "attend_paged_tiles_kernel", "attend_paged_rows_kernel"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mask", [0, 1, 5, 32])
@pytest.mark.parametrize("ps", [16, 32, 64, 128])
def test_tiles_kernel(d, mask, ps):
    """One and two row tiles, one key tile and many, empty sequences, ends inside a page and a tile; room that the lengths do not use."""
    lens, rows = [1, 70, 257, 0, 640, 385, 128, 900], [1, 33, 257, 2, 100, 60, 128, 17]
    run(BF, lens, rows, 6, 2, d, ps, mask, kernel=TILES, pad_rows=5, room=65536)


@pytest.mark.parametrize("d", [64, 128])
def test_tiles_kernel_second_pass(d):
    """Scores that leave the first pass's range: the unit is done again with running maxima, for one row tile and for two."""
    for mask in (0, 1):
        run(BF, [700, 300], [40, 200], 4, 2, d, 32, mask, kernel=TILES, scale_q=60.0, room=65536)


@pytest.mark.parametrize("hq,hkv,rows,kv", [(7, 1, 3, 4000), (1, 1, 200, 3000), (64, 2, 40, 700), (128, 1, 9, 300), (9, 9, 18, 2000)])
def test_tiles_kernel_cuts_and_groups(hq, hkv, rows, kv):
    run(BF, [kv, kv // 2 + 1], [rows, 1], hq, hkv, 128, 16, 1, kernel=TILES, room=1 << 18)


@pytest.mark.parametrize("rows", [9, 16, 3])
def test_rows_kernel_whole_and_cut(rows):
    for room, lens in ((0, [500, 77, 1]), (8000, [2500, 77, 1])):
        run(BF, lens, [min(rows, n) for n in lens], 1, 1, 128, 16, 1, kernel=ROWS, room=room)
        run(BF, lens, [min(rows, n) for n in lens], 2, 2, 64, 32, 0, kernel=ROWS, room=room)


@pytest.mark.parametrize("seed", range(12))
def test_random_batches(seed):
    g = np.random.default_rng(seed)
    hkv = int(g.choice([1, 2, 3]))
    hq, d, ps = hkv * int(g.choice([1, 2, 5, 8])), int(g.choice([64, 128])), int(g.choice([16, 32, 64, 128]))
    b = int(g.integers(1, 9))
    lens = [int(x) for x in g.integers(0, 1 + int(g.choice([40, 500, 1500])), b)]
    rows = [int(g.integers(0, min(n, int(g.choice([2, 40, 300]))) + 1)) for n in lens]
    if sum(rows) == 0:
        lens[0], rows[0] = 5, 1
    run(BF if seed % 4 else F32, lens, rows, hq, hkv, d, ps, int(g.choice([0, 1, 7, 32])), room=int(g.choice([0, 0, 40000])), pad_rows=int(g.integers(0, 3)))


def test_a_captured_call_serves_other_lengths_on_the_tiles_kernel():
    import paper_2603_18489_b200 as ec

    lens, rows = [2000, 1100, 300], [150, 40, 300]
    s = setup(BF, lens, rows, 8, 2, 128, 64, garbage=False, room=16384)
    desc = ec.make_paged_desc(3, 8, 2, 128, BF, 64, s["n_pages"], s["max_pages"], mask_block=1)
    assert ec.ec_attend_paged_kernel_name(desc, 300) == TILES
    ws = ec.new_workspace(ec.ec_attend_paged_workspace_bytes(desc, 300))
    out = torch.empty_like(s["q"])

    def call():
        ec.ec_attend_paged(desc, s["q"], s["offsets"], s["lens"], 300, s["table"], s["k"], s["v"], out=out, workspace=ws)

    call()
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)
    lens = [151, 1100, 300]
    s["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    check(s, out, lens, rows, 64, 1, 128, True)


@pytest.mark.parametrize("d,heads", [(64, 40), (128, 48)])
@pytest.mark.parametrize("mask", [0, 1])
def test_many_units_a_cta_some_of_them_done_twice(d, heads, mask):
    """Each CTA goes through several units of one and two row tiles, one key tile and more; in every other sequence the scores
    leave the first pass's range, so that units with and without a second pass follow one another."""
    import paper_2603_18489_b200 as ec

    lens, rows = [130, 20, 300, 257, 140, 1, 500, 129], [20, 20, 150, 257, 17, 1, 40, 129]
    s = setup(BF, lens, rows, heads, heads, d, 32, room=65536)
    at = 0
    for b, n in enumerate(rows):
        if b % 2 == 0:
            s["q"][at:at + n] *= 60
        at += n
    desc = ec.make_paged_desc(8, heads, heads, d, BF, 32, s["n_pages"], s["max_pages"], mask_block=mask)
    assert ec.ec_attend_paged_kernel_name(desc, max(rows)) == TILES
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = ec.ec_attend_paged(desc, s["q"], s["offsets"], s["lens"], max(rows), s["table"], s["k"], s["v"], dev_status=status)
    assert int(status) == 0
    check(s, out, lens, rows, 32, mask, d, True)


@pytest.mark.parametrize("dtype,room", [(BF, 0), (BF, 1 << 20), (F32, 0)])
def test_only_empty_sequences(dtype, room):
    import paper_2603_18489_b200 as ec

    s = setup(dtype, [40, 0, 7], [0, 0, 0], 40, 1, 64, 16, pad_rows=30, room=room)
    desc = ec.make_paged_desc(3, 40, 1, 64, dtype, 16, s["n_pages"], s["max_pages"], mask_block=1)
    out = torch.full_like(s["q"], 7.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ec.ec_attend_paged(desc, s["q"], s["offsets"], s["lens"], 30, s["table"], s["k"], s["v"], out=out, dev_status=status)
    assert (out == 7.0).all() and int(status) == 0


def test_the_largest_batch():
    g = np.random.default_rng(0)
    lens = [int(x) for x in g.integers(0, 40, 1024)]
    run(BF, lens, [min(n, 1 + i % 2) for i, n in enumerate(lens)], 2, 1, 64, 16, 1)
    run(BF, lens, [min(n, 1 + i % 19) for i, n in enumerate(lens)], 2, 1, 64, 16, 1, kernel=TILES, room=4096)


@pytest.mark.parametrize("rows", [1, 40])
def test_fewer_rows_than_the_offsets_say(rows):
    """Offsets beyond the rows of q: the rows that are there are computed, the rest is refused."""
    import paper_2603_18489_b200 as ec

    s = setup(BF, [100, 90], [rows, rows], 2, 2, 64, 16, room=1 << 18)
    desc = ec.make_paged_desc(2, 2, 2, 64, BF, 16, s["n_pages"], s["max_pages"], mask_block=0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = ec.ec_attend_paged(desc, s["q"], s["offsets"], s["lens"], rows, s["table"], s["k"], s["v"])
    out = ec.ec_attend_paged(desc, s["q"][:rows].contiguous(), s["offsets"], s["lens"], rows, s["table"], s["k"], s["v"], dev_status=status)
    assert int(status) == 2 and torch.equal(out, want[:rows])
