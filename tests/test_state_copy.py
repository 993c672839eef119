"""GPU: states moved between the slots of a cache, against indexing in one go on the CPU: equal, bit for bit."""
import pytest
import torch

from paper_2603_14360_b200 import binding as m

pytestmark = pytest.mark.gpu


def want(dst, to, src, frm, axis):
    out, read = dst.clone().movedim(axis, 0), src.movedim(axis, 0)
    for d, s in zip(to, frm):
        if d >= 0:
            out[d] = read[s] if s >= 0 else 0
    return out.movedim(0, axis)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.uint8])
@pytest.mark.parametrize("shape,axis", [((9, 2, 16, 16), 0), ((3, 9, 2, 16, 48), 1), ((40, 16), 0), ((2, 2, 300, 64), 2), ((700, 32), 0), ((5, 7, 33 * 16), 1)])
def test_moves(shape, axis, dtype):
    g = torch.Generator().manual_seed(sum(shape))
    pool = (torch.randn(*shape, generator=g) * 50).to(dtype)
    S = shape[axis]
    for n in {1, 2, S // 2, S - 1, S}:
        for kind in ("permutation", "fork", "shift", "mixed"):
            if kind == "permutation":
                to, frm = torch.randperm(S, generator=g)[:n].tolist(), torch.randperm(S, generator=g)[:n].tolist()
            elif kind == "fork":
                to, frm = torch.randperm(S, generator=g)[:n].tolist(), [S // 3] * n
            elif kind == "shift":
                to, frm = list(range(n)), [(i + 1) % S for i in range(n)]
            else:
                to = torch.randint(-2, S, (n,), generator=g).tolist()      # repeated destinations: the last counts
                frm = torch.randint(-2, S, (n,), generator=g).tolist()
            got = pool.cuda()
            back = m.m2rnn_state_copy(got, i32(to), i32(frm), axis=axis)
            assert back is got
            assert torch.equal(got.cpu(), want(pool, to, pool, frm, axis)), (n, kind)
    m.check_device_status()


def test_from_another_cache():
    src, dst = torch.randn(3, 5, 4, 64), torch.randn(3, 11, 4, 64)
    got, frm, to = dst.cuda(), [0, 4, 4, -1], [10, 0, 3, 7]
    m.m2rnn_state_copy(got, i32(to), i32(frm), src.cuda(), axis=1)
    assert torch.equal(got.cpu(), want(dst, to, src, frm, 1))


def test_slots_outside_are_reported_and_left_out():
    pool = torch.randn(4, 64)
    got = pool.cuda()
    m.m2rnn_state_copy(got, i32([0, 4, 1]), i32([3, 0, 4]))
    with pytest.raises(m.M2RNNError):
        m.check_device_status()
    assert torch.equal(got.cpu(), want(pool, [0], pool, [3], 0))


def test_as_many_pairs_as_a_call_takes():
    n = m._lib().m2rnn_state_copy_limit()
    pool = torch.randn(n + 3, 24)
    frm, to = torch.randperm(n + 3)[:n].tolist(), torch.randperm(n + 3)[:n].tolist()
    got = pool.cuda()
    m.m2rnn_state_copy(got, i32(to), i32(frm))
    assert torch.equal(got.cpu(), want(pool, to, pool, frm, 0))
    with pytest.raises(ValueError):
        m.m2rnn_state_copy(got, i32(to + [0]), i32(frm + [0]))


def test_large_cache_offsets():
    """Rows whose offsets pass 32 bits."""
    pool = torch.zeros(70, 1 << 26, dtype=torch.uint8, device="cuda")
    pool[69] = 7
    pool[1] = 3
    m.m2rnn_state_copy(pool, i32([68, 0, 67]), i32([69, 1, 68]))
    assert (pool[68] == 7).all() and (pool[0] == 3).all() and (pool[67] == 0).all() and (pool[69] == 7).all()


def test_captured_and_replayed():
    pool = torch.randn(6, 3, 32, device="cuda")
    was, to, frm = pool.clone(), i32([0, 1, 2]), i32([1, 2, 0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    m.device_status_word()
    with torch.cuda.graph(graph, stream=side):
        m.m2rnn_state_copy(pool, to, frm)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(pool, was[[2, 0, 1, 3, 4, 5]])
