"""GPU: the delta rule's calls as programs make them: on other streams, captured and replayed, at offsets past 32 bits, with
refused arguments, and next to the library's other calls."""
import pytest
import torch

from paper_2603_14360_b200 import binding as m

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def inputs(seed, B=2, T=150, N=4, K=64, V=32, dtype=BF):
    g = torch.Generator("cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    return [r(B, T, N, K), r(B, T, N, K), r(B, T, N, V), r(B, T, N), r(B, T, N)], r(B, T, N, V)


OPT = dict(gate_kind=m.GATE_LOGIT, step_kind=m.STEP_LOGIT, qk_norm=True)


def train(x, dy, **kw):
    y, hT, ckpt = m.m2rnn_delta_fwd(*x, save_ckpt=True, **OPT, **kw)
    g = m.m2rnn_delta_bwd(*x, None, dy, ckpt=ckpt, **OPT, **kw)
    return [y, hT, *g.values()]


@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=["bf16", "f32"])
def test_given_stream(dtype):
    x, dy = inputs(1, dtype=dtype)
    want = train(x, dy)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(5):      # workspaces of one call must not be another's before it is done
        got.append(train(x, dy, stream=side))
        torch.full((1 << 22,), 7.0, device="cuda")
    side.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(want, g))
    with torch.cuda.stream(side):
        assert all(torch.equal(a, b) for a, b in zip(want, train(x, dy)))


@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=["bf16", "f32"])
def test_two_streams_at_once(dtype):
    x1, dy1 = inputs(2, dtype=dtype)
    x2, dy2 = inputs(3, T=97, dtype=dtype)
    want = train(x1, dy1), train(x2, dy2)
    torch.cuda.synchronize()
    s1, s2, got = torch.cuda.Stream(), torch.cuda.Stream(), []
    for _ in range(4):
        with torch.cuda.stream(s1):
            a = train(x1, dy1)
        with torch.cuda.stream(s2):
            b = train(x2, dy2)
        got.append((a, b))
    torch.cuda.synchronize()
    for pair in got:
        for w, g in zip(want, pair):
            assert all(torch.equal(p, q) for p, q in zip(w, g))


@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=["bf16", "f32"])
def test_captured_and_replayed(dtype):
    x, dy = inputs(4, dtype=dtype)
    fresh, dy2 = inputs(5, dtype=dtype)
    want = train(fresh, dy2)
    m.device_status_word()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = train(x, dy)
    other = torch.cuda.CUDAGraph()      # a second graph with a workspace of its own
    with torch.cuda.graph(other):
        out2 = train(fresh, dy2)
    for a, b in zip([*x, dy], [*fresh, dy2]):
        a.copy_(b)
    graph.replay()
    other.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, out)) and all(torch.equal(a, b) for a, b in zip(want, out2))


def test_step_captured():
    x, _ = inputs(6, T=3)
    pool, slots = torch.randn(5, 4, 64, 32, device="cuda"), torch.tensor([3, 0], dtype=torch.int32, device="cuda")
    was = pool.clone()
    one = [t[:, 0].contiguous() for t in x]
    m.device_status_word()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = m.m2rnn_delta_decode_step(*one, pool, slots=slots, **OPT)
    want = []
    for t in range(3):
        for a, b in zip(one, x):
            a.copy_(b[:, t])
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        want.append((m.m2rnn_delta_decode_step(*(b[:, t].contiguous() for b in x), was, slots=slots, **OPT), got))
    assert all(torch.equal(a, b) for a, b in want) and torch.equal(was, pool)


def test_offsets_past_32_bits():
    """More than 2^31 entries to a tensor: what follows a dropped state is what a short call on it makes."""
    T, N, D, tail = 140_032, 128, 128, 96
    q = torch.randn(1, T, N, D, device="cuda", dtype=BF)
    assert q.numel() > 1 << 31
    gate = torch.full((1, T, N), -0.05, device="cuda", dtype=BF)
    gate[:, T - tail] = float("-inf")
    step = torch.full((1, T, N), 0.5, device="cuda", dtype=BF)
    o = dict(qk_norm=True, state_dtype=BF)
    y, hT, _ = m.m2rnn_delta_fwd(q, q, q, gate, step, **o)
    ys, hs, _ = m.m2rnn_delta_fwd(*(t[:, T - tail:].contiguous() for t in (q, q, q, gate, step)), **o)
    assert torch.equal(y[:, T - tail:], ys) and torch.equal(hT, hs)
    del y, q
    pool = torch.zeros(2200, 64, 128, 128, device="cuda", dtype=BF)      # a cache past 32 bits
    assert pool.numel() > 1 << 31
    pool[2199] = 1
    one = [torch.ones(1, 64, 128, device="cuda", dtype=BF) for _ in range(3)]
    g, s = torch.zeros(1, 64, device="cuda", dtype=BF), torch.zeros(1, 64, device="cuda", dtype=BF)
    yy = m.m2rnn_delta_decode_step(*one, g, s, pool, slots=torch.tensor([2199], dtype=torch.int32, device="cuda"))
    assert (yy == 128).all() and (pool[2199] == 1).all() and (pool[0] == 0).all()


def test_rows_behind_a_packed_batch_are_left_alone():
    x, dy = inputs(7, B=1, T=100)
    x, dy = [t[0] for t in x], dy[0]
    cu = torch.tensor([0, 30, 77, 90], dtype=torch.int32, device="cuda")      # ten tokens belong to no sequence
    mark = lambda like: torch.full_like(like, 3.0)  # noqa: E731
    out = dict(y=mark(x[2]))
    more = dict(cu_seqlens=cu, max_seqlen=47, **OPT)
    y, _, ckpt = m.m2rnn_delta_fwd(*x, save_ckpt=True, out=out, **more)
    g = dict(dq=mark(x[0]), dk=mark(x[1]), dv=mark(x[2]), dgate=mark(x[3]), dstep=mark(x[4]))
    m.m2rnn_delta_bwd(*x, None, dy, ckpt=ckpt, out=g, **more)
    for t in (y, *g.values()):
        assert (t[90:] == 3).all() and not (t[:90] == 3).all()


@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B", [1, 3])
def test_one_token_each_as_slices_of_a_projection(dtype, B):
    """An axis of one entry may have any stride: what a program's own operations leave there is not looked at."""
    x, dy = inputs(10, B=B, T=1, dtype=dtype)
    want = train(x, dy)
    wide = torch.cat([t.flatten(2) for t in x[:3]] + [torch.zeros(B, 1, 8, device="cuda", dtype=dtype)], 2)
    W = wide.shape[2]
    sizes = [t[0].numel() for t in x[:3]]
    for token in (W, 1, 7, sizes[0]):
        odd, at = [], 0
        for t, n in zip(x[:3], sizes):
            odd.append(torch.as_strided(wide, t.shape, (W, token, t.shape[3], 1), at))
            at += n
        assert all(torch.equal(a, b) for a, b in zip(odd, x))
        assert all(torch.equal(a, b) for a, b in zip(train(odd + x[3:], dy), want)), token
    one_head = [t[:, :, :1] for t in x[:2]] + x[2:]      # a single q and k head, sliced out of four
    dense = [t.contiguous() for t in one_head]
    assert all(torch.equal(a, b) for a, b in zip(train(one_head, dy), train(dense, dy)))


def test_first_call_captured():
    """In a process of its own: the status word that the first call makes is not the graph's."""
    import subprocess
    import sys
    code = """
import torch
from paper_2603_14360_b200 import binding as m
x = [torch.randn(2, 70, 2, 32, device="cuda").bfloat16() for _ in range(3)] + [-torch.rand(2, 70, 2, device="cuda").bfloat16() for _ in range(2)]
g = torch.cuda.CUDAGraph()
side = torch.cuda.Stream()
side.wait_stream(torch.cuda.current_stream())
with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
    y = m.m2rnn_delta_fwd(*x)[0]
assert m.device_status_word().item() == 0
for _ in range(2):
    m.device_status_word().fill_(5)
    g.replay()
    torch.cuda.synchronize()
    assert m.device_status_word().item() == 5
m.device_status_word().zero_()
assert torch.equal(y, m.m2rnn_delta_fwd(*x)[0]) and torch.isfinite(y).all()
print("fine")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr


def test_refusals():
    x, dy = inputs(8)
    q, k, v, gate, step = x
    for bad in ((q[:, :, :, :24], k, v, gate, step), (q, k, v, gate.float(), step), (q, k.float(), v, gate, step), (q, k, v, gate[:, :10], step),
                (q, k, v, gate.transpose(1, 2).contiguous().transpose(1, 2), step), (q.transpose(1, 2).contiguous().transpose(1, 2), k, v, gate, step),
                (q.cpu(), k, v, gate, step)):
        with pytest.raises((ValueError, TypeError)):
            m.m2rnn_delta_fwd(*bad, **OPT)
    for which in range(3):                                               # one token's memory for all: no layout of the calls
        same = list(x)
        same[which] = x[which][:1, :1].expand(2, 150, -1, -1)
        with pytest.raises(ValueError):
            m.m2rnn_delta_fwd(*same, **OPT)
    flat, cu = [t.flatten(0, 1) for t in x], torch.tensor([0, 150, 300], dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        m.m2rnn_delta_fwd(*flat, cu_seqlens=cu, max_seqlen=(1 << 32) + 5, **OPT)
    with pytest.raises(m.M2RNNError):
        m.m2rnn_delta_fwd(*x, gate_kind=m.GATE_VALUE)
    with pytest.raises(m.M2RNNError):
        m.m2rnn_delta_fwd(*x, gate_kind=m.GATE_PSI)                      # without alpha and beta
    with pytest.raises(TypeError):
        m.m2rnn_delta_fwd(*x, torch.zeros(2, 4, 64, 32, device="cuda", dtype=torch.float16), **OPT)
    with pytest.raises(TypeError):                                       # h0 and hT of two types
        m.m2rnn_delta_fwd(*x, torch.zeros(2, 4, 64, 32, device="cuda"), out=dict(hT=torch.zeros(2, 4, 64, 32, device="cuda", dtype=BF)), **OPT)
    with pytest.raises(ValueError):
        m.m2rnn_delta_bwd(*x, None, dy, ckpt=torch.zeros(100, device="cuda", dtype=torch.uint8), **OPT)
    with pytest.raises(m.M2RNNError):
        m.m2rnn_delta_fwd(*x, workspace=torch.zeros(16, device="cuda", dtype=torch.uint8), **OPT)
    one = [t[:, 0].contiguous() for t in x]
    with pytest.raises(ValueError):
        m.m2rnn_delta_decode_step(*one, torch.zeros(3, 4, 64, 32, device="cuda"), **OPT)      # three states, two rows, no slots
    with pytest.raises(TypeError):
        m.m2rnn_delta_decode_step(*one, torch.zeros(3, 4, 64, 32, device="cuda"), slots=torch.zeros(2, dtype=torch.int64, device="cuda"), **OPT)
    pool, i = torch.zeros(8, 32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (dict(dst=pool, dst_slots=i, src_slots=i[:1]), dict(dst=pool.t(), dst_slots=i, src_slots=i), dict(dst=pool, dst_slots=i.long(), src_slots=i.long()),
                dict(dst=pool, dst_slots=i, src_slots=i, axis=2), dict(dst=pool, dst_slots=i, src_slots=i, src=pool.half()),
                dict(dst=pool[:, :3].contiguous(), dst_slots=i, src_slots=i), dict(dst=pool[:7], dst_slots=i, src_slots=i, src=pool[1:])):
        with pytest.raises((ValueError, TypeError)):
            m.m2rnn_state_copy(**bad)


def test_a_layer_around_it():
    """conv + SiLU on the fused projection, the delta rule on its slices, the gated norm: a layer's path, prompt and then tokens."""
    B, T, N, K, V = 1, 45, 4, 32, 32
    torch.manual_seed(9)
    C = 3 * N * K
    x, w = torch.randn(B, T, C, device="cuda"), torch.randn(C, 4, device="cuda") * 0.5
    gate, step, gn, nw = (torch.randn(B, T, N, device="cuda") for _ in range(2)), None, torch.randn(B, T, N, V, device="cuda"), torch.rand(V, device="cuda") + 0.5
    gate, step = gate
    c = m.m2rnn_conv_silu_fwd(x, w)
    q, k, v = (c[..., i * N * K:(i + 1) * N * K].unflatten(-1, (N, K)) for i in range(3))
    y, hT, _ = m.m2rnn_delta_fwd(q, k, v, gate, step, **OPT)
    # a head's RMS norm: rows of V features
    out, _ = m.m2rnn_gated_norm_fwd(y.reshape(B, T * N, 1, V), gn.reshape(B, T * N, 1, V), nw, eps=1e-6)
    state = torch.zeros(B, N, K, V, device="cuda")
    for t in range(T):
        ct = m.m2rnn_conv_silu_fwd(x[:, t:t + 1].contiguous(), w, prev=torch.nn.functional.pad(x, (0, 0, 3, 0))[:, t:t + 3].contiguous())
        qt, kt, vt = (ct[:, 0, i * N * K:(i + 1) * N * K].unflatten(-1, (N, K)).contiguous() for i in range(3))
        yt = m.m2rnn_delta_decode_step(qt, kt, vt, gate[:, t].contiguous(), step[:, t].contiguous(), state, **OPT)
        ot, _ = m.m2rnn_gated_norm_fwd(yt.reshape(B, N, 1, V), gn[:, t].reshape(B, N, 1, V).contiguous(), nw, eps=1e-6)
        assert (ot.reshape(N, V) - out.reshape(B, T, N, V)[0, t]).abs().max() <= 1e-4 * out.abs().max()
    assert (state - hT).abs().max() <= 1e-4 * hT.abs().max()
