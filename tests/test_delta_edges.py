"""GPU: the delta rule at inputs where its chunks' arithmetic can go wrong, against its definition in 64 bits."""
import math

import pytest
import torch

import delta_reference as ref
from paper_2603_14360_b200 import binding as m
from test_delta_rule import make, on_gpu, rel

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def forward_and_gradients(x, on, H0, dy, d_hT, o):
    """Errors of every output against 64 bits, as shares of its largest entry."""
    y_r, hT_r, g_r = ref.gradients([t.double() for t in x], H0.double(), dy.double(), d_hT.double(), **o)
    y, hT, ckpt = m.m2rnn_delta_fwd(*on, H0.cuda(), save_ckpt=True, **on_gpu(o))
    g = m.m2rnn_delta_bwd(*on, H0.cuda(), dy.cuda(), d_hT.cuda(), ckpt=ckpt, **on_gpu(o))
    m.check_device_status()
    return dict(y=rel(y, y_r), hT=rel(hT, hT_r), **{n: rel(g[n], torch.nan_to_num(g_r[n])) for n in g_r})


@pytest.mark.parametrize("drop", [-math.inf, -60.0], ids=["dropped", "strong"])
@pytest.mark.parametrize("every", [16, 5, 2])
def test_digits_behind_dropped_states(every, drop):
    """fp32 keeps its digits behind tokens that drop the state, many to a chunk, whose log decays stay in the chunk's running sums.

    Bound: between an input and an output stand four sums of 16 terms (K = V = 16, chunks of 16, and at most as many of them between two such
    tokens) and some 32 single operations, each off by 2^-24 of its value at most: (4 * 16 + 32) 2^-24 = 5.8e-6.  (A sum of 12 * 104 in
    fp32 alone is off by 6e-5.)"""
    x, on, H0, dy, d_hT, o = make(30 + every, B=2, T=70, N=2, K=16, V=16, dtype=F32, gate="log", step="value")
    for t in range(70):
        if (t % 16 < 12 if every == 16 else t % every == 1):
            x[3][:, t] = drop
    on = [t.cuda() for t in x]
    errs = forward_and_gradients(x, on, H0, dy, d_hT, o)
    assert max(errs.values()) <= 96 * 2.0 ** -24, errs


def packed_with_marks(cu, tokens, most, N, Nq, dtype, seed):
    """Forward and gradients of a packed batch into buffers full of 3, on workspaces full of NaN, and what was given."""
    x, on, _, dy, d_hT, o = make(seed, B=len(cu) - 1, T=0, N=N, K=32, V=32, Nq=Nq, Nk=Nq, dtype=dtype, cu=[0, tokens])
    H0 = torch.randn(len(cu) - 1, N, 32, 32, generator=torch.Generator().manual_seed(seed))
    more = dict(on_gpu(o), cu_seqlens=torch.tensor(cu, dtype=torch.int32).cuda(), max_seqlen=most, workspace=torch.full((1 << 26,), 0xFF, dtype=torch.uint8).cuda())
    mark = lambda like: torch.full_like(like, 3.0)  # noqa: E731
    d_hT = torch.randn(H0.shape, generator=torch.Generator().manual_seed(seed + 1))
    y, hT, ckpt = m.m2rnn_delta_fwd(*on, H0.cuda(), save_ckpt=True, out=dict(y=mark(on[2])), **more)
    g = dict(zip(("dq", "dk", "dv", "dgate", "dstep"), map(mark, on)))
    g = m.m2rnn_delta_bwd(*on, H0.cuda(), dy.cuda(), d_hT.cuda(), ckpt=ckpt, out=g, **more)
    m.check_device_status()
    return (x, H0, dy, d_hT, o), dict(y=y, **g), hT


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("Nq", [1, 2, 4])
@pytest.mark.parametrize("cu,tokens,most", [([0, 30, 77, 90], 100, 47), ([0, 30, 77, 90], 90, 40), ([0, 0, 33, 33], 70, 33)], ids=["behind", "cut", "empty"])
def test_rows_of_no_sequence_are_left_alone(cu, tokens, most, Nq, dtype):
    """With q and k shared too, where sums over the heads follow the gradient kernel."""
    given, out, _ = packed_with_marks(cu, tokens, most, 4, Nq, dtype, 40)
    rows = torch.zeros(tokens, dtype=torch.bool)
    for a, b in zip(cu, cu[1:]):
        rows[a:min(b, a + most)] = True
    for name, t in out.items():
        if name != "dh0":
            t = t.flatten(1).float().cpu()
            assert (t[~rows] == 3).all(), name
            assert torch.isfinite(t).all() and not (t[rows] == 3).all(1).any(), name


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("Nq", [1, 4])
@pytest.mark.parametrize("first", [1, 40, 150, 331])
def test_offsets_that_begin_behind_the_first_token(first, Nq, dtype):
    """A slice of a larger batch's offsets: those sequences' results, rows of others left alone.  Bounds as in test_delta_rule.
    (A batch of more tokens than its sequences can have, B times the longest, is refused.)"""
    cu = [first + c for c in (0, 30, 30, 101, 150)]
    if first + 170 > 4 * 80:
        with pytest.raises(m.M2RNNError):
            packed_with_marks(cu, first + 170, 80, 4, Nq, dtype, 41)
        return
    (x, H0, dy, d_hT, o), out, hT = packed_with_marks(cu, first + 170, 80, 4, Nq, dtype, 41)
    rows = slice(first, cu[-1])
    y_r, hT_r, g_r = ref.gradients([t[rows].double() for t in x], H0.double(), dy[rows].double(), d_hT.double(), [c - first for c in cu], **o)
    tol = 2e-2 if dtype == BF else 1e-4
    assert rel(hT, hT_r) <= tol and rel(out.pop("dh0"), g_r["dh0"]) <= tol
    for name, t in out.items():
        assert rel(t[rows], y_r if name == "y" else g_r[name]) <= tol, name
        assert (t[:first] == 3).all() and (t[cu[-1]:] == 3).all(), name


@pytest.mark.parametrize("state", [BF, F32], ids=["sbf16", "sf32"])
@pytest.mark.parametrize("packed", [False, True])
def test_calls_without_tokens_hand_the_states_on(packed, state):
    """Every sequence of a call is empty: its final states are the initial ones, as of a single empty sequence."""
    lead = (0,) if packed else (3, 0)
    q, gt = torch.zeros(*lead, 2, 32, dtype=BF, device="cuda"), torch.zeros(*lead, 2, dtype=BF, device="cuda")
    more = dict(cu_seqlens=torch.zeros(4, dtype=torch.int32, device="cuda"), max_seqlen=8) if packed else {}
    h0 = torch.randn(3, 2, 32, 32, device="cuda").to(state)
    hT = torch.full_like(h0, math.nan)
    assert m.m2rnn_delta_fwd(q, q, q, gt, gt, h0, out=dict(hT=hT), **more)[1] is hT and torch.equal(hT, h0)
    assert torch.equal(m.m2rnn_delta_fwd(q, q, q, gt, gt, h0, **more)[1], h0)
    assert torch.equal(m.m2rnn_delta_fwd(q, q, q, gt, gt, hT, out=dict(hT=hT), **more)[1], h0)      # in place
    hT.fill_(math.nan)
    m.m2rnn_delta_fwd(q, q, q, gt, gt, out=dict(hT=hT), **more)
    assert (hT == 0).all()
    g = m.m2rnn_delta_bwd(q, q, q, gt, gt, h0, q, hT + 2, **more)
    assert (g["dh0"] == 2).all() and g["dh0"].dtype == state


@pytest.mark.parametrize("most", [-(1 << 32) + 80, 1 << 31])
def test_lengths_that_32_bits_do_not_hold(most):
    """Not cut to what is left of them in 32 bits (80 of the second)."""
    q, gt = torch.zeros(80, 2, 32, dtype=BF, device="cuda"), torch.zeros(80, 2, dtype=BF, device="cuda")
    cu = torch.tensor([0, 80], dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="max_seqlen"):
        m.m2rnn_delta_fwd(q, q, q, gt, gt, cu_seqlens=cu, max_seqlen=most)
    with pytest.raises(ValueError, match="max_seqlen"):
        m.m2rnn_fwd(q, q, q, gt.float(), torch.zeros(2, 32, 32, dtype=BF, device="cuda"), cu_seqlens=cu, max_seqlen=most)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("step,decay", [(1.0, 0.0), (0.98, -0.002), (0.7, -0.01), (0.5, -0.05)])
@pytest.mark.parametrize("cosine", [0.97, 0.994, 0.999, 1.0])
def test_keys_that_are_nearly_the_same(cosine, step, decay, dtype):
    """A run of one token, or of tokens much alike: (I + M)^-1 = T has entries near -1 below its diagonal, and what it carries from token to
    token cancels.

    Bounds: those of test_delta_rule, twice.  With keys of cosine c, M's entries are c b times the decays, at most m = c b in [0, 1], so T's rows
    hold 1 and m (1 - m)^i, which sum to 2 at most: as much of the roundings of X (of dU in the gradient) comes through it, where keys that
    point anywhere leave T near I.  (With T itself rounded to bf16, all its entries off to the same side, dstep was 1e-1 off.)"""
    o = dict(q_scale=1.0, qk_norm=True, norm_eps=1e-6, gate_kind=m.GATE_LOG, step_kind=m.STEP_VALUE)
    gen = torch.Generator().manual_seed(50)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    T, N, K, V = 150, 2, 64, 64
    base, other = ref.unit(r(1, 1, N, K), 0), r(1, T, N, K)
    other = ref.unit(other - (other * base).sum(-1, keepdim=True) * base, 0)
    k = math.sqrt(cosine) * base + math.sqrt(1 - cosine) * other
    x = [t.to(dtype) for t in (r(1, T, N, K), k, r(1, T, N, V), torch.full((1, T, N), decay), torch.full((1, T, N), step))]
    H0, d_hT = r(1, N, K, V) * 0.2, r(1, N, K, V) * 0.2
    errs = forward_and_gradients(x, [t.cuda() for t in x], H0, r(1, T, N, V).to(dtype), d_hT, o)
    assert max(errs.values()) <= (4e-2 if dtype == BF else 2e-4), errs
