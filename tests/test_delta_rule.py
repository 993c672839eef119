"""GPU: the gated delta rule -- forward, gradient, decoding step -- against its definition in 64 bits.

Bounds, per output tensor, on max |gpu - ref| / max |ref|.  bf16: an output passes at most five rounded operands in a row
(the state, T, X, U and itself), each off by 2^-8 of its value at most: 5/256 < 2e-2; the gradients pass two more, but
no entry takes the worst of all of its sums' terms.  fp32: 1e-4, the bound of the library's fp32 paths (sums of up to
128 terms, 2^-24 each, through chains of 16 rows: 2^-24 * 128 * 10)."""
import math

import pytest
import torch

import delta_reference as ref
from paper_2603_14360_b200 import binding as m

pytestmark = pytest.mark.gpu
TOL = {torch.bfloat16: 2e-2, torch.float32: 1e-4}
BF, F32 = torch.bfloat16, torch.float32


def rel(x, want):
    x, want = x.detach().double().cpu(), want.double()
    assert x.shape == want.shape
    assert torch.isfinite(x).all()
    top = want.abs().max().item() if want.numel() else 0.0
    off = (x - want).abs().max().item() if want.numel() else 0.0
    return off / top if top > 0 else off


def make(seed, B, T, N, K, V, Nq=None, Nk=None, dtype=BF, state=F32, norm=True, gate="psi", step="logit", cu=None, strided=False, h0=True):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    Nq, Nk = Nq or N, Nk or N
    lead = (cu[-1],) if cu else (B, T)
    q, k, v = torch.nn.functional.silu(r(*lead, Nq, K)), torch.nn.functional.silu(r(*lead, Nk, K)), r(*lead, N, V)
    if not norm:
        q, k = q * K ** -0.5, ref.unit(k, 1e-3)
    o = dict(q_scale=K ** -0.5 if norm else 1.0, qk_norm=norm, norm_eps=1e-6)
    if gate == "psi":
        gt = r(*lead, N)
        o.update(gate_kind=m.GATE_PSI, alpha=torch.rand(N, generator=g) * 4 + 0.5, beta=r(N) - 2)
    elif gate == "logit":
        gt = r(*lead, N) + 2
        o.update(gate_kind=m.GATE_LOGIT)
    else:
        gt = -torch.rand(*lead, N, generator=g) * 0.3
        o.update(gate_kind=m.GATE_LOG)
    st = r(*lead, N) if step == "logit" else torch.rand(*lead, N, generator=g)
    o["step_kind"] = m.STEP_LOGIT if step == "logit" else m.STEP_VALUE
    x = [t.to(dtype) for t in (q, k, v, gt, st)]
    H0 = (r(B, N, K, V) * 0.2).to(state) if h0 else None
    dy, d_hT = r(*lead, N, V).to(dtype), (r(B, N, K, V) * 0.2).to(state)
    on = [t.cuda() for t in x]
    if strided:      # slices of one tensor
        wide = torch.cat([t.flatten(-2) for t in on[:3]] + [torch.full((*lead, 32), math.nan, dtype=dtype, device="cuda")], -1)
        cut, parts = 0, []
        for t in on[:3]:
            w = t.shape[-1] * t.shape[-2]
            parts.append(wide[..., cut:cut + w].unflatten(-1, t.shape[-2:]))
            cut += w
        on[:3] = parts
    return x, on, H0, dy, d_hT, o


def on_gpu(o):
    return {k: (v.cuda() if isinstance(v, torch.Tensor) else v) for k, v in o.items()}


def run_both(seed=0, cu=None, use_ckpt=True, d_hT_given=True, **kw):
    x, on, H0, dy, d_hT, o = make(seed, cu=cu, **kw)
    dtype, state = kw.get("dtype", BF), kw.get("state", F32)
    B, N, K, V = kw["B"], kw["N"], kw["K"], kw["V"]
    h64 = H0.double() if H0 is not None else torch.zeros(B, N, K, V, dtype=torch.float64)
    y_r, hT_r, g_r = ref.gradients([t.double() for t in x], h64, dy.double(), d_hT.double() if d_hT_given else None, cu, **o)
    more = dict(on_gpu(o), state_dtype=state)
    if cu:
        more.update(cu_seqlens=torch.tensor(cu, dtype=torch.int32).cuda(), max_seqlen=max(b - a for a, b in zip(cu, cu[1:])))
    h0 = None if H0 is None else H0.cuda()
    y, hT, ckpt = m.m2rnn_delta_fwd(*on, h0, save_ckpt=use_ckpt, **more)
    g = m.m2rnn_delta_bwd(*on, h0, dy.cuda(), d_hT.cuda() if d_hT_given else None, ckpt=ckpt, **more)
    m.check_device_status()
    errs = dict(y=rel(y, y_r), hT=rel(hT, hT_r), **{n: rel(g[n], g_r[n]) for n in g_r})
    assert hT.dtype == state and g["dh0"].dtype == state and all(g[n].dtype == dtype for n in g_r if n != "dh0")
    return errs


SHAPES = [
    dict(B=1, T=1, N=1, K=16, V=16),
    dict(B=2, T=31, N=3, K=64, V=64),
    dict(B=1, T=32, N=2, K=48, V=32),
    dict(B=2, T=33, N=4, K=64, V=16, Nq=1, Nk=1),
    dict(B=1, T=65, N=6, K=112, V=64, Nq=2, Nk=3),
    dict(B=2, T=200, N=8, K=128, V=128, Nq=2, Nk=4),
    dict(B=1, T=130, N=2, K=80, V=128),
    dict(B=1, T=97, N=3, K=96, V=16),
    dict(B=3, T=70, N=2, K=32, V=128),
    dict(B=1, T=64, N=5, K=128, V=16, Nq=5, Nk=1),
]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(str(v) for v in s.values()))
def test_shapes(shape, dtype):
    errs = run_both(**shape, dtype=dtype)
    assert max(errs.values()) <= TOL[dtype], errs


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("gate", ["psi", "logit", "log"])
@pytest.mark.parametrize("step", ["logit", "value"])
@pytest.mark.parametrize("norm", [True, False])
def test_gates_steps_and_lengths(dtype, gate, step, norm):
    errs = run_both(seed=3, B=2, T=75, N=2, K=64, V=32, dtype=dtype, gate=gate, step=step, norm=norm)
    assert max(errs.values()) <= TOL[dtype], errs


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_without_optional_tensors(dtype):
    """No initial state, no gradient of the final one, no checkpoint."""
    errs = run_both(seed=4, B=2, T=50, N=4, K=64, V=64, Nq=2, Nk=2, dtype=dtype, h0=False, use_ckpt=False, d_hT_given=False)
    assert max(errs.values()) <= TOL[dtype], errs


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_states_of_bf16(dtype):
    errs = run_both(seed=5, B=2, T=40, N=2, K=64, V=64, dtype=dtype, state=BF)
    assert max(errs.values()) <= 2e-2, errs


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shared", [False, True])
def test_packed_and_strided(dtype, shared):
    cu = [0, 0, 1, 34, 34, 129, 161, 260]      # empty ones, single tokens, whole chunks, odd lengths
    errs = run_both(seed=6, B=7, T=0, N=4, K=64, V=32, Nq=1 if shared else 4, Nk=1 if shared else 4, cu=cu, dtype=dtype, strided=True)
    assert max(errs.values()) <= TOL[dtype], errs


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_many_shared_heads(dtype):
    """Heads that share q and k, several to a CTA of the gradient kernel: enough chunks for that."""
    errs = run_both(seed=7, B=5, T=97, N=84, K=32, V=16, Nq=1, Nk=1, dtype=dtype)
    assert max(errs.values()) <= TOL[dtype], errs


@pytest.mark.parametrize("K,V", [(16, 16), (48, 128), (64, 32), (64, 16)])
@pytest.mark.parametrize("B,N", [(100, 8), (9, 6), (150, 4)])
def test_jobs_of_the_gradient_kernel(B, N, K, V):
    """Numbers of chunks and heads for which it takes two and three CTAs to an SM, and one head and several to a job."""
    errs = run_both(seed=16, B=B, T=5, N=N, K=K, V=V, Nq=1, Nk=1)
    assert max(errs.values()) <= TOL[BF], errs


@pytest.mark.parametrize("use_ckpt", [True, False])
@pytest.mark.parametrize("N,K", [(3, 64), (60, 64), (148, 64), (3, 80), (60, 80), (148, 80)])
def test_numbers_of_chains(N, K, use_ckpt):
    """One, two and four chains to an SM, with y from the chains' own warps and from others."""
    errs = run_both(seed=17, B=1, T=40, N=N, K=K, V=64, Nq=1, Nk=1, use_ckpt=use_ckpt)
    assert max(errs.values()) <= TOL[BF], errs


@pytest.mark.parametrize("N", [200, 400, 560, 700])
@pytest.mark.parametrize("K", [16, 32, 64, 96])
def test_numbers_of_ctas_of_one_chain(N, K):
    errs = run_both(seed=19, B=1, T=40, N=N, K=K, V=16, Nq=1, Nk=1)
    assert max(errs.values()) <= TOL[BF], errs


@pytest.mark.parametrize("N,K", [(60, 64), (148, 64), (60, 80), (148, 80)])
def test_numbers_of_chains_and_a_value_that_is_not_finite(N, K):
    x, on, H0, dy, d_hT, o = make(18, B=1, T=75, N=N, K=K, V=64, gate="log", step="value")
    o = on_gpu(o)
    want = m.m2rnn_delta_fwd(*on, H0.cuda(), **o)[0]
    for at in (0, 20, 31, 40, 74):
        for which in (1, 2):
            bad = [t.clone() for t in on]
            bad[which][0, at, 1, 9] = math.nan
            for save in (False, True):
                y = m.m2rnn_delta_fwd(*bad, H0.cuda(), save_ckpt=save, **o)[0]
                others = [n for n in range(N) if n != 1]
                assert torch.equal(y[0][:, others], want[0][:, others])
                cols = slice(None) if which == 1 else slice(9, 10)
                assert torch.isnan(y[0, at:, 1, cols]).all()
                if at:
                    assert rel(y[0, :at, 1], want[0, :at, 1].cpu()) <= TOL[BF]


def test_keys_that_point_the_same_way():
    """T's diagonal blocks by substitution: with equal keys and steps of 1 M is a triangle of ones."""
    x, on, H0, dy, d_hT, o = make(8, B=1, T=96, N=2, K=64, V=32, gate="log", step="value")
    x[1] = x[1][:, :1].expand_as(x[1]).contiguous()
    x[3] = torch.zeros_like(x[3])
    x[4] = torch.ones_like(x[4])
    on = [t.cuda() for t in x]
    y_r, hT_r, g_r = ref.gradients([t.double() for t in x], H0.double(), dy.double(), None, **o)
    y, hT, ckpt = m.m2rnn_delta_fwd(*on, H0.cuda(), save_ckpt=True, **on_gpu(o))
    g = m.m2rnn_delta_bwd(*on, H0.cuda(), dy.cuda(), ckpt=ckpt, **on_gpu(o))
    errs = dict(y=rel(y, y_r), hT=rel(hT, hT_r), dv=rel(g["dv"], g_r["dv"]), dq=rel(g["dq"], g_r["dq"]), dh0=rel(g["dh0"], g_r["dh0"]))
    assert max(errs.values()) <= 2e-2, errs


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_dropped_states_and_skipped_tokens(dtype):
    """a = 0 (a log decay of -inf) drops the state, a = 1 with b = 0 leaves it; gradients stay finite and right."""
    x, on, H0, dy, d_hT, o = make(9, B=2, T=80, N=2, K=32, V=32, dtype=dtype, gate="log", step="value")
    x[3][:, 10] = -math.inf
    x[3][:, 33:36] = -math.inf
    x[3][1, 79] = -200.0
    x[3][:, 50:60] = 0
    x[4][:, 50:60] = 0
    on = [t.cuda() for t in x]
    y_r, hT_r, g_r = ref.gradients([t.double() for t in x], H0.double(), dy.double(), d_hT.double(), **o)
    y, hT, ckpt = m.m2rnn_delta_fwd(*on, H0.cuda(), save_ckpt=True, **on_gpu(o))
    g = m.m2rnn_delta_bwd(*on, H0.cuda(), dy.cuda(), d_hT.cuda(), ckpt=ckpt, **on_gpu(o))
    errs = dict(y=rel(y, y_r), hT=rel(hT, hT_r), **{n: rel(g[n], torch.nan_to_num(g_r[n])) for n in g_r})
    assert max(errs.values()) <= TOL[dtype], errs
    assert (g["dgate"][:, 10] == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_differences(dtype):
    """The gradient against central differences of the 64-bit definition along random directions."""
    x, on, H0, dy, d_hT, o = make(10, B=1, T=45, N=2, K=32, V=16, dtype=dtype)
    h0 = H0.cuda()
    _, _, ckpt = m.m2rnn_delta_fwd(*on, h0, save_ckpt=True, **on_gpu(o))
    g = m.m2rnn_delta_bwd(*on, h0, dy.cuda(), d_hT.cuda(), ckpt=ckpt, **on_gpu(o))
    x64, e = [t.double() for t in (*x, H0)], 1e-5
    gen = torch.Generator().manual_seed(1)
    for i, name in enumerate(("dq", "dk", "dv", "dgate", "dstep", "dh0")):
        d = torch.randn(x64[i].shape, generator=gen, dtype=torch.float64)

        def at(s):
            y, hT = ref.scan(*(t + s * d if j == i else t for j, t in enumerate(x64)), **o)
            return ((y * dy.double()).sum() + (hT * d_hT.double()).sum()).item()
        want, got = (at(e) - at(-e)) / (2 * e), (g[name].double().cpu() * d).sum().item()
        # a sum of independent errors of TOL of a typical entry each
        assert abs(want - got) <= TOL[dtype] * (g[name].double().norm().item() + abs(want)), (name, want, got)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_chunks_of_a_prompt_and_repeats(dtype):
    """A sequence in two calls, the state handed on, is the sequence in one; and a call repeats bit for bit."""
    x, on, H0, dy, d_hT, o = make(11, B=2, T=77, N=2, K=64, V=64, dtype=dtype)
    o = on_gpu(o)
    y, hT, _ = m.m2rnn_delta_fwd(*on, H0.cuda(), **o)
    y2, hT2, _ = m.m2rnn_delta_fwd(*on, H0.cuda(), **o)
    assert torch.equal(y, y2) and torch.equal(hT, hT2)
    cut = 32      # a multiple of the chunk: the same products
    ya, h, _ = m.m2rnn_delta_fwd(*(t[:, :cut].contiguous() for t in on), H0.cuda(), **o)
    yb, h, _ = m.m2rnn_delta_fwd(*(t[:, cut:].contiguous() for t in on), h, **o)
    assert torch.equal(torch.cat((ya, yb), 1), y) and torch.equal(h, hT)
    a = m.m2rnn_delta_bwd(*on, H0.cuda(), dy.cuda(), d_hT.cuda(), **o)
    b = m.m2rnn_delta_bwd(*on, H0.cuda(), dy.cuda(), d_hT.cuda(), **o)
    assert all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_lengths_without_epsilon(dtype):
    """norm_eps = 0: rows behind the last token, which are zeros, have no length to be divided by."""
    x, on, H0, dy, d_hT, o = make(13, B=2, T=43, N=2, K=48, V=32, dtype=dtype)
    o["norm_eps"] = 0.0
    y_r, hT_r, g_r = ref.gradients([t.double() for t in x], H0.double(), dy.double(), d_hT.double(), **o)
    y, hT, ckpt = m.m2rnn_delta_fwd(*on, H0.cuda(), save_ckpt=True, **on_gpu(o))
    g = m.m2rnn_delta_bwd(*on, H0.cuda(), dy.cuda(), d_hT.cuda(), ckpt=ckpt, **on_gpu(o))
    errs = dict(y=rel(y, y_r), hT=rel(hT, hT_r), **{n: rel(g[n], g_r[n]) for n in g_r})
    assert max(errs.values()) <= TOL[dtype], errs


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_rows_that_are_not_finite_stay_with_their_sequence(dtype):
    """A NaN in one sequence, or behind a packed batch's tokens, reaches no other."""
    x, on, H0, dy, d_hT, o = make(14, B=3, T=70, N=2, K=32, V=32, dtype=dtype)
    o = on_gpu(o)
    want = m.m2rnn_delta_fwd(*on, H0.cuda(), **o)[0]
    for t in on:
        t[1] = math.nan
    y, hT, ckpt = m.m2rnn_delta_fwd(*on, H0.cuda(), save_ckpt=True, **o)
    g = m.m2rnn_delta_bwd(*on, H0.cuda(), dy.cuda(), ckpt=ckpt, **o)
    keep = [0, 2]
    assert torch.equal(y[keep], want[keep]) and torch.isfinite(hT[keep]).all() and torch.isnan(y[1]).all()
    assert all(torch.isfinite(v[keep]).all() for v in g.values())
    flat = [t.flatten(0, 1)[:80].clone() for t in on]      # packed: sequences of 40 and 30 tokens, NaN in all that follows
    cu = torch.tensor([0, 40, 70], dtype=torch.int32, device="cuda")
    y, hT, _ = m.m2rnn_delta_fwd(*flat, cu_seqlens=cu, max_seqlen=40, **o)
    assert torch.isfinite(y[:70]).all() and torch.isfinite(hT).all()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("K,V", [(48, 32), (128, 64)])
@pytest.mark.parametrize("value", [math.nan, math.inf], ids=["nan", "inf"])
@pytest.mark.parametrize("at", [0, 3, 14, 21, 30, 47, 72])
def test_values_that_are_not_finite_reach_no_earlier_token(dtype, K, V, value, at):
    """As behind the last token of a right-padded batch: tokens before, other heads and other entries have the y that they had."""
    x, on, H0, dy, d_hT, o = make(15, B=2, T=75, N=4, K=K, V=V, Nq=2, Nk=2, dtype=dtype, gate="log", step="value")
    o = on_gpu(o)
    want = m.m2rnn_delta_fwd(*on, H0.cuda(), **o)[0]
    for which in range(5):
        # what it is planted in, and the heads that it may reach (q, k: head 0's group)
        bad = [t.clone() for t in on]
        bad[which][(0, at, 0) if which > 2 else (0, at, 0, 5)] = value
        heads = [0] if which > 1 else [0, 1]
        for save in (False, True):
            y, hT, _ = m.m2rnn_delta_fwd(*bad, H0.cuda(), save_ckpt=save, **o)
            others = [n for n in range(4) if n not in heads]
            assert torch.equal(y[1], want[1]) and torch.equal(y[0][:, others], want[0][:, others])
            assert torch.isfinite(hT[1]).all() and torch.isfinite(hT[0, others]).all()
            if at:
                assert rel(y[0, :at], want[0, :at].cpu()) <= TOL[dtype], which
            if which == 0:
                assert torch.isfinite(hT).all() and torch.equal(y[0, at + 1:], want[0, at + 1:]) and not torch.isfinite(y[0, at, heads]).any()
            elif which == 2:      # a column of the state
                rest = [v for v in range(V) if v != 5]
                assert not torch.isfinite(y[0, at:, 0, 5]).any() and not torch.isfinite(hT[0, 0, :, 5]).any()
                assert torch.equal(y[0][..., rest], want[0][..., rest]) and torch.isfinite(hT[0, 0][:, rest]).all()
            elif which != 3 or value != math.inf:      # (a decay of e^inf: by the formula, not asked for)
                assert not torch.isfinite(y[0, at:, heads]).any() and not torch.isfinite(hT[0, heads]).any()


def test_empty_calls():
    q = torch.zeros(2, 0, 2, 16, dtype=BF, device="cuda")
    v, gt = torch.zeros(2, 0, 2, 16, dtype=BF, device="cuda"), torch.zeros(2, 0, 2, dtype=BF, device="cuda")
    h0 = torch.ones(2, 2, 16, 16, device="cuda")
    y, _, _ = m.m2rnn_delta_fwd(q, q, v, gt, gt, h0)
    assert y.shape == v.shape
    g = m.m2rnn_delta_bwd(q, q, v, gt, gt, h0, v, 3 * h0)
    assert torch.equal(g["dh0"], 3 * h0)


STEP_SHAPES = [
    dict(B=1, N=84, K=64, V=16, Nq=1, Nk=1), dict(B=3, N=2, K=16, V=16), dict(B=5, N=4, K=48, V=32, Nq=2, Nk=4), dict(B=2, N=3, K=112, V=64),
    dict(B=7, N=2, K=128, V=128), dict(B=1, N=1, K=80, V=128), dict(B=300, N=5, K=64, V=64), dict(B=40, N=32, K=32, V=32), dict(B=2, N=2, K=112, V=16),
    dict(B=2, N=2, K=128, V=32), dict(B=400, N=8, K=128, V=16), dict(B=9, N=1, K=96, V=128),
]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("state", [BF, F32], ids=["sbf16", "sf32"])
@pytest.mark.parametrize("shape", STEP_SHAPES, ids=lambda s: "x".join(str(v) for v in s.values()))
def test_decode_step(shape, state, dtype):
    """All arithmetic in fp32: an output of bf16 is off by its own rounding (2^-8 of the value), one of fp32 by the sums
    (2^-24 times a few hundred terms)."""
    B = shape["B"]
    for gate, step, norm, pool in (("psi", "logit", True, 0), ("log", "value", False, 3), ("logit", "value", True, 5)):
        x, on, H0, _, _, o = make(20 + pool, T=1, dtype=dtype, state=state, gate=gate, step=step, norm=norm, **shape)
        x, on = [t[:, 0].contiguous() for t in x], [t[:, 0].contiguous() for t in on]
        S = B + pool
        slots = torch.randperm(S, generator=torch.Generator().manual_seed(B))[:B].to(torch.int32) if pool else None
        if pool:
            slots[B // 2] = -1
        at = slots.long() if pool else torch.arange(B)
        full = torch.randn(S, *H0.shape[1:], generator=torch.Generator().manual_seed(2)).to(state)
        q, k, v, gt, st = (t.double() for t in x)
        q, k, a, b = ref.prepared(q, k, gt, st, shape["N"], o)
        H, y_r = ref.one(full[at.clamp(min=0)].double(), q, k, v, a, b)
        y_r[at < 0] = 0
        want = full.double().clone()
        want[at[at >= 0]] = H[at >= 0]
        got = full.cuda()
        y = m.m2rnn_delta_decode_step(*on, got, slots=slots.cuda() if pool else None, **on_gpu(o))
        m.check_device_status()
        assert rel(y, y_r) <= (2.0 ** -8 if dtype == BF else 1e-5) * 1.01
        assert rel(got, want) <= (2.0 ** -8 if state == BF else 1e-5) * 1.01
        untouched = torch.ones(S, dtype=torch.bool)
        untouched[at[at >= 0]] = False
        assert torch.equal(got.cpu()[untouched], full[untouched])


def test_decode_slot_outside_the_pool_is_reported():
    x, on, H0, _, _, o = make(1, B=3, T=1, N=2, K=32, V=32)
    on = [t[:, 0].contiguous() for t in on]
    pool = torch.randn(4, 2, 32, 32, device="cuda")
    was = pool.clone()
    y = m.m2rnn_delta_decode_step(*on, pool, slots=torch.tensor([1, 4, -5], dtype=torch.int32).cuda(), **on_gpu(o))
    with pytest.raises(m.M2RNNError):
        m.check_device_status()
    assert (y[1:] == 0).all() and torch.equal(pool[[0, 2, 3]], was[[0, 2, 3]]) and not torch.equal(pool[1], was[1])


def test_steps_after_a_prompt():
    """A prompt, its states forked in the cache, tokens decoded: the sequence in one call."""
    N, K, V, T, more = 6, 64, 32, 41, 5
    x, on, _, _, _, o = make(12, B=1, T=T + more, N=N, K=K, V=V, dtype=F32)
    g = on_gpu(o)
    y, hT, _ = m.m2rnn_delta_fwd(*on, **g)
    _, h, _ = m.m2rnn_delta_fwd(*(t[:, :T].contiguous() for t in on), **g)
    pool = torch.full((8, N, K, V), math.nan, device="cuda")
    slots = torch.tensor([5, 0, 7], dtype=torch.int32).cuda()
    m.m2rnn_state_copy(pool, slots, torch.zeros(3, dtype=torch.int32).cuda(), h)
    for t in range(T, T + more):
        if t == T + 2:      # the sessions move
            to = torch.tensor([0, 5, 1], dtype=torch.int32).cuda()
            m.m2rnn_state_copy(pool, to, slots)
            slots = to
        yt = m.m2rnn_delta_decode_step(*(z[:, t].expand(3, *z.shape[2:]).contiguous() for z in on), pool, slots=slots, **g)
        for s in range(3):
            assert rel(yt[s], y[0, t].double().cpu()) <= 1e-4
    assert rel(pool[slots.long()[2]], hT[0].double().cpu()) <= 1e-4
