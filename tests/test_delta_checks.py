"""Host-side checks of the delta rule's and the state copy's C ABI that need no GPU: sizes of workspaces and checkpoints, and
what is refused before anything is launched."""
import ctypes

import pytest

from paper_2603_14360_b200 import binding as m

FAKE, ODD, WS = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10004), ctypes.c_void_p(0x20000)


@pytest.fixture(scope="module")
def lib():
    from paper_2603_14360_b200 import build
    build.build()
    return m._lib()


def par(**kw):
    base = dict(B=2, T=70, N=4, Nq=4, Nk=4, K=32, V=32, io_dtype=1, state_dtype=0, gate_kind=m.GATE_LOG, step_kind=0, qk_norm=0,
                norm_eps=1e-6, q_scale=1.0)
    base.update(kw)
    return m.DeltaParams(**base)


def fwd(lib, p, ws=WS, size=1 << 40, **over):
    a = dict(q=FAKE, k=FAKE, v=FAKE, gate=FAKE, step=FAKE, h0=None, alpha=None, beta=None, y=FAKE, hT=None, ckpt=None)
    a.update(over)
    return lib.m2rnn_delta_fwd(None if p is None else ctypes.byref(p), *a.values(), ws, size, None, None)


def bwd(lib, p, ws=WS, size=1 << 40, **over):
    a = dict(q=FAKE, k=FAKE, v=FAKE, gate=FAKE, step=FAKE, h0=None, alpha=None, beta=None, ckpt=None, dy=FAKE, d_hT=None, dq=FAKE, dk=FAKE,
             dv=FAKE, dgate=FAKE, dstep=FAKE, dh0=None)
    a.update(over)
    return lib.m2rnn_delta_bwd(ctypes.byref(p), *a.values(), ws, size, None, None)


def step(lib, p, n_slots=2, **over):
    a = dict(q=FAKE, k=FAKE, v=FAKE, gate=FAKE, step=FAKE, alpha=None, beta=None, state=FAKE, slots=None)
    tail = dict(y=FAKE)
    tail.update({k: over.pop(k) for k in list(over) if k == "y"})
    a.update(over)
    return lib.m2rnn_delta_decode_step(ctypes.byref(p), *a.values(), n_slots, tail["y"], None, None)


BAD = [(dict(N=0), -2), (dict(Nq=3), -2), (dict(Nk=8), -2), (dict(K=24), -3), (dict(K=144), -3), (dict(K=0), -2), (dict(V=48), -3), (dict(V=256), -3), (dict(io_dtype=2), -3),
       (dict(state_dtype=2), -3), (dict(gate_kind=m.GATE_VALUE), -3), (dict(gate_kind=4), -3), (dict(step_kind=2), -3), (dict(B=-1), -2),
       (dict(B=1 << 28, N=16), -2)]


@pytest.mark.parametrize("change,status", BAD, ids=str)
def test_sizes_and_kinds(lib, change, status):
    p = par(**change)
    assert fwd(lib, p) == status and bwd(lib, p) == status and step(lib, p, n_slots=p.B) == status
    assert lib.m2rnn_delta_ckpt_bytes(ctypes.byref(p)) == lib.m2rnn_delta_bwd_workspace_bytes(ctypes.byref(p), 1) == 0


def test_sequence_arguments(lib):
    assert fwd(lib, None) == -1
    assert fwd(lib, par(T=-1)) == -2
    assert fwd(lib, par(q_stride=64)) == -2 and fwd(lib, par(v_stride=132)) == -2      # shorter than a token's heads; not whole 16 bytes
    assert fwd(lib, par(total_tokens=5)) == -2                                          # without cu_seqlens
    assert fwd(lib, par(cu_seqlens=0x10000, total_tokens=141)) == -2                    # more than B T
    assert fwd(lib, par(B=1 << 20, T=1 << 20, N=64, Nq=64, Nk=64)) == -2                # more chunks than a launch has CTAs
    assert fwd(lib, par(gate_kind=m.GATE_PSI)) == -1 and bwd(lib, par(gate_kind=m.GATE_PSI), alpha=FAKE) == -1
    for name in ("q", "k", "v", "gate", "step", "y"):
        assert fwd(lib, par(), **{name: None}) == -1
        assert fwd(lib, par(), **{name: ODD}) == -4
    for name in ("q", "k", "v", "gate", "step", "dy", "dq", "dk", "dv", "dgate", "dstep"):
        assert bwd(lib, par(), **{name: None}) == -1
        assert bwd(lib, par(), **{name: ODD}) == -4
    for name in ("h0", "hT", "ckpt"):
        assert fwd(lib, par(), **{name: ODD}) == -4
    assert fwd(lib, par(), ckpt=ctypes.c_void_p(0x10010)) == -4                         # 256-byte aligned
    assert fwd(lib, par(T=0)) == 0 and fwd(lib, par(B=0)) == 0                          # empty calls launch nothing
    assert bwd(lib, par(B=0)) == 0 and bwd(lib, par(T=0)) == 0


@pytest.mark.parametrize("io", [0, 1])
def test_workspaces(lib, io):
    p = par(io_dtype=io)
    need = lib.m2rnn_delta_fwd_workspace_bytes(ctypes.byref(p), 0)
    assert need > 0 and lib.m2rnn_delta_fwd_workspace_bytes(ctypes.byref(p), 1) == 0
    assert fwd(lib, p, size=need - 1) == -5 and fwd(lib, p, ws=None) == -5 and fwd(lib, p, ws=ctypes.c_void_p(0x20010), size=need) == -4
    keep, with_it, without = lib.m2rnn_delta_ckpt_bytes(ctypes.byref(p)), *(lib.m2rnn_delta_bwd_workspace_bytes(ctypes.byref(p), h) for h in (1, 0))
    assert keep > need and without == with_it + keep
    assert bwd(lib, p, size=without - 1) == -5 and bwd(lib, p, ckpt=FAKE, size=with_it - 1) == -5
    # shared q and k: shares of dq and dk
    assert lib.m2rnn_delta_bwd_workspace_bytes(ctypes.byref(par(io_dtype=io, Nq=1, Nk=1)), 1) >= with_it
    # a packed batch is sized by its tokens, not by B times the longest
    packed = par(io_dtype=io, B=50, T=4096, cu_seqlens=0x10000, total_tokens=5000)
    assert lib.m2rnn_delta_ckpt_bytes(ctypes.byref(packed)) < lib.m2rnn_delta_ckpt_bytes(ctypes.byref(par(io_dtype=io, B=50, T=4096))) / 10


def test_longest_length(lib):
    """A packed batch may give any upper bound of its lengths, the largest number too: sizes follow its tokens."""
    most = (1 << 31) - 1
    for io in (0, 1):
        sizes = [lib.m2rnn_delta_ckpt_bytes(ctypes.byref(par(io_dtype=io, B=3, N=64, T=T, Nq=64, Nk=64, cu_seqlens=0x10000, total_tokens=5000))) for T in (5000, most)]
        assert sizes[0] == sizes[1] > 0
        # a dense one of that length: 2^31 tokens of 1 head, 5 120 (3 584) bytes of record to a chunk
        p = par(io_dtype=io, B=1, N=1, Nq=1, Nk=1, K=16, V=16, T=most)
        assert lib.m2rnn_delta_ckpt_bytes(ctypes.byref(p)) > (1 << 31) / 32 * 5120
        assert fwd(lib, p, size=1 << 20) == -5
    assert fwd(lib, par(T=most, N=64, Nq=64, Nk=64)) == -2


def test_decoding_step(lib):
    assert step(lib, par(), n_slots=3) == -2                    # without slots a state for every row
    assert step(lib, par(), n_slots=-1, slots=FAKE) == -2
    for name in ("q", "k", "v", "gate", "step", "state", "y"):
        assert step(lib, par(), **{name: None}) == -1
        assert step(lib, par(), **{name: ODD}) == -4
    assert step(lib, par(gate_kind=m.GATE_PSI)) == -1
    assert step(lib, par(B=0), n_slots=0) == 0 and step(lib, par(B=0, T=-7), n_slots=0) == 0


def test_state_copy(lib):
    most = lib.m2rnn_state_copy_limit()
    assert most >= 1024

    def copy(n=4, row=64, layers=1, rows=8, dst=FAKE, src=WS, to=FAKE, frm=FAKE, stride=512):
        return lib.m2rnn_state_copy(dst, to, rows, stride, src, frm, rows, stride, n, row, layers, None, None)
    assert copy(n=-1) == -2 and copy(row=40) == -2 and copy(rows=-1) == -2 and copy(layers=-1) == -2
    assert copy(n=most + 1) == -3
    assert copy(dst=None) == -1 and copy(to=None) == -1
    assert copy(src=ODD) == -4
    assert copy(layers=2, stride=500) == -2 and copy(layers=2, stride=256) == -2       # not whole 16 bytes; layers that overlap
    assert copy(layers=1 << 30, row=1 << 20, stride=1 << 40) == -2
    assert copy(n=0, dst=None) == 0 and copy(layers=0) == 0 and copy(row=0) == 0


def test_binding_refuses_on_the_host(lib):
    import torch
    q = torch.zeros(1, 4, 2, 16)
    with pytest.raises(ValueError, match="CUDA"):
        m.m2rnn_delta_fwd(q, q, q, torch.zeros(1, 4, 2), torch.zeros(1, 4, 2))
    with pytest.raises(ValueError, match="CUDA"):
        m.m2rnn_state_copy(torch.zeros(3, 16), torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(TypeError):
        m.m2rnn_delta_decode_step(q[0], q[0], q[0], None, None, q)
