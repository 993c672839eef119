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
