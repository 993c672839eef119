"""Performance cases of the gated delta rule and of the cache of recurrent states: what is measured of them.

The gated delta rule is the linear recurrence of the hybrid models that an M2RNN layer is put into: per
(batch b, head n), on a K x V state H, with a decay a_t in (0, 1] and a step b_t in [0, 1],

    u_t = b_t (v_t - a_t H_{t-1}^T k_t)        H_t = a_t H_{t-1} + k_t u_t^T        y_t = H_t^T (s q_t)

with q_t and k_t divided by their lengths and s = K^-1/2.  Decays come from a projection through the
forget gate a = (1 + e^{x+beta})^{-alpha}, steps through a sigmoid.  A case is a dict of plain values;
``kind`` says what one pass is:

  step      one decoded token of a serving batch on cached states, which lie in a pool of slots
  prefill   a prompt: the scan, its final state kept
  train     the scan and its gradient
  copy      states moved between the slots of a pool: forked, compacted, freed

With ``own`` false everything is computed with elementary torch operations in fp32 (the scans in chunks
of 64 tokens), with ``own`` true by the library's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False

IO = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6       # in the lengths of q and k
CHUNK = 64       # of the plain form


def listed():
    return [
        # one session, one token, a layer of 84 value heads that share one q/k head: latency
        dict(name="step_token", kind="step", dtype="bf16", state="f32", B=1, spare=0, N=84, shared=True, K=64, V=16),
        # a small serving batch on the same layer, its states scattered over a pool
        dict(name="step_layer", kind="step", dtype="bf16", state="f32", B=48, spare=16, N=84, shared=True, K=64, V=16),
        # 512 sessions of large states kept in 16 bits: bound by HBM
        dict(name="step_full", kind="step", dtype="bf16", state="bf16", B=512, spare=0, N=32, shared=False, K=128, V=128),
        # a prompt of odd length
        dict(name="prefill_prompt", kind="prefill", dtype="bf16", B=1, T=1001, N=84, shared=True, K=64, V=16),
        # a batch of prompts
        dict(name="prefill_batch", kind="prefill", dtype="bf16", B=8, T=2048, N=16, shared=False, K=64, V=64),
        # one very long prompt
        dict(name="prefill_long", kind="prefill", dtype="bf16", B=1, T=65536, N=32, shared=False, K=128, V=128),
        # a training step's layer at a training context of 4 096, 84 value heads to one q/k head
        dict(name="train_layer", kind="train", dtype="bf16", B=4, T=4096, N=84, shared=True, K=64, V=16, packed=False),
        # many heads of their own
        dict(name="train_batch", kind="train", dtype="bf16", B=8, T=4096, N=32, shared=False, K=64, V=64, packed=False),
        # documents of ragged lengths packed into one batch, q/k/v slices of a fused projection, large states
        dict(name="train_packed", kind="train", dtype="bf16", B=12, T=4000, N=16, shared=False, K=128, V=128, packed=True),
        # fp32, the accuracy path, with initial states and their gradient
        dict(name="train_f32", kind="train", dtype="f32", B=2, T=512, N=8, shared=False, K=64, V=64, packed=False),
        # a prompt's states (all layers of a small model) forked for eight samples
        dict(name="copy_fork", kind="copy", state="f32", layers=24, slots=64, n=8, fork=True, N=84, K=64, V=16),
        # a serving batch compacted: states move to the slots that finished sessions left, others are cleared
        dict(name="copy_compact", kind="copy", state="bf16", layers=1, slots=512, n=200, fork=False, N=32, K=128, V=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = [work(c) for c in listed()]
    most = {x: max(w[x] for w in top) for x in ("bytes", "flops")}
    while True:
        kind = rng.choice(("step", "step", "prefill", "prefill", "train", "train", "train", "copy"))
        V = rng.choice((16, 32, 64, 128))
        K = 64 if V == 16 and rng.random() < 0.5 else V if rng.random() < 0.5 else 16 * rng.randint(1, 8)
        case = dict(kind=kind, N=rng.randint(2, 96), K=K, V=V)
        if kind == "copy":
            slots = _log(rng, 4, 512)
            case.update(state=rng.choice(("f32", "bf16")), layers=rng.choice((1, 1, 2, 5, 24)), slots=slots,
                        n=rng.randint(1, max(1, slots // 2)), fork=rng.random() < 0.5)
        else:
            case.update(dtype="f32" if rng.random() < 0.15 else "bf16", shared=V == 16 or rng.random() < 0.3)
            if kind == "step":
                case.update(state=rng.choice(("f32", "bf16")), B=_log(rng, 1, 512), spare=rng.choice((0, 0, 3, 16)))
            else:
                case.update(B=_log(rng, 1, 12), T=_log(rng, 1, 65536 if kind == "prefill" else 8192))
                if kind == "train":
                    case.update(packed=rng.random() < 0.3)
                # the plain form's passes stay within seconds and the accuracy path within small models
                if case["dtype"] == "f32" and (case["T"] > 2048 or case["B"] * case["N"] > 148):
                    continue
                if case["B"] * case["T"] * case["N"] > 1 << 21 or (kind == "train" and case["B"] * case["T"] * case["N"] * max(K, V) > 1 << 26):
                    continue
        w = work(case)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return case


def _lengths(case):
    """Token counts of the documents of a packed batch; the longest is T."""
    rng = random.Random(1000003 * case["T"] + 101 * case["B"] + case["N"])
    return [case["T"]] + [max(1, int(case["T"] * rng.uniform(0.02, 1.0) ** 1.5)) for _ in range(case["B"] - 1)]


def _moves(case):
    """(sources, destinations) of a copy: a fork of slot 0, or states moved down into free slots and a few
    slots cleared (source -1)."""
    n, slots = case["n"], case["slots"]
    rng = random.Random(9176 * n + 31 * slots + case["layers"])
    places = list(range(1, slots))
    rng.shuffle(places)
    n = min(n, len(places))
    if case["fork"]:
        return [0] * n, places[:n]
    dst = sorted(places[:n])
    src = [d + 1 + rng.randrange(max(1, slots // 4)) if rng.random() < 0.9 else -1 for d in dst]
    return [s if s < slots else -1 for s in src], dst


def _tokens(case):
    return sum(_lengths(case)) if case.get("packed") else case["B"] * case["T"]


def work(case):
    N, K, V = case["N"], case["K"], case["V"]
    if case["kind"] == "copy":
        src, dst = _moves(case)
        row = case["layers"] * N * K * V * IO[case["state"]].itemsize
        return {"bytes": (len({s for s in src if s >= 0}) + len(dst)) * row, "flops": 0}
    e = IO[case["dtype"]].itemsize
    h = 1 if case["shared"] else N
    if case["kind"] == "step":
        units = case["B"] * N
        return {"bytes": case["B"] * (2 * h * K + 2 * N * V + 2 * N) * e + 2 * units * K * V * IO[case["state"]].itemsize, "flops": 7 * units * K * V}
    tok = _tokens(case)
    qkv, gates, y = tok * (2 * h * K + N * V) * e, 2 * tok * N * e, tok * N * V * e
    state = case["B"] * N * K * V * e
    flops = 7 * tok * N * K * V     # of the recurrence itself: decay, k.H, the outer product, q.H
    if case["kind"] == "prefill":
        return {"bytes": qkv + gates + y + state, "flops": flops}
    states = 4 * state if case["dtype"] == "f32" else 0     # h0, hT, their gradients
    return {"bytes": 2 * (qkv + gates) + 2 * y + states, "flops": 3 * flops}


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(int(seed))
    N, K, V = case["N"], case["K"], case["V"]

    def normal(*shape, std=1.0, mean=0.0, to=torch.float32):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=gen).to(to)

    def uniform(*shape, lo, hi):
        return torch.empty(shape, dtype=torch.float32, device="cuda").uniform_(lo, hi, generator=gen)

    if case["kind"] == "copy":
        src, dst = _moves(case)
        shape = (case["slots"], N, K, V)
        pool = normal(*((case["layers"],) if case["layers"] > 1 else ()), *shape, to=IO[case["state"]])
        return dict(kind="copy", pool=pool, axis=pool.dim() - 4, src=torch.tensor(src, dtype=torch.int32, device="cuda"),
                    dst=torch.tensor(dst, dtype=torch.int32, device="cuda"))
    io, B, h = IO[case["dtype"]], case["B"], 1 if case["shared"] else N
    # the gate's constants as such layers are initialised: alpha in 1 .. 16, softplus(beta) log-uniform in 0.001 .. 0.1
    dt = torch.exp(uniform(N, lo=math.log(1e-3), hi=math.log(1e-1)))
    s = dict(kind=case["kind"], alpha=uniform(N, lo=1.0, hi=16.0), beta=dt + torch.log(-torch.expm1(-dt)), scale=K ** -0.5, N=N)
    lead = (B,) if case["kind"] == "step" else (B, case["T"])
    s["more"], s["index"] = {}, None
    if case.get("packed"):
        lens = _lengths(case)
        lead = (sum(lens),)
        cu = torch.zeros(B + 1, dtype=torch.int32)
        cu[1:] = torch.tensor(lens, dtype=torch.int32).cumsum(0)
        s["more"] = dict(cu_seqlens=cu.cuda(), max_seqlen=case["T"])
        # where the plain form finds token t of document b, and which of its rows are tokens
        t = torch.arange(case["T"])
        s["index"] = (cu[:-1, None].long() + t).clamp_(max=sum(lens) - 1).cuda()
        s["valid"] = (t < torch.tensor(lens)[:, None]).cuda()
    # q, k, v come out of a convolution and SiLU as slices of one tensor; a decoding step takes dense rows
    x = torch.nn.functional.silu(normal(*lead, 2 * h * K + N * V)).to(io)
    q, k, v = x[..., : h * K].unflatten(-1, (h, K)), x[..., h * K: 2 * h * K].unflatten(-1, (h, K)), x[..., 2 * h * K:].unflatten(-1, (N, V))
    if case["kind"] == "step":
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    s.update(q=q, k=k, v=v, gate=normal(*lead, N, to=io), step=normal(*lead, N, to=io))
    if case["kind"] == "step":
        slots = B + case["spare"]
        s["pool"] = normal(slots, N, K, V, std=0.1, to=IO[case["state"]])
        order = list(range(slots))
        random.Random(slots).shuffle(order)
        s["slots"] = torch.tensor(order[:B], dtype=torch.int32, device="cuda")
    elif case["kind"] == "train":
        s["dy"] = normal(*lead, N, V, to=io)
        s["h0"] = s["d_hT"] = None
        if case["dtype"] == "f32":
            s["h0"], s["d_hT"] = normal(B, N, K, V, std=0.1), normal(B, N, K, V, std=0.1)
    return s


# ---- the plain form

def _softplus(x):
    return torch.clamp(x, min=0) + torch.log1p(torch.exp(-torch.abs(x)))


def _unit(x):
    return x * torch.rsqrt((x * x).sum(-1, keepdim=True) + EPS)


def _inverse(m):
    """(I + m)^-1 of strictly lower triangular m [..., CHUNK, CHUNK], by inverting diagonal blocks of 1, 2, 4, ... rows."""
    lead = m.shape[:-2]
    x = torch.eye(CHUNK, device=m.device, dtype=m.dtype).expand(m.shape)
    size = 1
    while size < CHUNK:
        pairs = CHUNK // (2 * size)
        at = torch.arange(pairs, device=m.device)
        blocks = lambda a: a.reshape(*lead, pairs, 2, size, pairs, 2, size)[..., at, :, :, at, :, :].movedim(0, -5)  # noqa: E731
        b, low = blocks(x), blocks(m)[..., 1, :, 0, :]
        x11, x22 = b[..., 0, :, 0, :], b[..., 1, :, 1, :]
        x21 = -(x22 @ low @ x11)
        both = torch.cat((torch.cat((x11, torch.zeros_like(x11)), -1), torch.cat((x21, x22), -1)), -2)     # [..., pairs, 2 size, 2 size]
        x = (both.unsqueeze(-2) * torch.eye(pairs, device=m.device, dtype=m.dtype)[:, None, :, None]).reshape(*lead, CHUNK, CHUNK)
        size *= 2
    return x


def _scan(q, k, v, log_a, step, h0):
    """q, k [B,N,T,K], v [B,N,T,V], log_a, step [B,N,T] in fp32 -> y [B,N,T,V] and the final state."""
    B, N, T, V = v.shape
    K, n = k.shape[-1], -(-T // CHUNK)
    more = n * CHUNK - T
    rows = lambda x: torch.nn.functional.pad(x, (0, 0, 0, more)).reshape(B, N, n, CHUNK, x.shape[-1])  # noqa: E731
    q, k, v = rows(q), rows(k), rows(v)
    log_a, step = rows(log_a.unsqueeze(-1)).squeeze(-1), rows(step.unsqueeze(-1))
    g = log_a.cumsum(-1)
    lower = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=v.device).tril()
    decay = torch.exp((g.unsqueeze(-1) - g.unsqueeze(-2)).masked_fill(~lower, -math.inf))
    eg, last = torch.exp(g).unsqueeze(-1), g[..., -1:]
    inv = _inverse(((k @ k.transpose(-1, -2)) * decay * step).tril(-1))
    w, u0 = inv @ (step * eg * k), inv @ (step * v)
    p = (q @ k.transpose(-1, -2)) * decay
    qe, ke, ec = q * eg, k * torch.exp(last - g).unsqueeze(-1), torch.exp(last).unsqueeze(-1)
    H = h0 if h0 is not None else torch.zeros(B, N, K, V, device=v.device, dtype=v.dtype)
    ys = []
    for c in range(n):
        u = u0[:, :, c] - w[:, :, c] @ H
        ys.append(qe[:, :, c] @ H + p[:, :, c] @ u)
        H = ec[:, :, c] * H + ke[:, :, c].transpose(-1, -2) @ u
    return torch.stack(ys, 2).reshape(B, N, n * CHUNK, V)[:, :, :T], H


def _plain_scan(s, q, k, v, gate, step, h0):
    io = v.dtype
    q, k, v, gate, step = (x.float() for x in (q, k, v, gate, step))
    if s["index"] is not None:      # documents as rows of a padded batch
        valid = s["valid"]
        q, k, v = (x[s["index"]] * valid[..., None, None] for x in (q, k, v))
        gate, step = gate[s["index"]], step[s["index"]]
    heads = lambda x: x.transpose(1, 2).expand(-1, s["N"], -1, -1) if x.shape[2] == 1 else x.transpose(1, 2)  # noqa: E731
    log_a = -s["alpha"] * _softplus(gate + s["beta"])
    step = 1 / (1 + torch.exp(-step))
    if s["index"] is not None:
        log_a, step = log_a * valid[..., None], step * valid[..., None]
    y, hT = _scan(_unit(heads(q)) * s["scale"], _unit(heads(k)), heads(v), log_a.transpose(1, 2), step.transpose(1, 2), None if h0 is None else h0.float())
    y = y.transpose(1, 2)
    return (y if s["index"] is None else y[valid]).to(io), hT


def _plain(s):
    if s["kind"] == "copy":
        pool, src, dst = s["pool"], s["src"].long(), s["dst"].long()
        fresh = (src >= 0).reshape(-1, 1, 1, 1)
        if s["axis"]:
            pool[:, dst] = torch.where(fresh, pool[:, src.clamp(min=0)], 0)
        else:
            pool[dst] = torch.where(fresh, pool[src.clamp(min=0)], 0)
        return pool
    if s["kind"] == "step":
        slots = s["slots"].long()
        H = s["pool"][slots].float()
        q, k, v, gate, step = (s[x].float() for x in ("q", "k", "v", "gate", "step"))
        a = torch.exp(-s["alpha"] * _softplus(gate + s["beta"]))[..., None, None]
        b = (1 / (1 + torch.exp(-step)))[..., None, None]
        H = a * H
        q, k = _unit(q) * s["scale"], _unit(k)
        H = H + k.unsqueeze(-1) * (b * (v.unsqueeze(-2) - k.unsqueeze(-2) @ H))
        y = (q.unsqueeze(-2) @ H).squeeze(-2)
        s["pool"][slots] = H.to(s["pool"].dtype)
        return y.to(s["v"].dtype), s["pool"]
    names = ("q", "k", "v", "gate", "step")
    if s["kind"] == "prefill":
        y, hT = _plain_scan(s, *(s[x] for x in names), None)
        return y, hT.to(y.dtype)
    leaves = [s[x].detach().requires_grad_() for x in names]
    h0 = None if s["h0"] is None else s["h0"].detach().requires_grad_()
    with torch.enable_grad():
        y, hT = _plain_scan(s, *leaves, h0)
    if h0 is None:
        return (y.detach(), *torch.autograd.grad(y, leaves, s["dy"]))
    return (y.detach(), hT.detach(), *torch.autograd.grad((y, hT), (*leaves, h0), (s["dy"], s["d_hT"])))


# ---- the library's calls

def _own(s):
    from paper_2603_14360_b200 import binding as m
    if s["kind"] == "copy":
        return m.m2rnn_state_copy(s["pool"], s["dst"], s["src"], axis=s["axis"])
    gates = dict(gate_kind=m.GATE_PSI, alpha=s["alpha"], beta=s["beta"], step_kind=m.STEP_LOGIT, qk_norm=True, norm_eps=EPS, q_scale=s["scale"])
    x = [s[name] for name in ("q", "k", "v", "gate", "step")]
    if s["kind"] == "step":
        return m.m2rnn_delta_decode_step(*x, s["pool"], slots=s["slots"], **gates), s["pool"]
    if s["kind"] == "prefill":
        y, hT, _ = m.m2rnn_delta_fwd(*x, state_dtype=s["v"].dtype, **gates)
        return y, hT
    h0, d_hT = s["h0"], s["d_hT"]
    y, hT, ckpt = m.m2rnn_delta_fwd(*x, h0, save_ckpt=True, want_hT=h0 is not None, **gates, **s["more"])
    g = m.m2rnn_delta_bwd(*x, h0, s["dy"], d_hT, ckpt=ckpt, want_dh0=h0 is not None, **gates, **s["more"])
    grads = tuple(g[name] for name in ("dq", "dk", "dv", "dgate", "dstep"))
    return (y, *grads) if h0 is None else (y, hT, *grads, g["dh0"])


def run(s):
    return _own(s) if own else _plain(s)


# ---- the definition in 64 bits, token after token

def _token(H, q, k, v, a, b):
    """One token of the recurrence: H [..., K, V], q, k [..., K], v [..., V], a, b [...]."""
    H = H * a[..., None, None]
    u = b[..., None] * (v - torch.einsum("...kv,...k->...v", H, k))
    H = H + torch.einsum("...k,...v->...kv", k, u)
    return H, torch.einsum("...kv,...k->...v", H, q)


def _gates64(s, gate, step):
    z = gate + s["beta"].double()
    a = torch.exp(-s["alpha"].double() * torch.logaddexp(z, torch.zeros_like(z)))
    return a, torch.sigmoid(step)


def _piece(H, q, k, v, a, b):
    ys = []
    for t in range(q.shape[1]):
        H, y = _token(H, q[:, t], k[:, t], v[:, t], a[:, t], b[:, t])
        ys.append(y)
    return H, torch.stack(ys, 1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "copy":
        was = s["pool"].clone().movedim(s["axis"], 0)
        now = s["pool"].movedim(s["axis"], 0)
        for i, j in zip(s["src"].tolist(), s["dst"].tolist()):
            now[j] = was[i] if i >= 0 else 0
        return s["pool"].double()
    names = ("q", "k", "v", "gate", "step")
    N = case["N"]
    if case["kind"] == "step":
        q, k, v, gate, step = (s[x].double() for x in names)
        q, k = (x / torch.sqrt((x ** 2).sum(-1, keepdim=True) + EPS) for x in (q, k))
        pool = s["pool"].double()
        a, b = _gates64(s, gate, step)
        at = s["slots"].long()
        pool[at], y = _token(pool[at], (q * s["scale"]).expand(-1, N, -1), k.expand(-1, N, -1), v, a, b)
        return y, pool
    if case["T"] * case["B"] * N * case["K"] * case["V"] * (8 if case["kind"] == "train" else 2) > 6e11 or case["T"] > 70000:
        return None
    leaves = [s[x].double().requires_grad_(case["kind"] == "train") for x in names]
    h0 = s.get("h0")
    h0 = torch.zeros(case["B"], N, case["K"], case["V"], dtype=torch.float64, device="cuda") if h0 is None else h0.double().requires_grad_()
    with torch.set_grad_enabled(case["kind"] == "train"):
        q, k, v, gate, step = leaves
        q, k = (x / torch.sqrt((x ** 2).sum(-1, keepdim=True) + EPS) for x in (q, k))
        a, b = _gates64(s, gate, step)
        x = [q * s["scale"], k, v, a, b]
        if s["index"] is not None:
            x = [y[s["index"]] for y in x]
            x[3] = torch.where(s["valid"][..., None], x[3], 1.0)      # behind a document's end nothing happens
            x[4] = torch.where(s["valid"][..., None], x[4], 0.0)
        x[:2] = [y.expand(-1, -1, N, -1) for y in x[:2]]
        H, ys = h0, []
        for t in range(0, case["T"], 64):
            part = [y[:, t:t + 64] for y in x]
            if case["kind"] == "train":     # states of a piece are recomputed in the gradient
                H, y = torch.utils.checkpoint.checkpoint(_piece, H, *part, use_reentrant=False)
            else:
                H, y = _piece(H, *part)
            ys.append(y)
        y = torch.cat(ys, 1)
        if s["index"] is not None:
            y = y[s["valid"]]
    if case["kind"] == "prefill":
        return y, H
    outs, seeds, wrt = [y], [s["dy"].double()], list(leaves)
    if s["h0"] is not None:
        outs, seeds, wrt = outs + [H], seeds + [s["d_hT"].double()], wrt + [h0]
    grads = torch.autograd.grad(outs, wrt, seeds)
    return (*(o.detach() for o in outs), *grads)
