"""The operators of a layer that forgets by its data, as cases that can be timed: the gated delta rule (prompts, training steps,
single tokens), the rotation of queries and keys by their positions, and the norms before and after a block with its gate and
residual stream, in float, bfloat16 and half.

A case is a dict of plain values; its "path" says which operator it belongs to.  With `own` false, run() computes the operator
by elementary torch operations in 32 bits (angles and sums of logarithms in 64), rounded once at the end; with `own` true it
makes the calls a program makes of this library.  exact() computes the same from the definitions in 64 bits.
"""
import math

import torch

own = False  # run(): the library's calls (True) or elementary torch operations (False)

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_CHUNK = 64  # steps that the plain delta rule takes as one dense block
_EPS = 1e-5


def listed():
    return [
        # decoding for one user: the smallest call, bound by its launch
        dict(name="delta_step_one", path="step", dtype="bf16", batch=1, heads=16, qk_heads=8, dk=64, dv=64),
        # decoding for 256 users of wide heads: every state read and written once
        dict(name="delta_step_many", path="step", dtype="bf16", batch=256, heads=16, qk_heads=16, dk=128, dv=128),
        # one long prompt of 65,536 tokens: few sequences, so the length has to be split
        dict(name="delta_prompt", path="delta", dtype="bf16", seqs=1, tokens=65536, packed=False, heads=16, qk_heads=16, dk=64, dv=64, state=False, grad=False),
        # prompts of different lengths packed behind one another, continued from kept states, with heads that no tile divides
        dict(name="delta_packed", path="delta", dtype="f32", seqs=37, tokens=30011, packed=True, heads=12, qk_heads=4, dk=50, dv=72, state=True, grad=False),
        # a training step, forward and backward: batch 8 x 4096 tokens, 16 heads of 128
        dict(name="delta_train", path="delta", dtype="bf16", seqs=8, tokens=32768, packed=False, heads=16, qk_heads=16, dk=128, dv=128, state=False, grad=True),
        # a training step in float over windows of 1000 tokens with carried states, queries and keys shared by four heads
        dict(name="delta_train_float", path="delta", dtype="f32", seqs=8, tokens=8000, packed=False, heads=8, qk_heads=2, dk=32, dv=64, state=True, grad=True),
        # the queries and keys of 256 decoded tokens, each at a position of its own, up to a million tokens in
        dict(name="rotary_decode", path="rotary", dtype="bf16", seqs=256, tokens=256, heads=16, kv_heads=4, dim=64, pairs=32, interleaved=False, factor=32.0, grad=False),
        # a training step's queries and keys, slices of one projection: 8 x 4096 tokens, 16 heads of 128, and the gradients' way back
        dict(name="rotary_train", path="rotary", dtype="bf16", seqs=8, tokens=32768, heads=16, kv_heads=16, dim=128, pairs=64, interleaved=False, factor=1.0, grad=True),
        # neighbouring entries as pairs, a part of heads that no vector divides, in float
        dict(name="rotary_part", path="rotary", dtype="f32", seqs=5, tokens=10005, heads=12, kv_heads=4, dim=77, pairs=19, interleaved=True, factor=4.0, grad=False),
        # the heads of one decoded token, normalised, gated and added to the residual stream: bound by its launch
        dict(name="norm_after_one", path="after", dtype="bf16", tokens=1, channels=2048, groups=16, kind="rms", act="silu", gate=True, residual=True, scale=False, grad=False),
        # the residual stream of a training step, 32,768 tokens of 2048 channels: block added with its scale, normalised for the next, both ways
        dict(name="norm_before_train", path="before", dtype="bf16", tokens=32768, channels=2048, groups=1, kind="rms", act="none", gate=False, residual=True, scale=True, grad=True),
        # heads of 107 channels with mean and bias, gate, scale and residual stream in float, both ways
        dict(name="norm_after_train", path="after", dtype="f32", tokens=6000, channels=1712, groups=16, kind="layer", act="gelu", gate=True, residual=True, scale=True, grad=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _head(rng):
    return _log_int(rng, 8, 128)


def draw(rng):
    path = rng.choice(["step", "delta", "delta", "delta", "rotary", "rotary", "before", "after"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32", "f32", "f16"])
    if path in ("step", "delta"):
        qk_heads = rng.choice([1, 2, 4, 8, 16])
        heads = qk_heads * rng.choice([1, 1, 2, 4])
        dk, dv = (_head(rng), _head(rng)) if rng.random() < 0.5 else (rng.choice([32, 64, 128]),) * 2
        if path == "step":
            return dict(path=path, dtype=dtype, batch=max(1, min(_log_int(rng, 1, 512), 4194304 * 16 // (heads * dk * dv))), heads=heads, qk_heads=qk_heads, dk=dk, dv=dv)
        grad = rng.random() < 0.5
        seqs = _log_int(rng, 1, 64)
        tokens = _log_int(rng, seqs, min(65536, 3 * 10**7 // (heads * max(dk, dv))))
        packed = rng.random() < 0.5
        if not packed:
            tokens = max(1, tokens // seqs) * seqs
        return dict(path=path, dtype=dtype, seqs=seqs, tokens=tokens, packed=packed, heads=heads, qk_heads=qk_heads, dk=dk, dv=dv, state=rng.random() < 0.5, grad=grad)
    if path == "rotary":
        kv_heads = rng.choice([1, 2, 4, 8, 16])
        heads = kv_heads * rng.choice([1, 1, 2, 4])
        dim = rng.choice([32, 64, 128]) if rng.random() < 0.5 else _log_int(rng, 8, 256)
        pairs = dim // 2 if rng.random() < 0.6 else rng.randint(1, dim // 2)
        seqs = _log_int(rng, 1, 64)
        tokens = max(1, _log_int(rng, seqs, min(65536, 6 * 10**7 // (heads * dim))) // seqs) * seqs
        return dict(path=path, dtype=dtype, seqs=seqs, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, pairs=pairs, interleaved=rng.random() < 0.5,
                    factor=rng.choice([1.0, 4.0, 32.0]), grad=rng.random() < 0.5)
    groups = rng.choice([1, 1, 1, 4, 16, 32])
    channels = groups * (_log_int(rng, 16, 8192) if groups == 1 else _log_int(rng, 2, 256))
    return dict(path=path, dtype=dtype, tokens=max(1, min(_log_int(rng, 1, 32768), 6 * 10**7 // channels)), channels=channels, groups=groups,
                kind=rng.choice(["rms", "rms", "layer"]), act=rng.choice(["none", "silu", "silu", "gelu"]), gate=rng.random() < 0.5, residual=rng.random() < 0.7,
                scale=rng.random() < 0.4, grad=rng.random() < 0.5)


# ---- inputs

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, dtype=torch.float32, device="cuda", generator=gen) * scale).to(dtype)


def _unit(gen, shape, dtype):
    """Rows of length one, as a layer's normalised queries and keys are."""
    x = torch.randn(shape, dtype=torch.float32, device="cuda", generator=gen)
    return (x / (x * x).sum(-1, keepdim=True).sqrt()).to(dtype)


def _lengths(case, seed):
    """Lengths of the sequences: equal ones, or ragged ones that add up to the tokens, one of them empty where there are several."""
    n, total = case["seqs"], case["tokens"]
    if not case["packed"]:
        return [total // n] * n
    if n == 1:
        return [total]
    w = torch.rand(n, generator=torch.Generator().manual_seed(int(seed)), dtype=torch.float64).pow(2) + 0.01
    w[n // 2] = 0.0
    cuts = (w.cumsum(0) / w.sum() * total).round().to(torch.int64).tolist()
    cuts[-1] = total
    return [b - a for a, b in zip([0] + cuts[:-1], cuts)]


def _frequencies(case):
    """base^(-i / pairs); for longer contexts, waves that the shorter context did not see whole are stretched by the factor, those that it
    saw often are left, and the others lie between."""
    i = torch.arange(case["pairs"], dtype=torch.float64)
    f = torch.pow(torch.tensor(10000.0, dtype=torch.float64), -i / case["pairs"])
    if case["factor"] > 1:
        turns = 4096 * f / (2 * math.pi)
        keep = ((turns - 1) / 31).clamp(0, 1)
        f = f * keep + f / case["factor"] * (1 - keep)
    return f.to(torch.float32).cuda()


def prepare(case, seed):
    gen, t = _generator(seed), _TYPES[case["dtype"]]
    s = {"case": case}
    if case["path"] in ("step", "delta"):
        H, Q, dk, dv = case["heads"], case["qk_heads"], case["dk"], case["dv"]
        if case["path"] == "step":
            lead, n = (case["batch"],), case["batch"]
        else:
            n = case["seqs"]
            lengths = _lengths(case, seed)
            lead = (case["tokens"],) if case["packed"] else (n, case["tokens"] // n)
            s["longest"] = max(lengths)
            s["offsets"] = torch.tensor([0] + lengths, dtype=torch.int64).cumsum(0).cuda() if case["packed"] else None
        s["q"] = _unit(gen, lead + (Q, dk), t)
        s["k"] = _unit(gen, lead + (Q, dk), t)
        s["v"] = _normal(gen, lead + (H, dv), t)
        # heads that forget within some ten tokens up to heads that remember thousands, each token in its own measure
        rate = torch.exp2(-torch.linspace(2.0, 11.0, H, device="cuda"))
        s["log_decay"] = -rate * torch.nn.functional.softplus(torch.randn(lead + (H,), device="cuda", generator=gen))
        s["beta"] = torch.sigmoid(torch.randn(lead + (H,), device="cuda", generator=gen))
        s["scale"] = 1.0 if case["path"] == "step" else dk ** -0.5
        s["state"] = _normal(gen, (n, H, dk, dv), torch.float32, 0.3) if case.get("state", True) else None
        if case["path"] == "step":
            s["next"] = torch.empty_like(s["state"])
        elif case["grad"]:
            s["grad_o"] = _normal(gen, lead + (H, dv), t)
            s["grad_state"] = _normal(gen, (n, H, dk, dv), torch.float32, 0.3) if case["state"] else None
    elif case["path"] == "rotary":
        H, G, d = case["heads"], case["kv_heads"], case["dim"]
        lead = (case["seqs"], case["tokens"] // case["seqs"])
        # slices of one projection to queries, keys and values
        fused = _normal(gen, lead + ((H + 2 * G) * d,), t)
        s["q"], s["k"] = fused[..., :H * d].unflatten(-1, (H, d)), fused[..., H * d:(H + G) * d].unflatten(-1, (G, d))
        start = torch.randint(0, 1 << 20 if case["factor"] > 1 else 4096, (lead[0], 1), device="cuda", generator=gen)
        s["positions"] = start + torch.arange(lead[1], device="cuda")
        s["frequencies"] = _frequencies(case)
        s["scale"] = 0.1 * math.log(case["factor"]) + 1.0
        if case["grad"]:
            s["grad_q"], s["grad_k"] = _normal(gen, lead + (H, d), t), _normal(gen, lead + (G, d), t)
    else:
        shape = (case["tokens"], case["channels"])
        s["x"] = (torch.randn(shape, device="cuda", generator=gen) * _spread(gen, shape[1]) + 0.3 * _spread(gen, shape[1])).to(t)
        s["gate"] = _normal(gen, shape, t) if case["gate"] else None
        s["residual"] = _normal(gen, shape, t, 2.0) if case["residual"] else None
        s["weight"] = _normal(gen, shape[1:], torch.float32, 0.1) + 1.0
        s["bias"] = _normal(gen, shape[1:], torch.float32, 0.1) if case["kind"] == "layer" else None
        s["scale"] = _normal(gen, shape[1:], torch.float32, 0.1) + 0.5 if case["scale"] else None
        if case["grad"]:
            s["grad_y"] = _normal(gen, shape, t)
            s["grad_h"] = _normal(gen, shape, t) if case["path"] == "before" else None
    return s


def _spread(gen, n):
    """Channels whose scales and means differ."""
    return 0.5 + torch.rand(n, device="cuda", generator=gen)


# ---- the library's calls

_kept = {}


def _library():
    """The context that a program opens once."""
    if "g" not in _kept:
        from paper_2510_03426_amd import Goom
        _kept["g"] = Goom(0)
    return _kept["g"]


def _named(**outputs):
    return {k: x for k, x in outputs.items() if x is not None}


def _run_own(s):
    g, case = _library(), s["case"]
    path = case["path"]
    if path == "step":
        return {"o": g.gated_delta_step(s["q"], s["k"], s["v"], s["log_decay"], s["beta"], s["state"], scale=s["scale"], out_state=s["next"]), "state": s["next"]}
    if path == "delta":
        q, k, v, a, b = (s[x] for x in ("q", "k", "v", "log_decay", "beta"))
        r = {}
        r["o"], r["state"] = g.gated_delta(q, k, v, a, b, state=s["state"], offsets=s["offsets"], scale=s["scale"], want_state=True)
        if case["grad"]:
            gq, gk, gv, ga, gb, gs = g.gated_delta_backward(q, k, v, a, b, s["grad_o"], state=s["state"], grad_state=s["grad_state"], offsets=s["offsets"], scale=s["scale"])
            r.update(_named(gq=gq, gk=gk, gv=gv, glog_decay=ga, gbeta=gb, gstate=gs))
        return r
    if path == "rotary":
        how = dict(interleaved=case["interleaved"], scale=s["scale"])
        r = {}
        r["q"], r["k"] = g.rotary(s["q"], s["k"], s["positions"], s["frequencies"], **how)
        if case["grad"]:
            r["gq"], r["gk"] = g.rotary_backward(s["grad_q"], s["grad_k"], s["positions"], s["frequencies"], **how)
        return r
    how = dict(groups=case["groups"], weight=s["weight"], bias=s["bias"], scale=s["scale"], gate=s["gate"], kind=case["kind"], activation=case["act"])
    if path == "after":
        y, mean, rstd = g.norm_after(s["x"], residual=s["residual"], eps=_EPS, want_stats=True, **how)
        r = _named(y=y, mean=mean, rstd=rstd)
        if case["grad"]:
            gx, ggate, gw, gb, gs = g.norm_after_backward(s["x"], s["grad_y"], mean, rstd, **how)
            r.update(_named(gx=gx, ggate=ggate, gweight=gw, gbias=gb, gscale=gs))
        return r
    y, h, mean, rstd = g.norm_before(s["x"], residual=s["residual"], eps=_EPS, want_stats=True, **how)
    r = _named(y=y, h=h, mean=mean, rstd=rstd)
    if case["grad"]:
        gres, gx, ggate, gw, gb, gs = g.norm_before_backward(s["x"], h, s["grad_y"], mean, rstd, grad_h=s["grad_h"], **how)
        r.update(_named(gresidual=gres, gx=gx, ggate=ggate, gweight=gw, gbias=gb, gscale=gs))
    return r


# ---- elementary torch operations, in 32 bits

def _padded(x, s, n):
    """Packed tokens [tokens, ...] -> [sequences, longest, ...], zeros after each sequence's end; float."""
    x = x.float()
    if s["offsets"] is None:
        return x
    off, at = s["offsets"], torch.arange(s["longest"], device=x.device)
    valid = at < (off[1:] - off[:-1])[:, None]
    index = torch.where(valid, off[:-1, None] + at, torch.zeros_like(at))
    return x[index] * valid[(...,) + (None,) * (x.dim() - 1)]


def _packed(x, s, dtype):
    """The way back, rounded to the type."""
    if s["offsets"] is not None:
        off, at = s["offsets"], torch.arange(s["longest"], device=x.device)
        x = x[at < (off[1:] - off[:-1])[:, None]]
    return x.to(dtype)


def _inverse(L):
    """(I + L)^-1 of strictly lower triangular L: blocks of one entry, then of two, of four, ..."""
    C = L.shape[-1]
    i = torch.arange(C, device=L.device)
    R = torch.eye(C, device=L.device).expand_as(L)
    size = 1
    while size < C:
        low = (i[:, None] // size % 2 == 1) & (i // size % 2 == 0) & (i[:, None] // (2 * size) == i // (2 * size))
        R = R - torch.matmul(torch.matmul(R, L * low), R)
        size *= 2
    return R


def _turn(x):
    return x.transpose(-1, -2).contiguous()


def _run_delta(s):
    """Chunks of _CHUNK tokens: what lies within them is dense and done for all at once; their states follow one another."""
    case, c = s["case"], s["scale"]
    n, H, Q, dk, dv = case["seqs"], case["heads"], case["qk_heads"], case["dk"], case["dv"]
    share = H // Q
    rows = {x: _padded(s[x], s, n) for x in ("q", "k", "v", "log_decay", "beta")}
    T = rows["q"].shape[1]
    C, m = _CHUNK, max(1, -(-T // _CHUNK))

    def blocks(x):  # [n, T, heads, d] -> [chunks, n, heads, C, d]
        x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, m * C - T))
        return x.reshape(n, m, C, x.shape[2], x.shape[3]).permute(1, 0, 3, 2, 4).contiguous()

    q, k = (blocks(rows[x].repeat_interleave(share, dim=2)) for x in "qk")
    v, beta = blocks(rows["v"]), blocks(rows["beta"][..., None])
    b = blocks(rows["log_decay"][..., None].double()).cumsum(-2)
    i = torch.arange(C, device=q.device)
    gap = (b - b.transpose(-1, -2)).masked_fill(i[:, None] < i, -math.inf).exp().float()
    up, down, whole = b.exp().float(), (b[..., -1:, :] - b).exp().float(), b[..., -1:, :].exp().float()
    kk = torch.matmul(k, _turn(k)) * gap * (i[:, None] > i)
    pairs = torch.matmul(q, _turn(k)) * gap
    R = _inverse(kk * beta.transpose(-1, -2))
    k_up, k_down, q_up = k * up, k * down, q * up
    k_down_t = _turn(k_down)
    S = s["state"] if s["state"] is not None else torch.zeros(n, H, dk, dv, device=q.device)
    states, E = [], []
    for t in range(m):
        states.append(S)
        E.append(torch.matmul(R[t], v[t] - torch.matmul(k_up[t], S)))
        S = whole[t] * S + torch.matmul(k_down_t[t], beta[t] * E[t])
    first, E = torch.stack(states), torch.stack(E)
    U = beta * E
    o = c * (torch.matmul(q_up, first) + torch.matmul(pairs, U))

    def rows_of(x, dtype, shared=False):  # and back
        x = x.permute(1, 0, 3, 2, 4).reshape(n, m * C, H, -1)[:, :T]
        return _packed(x.reshape(n, T, Q, share, -1).sum(3) if shared else x, s, dtype)

    t = s["q"].dtype
    r = {"o": rows_of(o, t), "state": S}
    if not case["grad"]:
        return r
    do = c * blocks(_padded(s["grad_o"], s, n))
    D = s["grad_state"] if s["grad_state"] is not None else torch.zeros_like(S)
    local, R_t = torch.matmul(_turn(pairs), do), _turn(_inverse(kk * beta))
    q_up_t, k_up_t = _turn(q_up), _turn(k_up)
    adjoints, W = [None] * m, [None] * m
    for j in reversed(range(m)):
        adjoints[j] = D
        W[j] = torch.matmul(R_t[j], local[j] + torch.matmul(k_down[j], D))
        D = whole[j] * D + torch.matmul(q_up_t[j], do[j]) - torch.matmul(k_up_t[j], beta[j] * W[j])
    last, W = torch.stack(adjoints), torch.stack(W)
    gv = beta * W
    first_t, U_t = _turn(first), _turn(U)
    dp = torch.matmul(do, U_t) * gap
    dk_pairs = torch.matmul(gv, U_t) * gap * (i[:, None] > i)
    gq = up * torch.matmul(do, first_t) + torch.matmul(dp, k)
    k_last = down * torch.matmul(U, _turn(last))
    k_row = -up * torch.matmul(gv, first_t) - torch.matmul(dk_pairs, k)
    k_col = torch.matmul(_turn(dp), q) - torch.matmul(_turn(dk_pairs), k) + k_last
    # every logarithm b_i stands in what row i reads, against what it gives away; the last one also in the next state
    gb = (q * gq + k * (k_row - k_col)).double().sum(-1)
    gb[..., -1] += (k * k_last).double().sum((-1, -2)) + whole[..., 0, 0] * (last * first).double().sum((-1, -2))
    ga = gb.flip(-1).cumsum(-1).flip(-1)[..., None]
    r.update(gq=rows_of(gq, t, True), gk=rows_of(k_row + k_col, t, True), gv=rows_of(gv, t),
             glog_decay=rows_of(ga, torch.float32)[..., 0], gbeta=rows_of((W * E).sum(-1, keepdim=True), torch.float32)[..., 0])
    if s["state"] is not None:
        r["gstate"] = D
    return r


def _run_step(s):
    share = s["case"]["heads"] // s["case"]["qk_heads"]
    q, k = (s[x].float().repeat_interleave(share, dim=1) for x in "qk")
    state = torch.exp(s["log_decay"])[..., None, None] * s["state"]
    u = s["beta"][..., None] * (s["v"].float() - (k[..., None] * state).sum(-2))
    state = state + k[..., None] * u[..., None, :]
    return {"o": (s["scale"] * (q[..., None] * state).sum(-2)).to(s["q"].dtype), "state": state}


def _rotated(x, angle, s, back=False):
    case = s["case"]
    p = case["pairs"]
    cos, sin = (s["scale"] * f(angle).float()[..., None, :] for f in (torch.cos, torch.sin))
    if back:
        sin = -sin
    z = x.float()
    head = z[..., :2 * p]
    one, two = (head[..., 0::2], head[..., 1::2]) if case["interleaved"] else (head[..., :p], head[..., p:])
    both = (one * cos - two * sin, one * sin + two * cos)
    head = torch.stack(both, -1).flatten(-2) if case["interleaved"] else torch.cat(both, -1)
    return torch.cat((head, z[..., 2 * p:]), -1).to(x.dtype)


def _run_rotary(s):
    angle = s["positions"].double()[..., None] * s["frequencies"].double()
    r = {"q": _rotated(s["q"], angle, s), "k": _rotated(s["k"], angle, s)}
    if s["case"]["grad"]:
        r.update(gq=_rotated(s["grad_q"], angle, s, True), gk=_rotated(s["grad_k"], angle, s, True))
    return r


def _act(z, act):
    """The activation and its derivative."""
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return z * p, p * (1 + z * (1 - p))
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * p, p + z * torch.exp(-0.5 * z * z) * (0.5 / math.pi) ** 0.5
    return z, torch.ones_like(z)


def _normed(x, case):
    """Normalised groups, and their mean (None where it is not taken off) and factor."""
    x = x.reshape(x.shape[0], case["groups"], -1)
    mean = x.mean(-1, keepdim=True) if case["kind"] == "layer" else None
    d = x - mean if mean is not None else x
    rstd = 1 / torch.sqrt((d * d).mean(-1, keepdim=True) + _EPS)
    return (d * rstd).reshape(x.shape[0], -1), mean, rstd


def _norm_back(dx, xhat, rstd, case):
    dx, h = (t.reshape(t.shape[0], case["groups"], -1) for t in (dx, xhat))
    g = dx - h * (dx * h).mean(-1, keepdim=True)
    if case["kind"] == "layer":
        g = g - dx.mean(-1, keepdim=True)
    return (rstd * g).reshape(xhat.shape)


def _run_norm(s):
    case, t = s["case"], s["x"].dtype
    x = s["x"].float()
    gate, slope = _act(s["gate"].float(), case["act"]) if case["gate"] else (1.0, None)
    scale = s["scale"] if case["scale"] else 1.0
    residual = s["residual"].float() if case["residual"] else 0.0
    bias = s["bias"] if s["bias"] is not None else 0.0
    before = case["path"] == "before"
    h = residual + scale * x * gate if before else x
    if before and s["x"].dtype != torch.float32:
        h = h.to(t).float()  # what the block's residual stream holds is what is normalised
    xhat, mean, rstd = _normed(h, case)
    n = xhat * s["weight"] + bias
    y = n if before else residual + scale * n * gate
    r = _named(y=y.to(t), h=h.to(t) if before else None, mean=mean[..., 0] if mean is not None else None, rstd=rstd[..., 0])
    if not case["grad"]:
        return r
    gy = s["grad_y"].float()
    if before:
        dn = gy
        total = _norm_back(dn * s["weight"], xhat, rstd, case) + s["grad_h"].float()
        r["gresidual"] = total.to(t)
        inner = x
        r["gx"] = (total * scale * gate).to(t)
    else:
        total, inner = gy, n
        dn = gy * scale * gate
        r["gx"] = _norm_back(dn * s["weight"], xhat, rstd, case).to(t)
    if case["gate"]:
        r["ggate"] = (total * scale * inner * slope).to(t)
    r["gweight"] = (dn * xhat).sum(0)
    if s["bias"] is not None:
        r["gbias"] = dn.sum(0)
    if case["scale"]:
        r["gscale"] = (total * inner * gate).sum(0)
    return r


def run(s):
    if own:
        return _run_own(s)
    return {"step": _run_step, "delta": _run_delta, "rotary": _run_rotary, "before": _run_norm, "after": _run_norm}[s["case"]["path"]](s)


# ---- what a pass cannot do without

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["path"] in ("step", "delta"):
        H, Q, dk, dv = case["heads"], case["qk_heads"], case["dk"], case["dv"]
        n, seqs = (case["batch"],) * 2 if case["path"] == "step" else (case["tokens"], case["seqs"])
        tensors = n * (size * (2 * Q * dk + H * dv) + 8 * H)  # q, k, v, decays and betas, or their gradients
        outs = n * size * H * dv
        states = 4 * seqs * H * dk * dv
        token = 7 * n * H * dk * dv  # decay, prediction, update and readout of each token: the recurrent form's operations
        if case["path"] == "step":
            return {"bytes": tensors + outs + 2 * states, "flops": token}
        nbytes, flops = tensors + outs + states * (2 if case["state"] else 1), token
        if case["grad"]:
            nbytes += 2 * tensors + outs + (3 * states if case["state"] else 0)
            flops += 2 * token
        return {"bytes": nbytes, "flops": flops}
    if case["path"] == "rotary":
        e = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["dim"]
        times = 2 if case["grad"] else 1
        return {"bytes": times * (2 * e * size + 8 * case["tokens"] + 4 * case["pairs"]), "flops": times * 3 * e}
    e = case["tokens"] * case["channels"]
    stats = 4 * case["tokens"] * case["groups"] * (2 if case["kind"] == "layer" else 1)
    before = case["path"] == "before"
    tensors = 2 + case["gate"] + case["residual"] + before
    params = 4 * case["channels"] * (1 + (case["kind"] == "layer") + case["scale"])
    nbytes, flops = tensors * e * size + stats + params, 12 * e
    if case["grad"]:
        # read: what was normalised, the gradients, the gate, the block's output where gate or scale want it; written: each gradient that is a tensor of its own
        back = (4 + 2 * (case["gate"] or case["scale"]) if before else 3) + 2 * case["gate"]
        nbytes += back * e * size + stats + 2 * params
        flops += 25 * e
    return {"bytes": nbytes, "flops": flops}


# ---- the definitions in 64 bits

def _exact_delta(case, s, seed):
    """The recurrence, token after token, and its adjoint walked back over kept states."""
    n, H, share, c = case["seqs"], case["heads"], case["heads"] // case["qk_heads"], s["scale"]
    lengths = _lengths(case, seed)
    T = max(lengths)
    if T * (3 if case["grad"] else 1) * max(1.0, n * H * case["dk"] * case["dv"] / 4e6) > 1.2e5:
        return None
    total, ends = sum(lengths), torch.tensor(lengths).cumsum(0)[:, None].cuda()
    at = torch.arange(T, device="cuda") + ends - torch.tensor(lengths, device="cuda")[:, None]
    alive, index = at < ends, at.clamp(max=total - 1)

    def steps(x, zero=0.0):  # [T, n, heads, ...]: what is beyond an end changes nothing
        x = x.double().reshape((total,) + x.shape[-2 if x is not s["log_decay"] and x is not s["beta"] else -1:])
        x = x[index]
        return torch.where(alive[(...,) + (None,) * (x.dim() - 2)], x, torch.full_like(x, zero)).transpose(0, 1).contiguous()

    q, k = (steps(s[x]).repeat_interleave(share, dim=2) for x in "qk")
    v, a, b = steps(s["v"]), torch.exp(steps(s["log_decay"])), steps(s["beta"])
    S = torch.zeros(n, H, case["dk"], case["dv"], dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()

    def forward(S, t):
        S = a[t][..., None, None] * S
        e = v[t] - (k[t].unsqueeze(-2) @ S).squeeze(-2)
        return S + k[t][..., None] * (b[t][..., None] * e)[..., None, :], e

    o = torch.empty_like(v)
    every = max(1, int(math.sqrt(T)))
    kept = []
    for t in range(T):
        if t % every == 0:
            kept.append(S)
        S, _ = forward(S, t)
        o[t] = c * (q[t].unsqueeze(-2) @ S).squeeze(-2)

    def back(x, tail, shared=False):
        x = x.transpose(0, 1)
        if shared:
            x = x.reshape(n, T, H // share, share, -1).sum(3)
        return x[alive].reshape(s["q"].shape[:-2] + tail)

    r = {"o": back(o, (H, case["dv"])), "state": S}
    if not case["grad"]:
        return r
    do = steps(s["grad_o"])
    D = torch.zeros_like(S) if s["grad_state"] is None else s["grad_state"].double()
    gq, gk, gv, ga, gb = (torch.zeros_like(x) for x in (q, k, v, a, b))
    for j in reversed(range(len(kept))):
        S, states = kept[j], []
        for t in range(j * every, min(T, (j + 1) * every)):
            old = S
            S, e = forward(S, t)
            states.append((old, S, e))
        for t in reversed(range(j * every, min(T, (j + 1) * every))):
            old, new, e = states.pop()
            gq[t] = c * (new @ do[t][..., None]).squeeze(-1)
            D = D + c * q[t][..., None] * do[t][..., None, :]
            du = (k[t].unsqueeze(-2) @ D).squeeze(-2)
            gb[t] = (du * e).sum(-1)
            gv[t] = b[t][..., None] * du
            gk[t] = (D @ (b[t][..., None] * e)[..., None]).squeeze(-1) - a[t][..., None] * (old @ gv[t][..., None]).squeeze(-1)
            D = a[t][..., None, None] * (D - k[t][..., None] * gv[t][..., None, :])
            ga[t] = (D * old).sum((-1, -2))
    r.update(gq=back(gq, (H // share, case["dk"]), True), gk=back(gk, (H // share, case["dk"]), True), gv=back(gv, (H, case["dv"])),
             glog_decay=back(ga, (H,)), gbeta=back(gb, (H,)))
    if s["state"] is not None:
        r["gstate"] = D
    return r


def _exact_rotary(case, s):
    """Pairs as complex numbers, times scale e^(i angle)."""
    p = case["pairs"]
    turn = s["scale"] * torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[..., None] * s["frequencies"].double())[..., None, :]

    def rotate(x, turn):
        out = x.double().clone()
        at = torch.arange(p, device="cuda")
        one, two = (2 * at, 2 * at + 1) if case["interleaved"] else (at, at + p)
        z = torch.complex(out[..., one], out[..., two]) * turn
        out[..., one], out[..., two] = z.real, z.imag
        return out

    r = {"q": rotate(s["q"], turn), "k": rotate(s["k"], turn)}
    if case["grad"]:
        r.update(gq=rotate(s["grad_q"], turn.conj()), gk=rotate(s["grad_k"], turn.conj()))
    return r


def _exact_norm(case, s):
    leaves = {k: s[k].double().requires_grad_(case["grad"]) for k in ("x", "gate", "residual", "weight", "bias", "scale") if s[k] is not None}
    inner = leaves["x"]
    one = torch.ones((), dtype=torch.float64, device="cuda")
    z = leaves.get("gate", one)
    gate = one if not case["gate"] else z if case["act"] == "none" else z * torch.sigmoid(z) if case["act"] == "silu" else z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    res, scale = leaves.get("residual", one * 0), leaves.get("scale", one)
    before = case["path"] == "before"
    stream = res + scale * inner * gate if before else inner
    if before:  # normalised as it is held, in the type of the stream
        stream = stream + (stream.detach().to(s["x"].dtype).double() - stream.detach())
    x = stream.reshape(case["tokens"], case["groups"], -1)
    mean = x.sum(-1, keepdim=True) / x.shape[-1] if case["kind"] == "layer" else 0.0 * x[..., :1]
    rstd = (((x - mean) ** 2).sum(-1, keepdim=True) / x.shape[-1] + _EPS) ** -0.5
    n = ((x - mean) * rstd).reshape(s["x"].shape) * leaves["weight"] + leaves.get("bias", 0.0)
    y = n if before else res + scale * n * gate
    r = _named(y=y.detach(), h=stream.detach() if before else None, mean=mean[..., 0].detach() if case["kind"] == "layer" else None, rstd=rstd[..., 0].detach())
    if case["grad"]:
        outs, grads = [y], [s["grad_y"].double()]
        if before:
            outs, grads = outs + [stream], grads + [s["grad_h"].double()]
        names = [k for k in leaves if k != "residual"]
        if before:
            total = torch.autograd.grad(outs, stream, grads, retain_graph=True)[0]
            r["gresidual"] = total.detach()
        got = torch.autograd.grad(outs, [leaves[k] for k in names], grads)
        r.update({"g" + k: x for k, x in zip(names, got)})
    return r


def exact(case, seed):
    s = prepare(case, seed)
    if case["path"] == "delta":
        return _exact_delta(case, s, seed)
    if case["path"] == "step":
        share = case["heads"] // case["qk_heads"]
        q, k = (s[x].double().repeat_interleave(share, dim=1) for x in "qk")
        eye = torch.eye(case["dk"], dtype=torch.float64, device="cuda")
        forget = eye - s["beta"].double()[..., None, None] * k[..., :, None] * k[..., None, :]
        state = torch.exp(s["log_decay"].double())[..., None, None] * (forget @ s["state"].double())
        state += s["beta"].double()[..., None, None] * k[..., :, None] * s["v"].double()[..., None, :]
        return {"o": s["scale"] * (q[..., None, :] @ state)[..., 0, :], "state": state}
    if case["path"] == "rotary":
        return _exact_rotary(case, s)
    return _exact_norm(case, s)
