"""The operators around the recurrences in a language model's layer, as cases that can be timed: token embeddings and their
gradient, linear attention with a decay for each head (prompts, training steps, single tokens), and group norm with an
activation, channels last, in float, bfloat16 and half.

A case is a dict of plain values; its "path" says which operator it belongs to.  With `own` false, run() computes the operator
by elementary torch operations in 32 bits, rounded once at the end; with `own` true it makes the calls a program makes of this
library.  exact() computes the same from the definitions in 64 bits.
"""
import math

import torch

own = False  # run(): the library's calls (True) or elementary torch operations (False)

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_CHUNK = 128  # steps that the plain linear attention takes as one dense block


def listed():
    return [
        # decoding for one user: the smallest call, bound by its launch
        dict(name="step_one", path="step", dtype="bf16", batch=1, heads=16, kv_heads=16, dk=64, dv=64),
        # decoding for 256 users of wide heads: every state read and written once
        dict(name="step_many", path="step", dtype="bf16", batch=256, heads=16, kv_heads=16, dk=128, dv=128),
        # one long prompt of 65,536 tokens: few sequences, so the length has to be split
        dict(name="attend_prompt", path="attend", dtype="bf16", seqs=1, tokens=65536, packed=False, heads=16, kv_heads=16, dk=64, dv=64, state=False, grad=False),
        # prompts of different lengths packed behind one another, continued from kept states, with heads that no tile divides
        dict(name="attend_packed", path="attend", dtype="f32", seqs=37, tokens=30011, packed=True, heads=12, kv_heads=4, dk=50, dv=72, state=True, grad=False),
        # a training step, forward and backward: batch 8 x 4096 tokens, 16 heads of 128
        dict(name="attend_train", path="attend", dtype="bf16", seqs=8, tokens=32768, packed=False, heads=16, kv_heads=16, dk=128, dv=128, state=False, grad=True),
        # a training step in float over windows of 1000 tokens with carried states, 64 heads in all, keys and values shared by four
        dict(name="attend_train_float", path="attend", dtype="f32", seqs=8, tokens=8000, packed=False, heads=8, kv_heads=2, dk=32, dv=64, state=True, grad=True),
        # every token's heads normalised after the recurrence, for one decoded token: bound by its launch
        dict(name="norm_one", path="norm", dtype="bf16", items=1, length=1, channels=1024, groups=16, act="silu", grad=False),
        # the same in a training step of 32,768 tokens, heads of 128
        dict(name="norm_train", path="norm", dtype="bf16", items=32768, length=1, channels=2048, groups=16, act="silu", grad=True),
        # statistics over whole sequences: 8 x 4096 positions, groups of 10 channels
        dict(name="norm_sequence_train", path="norm", dtype="f32", items=8, length=4096, channels=320, groups=32, act="gelu", grad=True),
        # the embeddings of 256 decoded tokens from a float table, with a width that no vector divides
        dict(name="embed_decode", path="embed", dtype="f32", tokens=256, vocab=50257, width=1001, grad=False),
        # a training step's embeddings and their gradient: 32,768 tokens of a vocabulary of 50,257
        dict(name="embed_train", path="embed", dtype="bf16", tokens=32768, vocab=50257, width=1024, grad=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    path = rng.choice(["step", "attend", "attend", "attend", "norm", "norm", "embed", "embed"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32", "f32", "f16"])
    if path == "step":
        kv_heads = rng.choice([1, 2, 4, 8, 16])
        heads = kv_heads * rng.choice([1, 1, 2, 4])
        dk, dv = (_head(rng), _head(rng)) if rng.random() < 0.5 else (rng.choice([32, 64, 128]),) * 2
        return dict(path=path, dtype=dtype, batch=min(_log_int(rng, 1, 512), 4194304 * 16 // (heads * dk * dv)), heads=heads, kv_heads=kv_heads, dk=dk, dv=dv)
    if path == "attend":
        kv_heads = rng.choice([1, 2, 4, 8, 16])
        heads = kv_heads * rng.choice([1, 1, 2])
        dk, dv = (_head(rng), _head(rng)) if rng.random() < 0.5 else (rng.choice([32, 64, 128]),) * 2
        grad = rng.random() < 0.5
        seqs = _log_int(rng, 1, 64)
        tokens = _log_int(rng, seqs, min(65536, 3 * 10**7 // (heads * max(dk, dv))))
        packed = rng.random() < 0.5
        if not packed:
            tokens = max(1, tokens // seqs) * seqs
        return dict(path=path, dtype=dtype, seqs=seqs, tokens=tokens, packed=packed, heads=heads, kv_heads=kv_heads, dk=dk, dv=dv,
                    state=rng.random() < 0.5, grad=grad)
    if path == "norm":
        groups = rng.choice([1, 4, 8, 16, 32])
        channels = groups * _log_int(rng, 2, 128)
        items = _log_int(rng, 1, 32768)
        length = 1 if rng.random() < 0.5 else _log_int(rng, 2, 4096)
        items = max(1, min(items, 3 * 10**7 // (length * channels)))
        return dict(path=path, dtype=dtype, items=items, length=length, channels=channels, groups=groups, act=rng.choice(["none", "silu", "gelu"]),
                    grad=rng.random() < 0.5)
    width = _log_int(rng, 16, 2048)
    return dict(path=path, dtype=dtype, tokens=min(_log_int(rng, 1, 32768), 3 * 10**7 // width), vocab=min(_log_int(rng, 64, 50257), 5 * 10**7 // width), width=width,
                grad=rng.random() < 0.6)


def _head(rng):
    return _log_int(rng, 8, 128)


# ---- inputs

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, dtype=torch.float32, device="cuda", generator=gen) * scale).to(dtype)


def _log_decays(heads):
    """Heads that forget within two tokens up to heads that remember some 500."""
    x = torch.linspace(1.0, 9.0, heads, dtype=torch.float64) if heads > 1 else torch.tensor([6.0], dtype=torch.float64)
    return torch.log1p(-torch.exp2(-x)).to(torch.float32).cuda()


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


def prepare(case, seed):
    gen, t = _generator(seed), _TYPES[case["dtype"]]
    s = {"case": case}
    if case["path"] in ("step", "attend"):
        H, G, dk, dv = case["heads"], case["kv_heads"], case["dk"], case["dv"]
        if case["path"] == "step":
            lead, n = (case["batch"],), case["batch"]
        else:
            n = case["seqs"]
            lengths = _lengths(case, seed)
            lead = (case["tokens"],) if case["packed"] else (n, case["tokens"] // n)
            s["longest"] = max(lengths)
            s["offsets"] = torch.tensor([0] + lengths, dtype=torch.int64).cumsum(0).cuda() if case["packed"] else None
        s["q"] = _normal(gen, lead + (H, dk), t)
        s["k"] = _normal(gen, lead + (G, dk), t, dk ** -0.5)
        s["v"] = _normal(gen, lead + (G, dv), t)
        s["log_decay"] = _log_decays(H)
        s["state"] = _normal(gen, (n, H, dk, dv), torch.float32) if case.get("state", True) else None
        if case["path"] == "step":
            s["next"] = torch.empty_like(s["state"])
        elif case["grad"]:
            s["grad_o"] = _normal(gen, lead + (H, dv), t)
            s["grad_state"] = _normal(gen, (n, H, dk, dv), torch.float32) if case["state"] else None
    elif case["path"] == "norm":
        shape = (case["items"], case["length"], case["channels"])
        s["x"] = (torch.randn(shape, device="cuda", generator=gen) * _spread(gen, case["channels"]) + _spread(gen, case["channels"])).to(t)
        s["weight"] = _normal(gen, shape[-1:], torch.float32, 0.1) + 1.0
        s["bias"] = _normal(gen, shape[-1:], torch.float32, 0.1)
        if case["grad"]:
            s["grad_y"] = _normal(gen, shape, t)
    else:
        # token frequencies fall with the rank, as in text; some positions are padding and hold no token (-1)
        V, n = case["vocab"], case["tokens"]
        u = torch.rand(n, device="cuda", generator=gen, dtype=torch.float64)
        tokens = torch.exp(u * math.log(V)).to(torch.int64).clamp_(1, V) - 1
        s["tokens"] = torch.where(torch.rand(n, device="cuda", generator=gen) < 0.02, torch.full_like(tokens, -1), tokens)
        s["table"] = _normal(gen, (V, case["width"]), t, 0.02)
        s["scale"] = math.sqrt(case["width"])
        if case["grad"]:
            s["grad"] = _normal(gen, (n, case["width"]), t)
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


def _run_own(s):
    g, case = _library(), s["case"]
    if case["path"] == "step":
        return {"o": g.linear_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"], out_state=s["next"]), "state": s["next"]}
    if case["path"] == "attend":
        r = {}
        r["o"], r["state"] = g.linear_attention(s["q"], s["k"], s["v"], s["log_decay"], state=s["state"], offsets=s["offsets"], want_state=True)
        if case["grad"]:
            r["gq"], r["gk"], r["gv"], gs = g.linear_attention_backward(s["q"], s["k"], s["v"], s["log_decay"], s["grad_o"], state=s["state"],
                                                                        grad_state=s["grad_state"], offsets=s["offsets"])
            if gs is not None:
                r["gstate"] = gs
        return r
    if case["path"] == "norm":
        y, mean, rstd = g.group_norm(s["x"], case["groups"], s["weight"], s["bias"], activation=case["act"], want_stats=True)
        r = {"y": y, "mean": mean, "rstd": rstd}
        if case["grad"]:
            r["gx"], r["gweight"], r["gbias"] = g.group_norm_backward(s["x"], s["grad_y"], mean, rstd, case["groups"], s["weight"], s["bias"], activation=case["act"])
        return r
    r = {"rows": g.embedding(s["table"], s["tokens"], scale=s["scale"])}
    if case["grad"]:
        r["gtable"] = g.embedding_backward(s["tokens"], s["grad"], case["vocab"], scale=s["scale"])
    return r


# ---- elementary torch operations, in 32 bits

def _padded(x, s, n):
    """Packed tokens [tokens, heads, d] -> [sequences, longest, heads, d], zeros after each sequence's end; float."""
    x = x.float()
    if s["offsets"] is None:
        return x.reshape((n, -1) + x.shape[-2:])
    off, at = s["offsets"], torch.arange(s["longest"], device=x.device)
    valid = at < (off[1:] - off[:-1])[:, None]
    index = torch.where(valid, off[:-1, None] + at, torch.zeros_like(at))
    return x[index] * valid[..., None, None]


def _packed(x, s, like):
    """The way back, rounded to the type of `like`."""
    if s["offsets"] is not None:
        off, at = s["offsets"], torch.arange(s["longest"], device=x.device)
        x = x[at < (off[1:] - off[:-1])[:, None]]
    return x.reshape(like.shape[:-2] + x.shape[-2:]).to(like.dtype)


def _turned(x, lengths):
    """Every sequence's tokens in reverse order (padding stays behind)."""
    at = lengths[:, None] - 1 - torch.arange(x.shape[1], device=x.device)
    return x[torch.arange(x.shape[0], device=x.device)[:, None], at.clamp_min(0)] * (at >= 0)[..., None, None]


def _decayed(a, b, c, log_decay):
    """y_i = sum over j <= i of exp(log_decay (i - j)) (a_i . b_j) c_j: dense blocks of _CHUNK steps, and between blocks a product
    with the decays from block to block.  a, b: [n, T, H, d]; c: [n, T, H, e]."""
    n, T, H, _ = a.shape
    C = min(_CHUNK, T)
    m = -(-T // C)
    blocks = lambda x: torch.nn.functional.pad(x, (0, 0, 0, 0, 0, m * C - T)).reshape(n, m, C, H, -1).permute(0, 3, 1, 2, 4)  # noqa: E731
    a, b, c = blocks(a), blocks(b), blocks(c)  # [n, H, m, C, .]
    i = torch.arange(C, device=a.device, dtype=torch.float32)
    g = log_decay[:, None, None]
    within = torch.exp((i[:, None] - i).clamp_min(0) * g) * (i[:, None] >= i)
    y = torch.matmul(torch.matmul(a, b.transpose(-1, -2).contiguous()) * within[:, None], c)
    if m > 1:
        local = torch.matmul((b * torch.exp((C - 1 - i) * log_decay[:, None])[:, None, :, None]).transpose(-1, -2).contiguous(), c)
        u = torch.arange(m, device=a.device, dtype=torch.float32)
        steps = u[:, None] - 1 - u
        carried = torch.exp(steps.clamp_min(0) * C * g) * (steps >= 0)
        before = torch.matmul(carried, local.reshape(n, H, m, -1)).reshape(local.shape)
        y = y + torch.exp((i + 1) * log_decay[:, None])[:, None, :, None] * torch.matmul(a, before)
    return y.permute(0, 2, 3, 1, 4).reshape(n, m * C, H, -1)[:, :T]


def _run_attend(s):
    case = s["case"]
    n, H, G, g = case["seqs"], case["heads"], case["kv_heads"], s["log_decay"]
    q = _padded(s["q"], s, n)
    k, v = (_padded(s[x], s, n).repeat_interleave(H // G, dim=2) for x in "kv")
    T = q.shape[1]
    lengths = s["offsets"][1:] - s["offsets"][:-1] if s["offsets"] is not None else torch.full((n,), T, device=q.device)
    at = torch.arange(T, device=q.device)
    up = torch.exp((at + 1)[:, None] * g)[None, :, :, None]  # from the initial state to each token
    down = torch.exp((lengths[:, None] - 1 - at).clamp_min(0)[..., None] * g)[..., None]  # from each token to the final state
    heads = lambda x: x.transpose(1, 2)  # noqa: E731
    o = _decayed(q, k, v, g)
    last = torch.matmul(heads(k * down).transpose(-1, -2).contiguous(), heads(v))
    whole = torch.exp(lengths[:, None] * g)[..., None, None]
    if s["state"] is not None:
        o = o + up * heads(torch.matmul(heads(q), s["state"]))
        last = last + whole * s["state"]
    r = {"o": _packed(o, s, s["q"]), "state": last}
    if not case["grad"]:
        return r
    do = _padded(s["grad_o"], s, n)
    gq = _decayed(do, v, k, g)
    turned = [_turned(x, lengths) for x in (q, k, v, do)]
    gk = _turned(_decayed(turned[2], turned[3], turned[0], g), lengths)
    gv = _turned(_decayed(turned[1], turned[0], turned[3], g), lengths)
    if s["state"] is not None:
        ds = s["grad_state"]
        gq = gq + up * heads(torch.matmul(heads(do), s["state"].transpose(-1, -2).contiguous()))
        gk = gk + down * heads(torch.matmul(heads(v), ds.transpose(-1, -2).contiguous()))
        gv = gv + down * heads(torch.matmul(heads(k), ds))
        r["gstate"] = whole * ds + torch.matmul(heads(q * up).transpose(-1, -2).contiguous(), heads(do))
    shared = lambda x: x.reshape(n, T, G, H // G, -1).sum(3)  # noqa: E731
    return {**r, "gq": _packed(gq, s, s["q"]), "gk": _packed(shared(gk), s, s["k"]), "gv": _packed(shared(gv), s, s["v"])}


def _run_step(s):
    case = s["case"]
    q = s["q"].float()
    k, v = (s[x].float().repeat_interleave(case["heads"] // case["kv_heads"], dim=1) for x in "kv")
    state = torch.exp(s["log_decay"])[:, None, None] * s["state"] + k[..., None] * v[..., None, :]
    return {"o": (q[..., None] * state).sum(-2).to(s["q"].dtype), "state": state}


def _act(z, act):
    """The activation and its derivative."""
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return z * p, p * (1 + z * (1 - p))
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * p, p + z * torch.exp(-0.5 * z * z) * (0.5 / math.pi) ** 0.5
    return z, torch.ones_like(z)


def _run_norm(s):
    case, x = s["case"], s["x"].float()
    G = case["groups"]
    shape = (case["items"], case["length"], G, case["channels"] // G)
    w, b = (s[k].reshape(shape[2:]) for k in ("weight", "bias"))
    x = x.reshape(shape)
    mean = x.mean((1, 3), keepdim=True)
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).mean((1, 3), keepdim=True) + 1e-5)
    xhat = d * rstd
    y, dy = _act(xhat * w + b, case["act"])
    r = {"y": y.reshape(s["x"].shape).to(s["x"].dtype), "mean": mean.reshape(-1, G), "rstd": rstd.reshape(-1, G)}
    if case["grad"]:
        dz = s["grad_y"].float().reshape(shape) * dy
        dx = dz * w
        dx = rstd * (dx - dx.mean((1, 3), keepdim=True) - xhat * (dx * xhat).mean((1, 3), keepdim=True))
        r.update(gx=dx.reshape(s["x"].shape).to(s["x"].dtype), gweight=(dz * xhat).sum((0, 1)).reshape(-1), gbias=dz.sum((0, 1)).reshape(-1))
    return r


def _run_embed(s):
    case, valid = s["case"], (s["tokens"] >= 0)[:, None]
    at = s["tokens"].clamp_min(0)
    r = {"rows": (s["table"][at].float() * valid * s["scale"]).to(s["table"].dtype)}
    if case["grad"]:
        total = torch.zeros((case["vocab"], case["width"]), device=at.device)
        r["gtable"] = total.index_add_(0, at, s["grad"].float() * valid).mul_(s["scale"]).to(s["table"].dtype)
    return r


def run(s):
    if own:
        return _run_own(s)
    return {"step": _run_step, "attend": _run_attend, "norm": _run_norm, "embed": _run_embed}[s["case"]["path"]](s)


# ---- what a pass cannot do without

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["path"] in ("step", "attend"):
        H, G, dk, dv = case["heads"], case["kv_heads"], case["dk"], case["dv"]
        n, seqs = (case["batch"],) * 2 if case["path"] == "step" else (case["tokens"], case["seqs"])
        tensors = n * size * (H * dk + G * dk + G * dv)  # q, k, v or their gradients
        outs = n * size * H * dv
        states = 4 * seqs * H * dk * dv
        token = 4 * n * H * dk * dv  # state update and readout of each token: the recurrent form's operations
        if case["path"] == "step":
            return {"bytes": tensors + outs + 2 * states, "flops": token + states // 4}
        nbytes, flops = tensors + outs + states * (2 if case["state"] else 1), token
        if case["grad"]:
            nbytes += 2 * tensors + outs + (3 * states if case["state"] else 0)
            flops += 2 * token
        return {"bytes": nbytes, "flops": flops}
    if case["path"] == "norm":
        e = case["items"] * case["length"] * case["channels"]
        stats = 8 * case["items"] * case["groups"]
        if case["grad"]:
            return {"bytes": 5 * e * size + 2 * stats + 24 * case["channels"], "flops": 30 * e}
        return {"bytes": 2 * e * size + stats + 8 * case["channels"], "flops": 10 * e}
    rows, table = case["tokens"] * case["width"] * size, case["vocab"] * case["width"] * size
    if case["grad"]:
        return {"bytes": 3 * rows + table + 16 * case["tokens"], "flops": 3 * case["tokens"] * case["width"]}
    return {"bytes": 2 * rows + 8 * case["tokens"], "flops": case["tokens"] * case["width"]}


# ---- the definitions in 64 bits

def _exact_attend(case, s, seed):
    """Every pair (i, j) of each sequence, blocks of rows at a time."""
    H, G = case["heads"], case["kv_heads"]
    lengths = _lengths(case, seed)
    if sum(t * t for t in lengths) * H * (case["dk"] + case["dv"]) * (3 if case["grad"] else 1) > 2e13:
        return None
    per_head = lambda x: x.double().reshape((-1,) + x.shape[-2:]).transpose(0, 1).contiguous()  # noqa: E731
    q, k, v = per_head(s["q"]), per_head(s["k"]), per_head(s["v"])
    kv = torch.arange(H, device=q.device) // (H // G)
    g = s["log_decay"].double()
    do = per_head(s["grad_o"]) if case["grad"] else None
    o = torch.zeros(H, q.shape[1], v.shape[2], dtype=torch.float64, device=q.device)
    last = torch.zeros(len(lengths), H, q.shape[2], v.shape[2], dtype=torch.float64, device=q.device)
    gq, gk, gv, gs = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), torch.zeros_like(last)
    start = 0
    for b, T in enumerate(lengths):
        here = slice(start, start + T)
        kb, vb = k[kv, here], v[kv, here]
        age = torch.arange(T, device=q.device, dtype=torch.float64)
        to_end = torch.exp(g[:, None] * (T - 1 - age))
        last[b] = (kb * to_end[..., None]).transpose(1, 2).contiguous() @ vb
        if s["state"] is not None:
            first = s["state"][b].double()
            from_start = torch.exp(g[:, None] * (age + 1))
            end = torch.exp(g * T)[:, None, None]
            last[b] += end * first
            o[:, here] += from_start[..., None] * (q[:, here] @ first)
            if case["grad"]:
                ds = s["grad_state"][b].double()
                gs[b] = end * ds + (q[:, here] * from_start[..., None]).transpose(1, 2).contiguous() @ do[:, here]
                gq[:, here] += from_start[..., None] * (do[:, here] @ first.transpose(1, 2).contiguous())
                gk[:, here].index_add_(0, kv, to_end[..., None] * (vb @ ds.transpose(1, 2).contiguous()))
                gv[:, here].index_add_(0, kv, to_end[..., None] * (kb @ ds))
        step = max(64, min(4096, 10**8 // max(1, T * H)))
        for i in range(0, T, step):
            rows, cols = slice(start + i, start + min(T, i + step)), slice(start, start + min(T, i + step))
            kc, vc = k[kv, cols], v[kv, cols]
            gap = age[i:i + step, None] - age[:min(T, i + step)]
            w = torch.exp(g[:, None, None] * gap.clamp_min(0)).masked_fill_(gap < 0, 0)
            a = (q[:, rows] @ kc.transpose(1, 2).contiguous()).mul_(w)
            o[:, rows] += a @ vc
            if case["grad"]:
                c = (do[:, rows] @ vc.transpose(1, 2).contiguous()).mul_(w)
                gq[:, rows] += c @ kc
                gk[:, cols].index_add_(0, kv, c.transpose(1, 2).contiguous() @ q[:, rows])
                gv[:, cols].index_add_(0, kv, a.transpose(1, 2).contiguous() @ do[:, rows])
        start += T
    lead = s["q"].shape[:-2]
    back = lambda x: x.transpose(0, 1).reshape(lead + (x.shape[0], x.shape[2]))  # noqa: E731
    r = {"o": back(o), "state": last}
    if case["grad"]:
        r.update(gq=back(gq), gk=back(gk), gv=back(gv))
        if s["state"] is not None:
            r["gstate"] = gs
    return r


def exact(case, seed):
    s = prepare(case, seed)
    if case["path"] == "attend":
        return _exact_attend(case, s, seed)
    if case["path"] == "step":
        share = case["heads"] // case["kv_heads"]
        q, k, v = s["q"].double(), *(s[x].double().repeat_interleave(share, dim=1) for x in "kv")
        state = s["state"].double() * torch.exp(s["log_decay"].double())[None, :, None, None]
        state += k[:, :, :, None] * v[:, :, None, :]
        return {"o": (q[:, :, None, :] @ state)[:, :, 0], "state": state}
    if case["path"] == "norm":
        leaves = [s[x].double().requires_grad_(case["grad"]) for x in ("x", "weight", "bias")]
        x = leaves[0].reshape(case["items"], case["length"], case["groups"], -1).transpose(1, 2)
        mean = x.sum((2, 3)) / (x.shape[2] * x.shape[3])
        rstd = (((x - mean[..., None, None]) ** 2).sum((2, 3)) / (x.shape[2] * x.shape[3]) + 1e-5) ** -0.5
        z = ((x - mean[..., None, None]) * rstd[..., None, None]).transpose(1, 2).reshape(s["x"].shape) * leaves[1] + leaves[2]
        y = z if case["act"] == "none" else z * torch.sigmoid(z) if case["act"] == "silu" else z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
        r = {"y": y.detach(), "mean": mean.detach(), "rstd": rstd.detach()}
        if case["grad"]:
            r["gx"], r["gweight"], r["gbias"] = torch.autograd.grad(y, leaves, s["grad_y"].double())
        return r
    some = s["tokens"] >= 0
    rows = torch.zeros(case["tokens"], case["width"], dtype=torch.float64, device="cuda")
    rows[some] = s["table"][s["tokens"][some]].double() * s["scale"]
    r = {"rows": rows}
    if case["grad"]:
        r["gtable"] = torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device="cuda")
        r["gtable"].index_add_(0, s["tokens"][some], s["grad"][some].double() * s["scale"])
    return r
