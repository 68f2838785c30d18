"""The operators around the recurrence, as cases to be timed and compared: the short causal convolution, the selective
state space scan and the row normalisation, each forward, backward and (the first two) for single tokens.

With `own` the calls of this library are made, else the same operators in elementary torch operations in 32 bits
(prefix sums of the scan's decay in 64).  Formulas:

    convolution    u_t = bias + sum_j w[:, j] x_{t-W+1+j},  y = u or u sigmoid(u)
    scan           dt = softplus(raw + bias),  S_t = exp(dt A) S_{t-1} + dt x_t B_t^T,  y_t = S_t C_t + D x_t
    norm           y = ((x - mean) / sqrt(var + eps) w + b) (g sigmoid(g)); "rms": no mean, no b; without g: no factor
"""
import itertools
import math

import torch

own = False

EPS = 1e-5


def _conv(way, batch, tokens, channels, width, dtype="bf16", silu=True, state=True, packed=False, name=None):
    """way: "train" (forward and backward), "prompt" (forward) or "step"; packed: `tokens` in all, in `batch` sequences."""
    c = dict(op="conv", way=way, batch=batch, tokens=tokens, channels=channels, width=width, dtype=dtype, silu=silu,
             state=state, packed=packed)
    return dict(c, name=name) if name else c


def _scan(way, batch, tokens, heads, groups, dp, dn, dtype="bf16", state=True, skip=True, packed=False, name=None):
    c = dict(op="scan", way=way, batch=batch, tokens=tokens, heads=heads, groups=groups, dp=dp, dn=dn, dtype=dtype,
             state=state, skip=skip, packed=packed)
    return dict(c, name=name) if name else c


def _norm(way, rows, size, kind, dtype="bf16", gate=False, name=None):
    c = dict(op="norm", way=way, rows=rows, size=size, kind=kind, dtype=dtype, gate=gate)
    return dict(c, name=name) if name else c


def listed():
    return [
        # training: the convolution over q, k and v of a layer with 16 heads of 128, model width 2048
        _conv("train", 4, 4096, 6144, 4, name="conv_train_bf16"),
        # training in fp32 on a packed batch of short documents, odd channels
        _conv("train", 9, 2003, 1001, 3, "f32", packed=True, name="conv_packed_f32"),
        # one decode step of a serving batch
        _conv("step", 64, 1, 6144, 4, name="conv_step"),
        # training: heads of 64 over a state of 128, one group, as a layer of model width 2048 expanded twice has them
        _scan("train", 4, 4096, 64, 1, 64, 128, name="scan_train_bf16"),
        # training in fp32 on ragged packed documents, two groups of heads
        _scan("train", 7, 3001, 8, 2, 64, 64, "f32", packed=True, name="scan_packed_f32"),
        # prefill of one long document over few heads
        _scan("prompt", 1, 65536, 16, 1, 128, 128, name="scan_long_bf16"),
        # the smallest prompt: launches and latency
        _scan("prompt", 1, 256, 2, 1, 64, 64, "f32", state=False, skip=False, name="scan_tiny_f32"),
        # one decode step of a serving batch
        _scan("step", 64, 1, 64, 1, 64, 128, name="scan_step_batch"),
        # one decode step of a single request
        _scan("step", 1, 1, 64, 1, 64, 128, name="scan_step_single"),
        # training: the norm before a layer
        _norm("train", 16384, 2048, "layer", name="norm_layer_bf16"),
        # training: the gated norm over each head's output
        _norm("train", 262144, 128, "rms", gate=True, name="norm_gated_heads_bf16"),
        # fp32 rows that no vector divides
        _norm("train", 777, 1003, "layer", "f32", name="norm_ragged_f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f32"])
    op = rng.choice(["conv", "scan", "scan", "norm"])
    if op == "norm":
        size = rng.choice([64, 128, 256, _log(rng, 64, 8192), _log(rng, 64, 1024) * 8])
        rows = max(1, min(_log(rng, 1, 1 << 18), (1 << 25) // size))
        return _norm(rng.choice(["train", "prompt"]), rows, size, rng.choice(["layer", "rms"]), dtype, rng.random() < 0.5)
    way = rng.choice(["train", "train", "prompt", "step"])
    batch, packed, state = rng.randint(1, 16), rng.random() < 0.4, rng.random() < 0.7
    if way == "step":
        batch, tokens, packed, state = _log(rng, 1, 256), 1, False, True
    if op == "conv":
        channels = rng.choice([_log(rng, 64, 1024) * 8, _log(rng, 65, 4099)])
        if way != "step":
            total = min(_log(rng, 16, 1 << 16), (1 << 26) // channels)
            tokens = max(total, batch) if packed else max(1, total // batch)
        return _conv(way, batch, tokens, channels, rng.randint(2, 4), dtype, rng.random() < 0.7, state, packed)
    groups = rng.choice([1, 1, 2, 4])
    heads = groups * rng.choice([1, 2, 3, 4, 8, 16])
    dp, dn = rng.choice([32, 64, 64, 128]), rng.choice([16, 32, 64, 128])
    if way == "step":
        batch = max(1, min(batch, (1 << 25) // (heads * dp * dn)))
    else:
        total = min(_log(rng, 16, 1 << 16), (1 << 25) // (heads * dp))
        tokens = max(total, batch) if packed else max(1, total // batch)
    return _scan(way, batch, tokens, heads, groups, dp, dn, dtype, state, rng.random() < 0.7, packed)


# ------------------------------------------------------------------------------------------------------------- inputs

def _lengths(tokens, n, rng):
    """n sequence lengths of at least one token that add up to `tokens`, spread over their logarithm."""
    w = torch.exp(torch.randn(n, generator=rng)) + 1e-3
    extra = torch.floor(w / w.sum() * (tokens - n)).long()
    extra[0] += tokens - n - extra.sum()
    return (extra + 1).tolist()


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")                       # noqa: E731
    un = lambda *s: torch.rand(s, generator=g, device="cuda")                        # noqa: E731
    act = lambda *s: torch.nn.functional.silu(rn(*s)).to(t)                          # noqa: E731
    st = dict(case=case)
    if case["op"] == "norm":
        r, d = case["rows"], case["size"]
        st.update(x=(rn(r, d) * 1.5 + 0.3).to(t), w=(1 + 0.1 * rn(d)).to(t),
                  b=(0.1 * rn(d)).to(t) if case["kind"] == "layer" else None,
                  g=rn(r, d).to(t) if case["gate"] else None, dy=rn(r, d).to(t))
        return st
    n, T = case["batch"], case["tokens"]
    lead = (n,) if case["way"] == "step" else (1, T) if case["packed"] else (n, T)
    st["cu"] = st["plan"] = None
    if case["packed"]:
        lens = _lengths(T, n, torch.Generator().manual_seed(seed))
        cu = list(itertools.accumulate(lens, initial=0))
        st["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
        longest = max(lens)
        at = torch.arange(longest).unsqueeze(0) + torch.tensor(cu[:-1]).unsqueeze(1)     # token of (sequence, position)
        real = torch.arange(longest).unsqueeze(0) < torch.tensor(lens).unsqueeze(1)
        st["plan"] = dict(at=at.clamp(max=T - 1).cuda(), real=real.cuda(), lens=torch.tensor(lens).cuda(),
                          back=torch.nonzero(real.reshape(-1)).squeeze(1).cuda())
    if case["op"] == "conv":
        d, w = case["channels"], case["width"]
        st.update(x=rn(*lead, d).to(t), w=(rn(d, w) / math.sqrt(w)).to(t), b=(0.1 * rn(d)).to(t),
                  s0=rn(n, w - 1, d).to(t) if case["state"] else None, dy=rn(*lead, d).to(t),
                  dsf=rn(n, w - 1, d).to(t) if case["state"] else None)
        return st
    h, gr, p, m = case["heads"], case["groups"], case["dp"], case["dn"]
    step = torch.exp(math.log(1e-3) + (math.log(0.1) - math.log(1e-3)) * un(h))          # time steps of 0.001 to 0.1
    st.update(x=act(*lead, h, p), dt=rn(*lead, h), A=-(1 + 15 * un(h)), B=act(*lead, gr, m), C=act(*lead, gr, m),
              D=1 + 0.1 * rn(h) if case["skip"] else None, bias=step + torch.log(-torch.expm1(-step)),
              s0=0.3 * rn(n, h, p, m) if case["state"] else None, dy=rn(*lead, h, p).to(t),
              dsf=0.1 * rn(n, h, p, m) if case["state"] else None)
    return st


# --------------------------------------------------------------------------------------------------------- plain forms

def _silu(u):
    return u / (1 + torch.exp(-u))


def _softplus(z):
    return torch.clamp(z, min=0) + torch.log1p(torch.exp(-torch.abs(z)))


def _spread(x, plan):
    """A packed batch [1, T, ...] as sequences padded with zeros."""
    if plan is None:
        return x
    y = x[0][plan["at"]]
    return y * plan["real"].reshape(plan["real"].shape + (1,) * (y.dim() - 2))


def _joined(y, plan):
    return y if plan is None else y.flatten(0, 1)[plan["back"]].unsqueeze(0)


def _plain_conv(x, w, b, s0, plan, silu):
    x = _spread(x, plan)
    n, T, d = x.shape
    W = w.shape[1]
    before = s0 if s0 is not None else torch.zeros(n, W - 1, d, device=x.device)
    ext = torch.cat([before, x], 1)
    u = b + sum(ext[:, j:j + T] * w[:, j] for j in range(W))
    lens = plan["lens"] if plan is not None else torch.full((n,), T, device=x.device)
    last = lens.unsqueeze(1) + torch.arange(W - 1, device=x.device)
    final = torch.gather(ext, 1, last.unsqueeze(2).expand(-1, -1, d))
    return _joined(_silu(u) if silu else u, plan), final


def _plain_scan(x, raw, A, B, C, D, bias, s0, plan, chunk=64):
    x, raw, B, C = (_spread(t, plan) for t in (x, raw, B, C))
    n, T, h, p = x.shape
    g, m = B.shape[2:]
    dt = _softplus(raw + bias)
    if plan is not None:
        dt = dt * plan["real"].unsqueeze(2)
    c = -(-T // chunk)
    fill = c * chunk - T
    cut = lambda t: torch.cat([t, t.new_zeros((n, fill) + t.shape[2:])], 1).reshape((n, c, chunk) + t.shape[2:])  # noqa: E731
    xc, dtc = cut(x).permute(0, 1, 3, 2, 4).contiguous(), cut(dt).permute(0, 1, 3, 2)      # [n c h q p], [n c h q]
    Bc, Cc = cut(B).permute(0, 1, 3, 2, 4).contiguous(), cut(C).permute(0, 1, 3, 2, 4).contiguous()   # [n c g q m]
    b = torch.cumsum((dtc.double() * A.double().unsqueeze(1)), 3)                          # in 64 bits: differences
    diff = b.unsqueeze(4) - b.unsqueeze(3)
    lower = torch.ones(chunk, chunk, dtype=torch.bool, device=x.device).tril()
    weight = torch.exp(diff.masked_fill(~lower, -math.inf)).float()                        # [n c h q q]
    per = h // g
    heads = lambda t: t.unsqueeze(3).expand(-1, -1, -1, per, -1, -1).reshape((n, c, h) + t.shape[3:])     # noqa: E731
    score = heads(torch.matmul(Cc, Bc.transpose(3, 4).contiguous()))
    dx = dtc.unsqueeze(4) * xc
    y = torch.matmul(weight * score, dx)
    Bh, Ch = heads(Bc), heads(Cc)
    tail = torch.exp(b[..., -1:] - b).float()
    add = torch.matmul((dx * tail.unsqueeze(4)).transpose(3, 4).contiguous(), Bh)          # [n c h p m]
    first = s0 if s0 is not None else torch.zeros(n, h, p, m, device=x.device)
    states = torch.cat([first.unsqueeze(1), add], 1).permute(0, 2, 1, 3, 4).reshape(n, h, c + 1, p * m)
    total = torch.cumsum(torch.cat([b.new_zeros(n, 1, h), b[..., -1]], 1), 1).permute(0, 2, 1)             # [n h c+1]
    low = torch.ones(c + 1, c + 1, dtype=torch.bool, device=x.device).tril()
    carry = torch.exp((total.unsqueeze(3) - total.unsqueeze(2)).masked_fill(~low, -math.inf)).float()
    entry = torch.matmul(carry, states).reshape(n, h, c + 1, p, m).permute(0, 2, 1, 3, 4)
    y = y + torch.exp(b).float().unsqueeze(4) * torch.matmul(Ch, entry[:, :-1].transpose(3, 4).contiguous())
    y = y.permute(0, 1, 3, 2, 4).reshape(n, c * chunk, h, p)[:, :T]
    if D is not None:
        y = y + D.unsqueeze(1) * x
    return _joined(y, plan), entry[:, -1]


def _plain_norm(x, w, b, g):
    if b is not None:                                   # "layer"
        x = x - x.mean(1, keepdim=True)
    y = x / torch.sqrt((x * x).mean(1, keepdim=True) + EPS) * w
    if b is not None:
        y = y + b
    return y if g is None else y * _silu(g)


def _grads(outs, back, leaves):
    """Gradients of the leaves (None kept) for the outputs' gradients."""
    keep = [i for i, v in enumerate(leaves) if v is not None]
    pairs = [(o, d) for o, d in zip(outs, back) if d is not None]
    got = torch.autograd.grad([o for o, _ in pairs], [leaves[i] for i in keep], [d.float() for _, d in pairs])
    full = dict(zip(keep, got))
    return [full.get(i) for i in range(len(leaves))]


def _leaf(t, train):
    return None if t is None else t.detach().float().requires_grad_(train)


def _as(t, like):
    return None if t is None else t.detach().to(like.dtype)


def _plain_step(s):
    """One token from the state: (outputs, state after it)."""
    if s["case"]["op"] == "conv":
        ext = torch.cat([s["s0"], s["x"].unsqueeze(1)], 1).float()                         # [n W d]
        u = (ext * s["w"].float().t()).sum(1) + s["b"].float()
        return _silu(u) if s["case"]["silu"] else u, ext[:, 1:]
    x, per = s["x"].float(), s["x"].shape[1] // s["B"].shape[1]
    B, C = (s[k].float().repeat_interleave(per, 1) for k in ("B", "C"))
    dt = _softplus(s["dt"] + s["bias"])
    S = torch.exp(dt * s["A"])[..., None, None] * s["s0"] + (dt.unsqueeze(2) * x).unsqueeze(3) * B.unsqueeze(2)
    y = (S * C.unsqueeze(2)).sum(3)
    return y + s["D"].unsqueeze(1) * x if s["D"] is not None else y, S


def _run_plain(s):
    case = s["case"]
    if case["way"] == "step":
        y, after = _plain_step(s)
        return dict(y=_as(y, s["x"]), state=_as(after, s["s0"]))
    train = case["way"] == "train"
    if case["op"] == "norm":
        names = ("x", "w", "b", "g")
        leaves = [_leaf(s[k], train) for k in names]
        outs = (_plain_norm(*leaves),)
        res, back = dict(y=_as(outs[0], s["x"])), (s["dy"],)
    elif case["op"] == "conv":
        names = ("x", "w", "b", "s0")
        leaves = [_leaf(s[k], train) for k in names]
        outs = _plain_conv(*leaves, s["plan"], case["silu"])
        res, back = dict(y=_as(outs[0], s["x"]), state=_as(outs[1], s["x"])), (s["dy"], s["dsf"])
    else:
        names = ("x", "dt", "A", "B", "C", "D", "bias", "s0")
        leaves = [_leaf(s[k], train) for k in names]
        outs = _plain_scan(*leaves, s["plan"])
        res, back = dict(y=_as(outs[0], s["x"]), state=outs[1].detach()), (s["dy"], s["dsf"])
    if train:
        for k, d in zip(names, _grads(outs, back, leaves)):
            if d is not None:
                res["d" + k] = _as(d, s[k])
    return res


# ------------------------------------------------------------------------------------------------------------ own calls

def _run_own(s):
    from paper_2606_08804_amd import mixer
    case = s["case"]
    if case["op"] == "norm":
        y, stats = mixer.norm_fwd(s["x"], s["w"], s["b"], s["g"], eps=EPS, kind=case["kind"])
        res = dict(y=y)
        if case["way"] == "train":
            d = mixer.norm_bwd(s["x"], s["w"], s["b"], s["g"], stats, s["dy"], kind=case["kind"])
            res.update(dx=d["dx"], dw=d["dweight"], db=d["dbias"], dg=d["dgate"])
        return {k: v for k, v in res.items() if v is not None}
    if case["op"] == "conv":
        act = "silu" if case["silu"] else None
        if case["way"] == "step":
            state = torch.empty_like(s["s0"])
            y = mixer.conv_step(s["x"], s["w"], s["b"], s["s0"], activation=act, state_out=state)
            return dict(y=y, state=state)
        y, state = mixer.conv_fwd(s["x"], s["w"], s["b"], s["s0"], cu_seqlens=s["cu"], activation=act)
        res = dict(y=y, state=state)
        if case["way"] == "train":
            d = mixer.conv_bwd(s["x"], s["w"], s["b"], s["s0"], s["dy"], s["dsf"], cu_seqlens=s["cu"], activation=act,
                               need_d_initial_state=case["state"])
            res.update(dx=d["dx"], dw=d["dweight"], db=d["dbias"], ds0=d["d_initial_state"])
        return {k: v for k, v in res.items() if v is not None}
    if case["way"] == "step":
        state = torch.empty_like(s["s0"])
        y = mixer.scan_step(s["x"], s["dt"], s["A"], s["B"], s["C"], s["s0"], s["D"], s["bias"], softplus=True,
                            state_out=state)
        return dict(y=y, state=state)
    y, state = mixer.scan_fwd(s["x"], s["dt"], s["A"], s["B"], s["C"], s["D"], s["bias"], s["s0"], cu_seqlens=s["cu"],
                              softplus=True)
    res = dict(y=y, state=state)
    if case["way"] == "train":
        d = mixer.scan_bwd(s["x"], s["dt"], s["A"], s["B"], s["C"], s["D"], s["bias"], s["s0"], s["dy"], s["dsf"],
                           cu_seqlens=s["cu"], softplus=True, need_d_initial_state=case["state"])
        res.update(dx=d["dx"], ddt=d["ddt"], dA=d["dA"], dB=d["dB"], dC=d["dC"], dD=d["dD"], dbias=d["ddt_bias"],
                   ds0=d["d_initial_state"])
    return {k: v for k, v in res.items() if v is not None}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# --------------------------------------------------------------------------------------------------------------- work

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    train = case["way"] == "train"
    if case["op"] == "norm":
        n = case["rows"] * case["size"]
        # x (and the gate) in, y out; backward: dy in, dx (and the gate's gradient) out
        tensors = (2 + case["gate"]) * (2 if train else 1)
        return {"bytes": n * e * tensors, "flops": n * (8 + 6 * case["gate"]) * (3 if train else 1)}
    tokens = case["tokens"] if case["packed"] else case["batch"] * case["tokens"]
    seqs = case["batch"]
    if case["op"] == "conv":
        n, w = tokens * case["channels"], case["width"]
        state = seqs * (w - 1) * case["channels"] * e * ((2 if train else 1) * case["state"] + 1 + (train and case["state"]))
        return {"bytes": n * e * (4 if train else 2) + state, "flops": n * (2 * w + 5 * case["silu"]) * (3 if train else 1)}
    h, g, p, m = case["heads"], case["groups"], case["dp"], case["dn"]
    x, bc, dt, S = tokens * h * p * e, 2 * tokens * g * m * e, tokens * h * 4, seqs * h * p * m * 4
    if train:
        # x, dy, y, dx; B, C and their gradients; dt and its gradient; states and their gradients
        return {"bytes": 4 * x + 2 * bc + 2 * dt + (1 + 3 * case["state"]) * S, "flops": tokens * h * p * m * 5 * 3}
    # the recurrence: decay, update and readout of every state element a token
    return {"bytes": 2 * x + bc + dt + (1 + case["state"]) * S, "flops": tokens * h * p * m * 5}


# --------------------------------------------------------------------------------- the definitions in 64 bits, by token

def _exact_norm(s, train):
    f = lambda t: None if t is None else t.double()                                  # noqa: E731
    x, w, b, g = f(s["x"]), f(s["w"]), f(s["b"]), f(s["g"])
    n = x.shape[1]
    mean = x.sum(1, keepdim=True) / n if b is not None else torch.zeros_like(x[:, :1])
    r = ((x - mean).square().sum(1, keepdim=True) / n + EPS).rsqrt()
    xh = (x - mean) * r
    lin = xh * w + (b if b is not None else 0)
    sg = torch.sigmoid(g) if g is not None else None
    res = dict(y=lin if g is None else lin * g * sg)
    if train:
        dy = f(s["dy"])
        dlin = dy if g is None else dy * g * sg
        res["dw"] = (dlin * xh).sum(0)
        if b is not None:
            res["db"] = dlin.sum(0)
        if g is not None:
            res["dg"] = dy * lin * sg * (1 + g * (1 - sg))
        d = dlin * w
        centre = d.sum(1, keepdim=True) / n if b is not None else 0
        res["dx"] = r * (d - centre - xh * (d * xh).sum(1, keepdim=True) / n)
    return res


def _sequences(s):
    """[(sequence, its tokens' place in the first two dimensions)]."""
    if s["cu"] is None:
        return [(i, (i, slice(None))) for i in range(s["x"].shape[0])]
    cu = s["cu"].tolist()
    return [(i, (0, slice(cu[i], cu[i + 1]))) for i in range(len(cu) - 1)]


def _exact_conv(s, case):
    f = lambda t: t.double()                                                         # noqa: E731
    w, b, W, train = f(s["w"]), f(s["b"]), case["width"], case["way"] == "train"
    if case["way"] == "step":
        ext = torch.cat([f(s["s0"]), f(s["x"]).unsqueeze(1)], 1)
        u = b + torch.einsum("nwd,dw->nd", ext, w)
        return dict(y=u * torch.sigmoid(u) if case["silu"] else u, state=ext[:, 1:])
    x = f(s["x"])
    y, state = torch.empty_like(x), torch.zeros(case["batch"], W - 1, x.shape[2], dtype=x.dtype, device=x.device)
    dx, dw, db, ds0 = torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(b), torch.zeros_like(state)
    for i, at in _sequences(s):
        xs = x[at]
        T = xs.shape[0]
        ext = torch.cat([f(s["s0"][i]) if s["s0"] is not None else torch.zeros_like(state[i]), xs])
        u = b.expand(T, -1).clone()
        for j in range(W):
            u += w[:, j] * ext[j:j + T]
        sg = torch.sigmoid(u)
        y[at] = u * sg if case["silu"] else u
        state[i] = ext[T:]
        if train:
            du = f(s["dy"])[at]
            if case["silu"]:
                du = du * (sg + u * sg * (1 - sg))
            dext = torch.zeros_like(ext)
            if s["dsf"] is not None:
                dext[T:] += f(s["dsf"][i])
            for j in range(W):
                dext[j:j + T] += w[:, j] * du
                dw[:, j] += (du * ext[j:j + T]).sum(0)
            db += du.sum(0)
            dx[at], ds0[i] = dext[W - 1:], dext[:W - 1]
    res = dict(y=y, state=state)
    if train:
        res.update(dx=dx, dw=dw, db=db)
        if s["s0"] is not None:
            res["ds0"] = ds0
    return res


def _exact_scan(s, case):
    """Token by token; sequences side by side, each put at the front of its row."""
    f = lambda t: t.double()                                                         # noqa: E731
    step, train = case["way"] == "step", case["way"] == "train"
    rows = (lambda t: f(t).unsqueeze(1)) if step else \
        (lambda t: torch.nn.utils.rnn.pad_sequence([f(t[at]) for _, at in _sequences(s)], batch_first=True))
    x, raw, B, C = (rows(s[k]) for k in ("x", "dt", "B", "C"))
    n, T, h, p = x.shape
    per, m = h // B.shape[2], B.shape[3]
    lens = torch.tensor([1] * n if step else [s["x"][at].shape[0] for _, at in _sequences(s)], device=x.device)
    there = (torch.arange(T, device=x.device) < lens.unsqueeze(1)).double()                # [n, T]
    z = raw + f(s["bias"])
    dt = torch.nn.functional.softplus(z, threshold=1e9) * there.unsqueeze(2)
    A, D = f(s["A"]), None if s["D"] is None else f(s["D"])
    a = torch.exp(dt * A)
    wide = lambda t: t.repeat_interleave(per, 1)                                     # noqa: E731
    S = f(s["s0"]).clone() if s["s0"] is not None else torch.zeros(n, h, p, m, dtype=x.dtype, device=x.device)
    y = torch.empty_like(x)
    every, kept = 64, []

    def advance(S, t):
        S = S * a[:, t, :, None, None]
        return S.addcmul_((dt[:, t].unsqueeze(2) * x[:, t]).unsqueeze(3), wide(B[:, t]).unsqueeze(2))

    for t in range(T):
        if train and t % every == 0:
            kept.append(S)
        S = advance(S, t)
        y[:, t] = torch.matmul(S, wide(C[:, t]).unsqueeze(3)).squeeze(3)
        if D is not None:
            y[:, t] += D.unsqueeze(1) * x[:, t]
    res = dict(y=y, state=S)
    if train:
        dy = rows(s["dy"])
        G = f(s["dsf"]).clone() if s["dsf"] is not None else torch.zeros_like(S)           # dL/dS_t
        dx, dd, dB, dC = torch.zeros_like(x), torch.zeros_like(dt), torch.zeros_like(B), torch.zeros_like(C)
        dA = torch.zeros_like(A)
        for c in reversed(range(len(kept))):
            t0, t1 = c * every, min((c + 1) * every, T)
            inner = [kept[c]]
            for t in range(t0, t1):
                inner.append(advance(inner[-1], t))
            for t in reversed(range(t0, t1)):
                Sp, St, gy = inner[t - t0], inner[t - t0 + 1], dy[:, t]
                dC[:, t] = torch.matmul(gy.unsqueeze(2), St).reshape(n, -1, per, m).sum(2)
                G = G.addcmul(gy.unsqueeze(3), wide(C[:, t]).unsqueeze(2))
                gb = torch.matmul(G, wide(B[:, t]).unsqueeze(3)).squeeze(3)
                dx[:, t] = dt[:, t].unsqueeze(2) * gb
                dB[:, t] = (dt[:, t].unsqueeze(2) * torch.matmul(x[:, t].unsqueeze(2), G).squeeze(2)).reshape(n, -1, per, m).sum(2)
                dl = (G * Sp).sum((2, 3)) * a[:, t]
                dd[:, t] = (gb * x[:, t]).sum(2) + A * dl
                dA += (dt[:, t] * dl).sum(0)
                G = G * a[:, t, :, None, None]
            kept[c] = None
        if D is not None:
            dx += D.unsqueeze(1) * dy
            res["dD"] = (dy * x).sum((0, 1, 3))
        dd = dd * torch.sigmoid(z) * there.unsqueeze(2)
        res.update(dx=dx, ddt=dd, dA=dA, dB=dB, dC=dC, dbias=dd.sum((0, 1)))
        if s["s0"] is not None:
            res["ds0"] = G
    if step:
        res["y"] = y.squeeze(1)
    elif s["cu"] is not None:
        flat = there.reshape(-1).nonzero().squeeze(1)
        for k in ("y", "dx", "ddt", "dB", "dC"):
            if k in res:
                res[k] = res[k].flatten(0, 1)[flat].unsqueeze(0)
    return res


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        res = _exact_norm(s, case["way"] == "train")
    elif case["op"] == "conv":
        res = _exact_conv(s, case)
    else:
        if case["tokens"] * (3 if case["way"] == "train" else 1) > 1.5e5:
            return None                                 # a loop over so many tokens takes too long
        res = _exact_scan(s, case)
    order = ("y", "state", "dx", "dw", "db", "dg", "ddt", "dA", "dB", "dC", "dD", "dbias", "ds0")
    return {k: res[k] for k in order if k in res}
