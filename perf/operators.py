"""Cases that the speed and the outputs of the operators around linear attention with a decay are judged on.

A case is one call of a user's program at one set of sizes.  `op` says which:

  decay     linear attention with a decay for each head, S_t = g S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t: prompts of
            N rows, or single tokens (N = 1) that are read against a state and added to it
  decay_bw  its gradients with respect to Q, K, V, the first state and the logarithm of the decays
  rotary    rotary positions applied to queries and keys
  norm      layer norm over groups of columns, with the statistics that its gradient needs
  norm_bw   its gradients with respect to input, weight and bias

B users, N rows per (padded) sequence, H heads of Q, Hkv heads of K and V (each shared by H / Hkv heads), D columns per head.
`ragged` draws the valid lengths from [0, N] (one user has all N rows, and with more than two users one has none) and fills the
rows past them with garbage; outputs are zero there.  For the norms `rows` rows hold `groups` groups of `d` columns.
Where `own` is false, `run` is the plain form of each operator in elementary torch operations.
"""
import math

import torch

own = False

F32, BF16 = "f32", "bf16"
_DT = {F32: torch.float32, BF16: torch.bfloat16}
_CHUNK = 128


def _decay(B, N, H, Hkv, D, dtype, name=None, op="decay", ragged=False, packed=False, state=True):
    c = dict(op=op, B=B, N=N, H=H, Hkv=Hkv, D=D, dtype=dtype, ragged=ragged, packed=packed, state=state)
    return dict(c, name=name) if name else c


def _rotary(B, N, H, Hkv, D, rot, dtype, name=None, interleaved=False, far=0, scaled=False):
    c = dict(op="rotary", B=B, N=N, H=H, Hkv=Hkv, D=D, rot=rot, dtype=dtype, interleaved=interleaved, far=far,
             scaled=scaled)
    return dict(c, name=name) if name else c


def _norm(rows, groups, d, dtype, name=None, op="norm"):
    c = dict(op=op, rows=rows, groups=groups, d=d, dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's next behaviour: a single token against a small state, where latency counts
        _decay(1, 1, 4, 4, 64, BF16, "step-one"),
        # a serving batch of single tokens: the states are read and written once
        _decay(128, 1, 16, 16, 128, BF16, "step-batch"),
        # the histories of the headline batch, one head of the full width: ten thousand rows, few heads
        _decay(64, 10000, 1, 1, 128, BF16, "prompt-history"),
        # float histories that fit no tile, keys and values shared by two heads
        _decay(12, 3001, 4, 2, 64, F32, "prompt-odd-ragged", ragged=True),
        # one long history of a model with heads, cut from one packed projection
        _decay(1, 65536, 16, 4, 128, BF16, "prompt-long", packed=True),
        # a training batch
        _decay(8, 4096, 16, 16, 128, BF16, "train", op="decay_bw", state=False),
        # a small float training batch of odd lengths with shared keys
        _decay(3, 1777, 6, 2, 64, F32, "train-odd-f32", op="decay_bw", ragged=True),
        # positions of one user's next token
        _rotary(1, 1, 4, 4, 64, 64, BF16, "positions-one", far=10000),
        # positions of a training batch, half of each head rotated, frequencies scaled for long contexts
        _rotary(8, 8192, 32, 8, 128, 64, BF16, "positions-batch", scaled=True),
        # output of the heads of a batch, normalised head by head
        _norm(65536, 16, 128, BF16, "norm-heads"),
        # hidden rows of a training batch
        _norm(32768, 1, 4096, BF16, "norm-train", op="norm_bw"),
        # a float layer whose width fits no vector
        _norm(3001, 1, 333, F32, "norm-odd-f32", op="norm_bw"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case: every size over the logarithm of its range, work no larger than the largest listed."""
    top = work(listed()[4])["bytes"]
    while True:
        op = rng.choice(["decay", "decay", "decay", "decay_bw", "decay_bw", "rotary", "norm", "norm_bw"])
        dtype = rng.choice([BF16, BF16, F32])
        if op in ("norm", "norm_bw"):
            groups = rng.choice([1, 1, rng.randint(2, 32)])
            d = rng.choice([64, 128, 256, _log_uniform(rng, 33, 1000)]) if groups > 1 else _log_uniform(rng, 64, 8192)
            if rng.random() < 0.6:
                d = max(8, d // 8 * 8)
            c = _norm(_log_uniform(rng, 1, 65536), groups, d, dtype, op=op)
        else:
            D = rng.choice([64, 128, 128, 256])
            Hkv = rng.choice([1, 2, 3, 4, 8])
            H = Hkv * rng.choice([1, 1, 2, 4])
            B = _log_uniform(rng, 1, 64)
            N = 1 if op == "decay" and rng.random() < 0.3 else _log_uniform(rng, 2, 32768)
            if op == "rotary":
                rot = rng.choice([D, D, D // 2, D // 4, 2 * rng.randint(1, D // 2)])
                c = _rotary(B, N, H, Hkv, D, rot, dtype, interleaved=rng.random() < 0.5,
                            far=rng.choice([0, 0, 100000, 2000000]), scaled=rng.random() < 0.3)
            else:
                c = _decay(B, N, H, Hkv, D, dtype, op=op, ragged=rng.random() < 0.5,
                           packed=op == "decay" and rng.random() < 0.4, state=rng.random() < 0.6)
        if work(c)["bytes"] <= (top if op in ("decay", "rotary", "norm") else top / 2):
            return c


def _scale(c):
    return c["D"] ** -0.5


def prepare(case, seed):
    """Inputs on the GPU, and the output buffers and workspace that a program keeps."""
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DT[c["dtype"]]
    s = {"case": c}

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def empty(*shape, dtype=torch.float32):
        return torch.zeros(*shape, dtype=dtype, device="cuda")

    if c["op"] in ("norm", "norm_bw"):
        R, G, d = c["rows"], c["groups"], c["d"]
        # rows of different size and with a mean, as hidden rows have
        x = randn(R, G, d) * (0.5 + 2 * torch.rand(R, G, 1, generator=gen, device="cuda")) + 0.5 * randn(R, G, 1)
        s["x"] = x.to(dt)
        s["weight"], s["bias"] = 1 + 0.2 * randn(G, d), 0.2 * randn(G, d)
        s["eps"] = 1e-5
        s["y"], s["mean"], s["rstd"] = empty(R, G, d, dtype=dt), empty(R, G), empty(R, G)
        if c["op"] == "norm_bw":
            v = s["x"].double()
            s["mean"] = v.mean(-1).float()
            s["rstd"] = (v.var(-1, unbiased=False) + s["eps"]).rsqrt().float()
            s["dy"] = randn(R, G, d).to(dt)
            s["dx"], s["dweight"], s["dbias"] = empty(R, G, d, dtype=dt), empty(G, d), empty(G, d)
            if own:
                from paper_2603_02561_amd import binding as sb
                s["workspace"] = torch.empty(max(256, sb.solar_layer_norm_workspace_bytes(R, G, d)), dtype=torch.uint8,
                                             device="cuda")
        return s

    B, N, H, Hkv, D = c["B"], c["N"], c["H"], c["Hkv"], c["D"]
    if c["op"] == "rotary":
        rot = c["rot"]
        s["q"], s["k"] = randn(B, N, H, D).to(dt), randn(B, N, Hkv, D).to(dt)
        s["freq"] = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
        s["amplitude"] = 1.0
        if c["scaled"]:
            # positions beyond the trained range: slow frequencies by a quarter, a slightly larger amplitude
            s["freq"] = torch.where(s["freq"] < 0.01, s["freq"] / 4, s["freq"])
            s["amplitude"] = 1.1386
        s["positions"] = None
        if c["far"]:
            first = torch.randint(0, c["far"], (B, 1), generator=gen, device="cuda")
            s["positions"] = (first + torch.arange(N, device="cuda")[None, :]).to(torch.int32)
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        return s

    if c["packed"]:
        # views of one projection's output [B, N, (H + 2 Hkv) D]
        z = randn(B, N, H + 2 * Hkv, D).to(dt)
        s["q"], s["k"], s["v"] = z[:, :, :H], z[:, :, H:H + Hkv], z[:, :, H + Hkv:]
    else:
        s["q"], s["k"], s["v"] = (randn(B, N, h, D).to(dt) for h in (H, Hkv, Hkv))
    # half-lives from a few rows to some thousands, as heads of one layer have them
    p = torch.linspace(3, 11, H, dtype=torch.float64, device="cuda") if H > 1 else torch.tensor([7.0], device="cuda").double()
    s["log_decay"] = torch.log1p(-(2.0 ** -(p + 0.25 * randn(H).double().abs()))).float()
    s["lengths"] = None
    if c["ragged"]:
        n = torch.randint(0, N + 1, (B,), generator=gen, device="cuda").to(torch.int32)
        n[0] = N
        if B > 2:
            n[B // 2] = 0
        s["lengths"] = n
        past = (torch.arange(N, device="cuda")[None, :] >= n[:, None])[:, :, None, None]
        for name in ("q", "k", "v"):
            s[name].copy_(torch.where(past, 1 + 3 * randn(*s[name].shape).to(dt), s[name]))
    s["state_in"] = randn(B, H, D, D) if c["state"] else None
    if c["op"] == "decay":
        s["o"] = empty(B, N, H, D, dtype=dt)
        s["state_out"] = empty(B, H, D, D)
    else:
        s["do"] = randn(B, N, H, D).to(dt)
        s["dstate_out"] = randn(B, H, D, D) / D ** 0.5 if c["state"] else None
        s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[n]) for n in ("q", "k", "v"))
        s["dstate_in"] = empty(B, H, D, D) if c["state"] else None
        s["dlog_decay"] = empty(H)
    if own:
        from paper_2603_02561_amd import binding as sb
        code = sb.SOLAR_BF16 if c["dtype"] == BF16 else sb.SOLAR_F32
        nbytes = sb.solar_decay_workspace_bytes(B, N, H, Hkv, D, code, c["op"] == "decay_bw")
        s["workspace"] = torch.empty(max(256, nbytes), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------------------
# Plain forms


def _valid(s, N, dev):
    """[B,N,1,1] truth values of the rows before each length, None where all are."""
    if s["lengths"] is None:
        return None
    return (torch.arange(N, device=dev)[None, :] < s["lengths"][:, None])[:, :, None, None]


def _masked(x, valid):
    return x if valid is None else torch.where(valid, x, torch.zeros((), dtype=x.dtype, device=x.device))


def _chunks(x, C):
    """[B,N,H,D] -> [B,H,chunks,C,D], zero rows at the end."""
    B, N, H, D = x.shape
    pad = -N % C
    if pad:
        x = torch.cat([x, torch.zeros(B, pad, H, D, dtype=x.dtype, device=x.device)], 1)
    return x.reshape(B, (N + pad) // C, C, H, D).permute(0, 3, 1, 2, 4).contiguous()


def _exp(log_decay, n):
    """g^n for whole numbers n >= 0 of any shape, per head: [H, *n.shape] in 32 bits, the exponents in 64."""
    e = log_decay.double().reshape(-1, *([1] * n.dim())) * n.double()
    return torch.exp(e).float()


def _attend(q, k, v, g, state, moment=False):
    """sum over s <= t of g^(t-s) (q_t . k_s) v_s, plus g^(t+1) state^T q_t; with `moment` its derivative by log g."""
    B, N, H, D = q.shape
    dev = q.device
    C = min(_CHUNK, N)
    qc, kc, vc = _chunks(q, C), _chunks(k, C), _chunks(v, C)
    nc = qc.shape[2]
    i = torch.arange(C, device=dev)
    ago = (i[:, None] - i[None, :]).clamp(min=0)
    causal = i[:, None] >= i[None, :]
    w = _exp(g, ago) * causal
    p = torch.matmul(qc, kc.transpose(-1, -2).contiguous())
    w_in = _exp(g, C - 1 - i)[None, :, None, :, None]
    inc = torch.matmul(kc.transpose(-1, -2).contiguous(), vc * w_in)                 # [B,H,nc,D,D]
    j = torch.arange(nc, device=dev)
    far = j[:, None] - 1 - j[None, :]
    before = far >= 0
    wj = _exp(g, C * far.clamp(min=0)) * before                                       # [H,nc,nc]
    start = torch.matmul(wj[None], inc.reshape(B, H, nc, D * D)).reshape(B, H, nc, D, D)
    if state is not None:
        start = start + _exp(g, C * j)[None, :, :, None, None] * state[:, :, None]
    w_t = _exp(g, i + 1)[None, :, None, :, None]
    if not moment:
        o = torch.matmul(p * w[None, :, None], vc) + w_t * torch.matmul(qc, start)
    else:
        inc_m = torch.matmul(kc.transpose(-1, -2).contiguous(), vc * (w_in * (C - 1 - i).float()[:, None]))
        start_m = torch.matmul(wj[None], inc_m.reshape(B, H, nc, D * D))
        start_m = start_m + torch.matmul((wj * (C * far.clamp(min=0)).float())[None], inc.reshape(B, H, nc, D * D))
        start_m = start_m.reshape(B, H, nc, D, D)
        if state is not None:
            start_m = start_m + (_exp(g, C * j) * (C * j).float())[None, :, :, None, None] * state[:, :, None]
        o = torch.matmul(p * (w * ago.float())[None, :, None], vc)
        o = o + w_t * (torch.matmul(qc, start_m) + (i + 1).float()[:, None] * torch.matmul(qc, start))
    return o.permute(0, 2, 3, 1, 4).reshape(B, nc * C, H, D)[:, :N]


def _last(k, v, g, n, state, moment=False):
    """sum over s < n of g^(n-1-s) k_s v_s^T, plus g^n state, for lengths n [B]; with `moment` its derivative by log g."""
    B, N, H, D = k.shape
    ago = (n[:, None] - 1 - torch.arange(N, device=k.device)[None, :]).clamp(min=0)
    w = _exp(g, ago)
    w0 = _exp(g, n)
    if moment:
        w, w0 = w * ago.float(), w0 * n.float()
    w = w.permute(1, 2, 0)[..., None]                                                 # [B,N,H,1]
    last = torch.matmul(k.permute(0, 2, 3, 1).contiguous(), (v * w).permute(0, 2, 1, 3).contiguous())
    return last if state is None else last + w0.t()[:, :, None, None] * state


def _heads(x, H):
    """Shared heads repeated for the heads that read them."""
    return x.repeat_interleave(H // x.shape[2], 2) if x.shape[2] != H else x


def _plain_decay(s):
    c = s["case"]
    N, H = c["N"], c["H"]
    valid = _valid(s, N, s["q"].device)
    q, k, v = (_heads(_masked(s[n], valid).float(), H) for n in ("q", "k", "v"))
    n = s["lengths"] if s["lengths"] is not None else torch.full((c["B"],), N, dtype=torch.int32, device=q.device)
    g = s["log_decay"]
    if N == 1:
        # a single token: the recurrence itself
        new = k[:, 0, :, :, None] * v[:, 0, :, None, :]
        if s["state_in"] is not None:
            kept = n.float()[:, None, None, None] * g[:, None, None]
            new = new + torch.exp(kept) * s["state_in"]
        o = _scale(c) * _masked(torch.matmul(q[:, 0, :, None, :], new).permute(0, 2, 1, 3), valid)
        return {"o": o.to(s["q"].dtype), "state": new}
    o = _scale(c) * _masked(_attend(q, k, v, g, s["state_in"]), valid)
    return {"o": o.to(s["q"].dtype), "state": _last(k, v, g, n, s["state_in"])}


def _back(x, n):
    """Rows of each user in reverse order: row i takes row n - 1 - i, rows past n are whatever."""
    at = (n[:, None] - 1 - torch.arange(x.shape[1], device=x.device)[None, :]) % x.shape[1]
    return torch.gather(x, 1, at[:, :, None, None].expand(-1, -1, x.shape[2], x.shape[3]))


def _plain_decay_bw(s):
    c = s["case"]
    B, N, H, Hkv, D = c["B"], c["N"], c["H"], c["Hkv"], c["D"]
    valid = _valid(s, N, s["q"].device)
    q, k, v, do = (_heads(_masked(s[n], valid).float(), H) for n in ("q", "k", "v", "do"))
    n = (s["lengths"] if s["lengths"] is not None else torch.full((B,), N, device=q.device)).long()
    g, do = s["log_decay"], do * _scale(c)
    turned = lambda x: None if x is None else x.transpose(-1, -2).contiguous()  # noqa: E731
    dq = _attend(do, v, k, g, turned(s["state_in"]))
    rq, rk, rv, rdo = (_masked(_back(x, n), valid) for x in (q, k, v, do))
    # the state that the reversed rows start from reaches row n - 1 with weight g^0, one less than _attend gives it
    e = s["dstate_out"]
    at = torch.arange(N, device=q.device)
    w = _exp(g, at).t()[None, :, :, None]
    dk, dv = _attend(rv, rdo, rq, g, None), _attend(rk, rq, rdo, g, None)
    if e is not None:
        dk = dk + w * torch.matmul(rv.permute(0, 2, 1, 3).contiguous(), turned(e)).permute(0, 2, 1, 3)
        dv = dv + w * torch.matmul(rk.permute(0, 2, 1, 3).contiguous(), e).permute(0, 2, 1, 3)
    dk, dv = (_masked(_back(x, n), valid).reshape(B, N, Hkv, H // Hkv, D).sum(3) for x in (dk, dv))
    z = (do.double() * _attend(q, k, v, g, s["state_in"], moment=True).double()).sum((0, 1, 3))
    out = {"dq": _masked(dq, valid), "dk": dk, "dv": dv}
    out = {name: x.to(s["q"].dtype) for name, x in out.items()}
    if e is not None:
        w_t = _exp(g, at + 1).t()[None, :, :, None]
        out["dstate"] = torch.matmul((q * w_t).permute(0, 2, 3, 1).contiguous(), do.permute(0, 2, 1, 3).contiguous())
        out["dstate"] = out["dstate"] + _exp(g, n).t()[:, :, None, None] * e
        z = z + (e.double() * _last(k, v, g, n, s["state_in"], moment=True).double()).sum((0, 2, 3))
    return {**out, "dlog_decay": z.float()}


def _turn(x, angle, amplitude, interleaved):
    """Rotates the first pairs of the columns of x [B,N,H,D] by angle [B,N,1,pairs], which is in 64 bits."""
    n = angle.shape[-1]
    cos, sin = (amplitude * torch.cos(angle)).float(), (amplitude * torch.sin(angle)).float()
    xf = x.float()
    a, b = (xf[..., 0:2 * n:2], xf[..., 1:2 * n:2]) if interleaved else (xf[..., :n], xf[..., n:2 * n])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned, xf[..., 2 * n:]], -1).to(x.dtype)


def _plain_rotary(s):
    c = s["case"]
    pos = s["positions"] if s["positions"] is not None else torch.arange(c["N"], device="cuda")[None, :]
    angle = (pos.double()[:, :, None] * s["freq"])[:, :, None, :]
    return {n: _turn(s[n], angle, s["amplitude"], c["interleaved"]) for n in ("q", "k")}


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(-1, keepdim=True)
    diff = x - mean
    rstd = torch.rsqrt((diff * diff).mean(-1, keepdim=True) + s["eps"])
    y = diff * rstd * s["weight"] + s["bias"]
    return {"y": y.to(s["x"].dtype), "mean": mean[..., 0], "rstd": rstd[..., 0]}


def _plain_norm_bw(s):
    dy = s["dy"].float()
    xhat = (s["x"].float() - s["mean"][..., None]) * s["rstd"][..., None]
    g = dy * s["weight"]
    dx = s["rstd"][..., None] * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * xhat).sum(0), "dbias": dy.sum(0)}


_PLAIN = {"decay": _plain_decay, "decay_bw": _plain_decay_bw, "rotary": _plain_rotary, "norm": _plain_norm,
          "norm_bw": _plain_norm_bw}


def run(s):
    """One pass."""
    c = s["case"]
    if not own:
        return _PLAIN[c["op"]](s)
    from paper_2603_02561_amd import binding as sb
    op = c["op"]
    if op == "decay":
        sb.solar_decay_attention(s["q"], s["k"], s["v"], s["log_decay"], s["lengths"], _scale(c), s["o"], s["state_in"],
                                 s["state_out"], s["workspace"])
        return {"o": s["o"], "state": s["state_out"]}
    if op == "decay_bw":
        sb.solar_decay_attention_backward(s["q"], s["k"], s["v"], s["do"], s["log_decay"], s["lengths"], _scale(c),
                                          s["state_in"], s["dstate_out"], s["dq"], s["dk"], s["dv"], s["dstate_in"],
                                          s["dlog_decay"], s["workspace"])
        out = {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"], "dlog_decay": s["dlog_decay"]}
        return {**out, "dstate": s["dstate_in"]} if c["state"] else out
    if op == "rotary":
        sb.solar_rotary(s["q"], s["k"], s["freq"], s["q_out"], s["k_out"], positions=s["positions"],
                        layout=sb.SOLAR_ROTARY_INTERLEAVED if c["interleaved"] else sb.SOLAR_ROTARY_HALF,
                        amplitude=s["amplitude"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "norm":
        sb.solar_layer_norm(s["x"], s["weight"], s["bias"], s["eps"], s["y"], s["mean"], s["rstd"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    sb.solar_layer_norm_backward(s["x"], s["weight"], s["mean"], s["rstd"], s["dy"], s["dx"], s["dweight"], s["dbias"],
                                 s["workspace"])
    return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}


def exact(case, seed):
    """What run() returns, in 64 bits and row by row from the definitions."""
    c = dict(case)
    op = c["op"]
    if op in ("decay", "decay_bw") and c["N"] * (3 if op == "decay_bw" else 1) > 70000:
        return None
    s = prepare(c, seed)
    f = {n: x.double() for n, x in s.items() if isinstance(x, torch.Tensor) and x.is_floating_point()}
    if op == "rotary":
        n = c["rot"] // 2
        pos = torch.arange(c["N"], device="cuda").expand(c["B"], -1) if s["positions"] is None else s["positions"]
        unit = torch.polar(torch.full_like(f["freq"], s["amplitude"]) * torch.ones_like(pos[..., None]),
                           pos.double()[..., None] * f["freq"])[:, :, None]
        out = {}
        for name in ("q", "k"):
            x = f[name]
            at = torch.arange(2 * n, device="cuda")
            first, second = (at[0::2], at[1::2]) if c["interleaved"] else (at[:n], at[n:])
            z = torch.complex(x[..., first], x[..., second]) * unit
            y = x.clone()
            y[..., first], y[..., second] = z.real, z.imag
            out[name] = y
        return out
    if op == "norm":
        var, mean = torch.var_mean(f["x"], -1, unbiased=False)
        rstd = 1 / torch.sqrt(var + s["eps"])
        return {"y": (f["x"] - mean[..., None]) * rstd[..., None] * f["weight"] + f["bias"], "mean": mean, "rstd": rstd}
    if op == "norm_bw":
        d = c["d"]
        xhat = (f["x"] - f["mean"][..., None]) * f["rstd"][..., None]
        a = f["dy"] * f["weight"]
        dx = f["rstd"][..., None] / d * (d * a - a.sum(-1, keepdim=True) - xhat * (a * xhat).sum(-1, keepdim=True))
        return {"dx": dx, "dweight": (f["dy"] * xhat).sum(0), "dbias": f["dy"].sum(0)}
    # the recurrence itself, a row at a time
    B, N, H, Hkv, D = c["B"], c["N"], c["H"], c["Hkv"], c["D"]
    group = H // Hkv
    q, k, v = f["q"], f["k"].repeat_interleave(group, 2), f["v"].repeat_interleave(group, 2)
    lengths = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), N, device="cuda")
    lam = torch.exp(f["log_decay"])[None, :, None, None]
    S = f["state_in"] if c["state"] else torch.zeros(B, H, D, D, dtype=torch.float64, device="cuda")
    live = (torch.arange(N, device="cuda")[:, None] < lengths)[:, :, None, None, None]          # [N,B,1,1,1]

    def dot(x, m):  # x [B,H,D], m [B,H,D,E] -> [B,H,E]
        return (x[..., None] * m).sum(-2)

    def outer(x, y):
        return x[..., :, None] * y[..., None, :]

    scale = _scale(c)
    T = torch.zeros_like(S)
    z = torch.zeros(H, dtype=torch.float64, device="cuda")
    out = torch.zeros(B, N, H, D, dtype=torch.float64, device="cuda")
    do = f["do"] * scale if op == "decay_bw" else None
    for t in range(N):
        on = live[t]
        if op == "decay_bw":
            T = torch.where(on, lam * (T + S), T)
        S = torch.where(on, lam * S + outer(k[:, t], v[:, t]), S)
        if op == "decay":
            out[:, t] = torch.where(on[..., 0], scale * dot(q[:, t], S), 0.0)
        else:
            out[:, t] = torch.where(on[..., 0], dot(do[:, t], S.transpose(-1, -2)), 0.0)
            z += (torch.where(on[..., 0], do[:, t], 0.0) * dot(q[:, t], T)).sum((0, 2))
    if op == "decay":
        return {"o": out, "state": S}
    dk, dv = torch.zeros_like(out), torch.zeros_like(out)
    G = f["dstate_out"] if c["state"] else torch.zeros_like(S)                                   # dL/dS_t before row t's own
    z += (G * T).sum((0, 2, 3))
    for t in range(N - 1, -1, -1):
        on = live[t]
        full = G + outer(q[:, t], do[:, t])
        dk[:, t] = torch.where(on[..., 0], dot(v[:, t], full.transpose(-1, -2)), 0.0)
        dv[:, t] = torch.where(on[..., 0], dot(k[:, t], full), 0.0)
        G = torch.where(on, lam * full, G)
    dk, dv = (x.reshape(B, N, Hkv, group, D).sum(3) for x in (dk, dv))
    r = {"dq": out, "dk": dk, "dv": dv, "dlog_decay": z}
    return {**r, "dstate": G} if c["state"] else r


def work(case):
    """Bytes (each input read once, each output written once) and operations of one pass, the recurrent form's.  Ragged
    batches are counted at their mean length, outputs at their full one."""
    c = case
    e = 2 if c["dtype"] == BF16 else 4
    if c["op"] in ("norm", "norm_bw"):
        n, p = c["rows"] * c["groups"] * c["d"], c["groups"] * c["d"] * 4
        if c["op"] == "norm":
            return {"bytes": float(2 * n * e + 8 * c["rows"] * c["groups"] + 2 * p), "flops": float(8 * n)}
        return {"bytes": float(3 * n * e + 8 * c["rows"] * c["groups"] + 3 * p), "flops": float(14 * n)}
    B, N, H, Hkv, D = c["B"], c["N"], c["H"], c["Hkv"], c["D"]
    if c["op"] == "rotary":
        nbytes = 2 * B * N * (H + Hkv) * D * e + (4 * B * N if c["far"] else 0) + 4 * c["rot"]
        return {"bytes": float(nbytes), "flops": float(3 * B * N * (H + Hkv) * c["rot"])}
    n = B * (N / 2 if c["ragged"] else N)
    q, kv, st = n * H * D * e, n * Hkv * D * e, 4 * B * H * D * D
    if c["op"] == "decay":
        nbytes = q + 2 * kv + B * N * H * D * e + st + (st if c["state"] else 0)
        return {"bytes": float(nbytes), "flops": float(4 * n * H * D * D)}
    nbytes = 2 * q + 2 * kv + B * N * (H + 2 * Hkv) * D * e + (3 * st if c["state"] else 0)
    return {"bytes": float(nbytes), "flops": float(14 * n * H * D * D)}
