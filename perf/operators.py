"""The activation side of a training step, timed: what a program that trains with the page update does
with a block's activations between the forward and the backward pass.

  write   apm_ckpt_write: activations [tokens, channels] into 8 bits, a scale for each 32 channels
  read    apm_ckpt_read: the values again
  fwd     apm_norm_join_forward: where one block ends and the next begins,
              y = residual_scale x + gate (post_norm(branch) w2 + b2),   n = pre_norm(y) w1 + b1,
          which keeps both normalised tensors in 8 bits for the backward pass
  bwd     apm_norm_join_backward: the gradients of all of it, out of the 8-bit tensors
  wgrad   apm_ckpt_weight_grad: the gradient of the weights of the linear layer behind a kept tensor,
              dW[o, k] = sum over tokens of dy[t, o] (w1[k] kept[t, k] + b1[k]),  db[o] = sum of dy[t, o],
          one product, or one for each expert of a mixture over that expert's tokens

A kept tensor is q and scale: a byte for each element (a whole number -127 .. 127, in units of 2^-6, or a
float of 4 exponent and 3 mantissa bits) and for each 32 channels of a token a byte s, which stands for
2^(s-127) and is the smallest for which no element is out of range.

Widths, hidden sizes and expert counts are those of the 124 M, 1.3 B, 13 B and mixture-of-experts shapes.
"""
import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 32
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases --------------------------------------------------------------------------------

def listed():
    return [
        # the last few tokens of a small fine-tuning batch: what a call costs that moves next to nothing
        {"name": "write_few_tokens", "kind": "write", "rows": 8, "cols": 768, "type": "bf16", "format": "i8", "pad": 0},
        # hidden activations of the 1.3 B shape, 16 sequences of 1024 tokens, in the floating format
        {"name": "write_hidden_1p3b", "kind": "write", "rows": 16384, "cols": 8192, "type": "bf16", "format": "f8", "pad": 0},
        # a slice of an odd-width model's activations, read back in 32 bits into a wider buffer
        {"name": "read_odd_f32", "kind": "read", "rows": 777, "cols": 1001, "type": "f32", "format": "i8", "pad": 7},
        # hidden activations of the 13 B shape, read back for the activation function's backward pass
        {"name": "read_hidden_13b", "kind": "read", "rows": 8192, "cols": 20480, "type": "bf16", "format": "i8", "pad": 0},
        # few tokens through one join of the 124 M shape
        {"name": "fwd_few_tokens", "kind": "fwd", "rows": 8, "cols": 768, "res": "bf16", "act": "bf16", "par": "bf16",
         "pre": "layer", "post": "none", "gate": "none", "bias": True, "scale": 1.0, "format": "f8"},
        # the 1.3 B shape, norms before and after a block, a learned gate for each channel
        {"name": "fwd_1p3b", "kind": "fwd", "rows": 8192, "cols": 2048, "res": "bf16", "act": "bf16", "par": "bf16",
         "pre": "rms", "post": "rms", "gate": "channel", "bias": False, "scale": 1.0, "format": "f8"},
        # an odd width, 32-bit residual stream, a gate for each token as a router gives it
        {"name": "fwd_odd_token_gate", "kind": "fwd", "rows": 3001, "cols": 1001, "res": "f32", "act": "bf16", "par": "f32",
         "pre": "layer", "post": "layer", "gate": "token", "bias": True, "scale": 1.7, "format": "i8"},
        # the gradients of the small join
        {"name": "bwd_few_tokens", "kind": "bwd", "rows": 8, "cols": 768, "res": "bf16", "act": "bf16", "par": "bf16",
         "pre": "layer", "post": "none", "gate": "none", "bias": True, "scale": 1.0, "format": "f8"},
        # the 13 B shape with a 32-bit residual stream
        {"name": "bwd_13b", "kind": "bwd", "rows": 8192, "cols": 5120, "res": "f32", "act": "bf16", "par": "bf16",
         "pre": "rms", "post": "rms", "gate": "channel", "bias": False, "scale": 0.9, "format": "i8"},
        # a square matrix of the 124 M shape over one odd batch
        {"name": "wgrad_124m_odd_batch", "kind": "wgrad", "tokens": 1000, "out": 768, "in": 768, "groups": 0,
         "format": "i8", "type": "f32", "affine": "weight", "bias": True},
        # the first matrix of the 1.3 B shape's feed-forward part, 16 sequences of 1024 tokens
        {"name": "wgrad_1p3b", "kind": "wgrad", "tokens": 16384, "out": 8192, "in": 2048, "groups": 0,
         "format": "i8", "type": "bf16", "affine": "both", "bias": True},
        # the experts of the mixture shape: 64 experts, an eighth of them with tokens
        {"name": "wgrad_experts", "kind": "wgrad", "tokens": 8192, "out": 4096, "in": 1024, "groups": 64, "active": 8,
         "format": "f8", "type": "bf16", "affine": "none", "bias": False},
    ]


def _log_between(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    n = _log_between(rng, lo, hi)
    return max(lo, n - n % 64) if rng.random() < 0.5 else n


def draw(rng):
    """One more case of the ranges above: a few tokens up to 16384, odd and even widths, every format, type, norm and gate."""
    kind = rng.choice(["write", "read", "fwd", "fwd", "bwd", "bwd", "wgrad", "wgrad", "wgrad"])
    form = rng.choice(["i8", "f8"])
    if kind in ("write", "read"):
        cols = _width(rng, 40, 20480)
        rows = _log_between(rng, 1, min(16384, 16384 * 8192 // cols))
        return {"kind": kind, "rows": rows, "cols": cols, "type": rng.choice(["bf16", "bf16", "f32"]), "format": form,
                "pad": rng.choice([0, 0, 8, 7])}
    if kind in ("fwd", "bwd"):
        cols = _width(rng, 64, 12288)
        rows = _log_between(rng, 1, min(16384, 8192 * 5120 // cols))
        res = rng.choice(["bf16", "f32"])
        norm = rng.choice(["rms", "layer"])
        return {"kind": kind, "rows": rows, "cols": cols, "res": res, "act": "bf16" if res == "bf16" else rng.choice(["bf16", "bf16", "f32"]),
                "par": rng.choice(["bf16", "f32"]), "pre": norm, "post": rng.choice(["none", norm, norm]),
                "gate": rng.choice(["none", "channel", "channel", "token", "full"]), "bias": norm == "layer",
                "scale": rng.choice([1.0, 1.0, 0.7, 1.9]), "format": form}
    groups = rng.choice([0, 0, 0, 8, 64])
    most = 16384 * 8192 * 2048
    if groups:
        wide, narrow = _width(rng, 64, 4096), _width(rng, 64, 1024)
        tokens = _log_between(rng, 1, 8192)
    else:
        wide, narrow = _width(rng, 64, 8192), _width(rng, 64, 4096)
        tokens = _log_between(rng, 1, min(16384, most // (wide * narrow)))
    out, k = (wide, narrow) if rng.random() < 0.5 else (narrow, wide)
    case = {"kind": kind, "tokens": tokens, "out": out, "in": k, "groups": groups, "format": form,
            "type": rng.choice(["bf16", "bf16", "f32"]), "affine": rng.choice(["none", "weight", "both"]), "bias": rng.random() < 0.5}
    return dict(case, active=rng.randint(1, groups)) if groups else case


def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["kind"] in ("write", "read"):
        n = case["rows"] * case["cols"]
        return {"bytes": n * (size[case["type"]] + 1) + case["rows"] * -(-case["cols"] // BLOCK), "flops": 0}
    if case["kind"] in ("fwd", "bwd"):
        r, c = case["rows"], case["cols"]
        # x, branch, y, n and the two kept tensors; backward: dy, dn, dx, dbranch and the two kept tensors
        n = r * c * 2 * (size[case["res"]] + size[case["act"]] + 1) + 2 * r * -(-c // BLOCK) + 8 * r
        n += {"none": 0, "channel": c, "token": r, "full": r * c}[case["gate"]] * size[case["par"]] * (1 if case["kind"] == "fwd" else 2)
        return {"bytes": n, "flops": 0}
    t, o, k = case["tokens"], case["out"], case["in"]
    return {"bytes": t * o * 2 + t * (k + -(-k // BLOCK)) + max(1, case["groups"]) * o * k * size[case["type"]], "flops": 2 * t * o * k}


# ---- inputs -----------------------------------------------------------------------------------

def _times_power(v, n):
    """v 2^n, exactly: exp2 rounds, and 2^n may lie outside the range where the two parts that are multiplied by do not."""
    half = torch.div(n, 2, rounding_mode="floor")
    return v * ((half + 127) << 23).view(torch.float32) * ((n - half + 127) << 23).view(torch.float32)


def _encode(x, form):
    """x [rows, cols] in 32 bits -> (bytes [rows, cols], scale bytes [rows, blocks]), both uint8."""
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    v = torch.nn.functional.pad(x, (0, nb * BLOCK - cols)).view(rows, nb, BLOCK)
    bits = v.abs().amax(dim=2).view(torch.int32)       # the bits of a float that is not negative count up with it
    lost = bits >= 0x7F800000                          # an infinity or a NaN in the block
    if form == "i8":                                   # largest / scale < 127.5 / 64
        s = ((bits + 0x00010000) >> 23).clamp(0, 254)
        shift = 133 - s
    else:                                              # largest / scale <= 464, which rounds to 448
        s = (((bits + 0x0017FFFF) >> 23) - 8).clamp(0, 254)
        shift = 127 - s
    v = torch.where(lost[..., None], torch.zeros_like(v), _times_power(v, shift[..., None]))
    q = v.round().clamp(-127, 127).to(torch.int8) if form == "i8" else v.to(torch.float8_e4m3fn)
    q = q.view(torch.uint8).reshape(rows, nb * BLOCK)[:, :cols].contiguous()
    return q, torch.where(lost, 255, s).to(torch.uint8)


def _decode(q, scale, form):
    """The values in 32 bits."""
    rows, cols = q.shape
    s = scale.to(torch.int32)
    m = torch.where(s == 255, torch.full((), float("nan"), device=q.device), _times_power(torch.ones((), device=q.device), s - 127))
    v = q.view(torch.int8).float() * (1 / 64) if form == "i8" else q.view(torch.float8_e4m3fn).float()
    return v * m.repeat_interleave(BLOCK, dim=1)[:, :cols]


def _stream_like(rows, cols, g, spread=1.0):
    """A residual stream or hidden activations: channels of different size, a few of them large."""
    size = torch.exp(0.5 * torch.randn(cols, device=DEV, generator=g))
    size[torch.randint(0, cols, (max(1, cols // 200),), device=DEV, generator=g)] *= 15.0
    return torch.randn(rows, cols, device=DEV, generator=g) * size * spread


def _hat(v, norm):
    """(normalised v, 1 / its standard deviation or root mean square, a value for each row), in v's own type"""
    if norm == "none":
        return v, torch.ones(v.shape[0], dtype=v.dtype, device=v.device)
    c = v - v.mean(dim=1, keepdim=True) if norm == "layer" else v
    r = 1.0 / torch.sqrt(c.square().mean(dim=1, keepdim=True) + EPS)
    return c * r, r[:, 0].contiguous()


def _blank(rows, cols, form):
    return (torch.empty(rows, cols, dtype=torch.uint8, device=DEV), torch.empty(rows, -(-cols // BLOCK), dtype=torch.uint8, device=DEV))


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case)

    def randn(*shape):
        return torch.randn(*shape, device=DEV, generator=g)

    if case["kind"] in ("write", "read"):
        rows, cols, t = case["rows"], case["cols"], TYPES[case["type"]]
        x = _stream_like(rows, cols, g)
        if case["kind"] == "write":
            wide = torch.zeros(rows, cols + case["pad"], dtype=t, device=DEV)
            wide[:, :cols] = x.to(t)
            s["x"], s["kept"] = wide[:, :cols], _blank(rows, cols, case["format"])
        else:
            s["kept"] = _encode(x, case["format"])
            s["x"] = torch.empty(rows, cols + case["pad"], dtype=t, device=DEV)[:, :cols]
        return s
    if case["kind"] in ("fwd", "bwd"):
        rows, cols, par = case["rows"], case["cols"], TYPES[case["par"]]
        res, act = TYPES[case["res"]], TYPES[case["act"]]
        s["w1"], s["w2"] = (1 + 0.2 * randn(cols)).to(par), (0.5 + 0.1 * randn(cols)).to(par)
        s["b1"], s["b2"] = ((0.1 * randn(cols)).to(par), (0.1 * randn(cols)).to(par)) if case["bias"] else (None, None)
        shape = {"none": None, "channel": (1, cols), "token": (rows, 1), "full": (rows, cols)}[case["gate"]]
        s["gated"] = case["gate"]
        s["gate"] = None if shape is None else torch.sigmoid(randn(*shape)).to(par)
        x, branch = _stream_like(rows, cols, g).to(res), (0.4 * randn(rows, cols)).to(act)
        s["rstd1"], s["rstd2"] = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        if case["kind"] == "fwd":
            s["x"], s["branch"], s["y"], s["n"] = x, branch, torch.empty_like(x), torch.empty_like(branch)
            s["kept1"], s["kept2"] = _blank(rows, cols, case["format"]), _blank(rows, cols, case["format"])
            s["back1"], s["back2"] = (torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV) for _ in range(2))
            return s
        hat, s["rstd1"] = _hat(x.float(), case["pre"])
        s["kept1"] = _encode(hat, case["format"])
        hat, s["rstd2"] = _hat(branch.float(), case["post"])
        s["kept2"] = _encode(hat, case["format"])
        s["dy"], s["dn"] = (1e-3 * randn(rows, cols)).to(res), (1e-3 * randn(rows, cols)).to(act)
        s["dx"], s["dbranch"] = torch.empty_like(s["dy"]), torch.empty_like(s["dn"])
        for name in ("w1", "b1", "w2", "b2", "gate"):
            s["d" + name] = None if s[name] is None else torch.empty_like(s[name])
        return s
    t, o, k = case["tokens"], case["out"], case["in"]
    s["dy"] = (1e-3 * randn(t, o)).to(torch.bfloat16)
    s["kept"] = _encode(randn(t, k), case["format"])
    s["w"] = (1 + 0.2 * randn(k)).to(torch.bfloat16) if case["affine"] != "none" else None
    s["b"] = (0.1 * randn(k)).to(torch.bfloat16) if case["affine"] == "both" else None
    s["ends"], s["offsets"] = None, None
    if case["groups"]:  # tokens sorted by expert; the active ones take uneven shares
        n, live = case["groups"], torch.randperm(case["groups"], device=DEV, generator=g)[:case["active"]]
        share = torch.zeros(n, device=DEV)
        share[live] = torch.rand(case["active"], device=DEV, generator=g) + 0.2
        at = (torch.cumsum(share, 0) / share.sum() * t).round().to(torch.int64).clamp(0, t)
        s["offsets"] = torch.cat([at.new_zeros(1), at])
        s["offsets"][int(live.max()) + 1:] = t
        s["ends"] = s["offsets"].tolist()
    lead = (case["groups"],) if case["groups"] else ()
    s["dw"] = torch.empty(*lead, o, k, dtype=TYPES[case["type"]], device=DEV)
    s["db"] = torch.empty(*lead, o, dtype=TYPES[case["type"]], device=DEV) if case["bias"] else None
    return s


# ---- one pass ---------------------------------------------------------------------------------

def _seen(q, scale, form):
    """A kept tensor as what its bytes stand for."""
    return (q.view(torch.int8) if form == "i8" else q.view(torch.float8_e4m3fn)), scale


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2303_02868_amd as apm

    form = apm.APM_CKPT_I8 if s["format"] == "i8" else apm.APM_CKPT_F8
    kind = s["kind"]
    if kind == "write":
        apm.apm_ckpt_write(s["x"], apm.make_ckpt(*s["kept"], form))
        return _seen(*s["kept"], s["format"])
    if kind == "read":
        apm.apm_ckpt_read(apm.make_ckpt(*s["kept"], form), s["x"])
        return s["x"]
    if kind == "wgrad":
        grad = apm.make_weight_grad(s["dy"], apm.make_ckpt(*s["kept"], form), s["dw"], db=s["db"], weight=s["w"], bias=s["b"], offsets=s["offsets"])
        room = torch.empty(apm.apm_ckpt_weight_grad_workspace_bytes(grad), dtype=torch.uint8, device=DEV)
        apm.apm_ckpt_weight_grad(grad, room)
        return s["dw"], s["db"]
    norm = {"none": apm.APM_NORM_NONE, "rms": apm.APM_NORM_RMS, "layer": apm.APM_NORM_LAYER}
    gate = {"none": apm.APM_GATE_NONE, "channel": apm.APM_GATE_CHANNEL, "token": apm.APM_GATE_TOKEN, "full": apm.APM_GATE_FULL}
    kept = [apm.make_ckpt(*s["kept1"], form), apm.make_ckpt(*s["kept2"], form)]
    join = apm.make_norm_join(s["rows"], s["cols"], x=s.get("x"), branch=s.get("branch"), y=s.get("y"), n=s.get("n"),
                              residual_scale=s["scale"], pre_norm=norm[s["pre"]], pre_eps=EPS, pre_weight=s["w1"], pre_bias=s["b1"],
                              pre_ckpt=kept[0], pre_rstd=s["rstd1"], post_norm=norm[s["post"]], post_eps=EPS, post_weight=s["w2"],
                              post_bias=s["b2"], post_ckpt=kept[1], post_rstd=s["rstd2"], gate_kind=gate[s["gated"]], gate=s["gate"])
    if kind == "fwd":
        apm.apm_norm_join_forward(join)
        if s["format"] == "i8":  # whole numbers of a value computed in 32 bits: as the values that they stand for
            apm.apm_ckpt_read(kept[0], s["back1"])
            apm.apm_ckpt_read(kept[1], s["back2"])
            return s["y"], s["n"], s["rstd1"], s["rstd2"], s["back1"], s["back2"]
        return (s["y"], s["n"], s["rstd1"], s["rstd2"], *_seen(*s["kept1"], "f8")[:1], s["kept1"][1].view(torch.float8_e8m0fnu),
                *_seen(*s["kept2"], "f8")[:1], s["kept2"][1].view(torch.float8_e8m0fnu))
    grads = apm.make_norm_join_grads(join, dn=s["dn"], dy=s["dy"], dx=s["dx"], dbranch=s["dbranch"], dgate=s["dgate"], dpre_weight=s["dw1"],
                                     dpre_bias=s["db1"], dpost_weight=s["dw2"], dpost_bias=s["db2"])
    room = torch.empty(apm.apm_norm_join_workspace_bytes(s["rows"], s["cols"]), dtype=torch.uint8, device=DEV)
    apm.apm_norm_join_backward(join, grads, room)
    return s["dx"], s["dbranch"], s["dgate"], s["dw1"], s["db1"], s["dw2"], s["db2"]


def _run_plain(s):
    kind = s["kind"]
    if kind == "write":
        return _seen(*_encode(s["x"].float(), s["format"]), s["format"])
    if kind == "read":
        return _decode(*s["kept"], s["format"]).to(s["x"].dtype)
    if kind == "wgrad":
        kept, dy, t = _decode(*s["kept"], s["format"]), s["dy"].float(), s["dw"].dtype
        if s["w"] is not None:
            kept = kept * s["w"].float()
        if s["b"] is not None:
            kept = kept + s["b"].float()
        if s["ends"] is None:
            return (dy.T @ kept).to(t), (dy.sum(0).to(t) if s["db"] is not None else None)
        parts = list(zip(s["ends"][:-1], s["ends"][1:]))
        return (torch.stack([(dy[a:b].T @ kept[a:b]).to(t) for a, b in parts]),
                torch.stack([dy[a:b].sum(0).to(t) for a, b in parts]) if s["db"] is not None else None)
    w1, w2, b1, b2, gate = (None if s[n] is None else s[n].float() for n in ("w1", "w2", "b1", "b2", "gate"))
    one = torch.ones((), device=DEV)
    gate = one if gate is None else gate
    if kind == "fwd":
        hat2, r2 = _hat(s["branch"].float(), s["post"])
        y = s["scale"] * s["x"].float() + gate * (hat2 * w2 + (b2 if b2 is not None else 0.0))
        hat1, r1 = _hat(y, s["pre"])
        n = hat1 * w1 + (b1 if b1 is not None else 0.0)
        kept1, kept2 = _encode(hat1, s["format"]), _encode(hat2, s["format"])
        if s["format"] == "i8":
            kept = _decode(*kept1, "i8").bfloat16(), _decode(*kept2, "i8").bfloat16()
        else:
            kept = (_seen(*kept1, "f8")[0], kept1[1].view(torch.float8_e8m0fnu), _seen(*kept2, "f8")[0], kept2[1].view(torch.float8_e8m0fnu))
        return (y.to(s["x"].dtype), n.to(s["branch"].dtype), r1, r2, *kept)
    hat1, hat2 = _decode(*s["kept1"], s["format"]), _decode(*s["kept2"], s["format"])
    dn = s["dn"].float()
    dy = s["dy"].float() + _through_norm(dn * w1, hat1, s["rstd1"], s["pre"])
    dc, c = dy * gate, hat2 * w2 + (b2 if b2 is not None else 0.0)
    dbranch = _through_norm(dc * w2, hat2, s["rstd2"], s["post"])
    dgate = {"none": lambda v: None, "channel": lambda v: v.sum(0, keepdim=True), "token": lambda v: v.sum(1, keepdim=True), "full": lambda v: v}[s["gated"]](dy * c)
    par = s["w1"].dtype
    return ((s["scale"] * dy).to(s["dy"].dtype), dbranch.to(s["dn"].dtype), None if dgate is None else dgate.to(par), (dn * hat1).sum(0).to(par),
            None if b1 is None else dn.sum(0).to(par), (dc * hat2).sum(0).to(par), None if b2 is None else dc.sum(0).to(par))


def _through_norm(t, hat, rstd, norm):
    """The gradient of what was normalised to `hat`, where that of hat is t."""
    if norm == "none":
        return t
    u = t - hat * (t * hat).mean(dim=1, keepdim=True)
    if norm == "layer":
        u = u - t.mean(dim=1, keepdim=True)
    return u * rstd[:, None]


# ---- the definition, in 64 bits ---------------------------------------------------------------

def _power_64(e):
    return (e.to(torch.int64) + 1023 << 52).view(torch.float64)


def _kept_64(v, form):
    """(element values, scales, values) of the 8-bit form of v, each in 64 bits, found by exponents and remainders."""
    rows, cols = v.shape
    out_q, out_s = torch.zeros_like(v), torch.zeros(rows, -(-cols // BLOCK), dtype=torch.float64, device=v.device)
    for j in range(out_s.shape[1]):
        part = v[:, j * BLOCK:(j + 1) * BLOCK]
        top = part.abs().max(dim=1).values
        m, e = torch.frexp(top)                                        # top = m 2^e, 1/2 <= m < 1
        e = torch.where(top == 0, torch.full_like(e, -200), e - 1)     # top = 2 m 2^(e-1)
        e = e + (2 * m >= 127.5 / 64) if form == "i8" else e - 8 + (2 * m > 1.8125)
        unit = _power_64(e.clamp(-127, 127))
        r = part / unit[:, None]
        if form == "i8":
            r = torch.round(r * 64).clamp(-127, 127) / 64
        else:
            step = _power_64((torch.frexp(r)[1] - 1).clamp(min=-6) - 3)
            r = torch.round(r / step) * step
        out_q[:, j * BLOCK:(j + 1) * BLOCK], out_s[:, j] = r, unit
    return out_q, out_s, out_q * out_s.repeat_interleave(BLOCK, 1)[:, :cols]


def _values_64(q, scale, form):
    u = _power_64(scale.to(torch.int64) - 127)
    e = q.view(torch.int8).double() / 64.0 if form == "i8" else q.view(torch.float8_e4m3fn).double()
    return torch.cat([e[:, a:a + BLOCK] * u[:, a // BLOCK, None] for a in range(0, q.shape[1], BLOCK)], dim=1)


def _normed_64(v, norm):
    if norm == "none":
        return v, torch.ones_like(v[:, 0])
    mean = v.sum(1) / v.shape[1] if norm == "layer" else torch.zeros_like(v[:, 0])
    r = ((v - mean[:, None]).pow(2).sum(1) / v.shape[1] + EPS).pow(-0.5)
    return (v - mean[:, None]) * r[:, None], r


def exact(case, seed):
    s, form = prepare(case, seed), case["format"]
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.dtype in (torch.bfloat16, torch.float32)}
    if case["kind"] == "write":
        q, scale, _ = _kept_64(d["x"], form)
        return (q * 64).to(torch.int8) if form == "i8" else q, (torch.frexp(scale)[1] + 126).to(torch.uint8)
    if case["kind"] == "read":
        return _values_64(*s["kept"], form)
    if case["kind"] == "wgrad":
        z = _values_64(*s["kept"], form) * d.get("w", 1.0) + d.get("b", 0.0)
        ends = s["ends"] or [0, case["tokens"]]
        dw = torch.stack([torch.mm(d["dy"][a:b].t().contiguous(), z[a:b]) for a, b in zip(ends, ends[1:])])
        db = torch.stack([d["dy"][a:b].sum(0) for a, b in zip(ends, ends[1:])]) if case["bias"] else None
        return (dw, db) if s["ends"] else (dw[0], None if db is None else db[0])
    w1, w2, b1, b2, gate = d["w1"], d["w2"], d.get("b1", 0.0), d.get("b2", 0.0), d.get("gate", 1.0)
    if case["kind"] == "fwd":
        z2, r2 = _normed_64(d["branch"], case["post"])
        y = d["x"] * case["scale"] + (z2 * w2 + b2) * gate
        z1, r1 = _normed_64(y, case["pre"])
        kept = [_kept_64(z1, form), _kept_64(z2, form)]
        return (y, z1 * w1 + b1, r1, r2, *([k[2] for k in kept] if form == "i8" else [v for k in kept for v in k[:2]]))
    # the chain rule with the normalised tensors as they are kept
    z1, z2 = _values_64(*s["kept1"], form), _values_64(*s["kept2"], form)
    n = case["cols"]

    def back(t, z, r, norm):
        if norm == "none":
            return t
        inner = (t * z).sum(1) / n
        mean = t.sum(1) / n if norm == "layer" else torch.zeros_like(inner)
        return r[:, None] * (t - mean[:, None] - z * inner[:, None])

    dy = d["dy"] + back(d["dn"] * w1, z1, d["rstd1"], case["pre"])
    dz2 = dy * gate
    db = back(dz2 * w2, z2, d["rstd2"], case["post"])
    dg = dy * (z2 * w2 + b2)
    dg = {"none": None, "channel": dg.sum(0)[None], "token": dg.sum(1)[:, None], "full": dg}[case["gate"]]
    return (dy * case["scale"], db, dg, (d["dn"] * z1).sum(0), d["dn"].sum(0) if case["bias"] else None, (dz2 * z2).sum(0),
            dz2.sum(0) if case["bias"] else None)
