"""The token-wise operators of a transformer layer that stand beside the packed attention of a nested sequence-parallel
plan, as cases that can be timed and compared: the rotation of queries and keys by their positions on the way into the
attention, the normalisation of hidden states and of heads, and the gated half of the feed-forward block, each with its
backward pass.

A case describes one call with plain values:
  op          "rope"   queries and keys of one GPU's share, "tokens@hq/hkv; ..." for the nodes of its chain (`runs`)
              "norm"   `rows` rows (times `heads`, where heads are normalised) of `dim` values
              "glu"    `rows` tokens of `dim` features against two weights of `ff` rows
  direction   "forward" or "backward"
  own = True takes the library's calls, own = False the same operators written out in elementary operations.
"""
import math
import random

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rope(name, runs, direction="forward", head_dim=128, rot_dim=128, layout="half", q_type="bf16", k_type="bf16", base=10000.0,
          scaling="none", scale=1.0, segments=1, first=0, fused=False):
    return {"name": name, "op": "rope", "direction": direction, "runs": runs, "head_dim": head_dim, "rot_dim": rot_dim,
            "layout": layout, "q_type": q_type, "k_type": k_type, "base": base, "scaling": scaling, "scale": scale,
            "segments": segments, "first": first, "fused": fused}


def _norm(name, direction, rows, dim, heads=0, kind="layer", dtype="bf16", w_type="f32", bias=True, fused=False):
    return {"name": name, "op": "norm", "direction": direction, "rows": rows, "heads": heads, "dim": dim, "kind": kind,
            "type": dtype, "w_type": w_type, "bias": bias, "fused": fused}


def _glu(name, direction, rows, dim, ff, act="silu", saved=True):
    return {"name": name, "op": "glu", "direction": direction, "rows": rows, "dim": dim, "ff": ff, "act": act, "saved": saved}


def listed():
    return [
        # a micro-batch of four short sequences of a small model: launches and host time count
        _rope("rope_small", "960@8/2", segments=4),
        # one GPU's token slices at degree 8, cut out of the output of a joint q, k, v projection; half of each head is
        # rotated, in neighbouring pairs; ragged sequences
        _rope("rope_slice_interleaved", "53001@32/4", rot_dim=64, layout="interleaved", segments=13, first=49152, fused=True),
        # the 393,216-token sequence at degree 8 beside its degree-1 tail, frequencies by parts for the long context
        _rope("rope_nested_shard", "393216@4/1; 32768@32/4", base=1e6, scaling="parts", scale=8.0),
        # the way back of a batch of equal sequences: gradients in the types the attention's backward pass leaves them in
        _rope("rope_gradients", "131072@32/4", "backward", k_type="f32", base=5e5, scaling="linear", scale=4.0, segments=16),
        # hidden states of a small micro-batch
        _norm("norm_small", "forward", 333, 2048),
        # hidden states of 32,768 tokens, the way there and the way back with both parameters' gradients
        _norm("norm_hidden", "forward", 32768, 4096),
        _norm("norm_hidden_backward", "backward", 32768, 4096),
        # queries and keys normalised head by head inside the joint projection's output: 2.1 million rows of 128
        _norm("norm_heads_backward", "backward", 57344, 128, heads=36, kind="rms", w_type="bf16", bias=False, fused=True),
        # a small micro-batch against the weights of a small model: the weights' bytes count
        _glu("glu_small", "forward", 77, 1024, 2816),
        # 16,384 tokens of a model with 32 heads of 128, the way there with what the way back needs
        _glu("glu_hidden", "forward", 16384, 4096, 12288),
        # odd sizes, the other activation
        _glu("glu_odd_backward", "backward", 4099, 2056, 5512, act="gelu"),
        # the largest: the way back of 16,384 tokens
        _glu("glu_hidden_backward", "backward", 16384, 4096, 12288),
    ]


def draw(rng):
    """Another call of the same ranges."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    while True:
        direction = rng.choice(["forward", "backward"])
        op = rng.choice(["rope", "norm", "glu"])
        if op == "rope":
            head_dim = rng.choice([64, 128, 128])
            heads = [rng.choice([(8, 2), (32, 4), (32, 4), (64, 4), (16, 16)])]
            if rng.random() < 0.4:  # a node of a higher degree in front
                d = rng.choice([2, 4, 8])
                heads.insert(0, (heads[0][0] // d, max(1, heads[0][1] // d)))
            runs = "; ".join("%d@%d/%d" % (log(1, 393216), q, k) for q, k in heads)
            scaling = rng.choice(["none", "none", "linear", "parts"])
            layout = rng.choice(["half", "half", "interleaved"])
            c = _rope("", runs, direction, head_dim, rng.choice([head_dim, head_dim, head_dim // 2, 24, 2 * rng.randint(1, head_dim // 2)]),
                      layout, rng.choice(["bf16", "bf16", "f32"]), rng.choice(["bf16", "f32"]), rng.choice([1e4, 5e5, 1e6]), scaling,
                      1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]), rng.randint(1, 40), rng.choice([0, 0, log(1, 1 << 20)]),
                      rng.random() < 0.3)
            if c["fused"]:
                c["k_type"] = c["q_type"]  # one projection, one type
        elif op == "norm":
            heads = rng.choice([0, 0, 0, 5, 10, 36])
            c = _norm("", direction, log(1, 65536), rng.choice([64, 128, 128]) if heads else log(48, 16384), heads,
                      rng.choice(["layer", "rms"]), rng.choice(["bf16", "bf16", "f32"]), rng.choice(["bf16", "f32"]), rng.random() < 0.6,
                      rng.random() < 0.3)
            if not heads and rng.random() < 0.7:
                c["dim"] = max(64, c["dim"] // 64 * 64)
        else:
            unit = rng.choice([8, 64])
            c = _glu("", direction, log(1, 16384), unit * log(max(1, 128 // unit), 5120 // unit), unit * log(max(1, 256 // unit), 14336 // unit),
                     rng.choice(["silu", "silu", "gelu"]), rng.random() < 0.5)
        if work(c)["bytes"] <= 3.0e9 and work(c)["flops"] <= 6.6e12:
            del c["name"]
            return c


# ---- from a case to its call
def _runs(case):
    for r in case["runs"].split(";"):
        tokens, heads = r.split("@")
        hq, hkv = heads.split("/")
        yield int(tokens), int(hq), int(hkv)


def _frequencies(case):
    """Radians per position of each rotated pair (64 bits), and the factor on cosine and sine."""
    rot, base, s = case["rot_dim"], case["base"], case["scale"]
    f = base ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    if case["scaling"] == "linear":  # positions pressed together
        return f / s, 1.0
    if case["scaling"] == "parts":  # slow pairs pressed together, fast ones left, a ramp between 32 turns and 1 in 32,768 tokens
        pair_of = lambda turns: rot * math.log(32768 / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair_of(32.0)), 0), min(math.ceil(pair_of(1.0)), rot - 1)
        keep = 1 - np.clip((np.arange(rot // 2) - lo) / max(hi - lo, 1e-3), 0, 1)
        return f / s * (1 - keep) + f * keep, 0.1 * math.log(s) + 1.0
    return f, 1.0


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))

    def normal(shape, dtype, scale=1.0, mean=0.0):
        t = torch.empty(shape, dtype=dtype, device=DEVICE)
        flat = t.view(-1)
        for a in range(0, flat.numel(), 1 << 26):
            n = min(1 << 26, flat.numel() - a)
            flat[a:a + n] = torch.randn(n, generator=g, device=DEVICE) * scale + mean
        return t

    s = {"case": case, "kept": {}}
    if case["op"] == "rope":
        D = case["head_dim"]
        s["inv_freq"], s["magnitude"] = _frequencies(case)
        s["x"], s["positions"], s["y"] = [], [], []
        rng = random.Random(int(seed))
        for tokens, hq, hkv in _runs(case):
            cuts = sorted(rng.randint(0, tokens) for _ in range(case["segments"] - 1))
            pos = torch.arange(tokens, device=DEVICE)
            for a, b in zip(cuts, cuts[1:] + [tokens]):
                pos[a:b] = torch.arange(b - a, device=DEVICE)
            pos += case["first"]
            if case["fused"]:  # views into the joint projection's output
                qkv = normal((tokens, hq + 2 * hkv, D), TYPES[case["q_type"]])
                s["x"] += [qkv[:, :hq], qkv[:, hq:hq + hkv]]
            else:
                s["x"] += [normal((tokens, hq, D), TYPES[case["q_type"]]), normal((tokens, hkv, D), TYPES[case["k_type"]])]
            s["positions"] += [pos, pos]
        s["y"] = [torch.empty(x.shape, dtype=x.dtype, device=DEVICE) for x in s["x"]]
    elif case["op"] == "norm":
        rows, heads, dim, dt = case["rows"], case["heads"], case["dim"], TYPES[case["type"]]
        shape = (rows, heads, dim) if heads else (rows, dim)
        if case["fused"]:  # views into rows that are half as long again
            more = (rows, heads + heads // 2 + 1, dim) if heads else (rows, dim + 8 * (dim // 16) + 8)
            whole = normal(more, dt, 1.5, 0.25)
            s["x"] = whole[:, :heads] if heads else whole[:, :dim]
        else:
            s["x"] = normal(shape, dt, 1.5, 0.25)
        s["weight"] = normal((dim,), TYPES[case["w_type"]], 0.2, 1.0)
        s["bias"] = normal((dim,), TYPES[case["w_type"]], 0.1) if case["bias"] else None
        s["eps"] = 1e-5
        empty = lambda shape, t: torch.empty(shape, dtype=t, device=DEVICE)
        if case["direction"] == "forward":
            s["y"] = empty(shape, dt)
            s["mean"] = empty(shape[:-1], torch.float32) if case["kind"] == "layer" else None
            s["rstd"] = empty(shape[:-1], torch.float32)
        else:
            x = s["x"].double()
            mean = x.mean(-1) if case["kind"] == "layer" else None
            centred = x - mean[..., None] if mean is not None else x
            s["rstd"] = (centred.square().mean(-1) + s["eps"]).rsqrt().float()
            s["mean"] = mean.float() if mean is not None else None
            s["dy"] = normal(shape, dt)
            s["dx"] = empty(shape, dt)
            s["dweight"], s["dbias"] = empty((dim,), torch.float32), empty((dim,), torch.float32) if case["bias"] else None
    else:
        rows, dim, ff, bf = case["rows"], case["dim"], case["ff"], torch.bfloat16
        empty = lambda *shape: torch.empty(shape, dtype=bf, device=DEVICE)
        s["x"] = normal((rows, dim), bf)
        s["w_gate"], s["w_up"] = normal((ff, dim), bf, dim ** -0.5), normal((ff, dim), bf, dim ** -0.5)
        if case["direction"] == "forward":
            s["h"] = empty(rows, ff)
            s["g"], s["u"] = (empty(rows, ff), empty(rows, ff)) if case["saved"] else (None, None)
        else:
            s["g"], s["u"], s["dh"] = normal((rows, ff), bf), normal((rows, ff), bf), normal((rows, ff), bf)
            s["dx"], s["dw_gate"], s["dw_up"] = empty(rows, dim), empty(ff, dim), empty(ff, dim)
    return s


def _workspace(s, nbytes):
    """The workspace that a program keeps from step to step."""
    if s["kept"].get("ws") is None:
        s["kept"]["ws"] = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=DEVICE)
    return s["kept"]["ws"]


def run(s):
    case = s["case"]
    there = case["direction"] == "forward"
    if own:
        from paper_2609_22755_b200 import binding as B

        if case["op"] == "rope":
            layout = B.NSP_ROPE_HALF if case["layout"] == "half" else B.NSP_ROPE_INTERLEAVED
            B.nsp_rope(s["x"], s["y"], s["positions"], s["inv_freq"], layout=layout, magnitude=s["magnitude"], inverse=not there)
            return s["y"]
        if case["op"] == "norm":
            kind = B.NSP_NORM_LAYER if case["kind"] == "layer" else B.NSP_NORM_RMS
            if there:
                B.nsp_norm_fwd(s["x"], s["weight"], s["bias"], s["y"], s["mean"], s["rstd"], eps=s["eps"], kind=kind)
                return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
            ws = _workspace(s, B.nsp_norm_bwd_ws_bytes(s["rstd"].numel(), case["dim"]))
            B.nsp_norm_bwd(s["x"], s["dy"], s["weight"], s["mean"], s["rstd"], s["dx"], s["dweight"], s["dbias"], ws, kind=kind)
            return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
        act = B.NSP_ACT_SILU if case["act"] == "silu" else B.NSP_ACT_GELU
        if there:
            B.nsp_glu_fwd(s["x"], s["w_gate"], s["w_up"], s["h"], s["g"], s["u"], act=act)
            return {"h": s["h"], "g": s["g"], "u": s["u"]}
        ws = _workspace(s, B.nsp_glu_bwd_ws_bytes(case["rows"], case["dim"], case["ff"]))
        B.nsp_glu_bwd(s["dh"], s["x"], s["w_gate"], s["w_up"], s["g"], s["u"], s["dx"], s["dw_gate"], s["dw_up"], ws, act=act)
        return {"dx": s["dx"], "dw_gate": s["dw_gate"], "dw_up": s["dw_up"]}
    if case["op"] == "rope":
        return _plain_rope(s, case, there)
    if case["op"] == "norm":
        return _plain_norm_forward(s, case) if there else _plain_norm_backward(s, case)
    return _plain_glu_forward(s, case) if there else _plain_glu_backward(s, case)


# ---- the operators in elementary operations, in 32 bits (angles in 64)
def _plain_rope(s, case, there):
    rot, half = case["rot_dim"], case["rot_dim"] // 2
    freq = torch.from_numpy(s["inv_freq"]).to(DEVICE)
    outs = []
    for x, pos in zip(s["x"], s["positions"]):
        angle = pos.double()[:, None] * freq
        cos = (torch.cos(angle) * s["magnitude"]).float()[:, None]
        sin = (torch.sin(angle) * (s["magnitude"] if there else -s["magnitude"])).float()[:, None]
        v = x[..., :rot].float()
        if case["layout"] == "half":
            a, b = v[..., :half], v[..., half:]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        else:
            a, b = v[..., 0::2], v[..., 1::2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        outs.append(torch.cat([turned.to(x.dtype), x[..., rot:]], -1))
    return outs


def _plain_norm_forward(s, case):
    x = s["x"].float()
    mean = x.mean(-1, keepdim=True) if case["kind"] == "layer" else None
    centred = x - mean if mean is not None else x
    rstd = (centred.square().mean(-1, keepdim=True) + s["eps"]).rsqrt()
    y = centred * rstd * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return {"y": y.to(s["x"].dtype), "mean": mean[..., 0] if mean is not None else None, "rstd": rstd[..., 0]}


def _plain_norm_backward(s, case):
    x, dy, w = s["x"].float(), s["dy"].float(), s["weight"].float()
    hat = (x - s["mean"][..., None] if s["mean"] is not None else x) * s["rstd"][..., None]
    wdy = dy * w
    dx = wdy - hat * (wdy * hat).mean(-1, keepdim=True)
    if case["kind"] == "layer":
        dx = dx - wdy.mean(-1, keepdim=True)
    every = tuple(range(x.dim() - 1))
    return {"dx": (dx * s["rstd"][..., None]).to(s["x"].dtype), "dweight": (dy * hat).sum(every),
            "dbias": dy.sum(every) if s["dbias"] is not None else None}


def _plain_glu_forward(s, case):
    x = s["x"].float()
    g, u = x @ s["w_gate"].float().t(), x @ s["w_up"].float().t()
    a = g / (1 + torch.exp(-g)) if case["act"] == "silu" else 0.5 * g * (1 + torch.erf(g * 2 ** -0.5))
    h, bf = a * u, torch.bfloat16
    return {"h": h.to(bf), "g": g.to(bf) if s["g"] is not None else None, "u": u.to(bf) if s["u"] is not None else None}


def _plain_glu_backward(s, case):
    g, u, dh, x, bf = s["g"].float(), s["u"].float(), s["dh"].float(), s["x"].float(), torch.bfloat16
    if case["act"] == "silu":
        p = 1 / (1 + torch.exp(-g))
        a, slope = g * p, p * (1 + g * (1 - p))
    else:
        p = 0.5 * (1 + torch.erf(g * 2 ** -0.5))
        a, slope = g * p, p + g * torch.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5
    dg, du = dh * u * slope, dh * a
    dx = dg @ s["w_gate"].float() + du @ s["w_up"].float()
    return {"dx": dx.to(bf), "dw_gate": (dg.t() @ x).to(bf), "dw_up": (du.t() @ x).to(bf)}


def work(case):
    there = case["direction"] == "forward"
    size = {"bf16": 2, "f32": 4}
    if case["op"] == "rope":
        moved, pairs = 0, 0
        for tokens, hq, hkv in _runs(case):
            moved += tokens * case["head_dim"] * 2 * (hq * size[case["q_type"]] + hkv * size[case["k_type"]]) + 8 * tokens
            pairs += tokens * (hq + hkv) * case["rot_dim"] // 2
        return {"bytes": moved, "flops": 6 * pairs}
    if case["op"] == "norm":
        rows = case["rows"] * max(case["heads"], 1)
        values, per_row = rows * case["dim"], rows * (8 if case["kind"] == "layer" else 4)
        params = case["dim"] * size[case["w_type"]] * (2 if case["bias"] and there else 1)
        grads = 0 if there else case["dim"] * 4 * (2 if case["bias"] else 1)
        return {"bytes": values * size[case["type"]] * (2 if there else 3) + per_row + params + grads, "flops": values * (8 if there else 14)}
    rows, dim, ff = case["rows"], case["dim"], case["ff"]
    wide = (3 if case["saved"] else 1) if there else 3
    return {"bytes": 2 * (rows * ff * wide + rows * dim * (1 if there else 2) + ff * dim * (2 if there else 4)),
            "flops": (4 if there else 8) * rows * dim * ff + rows * ff * 8}


# ---- the operators' definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    there = case["direction"] == "forward"
    if case["op"] == "rope":  # a pair as a complex number, turned by exp(i * position * frequency)
        rot, outs = case["rot_dim"], []
        for x, pos in zip(s["x"], s["positions"]):
            phase = torch.outer(pos.to(torch.float64), torch.as_tensor(s["inv_freq"], dtype=torch.float64, device=DEVICE))
            turn = torch.polar(torch.full_like(phase, s["magnitude"]), phase if there else -phase).unsqueeze(1)
            out = x.to(torch.float64)
            pairs = out[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2) if case["layout"] == "half" else out[..., :rot].unflatten(-1, (rot // 2, 2))
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            out[..., :rot] = (z.transpose(-1, -2) if case["layout"] == "half" else z).flatten(-2)
            outs.append(out)
        return outs
    d = {k: v.to(torch.float64) for k, v in s.items() if isinstance(v, torch.Tensor)}
    if case["op"] == "norm":
        x, n = d["x"], case["dim"]
        if there:
            mean = x.sum(-1) / n if case["kind"] == "layer" else torch.zeros_like(x[..., 0])
            rstd = 1 / torch.sqrt(((x - mean.unsqueeze(-1)) ** 2).sum(-1) / n + s["eps"])
            y = torch.einsum("...d,...,d->...d", x - mean.unsqueeze(-1), rstd, d["weight"])
            return {"y": y + d["bias"] if case["bias"] else y, "mean": mean if case["kind"] == "layer" else None, "rstd": rstd}
        x, dy = x.reshape(-1, n), d["dy"].reshape(-1, n)
        centre = d["mean"].reshape(-1, 1) if case["kind"] == "layer" else 0.0
        r = d["rstd"].reshape(-1, 1)
        hat, t = (x - centre) * r, dy * d["weight"]
        dx = t - hat * torch.einsum("rd,rd->r", t, hat).unsqueeze(-1) / n
        if case["kind"] == "layer":
            dx -= t.sum(-1, keepdim=True) / n
        return {"dx": (dx * r).reshape(s["dx"].shape), "dweight": torch.einsum("rd,rd->d", dy, hat), "dbias": dy.sum(0) if case["bias"] else None}
    wg, wu, x = d["w_gate"], d["w_up"], d["x"]
    cdf = lambda t: 0.5 * torch.erfc(-t / math.sqrt(2.0))
    if there:
        g, u = torch.einsum("td,fd->tf", x, wg), torch.einsum("td,fd->tf", x, wu)
        h = (g * torch.sigmoid(g) if case["act"] == "silu" else g * cdf(g)) * u
        return {"h": h, "g": g if case["saved"] else None, "u": u if case["saved"] else None}
    g, u, dh = d["g"], d["u"], d["dh"]
    if case["act"] == "silu":
        slope = torch.sigmoid(g) + g * torch.sigmoid(g) * torch.sigmoid(-g)
        value = g * torch.sigmoid(g)
    else:
        slope = cdf(g) + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        value = g * cdf(g)
    dg, du = dh * slope * u, dh * value
    return {"dx": torch.einsum("tf,fd->td", dg, wg) + torch.einsum("tf,fd->td", du, wu),
            "dw_gate": torch.einsum("tf,td->fd", dg, x), "dw_up": torch.einsum("tf,td->fd", du, x)}
