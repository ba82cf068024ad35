"""Operators beside the routed FFN layer's own: the scored router and microscaled 4-bit experts, as a program calls them.

A case is a dict of plain values.  `op` says which operator it times:
  route      token-choice routing by softmax or sigmoid scores, with a selection bias, expert groups and renormalised weights
  route_bwd  its backward pass: gradients of the gate weights to gradients of the logits
  quantize   rows to blocks of 32 four-bit values with a shared power-of-two scale (MXFP4), and back
  ffn        the grouped SwiGLU FFN on MXFP4 weights: activations quantised on the way, rows read in expert order from token order
Logits are N(0,1) with a Zipf bias over the experts, activations N(0,1), weights N(0, 0.02^2).
"""
import math

import torch

own = False


def listed():
    return [
        # One token of a decode step through a Mixtral-shaped layer's router: latency alone.
        dict(name="route_one_token", op="route", T=1, E=8, k=2, score="softmax", groups=1, top_groups=1, group_best=1, renormalize=True, scale=1.0, bias=False),
        # 256 experts in eight groups, sigmoid scores, the balancing bias: two sequences of a training step.
        dict(name="route_groups", op="route", T=4096, E=256, k=8, score="sigmoid", groups=8, top_groups=4, group_best=2, renormalize=True, scale=2.5, bias=True),
        # An odd token count, a number of experts and a group size that are no powers of two, weights as the softmax gives them.
        dict(name="route_odd", op="route", T=3001, E=60, k=6, score="softmax", groups=5, top_groups=2, group_best=1, renormalize=False, scale=1.0, bias=False),
        # A large batch on the widest expert list of the layer itself.
        dict(name="route_large", op="route", T=65536, E=64, k=8, score="sigmoid", groups=1, top_groups=1, group_best=1, renormalize=True, scale=1.0, bias=True),
        dict(name="route_bwd_odd", op="route_bwd", T=3001, E=60, k=6, score="softmax", groups=5, top_groups=2, group_best=1, renormalize=False, scale=1.0, bias=False),
        dict(name="route_bwd_large", op="route_bwd", T=65536, E=256, k=8, score="sigmoid", groups=8, top_groups=4, group_best=2, renormalize=True, scale=2.5, bias=True),
        # Activations of a prompt of odd length, rows that end inside a block.
        dict(name="quantize_rows", op="quantize", dtype="bf16", n=1, rows=1003, K=1032),
        # One weight tensor of a Mixtral-shaped layer from its fp32 masters: done once for a model.
        dict(name="quantize_weights", op="quantize", dtype="f32", n=8, rows=14336, K=4096),
        # One token, two of eight experts: the weights of two experts are read once.
        dict(name="ffn_one_token", op="ffn", T=1, H=4096, F=14336, E=8, k=2, zipf=1.1),
        # One decode step of 32 sequences: every expert's weights are read once.
        dict(name="ffn_decode", op="ffn", T=32, H=4096, F=14336, E=8, k=2, zipf=1.1),
        # Many small experts with some hundred rows each, sizes off every tile boundary.
        dict(name="ffn_many_ragged", op="ffn", T=1999, H=2056, F=1032, E=64, k=8, zipf=1.1),
        # Prefill of two sequences of 2048 tokens: the largest product.
        dict(name="ffn_prefill", op="ffn", T=4096, H=4096, F=14336, E=8, k=2, zipf=1.1),
    ]


MAX_FLOPS, MAX_WEIGHTS = 2.8e12, 4.6e8  # a drawn product stays below the largest listed one


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A feature size: half the time a multiple of 128, as models have them, else any multiple of 8."""
    v = _log(rng, lo, hi)
    step = 128 if v >= 128 and rng.random() < 0.5 else 8
    return min(hi, max(step, v // step * step))


def draw(rng):
    while True:
        op = rng.choice(["route", "route", "route_bwd", "quantize", "ffn", "ffn", "ffn"])
        if op in ("route", "route_bwd"):
            groups = rng.choice([1, 1, 2, 3, 4, 8, 16])
            size = _log(rng, 2, max(2, 256 // groups))
            top = rng.randint(1, groups)
            E = groups * size
            return dict(op=op, T=_log(rng, 1, 65536), E=E, k=rng.randint(1, min(8, top * size)), score=rng.choice(["softmax", "sigmoid"]),
                        groups=groups, top_groups=top, group_best=rng.choice([1, 2]), renormalize=rng.random() < 0.7,
                        scale=rng.choice([1.0, 2.5]), bias=rng.random() < 0.6)
        if op == "quantize":
            c = dict(op=op, dtype=rng.choice(["bf16", "f32"]), n=rng.randint(1, 8), rows=_log(rng, 1, 16384), K=_size(rng, 32, 14336))
            if c["n"] * c["rows"] * c["K"] <= MAX_WEIGHTS:
                return c
        else:
            E = _log(rng, 1, 64)
            c = dict(op=op, T=_log(rng, 1, 8192), H=_size(rng, 128, 4096), F=_size(rng, 128, 14336), E=E,
                     k=rng.randint(1, min(E, 8)), zipf=round(rng.uniform(0.0, 2.0), 2))
            if 6 * c["T"] * c["k"] * c["H"] * c["F"] <= MAX_FLOPS and E * c["H"] * c["F"] <= MAX_WEIGHTS:
                return c


def _ceil(a, b):
    return -(-a // b)


def _packed_bytes(rows, K):
    return _ceil(rows, 16) * (_ceil(K, 128) * 1024 + _ceil(K, 512) * 256)


def work(case):
    c = case
    if c["op"] == "route":
        return {"bytes": 4 * c["T"] * c["E"] + 8 * c["T"] * c["k"], "flops": 8 * c["T"] * c["E"]}
    if c["op"] == "route_bwd":
        return {"bytes": 8 * c["T"] * c["E"] + 8 * c["T"] * c["k"], "flops": 8 * c["T"] * c["E"]}
    if c["op"] == "quantize":
        v = c["n"] * c["rows"] * c["K"]  # read, the packed form written and read, written
        return {"bytes": 2 * v * (2 if c["dtype"] == "bf16" else 4) + 2 * v * 17 // 32, "flops": 6 * v}
    R = c["T"] * c["k"]
    used = min(c["E"], R)
    return {"bytes": used * 3 * c["H"] * c["F"] * 17 // 32 + 2 * (c["T"] + R) * c["H"], "flops": 6 * R * c["H"] * c["F"]}


# ---- inputs ------------------------------------------------------------------------------------------------------------

# the four-bit codes in order: sign in the top bit, then the magnitude's place among these values
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _block_scale(amax):
    """floor(log2(amax)) - 2 in [-127, 127]; -127 for a block of zeros."""
    e = torch.frexp(amax).exponent - 3
    return torch.where(amax > 0, e, torch.full_like(e, -127)).clamp(-127, 127)


def _power_of_two(e):
    """2^e in 32 bits for e in [-127, 127]: a library's power or ldexp may be off by a rounding."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _blocks(x):
    """x [..., K] as [..., ceil(K / 32), 32], zeros behind the end."""
    K = x.shape[-1]
    return torch.nn.functional.pad(x, (0, -K % 32)).unflatten(-1, (-1, 32))


def _on_grid(v):
    """|v| / scale to the nearest of MAGNITUDES, ties to the even code; the step is 1/2 below 2, 1 below 4, 2 above."""
    step = torch.where(v < 2, 0.5, torch.where(v < 4, 1.0, 2.0))
    return torch.clamp(torch.round(v / step) * step, max=6.0)


def _quantized(x):
    """x [..., K] in 32 bits -> the values that its MXFP4 form stands for."""
    b = _blocks(x)
    scale = _power_of_two(_block_scale(b.abs().amax(-1, keepdim=True)))
    return (torch.sign(b) * _on_grid((b / scale).abs()) * scale).flatten(-2)[..., : x.shape[-1]]


def _pack(w):
    """One matrix [rows, K] in its packed form: codes of 16 rows x 128 values in 1 KiB tiles, 16 bytes for a row's block of
    32, the blocks' rows side by side; behind them the scales of 16 rows x 512 values in 256 bytes."""
    rows, K = w.shape
    b = _blocks(w)
    e = _block_scale(b.abs().amax(-1))
    v = _on_grid((b / _power_of_two(e)[..., None]).abs())
    code = torch.where(v < 2, v * 2, torch.where(v < 4, v + 2, v * 0.5 + 4)).to(torch.uint8) + (b < 0).to(torch.uint8) * 8
    code = (code[..., 0::2] + code[..., 1::2] * 16).flatten(1)
    code = torch.nn.functional.pad(code, (0, -code.shape[1] % 64, 0, -rows % 16))
    scale = (e + 127).to(torch.uint8)
    scale = torch.nn.functional.pad(scale, (0, -scale.shape[1] % 16, 0, -rows % 16))
    code = code.view(code.shape[0] // 16, 16, -1, 4, 16).permute(0, 2, 3, 1, 4)
    scale = scale.view(scale.shape[0] // 16, 16, -1, 4, 4).permute(0, 2, 4, 1, 3)
    return torch.cat([code.reshape(-1), scale.reshape(-1)])


def _zipf(E, s, dev):
    return torch.arange(1, E + 1, device=dev, dtype=torch.float32) ** -s


def prepare(case, seed):
    c, dev = case, "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device=dev)  # noqa: E731
    s = dict(case=c)
    if c["op"] in ("route", "route_bwd"):
        T, E, k = c["T"], c["E"], c["k"]
        s["logits"] = normal(T, E) + _zipf(E, 1.1, dev)
        # a bias that has been steered for a while: small beside the scores, against the frequent experts
        s["bias"] = 0.02 * normal(E) - 0.05 * _zipf(E, 1.1, dev) if c["bias"] else None
        s["expert_idx"] = torch.empty((T, k), dtype=torch.int32, device=dev)
        s["gate_w"] = torch.empty((T, k), device=dev)
        if c["op"] == "route_bwd":
            s["expert_idx"] = _route(c, s["logits"], s["bias"])[0]
            s["dgate"] = normal(T, k)
            s["dlogits"] = torch.empty((T, E), device=dev)
        return s
    if c["op"] == "quantize":
        td = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        s["src"] = (0.02 * normal(c["n"], c["rows"], c["K"])).to(td)
        s["packed"] = torch.empty((c["n"], _packed_bytes(c["rows"], c["K"])), dtype=torch.uint8, device=dev)
        s["values"] = torch.empty_like(s["src"])
        return s
    T, H, F, E, k = (c[n] for n in ("T", "H", "F", "E", "k"))
    s["x"] = normal(T, H).bfloat16()
    for name, rows, K in (("Wg", F, H), ("Wu", F, H), ("Wd", H, F)):
        w = torch.empty((E, _packed_bytes(rows, K)), dtype=torch.uint8, device=dev)
        for e in range(E):
            w[e] = _pack(0.02 * normal(rows, K))
        s[name] = w
    # the permutation of the routed slots: sorted by expert, in their order within one
    chosen = torch.topk(normal(T, E) + _zipf(E, c["zipf"], dev), k).indices.reshape(-1)
    order = torch.argsort(chosen, stable=True)
    counts = torch.bincount(chosen, minlength=E)
    s["src_slot"] = order.to(torch.int32)
    s["seg_offsets"] = torch.cat([counts.new_zeros(1), torch.cumsum(counts, 0)]).to(torch.int32)
    s["most"] = int(counts.max())
    s["y_p"] = torch.empty((T * k, H), dtype=torch.bfloat16, device=dev)
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------------------


def _scores(c, logits):
    """In 64 bits: which of two experts is ahead is decided by the scores, not by their rounding."""
    z = logits.double()
    if c["score"] == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    p = torch.exp(z - z.amax(-1, keepdim=True))
    return p / p.sum(-1, keepdim=True)


def _route(c, logits, bias):
    T, E = logits.shape
    s = _scores(c, logits)
    v = s if bias is None else s + bias.double()
    if c["groups"] > 1:
        by_group = v.view(T, c["groups"], -1)
        best = torch.sort(by_group, dim=-1, descending=True).values[..., : c["group_best"]].sum(-1)
        stay = torch.sort(best, dim=-1, descending=True, stable=True).indices[:, : c["top_groups"]]
        keep = torch.zeros_like(best, dtype=torch.bool).scatter_(1, stay, True)
        v = torch.where(keep[..., None], by_group, -math.inf).view(T, E)
    idx = torch.sort(v, dim=-1, descending=True, stable=True).indices[:, : c["k"]]
    w = s.gather(1, idx)
    if c["renormalize"]:
        w = w / w.sum(-1, keepdim=True)
    return idx.to(torch.int32), (w * c["scale"]).float()


def _route_bwd(c, dgate, logits, expert_idx):
    s = _scores(c, logits)
    idx = expert_idx.long()
    w, d = s.gather(1, idx), dgate.double() * c["scale"]
    if c["renormalize"]:
        total = w.sum(-1, keepdim=True)
        d = (d - (d * w).sum(-1, keepdim=True) / total) / total
    ds = torch.zeros_like(s).scatter_add_(1, idx, d)
    if c["score"] == "sigmoid":
        return (ds * s * (1 - s)).float()
    return (s * (ds - (ds * s).sum(-1, keepdim=True))).float()


def _unpack(packed, rows, K):
    """[E, bytes] -> the values [E, rows, K] in 32 bits."""
    E, R, Kb = packed.shape[0], _ceil(rows, 16), _ceil(K, 128)
    code = packed[:, : R * Kb * 1024].view(E, R, Kb, 4, 16, 16).permute(0, 1, 4, 2, 3, 5)
    code = torch.stack([code & 15, code >> 4], -1).reshape(E, R * 16, Kb * 4, 32)
    scale = packed[:, R * Kb * 1024 :].view(E, R, -1, 4, 16, 4).permute(0, 1, 4, 2, 5, 3).reshape(E, R * 16, -1)[:, :, : Kb * 4]
    table = torch.tensor(MAGNITUDES + tuple(-v for v in MAGNITUDES), device=packed.device)
    value = table[code.int()] * _power_of_two(scale.int() - 127)[..., None]
    return value.reshape(E, R * 16, Kb * 128)[:, :rows, :K]


def _ffn(c, s):
    H, F, E, most = c["H"], c["F"], c["E"], s["most"]
    seg = s["seg_offsets"].long()
    row = torch.arange(s["src_slot"].shape[0], device=seg.device)
    expert = torch.searchsorted(seg[1:], row, right=True)
    place = expert * most + row - seg[expert]
    x = torch.zeros((E * most, H), device=seg.device)
    x[place] = _quantized(s["x"].float())[s["src_slot"].long() // c["k"]]
    x = x.view(E, most, H)
    g = torch.bmm(x, _unpack(s["Wg"], F, H).transpose(1, 2).contiguous())
    u = torch.bmm(x, _unpack(s["Wu"], F, H).transpose(1, 2).contiguous())
    a = _quantized(g / (1 + torch.exp(-g)) * u)
    y = torch.bmm(a, _unpack(s["Wd"], H, F).transpose(1, 2).contiguous())
    return y.view(E * most, H)[place].to(s["x"].dtype)


def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(c, s)
    if c["op"] == "route":
        return _route(c, s["logits"], s["bias"])
    if c["op"] == "route_bwd":
        return _route_bwd(c, s["dgate"], s["logits"], s["expert_idx"])
    if c["op"] == "quantize":
        return _quantized(s["src"].float()).to(s["src"].dtype)
    return _ffn(c, s)


# ---- the framework's calls -------------------------------------------------------------------------------------------------


def _run_own(c, s):
    from paper_2505_14864_amd import binding as B
    if "d" not in s and c["op"] != "quantize":  # the descriptors and the workspace that a program keeps
        if c["op"] in ("route", "route_bwd"):
            s["d"] = B.make_desc(c["T"], 8, 8, c["E"], c["k"], "bf16")
            s["rule"] = B.make_rule(c["score"], groups=c["groups"], top_groups=c["top_groups"], group_best=c["group_best"],
                                    renormalize=c["renormalize"], scale=c["scale"])
        else:
            s["d"] = B.make_desc(c["T"], c["H"], c["F"], c["E"], c["k"], "bf16")
            s["workspace"] = torch.empty(B.dynmo_grouped_ffn_mxfp4_workspace_bytes(s["d"]), dtype=torch.uint8, device="cuda")
    if c["op"] == "route":
        B.dynmo_route_scored(s["d"], s["rule"], s["logits"], s["bias"], s["expert_idx"], s["gate_w"])
        return s["expert_idx"], s["gate_w"]
    if c["op"] == "route_bwd":
        B.dynmo_route_scored_bwd(s["d"], s["rule"], s["dgate"], s["logits"], s["expert_idx"], s["dlogits"])
        return s["dlogits"]
    if c["op"] == "quantize":
        B.dynmo_mxfp4_quantize(s["src"], s["packed"])
        B.dynmo_mxfp4_dequantize(s["packed"], s["values"])
        return s["values"]
    B.dynmo_grouped_ffn_mxfp4(s["d"], s["x"], s["src_slot"], s["seg_offsets"], s["Wg"], s["Wu"], s["Wd"], s["y_p"], None, None, s["workspace"])
    return s["y_p"]


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------


def _exact_route(c, logits, bias):
    z = logits.double()
    s = torch.sigmoid(z) if c["score"] == "sigmoid" else torch.softmax(z, -1)
    T, E = z.shape
    v = s.clone() if bias is None else s + bias.double()[None]
    size = E // c["groups"]
    alive = torch.ones_like(v, dtype=torch.bool)
    if c["groups"] > 1:
        best = torch.stack([v[:, i * size : (i + 1) * size].topk(min(size, c["group_best"]), -1).values.sum(-1) for i in range(c["groups"])], -1)
        alive[:] = False
        for _ in range(c["top_groups"]):
            at = best.argmax(-1)
            alive |= (torch.arange(E, device=z.device)[None] // size) == at[:, None]
            best[torch.arange(T, device=z.device), at] = -math.inf
    v[~alive] = -math.inf
    chosen = []
    for _ in range(c["k"]):
        chosen.append((v == v.amax(-1, keepdim=True)).int().argmax(-1))  # the first of equal ones
        v[torch.arange(T, device=z.device), chosen[-1]] = -math.inf
    idx = torch.stack(chosen, -1)
    w = torch.gather(s, 1, idx)
    return s, idx, (w / w.sum(-1, keepdim=True) if c["renormalize"] else w) * c["scale"]


def _exact_route_bwd(c, s, idx, dgate):
    w, d = torch.gather(s, 1, idx), dgate.double()
    if c["renormalize"]:  # the Jacobian of w_i / sum w, a row per slot
        n = w / w.sum(-1, keepdim=True)
        jac = (torch.eye(c["k"], device=w.device, dtype=w.dtype)[None] - n[:, :, None]) / w.sum(-1)[:, None, None]
        d = (d[:, :, None] * jac).sum(1)
    d = d * c["scale"]
    out = torch.zeros_like(s)
    if c["score"] == "sigmoid":
        for j in range(c["k"]):
            out.scatter_add_(1, idx[:, j : j + 1], (d * w * (1 - w))[:, j : j + 1])
        return out
    for j in range(c["k"]):  # d softmax_j / d logits = p_j (delta - p)
        out -= (d[:, j] * w[:, j])[:, None] * s
        out.scatter_add_(1, idx[:, j : j + 1], (d * w)[:, j : j + 1])
    return out


def _exact_power(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_quantized(x):
    x = x.double()
    K = x.shape[-1]
    whole = torch.zeros(x.shape[:-1] + (_ceil(K, 32) * 32,), dtype=torch.float64, device=x.device)
    whole[..., :K] = x
    b = whole.view(x.shape[:-1] + (-1, 32))
    amax = b.abs().amax(-1, keepdim=True)
    unit = _exact_power(torch.floor(torch.log2(torch.where(amax > 0, amax, 1.0))) - 2)
    unit = torch.where(amax < 4 * unit, unit / 2, torch.where(amax >= 8 * unit, unit * 2, unit))  # log2 may round over a power
    v = b.abs() / unit
    # the midpoints between neighbours; one whose lower neighbour has an odd code goes up
    r = torch.zeros_like(v)
    for lower, mid, step, up in ((0.0, 0.25, 0.5, False), (0.5, 0.75, 0.5, True), (1.0, 1.25, 0.5, False), (1.5, 1.75, 0.5, True),
                                 (2.0, 2.5, 1.0, False), (3.0, 3.5, 1.0, True), (4.0, 5.0, 2.0, False)):
        r += step * ((v >= mid) if up else (v > mid))
    return (torch.copysign(r, b) * unit).view(whole.shape)[..., :K]


def _exact_matrix(packed, rows, K):
    """One packed matrix: every value looked up at its place."""
    dev = packed.device
    r, k = torch.arange(rows, device=dev)[:, None], torch.arange(K, device=dev)[None]
    Kb, Kq = _ceil(K, 128), _ceil(K, 512)
    byte = packed[((r // 16) * Kb + k // 128) * 1024 + (k % 128) // 32 * 256 + r % 16 * 16 + k % 32 // 2].int()
    code = torch.where(k % 2 == 1, byte >> 4, byte & 15)
    k = torch.arange(0, K, 32, device=dev)[None]
    exp = packed[_ceil(rows, 16) * Kb * 1024 + ((r // 16) * Kq + k // 512) * 256 + (k % 128) // 32 * 64 + r % 16 * 4 + (k % 512) // 128]
    exp = _exact_power(exp.long() - 127).repeat_interleave(32, 1)[:, :K]
    e, m = (code >> 1) & 3, (code & 1).double()
    mag = torch.where(e == 0, m * 0.5, (1 + m / 2) * (1 << e) / 2)
    return torch.where(code >= 8, -mag, mag) * exp


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "route":
        _, idx, w = _exact_route(c, s["logits"], s["bias"])
        return idx.to(torch.int32), w
    if c["op"] == "route_bwd":
        scores, idx, _ = _exact_route(c, s["logits"], s["bias"])
        return _exact_route_bwd(c, scores, idx, s["dgate"])
    if c["op"] == "quantize":
        return _exact_quantized(s["src"])
    x, y, seg = _exact_quantized(s["x"]), [], s["seg_offsets"].tolist()
    token = s["src_slot"].long() // c["k"]
    for e in range(c["E"]):
        if seg[e] == seg[e + 1]:
            continue
        rows = x[token[seg[e] : seg[e + 1]]]
        g = rows @ _exact_matrix(s["Wg"][e], c["F"], c["H"]).T
        g = g * torch.sigmoid(g)
        g *= rows @ _exact_matrix(s["Wu"][e], c["F"], c["H"]).T
        y.append(_exact_quantized(g) @ _exact_matrix(s["Wd"][e], c["H"], c["F"]).T)
    return torch.cat(y)
