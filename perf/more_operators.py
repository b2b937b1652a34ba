"""Operators of a block served in 4 bits, as timed cases: rows held as 4-bit
floating-point codes with a scale for every 32 values, matrix products of such
rows, rotary positions on queries and keys, and the norms on both sides of a
sub-layer with its gate and residual.

Each case is one pass through an operator of `paper_2608_02474_amd.api` as a
program calls it: a linear layer quantises its input and multiplies, with the
weights' codes in hand; positions turn queries and keys in one call.

own               False: the plain forms in elementary torch; True: the library
listed()          the cases
draw(rng)         one more case of the same ranges
prepare / run     a program's state before the call, and the call
work              bytes and operations of a pass
exact             the outputs in 64 bits
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
BASE = 10000.0
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------- cases

def _quantize(name, M, D, dtype="bf16", ld=0):
    """M rows of D values (rows `ld` apart; 0: contiguous) to codes and back."""
    return {"name": name, "kind": "quantize", "M": M, "D": D, "dtype": dtype, "ld": ld}


def _linear(name, M, N, K, dtype="bf16", act="none", ln=False, gated=False, gather=0):
    """M rows of K values through a layer of N channels.  ln: modulated
    LayerNorm in front; gated: gate and residual behind (an fp32 output);
    gather: the M rows are picked from that many."""
    return {"name": name, "kind": "linear", "M": M, "N": N, "K": K, "dtype": dtype, "act": act, "ln": ln,
            "gated": gated, "gather": gather}


def _rotary(name, B, L, H, Hk, dh, dims, layout, dtype="bf16", frames=0, rows=0, cols=0, far=0, factor=1.0):
    """Queries of H heads and keys of Hk heads (0: queries alone) of L tokens of B
    elements; the first `dims` channels of a head turn.  frames x rows x cols: tokens
    of that grid, picked where L is less; else positions in order from near `far` on.
    factor > 1: frequencies of a context that many times as long."""
    return {"name": name, "kind": "rotary", "B": B, "L": L, "H": H, "Hk": Hk, "dh": dh, "dims": dims, "layout": layout,
            "dtype": dtype, "frames": frames, "rows": rows, "cols": cols, "far": far, "factor": factor}


def _norm(name, M, D, after, before, G=1, dtype="bf16", res="f32", gather=0, alpha=1.0):
    """M rows of D values: the norm `after` a sub-layer ("rms", "layer" or "none"),
    gate, residual, and the norm `before` the next one, modulated by one of G
    vectors; the residual in `res`, its rows picked from `gather`, scaled by alpha."""
    return {"name": name, "kind": "norm", "M": M, "D": D, "after": after, "before": before, "G": G, "dtype": dtype,
            "res": res, "gather": gather, "alpha": alpha}


def listed() -> list:
    return [
        # a small fp32 state of an odd width (launch and latency)
        _quantize("quantize4_300tok_f32", 300, 250, "f32"),
        # the block input of a 14B-shaped block at 480p, all tokens
        _quantize("quantize4_480p", 32760, 5120),
        # one row: the projection of a step's time embedding to six modulation rows
        _linear("linear4_token", 1, 30720, 5120),
        # the FFN's first product of a small block with ragged tails
        _linear("linear4_300tok", 111, 512, 256, act="gelu"),
        # the FFN's first product of the 7800-token block at a ratio of 0.25, LayerNorm in front
        _linear("linear4_7800tok_up", 1950, 8960, 1536, act="gelu", ln=True),
        # keys and values of every token at 480p
        _linear("linear4_480p_kv", 32760, 10240, 5120, ln=True),
        # the FFN's second product of the selected tokens at 480p, gate and residual behind
        _linear("linear4_480p_down", 13104, 5120, 13824, gated=True),
        # one token each of many streams far into a long context, shared heads
        _rotary("rotary_token", 32, 1, 40, 8, 128, 128, "half", far=1000000, factor=8.0),
        # fp32 exactness: odd counts, half of the head
        _rotary("rotary_f32_part", 2, 301, 3, 3, 64, 32, "interleaved", "f32", far=70000, factor=4.0),
        # queries and keys of every token of the 14B-shaped block at 480p
        _rotary("rotary_480p", 1, 32760, 40, 40, 128, 128, "interleaved", frames=21, rows=30, cols=52),
        # the 7800-token block's selected tokens: norms on both sides of a sub-layer
        _norm("norm_7800tok", 1950, 1536, "rms", "rms", dtype="bf16", gather=7800),
        # the selected tokens at 480p of a batch of two, a modulation for each element
        _norm("norm_480p_b2", 26208, 5120, "rms", "layer", G=2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng) -> dict:
    """One more case of these ranges; what would cost more than the listed ones is drawn again."""
    while True:
        kind = rng.choice(["quantize", "linear", "linear", "rotary", "norm"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if kind == "quantize":
            M, D = _log_int(rng, 1, 75600), _log_int(rng, 8, 13824)
            if rng.random() < 0.5:
                D = 8 * max(1, D // 8)
            c = _quantize("", M, D, dtype, rng.choice([0, 0, D + 8 * rng.randint(1, 64)]))
            if M * max(D, c["ld"]) > 32760 * 5120:
                continue
        elif kind == "linear":
            M, N, K = _log_int(rng, 1, 32760), _log_int(rng, 8, 30720), _log_int(rng, 16, 13824)
            if rng.random() < 0.6:
                N, K = 64 * max(1, N // 64), 64 * max(1, K // 64)
            gated = rng.random() < 0.3
            ln = not gated and dtype == "bf16" and rng.random() < 0.4
            c = _linear("", M, N, K, dtype, "none" if gated else rng.choice(["none", "gelu"]), ln, gated,
                        rng.choice([0, 0, M + _log_int(rng, 1, 2 * M + 1)]))
            if M * N * K > 32760 * 10240 * 5120 or M * N > 32760 * 10240 or N * K > 30720 * 5120:
                continue
        elif kind == "rotary":
            dh = rng.choice([16, 64, 80, 128, 128, 256])
            dims = rng.choice([dh, dh, dh // 2, max(2, dh // 4)])
            Hk, G, B = rng.choice([0, 1, 2, 4, 8, 12, 40]), rng.choice([1, 1, 2, 5]), _log_int(rng, 1, 48)
            H = Hk * G if Hk else rng.choice([1, 12, 40])
            layout = rng.choice(["half", "interleaved"])
            if rng.random() < 0.4:
                f, r, w = rng.randint(1, 21), rng.randint(1, 45), rng.randint(1, 80)
                c = _rotary("", B, rng.choice([f * r * w, max(1, f * r * w // 3)]), H, Hk, dh, dims, layout, dtype, f, r, w)
            else:
                c = _rotary("", B, _log_int(rng, 1, 32760), H, Hk, dh, dims, layout, dtype, far=_log_int(rng, 1, 4000000),
                            factor=rng.choice([1.0, 2.0, 8.0, 32.0]))
            if B * c["L"] * (H + Hk) * dh * (2 if dtype == "f32" else 1) > 32760 * 80 * 128:
                continue
        else:
            M, D, G = _log_int(rng, 1, 75600), _log_int(rng, 8, 13824), rng.choice([1, 1, 2, 3])
            if rng.random() < 0.6:
                D = 8 * max(1, D // 8)
            c = _norm("", M * G, D, rng.choice(["rms", "rms", "layer", "none"]), rng.choice(["rms", "layer"]), G, dtype,
                      rng.choice(["f32", "bf16"]), rng.choice([0, 0, M * G + _log_int(rng, 1, M + 1)]),
                      rng.choice([1.0, 1.0, 0.5, 1.7]))
            if M * G * D > 26208 * 5120:
                continue
        del c["name"]
        return c


def work(c) -> dict:
    es = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "quantize":
        # the values once, the codes and scales written and read once, the values read back written
        n = c["M"] * c["D"]
        return {"bytes": 2 * n * es + 2 * (n // 2 + n // 32), "flops": 4 * n}
    if c["kind"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        eo = 4 if c["gated"] else es
        extra = 2 * N * 4 + (M * N * es if c["gated"] else 0) + (2 * K * 4 if c["ln"] else 0)
        return {"bytes": M * K * es + N * K // 2 + N * K // 32 + M * N * eo + extra, "flops": 2 * M * N * K}
    if c["kind"] == "rotary":
        n = c["B"] * c["L"] * (c["H"] + c["Hk"]) * c["dh"]
        return {"bytes": 2 * n * es + 4 * c["B"] * c["L"], "flops": 3 * n}
    n, er = c["M"] * c["D"], 2 if c["res"] == "bf16" else 4
    return {"bytes": n * (2 * es + 2 * er) + 5 * 4 * c["G"] * c["D"], "flops": 12 * n}


# ------------------------------------------------------------------ states

def _tokens(g, M, D, dtype, ld=0):
    """Activations: N(0, 1) with a few channels of ten times the others, as blocks have them."""
    gain = torch.ones(ld or D, device="cuda")
    gain[torch.randint(0, ld or D, (max(1, D // 512),), device="cuda", generator=g)] = 10.0
    x = (torch.randn(M, ld or D, device="cuda", generator=g) * gain).to(_DT[dtype])
    return x[:, :D]


def _pick(g, n, M):
    return torch.randperm(n, device="cuda", generator=g)[:M].sort().values.to(torch.int32)


def _frequencies(c):
    """Radians per position of each pair, and how many pairs turn by each axis of the
    grid (frames, rows, columns; without a grid all by the one position)."""
    n = c["dims"] // 2
    if c["frames"]:
        side = n // 3
        counts = (n - 2 * side, side, side)
        f = [BASE ** (-j / k) for k in counts for j in range(k)]
        return f, counts
    f = [BASE ** (-j / n) for j in range(n)]
    if c["factor"] > 1:
        # pairs of few rotations over 4096 positions are slowed by the factor, those of many kept, a ramp between
        out = []
        for v in f:
            keep = min(1.0, max(0.0, (4096 * v / (2 * math.pi) - 1.0) / 31.0))
            out.append(v * (keep + (1.0 - keep) / c["factor"]))
        f = out
    return f, None


def prepare(c, seed) -> dict:
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def randn(*shape, std=1.0, mean=0.0, dtype=torch.float32):
        return (torch.randn(*shape, device="cuda", generator=g) * std + mean).to(dtype)

    s, dt = dict(c), _DT[c["dtype"]]
    if c["kind"] == "quantize":
        s["x"] = _tokens(g, c["M"], c["D"], c["dtype"], c["ld"])
    elif c["kind"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        s["x"] = _tokens(g, c["gather"] or M, K, c["dtype"])
        s["pick"] = _pick(g, c["gather"], M) if c["gather"] else None
        # the layer as a program holds it: two codes a byte in rows of whole 128 bytes, a scale byte for every 32 in
        # rows of whole 16, zeros behind the last column
        cols = torch.arange((K + 255) // 256 * 128, device="cuda") * 2
        codes = torch.randint(0, 256, (N, len(cols)), device="cuda", generator=g, dtype=torch.uint8)
        s["w_codes"] = codes & ((cols < K) * 15 + (cols + 1 < K) * 240).to(torch.uint8)
        blocks = torch.arange((K + 511) // 512 * 16, device="cuda") * 32
        scales = torch.randint(119, 122, (N, len(blocks)), device="cuda", generator=g, dtype=torch.uint8)
        s["w_scales"] = scales * (blocks < K)
        s["bias"] = randn(N, std=0.02, dtype=dt)
        s["shift"], s["scale"] = (randn(K, std=0.1), randn(K, std=0.1)) if c["ln"] else (None, None)
        s["gate"], s["res"] = (randn(N, std=0.05, mean=0.25), randn(M, N, dtype=dt)) if c["gated"] else (None, None)
    elif c["kind"] == "rotary":
        B, L, H, Hk, dh = c["B"], c["L"], c["H"], c["Hk"], c["dh"]
        qkv = randn(B, L, H + 2 * Hk, dh, dtype=dt)                 # queries, keys and values of one product
        s["q"], s["k"] = qkv[:, :, :H], qkv[:, :, H:H + Hk] if Hk else None
        f, s["counts"] = _frequencies(c)
        s["freq"] = torch.tensor(f, dtype=torch.float64, device="cuda")
        s["magnitude"] = 0.1 * math.log(c["factor"]) + 1.0
        if c["frames"]:
            n = c["frames"] * c["rows"] * c["cols"]
            s["pos"] = _pick(g, n, L)                               # the same tokens of every element
        else:
            start = torch.randint(c["far"] // 2, c["far"] + 1, (B, 1), device="cuda", generator=g)
            s["pos"] = (start + torch.arange(L, device="cuda")).to(torch.int32)
    else:
        M, D, G = c["M"], c["D"], c["G"]
        s["z"] = _tokens(g, M, D, c["dtype"])
        s["x"] = randn(c["gather"] or M, D, dtype=_DT[c["res"]])
        s["pick"] = _pick(g, c["gather"], M) if c["gather"] else None
        s["w1"] = randn(D, std=0.1, mean=1.0) if c["after"] != "none" else None
        s["w2"] = randn(D, std=0.1, mean=1.0) if c["before"] == "rms" else None
        mod = randn(G, 3, D, std=0.1)                               # gate, scale and shift of each element
        s["gate"], s["scale"], s["shift"] = mod[:, 0], mod[:, 1], mod[:, 2]
    return s


# --------------------------------------------------------------- the passes

def _codes(a):
    """Values of the 4-bit codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) and
    the power of two they are multiplied by, of 32 columns at a time."""
    M, D = a.shape
    a = torch.nn.functional.pad(a, (0, -D % 32)).view(M, -1, 32)
    _, e = torch.frexp(a.abs().amax(2, keepdim=True))              # top = f 2^e, f in [0.5, 1)
    unit = torch.exp2((e - 3).clamp(min=-127).float())
    q = a / unit                                                   # exact: below 8 in magnitude
    step = torch.where(q.abs() < 2, 0.5, torch.where(q.abs() < 4, 1.0, 2.0))
    q = (torch.round(q / step) * step).clamp(-6, 6)                # halves to the even code
    return q, unit


def _values(a):
    q, unit = _codes(a)
    return (q * unit).flatten(1)[:, : a.shape[1]]


def _weights(s):
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    c = s["w_codes"].int()
    w = table[torch.stack((c & 15, c >> 4), 2).flatten(1)]
    unit = torch.exp2(s["w_scales"].float() - 127)
    return (w.view(len(w), -1, 32) * unit[:, : w.shape[1] // 32, None]).flatten(1)[:, : s["K"]]


def _gelu(z):
    return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))


def _norm_of(a, kind):
    if kind == "none":
        return a
    if kind == "layer":
        a = a - a.mean(1, keepdim=True)
    return a * torch.rsqrt((a * a).mean(1, keepdim=True) + EPS)


def _plain_linear(s):
    x = s["x"] if s["pick"] is None else s["x"][s["pick"].long()]
    a = x.float()
    if s["ln"]:
        a = _norm_of(a, "layer") * (1.0 + s["scale"]) + s["shift"]
    y = torch.matmul(_values(a), _weights(s).t()) + s["bias"].float()
    if s["act"] == "gelu":
        y = _gelu(y)
    if s["gated"]:
        return s["res"].float() + s["gate"] * y
    return y.to(s["x"].dtype)


def _turn(x, s, cos, sin):
    n = s["dims"] // 2
    a = x.float()
    if s["layout"] == "half":
        u, v = a[..., :n], a[..., n: 2 * n]
        turned = torch.cat((u * cos - v * sin, u * sin + v * cos), -1)
    else:
        u, v = a[..., 0: 2 * n: 2], a[..., 1: 2 * n: 2]
        turned = torch.stack((u * cos - v * sin, u * sin + v * cos), -1).flatten(-2)
    return torch.cat((turned, a[..., 2 * n:]), -1).to(x.dtype)


def _plain_rotary(s):
    p = s["pos"].double()[..., None]
    if s["frames"]:
        t, r, w = s["counts"]
        i = s["pos"].long()[:, None]
        p = torch.cat(((i // (s["rows"] * s["cols"])).expand(-1, t), (i // s["cols"] % s["rows"]).expand(-1, r),
                       (i % s["cols"]).expand(-1, w)), 1).double()
    angle = p * s["freq"]                                          # 64 bits: far positions turn many times
    cos, sin = (torch.cos(angle) * s["magnitude"]).float(), (torch.sin(angle) * s["magnitude"]).float()
    cos, sin = cos[..., None, :], sin[..., None, :]                # the same for every head
    out = {"q": _turn(s["q"], s, cos, sin)}
    if s["k"] is not None:
        out["k"] = _turn(s["k"], s, cos, sin)
    return out


def _plain_norm(s):
    M, G = s["M"], s["G"]
    gate, scale, shift = (s[n].repeat_interleave(M // G, 0) if G > 1 else s[n] for n in ("gate", "scale", "shift"))
    x = s["x"] if s["pick"] is None else s["x"][s["pick"].long()]
    z = _norm_of(s["z"].float(), s["after"])
    if s["w1"] is not None:
        z = z * s["w1"]
    y = s["alpha"] * x.float() + gate * z
    h = _norm_of(y, s["before"])
    if s["w2"] is not None:
        h = h * s["w2"]
    h = h * (1.0 + scale) + shift
    return {"y": y.to(s["x"].dtype), "h": h.to(s["z"].dtype)}


def run(s):
    if own:
        from paper_2608_02474_amd import api
        if s["kind"] == "quantize":
            return api.dequantize_rows_fp4(api.quantize_rows_fp4(s["x"]), s["x"].dtype)
        if s["kind"] == "linear":
            a = api.quantize_rows_fp4(s["x"], rows=s["pick"], shift=s["shift"], scale=s["scale"], ln_eps=EPS)
            w = api.Fp4Rows(s["w_codes"], s["w_scales"], s["K"])
            return api.linear_fp4(a, w, s["bias"], activation=None if s["act"] == "none" else s["act"],
                                  gate=s["gate"], residual=s["res"],
                                  dtype=torch.float32 if s["gated"] else s["x"].dtype)
        if s["kind"] == "rotary":
            grid = (s["rows"], s["cols"]) if s["frames"] else None
            rot = api.Rotary(s["freq"], s["layout"], s["magnitude"], grid, s["counts"])
            q, k = api.rotary(s["q"], rot, s["k"], positions=s["pos"])
            return {"q": q} if k is None else {"q": q, "k": k}
        y, h = api.gated_norm(s["z"], s["x"], after=None if s["after"] == "none" else s["after"], after_weight=s["w1"],
                              gate=s["gate"], residual_scale=s["alpha"], residual_rows=s["pick"], before=s["before"],
                              before_weight=s["w2"], scale=s["scale"], shift=s["shift"], eps=EPS)
        return {"y": y, "h": h}
    if s["kind"] == "quantize":
        return _values(s["x"].float()).to(s["x"].dtype)
    if s["kind"] == "linear":
        return _plain_linear(s)
    return _plain_rotary(s) if s["kind"] == "rotary" else _plain_norm(s)


# -------------------------------------------------------------------- exact

def _exact_values(x):
    """The nearest of the eight magnitudes: how many of their borders lie below, the ones
    above an odd code reached from below."""
    M, D = x.shape
    out = torch.empty(M, (D + 31) // 32 * 32, dtype=torch.float64, device="cuda")
    out[:, :D], out[:, D:] = x, 0
    for part in out.split(4096):
        b = part.view(len(part), -1, 32)
        top = b.abs().max(dim=2, keepdim=True).values
        unit = (((top.view(torch.int64) >> 52) - 1023 - 2).clamp(min=-127) + 1023 << 52).view(torch.float64)
        m = b.abs() / unit
        code = torch.zeros_like(m, dtype=torch.int64)
        for border in (0.25, 1.25, 2.5, 5.0):
            code += m > border
        for border in (0.75, 1.75, 3.5):
            code += m >= border
        grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
        b.copy_(torch.copysign(grid[code], b) * unit)
    return out[:, :D]


def _exact_norm(x, kind):
    if kind == "none":
        return x
    if kind == "rms":
        return x / (x.square().mean(1, keepdim=True) + EPS).sqrt()
    var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
    return (x - mean) / (var + EPS).sqrt()


def exact(c, seed):
    s = prepare(c, seed)
    f64 = torch.float64
    if c["kind"] == "quantize":
        return _exact_values(s["x"])
    if c["kind"] == "linear":
        x = s["x"].to(f64)
        if s["pick"] is not None:
            x = x.index_select(0, s["pick"].long())
        if c["ln"]:
            x = _exact_norm(x, "layer") * (1 + s["scale"].to(f64)) + s["shift"].to(f64)
        x = _exact_values(x)
        codes = s["w_codes"]
        w = torch.empty(c["N"], 2 * codes.shape[1], dtype=f64, device="cuda")
        for at, nibble in ((0, codes % 16), (1, codes // 16)):
            e, odd = (nibble % 8) // 2, (nibble % 2).to(f64)       # two bits of exponent and one of the fraction
            v = torch.where(e == 0, odd / 2, (1 + odd / 2) * torch.exp2(e.to(f64) - 1))
            w[:, at::2] = torch.where(nibble >= 8, -v, v)
        unit = torch.exp2(s["w_scales"].to(f64) - 127).repeat_interleave(32, 1)[:, : w.shape[1]]
        w = (w * unit)[:, : c["K"]]
        y = torch.addmm(s["bias"].to(f64), x, w.T)
        del x, w, unit
        if c["act"] == "gelu":
            y = y / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
        if c["gated"]:
            y = s["res"].to(f64) + s["gate"].to(f64) * y
        return y
    if c["kind"] == "rotary":
        pos = s["pos"].to(torch.int64)
        if c["frames"]:
            per = c["rows"] * c["cols"]
            axes = (pos // per, pos % per // c["cols"], pos % c["cols"])
            angle = torch.cat([a[:, None].to(f64) * f for a, f in zip(axes, s["freq"].split(s["counts"]))], 1)
            angle = angle.expand(c["B"], -1, -1)
        else:
            angle = pos[:, :, None].to(f64) * s["freq"]
        turn = torch.polar(torch.full_like(angle, s["magnitude"]), angle)[:, :, None]
        out = {}
        for name in ("q", "k"):
            if s[name] is None:
                continue
            o = s[name].to(f64)
            p = o[..., : c["dims"]]
            if c["layout"] == "half":
                z = torch.complex(*p.chunk(2, -1)) * turn
                o[..., : c["dims"]] = torch.cat((z.real, z.imag), -1)
            else:
                z = torch.view_as_complex(p.unflatten(-1, (-1, 2)).contiguous()) * turn
                o[..., : c["dims"]] = torch.view_as_real(z).flatten(-2)
            out[name] = o
        return out
    z, x = s["z"].to(f64), s["x"].to(f64)
    if s["pick"] is not None:
        x = x.index_select(0, s["pick"].long())
    per = c["M"] // c["G"]
    z = _exact_norm(z, c["after"])
    if s["w1"] is not None:
        z *= s["w1"].to(f64)
    y = c["alpha"] * x
    for i in range(c["G"]):
        y[i * per:(i + 1) * per] += s["gate"][i].to(f64) * z[i * per:(i + 1) * per]
    h = _exact_norm(y, c["before"])
    if s["w2"] is not None:
        h = h * s["w2"].to(f64)
    for i in range(c["G"]):
        h[i * per:(i + 1) * per] *= 1 + s["scale"][i].to(f64)
        h[i * per:(i + 1) * per] += s["shift"][i].to(f64)
    return {"y": y, "h": h}
