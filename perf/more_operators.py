"""Cases that time the operators on hidden rows: rows in 8 bits, the layers that read them, gated or not, and their gradients.

A row of D columns is one piece of bytes: a byte of E4M3 code per column, zeros up to a multiple of sixteen, one E8M0 scale
byte per block of 128 columns, zeros up to a multiple of sixteen.  A block's scale is the smallest power of two, from 2^-117 to
2^119, under which none of its finite values is above 448, the largest E4M3.  Minibatches are those of the repository's
workloads (some 45 thousand vertices, 64 in flight), widths its benchmark's hidden ones of 256 and 1024, or odd.

`own` False: the operators in elementary torch operations, 32 bits.  True: the library's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
BYTES = {"float32": 4, "float16": 2, "bfloat16": 2}
BLOCK = 128                 # columns that share a scale
MOST = 448.0                # the largest E4M3
LEAST_E, MOST_E = -117, 119


def listed():
    return [
        # The two matrices of a gated layer, quantised again after every step: all latency.
        dict(name="rows_weight", kind="rows", n=512, D=256, dtype="float32", out="float32"),
        # The hidden rows of the 64 minibatches that a pipeline keeps in flight, kept in 8 bits for the backward pass, and read back.
        dict(name="rows_in_flight", kind="rows", n=2_560_000, D=256, dtype="bfloat16", out="bfloat16"),
        # One vertex served by itself.
        dict(name="product_one", kind="product", lists=1, rows=1, groups=1, D=256, H=256, dtype="float32"),
        # The second layer of 64 minibatches, each with its count on the device.
        dict(name="product_in_flight", kind="product", lists=64, rows=40_000, groups=1, D=256, H=256, dtype="bfloat16"),
        # A hidden layer of mag240c's width.
        dict(name="product_wide", kind="product", lists=3, rows=130_000, groups=1, D=1024, H=1024, dtype="bfloat16"),
        # A gated layer of one minibatch.
        dict(name="gated_batch", kind="gated", lists=1, rows=45_000, groups=1, D=256, H=256, act="silu", dtype="bfloat16"),
        # Of the 64 minibatches in flight.
        dict(name="gated_in_flight", kind="gated", lists=64, rows=40_000, groups=1, D=256, H=256, act="silu", dtype="bfloat16"),
        # Rows of eight kinds of vertices, each kind with matrices of its own; odd widths, some kinds absent.
        dict(name="gated_kinds", kind="gated", lists=24, rows=5_001, groups=8, D=172, H=100, act="gelu", dtype="float32"),
        # Its backward pass: the 64 minibatches, the kinds in 32 bits.
        dict(name="gated_grad_in_flight", kind="gated_grad", lists=64, rows=40_000, groups=1, D=256, H=256, act="silu", dtype="bfloat16"),
        dict(name="gated_grad_kinds", kind="gated_grad", lists=24, rows=5_001, groups=8, D=172, H=100, act="gelu", dtype="float32"),
        # The gradients of the two matrices of the gated layer, of the kinds' matrices.
        dict(name="grad_in_flight", kind="grad", lists=64, rows=40_000, groups=1, D=256, H=512, dtype="bfloat16"),
        dict(name="grad_kinds", kind="grad", lists=24, rows=5_001, groups=8, D=172, H=200, dtype="float32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rows", "product", "product", "gated", "gated", "gated_grad", "gated_grad", "grad"])
    D = rng.choice([256, 1024, 100, 128, 512, rng.randint(1, 1100)])
    if kind == "rows":
        return dict(kind=kind, n=_log(rng, 1, 600_000_000 // max(D, 300)), D=D, dtype=rng.choice(list(TYPES)), out=rng.choice(list(TYPES)))
    H = rng.choice([256, 1024, 47, 172, rng.randint(1, 1100)])
    if kind != "product" and kind != "grad":
        H = (H + 1) // 2
    lists = rng.choice([1, 1, rng.randint(2, 64), 64])
    groups = rng.choice([1, 1, rng.randint(1, min(lists, 12))])
    total = min(2_500_000, int(1.5e11 / (D * H)), int(3e8 / H))
    case = dict(kind=kind, lists=lists, rows=max(1, _log(rng, 1, max(2, total)) // lists), groups=groups, D=D, H=H)
    if kind in ("gated", "gated_grad"):
        case["act"] = rng.choice(["silu", "silu", "gelu", "sigmoid"])
    case["dtype"] = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    return case


# ---- sizes --------------------------------------------------------------------------------------

def _code_bytes(D):
    return (D + 15) // 16 * 16


def _row_bytes(D):
    return _code_bytes(D) + ((D + BLOCK - 1) // BLOCK + 15) // 16 * 16


def _lists(case):
    """(first row, capacity, rows, group) of each list; lists of several groups come ragged, some of them empty."""
    rng = random.Random("%d %d %d" % (case["lists"], case["rows"], case["groups"]))
    at, out = 0, []
    for j in range(case["lists"]):
        if case["lists"] == 1:
            n = case["rows"]
        elif case["groups"] > 1:
            n = 0 if rng.random() < 0.15 else rng.randint(0, 2 * case["rows"])
        else:
            n = rng.randint(case["rows"] * 4 // 5, case["rows"] * 6 // 5)
        cap = n if case["lists"] == 1 else n + n // 16 + 3
        out.append((at, cap, n, j % case["groups"]))
        at += cap
    return out, at


def work(case):
    if case["kind"] == "rows":
        n, D = case["n"], case["D"]
        return {"bytes": n * D * (BYTES[case["dtype"]] + BYTES[case["out"]]) + n * _row_bytes(D), "flops": 4 * n * D}
    lists, _ = _lists(case)
    n, rb, H, D, G, b = sum(x[2] for x in lists), _row_bytes(case["D"]), case["H"], case["D"], case["groups"], BYTES[case["dtype"]]
    if case["kind"] == "product":
        return {"bytes": n * (rb + H * b) + G * H * rb, "flops": 2 * n * H * D}
    if case["kind"] == "grad":
        return {"bytes": n * (rb + H * b) + 4 * G * H * D, "flops": 2 * n * H * D}
    return {"bytes": n * (rb + H * b * (1 if case["kind"] == "gated" else 3)) + 2 * G * H * rb, "flops": 4 * n * H * D}


# ---- rows in 8 bits, in elementary operations ------------------------------------------------------

def _quantize(x):
    """[n, D] -> packed rows uint8 [n, row bytes]."""
    n, D = x.shape
    nb, cb = (D + BLOCK - 1) // BLOCK, _code_bytes(D)
    x = torch.nn.functional.pad(x.float(), (0, nb * BLOCK - D)).view(n, nb, BLOCK)
    ok = torch.isfinite(x)
    f, k = torch.frexp(torch.where(ok, x.abs(), 0).amax(2))
    e = torch.where(f > 0, k.to(torch.int32) - 8 - (f <= MOST / 512).to(torch.int32), LEAST_E).clamp(LEAST_E, MOST_E)
    a = (x * ((127 - e) << 23).view(torch.float32).unsqueeze(2)).clamp(-MOST, MOST)
    code = torch.where(ok, a, math.nan).to(torch.float8_e4m3fn).view(torch.uint8)
    rows = torch.zeros(n, _row_bytes(D), dtype=torch.uint8, device=x.device)
    rows[:, :cb] = code.reshape(n, nb * BLOCK)[:, :cb]
    rows[:, cb:cb + nb] = (e + 127).to(torch.uint8)
    return rows


def _values(rows, D):
    """fp32 values of packed rows [..., row bytes]."""
    rows = rows.reshape(-1, rows.shape[-1])
    n, nb, cb = rows.shape[0], (D + BLOCK - 1) // BLOCK, _code_bytes(D)
    v = torch.nn.functional.pad(rows[:, :cb], (0, nb * BLOCK - cb)).view(torch.float8_e4m3fn).float().view(n, nb, BLOCK)
    s = (rows[:, cb:cb + nb].to(torch.int32) << 23).view(torch.float32)
    return (v * s.unsqueeze(2)).view(n, nb * BLOCK)[:, :D]


def _gate(g, act):
    """act(g) and its derivative."""
    if act == "gelu":
        p = 0.5 * torch.special.erfc(g * -math.sqrt(0.5))
        return g * p, p + g * torch.exp(g * g * -0.5) * (1 / math.sqrt(2 * math.pi))
    s = 1 / (1 + torch.exp(-g))
    r = 1 / (1 + torch.exp(g))
    return (g * s, s * (1 + g * r)) if act == "silu" else (s, s * r)


# ---- inputs and passes ---------------------------------------------------------------------------

def _hidden(gen, n, D):
    """Hidden rows: columns of unit variance, rows of differing size."""
    x = torch.randn(n, D, generator=gen, device=DEV)
    return x * torch.exp2(torch.randn(n, 1, generator=gen, device=DEV) * 0.5)


def _packed(gen, n, D, size):
    at = [_quantize(_hidden(gen, min(n - i, 400_000), D) * size) for i in range(0, n, 400_000)]
    return torch.cat(at) if at else torch.zeros(0, _row_bytes(D), dtype=torch.uint8, device=DEV)


def _inputs(case, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind == "rows":
        s["x"] = _hidden(gen, case["n"], case["D"]).to(TYPES[case["dtype"]])
        return s
    lists, total = _lists(case)
    D, H, G, ty = case["D"], case["H"], case["groups"], TYPES[case["dtype"]]
    s["rows"] = _packed(gen, total, D, 1.0)
    s["n"] = torch.tensor([x[2] for x in lists], dtype=torch.int64, device=DEV)
    if kind != "grad":
        each = H if kind == "product" else 2 * H
        s["w"] = _packed(gen, G * each, D, D ** -0.5).view(G, each, -1)
    if kind in ("product", "gated"):
        s["y"] = torch.zeros(total, H, dtype=ty, device=DEV)
    else:
        s["y"] = (torch.randn(total, H, generator=gen, device=DEV) * 0.01).to(ty)
    if kind == "gated_grad":
        s["dp"] = torch.zeros(total, 2 * H, dtype=ty, device=DEV)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "rows":
        if own:
            import paper_2305_03152_amd as spp
            s["spp"], s["ctx"] = spp, spp.Context(0)
        return s
    lists, _ = _lists(case)
    if own:
        import paper_2305_03152_amd as spp
        s["spp"], s["ctx"] = spp, spp.Context(0)
        s["lists"] = spp.RowLists([(s["rows"][a:a + c], c, s["n"][j:j + 1], s["y"][a:a + c], k) for j, (a, c, n, k) in enumerate(lists)])
        if "dp" in s:
            s["grads"] = spp.RowLists([(s["rows"][a:a + c], c, s["n"][j:j + 1], s["dp"][a:a + c], k) for j, (a, c, n, k) in enumerate(lists)])
    else:
        s["from"] = torch.tensor([x[0] for x in lists], device=DEV)
        s["parts"] = [(a, a + c, k) for a, c, n, k in lists]
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    case, spp, ctx = s["case"], s["spp"], s["ctx"]
    if case["kind"] == "rows":
        rows = spp.fp8_quantize(ctx, s["x"], sync=False)
        return spp.fp8_dequantize(ctx, rows, case["D"], dtype=TYPES[case["out"]], sync=False)
    if case["kind"] == "product":
        spp.fp8_product_multi(ctx, s["lists"], s["w"], case["D"], sync=False)
        return s["y"]
    if case["kind"] == "gated":
        spp.fp8_gated_multi(ctx, s["lists"], s["w"], case["D"], activation=case["act"], sync=False)
        return s["y"]
    if case["kind"] == "gated_grad":
        spp.fp8_gated_grad(ctx, s["lists"], s["grads"], s["w"], case["D"], activation=case["act"], sync=False)
        return s["dp"]
    return spp.fp8_weight_grad(ctx, s["lists"], case["H"], case["D"], groups=case["groups"], sync=False)


def _inside(s):
    """Which rows of the buffer a list holds: those before its count."""
    i = torch.arange(s["y"].shape[0], device=DEV)
    j = torch.searchsorted(s["from"], i, right=True) - 1
    return ((i - s["from"][j]) < s["n"][j]).unsqueeze(1)


def _run_plain(s):
    case, D = s["case"], s["case"]["D"]
    if case["kind"] == "rows":
        return _values(_quantize(s["x"]), D).to(TYPES[case["out"]])
    x, G, H = _values(s["rows"], D), case["groups"], case["H"]
    if case["kind"] == "grad":
        y = torch.where(_inside(s), s["y"].float(), 0)
        if G == 1:
            return (y.T @ x).unsqueeze(0)
        w = torch.zeros(G, H, D, device=DEV)
        [w[k].add_(y[a:b].T @ x[a:b]) for a, b, k in s["parts"]]
        return w
    w = _values(s["w"], D).view(G, -1, D)
    p = x @ w[0].T if G == 1 else torch.cat([x[a:b] @ w[k].T for a, b, k in s["parts"]])
    del x
    if case["kind"] == "product":
        s["y"] = torch.where(_inside(s), p.to(s["y"].dtype), s["y"])
        return s["y"]
    f, d = _gate(p[:, :H], case["act"])
    if case["kind"] == "gated":
        s["y"] = torch.where(_inside(s), (f * p[:, H:]).to(s["y"].dtype), s["y"])
        return s["y"]
    y = s["y"].float()
    s["dp"] = torch.where(_inside(s), torch.cat([y * p[:, H:] * d, y * f], 1).to(s["dp"].dtype), s["dp"])
    return s["dp"]


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _exact_rounded(x):
    """x [n, D] in float64, rounded by the definition: under its block's scale, to three bits behind the leading one, or to a
    multiple of 2^-9 below 2^-6."""
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], BLOCK):
        b = x[:, c:c + BLOCK]
        top = b.abs().max(1, keepdim=True).values
        e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / MOST))
        e = e + (MOST * torch.exp2(e) < top).double() - (MOST * torch.exp2(e - 1) >= top).double()     # log2 may be off next to a border
        e = e.clamp(LEAST_E, MOST_E)
        q = (b / torch.exp2(e)).clamp(-MOST, MOST)
        step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6) * (1 + 2.0 ** -40))) - 3)
        out[:, c:c + BLOCK] = torch.round(q / step) * step * torch.exp2(e)
    return out


def _exact_values(rows, D):
    """By the fields of a code: sign, four bits of exponent with bias 7, three of fraction."""
    r = rows.reshape(-1, rows.shape[-1])
    c = r[:, :D].to(torch.int32)
    power, fraction = (c >> 3) & 15, (c & 7).double()
    v = torch.where(power == 0, fraction * 2.0 ** -9, (8 + fraction) * torch.exp2(power.double() - 10))
    v = torch.where(c >= 128, -v, v)
    at = _code_bytes(D) + torch.arange(D, device=r.device) // BLOCK
    return v * torch.exp2(r[:, at].double() - 127)


def _exact_layer(case, x, w, dy):
    """Rows x and their part of the output, w [H or 2H, D], dy the output's gradient."""
    kind, H = case["kind"], case["H"]
    if kind == "product":
        return x @ w.T
    g, u = x @ w[:H].T, x @ w[H:].T
    normal = torch.distributions.Normal(torch.zeros((), dtype=torch.float64, device=x.device), 1.0)
    if case["act"] == "gelu":
        f, d = g * normal.cdf(g), normal.cdf(g) + g * torch.exp(normal.log_prob(g))
    elif case["act"] == "silu":
        t = torch.tanh(g / 2)
        f, d = g * (1 + t) / 2, (1 + t) / 2 + g * (1 - t * t) / 4
    else:
        t = torch.tanh(g / 2)
        f, d = (1 + t) / 2, (1 - t * t) / 4
    return f * u if kind == "gated" else torch.cat([dy * u * d, dy * f], 1)


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "rows":
        return torch.cat([_exact_rounded(s["x"][i:i + 100_000].double()) for i in range(0, case["n"], 100_000)])
    lists, total = _lists(case)
    D, H, G = case["D"], case["H"], case["groups"]
    if kind == "grad":
        w = torch.zeros(G, H, D, dtype=torch.float64, device=DEV)
        for a, cap, n, k in lists:
            w[k] += s["y"][a:a + n].double().T @ _exact_values(s["rows"][a:a + n], D)
        return w
    w = _exact_values(s["w"], D).view(G, -1, D)
    y = torch.zeros(total, 2 * H if kind == "gated_grad" else H, dtype=torch.float64, device=DEV)
    for a, cap, n, k in lists:
        y[a:a + n] = _exact_layer(case, _exact_values(s["rows"][a:a + n], D), w[k], s["y"][a:a + n].double())
    return y
