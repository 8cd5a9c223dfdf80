"""Cases that time the operators on gathered rows: 4-bit rows, the layer that reads them, its gradient, the optimiser's step.

A row of D columns in MXFP4 is one piece of bytes: blocks of 32 columns as sixteen bytes of E2M1 codes each (the even
column in the low half of a byte), then one E8M0 scale byte per block, then zeros up to a multiple of sixteen.  The sizes
are those of the repository's workloads (row widths 32, 100, 128, 256, 768; minibatches of some 45 to 66 thousand vertices,
64 in flight) with hidden widths of 256 and 1024.

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
BLOCK = 256                 # elements of an 8-bit state that share a scale
HYPER = dict(lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01)
SAGE = "25600,25600,256,65536,65536,256,12032,12032,47"      # three layers 100 -> 256 -> 256 -> 47, two matrices and a bias each


def listed():
    return [
        # The weights of one layer, quantised again after every step: all latency.
        dict(name="rows_weight", kind="rows", n=256, D=128, dtype="float32", out="float32"),
        # One Mid minibatch's rows (100 columns: the last block is a part), as a program that compresses on the fly does.
        dict(name="rows_mid_batch", kind="rows", n=66_003, D=100, dtype="float32", out="bfloat16"),
        # A share of Wide's feature store, compressed once and read back for a layer that wants 16 bits.
        dict(name="rows_wide_store", kind="rows", n=800_000, D=768, dtype="float16", out="bfloat16"),
        # One vertex served by itself.
        dict(name="product_one", kind="product", lists=1, rows=1, groups=1, D=128, H=256, out="float32"),
        # One minibatch of the papers shape.
        dict(name="product_batch", kind="product", lists=1, rows=45_000, groups=1, D=128, H=256, out="bfloat16"),
        # The 64 minibatches that a pipeline keeps in flight, each with its count on the device.
        dict(name="product_in_flight", kind="product", lists=64, rows=40_000, groups=1, D=128, H=256, out="bfloat16"),
        # mag240c's shape: wide rows, a hidden width of 1024.
        dict(name="product_wide", kind="product", lists=3, rows=130_000, groups=1, D=768, H=1024, out="bfloat16"),
        # Rows of eight kinds of vertices, each kind with weights of its own; odd widths, some kinds absent.
        dict(name="product_kinds", kind="product", lists=24, rows=5_001, groups=8, D=100, H=172, out="float32"),
        # The gradient of the 64 minibatches' layer: one matrix for all lists.
        dict(name="grad_in_flight", kind="grad", lists=64, rows=40_000, groups=1, D=128, H=256, dtype="bfloat16"),
        # The gradient of the kinds' matrices, and in 32 bits.
        dict(name="grad_kinds", kind="grad", lists=24, rows=5_001, groups=8, D=100, H=172, dtype="float32"),
        # The step of a three-layer model's nine tensors: launches and latency.
        dict(name="adamw_model", kind="adamw", sizes=SAGE, bits=32, param="float32", grad="float32"),
        # A learned table for the partition's vertices beside the model, states in 8 bits.
        dict(name="adamw_table_8", kind="adamw", sizes="128000001," + SAGE, bits=8, param="float32", grad="bfloat16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rows", "product", "product", "grad", "grad", "adamw"])
    D = rng.choice([32, 100, 128, 256, 768, rng.randint(1, 800)])
    if kind == "rows":
        return dict(kind=kind, n=_log(rng, 1, 600_000_000 // max(D, 500)), D=D, dtype=rng.choice(list(TYPES)), out=rng.choice(list(TYPES)))
    if kind == "adamw":
        sizes = [_log(rng, 1, 100_000_000)] + [_log(rng, 1, 1_000_000) for _ in range(rng.randint(0, 20))]
        return dict(kind=kind, sizes=",".join(map(str, sizes)), bits=rng.choice([8, 32]), param=rng.choice(["float32", "bfloat16"]),
                    grad=rng.choice(list(TYPES)))
    H = rng.choice([256, 1024, 47, 172, rng.randint(1, 1100)])
    lists = rng.choice([1, 1, rng.randint(2, 64), 64])
    groups = rng.choice([1, 1, rng.randint(1, min(lists, 12))])
    total = min(2_500_000, int(3e11 / (D * H)), int(6e8 / H))
    case = dict(kind=kind, lists=lists, rows=max(1, _log(rng, 1, max(2, total)) // lists), groups=groups, D=D, H=H)
    case["out" if kind == "product" else "dtype"] = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    return case


# ---- sizes --------------------------------------------------------------------------------------

def _row_bytes(D):
    return (17 * ((D + 31) // 32) + 15) // 16 * 16


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


def _sizes(case):
    return [int(s) for s in case["sizes"].split(",")]


def work(case):
    if case["kind"] == "rows":
        n, D = case["n"], case["D"]
        return {"bytes": n * D * (BYTES[case["dtype"]] + BYTES[case["out"]]) + n * _row_bytes(D), "flops": 4 * n * D}
    if case["kind"] == "adamw":
        state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK + 8        # in 8 bits the states come back as values too
        return {"bytes": sum(_sizes(case)) * (2 * BYTES[case["param"]] + BYTES[case["grad"]] + state), "flops": 16 * sum(_sizes(case))}
    lists, _ = _lists(case)
    n, rb, H, D, G = sum(x[2] for x in lists), _row_bytes(case["D"]), case["H"], case["D"], case["groups"]
    if case["kind"] == "product":
        return {"bytes": n * (rb + H * BYTES[case["out"]]) + G * H * rb, "flops": 2 * n * H * D}
    return {"bytes": n * (rb + H * BYTES[case["dtype"]]) + 4 * G * H * D, "flops": 2 * n * H * D}


# ---- MXFP4 in elementary operations --------------------------------------------------------------

def _quantize(x):
    """[n, D] -> (packed rows uint8 [n, row bytes], values fp32 [n, D])."""
    n, D = x.shape
    nb = (D + 31) // 32
    x = torch.nn.functional.pad(x.float(), (0, nb * 32 - D)).view(n, nb, 32)
    top = x.abs().amax(2)
    bad = ~torch.isfinite(top)
    e = torch.where(top > 0, torch.frexp(top)[1].to(torch.int32) - 3, -127).clamp(-127, 125)
    a = x * ((127 - e) << 23).view(torch.float32).unsqueeze(2)
    neg = torch.signbit(x).to(torch.uint8) << 3
    a = a.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)) | neg
    code = torch.where(bad.unsqueeze(2), torch.zeros_like(code), code)
    scale = torch.where(bad, 255, e + 127).to(torch.uint8)
    rows = torch.zeros(n, _row_bytes(D), dtype=torch.uint8, device=x.device)
    code = code.reshape(n, nb * 32)
    rows[:, :nb * 16] = code[:, 0::2] | (code[:, 1::2] << 4)
    rows[:, nb * 16:nb * 17] = scale
    return rows


def _values(rows, D):
    """fp32 values of packed rows [..., row bytes]."""
    rows = rows.reshape(-1, rows.shape[-1])
    n, nb = rows.shape[0], (D + 31) // 32
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=rows.device)
    c = rows[:, :nb * 16]
    c = torch.stack([c & 15, c >> 4], 2).view(-1)
    s = rows[:, nb * 16:nb * 17].to(torch.int32)
    s = torch.where(s == 255, math.nan, torch.where(s > 0, s << 23, 0x00400000).view(torch.float32))
    v = table.index_select(0, c.to(torch.int32)).view(n, nb, 32) * s.unsqueeze(2)
    return v.view(n, nb * 32)[:, :D]


# ---- AdamW in elementary operations --------------------------------------------------------------

def _blocks(x):
    return torch.nn.functional.pad(x, (0, -x.numel() % BLOCK)).view(-1, BLOCK)


def _pack(a, most, drop, base, top):
    """Codes of non-negative values a [blocks, BLOCK] as small floats below the block's largest, and the blocks' scales."""
    R = a.amax(1, keepdim=True)
    has = R >= 2.0 ** -100
    inv = torch.where(has, torch.full_like(R, most) / R, 0)
    u = (a * inv).view(torch.int32)
    code = (((u + ((1 << (drop - 1)) - 1) + ((u >> drop) & 1)) >> drop) - base).clamp(0, top)
    return code, torch.where(has, R * (1 / most), 0)


def _pack_m(m):
    b = _blocks(m)
    code, s = _pack(b.abs(), 1.875, 20, 896, 127)
    return torch.where(code > 0, code | (torch.signbit(b).to(torch.int32) << 7), 0).to(torch.uint8), s


def _pack_v(v):
    r = _blocks(torch.sqrt(v))
    code, s = _pack(r, 1.9375, 19, 1792, 255)
    return torch.where((r > 0) & (s > 0), code.clamp(min=1), 0).to(torch.uint8), s


def _unpack_m(code, s, n):
    c = code.to(torch.int32)
    a = (((c & 127) + 896) << 20).view(torch.float32) * s
    return torch.where((c & 127) == 0, 0, torch.where(c > 127, -a, a)).view(-1)[:n]


def _unpack_v(code, s, n):
    c = code.to(torch.int32)
    r = ((c + 1792) << 19).view(torch.float32) * s
    return torch.where(c == 0, 0, r * r).view(-1)[:n]


def _step(p, g, m, v, t):
    """One step in 32 bits; an element whose new second moment is not finite stays as it was."""
    (b1, b2), lr, eps = HYPER["betas"], HYPER["lr"], HYPER["eps"]
    g, q = g.float(), p.float()
    m1 = m * b1 + g * (1 - b1)
    v1 = v * b2 + (g * g) * (1 - b2)
    den = torch.sqrt(v1) * (1 / math.sqrt(1 - b2 ** t)) + eps
    q1 = q * (1 - lr * HYPER["weight_decay"]) - (m1 / den) * (lr / (1 - b1 ** t))
    ok = torch.isfinite(v1)
    return torch.where(ok, q1, q).to(p.dtype), torch.where(ok, m1, m), torch.where(ok, v1, v)


# ---- inputs and passes ---------------------------------------------------------------------------

def _features(gen, n, D):
    """Feature rows: columns of unit variance, rows and blocks of differing size as normalised embeddings have."""
    x = torch.randn(n, D, generator=gen, device=DEV)
    return x * torch.exp2(torch.randn(n, 1, generator=gen, device=DEV))


def _packed(gen, n, D):
    at = [_quantize(_features(gen, min(n - i, 400_000), D)) for i in range(0, n, 400_000)]
    return torch.cat(at) if at else torch.zeros(0, _row_bytes(D), dtype=torch.uint8, device=DEV)


def _inputs(case, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind == "rows":
        s["x"] = _features(gen, case["n"], case["D"]).to(TYPES[case["dtype"]])
    elif kind == "adamw":
        ns = _sizes(case)
        s["p"] = [(torch.randn(n, generator=gen, device=DEV) * 0.05).to(TYPES[case["param"]]) for n in ns]
        s["g"] = [(torch.randn(n, generator=gen, device=DEV) * 0.01).to(TYPES[case["grad"]]) for n in ns]
        s["m"] = [torch.randn(n, generator=gen, device=DEV) * 0.003 for n in ns]
        s["v"] = [(torch.randn(n, generator=gen, device=DEV) * 0.01).square() for n in ns]
        s["t"] = 100
    else:
        lists, total = _lists(case)
        D, H, G = case["D"], case["H"], case["groups"]
        s["rows"] = _packed(gen, total, D)
        s["n"] = torch.tensor([x[2] for x in lists], dtype=torch.int64, device=DEV)
        if kind == "product":
            s["w"] = _packed(gen, G * H, D).view(G, H, -1)
            s["y"] = torch.zeros(total, H, dtype=TYPES[case["out"]], device=DEV)
        else:
            s["y"] = (torch.randn(total, H, generator=gen, device=DEV) * 0.01).to(TYPES[case["dtype"]])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if own:
        import paper_2305_03152_amd as spp
        s["spp"], s["ctx"] = spp, spp.Context(0)
        if kind == "adamw":
            s["opt"] = spp.AdamW(s["ctx"], s["p"], state_bits=case["bits"], **HYPER)
            s["opt"].load(s.pop("m"), s.pop("v"), s["t"])
        elif kind != "rows":
            lists, _ = _lists(case)
            s["lists"] = spp.RowLists([(s["rows"][a:a + c], c, s["n"][j:j + 1], s["y"][a:a + c], k) for j, (a, c, n, k) in enumerate(lists)])
    elif kind == "adamw":
        if case["bits"] == 8:
            s["m"], s["v"] = [_pack_m(m) for m in s["m"]], [_pack_v(v) for v in s["v"]]
    elif kind != "rows":
        lists, _ = _lists(case)
        s["from"] = torch.tensor([x[0] for x in lists], device=DEV)
        s["parts"] = [(a, a + c, k) for a, c, n, k in lists]
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    case, spp, ctx = s["case"], s["spp"], s["ctx"]
    if case["kind"] == "rows":
        rows = spp.mx4_quantize(ctx, s["x"], sync=False)
        return spp.mx4_dequantize(ctx, rows, case["D"], dtype=TYPES[case["out"]], sync=False)
    if case["kind"] == "product":
        spp.mx4_product_multi(ctx, s["lists"], s["w"], case["D"], sync=False)
        return s["y"]
    if case["kind"] == "grad":
        return spp.mx4_weight_grad(ctx, s["lists"], case["H"], case["D"], groups=case["groups"], sync=False)
    s["opt"].step(s["g"], sync=False)
    m, v = s["opt"].state(sync=False)
    return {"p": s["p"], "m": m, "v": v}


def _inside(s):
    """Which rows of the buffer a list holds: those before its count."""
    i = torch.arange(s["y"].shape[0], device=DEV)
    j = torch.searchsorted(s["from"], i, right=True) - 1
    return ((i - s["from"][j]) < s["n"][j]).unsqueeze(1)


def _run_plain(s):
    case, D = s["case"], s["case"]["D"] if "D" in s["case"] else 0
    if case["kind"] == "rows":
        return _values(_quantize(s["x"]), D).to(TYPES[case["out"]])
    if case["kind"] == "product":
        x, w = _values(s["rows"], D), _values(s["w"], D).view(case["groups"], case["H"], D)
        if case["groups"] == 1:
            y = x @ w[0].T
        else:
            y = torch.cat([x[a:b] @ w[k].T for a, b, k in s["parts"]])
        s["y"] = torch.where(_inside(s), y.to(s["y"].dtype), s["y"])
        return s["y"]
    if case["kind"] == "grad":
        x, y = _values(s["rows"], D), torch.where(_inside(s), s["y"].float(), 0)
        if case["groups"] == 1:
            return (y.T @ x).unsqueeze(0)
        w = torch.zeros(case["groups"], case["H"], D, device=DEV)
        [w[k].add_(y[a:b].T @ x[a:b]) for a, b, k in s["parts"]]
        return w
    s["t"] += 1
    small = case["bits"] == 8
    m = [_unpack_m(*q, p.numel()) for p, q in zip(s["p"], s["m"])] if small else s["m"]
    v = [_unpack_v(*q, p.numel()) for p, q in zip(s["p"], s["v"])] if small else s["v"]
    s["p"], m, v = map(list, zip(*[_step(p, g, a, b, s["t"]) for p, g, a, b in zip(s["p"], s["g"], m, v)]))
    if not small:
        s["m"], s["v"] = m, v
        return {"p": s["p"], "m": m, "v": v}
    s["m"], s["v"] = [_pack_m(a) for a in m], [_pack_v(b) for b in v]
    return {"p": s["p"], "m": [_unpack_m(*q, p.numel()) for p, q in zip(s["p"], s["m"])],
            "v": [_unpack_v(*q, p.numel()) for p, q in zip(s["p"], s["v"])]}


# ---- the definitions in 64 bits ------------------------------------------------------------------

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_rounded(x):
    """x [n, D] in float64, rounded to MXFP4 by the definition: the nearest of the eight magnitudes, ties to the even one."""
    n, D = x.shape
    out = torch.empty_like(x)
    mag = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    for c in range(0, D, 32):
        b = x[:, c:c + 32]
        top = b.abs().max(1, keepdim=True).values
        e = torch.floor(torch.log2(top.clamp(min=2.0 ** -125))) - 2
        q = (b.abs() / torch.exp2(e)).clamp(max=6.0)
        hi = torch.searchsorted(mag, q).clamp(1, 7)
        lo = hi - 1
        up, down = mag[hi] - q, q - mag[lo]
        pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
        out[:, c:c + 32] = torch.sign(b) * mag[pick] * torch.exp2(e)
    return out


def _exact_values(rows, D):
    r = rows.reshape(-1, rows.shape[-1])
    out = torch.empty(r.shape[0], D, dtype=torch.float64, device=r.device)
    mag = torch.tensor(E2M1, dtype=torch.float64, device=r.device)
    last = 16 * ((D + 31) // 32)
    for c in range(D):
        code = (r[:, c // 2] >> (4 * (c % 2))).long() & 15
        scale = torch.exp2(r[:, last + c // 32].double() - 127)
        out[:, c] = torch.where(code >= 8, -1.0, 1.0) * mag[code & 7] * scale
    return out


def _exact_state(x, least, mantissa, root):
    """A moment as an 8-bit state holds it: in blocks, floats of `mantissa` bits below the block's largest."""
    pad = torch.zeros((x.numel() + BLOCK - 1) // BLOCK * BLOCK, dtype=torch.float64, device=x.device)
    pad[:x.numel()] = x.sqrt() if root else x
    b = pad.view(-1, BLOCK)
    steps = 2 ** mantissa
    grid = torch.tensor([(1 + (c % steps) / steps) * 2.0 ** (c // steps - 15) for c in range(16 * steps)], dtype=torch.float64, device=x.device)
    grid[0] = 0
    unit = b.abs().max(1, keepdim=True).values / (2 - 1 / steps)
    q = b.abs() / torch.where(unit > 0, unit, 1)
    edge = torch.cat([torch.tensor([2.0 ** -15 * (1 + 0.5 / steps)], dtype=torch.float64, device=x.device), (grid[1:-1] + grid[2:]) / 2])
    code = torch.searchsorted(edge, q)
    if least:
        code = torch.where(q > 0, code.clamp(min=1), code)
    y = torch.sign(b) * grid[code] * unit
    return (y * y if root else y).view(-1)[:x.numel()]


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "rows":
        return torch.cat([_exact_rounded(s["x"][i:i + 100_000].double()) for i in range(0, case["n"], 100_000)])
    if kind == "adamw":
        (b1, b2), t, out = HYPER["betas"], s["t"] + 1, {"p": [], "m": [], "v": []}
        held = case["bits"] == 8
        for p, g, m, v in zip(s["p"], s["g"], s["m"], s["v"]):
            p, g, m, v = p.double(), g.double(), m.double(), v.double()
            if held:
                m, v = _exact_state(m, False, 3, False), _exact_state(v, True, 4, True)
            m = b1 * m + (1 - b1) * g
            v = b2 * v + (1 - b2) * g * g
            p = p - HYPER["lr"] * HYPER["weight_decay"] * p - HYPER["lr"] * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + HYPER["eps"])
            if held:
                m, v = _exact_state(m, False, 3, False), _exact_state(v, True, 4, True)
            out["p"].append(p)
            out["m"].append(m)
            out["v"].append(v)
        return out
    lists, total = _lists(case)
    D, H, G = case["D"], case["H"], case["groups"]
    if kind == "product":
        w = _exact_values(s["w"], D).view(G, H, D)
        y = torch.zeros(total, H, dtype=torch.float64, device=DEV)
        for a, cap, n, k in lists:
            y[a:a + n] = _exact_values(s["rows"][a:a + n], D) @ w[k].T
        return y
    w = torch.zeros(G, H, D, dtype=torch.float64, device=DEV)
    for a, cap, n, k in lists:
        w[k] += s["y"][a:a + n].double().T @ _exact_values(s["rows"][a:a + n], D)
    return w
