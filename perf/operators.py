"""The operators of an 8-bit decoder as cases that can be timed and checked: rows to 8 bits, the RMS norm in front of a
projection with the residual's addition and 8-bit rows as its result, the projection itself in 8-bit integers, appending
to a key-value cache held in 8 bits, and the attention that reads it.

`own` chooses between the operators' plain forms in elementary torch operations and the package's calls.  Sizes are those
of the shapes in `workload/shapes.py` ("8b": d 4096, 32/8 heads of 128, F 14336, V 128256; "1b": d 2048, 32/8 heads of
64, F 8192) and generic ones around them.

Rows in 8 bits come back as the values that they stand for, in bfloat16, next to their scales.
"""
import math

import torch

own = False

_T = {"fp32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases
def _rows(name, op, rows, n, dtype, add=""):
    return _named(name, {"op": op, "rows": rows, "n": n, "dtype": dtype, "add": add})


def _gemm(name, rows, n, k, dtype, gated=False):
    return _named(name, {"op": "gemm", "rows": rows, "n": n, "k": k, "dtype": dtype, "gated": gated})


def _kv(name, op, heads, seqs, ctx, rows, block, rope=True):
    """ctx: tokens that the longest sequence holds; rows: new tokens (append) or queries (attention) of all sequences."""
    hq, hkv, hd = heads
    return _named(name, {"op": op, "hq": hq, "hkv": hkv, "hd": hd, "seqs": seqs, "ctx": ctx, "rows": rows, "block": block, "rope": rope})


def _named(name, case):
    if name:
        case["name"] = name
    return case


_8B, _1B = (32, 8, 128), (32, 8, 64)


def listed():
    return [
        # the attention's result of one token of the 1B shape, on its way into the O-projection: nothing but latency
        _rows("quantize_1x2048_bf16", "quantize", 1, 2048, "bf16"),
        # the SwiGLU rows of a prompt of the 8B shape, on their way into the down projection
        _rows("quantize_2048x14336_bf16", "quantize", 2048, 14336, "bf16"),
        # eight draft rows between two blocks of the 8B shape: residual stream in fp32, what the projection adds in bf16
        _rows("rmsnorm_8x4096_fp32_bf16", "rmsnorm", 8, 4096, "fp32", "bf16"),
        # an odd number of prompt rows of an odd width
        _rows("rmsnorm_1531x2055_fp32_bf16", "rmsnorm", 1531, 2055, "fp32", "bf16"),
        # one token through the 1B shape's gate and up projections, SwiGLU in the epilogue
        _gemm("gemm_1x8192x2048_gated", 1, 8192, 2048, "bf16", True),
        # eight draft rows through the 8B shape's down projection, the longest contraction
        _gemm("gemm_8x4096x14336", 8, 4096, 14336, "bf16"),
        # the whole headline prompt through gate and up of the 8B shape
        _gemm("gemm_2048x14336x4096_gated", 2048, 14336, 4096, "bf16", True),
        # a verify window of five drafts behind an odd context, a scale for each token
        _kv("append_1b_ctx517_5rows", "append", _1B, 1, 517, 5, 1),
        # a prompt's stretch into blocks of 32 tokens, the first of them partly filled
        _kv("append_8b_ctx1000_2048rows_block32", "append", _8B, 1, 1000, 2048, 32),
        # one token of the 1B shape as a draft model
        _kv("attention_1b_ctx512_1row", "attention", _1B, 1, 512, 1, 1),
        # the longest verify window: 16 rows behind 16384 tokens
        _kv("attention_8b_ctx16384_16rows", "attention", _8B, 1, 16384, 16, 1),
        # the second half of a prompt of 2048 tokens and a bit, blocks of 64 tokens
        _kv("attention_8b_ctx1024_1111rows_block64", "attention", _8B, 1, 1024, 1111, 64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(("quantize", "rmsnorm", "gemm", "gemm", "append", "attention", "attention"))
    if op in ("quantize", "rmsnorm"):
        n = _log_int(rng, 64, 14336)
        rows = _log_int(rng, 1, 2048)
        return _rows(None, op, rows, n, rng.choice(("fp32", "bf16")), rng.choice(("", "bf16", "fp32")) if op == "rmsnorm" else "")
    if op == "gemm":
        n, k = _log_int(rng, 64, 16384), _log_int(rng, 64, 14336)
        if rng.random() < 0.5:
            n, k = (n + 15) // 16 * 16, (k + 63) // 64 * 64
        gated = rng.random() < 0.3
        n = min(n, (1 << 26) // k)
        rows = rng.choice((rng.randint(1, 16), _log_int(rng, 1, 2048)))
        if rng.random() < 0.15:
            n, k, rows, gated = rng.choice((32000, 128256)), min(k, 4096), rng.randint(1, 16), False    # the vocabularies
        return _gemm(None, rows, n, k, "bf16" if gated else rng.choice(("bf16", "fp32")), gated)
    heads = rng.choice((_8B, _1B, (4, 4, 64), (8, 4, 128), (8, 1, 64), (16, 2, 128)))
    block, seqs = rng.choice((1, 1, 16, 32, 64)), rng.choice((1, 1, rng.randint(2, 8)))
    rows = rng.randint(seqs, 16) if rng.random() < 0.6 else _log_int(rng, 17, 2000 if op == "append" else 1000)
    ctx = _log_int(rng, 1, 16384 if rows <= 16 else 1200)
    if seqs > 1:
        ctx = min(ctx, 5000)
    return _kv(None, op, heads, seqs, ctx, rows, block, rng.random() < 0.8)


# ---------------------------------------------------------------- inputs
def _lengths(case, seed):
    """Tokens held and new tokens of each sequence; the first holds the most."""
    gen = torch.Generator().manual_seed((seed * 2 + 1) % (1 << 62))
    n, rows = case["seqs"], case["rows"]
    ctx = [case["ctx"]] + torch.randint(case["ctx"] // 4, case["ctx"] + 1, (n - 1,), generator=gen).tolist()
    cuts = sorted((torch.randperm(rows - 1, generator=gen)[:n - 1] + 1).tolist()) if rows > 1 else []
    ends = cuts + [rows]
    return ctx, [e - b for b, e in zip([0] + cuts, ends)]


def _rope_tables(positions, hd):
    """cos and sin of position * 500000^(-2i/hd) in fp32, angles in 64 bits."""
    inv = 500000.0 ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64) / hd)
    ang = torch.arange(positions, dtype=torch.float64)[:, None] * inv
    return torch.cos(ang).float().cuda(), torch.sin(ang).float().cuda()


def _inputs(case, seed):
    """The tensors that a case begins with, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std)

    if op in ("quantize", "rmsnorm"):
        rows, n = case["rows"], case["n"]
        t = {"x": (normal(rows, n) * torch.exp(normal(rows, 1))).to(_T[case["dtype"]])}
        if op == "rmsnorm":
            t["gain"] = 1.0 + normal(n, std=0.02)
            t["eps"] = 1e-5
            if case["add"]:
                t["add"] = normal(rows, n, std=0.3).to(_T[case["add"]])
        return t
    if op == "gemm":
        rows, n, k = case["rows"], case["n"], case["k"]
        m = 2 * n if case["gated"] else n
        # weights and rows as symmetric quantisation of normal values leaves them
        w = normal(m, k, std=127 / 4.5).round_().clamp_(-127, 127).to(torch.int8)
        x = normal(rows, k, std=127 / 4.0).round_().clamp_(-127, 127).to(torch.int8)
        sw = torch.exp(normal(m, std=0.1)) * (0.02 * 4.5 / 127)
        sx = torch.exp(normal(rows, std=0.3)) * (4.0 / 127)
        return {"w": w, "sw": sw, "x": x, "sx": sx}
    ctx, new = _lengths(case, seed)
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    t = {"ctx": ctx, "new": new}
    # attention: the rows that are asked about are in the cache like all others
    held = [c + (k if op == "attention" else 0) for c, k in zip(ctx, new)]
    t["k_held"] = [(normal(n, hkv, hd) * torch.exp(normal(1, hkv, hd, std=0.5))).to(torch.bfloat16) for n in held]
    t["v_held"] = [normal(n, hkv, hd).to(torch.bfloat16) for n in held]
    t["held"] = held
    if op == "append":
        t["k"] = (normal(case["rows"], hkv, hd) * torch.exp(normal(1, hkv, hd, std=0.5))).to(torch.bfloat16)
        t["v"] = normal(case["rows"], hkv, hd).to(torch.bfloat16)
    else:
        t["q"] = normal(case["rows"], hq, hd).to(torch.bfloat16)
    t["cos"], t["sin"] = _rope_tables(max(c + k for c, k in zip(ctx, new)), hd) if case["rope"] else (None, None)
    return t


def _pad16(n):
    return (n + 15) // 16 * 16


def _pad_rows(t):
    """Rows of bytes at a distance that is a multiple of 16."""
    out = torch.zeros(t.shape[0], _pad16(t.shape[1]), dtype=t.dtype, device="cuda")
    out[:, :t.shape[1]] = t
    return out


def _capacity(t, block):
    return (max(c + k for c, k in zip(t["ctx"], t["new"])) + 63) // 64 * 64


def prepare(case, seed):
    t = _inputs(case, seed)
    op = case["op"]
    s = {"op": op, **{k: v for k, v in case.items() if k != "name"}}
    if op in ("quantize", "rmsnorm"):
        rows, n = case["rows"], case["n"]
        s.pop("add")                                              # (the case's: a type, or that there is none)
        s.update(t)
        s["q8"] = torch.zeros(rows, _pad16(n), dtype=torch.int8, device="cuda")
        s["scale"] = torch.empty(rows, device="cuda")
        s["values"] = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
        s["sum"] = torch.empty_like(t["x"])
    elif op == "gemm":
        s["x"], s["sx"] = _pad_rows(t["x"]), t["sx"]
        s["out"] = torch.empty(case["rows"], case["n"], dtype=_T[case["dtype"]], device="cuda")
        if own:
            import paper_2410_17375_amd as A
            torch.cuda.synchronize()
            s["matrix"] = A.Q8Matrix(t["w"].data_ptr(), A.DTYPE_INT8, t["w"].shape[0], case["k"], scale=t["sw"].data_ptr(),
                                     gated=case["gated"], on_device=True)
            s["work"] = torch.zeros(max(16, s["matrix"].workspace_bytes(case["rows"])), dtype=torch.uint8, device="cuda")
        else:
            s["w"], s["sw"] = t["w"], t["sw"]
    else:
        _prepare_cache(case, t, s)
    return s


def _prepare_cache(case, t, s):
    """The cache with what its sequences hold, and for the plain form where each new row goes in padded arrays."""
    hkv, hd, block, n = case["hkv"], case["hd"], case["block"], case["seqs"]
    cap = _capacity(t, block)
    s.update({k: t[k] for k in ("ctx", "new", "cos", "sin")})
    s["ids"] = list(range(n))
    for name in ("q", "k", "v"):
        if name in t:
            s[name] = t[name]
    if case["op"] == "attention":
        s["out"] = torch.empty(case["rows"], case["hq"], hd, dtype=torch.bfloat16, device="cuda")
    else:
        # what comes back: every row of the blocks that the new rows reach into
        s["first"] = [c // block * block for c in t["ctx"]]
        s["back"] = [c + k - f for c, k, f in zip(t["ctx"], t["new"], s["first"])]
        for name in ("k_back", "v_back"):
            s[name] = torch.empty(sum(s["back"]), hkv, hd, dtype=torch.bfloat16, device="cuda")
    if own:
        import paper_2410_17375_amd as A
        cache = A.Q8Cache(n_layers=1, n_seqs=n, n_q_heads=case["hq"], n_kv_heads=hkv, head_dim=hd, capacity=cap, block=block)
        torch.cuda.synchronize()
        ptr = [0, 0] if t["cos"] is None else [t["cos"].data_ptr(), t["sin"].data_ptr()]
        for i, held in enumerate(t["held"]):
            if held:
                cache.append(0, [i], [0], [held], t["k_held"][i].data_ptr(), t["v_held"][i].data_ptr(), hkv * hd, *ptr)
        torch.cuda.synchronize()
        s["cache"] = cache
        return
    blocks = cap // block + 1                                     # the last one takes what pads the index arrays
    s["k8"], s["ks"] = _blank(n, hkv, blocks, block, hd)
    s["v8"], s["vs"] = _blank(n, hkv, blocks, block, hd)
    for i, held in enumerate(t["held"]):
        for x, q8, sc, turn in ((t["k_held"][i], s["k8"], s["ks"], True), (t["v_held"][i], s["v8"], s["vs"], False)):
            x = x.float()
            if turn and t["cos"] is not None:
                x = _turn(x, t["cos"][:held], t["sin"][:held])
            full = torch.zeros(blocks * block, hkv, hd, device="cuda")
            full[:held] = x
            full = full.view(blocks, block, hkv, hd).permute(2, 0, 1, 3)
            scale = full.abs().amax((2, 3)) / 127
            sc[i] = scale
            q8[i] = torch.round(full / torch.where(scale > 0, scale, 1.0)[:, :, None, None]).to(torch.int8)
    dev = lambda v: torch.tensor(v, device="cuda")   # noqa: E731
    seq = [i for i, k in enumerate(t["new"]) for _ in range(k)]
    pos = [c + j for c, k in zip(t["ctx"], t["new"]) for j in range(k)]
    s["row_seq"], s["row_pos"] = dev(seq), dev(pos)
    s["row_at"] = dev([j for k in t["new"] for j in range(k)])
    if case["op"] == "append":
        touched = [list(range(c // block, (c + k - 1) // block + 1)) for c, k in zip(t["ctx"], t["new"])]
        most = max(len(b) for b in touched)
        s["touched"] = dev([b + [blocks - 1] * (most - len(b)) for b in touched])
        s["row_touched"] = dev([p // block - t["ctx"][i] // block for i, p in zip(seq, pos)])
        s["row_off"] = dev([p % block for p in pos])
        at = s["touched"][:, :, None] * block + torch.arange(block, device="cuda")
        s["held_mask"] = at < dev(t["ctx"])[:, None, None]
        bseq = [i for i, b in enumerate(s["back"]) for _ in range(b)]
        bpos = [f + j for f, b in zip(s["first"], s["back"]) for j in range(b)]
        s["back_seq"], s["back_block"], s["back_off"] = dev(bseq), dev([p // block for p in bpos]), dev([p % block for p in bpos])


def _blank(n, hkv, blocks, block, hd):
    return (torch.zeros(n, hkv, blocks, block, hd, dtype=torch.int8, device="cuda"), torch.zeros(n, hkv, blocks, device="cuda"))


# ---------------------------------------------------------------- one pass
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2410_17375_amd as A
    op, stream = s["op"], torch.cuda.current_stream().cuda_stream
    code = {torch.float32: A.DTYPE_FP32, torch.bfloat16: A.DTYPE_BF16}
    if op == "quantize":
        x, q8 = s["x"], s["q8"]
        A.q8_quantize(x.data_ptr(), code[x.dtype], s["n"], s["rows"], s["n"], q8.data_ptr(), q8.shape[1], s["scale"].data_ptr(), stream)
        return {"values": torch.mul(q8[:, :s["n"]], s["scale"][:, None], out=s["values"]), "scale": s["scale"]}
    if op == "rmsnorm":
        x, q8, add = s["x"], s["q8"], s.get("add")
        A.q8_rmsnorm(x.data_ptr(), code[x.dtype], s["n"], 0 if add is None else add.data_ptr(), code[x.dtype if add is None else add.dtype], s["n"],
                     s["gain"].data_ptr(), s["eps"], s["rows"], s["n"], s["sum"].data_ptr(), s["n"], q8.data_ptr(), q8.shape[1],
                     s["scale"].data_ptr(), stream)
        return {"sum": s["sum"], "values": torch.mul(q8[:, :s["n"]], s["scale"][:, None], out=s["values"]), "scale": s["scale"]}
    if op == "gemm":
        x, out, work = s["x"], s["out"], s["work"]
        A.q8_gemm(s["matrix"], x.data_ptr(), x.shape[1], s["sx"].data_ptr(), s["rows"], out.data_ptr(), code[out.dtype], s["n"],
                  work.data_ptr(), work.numel(), stream)
        return {"out": out}
    cos, sin = (0, 0) if s["cos"] is None else (s["cos"].data_ptr(), s["sin"].data_ptr())
    width = s["hkv"] * s["hd"]
    if op == "append":
        s["cache"].append(0, s["ids"], s["ctx"], s["new"], s["k"].data_ptr(), s["v"].data_ptr(), width, cos, sin, stream)
        s["cache"].read(0, s["ids"], s["first"], s["back"], s["k_back"].data_ptr(), s["v_back"].data_ptr(), A.DTYPE_BF16, width, stream)
        return {"k": s["k_back"], "v": s["v_back"]}
    s["cache"].attention(0, s["ids"], s["ctx"], s["new"], s["q"].data_ptr(), s["hq"] * s["hd"], s["hd"] ** -0.5, cos, sin,
                         s["out"].data_ptr(), s["hq"] * s["hd"], stream)
    return {"out": s["out"]}


def _to_q8(v):
    """Rows in 8 bits and their scales; v in 64 bits where it is the result of sums, whose last bits decide at borders."""
    scale = (v.abs().amax(1) / 127).float()
    q = torch.round(v / torch.where(scale > 0, scale, 1.0)[:, None].to(v.dtype))
    return {"values": (q.float() * scale[:, None]).to(torch.bfloat16), "scale": scale}


def _turn(x, cos, sin):
    """Rotary: pairs (i, i + hd/2) of [n, heads, hd] turned by the angles of their rows."""
    h = x.shape[-1] // 2
    a, b, c, d = x[..., :h], x[..., h:], cos[:, None, :], sin[:, None, :]
    return torch.cat([a * c - b * d, a * d + b * c], -1)


def _grow(q8, scale, touched, held, new):
    """The touched blocks of a cache after new values: q8 [n, hkv, blocks, block, hd], new [n, touched, block, hkv, hd]."""
    n, hkv = q8.shape[:2]
    seq = torch.arange(n, device="cuda")[:, None]
    old = q8[seq, :, touched].float()                                             # [n, touched, hkv, block, hd]
    was = scale[seq, :, touched] * held.any(-1)[:, :, None]                       # blocks that begin here have no scale yet
    new = new.transpose(2, 3)
    now = torch.maximum(was, new.abs().amax((3, 4)) / 127)
    safe = torch.where(now > 0, now, 1.0)[..., None, None]
    kept = torch.round(old * (was[..., None, None] / safe)) * held[:, :, None, :, None]
    q8[seq, :, touched] = (kept + torch.round(new / safe)).to(torch.int8)
    scale[seq, :, touched] = now


def _run_plain(s):
    op = s["op"]
    if op == "quantize":
        return _to_q8(s["x"].float())
    if op == "rmsnorm":
        x = s["x"].float()
        if "add" in s:
            x = x + s["add"].float()
        w = x.double()
        y = w / torch.sqrt((w * w).mean(1, keepdim=True) + s["eps"]) * s["gain"]
        return {"sum": x.to(s["x"].dtype), **_to_q8(y)}
    if op == "gemm":
        k = s["k"]
        y = (s["x"][:, :k].float() @ s["w"].float().T) * s["sx"][:, None] * s["sw"]
        if s["gated"]:
            g, u = y[:, :s["n"]], y[:, s["n"]:]
            y = g / (1 + torch.exp(-g)) * u
        return {"out": y.to(s["out"].dtype)}
    n, hkv, hd, block = s["seqs"], s["hkv"], s["hd"], s["block"]
    if op == "append":
        k, v = s["k"].float(), s["v"].float()
        if s["cos"] is not None:
            k = _turn(k, s["cos"][s["row_pos"]], s["sin"][s["row_pos"]])
        k_new, v_new = (torch.zeros(n, s["touched"].shape[1], block, hkv, hd, device="cuda") for _ in range(2))
        k_new[s["row_seq"], s["row_touched"], s["row_off"]] = k
        v_new[s["row_seq"], s["row_touched"], s["row_off"]] = v
        _grow(s["k8"], s["ks"], s["touched"], s["held_mask"], k_new)
        _grow(s["v8"], s["vs"], s["touched"], s["held_mask"], v_new)
        at = (s["back_seq"], slice(None), s["back_block"])
        return {"k": (s["k8"][at + (s["back_off"],)].float() * s["ks"][at][..., None]).to(torch.bfloat16),
                "v": (s["v8"][at + (s["back_off"],)].float() * s["vs"][at][..., None]).to(torch.bfloat16)}
    group, most, keys = s["hq"] // hkv, max(s["new"]), max(c + k for c, k in zip(s["ctx"], s["new"]))
    q = s["q"].float()
    if s["cos"] is not None:
        q = _turn(q, s["cos"][s["row_pos"]], s["sin"][s["row_pos"]])
    padded = torch.zeros(n, most, hkv, group, hd, device="cuda")
    padded[s["row_seq"], s["row_at"]] = q.view(-1, hkv, group, hd)
    padded = padded.permute(0, 2, 1, 3, 4).reshape(n, hkv, most * group, hd)
    k = (s["k8"].float() * s["ks"][..., None, None]).view(n, hkv, -1, hd)[:, :, :keys]
    v = (s["v8"].float() * s["vs"][..., None, None]).view(n, hkv, -1, hd)[:, :, :keys]
    score = (padded @ k.transpose(2, 3)).view(n, hkv, most, group, keys) * hd ** -0.5
    last = torch.tensor(s["ctx"], device="cuda")[:, None] + torch.arange(most, device="cuda")
    score = score.masked_fill(torch.arange(keys, device="cuda") > last[:, None, :, None, None], float("-inf"))
    p = torch.exp(score - score.amax(-1, keepdim=True))
    o = (p.view(n, hkv, most * group, keys) @ v) / p.sum(-1).view(n, hkv, most * group, 1)
    o = o.view(n, hkv, most, group, hd).permute(0, 2, 1, 3, 4)[s["row_seq"], s["row_at"]]
    return {"out": o.reshape(-1, s["hq"], hd).to(torch.bfloat16)}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    op = case["op"]
    size = {"fp32": 4, "bf16": 2, "": 0}
    if op in ("quantize", "rmsnorm"):
        rows, n = case["rows"], case["n"]
        e = size[case["dtype"]]
        nbytes = rows * (n * (e + 1) + 4)
        if op == "rmsnorm":
            nbytes += rows * n * (e + size[case["add"]]) + 4 * n
        return {"bytes": nbytes, "flops": rows * n * (3 if op == "quantize" else 8)}
    if op == "gemm":
        rows, n, k = case["rows"], case["n"], case["k"]
        m = 2 * n if case["gated"] else n
        return {"bytes": m * k + 4 * m + rows * k + 4 * rows + rows * n * size[case["dtype"]], "flops": 2 * rows * m * k}
    rows, hkv, hd, block, n = case["rows"], case["hkv"], case["hd"], case["block"], case["seqs"]
    held = case["ctx"] + (n - 1) * (5 * case["ctx"] // 8)                # drawn lengths: their mean
    if op == "append":
        partly = n * (block - 1) // 2 if block > 1 else 0               # held rows of the first blocks, read and written
        return {"bytes": 2 * hkv * hd * (2 * rows + rows + 2 * partly), "flops": 2 * hkv * hd * rows * 6}
    per = rows / n
    pairs = sum(per * c + per * (per + 1) / 2 for c in [case["ctx"]] + [5 * case["ctx"] / 8] * (n - 1))
    nbytes = 2 * hkv * (held + rows) * (hd + 4 / block) + rows * case["hq"] * hd * 4
    return {"bytes": int(nbytes), "flops": int(4 * case["hq"] * hd * pairs)}


# ---------------------------------------------------------------- the same in 64 bits
def _exact_q8(v):
    scale = v.abs().max(1).values / 127
    whole = (v / scale.clamp_min(1e-300)[:, None]).round()
    return {"values": whole * scale[:, None], "scale": scale}


def _exact_rotated(x, first, theta_on):
    """[n, heads, hd] at positions first, first + 1, ..: every pair as a complex number times e^(i angle)."""
    x = x.double()
    if not theta_on:
        return x
    n, _, hd = x.shape
    freq = 500000.0 ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64) / hd)
    ang = (torch.arange(first, first + n, dtype=torch.float64)[:, None] * freq).cuda()
    z = torch.complex(x[..., :hd // 2].contiguous(), x[..., hd // 2:].contiguous()) * torch.polar(torch.ones_like(ang), ang)[:, None, :]
    return torch.cat([z.real, z.imag], -1)


def _exact_blocks(x, block):
    """The integers and the scales (a row each) of rows [n, heads, hd] that come into empty blocks together."""
    n, heads, hd = x.shape
    whole = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, -n % block)).view(-1, block, heads, hd)
    scale = whole.abs().amax((1, 3), keepdim=True) / 127
    ints = (whole / scale.clamp_min(1e-300)).round()
    return ints.reshape(-1, heads, hd)[:n], scale.expand(-1, block, -1, 1).reshape(-1, heads, 1)[:n]


def exact(case, seed):
    t = _inputs(case, seed)
    op = case["op"]
    if op == "quantize":
        return _exact_q8(t["x"].double())
    if op == "rmsnorm":
        x = t["x"].double() + (t["add"].double() if "add" in t else 0)
        rms = ((x ** 2).sum(1) / x.shape[1] + t["eps"]).sqrt()
        return {"sum": x, **_exact_q8(x * t["gain"].double() / rms[:, None])}
    if op == "gemm":
        w = t["w"].double() * t["sw"].double()[:, None]
        y = torch.matmul(t["x"].double() * t["sx"].double()[:, None], w.t())
        if case["gated"]:
            y = y[:, :case["n"]] * torch.sigmoid(y[:, :case["n"]]) * y[:, case["n"]:]
        return {"out": y}
    hq, hkv, hd, block, rope = (case[k] for k in ("hq", "hkv", "hd", "block", "rope"))
    outs = {"k": [], "v": []} if op == "append" else {"out": []}
    row = 0
    for c, n, k_held, v_held in zip(t["ctx"], t["new"], t["k_held"], t["v_held"]):
        pair = [_exact_rotated(k_held, 0, rope), v_held.double()]
        if op == "append":
            new = [_exact_rotated(t["k"][row:row + n], c, rope), t["v"][row:row + n].double()]
            first = c // block * block
            for key, held, x in (("k", pair[0], new[0]), ("v", pair[1], new[1])):
                ints, scale = _exact_blocks(held[first:], block)             # what the first block holds
                end = min(n, first + block - c)
                s1 = x[:end].abs().amax((0, 2))[:, None] / 127
                if c > first:
                    s0 = scale[0]
                    s1 = torch.maximum(s0, s1)
                    kept = (ints * (s0 / s1)).round() * s1
                else:
                    kept = x[:0]
                into = (x[:end] / s1).round() * s1
                q, sc = _exact_blocks(x[end:], block) if end < n else (x[:0], 1.0)
                outs[key].append(torch.cat([kept, into, q * sc]))
        else:
            k, v = (q * sc for q, sc in (_exact_blocks(x, block) for x in pair))
            q = _exact_rotated(t["q"][row:row + n], c, rope)
            o = torch.empty(n, hq, hd, dtype=torch.float64, device="cuda")
            for h in range(hq):
                kh, vh = k[:, h * hkv // hq].contiguous(), v[:, h * hkv // hq].contiguous()
                z = (q[:, h].contiguous() @ kh.t().contiguous()) / math.sqrt(hd)
                z.masked_fill_(torch.ones_like(z, dtype=torch.bool).triu_(c + 1), -math.inf)
                o[:, h] = torch.softmax(z, 1) @ vh
            outs["out"].append(o)
        row += n
    return {k: torch.cat(v) for k, v in outs.items()}
