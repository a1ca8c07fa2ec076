"""Operators on 4-bit floating point and on experts, as cases that can be timed and compared: quantisation of
activations, the product of two quantised matrices, the same product grouped by expert, the router that groups the
tokens, and the weighted sum that brings the experts' results back to them.

Storage of a quantised matrix (the library's own, include/bnn.h):
  codes   uint8 [rows][pitch], pitch = ceil(K / 32) * 16: element k of a row is the low (k even) or high nibble of byte
          k / 2, an e2m1 number (sign, two exponent bits, one mantissa bit: 0 .5 1 1.5 2 3 4 6); positions >= K hold 0.
  scales  uint8, tiles of 128 rows x 4 scales of 512 bytes, [row tile][tile of scales]: the scale of row r and block b of
          a tile is byte (r % 32) * 16 + (r / 32) * 4 + b.  "mx": one scale per 32 elements, 2^(byte - 127); "nv": one per
          16 elements, an e4m3 number.  Scales of blocks at or beyond K hold 0.
  Rows in groups (experts): group g has rows offsets[g] .. offsets[g + 1] - 1 and its own row tiles, the first of which
          is tile offsets[g] / 128 + g, so that a group starts at row 0 of a tile.

Plain forms: torch in 32 bits, one operation after another.  ``own`` switches ``run`` to the library's entry points."""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
BLOCK = {"mx": 32, "nv": 16}
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # ten live 11-frame windows of 40 features before a 4-bit first layer
        dict(name="quantize_chunk", op="quantize", rows=10, K=440, fmt="nv", dtype="f32", experts=0, tokens=0),
        # the activations of 4096 tokens, four experts each, gathered in the experts' order
        dict(name="quantize_experts", op="quantize", rows=16384, K=4096, fmt="mx", dtype="bf16", experts=32, tokens=4096),
        # one token through one 4-bit layer
        dict(name="gemm_token", op="gemm", M=1, K=2048, N=2048, fmt="mx", dtype="bf16", bias=False),
        # one 7 s utterance through a top layer of 3307 states, with its bias
        dict(name="gemm_utterance", op="gemm", M=731, K=2048, N=3307, fmt="nv", dtype="f32", bias=True),
        # a batch through a wide layer
        dict(name="gemm_batch", op="gemm", M=8192, K=4096, N=8192, fmt="mx", dtype="bf16", bias=False),
        # a decoding step of eight tokens, eight of 64 experts each: mostly one row to an expert, some without
        dict(name="experts_step", op="grouped", rows=64, K=2048, N=2048, experts=64, fmt="mx", dtype="bf16"),
        # an utterance, two of 16 experts each, on widths that fill no tile
        dict(name="experts_ragged", op="grouped", rows=1462, K=1000, N=1333, experts=16, fmt="nv", dtype="f32"),
        # a batch of 8192 tokens, two of 32 experts each
        dict(name="experts_batch", op="grouped", rows=16384, K=2048, N=4096, experts=32, fmt="mx", dtype="bf16"),
        # the router on a decoding step, and on a batch with padded positions
        dict(name="route_step", op="route", T=8, E=64, k=8, dtype="bf16", chosen=True, padded=False),
        dict(name="route_batch", op="route", T=16384, E=256, k=8, dtype="f32", chosen=False, padded=True),
        # the experts' results of a decoding step, and of a batch
        dict(name="combine_step", op="combine", T=8, k=8, N=2048, dtype="bf16"),
        dict(name="combine_batch", op="combine", T=8192, k=4, N=4096, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.4 else max(lo, n // 64 * 64)


def draw(rng):
    op = rng.choice(["quantize", "gemm", "gemm", "grouped", "grouped", "route", "combine"])
    fmt, dtype = rng.choice(["mx", "nv"]), rng.choice(["f32", "f16", "bf16"])
    if op == "quantize":
        c = dict(op=op, rows=_log_int(rng, 1, 16384), K=_width(rng, 200, 8192), fmt=fmt, dtype=dtype, experts=0, tokens=0)
        if rng.random() < 0.5:
            c["experts"] = _log_int(rng, 2, 128)
            c["tokens"] = max(1, c["rows"] // rng.randint(1, 8))
        while c["rows"] > 1 and c["rows"] * c["K"] > 16384 * 4096:
            c["rows"] = c["rows"] // 2 + 1
        return c
    if op == "gemm":
        c = dict(op=op, M=_log_int(rng, 1, 8192), K=_width(rng, 200, 8192), N=_width(rng, 200, 8192), fmt=fmt, dtype=dtype, bias=rng.random() < 0.5)
        c["M"] = max(1, min(c["M"], 8192 * 4096 * 8192 // (c["K"] * c["N"])))
        return c
    if op == "grouped":
        c = dict(op=op, rows=_log_int(rng, 1, 16384), K=_width(rng, 200, 4096), N=_width(rng, 200, 4096), experts=_log_int(rng, 2, 128), fmt=fmt, dtype=dtype)
        c["experts"] = max(2, min(c["experts"], 64 * 2048 * 2048 // (c["K"] * c["N"])))
        c["rows"] = max(1, min(c["rows"], 16384 * 2048 * 4096 // (c["K"] * c["N"])))
        return c
    if op == "route":
        return dict(op=op, T=_log_int(rng, 1, 16384), E=_log_int(rng, 8, 256), k=rng.randint(1, 8), dtype=dtype, chosen=rng.random() < 0.5, padded=rng.random() < 0.5)
    c = dict(op=op, T=_log_int(rng, 1, 8192), k=rng.randint(1, 8), N=_width(rng, 200, 8192), dtype=dtype)
    while c["T"] > 1 and c["T"] * (c["k"] + 1) * c["N"] > 8192 * 5 * 4096 // (2 if dtype == "f32" else 1):
        c["T"] = c["T"] // 2 + 1
    return c


# ---- the quantised form in plain torch ------------------------------------------------------------------

def _pitch(K):
    return (K + 31) // 32 * 16


def _scale_tiles(fmt, K):
    return (K + 4 * BLOCK[fmt] - 1) // (4 * BLOCK[fmt])


def _power(e):
    """2^e for whole numbers e, as doubles, by the exponent's bits (an exp2 may be off in the last place)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _blocks(x, fmt):
    """[rows][K] -> fp32 [rows][blocks][32 or 16], zero behind K, blocks to a multiple of four."""
    rows, K = x.shape
    wide = _scale_tiles(fmt, K) * 4 * BLOCK[fmt]
    return torch.nn.functional.pad(x.float(), (0, wide - K)).view(rows, -1, BLOCK[fmt])


def _codes_and_scales(x, fmt, exponent=0):
    """e2m1 codes (int, one per element, [rows][padded K]) and scale bytes ([rows][scales])."""
    b = _blocks(x, fmt) * 2.0 ** exponent
    most = b.abs().amax(-1)
    if fmt == "mx":
        e = (torch.frexp(most).exponent - 1 - 2).clamp(-127, 127)   # floor(log2(most)) - 2
        e = torch.where(most == 0, -127, e)
        byte = (e + 127).to(torch.uint8)
        scaled = b.double().abs() * _power(-e).unsqueeze(-1)
    else:
        s = (most / 6).clamp(max=448.0).to(torch.float8_e4m3fn)
        byte = s.view(torch.uint8)
        s = s.double().unsqueeze(-1)
        scaled = torch.where(s > 0, b.double().abs() / s, 0.0)
    # to the nearest, ties to the even code
    code = ((scaled > 0.25).int() + (scaled >= 0.75).int() + (scaled > 1.25).int() + (scaled >= 1.75).int() +
            (scaled > 2.5).int() + (scaled >= 3.5).int() + (scaled > 5.0).int())
    code = (code + 8 * torch.signbit(b).int()).to(torch.uint8)
    there = torch.arange(byte.shape[1], device=x.device) * BLOCK[fmt] < x.shape[1]
    return code.flatten(1), torch.where(there, byte, torch.zeros_like(byte))


def _row_places(rows, offsets):
    """Row of the scale tiles that each row's scales are in."""
    r = torch.arange(rows, device=DEV)
    if offsets is None:
        return r
    off = offsets.long()
    g = (torch.searchsorted(off, r, right=True) - 1).clamp(0, off.numel() - 2)
    return (off[g] // 128 + g) * 128 + r - off[g]


def _store(code, byte, K, fmt, offsets, groups):
    """The stored form: (codes, scales)."""
    rows = code.shape[0]
    wide = _pitch(K) * 2
    code = torch.nn.functional.pad(code, (0, max(0, wide - code.shape[1])))[:, :wide]
    packed = code[:, 0::2] | (code[:, 1::2] << 4)
    tiles, kt = rows // 128 + groups, byte.shape[1] // 4
    flat = torch.zeros((tiles * 128, kt * 4), dtype=torch.uint8, device=DEV)
    flat[_row_places(rows, offsets)] = byte
    return packed.contiguous(), flat.view(tiles, 4, 32, kt, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _values(codes, scales, K, fmt, offsets=None, groups=1):
    """Stored form -> fp32 [rows][K]."""
    rows = codes.shape[0]
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
    v = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), -1).flatten(1)[:, :K]
    tiles, kt = rows // 128 + groups, _scale_tiles(fmt, K)
    s = scales.view(tiles, kt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(tiles * 128, kt * 4)[_row_places(rows, offsets)]
    s = _power(s.int() - 127).float() if fmt == "mx" else s.view(torch.float8_e4m3fn).float()
    return v * s.repeat_interleave(BLOCK[fmt], 1)[:, :K]


def _stored(x, fmt, exponent=0, offsets=None, groups=1):
    code, byte = _codes_and_scales(x, fmt, exponent)
    return _store(code, byte, x.shape[1], fmt, offsets, groups)


# ---- inputs -----------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _activations(g, rows, K):
    """N(0, 1) with a few channels that are much larger, as hidden activations have them."""
    loud = torch.where(torch.rand((K,), generator=g, device=DEV) < 0.01, 8.0, 1.0)
    return torch.randn((rows, K), generator=g, device=DEV) * loud


def _offsets(g, rows, experts):
    """Rows spread over experts of unequal popularity: int32 [experts + 1]."""
    p = torch.softmax(0.7 * torch.randn((experts,), generator=g, device=DEV), 0)
    e = torch.multinomial(p, rows, replacement=True, generator=g)
    return torch.nn.functional.pad(torch.bincount(e, minlength=experts).cumsum(0), (1, 0)).int()


#: Weights have a spread of about 1 / sqrt(K): as e4m3 scales they would lie among the subnormal ones, so they are
#: multiplied by 2^6 before quantisation and the product by 2^-6.
EXPONENT = {"mx": 0, "nv": 6}


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    dt = DTYPE[case["dtype"]]
    if op == "quantize":
        rows, K, fmt, n = case["rows"], case["K"], case["fmt"], case["experts"]
        offsets = source = None
        x = _activations(g, case["tokens"] if n else rows, K).to(dt)
        if n:
            offsets = _offsets(g, rows, n)
            source = torch.randint(0, case["tokens"], (rows,), generator=g, device=DEV, dtype=torch.int32)
        return dict(op=op, x=x, K=K, fmt=fmt, offsets=offsets, source=source, groups=max(n, 1),
                    codes=torch.zeros((rows, _pitch(K)), dtype=torch.uint8, device=DEV),
                    scales=torch.zeros(((rows // 128 + max(n, 1)) * _scale_tiles(fmt, K) * 512,), dtype=torch.uint8, device=DEV),
                    values=torch.empty((rows, K), dtype=torch.bfloat16, device=DEV))
    if op in ("gemm", "grouped"):
        rows, K, N, fmt, n = case.get("M") or case["rows"], case["K"], case["N"], case["fmt"], case.get("experts", 1)
        offsets = _offsets(g, rows, n) if op == "grouped" else None
        a, a_scales = _stored(_activations(g, rows, K), fmt, 0, offsets, n)
        w_offsets = torch.arange(n + 1, device=DEV, dtype=torch.int32) * N if op == "grouped" else None
        w = torch.cat([torch.randn((N, K), generator=g, device=DEV).to(torch.bfloat16) for _ in range(n)]) / math.sqrt(K)
        parts = [_codes_and_scales(w[i:i + 65536], fmt, EXPONENT[fmt]) for i in range(0, n * N, 65536)]
        w, w_scales = _store(torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts]), K, fmt, w_offsets, n)
        most = int((offsets[1:] - offsets[:-1]).max()) if op == "grouped" else rows
        return dict(op=op, a=a, a_scales=a_scales, w=w.view(n, N, -1) if op == "grouped" else w, w_scales=w_scales, K=K, N=N, fmt=fmt,
                    offsets=offsets, w_offsets=w_offsets, groups=n, most=most, exponent=-EXPONENT[fmt],
                    bias=torch.randn((N,), generator=g, device=DEV) if case.get("bias") else None,
                    y=torch.empty((rows, N), dtype=dt, device=DEV))
    T, k = case["T"], case["k"]
    if op == "route":
        E = case["E"]
        logits = (torch.randn((T, E), generator=g, device=DEV) + torch.randn((E,), generator=g, device=DEV)).to(dt)
        if case["padded"]:   # positions without a token
            logits[torch.rand((T,), generator=g, device=DEV) < 0.1] = -math.inf
        i32 = dict(dtype=torch.int32, device=DEV)
        # what no token was routed to stays as it was: -1
        return dict(op=op, logits=logits, k=k, chosen=case["chosen"], index=torch.empty((T, k), **i32), weight=torch.empty((T, k), device=DEV),
                    offsets=torch.empty((E + 1,), **i32), slot=torch.empty((T, k), **i32), source=torch.full((T * k,), -1, **i32),
                    workspace=None)
    z = torch.randn((T * k, case["N"]), generator=g, device=DEV).to(dt)
    slot = torch.randperm(T * k, generator=g, device=DEV).int().view(T, k)
    weight = torch.softmax(torch.randn((T, k), generator=g, device=DEV), -1)
    return dict(op=op, z=z, slot=slot, weight=weight, y=torch.empty((T, case["N"]), dtype=dt, device=DEV))


# ---- one pass ---------------------------------------------------------------------------------------------

def _run_own(s):
    from paper_1706_09453_b200 import binding as B
    op = s["op"]
    if "fmt" in s:
        fmt = B.F4_E8M0_32 if s["fmt"] == "mx" else B.F4_E4M3_16
    if op == "quantize":
        B.bnn_f4_quantize(s["x"], s["codes"], s["scales"], fmt, source=s["source"], offsets=s["offsets"])
        return B.bnn_f4_dequantize(s["codes"], s["scales"], s["values"], fmt, offsets=s["offsets"])
    if op == "gemm":
        return B.bnn_f4_gemm(s["a"], s["a_scales"], s["w"], s["w_scales"], s["K"], s["y"], fmt, exponent=s["exponent"], shift=s["bias"])
    if op == "grouped":
        return B.bnn_f4_gemm_grouped(s["a"], s["a_scales"], s["offsets"], s["w"], s["w_scales"], s["K"], s["y"], fmt, exponent=s["exponent"])
    if op == "route":
        if s["workspace"] is None:   # kept, as a user's program keeps it
            s["workspace"] = torch.empty((B.bnn_route_workspace_bytes(*s["logits"].shape),), dtype=torch.uint8, device=DEV)
        B.bnn_route_experts(s["logits"], s["index"], s["weight"], s["offsets"], s["slot"], s["source"], s["workspace"],
                            B.ROUTE_SOFTMAX_CHOSEN if s["chosen"] else B.ROUTE_SOFTMAX)
        return {n: s[n] for n in ("index", "weight", "offsets", "slot", "source")}
    return B.bnn_combine_experts(s["z"], s["slot"], s["weight"], s["y"])


def run(s):
    if own:
        return _run_own(s)
    op = s["op"]
    if op == "quantize":
        x = s["x"] if s["source"] is None else s["x"][s["source"].long()]
        codes, scales = _stored(x, s["fmt"], 0, s["offsets"], s["groups"])
        return _values(codes, scales, s["K"], s["fmt"], s["offsets"], s["groups"]).to(torch.bfloat16)
    if op == "gemm":
        a = _values(s["a"], s["a_scales"], s["K"], s["fmt"])
        w = _values(s["w"], s["w_scales"], s["K"], s["fmt"])
        y = (a @ w.t()) * 2.0 ** s["exponent"]
        return (y if s["bias"] is None else y + s["bias"]).to(s["y"].dtype)
    if op == "grouped":
        rows, off = s["a"].shape[0], s["offsets"].long()
        a = _values(s["a"], s["a_scales"], s["K"], s["fmt"], s["offsets"], s["groups"])
        w = _values(s["w"].flatten(0, 1), s["w_scales"], s["K"], s["fmt"], s["w_offsets"], s["groups"]).view(s["groups"], s["N"], s["K"])
        # every group padded to the longest
        at = (off[:-1, None] + torch.arange(s["most"], device=DEV)).clamp(max=rows - 1)
        y = torch.bmm(a[at], w.transpose(1, 2))
        r = torch.arange(rows, device=DEV)
        g = torch.searchsorted(off, r, right=True) - 1
        return (y[g, r - off[g]] * 2.0 ** s["exponent"]).to(s["y"].dtype)
    if op == "route":
        x, k = s["logits"].float(), s["k"]
        T, E = x.shape
        top, index = torch.sort(x, dim=-1, descending=True, stable=True)
        first, top, index = top[:, :1], top[:, :k], index[:, :k]
        real = top > -math.inf
        first = torch.where(first > -math.inf, first, 0.0)
        part = torch.exp(top - first)
        total = part.sum(-1, keepdim=True) if s["chosen"] else torch.exp(x - first).sum(-1, keepdim=True)
        weight = torch.where(real, part / total, 0.0)
        expert = torch.where(real, index, E).flatten()
        order = torch.argsort(expert, stable=True)
        place = torch.empty_like(order)
        place[order] = torch.arange(T * k, device=DEV)
        count = (expert[:, None] == torch.arange(E, device=DEV)).sum(0)
        offsets = torch.nn.functional.pad(count.cumsum(0), (1, 0)).int()
        slot = torch.where(real, place.view(T, k), -1).int()
        source = torch.where(torch.arange(T * k, device=DEV) < offsets[-1], order // k, -1).int()
        return {"index": torch.where(real, index, -1).int(), "weight": weight, "offsets": offsets, "slot": slot, "source": source}
    z = s["z"].float()[s["slot"].long()]
    return (z * s["weight"].unsqueeze(-1)).sum(1).to(s["y"].dtype)


# ---- what a pass cannot do without ------------------------------------------------------------------------

SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def work(case):
    op, size = case["op"], SIZE[case["dtype"]]
    if op == "quantize":   # activations (gathered rows are read again from a cache), the values' 16 bits
        n = case["rows"] * case["K"]
        return {"bytes": float((min(case["tokens"], case["rows"]) if case["experts"] else case["rows"]) * case["K"] * size + 2 * n), "flops": 2.0 * n}
    if op in ("gemm", "grouped"):
        rows, K, N = case.get("M") or case["rows"], case["K"], case["N"]
        live = min(case.get("experts", 1), rows)     # experts that can have a row
        return {"bytes": (rows + live * N) * K * (0.5 + 1 / BLOCK[case["fmt"]]) + float(rows * N * size), "flops": 2.0 * rows * K * N}
    if op == "route":
        return {"bytes": float(case["T"] * case["E"] * size + 16 * case["T"] * case["k"]), "flops": 4.0 * case["T"] * case["E"]}
    T, k, N = case["T"], case["k"], case["N"]
    return {"bytes": float((T * k + T) * N * size + 8 * T * k), "flops": 2.0 * T * k * N}


# ---- the definition in 64 bits ----------------------------------------------------------------------------

def _number(code):
    """e2m1 code -> double, from its fields."""
    c = code.long()
    e, m = ((c >> 1) & 3).double(), (c & 1).double()
    v = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * torch.exp2(e - 1))
    return torch.where((c & 8) != 0, -v, v)


def _e4m3(byte):
    b = byte.long() & 127
    e, m = (b >> 3).double(), (b & 7).double()
    return torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.exp2(e - 7))


def _read(codes, scales, K, fmt, first=0, base=0):
    """Doubles [rows][K] of rows whose scales begin at row 0 of tile ``base``; codes from row ``first`` on."""
    rows = codes.shape[0] - first
    k, r = torch.arange(K, device=DEV), torch.arange(rows, device=DEV)[:, None]
    nib = (codes[first:][:, k // 2].int() >> (4 * (k % 2)).int()) & 15
    block = k // BLOCK[fmt]
    at = ((base + r // 128) * _scale_tiles(fmt, K) + block // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + block % 4
    byte = scales[at]
    return _number(nib) * (((byte.long() - 127 + 1023) << 52).view(torch.float64) if fmt == "mx" else _e4m3(byte))


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "quantize":
        x = s["x"].double()
        if s["source"] is not None:
            x = x[s["source"].long()]
        rows, K = x.shape
        n = BLOCK[s["fmt"]]
        wide = (K + n - 1) // n * n
        b = torch.cat((x, torch.zeros((rows, wide - K), dtype=torch.float64, device=DEV)), 1).view(rows, wide // n, n)
        most = b.abs().max(-1, keepdim=True).values
        if s["fmt"] == "mx":
            e = (most.clamp(min=2.0 ** -125).view(torch.int64) >> 52) - 1023     # floor(log2(most)), from the double's exponent
            scale = ((e - 2 + 1023) << 52).view(torch.float64)
        else:
            # the nearest of all e4m3 numbers, the even code of two that are equally near
            grid = _e4m3(torch.arange(127, device=DEV))
            want = (most / 6).clamp(max=448.0)
            hi = torch.searchsorted(grid, want.contiguous()).clamp(1, 126)
            lo = hi - 1
            up, down = grid[hi] - want, want - grid[lo]
            scale = grid[torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)]
        q = torch.where(scale > 0, b.abs() / torch.where(scale > 0, scale, 1.0), 0.0).clamp(max=6.0)
        step = torch.where(q < 2, 0.5, torch.where(q < 4, 1.0, 2.0))
        return (torch.round(q / step) * step * torch.sign(b) * scale).reshape(rows, wide)[:, :K]
    if op == "gemm":
        y = _read(s["a"], s["a_scales"], s["K"], s["fmt"]) @ _read(s["w"], s["w_scales"], s["K"], s["fmt"]).t()
        y = y * 2.0 ** s["exponent"]
        return y if s["bias"] is None else y + s["bias"].double()
    if op == "grouped":
        y = torch.zeros((s["a"].shape[0], s["N"]), dtype=torch.float64, device=DEV)
        off = s["offsets"].tolist()
        for g in range(s["groups"]):
            lo, hi = off[g], off[g + 1]
            if hi > lo:
                a = _read(s["a"][:hi], s["a_scales"], s["K"], s["fmt"], lo, lo // 128 + g)
                w = _read(s["w"][g], s["w_scales"], s["K"], s["fmt"], 0, g * s["N"] // 128 + g)
                y[lo:hi] = (a @ w.t()) * 2.0 ** s["exponent"]
        return y
    if op == "route":
        x, k = s["logits"].double(), s["k"]
        T, E = x.shape
        # by rank: how many experts come before this one
        e = torch.arange(E, device=DEV)
        lead = torch.stack([((r[None, :] > r[:, None]) | ((r[None, :] == r[:, None]) & (e[None, :] < e[:, None]))).sum(-1)
                            for r in x]) if T * E * E < 1 << 22 else None
        if lead is None:
            index = torch.argsort(-x, dim=-1, stable=True)[:, :k]
        else:
            index = torch.argsort(lead, dim=-1)[:, :k]
        live = torch.isfinite(x)
        p = torch.where(live, torch.exp(x - torch.where(live, x, -math.inf).max(-1, keepdim=True).values.clamp(min=-1e9)), 0.0)
        w = p.gather(1, index)
        total = (w if s["chosen"] else p).sum(-1, keepdim=True)
        return {"index": None, "weight": torch.where(total > 0, w / torch.where(total > 0, total, 1.0), 0.0), "offsets": None, "slot": None, "source": None}
    y = torch.zeros(s["y"].shape, dtype=torch.float64, device=DEV)
    for j in range(s["slot"].shape[1]):
        y += s["weight"][:, j:j + 1].double() * s["z"][s["slot"][:, j].long()].double()
    return y
