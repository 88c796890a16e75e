"""The operators of a KV cache held in 4 bits, as the speed of this library is
measured on them: quantising the entries of new tokens as they are written
("write"), reading entries back in 16 bits ("read"), and attention over the
cache as it is held ("attend").

An entry's key or value is D codes of 4 bits (floats of 1 sign, 2 exponent and 1
mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) and one scale of 8 bits (5 exponent and
3 mantissa bits, the upper bits of a half-precision number without its sign) per
16 elements.

A case is a dict of plain values; "kind" names the operator.  With `own` false,
run() computes it from elementary torch operations in 32 bits; with `own` true
it makes the calls that a user makes.  Inputs are drawn on the GPU from the
seed.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
MAX_SCALE = 10240.0           # 6 times it is within half precision


def listed():
    return [
        # the smallest call: the one new token of one sequence
        dict(name="write_one", kind="write", B=1, T=1, Hkv=4, D=128, C=512, ragged=False, dtype="bf16", heads_first=True),
        # a decode step of a batch of drafting sequences, 0 to 5 tokens each, behind what their caches hold
        dict(name="write_drafts", kind="write", B=128, T=5, Hkv=8, D=64, C=1024, ragged=True, dtype="fp16",
             heads_first=False),
        # the prompts of a batch, of different lengths, 80-wide heads
        dict(name="write_prompts", kind="write", B=7, T=3001, Hkv=8, D=80, C=4096, ragged=True, dtype="bf16",
             heads_first=False),
        # the largest: long documents
        dict(name="write_documents", kind="write", B=4, T=32768, Hkv=8, D=128, C=32768, ragged=False, dtype="bf16",
             heads_first=True),
        # one short conversation is taken up again
        dict(name="read_one", kind="read", B=1, T=60, Hkv=4, D=128, C=512, ragged=False, dtype="bf16", heads_first=True),
        # caches of different lengths go back to 16 bits
        dict(name="read_batch", kind="read", B=48, T=2047, Hkv=8, D=128, C=2048, ragged=True, dtype="fp16",
             heads_first=False),
        # the smallest call: one token of one sequence
        dict(name="attend_one", kind="attend", B=1, T=1, Hq=12, Hkv=4, D=128, lo=60, hi=60, C=512, dtype="bf16",
             join=False, heads_first=True),
        # an ordinary batch of chats, behind a shared system prompt in 16 bits whose attention is joined
        dict(name="attend_chats", kind="attend", B=64, T=1, Hq=12, Hkv=4, D=128, lo=1, hi=4096, C=4096, dtype="bf16",
             join=True, heads_first=False),
        # four drafts a sequence, 64-wide heads, half precision, odd lengths
        dict(name="attend_drafts", kind="attend", B=32, T=5, Hq=24, Hkv=8, D=64, lo=100, hi=8001, C=8192, dtype="fp16",
             join=False, heads_first=True),
        # one question about one long document
        dict(name="attend_document", kind="attend", B=1, T=1, Hq=12, Hkv=4, D=128, lo=262144, hi=262144, C=262144,
             dtype="bf16", join=False, heads_first=True),
        # many drafts over heads that many queries share
        dict(name="attend_rows", kind="attend", B=16, T=8, Hq=64, Hkv=8, D=128, lo=1000, hi=6000, C=6000, dtype="bf16",
             join=False, heads_first=True),
        # the largest: a full batch of long contexts
        dict(name="attend_long", kind="attend", B=64, T=1, Hq=32, Hkv=8, D=128, lo=4096, hi=16384, C=16384, dtype="bf16",
             join=False, heads_first=True),
    ]


def _seconds(case):
    """A case's floor on this card, to compare costs."""
    w = work(case)
    return max(w["bytes"] / 6.7e12, w["flops"] / 1.9e15)


def _log(rng, lo, hi):
    """An integer from lo to hi, even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _seconds(c))
    while True:
        kind = rng.choice(["write", "read", "attend", "attend"])
        hkv, D = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128, 64, 128, 32, 80, 96, 112])
        more = dict(Hkv=hkv, D=D, dtype=rng.choice(["bf16", "fp16"]), heads_first=rng.random() < 0.6)
        if kind == "attend":
            T, hi = rng.choice([1, 1, 1, 2, 3, 4, 5, 6, 8]), _log(rng, 1, 200000)
            lo = rng.choice([0, 1, hi, max(1, hi // 3)])
            c = dict(kind=kind, B=_log(rng, 1, 160), T=T, Hq=hkv * rng.choice([1, 2, 3, 4, 5, 8]), lo=lo, hi=hi,
                     C=hi + rng.choice([0, 0, 1, 7, 100]), join=rng.random() < 0.4, **more)
        else:
            T = rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, 32768)])
            c = dict(kind=kind, B=_log(rng, 1, 200), T=T, C=T + rng.choice([0, 1, 13, 500]), ragged=rng.random() < 0.5, **more)
        if c["B"] * c["C"] * hkv * D <= 1 << 29 and _seconds(c) <= most[kind]:
            return c


def _rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _held(c, width, fill=None):
    """Bytes [B][C][Hkv][width], stored with the heads before the entries where heads_first says so."""
    shape = (c["B"], c["Hkv"], c["C"], width) if c["heads_first"] else (c["B"], c["C"], c["Hkv"], width)
    x = torch.zeros(shape, dtype=torch.uint8, device="cuda")
    return x.transpose(1, 2) if c["heads_first"] else x


def _cache(c):
    return _held(c, c["D"] // 2), _held(c, c["D"] // 16)


def _activations(g, shape, dtype):
    """What projections give: heads of different size, and some channels well above the others."""
    heads = 0.5 + torch.rand(shape[-2], 1, generator=g, device="cuda") * 1.5
    loud = 1 + 7 * (torch.rand(shape[-2], shape[-1], generator=g, device="cuda") < 0.03)
    x = torch.empty(shape, dtype=dtype, device="cuda")
    rows = x.view(-1, *shape[-2:])
    for part in rows.split(max(1, (1 << 26) // (shape[-2] * shape[-1]))):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * heads * loud)
    return x


def _quantise(x):
    """Codes (two to a byte, the first in the lower half), scale bytes and the values they stand for, of x [..., D]."""
    x = x.float().unflatten(-1, (x.shape[-1] // 16, 16))
    top = x.abs().amax(-1, keepdim=True)
    fine = torch.isfinite(x).all(-1, keepdim=True)
    want = torch.where(fine, top, 0.0) / 6
    step = torch.exp2((torch.frexp(want).exponent - 1).clamp(min=-14).float() - 3)
    s = (torch.round(want / step) * step).clamp(max=MAX_SCALE)
    byte = (s.half().view(torch.int16) >> 7).to(torch.uint8)
    y = x.abs()
    # ties go to the even code
    code = (y > 0.25 * s).to(torch.uint8)
    code += y >= 0.75 * s
    code += y > 1.25 * s
    code += y >= 1.75 * s
    code += y > 2.5 * s
    code += y >= 3.5 * s
    code += y > 5 * s
    some = fine & (s > 0)
    size = torch.where(code < 4, code * 0.5, torch.where(code < 6, code - 2.0, code * 2.0 - 8))
    value = torch.where(some, torch.copysign(size * s, x), torch.where(fine, 0.0, math.nan))
    code = torch.where(some, code + 8 * torch.signbit(x), 0).to(torch.uint8)
    byte = torch.where(fine, byte, 255).squeeze(-1)
    code = code.flatten(-2)
    return code[..., 0::2] + code[..., 1::2] * 16, byte, value.flatten(-2)


def _values(codes, scales):
    """What codes [..., D / 2] and scales [..., D / 16] stand for, in 32 bits."""
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    size = (code & 7).float()
    size = torch.where(size < 4, size * 0.5, torch.where(size < 6, size - 2.0, size * 2.0 - 8))
    s = (scales.to(torch.int16) << 7).view(torch.half).float()
    return (torch.where(code > 7, -size, size).unflatten(-1, (scales.shape[-1], 16)) * s.unsqueeze(-1)).flatten(-2)


def _fill(g, c, held):
    """Entries of a cache, made and quantised a piece at a time."""
    codes, scales = held
    per = max(1, (1 << 25) // (c["Hkv"] * c["D"]))
    for b in range(c["B"]):
        for i in range(0, c["C"], per):
            n = min(per, c["C"] - i)
            codes[b, i:i + n], scales[b, i:i + n], _ = _quantise(_activations(g, (n, c["Hkv"], c["D"]), TYPES[c["dtype"]]))


def prepare(case, seed):
    c, g = case, _rng(seed)
    B, T, Hkv, D, C = (c[k] for k in ("B", "T", "Hkv", "D", "C"))
    t = TYPES[c["dtype"]]
    s = {"case": c, "k4": _cache(c), "v4": _cache(c), "n": None}
    if c["kind"] == "attend":
        Hq = c["Hq"]
        _fill(g, c, s["k4"])
        _fill(g, c, s["v4"])
        s["lens"] = torch.randint(c["lo"], c["hi"] + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        s["q"] = torch.randn(B, T, Hq, D, generator=g, device="cuda").to(t)
        s["out"], s["lse"] = torch.empty(B, T, Hq, D, dtype=t, device="cuda"), torch.empty(B, T, Hq, device="cuda")
        # what the attention over the shared prompt left
        s["out_a"] = (0.3 * torch.randn(B, T, Hq, D, generator=g, device="cuda")).to(t)
        s["lse_a"] = 6 + torch.randn(B, T, Hq, generator=g, device="cuda")
    else:
        if c["ragged"]:
            s["n"] = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        s["at"] = torch.randint(0, C - T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        if c["kind"] == "write":
            s["k"], s["v"] = _activations(g, (B, T, Hkv, D), t), _activations(g, (B, T, Hkv, D), t)
        else:
            _fill(g, c, s["k4"])
            _fill(g, c, s["v4"])
        s["k_out"], s["v_out"] = (torch.zeros(B, T, Hkv, D, dtype=t, device="cuda") for _ in range(2))
    if own:
        from paper_2606_03026_gb300 import spikeproj as sp
        s["cache"] = sp.Cache4(Hq=c.get("Hq", Hkv), Hkv=Hkv, D=D, capacity=C, max_T=T if c["kind"] == "attend" else 1,
                               dtype=c["dtype"])
    return s


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"write": _own_write, "read": _own_read, "attend": _own_attend}[kind](state)
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[kind](state)


def _written(s):
    return {"k": s["k_out"], "v": s["v_out"], "k4": s["k4"], "v4": s["v4"]}


def _own_write(s):
    s["cache"].write(s["k"], s["v"], s["k4"], s["v4"], at=s["at"], n=s["n"], k_out=s["k_out"], v_out=s["v_out"])
    return _written(s)


def _own_read(s):
    s["cache"].read(s["k4"], s["v4"], s["k_out"], s["v_out"], at=s["at"], n=s["n"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_attend(s):
    join = s["case"]["join"]
    s["cache"].attend(s["q"], s["k4"], s["v4"], s["lens"], s["out"], lse=s["lse"],
                      other_out=s["out_a"] if join else None, other_lse=s["lse_a"] if join else None)
    return {"out": s["out"], "lse": s["lse"]}


def _there(s):
    """Sequences and tokens of the entries that a write or read is of, and their slots."""
    B, T = s["case"]["B"], s["case"]["T"]
    at = s["at"].long().unsqueeze(1) + torch.arange(T, device="cuda")
    if s["n"] is None:
        b, t = torch.arange(B, device="cuda").repeat_interleave(T), torch.arange(T, device="cuda").repeat(B)
    else:
        b, t = torch.nonzero(torch.arange(T, device="cuda") < s["n"].unsqueeze(1), as_tuple=True)
    return b, t, at[b, t]


def _plain_write(s):
    b, t, slot = _there(s)
    for x in "kv":
        codes, scales, values = _quantise(s[x][b, t])
        s[x + "4"][0][b, slot], s[x + "4"][1][b, slot] = codes, scales
        s[x + "_out"][b, t] = values.to(s[x].dtype)
    return _written(s)


def _plain_read(s):
    b, t, slot = _there(s)
    for x in "kv":
        codes, scales = s[x + "4"]
        s[x + "_out"][b, t] = _values(codes[b, slot], scales[b, slot]).to(s[x + "_out"].dtype)
    return {"k": s["k_out"], "v": s["v_out"]}


def _plain_attend(s):
    c = s["case"]
    B, T, Hq, Hkv, D, C = (c[k] for k in ("B", "T", "Hq", "Hkv", "D", "C"))
    G = Hq // Hkv
    last = s["lens"].view(-1, 1) - (T - 1 - torch.arange(T, device="cuda")).view(1, -1)
    seen = (torch.arange(C, device="cuda").view(1, 1, -1) < last.unsqueeze(2)).view(B, 1, T, 1, C)
    q = s["q"].float().view(B, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, D) * D ** -0.5
    z = (q @ _values(*s["k4"]).permute(0, 2, 3, 1)).view(B, Hkv, T, G, C).masked_fill(~seen, -math.inf)
    m = z.amax(4)
    if c["join"]:
        la = s["lse_a"].view(B, T, Hkv, G).permute(0, 2, 1, 3)
        m = torch.maximum(m, la)
    m = torch.where(m == -math.inf, 0.0, m)
    a = torch.exp(z - m.unsqueeze(4))
    total = a.sum(4)
    o = (a.view(B, Hkv, T * G, C) @ _values(*s["v4"]).permute(0, 2, 1, 3)).view(B, Hkv, T, G, D)
    if c["join"]:
        w = torch.exp(la - m)
        total = total + w
        o = o + w.unsqueeze(4) * s["out_a"].float().view(B, T, Hkv, G, D).permute(0, 2, 1, 3, 4)
    o = torch.where(total.unsqueeze(4) > 0, o / total.unsqueeze(4), 0.0)
    o = o.permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D)
    lse = (m + torch.log(total)).permute(0, 2, 1, 3).reshape(B, T, Hq)
    return {"out": o.to(s["q"].dtype), "lse": lse}


def work(case):
    c = case
    held = c["D"] / 2 + c["D"] / 16               # bytes of a row of 4 bits
    if c["kind"] == "attend":
        mean = (c["lo"] + c["hi"]) / 2
        rows = c["B"] * c["T"] * c["Hq"]
        b = c["B"] * mean * c["Hkv"] * 2 * held + rows * (2 * c["D"] * 2 + 4)
        if c["join"]:
            b += rows * (2 * c["D"] + 4)
        return {"bytes": b, "flops": 4.0 * c["D"] * rows * mean}
    rows = 2 * c["B"] * c["T"] * c["Hkv"] * (0.5 if c["ragged"] and c["T"] > 1 else 1.0)
    return {"bytes": rows * (held + (4 if c["kind"] == "write" else 2) * c["D"]), "flops": 0.0}


def exact(case, seed):
    s = prepare(case, seed)
    return {"write": _exact_write, "read": _exact_read, "attend": _exact_attend}[case["kind"]](case, s)


CODE_VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def _scale_values():
    """All scales from 0 to the largest in order, in 64 bits: number i has exponent i // 8 and fraction i % 8."""
    all_of = [i / 8 * 2.0 ** -14 if i < 8 else (1 + i % 8 / 8) * 2.0 ** (i // 8 - 15) for i in range(227)]
    return torch.tensor(all_of, dtype=torch.float64, device="cuda")


def _nearest(x, table):
    """The index of the value nearest to each x >= 0 in a rising table, the even one of two as near."""
    i = torch.searchsorted(table, x).clamp(1, len(table) - 1)
    below, above = x - table[i - 1], table[i] - x
    return torch.where((below < above) | ((below == above) & (i % 2 == 1)), i - 1, i)


def _exact_row(x):
    """Code bytes, scale bytes, values of rows [..., D]."""
    x = x.double().unflatten(-1, (x.shape[-1] // 16, 16))
    scales, codes = _scale_values(), torch.tensor(CODE_VALUES[:8], dtype=torch.float64, device="cuda")
    top = x.abs().max(-1).values
    byte = _nearest(top / 6, scales)
    s = scales[byte].unsqueeze(-1)
    code = _nearest(torch.where(s > 0, x.abs() / s, 0.0), codes)
    value = codes[code] * s * torch.where(torch.signbit(x), -1.0, 1.0)
    code = torch.where((s > 0) & torch.signbit(x), code + 8, code)
    code = code.flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), byte.to(torch.uint8), value.flatten(-2)


def _exact_value(codes, scales):
    bits = codes.long()
    table = torch.tensor(CODE_VALUES, dtype=torch.float64, device="cuda")
    value = torch.stack([table[bits % 16], table[bits // 16]], -1).flatten(-2)
    return value * _scale_values()[scales.long()].repeat_interleave(16, -1)


def _exact_write(c, s):
    """Sequence by sequence, in 64 bits."""
    if c["B"] * c["T"] * c["Hkv"] * c["D"] > 1 << 28:
        return None
    out = {x: s[x + "_out"].double() for x in "kv"}
    for b, at in enumerate(s["at"].tolist()):
        n = c["T"] if s["n"] is None else int(s["n"][b])
        for x in "kv":
            codes, scales, out[x][b, :n] = _exact_row(s[x][b, :n])
            s[x + "4"][0][b, at:at + n], s[x + "4"][1][b, at:at + n] = codes, scales
    return {**out, "k4": s["k4"], "v4": s["v4"]}


def _exact_read(c, s):
    if c["B"] * c["T"] * c["Hkv"] * c["D"] > 1 << 28:
        return None
    out = {x: s[x + "_out"].double() for x in "kv"}
    for b, at in enumerate(s["at"].tolist()):
        n = c["T"] if s["n"] is None else int(s["n"][b])
        for x in "kv":
            out[x][b, :n] = _exact_value(s[x + "4"][0][b, at:at + n], s[x + "4"][1][b, at:at + n])
    return out


def _exact_attend(c, s):
    """Row by row of the definition, sequence by sequence, in 64 bits."""
    B, T, Hq, Hkv, D = (c[k] for k in ("B", "T", "Hq", "Hkv", "D"))
    if 4.0 * D * B * T * Hq * c["hi"] > 3e11:
        return None
    G = Hq // Hkv
    out = torch.zeros(B, T, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.full((B, T, Hq), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lens"].tolist()):
        keys = _exact_value(s["k4"][0][b, :n], s["k4"][1][b, :n])
        vals = _exact_value(s["v4"][0][b, :n], s["v4"][1][b, :n])
        for t in range(T):
            far = max(0, n - (T - 1 - t))
            if far == 0:
                continue
            for h in range(Hkv):
                rows = slice(h * G, (h + 1) * G)
                z = s["q"][b, t, rows].double() @ keys[:far, h].T / math.sqrt(D)
                lse[b, t, rows] = torch.logsumexp(z, 1)
                out[b, t, rows] = torch.softmax(z, 1) @ vals[:far, h]
    if c["join"]:
        la, oa = s["lse_a"].double(), s["out_a"].double()
        both = torch.logaddexp(lse, la)
        out = out * torch.exp(lse - both).unsqueeze(3) + oa * torch.exp(la - both).unsqueeze(3)
        lse = both
    return {"out": out, "lse": lse}
