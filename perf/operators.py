"""The operators of a drafted decode step over a shared prompt, as the speed of
this library is measured on them: attention of a batch whose sequences share a
long prefix and keep caches of their own ("attend"), eviction from those caches
by accumulated attention weight ("evict"), and verification of drafted tokens
against the target's probabilities ("verify").

A case is a dict of plain values; "kind" names the operator.  With `own` false,
run() computes it from elementary torch operations in 32 bits; with `own` true
it makes the calls that a user makes.  Inputs are drawn on the GPU from the
seed.  Widths follow the paper's decoder (residual 1536, vocabulary 57,344).
"""
import math

import torch

own = False

VOCAB = 57344
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
KEEP_RATE = 0.75              # a draft's chance to be kept, about what the inputs of "verify" give


def listed():
    return [
        # the smallest call: one sequence, one token, a short system prompt
        dict(name="attend_one", kind="attend", B=1, T=1, Hq=12, Hkv=4, D=128, P=512, lo=60, hi=60, C=64,
             dtype="bf16", weights=False, heads_first=False),
        # an ordinary batch of chats that share a system prompt of 2048 tokens
        dict(name="attend_chat", kind="attend", B=64, T=1, Hq=12, Hkv=4, D=128, P=2048, lo=1, hi=1024, C=1024,
             dtype="bf16", weights=True, heads_first=False),
        # four drafts a sequence after an odd-sized prefix, 64-wide heads, half precision
        dict(name="attend_draft", kind="attend", B=32, T=5, Hq=24, Hkv=8, D=64, P=8191, lo=100, hi=2000, C=2048,
             dtype="fp16", weights=True, heads_first=True),
        # questions about one long document
        dict(name="attend_document", kind="attend", B=16, T=1, Hq=12, Hkv=4, D=128, P=131072, lo=16, hi=500, C=512,
             dtype="bf16", weights=False, heads_first=False),
        # the largest: many drafting sequences over a shared prefix of few-shot examples
        dict(name="attend_many", kind="attend", B=128, T=5, Hq=16, Hkv=4, D=128, P=16384, lo=512, hi=2048, C=2048,
             dtype="bf16", weights=True, heads_first=False),
        # one sequence whose own cache is a few entries over its budget
        dict(name="evict_one", kind="evict", B=1, Hkv=4, D=128, C=1032, lo=1029, hi=1029, budget=1024, recent=64,
             dtype="bf16", shuffled=True),
        # the same after every step of a batch, 0 to 8 new entries a sequence
        dict(name="evict_step", kind="evict", B=64, Hkv=4, D=128, C=2056, lo=2048, hi=2056, budget=2048, recent=128,
             dtype="bf16", shuffled=True),
        # long prompts cut down to the budget once
        dict(name="evict_prompt", kind="evict", B=16, Hkv=8, D=64, C=16384, lo=3000, hi=16384, budget=4096, recent=256,
             dtype="fp16", shuffled=False),
        # one drafting sequence
        dict(name="verify_one", kind="verify", B=1, T=4, V=VOCAB, ragged=False),
        # a batch of drafting sequences
        dict(name="verify_batch", kind="verify", B=64, T=4, V=VOCAB, ragged=False),
        # many sequences, each with its own number of drafts, an odd vocabulary
        dict(name="verify_many", kind="verify", B=200, T=7, V=50001, ragged=True),
    ]


def _seconds(case):
    """A case's floor on this card, to compare costs."""
    w = work(case)
    return max(w["bytes"] / 6.8e12, w["flops"] / 1.9e15)


def _log(rng, lo, hi):
    """An integer from lo to hi, even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _seconds(c))
    while True:
        kind = rng.choice(["attend", "attend", "evict", "verify"])
        if kind == "attend":
            hkv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 8])
            hi = _log(rng, 1, 4096)
            c = dict(kind=kind, B=_log(rng, 1, 160), T=rng.choice([1, 1, 2, 3, 4, 5, 6, 8]), Hq=hkv * group, Hkv=hkv,
                     D=rng.choice([64, 64, 128, 128, 80, 96]), P=_log(rng, 1, 131072), lo=rng.choice([1, hi, max(1, hi // 3)]),
                     hi=hi, C=hi + rng.choice([0, 0, 1, 7, 100]), dtype=rng.choice(["bf16", "fp16"]),
                     weights=rng.random() < 0.5, heads_first=rng.random() < 0.3)
            c["lo"] = min(c["hi"], max(c["lo"], c["T"]))
            c["hi"] = max(c["lo"], c["hi"])
            if c["hi"] < c["T"] or c["B"] * c["C"] * c["Hkv"] * c["D"] > 1 << 28:
                continue
        elif kind == "evict":
            budget = _log(rng, 16, 8192)
            over = _log(rng, 1, 4 * budget)
            c = dict(kind=kind, B=_log(rng, 1, 128), Hkv=rng.choice([1, 2, 4, 8]), D=rng.choice([64, 128, 80]),
                     C=budget + over, lo=rng.choice([budget, budget + over, max(1, budget // 2)]), hi=budget + over,
                     budget=budget, recent=rng.randint(0, budget // 2), dtype=rng.choice(["bf16", "fp16"]),
                     shuffled=rng.random() < 0.5)
            if c["B"] * c["C"] * c["Hkv"] * c["D"] > 1 << 28:
                continue
        else:
            c = dict(kind=kind, B=_log(rng, 1, 256), T=rng.randint(1, 8), V=_log(rng, 1000, 160000), ragged=rng.random() < 0.5)
            if c["B"] * (c["T"] + 1) * c["V"] > 1 << 28:
                continue
        if _seconds(c) <= most[kind] and 3072 not in c.values():
            return c


def _rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, dtype):
    """N(0, 1) values made in pieces, so that no 32-bit copy of a large cache is held."""
    x = torch.empty(shape, dtype=dtype, device="cuda")
    for part in x.view(-1).split(1 << 26):
        part.copy_(torch.randn(part.numel(), generator=g, device="cuda"))
    return x


def _lens(g, c):
    return torch.randint(c["lo"], c["hi"] + 1, (c["B"],), generator=g, device="cuda", dtype=torch.int32)


def _cache(g, c):
    """A K or V cache [B][C][Hkv][D], stored with the heads before the entries where heads_first says so."""
    if c.get("heads_first"):
        return _normal(g, (c["B"], c["Hkv"], c["C"], c["D"]), TYPES[c["dtype"]]).transpose(1, 2)
    return _normal(g, (c["B"], c["C"], c["Hkv"], c["D"]), TYPES[c["dtype"]])


def prepare(case, seed):
    c, g = case, _rng(seed)
    s = {"case": c}
    if c["kind"] == "attend":
        B, T, Hq, Hkv, D, P, C = (c[k] for k in ("B", "T", "Hq", "Hkv", "D", "P", "C"))
        t = TYPES[c["dtype"]]
        s["lens"] = _lens(g, c)
        s["q"] = (1.5 * torch.randn(B, T, Hq, D, generator=g, device="cuda")).to(t)
        s["pk"], s["pv"] = _normal(g, (P, Hkv, D), t), _normal(g, (P, Hkv, D), t)
        s["k"], s["v"] = _cache(g, c), _cache(g, c)
        s["out"] = torch.empty(B, T, Hq, D, dtype=t, device="cuda")
        s["lse"] = torch.empty(B, T, Hq, device="cuda")
        s["weights"] = torch.zeros(B, Hkv, C, device="cuda") if c["weights"] else None
        if own:
            from paper_2606_03026_gb300 import spikeproj as sp
            s["cache"] = sp.Cache(max_batch=B, Hq=Hq, Hkv=Hkv, D=D, capacity=C, max_T=T, dtype=c["dtype"],
                                  weights=c["weights"])
    elif c["kind"] == "evict":
        B, Hkv, D, C = (c[k] for k in ("B", "Hkv", "D", "C"))
        s["lens"] = _lens(g, c)
        s["k"], s["v"] = _cache(g, c), _cache(g, c)
        # accumulated attention: a few entries hold most of it, some none
        w = torch.exp(2.0 * torch.randn(B, Hkv, C, generator=g, device="cuda")) / 100
        s["weights"] = w * (torch.rand(B, Hkv, C, generator=g, device="cuda") > 0.02)
        # order of arrival: as stored, or mixed by earlier evictions
        pos = torch.arange(C, device="cuda", dtype=torch.int32).expand(B, Hkv, C).contiguous()
        if c["shuffled"]:
            at = torch.arange(C, device="cuda").expand(B, Hkv, C)
            mix = torch.rand(B, Hkv, C, generator=g, device="cuda")
            order = torch.argsort(torch.where(at < s["lens"].view(-1, 1, 1), mix, 2.0 + at), dim=2)
            pos = order.to(torch.int32)
        s["pos"] = pos
        s["now"] = s["lens"].clone()
        s["weights_out"] = torch.zeros(B, Hkv, C, device="cuda")
        s["pos_out"] = torch.zeros(B, Hkv, C, device="cuda", dtype=torch.int32)
        s["lens_out"] = torch.zeros(B, device="cuda", dtype=torch.int32)
        if own:
            from paper_2606_03026_gb300 import spikeproj as sp
            s["cache"] = sp.Cache(max_batch=B, Hq=Hkv, Hkv=Hkv, D=D, capacity=C, dtype=c["dtype"])
    else:
        B, T, V = c["B"], c["T"], c["V"]
        z = 2.5 * torch.randn(B, T + 1, V, generator=g, device="cuda")
        s["p"] = torch.softmax(z, 2)
        # the drafting model's logits: the target's with noise
        s["q"] = torch.softmax(z[:, :T] + 0.6 * torch.randn(B, T, V, generator=g, device="cuda"), 2)
        del z
        cdf = s["q"].cumsum(2)
        s["draft"] = torch.searchsorted(cdf, torch.rand(B, T, 1, generator=g, device="cuda") * cdf[:, :, -1:])
        s["draft"] = s["draft"].squeeze(2).clamp_(max=V - 1).to(torch.int32)
        s["n_draft"] = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32) if c["ragged"] else None
        s["u"] = torch.rand(B, T, generator=g, device="cuda")
        s["u_sample"] = torch.rand(B, generator=g, device="cuda")
        s["n_accept"] = torch.empty(B, device="cuda", dtype=torch.int32)
        s["tokens"] = torch.empty(B, T + 1, device="cuda", dtype=torch.int32)
    return s


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"attend": _own_attend, "evict": _own_evict, "verify": _own_verify}[kind](state)
    return {"attend": _plain_attend, "evict": _plain_evict, "verify": _plain_verify}[kind](state)


def _own_attend(s):
    s["cache"].attend(s["q"], s["k"], s["v"], s["lens"], s["out"], prefix_k=s["pk"], prefix_v=s["pv"],
                      weights=s["weights"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"], "weights": s["weights"]}


def _own_evict(s):
    c = s["case"]
    s["cache"].evict(s["k"], s["v"], s["weights"], s["pos"], s["lens"], s["now"], c["budget"], c["recent"],
                     s["weights_out"], s["pos_out"], s["lens_out"])
    return {x: s[x] for x in ("k", "v", "weights_out", "pos_out", "lens_out")}


def _own_verify(s):
    from paper_2606_03026_gb300 import spikeproj as sp
    sp.verify(s["p"], s["q"], s["draft"], s["u"], s["u_sample"], s["n_accept"], s["tokens"], n_draft=s["n_draft"])
    return {"n_accept": s["n_accept"], "tokens": s["tokens"]}


def _visible(c, lens):
    """[B, 1, T, 1, C]: whether own entry j is seen by query t."""
    last = lens.view(-1, 1) - (c["T"] - 1 - torch.arange(c["T"], device="cuda")).view(1, -1)
    return (torch.arange(c["C"], device="cuda").view(1, 1, -1) < last.unsqueeze(2)).view(c["B"], 1, c["T"], 1, c["C"])


def _plain_attend(s):
    c = s["case"]
    B, T, Hq, Hkv, D, P, C = (c[k] for k in ("B", "T", "Hq", "Hkv", "D", "P", "C"))
    G = Hq // Hkv
    q = s["q"].float().view(B, T, Hkv, G, D) * D ** -0.5
    seen = _visible(c, s["lens"])
    # the shared part, once for the rows of all sequences
    sp = q.permute(2, 0, 1, 3, 4).reshape(Hkv, B * T * G, D) @ s["pk"].float().permute(1, 2, 0)
    so = q.permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, D) @ s["k"].float().permute(0, 2, 3, 1)
    so = so.view(B, Hkv, T, G, C).masked_fill(~seen, -math.inf)
    m = torch.maximum(sp.amax(2).view(Hkv, B, T, G).permute(1, 0, 2, 3), so.amax(4))
    sp = torch.exp(sp.view(Hkv, B, T, G, P) - m.permute(1, 0, 2, 3).unsqueeze(4))
    so = torch.exp(so - m.unsqueeze(4))
    total = sp.sum(4).permute(1, 0, 2, 3) + so.sum(4)
    o = (sp.view(Hkv, B * T * G, P) @ s["pv"].float().permute(1, 0, 2)).view(Hkv, B, T, G, D).permute(1, 0, 2, 3, 4)
    v = s["v"].float().permute(0, 2, 1, 3) * (torch.arange(C, device="cuda") < s["lens"].view(-1, 1)).view(B, 1, C, 1)
    o = o + (so.view(B, Hkv, T * G, C) @ v).view(B, Hkv, T, G, D)
    o = (o / total.unsqueeze(4)).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D)
    if s["weights"] is not None:
        s["weights"] += (so / total.unsqueeze(4)).sum((2, 3))
    lse = (m + torch.log(total)).permute(0, 2, 1, 3).reshape(B, T, Hq)
    return {"out": o.to(s["q"].dtype), "lse": lse, "weights": s["weights"]}


def _plain_evict(s):
    c = s["case"]
    B, Hkv, D, C, budget = (c[k] for k in ("B", "Hkv", "D", "C", "budget"))
    n = s["lens"].view(B, 1, 1)
    at = torch.arange(C, device="cuda").expand(B, Hkv, C)
    # kept first: the newest, then by weight, then by slot; entries that are not there last
    group = torch.where(at >= n, 2, torch.where(s["pos"] >= s["now"].view(B, 1, 1) - c["recent"], 0, 1))
    by_weight = torch.sort(torch.where(group == 1, s["weights"], 0.0), dim=2, descending=True, stable=True).indices
    order = by_weight.gather(2, torch.sort(group.gather(2, by_weight), dim=2, stable=True).indices)
    rank = torch.empty_like(order).scatter_(2, order, at)
    kept = (rank < budget) & (at < n)
    # kept entries from behind the budget move into the slots that others leave
    hole, moved = ~kept & (at < torch.clamp(n, max=budget)), kept & (at >= budget)
    place = torch.where(moved, moved.cumsum(2) - 1, C)
    source = torch.zeros(B, Hkv, C + 1, device="cuda", dtype=torch.long).scatter_(2, place, at)
    source = torch.where(hole, source.gather(2, (hole.cumsum(2) - 1).clamp(min=0)), at)[:, :, :min(budget, C)]
    there = at[:, :, :source.shape[2]] < torch.clamp(n, max=budget)
    for x in ("k", "v"):
        rows = s[x].gather(1, source.permute(0, 2, 1).unsqueeze(3).expand(B, source.shape[2], Hkv, D))
        s[x][:, :source.shape[2]] = rows
    for x in ("weights", "pos"):
        out = s[x + "_out"][:, :, :source.shape[2]]
        out.copy_(torch.where(there, s[x].gather(2, source), out))
    s["lens_out"].copy_(torch.clamp(s["lens"], max=budget))
    return {x: s[x] for x in ("k", "v", "weights_out", "pos_out", "lens_out")}


def _plain_verify(s):
    B, T, V = (s["case"][k] for k in ("B", "T", "V"))
    b, t = torch.arange(B, device="cuda"), torch.arange(T, device="cuda")
    count = torch.full((B,), T, device="cuda") if s["n_draft"] is None else s["n_draft"].long()
    x = s["draft"].long().unsqueeze(2)
    px, qx = s["p"][:, :T].gather(2, x).squeeze(2), s["q"].gather(2, x).squeeze(2)
    ok = (s["u"] * qx < px) & (t < count.view(B, 1))
    n = ok.long().cumprod(1).sum(1)
    p = s["p"][b, n]
    r = p - torch.where((n < count).unsqueeze(1), s["q"][b, n.clamp(max=T - 1)], 0.0)

    def whole(r):
        return torch.round(torch.where(r > 0, r.clamp(max=1.0), 0.0) * 2.0 ** 36).long()

    w = whole(r)
    w = torch.where((w.sum(1) > 0).unsqueeze(1), w, whole(p))
    total = w.sum(1)
    u = torch.floor(s["u_sample"].clamp(0, 1 - 2.0 ** -24) * 2.0 ** 24).long()
    first = (w.cumsum(1) <= ((u * total) >> 24).unsqueeze(1)).sum(1)
    first = torch.where(total > 0, first, -1)
    at = torch.arange(T + 1, device="cuda").view(1, -1)
    drafts = torch.cat([s["draft"].long(), torch.full((B, 1), -1, device="cuda")], 1)
    tokens = torch.where(at < n.view(B, 1), drafts, torch.where(at == n.view(B, 1), first.view(B, 1), -1))
    return {"n_accept": n.to(torch.int32), "tokens": tokens.to(torch.int32)}


def work(case):
    c = case
    if c["kind"] == "attend":
        mean = (c["lo"] + c["hi"]) / 2
        keys = c["P"] + c["B"] * mean
        rows = c["B"] * c["T"] * c["Hq"]
        b = keys * c["Hkv"] * 2 * c["D"] * 2 + rows * (2 * c["D"] * 2 + 4)
        if c["weights"]:
            b += 8 * c["B"] * mean * c["Hkv"]
        return {"bytes": b, "flops": 4.0 * c["D"] * rows * (c["P"] + mean)}
    if c["kind"] == "evict":
        heads, budget = c["B"] * c["Hkv"], c["budget"]
        b, steps = 0.0, 16
        for i in range(steps):            # lengths are even between lo and hi
            n = c["lo"] + (c["hi"] - c["lo"]) * (i + 0.5) / steps
            left = min(n, budget)
            moved = 0.0
            if n > budget:                # survivors behind the budget: the newest, and their share of the rest
                recent = c["recent"] * ((n - budget) / n if c["shuffled"] else min(1.0, (n - budget) / max(1, c["recent"])))
                moved = recent + (n - budget - recent) * max(0.0, budget - c["recent"]) / (n - c["recent"])
            b += (8 * n + 8 * left + moved * 2 * 2 * c["D"] * 2) / steps
        return {"bytes": heads * b, "flops": 0.0}
    # the target's row of the one more token, and the draft's unless all drafts are kept
    kept = KEEP_RATE ** (c["T"] / 2 if c["ragged"] else c["T"])
    return {"bytes": c["B"] * (c["V"] * 4 * (2 - kept) + 20 * c["T"]), "flops": 0.0}


def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "evict": _exact_evict, "verify": _exact_verify}[case["kind"]](case, s)


def _exact_attend(c, s):
    """Row by row of the definition, sequence by sequence, in 64 bits."""
    B, T, Hq, Hkv, D, P, C = (c[k] for k in ("B", "T", "Hq", "Hkv", "D", "P", "C"))
    if 4.0 * D * B * T * Hq * (P + C) > 4e12:
        return None
    G = Hq // Hkv
    out = torch.empty(B, T, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.empty(B, T, Hq, dtype=torch.float64, device="cuda")
    wts = torch.zeros(B, Hkv, C, dtype=torch.float64, device="cuda") if c["weights"] else None
    pk, pv = s["pk"].double(), s["pv"].double()
    for b, n in enumerate(s["lens"].tolist()):
        keys = torch.cat([pk, s["k"][b, :n].double()])
        vals = torch.cat([pv, s["v"][b, :n].double()])
        for t in range(T):
            far = P + max(0, n - (T - 1 - t))
            for h in range(Hkv):
                z = s["q"][b, t, h * G:(h + 1) * G].double() @ keys[:far, h].T / math.sqrt(D)
                lse[b, t, h * G:(h + 1) * G] = torch.logsumexp(z, 1)
                a = torch.softmax(z, 1)
                out[b, t, h * G:(h + 1) * G] = a @ vals[:far, h]
                if wts is not None:
                    wts[b, h, :far - P] += a[:, P:].sum(0)
    return {"out": out, "lse": lse, "weights": wts}


def _exact_evict(c, s):
    """One (sequence, head) after another on the host; only values are moved, none computed."""
    B, Hkv, C, budget = (c[k] for k in ("B", "Hkv", "C", "budget"))
    if B * Hkv * C > 600_000:
        return None
    k, v = s["k"].float().cpu().double(), s["v"].float().cpu().double()
    w, pos = s["weights"].cpu().double(), s["pos"].cpu()
    w_out, pos_out = torch.zeros(B, Hkv, C, dtype=torch.float64), torch.zeros(B, Hkv, C, dtype=torch.int32)
    lens, now = s["lens"].tolist(), s["now"].tolist()
    for b in range(B):
        n = lens[b]
        for h in range(Hkv):
            ws, ps = w[b, h, :n].tolist(), pos[b, h, :n].tolist()
            best = sorted(range(n), key=lambda j: (ps[j] < now[b] - c["recent"], -ws[j] if ps[j] < now[b] - c["recent"] else 0, j))
            keep = set(best[:budget])
            late = sorted(j for j in keep if j >= budget)
            for j in range(min(n, budget)):
                i = j if j in keep else late.pop(0)
                if i != j:
                    k[b, j, h], v[b, j, h] = k[b, i, h], v[b, i, h]
                w_out[b, h, j], pos_out[b, h, j] = ws[i], ps[i]
    return {"k": k, "v": v, "weights_out": w_out, "pos_out": pos_out,
            "lens_out": torch.tensor([min(n, budget) for n in lens], dtype=torch.int32)}


def _exact_verify(c, s):
    """Draft after draft on the host; the outputs are whole numbers."""
    import numpy as np
    B, T, V = c["B"], c["T"], c["V"]
    if B * V > 5_000_000:
        return None
    count = [T] * B if s["n_draft"] is None else s["n_draft"].tolist()
    draft, u, us = s["draft"].tolist(), s["u"].cpu().numpy(), s["u_sample"].cpu().numpy()
    n_accept, tokens = [], []
    for b in range(B):
        p, q = s["p"][b].cpu().numpy(), s["q"][b].cpu().numpy()
        n = 0
        while n < count[b] and u[b, n] * q[n, draft[b][n]] < p[n, draft[b][n]]:
            n += 1
        r = p[n].astype(np.float64)
        if n < count[b]:
            r = (p[n] - q[n]).astype(np.float64)
        w = np.rint(np.clip(r, 0, 1) * 2.0 ** 36).astype(np.int64)
        if not w.sum():
            w = np.rint(np.clip(p[n].astype(np.float64), 0, 1) * 2.0 ** 36).astype(np.int64)
        bound = int(float(us[b]) * 2 ** 24) * int(w.sum()) // 2 ** 24
        n_accept.append(n)
        tokens.append(draft[b][:n] + [int(np.searchsorted(np.cumsum(w), bound, side="right"))] + [-1] * (T - n))
    return {"n_accept": torch.tensor(n_accept, dtype=torch.int32), "tokens": torch.tensor(tokens, dtype=torch.int32)}
