"""The row-wise choice operators as cases: what they are called with, their plain form, and their exact values.

Operators (paper_2609_27209_gb300.erc):
  sample   erc_sample_rows: one draw per row of scores after temperature, min-p, top-k and top-p
  route    erc_route, erc_route_backward: experts of a row from its scores, and the scores' gradient
  plan     erc_expert_plan: the chosen (row, choice) pairs in expert order
  combine  erc_expert_gather, erc_expert_combine, erc_expert_combine_backward: rows to expert order and back

Whole-number results are defined exactly.  An entry's weight is an integer, 2^t in 40 fractional bits, t the
scaled distance from the row's maximum, 2^t from a polynomial whose products and sums are rounded one by one,
and every sum of weights is a sum of integers, so no order of summation changes a choice.
"""
import math

import numpy as np
import torch

own = False

LOG2E = 1.4426950408889634
COEF = (1.0, 0.693147, 0.24022242, 0.055507336, 0.009671513, 0.0013264727)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one walker's next node on the 20,000-node graph: a single short call, where latency counts
        dict(name="sample_single", op="sample", rows=1, n=20000, type="f32", stride=20000, rule="kp", mask=0.0),
        # a serving batch over the 169,343-node graph, every row with settings of its own
        dict(name="sample_batch", op="sample", rows=64, n=169343, type="bf16", stride=169343, rule="mixed", mask=0.0),
        # many walkers over padded neighbour lists of odd length; some lists are empty
        dict(name="sample_walkers", op="sample", rows=16384, n=257, type="f32", stride=260, rule="plain", mask=0.6),
        # nucleus sampling over the 232,965-node graph: the kept sets run from a handful to thousands
        dict(name="sample_nucleus", op="sample", rows=256, n=232965, type="bf16", stride=232968, rule="p", mask=0.0),
        # the 2,449,029-node graph: few rows, each many times a block's on-chip memory
        dict(name="sample_long", op="sample", rows=8, n=2449029, type="f32", stride=2449029, rule="m", mask=0.1),
        # a few nodes routed between training steps or while answering: latency
        dict(name="route_few", op="route", way="forward", rows=7, n=64, k=4, type="f32", score="softmax", bias=False,
             groups=1, top=1, best=1, renorm=True),
        # grouped sigmoid routing with a balance bias over a large batch
        dict(name="route_groups", op="route", way="forward", rows=32768, n=256, k=8, type="bf16", score="sigmoid",
             bias=True, groups=8, top=4, best=2, renorm=True),
        # the gradient for every node of the 169,343-node graph, softmax scores
        dict(name="route_gradient", op="route", way="backward", rows=169343, n=64, k=2, type="f32", score="softmax",
             bias=False, groups=1, top=1, best=1, renorm=False),
        # the plan of one small step
        dict(name="plan_few", op="plan", rows=130, n=64, k=4, drop=0.0),
        # the plan of every node of the 169,343-node graph, a tenth of the choices empty
        dict(name="plan_nodes", op="plan", rows=169343, n=256, k=8, drop=0.1),
        # expert results summed back for the 20,000-node graph
        dict(name="combine_forward", op="combine", way="forward", rows=20000, n=64, k=4, width=512, type="bf16", drop=0.0),
        # the gradient of a large batch
        dict(name="combine_gradient", op="combine", way="backward", rows=32768, n=128, k=8, width=1024, type="bf16",
             drop=0.05),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sample", "sample", "route", "plan", "combine"])
    if op == "sample":
        n = _log(rng, 33, 2449029)
        rows = _log(rng, 1, max(1, min(16384, 50_000_000 // n)))
        pad = rng.choice([0, 0, 1, 7, 8])
        return dict(op=op, rows=rows, n=n, type=rng.choice(["f32", "bf16", "f16"]), stride=n + pad,
                    rule=rng.choice(["plain", "k", "p", "m", "kp", "mixed"]), mask=rng.choice([0.0, 0.1, 0.6]))
    if op == "route":
        groups = rng.choice([1, 1, 4, 8])
        n = groups * _log(rng, 8, 512 // groups)
        top = rng.randint(1, groups)
        k = min(rng.choice([1, 2, 4, 6, 8]), top * (n // groups))
        rows = _log(rng, 1, min(169343, 16_000_000 // n))
        return dict(op=op, way=rng.choice(["forward", "backward"]), rows=rows, n=n, k=k,
                    type=rng.choice(["f32", "bf16", "f16"]), score=rng.choice(["softmax", "sigmoid"]),
                    bias=rng.random() < 0.5, groups=groups, top=top, best=rng.choice([1, 2]),
                    renorm=rng.random() < 0.5)
    k = rng.choice([1, 2, 4, 6, 8])
    n = max(k, _log(rng, 8, 512))
    if op == "plan":
        return dict(op=op, rows=_log(rng, 1, 169343), n=n, k=k, drop=rng.choice([0.0, 0.1, 0.5]))
    width = _log(rng, 16, 2048)
    width = rng.choice([width, width // 8 * 8])
    return dict(op=op, way=rng.choice(["forward", "backward", "gather"]), rows=_log(rng, 1, min(65536, 200_000_000 // (k * width))),
                n=n, k=k, width=width, type=rng.choice(["f32", "bf16", "f16"]), drop=rng.choice([0.0, 0.05]))


# ---------------------------------------------------------------------------------------------- inputs


def _scores(g, rows, n, spread):
    """Rows of scores between undecided and confident: normal with a spread of the row's own, a few entries favoured."""
    x = torch.randn(rows, n, generator=g, device="cuda")
    lo, hi = spread
    x *= lo + (hi - lo) * torch.rand(rows, 1, generator=g, device="cuda")
    few = max(1, min(32, n // 16))
    at = torch.randint(0, n, (rows, few), generator=g, device="cuda")
    return x.scatter_add_(1, at, 8.0 * torch.rand(rows, few, generator=g, device="cuda"))


def _experts(g, rows, n, k, drop):
    """k different experts a row, some favoured; -1 where a choice is empty."""
    noise = torch.rand(rows, n, generator=g, device="cuda") + torch.linspace(0, 0.3, n, device="cuda")
    experts = noise.topk(k, 1).indices.to(torch.int32)
    return torch.where(torch.rand(rows, k, generator=g, device="cuda") < drop, -1, experts).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 17)
    rows, n, op = case["rows"], case["n"], case["op"]
    s = dict(case)
    if op == "sample":
        x = _scores(g, rows, n, (0.5, 3.0))
        if case["mask"]:
            # a row's list ends somewhere, at its very start in some rows
            ends = (torch.rand(rows, 1, generator=g, device="cuda") * (n + n * case["mask"]) - n * case["mask"] / 2).clamp(0, n)
            x.masked_fill_(torch.arange(n, device="cuda") >= ends, -math.inf)
        buffer = torch.zeros(rows, case["stride"], dtype=TYPES[case["type"]], device="cuda")
        buffer[:, :n] = x
        s["logits"] = buffer[:, :n]
        s["words"] = torch.randint(-(2**63), 2**63 - 1, (rows,), generator=g, device="cuda")
        rule = case["rule"]
        s["settings"] = dict(temperature=0.8, top_k=50 if "k" in rule else 0, top_p=0.95 if "p" in rule and rule != "plain" else 1.0,
                             min_p=0.05 if rule == "m" else 0.0)
        if rule == "mixed":
            pick = lambda v, t: torch.tensor(v, dtype=t, device="cuda")[  # noqa: E731
                torch.randint(0, len(v), (rows,), generator=g, device="cuda")]
            s["settings"] = dict(temperature=pick([0.0, 0.6, 0.8, 1.0, 1.0, 1.3], torch.float32),
                                 top_k=pick([0, 0, 1, 40, 200, 2000], torch.int32),
                                 top_p=pick([0.5, 0.9, 0.95, 1.0], torch.float32),
                                 min_p=pick([0.0, 0.0, 0.02, 0.1], torch.float32))
    elif op == "route":
        s["logits"] = _scores(g, rows, n, (0.5, 1.5)).to(TYPES[case["type"]])
        s["bias_values"] = 0.05 * torch.randn(n, generator=g, device="cuda") if case["bias"] else None
        if case["way"] == "backward":
            s["experts"], _ = _route_plain(s)
            s["grad"] = torch.randn(rows, case["k"], generator=g, device="cuda")
    else:
        s["experts"] = _experts(g, rows, n, case["k"], case["drop"])
        if op == "combine":
            slots = rows * case["k"]
            s["offsets"], _, s["slot"] = _plan_plain(s)
            kind = TYPES[case["type"]]
            s["x"] = torch.randn(rows, case["width"], generator=g, device="cuda").to(kind)
            if case["way"] != "gather":
                s["y"] = torch.randn(slots, case["width"], generator=g, device="cuda").to(kind)
                s["weights"] = torch.rand(rows, case["k"], generator=g, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------- plain forms


def _power(t):
    """2^t for t <= 0 as a polynomial p in [0.7, 1.42] and an exponent: every product and sum is rounded once."""
    e = torch.round(t)
    f = t - e
    c0, c1, c2, c3, c4, c5 = COEF
    p = f * c5 + c4
    p = p * f + c3
    p = p * f + c2
    p = p * f + c1
    return p * f + c0, e


def _fixed(t):
    """round(2^t 2^40) as an integer, 0 below 2^-41."""
    p, e = _power(t)
    down = (-e).clamp(0, 62)
    live = e >= -41
    m = torch.where(live, p, 0.0) * 16777216.0
    w = (((m.to(torch.int64) << 17) >> torch.where(live, down, 62.0).to(torch.int64)) + 1) >> 1
    return torch.where(live, w, 0)


def _scaled(p, e, least):
    """p 2^e, 0 for e < least."""
    two = ((e.clamp(-126, 0) + 127).to(torch.int32) << 23).view(torch.float32)
    return torch.where(e >= least, torch.where(e >= least, p, 0.0) * two, 0.0)


def _below(x, scale):
    """(l - max) scale, 0 at the maximum, whatever the scale is."""
    m = x.amax(1, keepdim=True)
    return torch.where(x == m, 0.0, (x - m) * scale)


def _high(x, w):
    """floor(x w / 2^64) of 64-bit words: schoolbook in 16-bit digits."""
    a = torch.stack([(x >> s) & 0xFFFF for s in (0, 16, 32, 48)])
    b = torch.stack([(w >> s) & 0xFFFF for s in (0, 16, 32, 48)])
    c = a[:, None] * b[None]
    carry = c[0, 0] >> 16
    carry = (c[0, 1] + c[1, 0] + carry) >> 16
    carry = (c[0, 2] + c[1, 1] + c[2, 0] + carry) >> 16
    carry = (c[0, 3] + c[1, 2] + c[2, 1] + c[3, 0] + carry)
    d3, carry = carry & 0xFFFF, carry >> 16
    d4 = c[1, 3] + c[2, 2] + c[3, 1] + carry
    d5 = c[2, 3] + c[3, 2] + (d4 >> 16)
    d6 = c[3, 3] + (d5 >> 16)
    return (d4 & 0xFFFF) + ((d5 & 0xFFFF) << 16) + (d6 << 32)


def _column(v, rows, kind):
    v = v if isinstance(v, torch.Tensor) else torch.full((rows,), v, device="cuda")
    return v.to(kind)[:, None]


def _sample_plain(s):
    x = s["logits"].float()
    rows, n = x.shape
    x = torch.where(torch.isnan(x), -math.inf, x)
    heat = _column(s["settings"]["temperature"], rows, torch.float32)
    top_k = _column(s["settings"]["top_k"], rows, torch.int64)
    top_p = _column(s["settings"]["top_p"], rows, torch.float32)
    min_p = _column(s["settings"]["min_p"], rows, torch.float32)
    greedy = ~(heat > 0)
    scale = torch.where(greedy, 1.0, LOG2E_32() / torch.where(greedy, 1.0, heat))
    top_k = torch.where(greedy, 1, torch.where(top_k > 0, top_k, n))
    w = _fixed(_below(x, scale))
    w = torch.where(x == -math.inf, 0, w)
    least = (min_p.clamp(0, 1) * 1099511627776.0).to(torch.int64).clamp(min=1)
    w = torch.where(w >= least, w, 0)
    # eligible entries first, best first, lowest index first among equals
    order = torch.sort(torch.where(w > 0, x, -math.inf), dim=1, descending=True, stable=True).indices
    ranked = torch.gather(w, 1, order)
    ranked = torch.where(torch.arange(n, device=x.device) < top_k, ranked, 0)
    total = ranked.sum(1, keepdim=True)
    before = ranked.cumsum(1) - ranked
    part = (top_p.clamp(0, 1) * 2147483648.0).to(torch.int64)
    target = ((total >> 31) * part + (((total & 0x7FFFFFFF) * part) >> 31)).clamp(min=1)
    ranked = torch.where((before < target) | (top_p >= 1), ranked, 0)
    w = torch.zeros_like(w).scatter_(1, order, ranked)
    total = w.sum(1)
    at = _high(s["words"], total)
    ids = (w.cumsum(1) <= at[:, None]).sum(1)
    some = total > 0
    ids = torch.where(some, ids, 0)
    mine = torch.gather(w, 1, ids[:, None])[:, 0]
    rest, whole = (total - mine).float(), total.float().clamp(min=1)
    logp = torch.where(mine * 2 > total, torch.log1p(-(rest / whole)), torch.log(mine.float() / whole))
    return dict(ids=torch.where(some, ids, -1).to(torch.int32), logp=torch.where(some, logp, -math.inf),
                kept=(w > 0).sum(1).to(torch.int32))


def LOG2E_32():
    return torch.tensor(LOG2E, dtype=torch.float32, device="cuda")


def _score(s):
    """Scores in [0, 1] in 32 bits, and which entries are masked."""
    x = s["logits"].float()
    masked = torch.isnan(x) | (x == -math.inf)
    x = torch.where(masked, -math.inf, x)
    if s["score"] == "sigmoid":
        p, e = _power(-(x.abs() * LOG2E_32()))
        e = _scaled(p, e, -126)
        v = torch.where(x >= 0, 1.0, e) / (1.0 + e)
    else:
        t = _below(x, LOG2E_32())
        p, e = _power(t)
        total = torch.where(masked, 0, _fixed(t)).sum(1, keepdim=True).clamp(min=1).float() * 2.0**-40
        v = _scaled(p, e, -41) * (1.0 / total)
    return torch.where(masked, 0.0, v), masked


def _route_plain(s):
    v, masked = _score(s)
    rows, n = v.shape
    c = v if s["bias_values"] is None else v + s["bias_values"]
    c = torch.where(masked | torch.isnan(c), -math.inf, c)
    if s["groups"] > 1:
        by = c.view(rows, s["groups"], -1)
        best = torch.sort(by, dim=2, descending=True).values[:, :, : s["best"]]
        score = torch.where(best == -math.inf, 0.0, best).sum(2)
        score = torch.where(best[:, :, 0] == -math.inf, -math.inf, score)
        ranked = torch.sort(score, dim=1, descending=True, stable=True).indices[:, : s["top"]]
        take = torch.zeros(rows, s["groups"], dtype=torch.bool, device=c.device).scatter_(1, ranked, True)
        c = torch.where(take[:, :, None], by, -math.inf).view(rows, n)
    ranked = torch.sort(c, dim=1, descending=True, stable=True).indices[:, : s["k"]]
    none = torch.gather(c, 1, ranked) == -math.inf
    w = torch.where(none, 0.0, torch.gather(v, 1, ranked))
    if s["renorm"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    return torch.where(none, -1, ranked).to(torch.int32), w * SCALE


SCALE = 2.5


def _route_back_plain(s):
    v, _ = _score(s)
    some = s["experts"] >= 0
    at = s["experts"].clamp(min=0).long()
    picked = torch.where(some, torch.gather(v, 1, at), 0.0)
    ds = torch.where(some, s["grad"] * SCALE, 0.0)
    if s["renorm"]:
        total = picked.sum(1, keepdim=True)
        live = torch.where(total > 0, total, 1.0)
        ds = torch.where(total > 0, (ds - (ds * (picked / live)).sum(1, keepdim=True)) / live, 0.0)
        ds = torch.where(some, ds, 0.0)
    dv = torch.zeros_like(v).scatter_add_(1, at, ds)
    if s["score"] == "sigmoid":
        out = dv * v * (1.0 - v)
    else:
        out = v * (dv - (ds * picked).sum(1, keepdim=True))
    return out.to(s["logits"].dtype)


def _plan_plain(s):
    flat = s["experts"].reshape(-1).long()
    flat = torch.where(flat < 0, s["n"], flat)
    kept = torch.bincount(flat, minlength=s["n"] + 1)[: s["n"]]
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=flat.device), kept.cumsum(0)])
    order = torch.sort(flat, stable=True).indices
    empty = flat[order] == s["n"]
    slot = torch.empty_like(order).scatter_(0, order, torch.where(empty, -1, torch.arange(order.numel(), device=flat.device)))
    return offsets, torch.where(empty, -1, order).to(torch.int32), slot.to(torch.int32).view_as(s["experts"])


def _at_slots(s):
    some = s["slot"] >= 0
    return some, s["slot"].clamp(min=0).long()


def _to_slots(s, values):
    """Rows of `values` at their slots, zeros at the others (one more row takes what has none)."""
    some, at = _at_slots(s)
    slots = at.numel()
    out = torch.zeros(slots + 1, values.shape[-1], dtype=values.dtype, device=values.device)
    out[torch.where(some, at, slots)] = values
    return out[:slots]


def _gather_plain(s):
    return _to_slots(s, s["x"][:, None].expand(-1, s["k"], -1))


def _combine_plain(s):
    some, at = _at_slots(s)
    w = torch.where(some, s["weights"], 0.0)
    return (s["y"][at].float() * w[:, :, None]).sum(1).to(s["y"].dtype)


def _combine_back_plain(s):
    some, at = _at_slots(s)
    g = s["x"].float()[:, None]
    dy = _to_slots(s, (g * s["weights"][:, :, None]).to(s["y"].dtype))
    return dy, torch.where(some, (g * s["y"][at].float()).sum(2), 0.0)


# ---------------------------------------------------------------------------------------------- one pass


def run(state):
    s, op = state, state["op"]
    if own:
        from paper_2609_27209_gb300 import erc

        if op == "sample":
            ids, logp, kept = erc.erc_sample_rows(s["logits"], s["words"], **s["settings"])
            return dict(ids=ids, logp=logp, kept=kept)
        if op == "route":
            score = erc.ERC_SCORE_SOFTMAX if s["score"] == "softmax" else erc.ERC_SCORE_SIGMOID
            if s["way"] == "backward":
                return dict(dlogits=erc.erc_route_backward(s["logits"], s["experts"], s["grad"], score=score,
                                                           renorm=s["renorm"], scale=SCALE))
            experts, weights = erc.erc_route(s["logits"], s["k"], score=score, bias=s["bias_values"], groups=s["groups"],
                                             top_groups=s["top"], group_best=s["best"], renorm=s["renorm"], scale=SCALE)
            return dict(experts=experts, weights=weights)
        if op == "plan":
            offsets, order, slot = erc.erc_expert_plan(s["experts"], s["n"])
            return dict(offsets=offsets, order=order, slot=slot)
        if s["way"] == "gather":
            return dict(xs=erc.erc_expert_gather(s["x"], s["slot"], s["offsets"]))
        if s["way"] == "forward":
            return dict(out=erc.erc_expert_combine(s["y"], s["slot"], s["weights"]))
        dy, dweights = erc.erc_expert_combine_backward(s["x"], s["y"], s["slot"], s["offsets"], s["weights"])
        return dict(dy=dy, dweights=dweights)
    if op == "sample":
        return _sample_plain(s)
    if op == "route":
        if s["way"] == "backward":
            return dict(dlogits=_route_back_plain(s))
        experts, weights = _route_plain(s)
        return dict(experts=experts, weights=weights)
    if op == "plan":
        offsets, order, slot = _plan_plain(s)
        return dict(offsets=offsets, order=order, slot=slot)
    if s["way"] == "gather":
        return dict(xs=_gather_plain(s))
    if s["way"] == "forward":
        return dict(out=_combine_plain(s))
    dy, dweights = _combine_back_plain(s)
    return dict(dy=dy, dweights=dweights)


def work(case):
    rows, n = case["rows"], case["n"]
    if case["op"] == "sample":
        return {"bytes": rows * (n * BYTES[case["type"]] + 8 + 12), "flops": 2 * rows * n}
    k = case["k"]
    if case["op"] == "route":
        if case["way"] == "backward":
            return {"bytes": rows * (2 * n * BYTES[case["type"]] + 8 * k), "flops": 6 * rows * n}
        return {"bytes": rows * (n * BYTES[case["type"]] + 8 * k), "flops": 4 * rows * n}
    if case["op"] == "plan":
        return {"bytes": 12 * rows * k + 8 * (n + 1), "flops": 0}
    row = case["width"] * BYTES[case["type"]]
    if case["way"] == "gather":
        return {"bytes": rows * (row + k * (row + 4)), "flops": 0}
    if case["way"] == "forward":
        return {"bytes": rows * (row + k * (row + 8)), "flops": 2 * rows * k * case["width"]}
    return {"bytes": rows * (row + k * (2 * row + 12)), "flops": 3 * rows * k * case["width"]}


# ---------------------------------------------------------------------------------------------- 64 bits


def _host(t):
    return t.detach().cpu().to(torch.float64 if t.is_floating_point() else torch.int64).numpy()


def _exact_sample(s):
    x = _host(s["logits"])
    rows, n = x.shape
    words = s["words"].cpu().numpy().view(np.uint64)
    each = {k: (_host(v) if isinstance(v, torch.Tensor) else np.full(rows, np.float32(v) if isinstance(v, float) else v))
            for k, v in s["settings"].items()}
    logp = np.empty(rows)
    for i in range(rows):
        live = np.flatnonzero(x[i] > -np.inf)
        if not live.size:
            logp[i] = -np.inf
            continue
        l = x[i][live]
        if not each["temperature"][i] > 0:
            logp[i] = 0.0
            continue
        p = np.exp((l - l.max()) / float(each["temperature"][i]))
        ok = (p >= float(each["min_p"][i])) & (p >= 2.0**-41)
        live, l, p = live[ok], l[ok], p[ok]
        if each["top_k"][i] > 0 or each["top_p"][i] < 1:
            by = np.argsort(-l, kind="stable")
            if each["top_k"][i] > 0:
                by = by[: int(each["top_k"][i])]
            if each["top_p"][i] < 1:
                mass = np.cumsum(p[by])
                by = by[: 1 + int(np.searchsorted(mass, float(each["top_p"][i]) * mass[-1]))]
            by.sort()
            p = p[by]
        mass = np.cumsum(p)
        j = min(int(np.searchsorted(mass, float(words[i]) / 2.0**64 * mass[-1], side="right")), p.size - 1)
        rest = mass[-1] - p[j]
        logp[i] = math.log1p(-rest / mass[-1]) if 2 * p[j] > mass[-1] else math.log(p[j] / mass[-1])
    return dict(ids=None, logp=logp, kept=None)


def _exact_score(s):
    x = _host(s["logits"])
    if s["score"] == "sigmoid":
        e = np.exp(-np.abs(x))
        return np.where(x >= 0, 1.0, e) / (1.0 + e)
    e = np.exp(x - x.max(1, keepdims=True))
    return e / e.sum(1, keepdims=True)


def _exact_route(s):
    v = _exact_score(s)
    rows, n = v.shape
    if s["way"] == "backward":
        at, g = _host(s["experts"]), _host(s["grad"]) * SCALE
        picked = np.take_along_axis(v, at, 1)
        if s["renorm"]:
            total = picked.sum(1, keepdims=True)
            g = (g - (g * (picked / total)).sum(1, keepdims=True)) / total
        if s["score"] == "sigmoid":
            out = np.zeros_like(v)
            np.put_along_axis(out, at, g * picked * (1 - picked), 1)
        else:
            out = -v * (g * picked).sum(1, keepdims=True)
            np.put_along_axis(out, at, picked * (g - (g * picked).sum(1, keepdims=True)), 1)
        return dict(dlogits=out)
    c = v if s["bias_values"] is None else v + _host(s["bias_values"])
    if s["groups"] > 1:
        by = c.reshape(rows, s["groups"], -1)
        score = -np.sort(-by, 2)[:, :, : s["best"]].sum(2)
        worst = np.argsort(-score, 1, kind="stable")[:, s["top"]:]
        by = by.copy()
        np.put_along_axis(by, worst[:, :, None], -np.inf, 1)
        c = by.reshape(rows, n)
    at = np.argsort(-c, 1, kind="stable")[:, : s["k"]]
    w = np.take_along_axis(v, at, 1)
    if s["renorm"]:
        w = w / w.sum(1, keepdims=True)
    return dict(experts=None, weights=w * SCALE)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "sample":
        return _exact_sample(s) if case["rows"] * case["n"] <= 64_000_000 else None
    if case["op"] == "route":
        return _exact_route(s)
    if case["op"] == "plan" or case["way"] == "gather" or case["rows"] * case["k"] * case["width"] > 300_000_000:
        return None
    slot, y = _host(s["slot"]), _host(s["y"])
    w = np.where(slot >= 0, _host(s["weights"]), 0.0)
    at = np.maximum(slot, 0)
    if case["way"] == "forward":
        out = np.zeros((case["rows"], case["width"]))
        for j in range(case["k"]):
            out += y[at[:, j]] * w[:, j, None]
        return dict(out=out)
    g, some = _host(s["x"]), slot >= 0
    dy, dw = np.zeros_like(y), np.zeros(slot.shape)
    for j in range(case["k"]):
        dy[slot[some[:, j], j]] = g[some[:, j]] * w[some[:, j], j, None]
        dw[:, j] = np.where(some[:, j], np.einsum("td,td->t", g, y[at[:, j]]), 0.0)
    return dict(dy=dy, dweights=dw)
