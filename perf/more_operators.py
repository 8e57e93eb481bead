"""Operators of training and answering with experts over a graph's nodes, as cases: plain forms and exact values.

Operators (paper_2609_27209_gb300.erc):
  score    erc_score_rows, erc_score_rows_backward: log probability of a given entry of each row of scores, the row's
           entropy and its best entries, and the scores' gradient
  ffn      erc_expert_ffn, erc_expert_ffn_backward: the gated feed-forward block of each expert on its rows, and the
           gradients of rows and weights
  dropout  erc_dropout: dropout from a counter-based generator, with the residual's addition

Which entries dropout keeps and which entries are a row's best are defined exactly; the rest are computed numbers.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one walker's step on the 20,000-node graph, scored with its five best alternatives: latency
        dict(name="score_single", op="score", way="forward", rows=1, n=20000, type="f32", stride=20000, k=5,
             temperature=0.8, mask=0.0),
        # answers over the 169,343-node graph, with the alternatives that a service shows
        dict(name="score_batch", op="score", way="forward", rows=64, n=169343, type="bf16", stride=169343, k=20,
             temperature=1.0, mask=0.0),
        # the steps of many walkers over padded neighbour lists of odd length, some lists empty
        dict(name="score_walkers", op="score", way="forward", rows=16384, n=257, type="f32", stride=260, k=0,
             temperature=0.7, mask=0.6),
        # the loss of a training batch over the 20,000-node graph: the gradient of log probability and entropy
        dict(name="score_gradient", op="score", way="backward", rows=4096, n=20000, type="bf16", stride=20000, k=0,
             temperature=1.0, mask=0.0),
        # a few nodes answered at once: every expert's weights for a row or two
        dict(name="ffn_few", op="ffn", way="forward", slots=14, experts=8, width=512, inner=1024, type="bf16", act="silu",
             drop=0.0),
        # answering for a large batch: 64 experts of uneven load
        dict(name="ffn_batch", op="ffn", way="forward", slots=32768, experts=64, width=1024, inner=512, type="bf16",
             act="silu", drop=0.05),
        # a dense block in training: one expert, its projections kept for the backward pass
        dict(name="ffn_dense", op="ffn", way="train", slots=8192, experts=1, width=2048, inner=4096, type="f16", act="gelu",
             drop=0.0),
        # the gradients for the 20,000-node graph, four experts a node
        dict(name="ffn_gradient", op="ffn", way="backward", slots=80000, experts=64, width=512, inner=1024, type="bf16",
             act="silu", drop=0.0),
        # a small model in float32 with odd widths, as in a first experiment
        dict(name="ffn_odd", op="ffn", way="backward", slots=515, experts=5, width=100, inner=67, type="f32", act="relu",
             drop=0.1),
        # dropout inside a small training step: latency
        dict(name="dropout_few", op="dropout", rows=512, width=64, type="f32", p=0.1, residual=True),
        # every node of the 169,343-node graph, added to the residual
        dict(name="dropout_nodes", op="dropout", rows=169343, width=512, type="bf16", p=0.1, residual=True),
        # the gradient through it: the same call without a residual, odd width
        dict(name="dropout_gradient", op="dropout", rows=20000, width=1001, type="f16", p=0.3, residual=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["score", "score", "ffn", "ffn", "dropout"])
    if op == "score":
        n = _log(rng, 33, 2449029)
        rows = _log(rng, 1, max(1, min(32768, 50_000_000 // n)))
        return dict(op=op, way=rng.choice(["forward", "forward", "backward"]), rows=rows, n=n,
                    type=rng.choice(["f32", "bf16", "f16"]), stride=n + rng.choice([0, 0, 1, 7, 8]),
                    k=min(n, rng.choice([0, 1, 5, 20, 32])), temperature=rng.choice([0.7, 1.0, 1.3]),
                    mask=rng.choice([0.0, 0.1, 0.6]))
    if op == "ffn":
        kind, way = rng.choice(["f32", "bf16", "bf16", "f16"]), rng.choice(["forward", "train", "backward"])
        experts = rng.choice([1, 3, 8, 64, 128])
        odd = kind != "f32" and rng.random() < 0.2
        step = 1 if kind == "f32" or odd else 8
        most = 2_000_000_000 if step == 1 else 40_000_000_000  # slots * width * inner
        width = max(step, _log(rng, 16, 2048) // step * step)
        inner = max(step, _log(rng, 16, 2048) // step * step)
        while experts * width * inner > 150_000_000:
            experts = (experts + 1) // 2
        return dict(op=op, way=way, slots=_log(rng, 1, max(1, min(131072, most // (width * inner)))), experts=experts,
                    width=width, inner=inner, type=kind, act=rng.choice(["silu", "gelu", "relu"]),
                    drop=rng.choice([0.0, 0.0, 0.1]))
    width = _log(rng, 16, 4096)
    return dict(op=op, rows=_log(rng, 1, max(1, 80_000_000 // width)), width=width, type=rng.choice(["f32", "bf16", "f16"]),
                p=rng.choice([0.1, 0.25, 0.5]), residual=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------- inputs


def _scores(g, rows, n):
    """Rows of scores between undecided and confident: normal with a spread of the row's own, a few entries favoured."""
    x = torch.randn(rows, n, generator=g, device="cuda")
    x *= 0.5 + 2.5 * torch.rand(rows, 1, generator=g, device="cuda")
    few = max(1, min(32, n // 16))
    at = torch.randint(0, n, (rows, few), generator=g, device="cuda")
    return x.scatter_add_(1, at, 8.0 * torch.rand(rows, few, generator=g, device="cuda"))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 29)
    s = dict(case)
    kind = TYPES[case["type"]]
    if case["op"] == "score":
        rows, n = case["rows"], case["n"]
        x = _scores(g, rows, n)
        if case["mask"]:
            # a row's list ends somewhere, at its very start in some rows
            ends = (torch.rand(rows, 1, generator=g, device="cuda") * (n + n * case["mask"]) - n * case["mask"] / 2).clamp(0, n)
            x.masked_fill_(torch.arange(n, device="cuda") >= ends, -math.inf)
        buffer = torch.zeros(rows, case["stride"], dtype=kind, device="cuda")
        buffer[:, :n] = x
        s["logits"] = buffer[:, :n]
        # mostly likely entries, as a walk or an answer holds them; a few rows have none
        ids = torch.argmax(x + 2.0 * torch.randn(rows, n, generator=g, device="cuda"), 1).to(torch.int32)
        s["ids"] = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.02, -1, ids).to(torch.int32)
        if case["way"] == "backward":
            full = _score_plain(s)
            s["norm"], s["entropy"] = full["norm"], full["entropy"]
            s["dlogp"] = torch.rand(rows, generator=g, device="cuda") - 1.5
            s["dentropy"] = 0.01 * torch.randn(rows, generator=g, device="cuda")
    elif case["op"] == "ffn":
        slots, experts, width, inner = case["slots"], case["experts"], case["width"], case["inner"]
        share = 0.3 + torch.rand(experts, generator=g, device="cuda")
        expert = torch.multinomial(share, slots, replacement=True, generator=g)
        expert = torch.where(torch.rand(slots, generator=g, device="cuda") < case["drop"], experts, expert)
        count = torch.bincount(expert, minlength=experts + 1)[:experts]
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), count.cumsum(0)])
        s["ends"] = s["offsets"].tolist()

        def normal(*shape, scale=1.0):
            return (scale * torch.randn(*shape, generator=g, device="cuda")).to(kind)

        s["x"] = normal(slots, width)
        s["x"][s["ends"][-1]:] = 0
        s["w_in"] = normal(experts, 2 * inner, width, scale=width**-0.5)
        s["w_out"] = normal(experts, width, inner, scale=inner**-0.5)
        if case["way"] == "backward":
            s["pre"] = _ffn_plain(s)["pre"]
            s["dy"] = normal(slots, width)
            s["dy"][s["ends"][-1]:] = 0
    else:
        s["x"] = torch.randn(case["rows"], case["width"], generator=g, device="cuda").to(kind)
        if case["residual"]:
            s["added"] = torch.randn(case["rows"], case["width"], generator=g, device="cuda").to(kind)
        s["key"] = torch.randint(-(2**63), 2**63 - 1, (1,), generator=g, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------- plain forms


def _below(s):
    """(scores without masked entries, distance from the row's maximum over the temperature, maximum)"""
    x = s["logits"].float()
    x = torch.where(torch.isnan(x), -math.inf, x)
    m = x.amax(1, keepdim=True)
    t = torch.where(x == m, 0.0, (x - m) / s["temperature"])
    return x, torch.where(x == -math.inf, -math.inf, t), m


def _score_plain(s):
    x, t, m = _below(s)
    some = m[:, 0] > -math.inf
    e = torch.exp(t)
    total = e.sum(1, dtype=torch.float64)
    log_sum = torch.where(some, torch.log(total), -math.inf).float()
    mean = torch.where(t == -math.inf, 0.0, e * t).sum(1, dtype=torch.float64)
    entropy = torch.where(some, torch.log(total) - mean / total, 0.0).float()
    given = (s["ids"] >= 0) & (s["ids"] < x.shape[1])
    at = torch.where(given, s["ids"], 0).long()[:, None]
    log_all = t.double() - torch.log(total)[:, None]
    logp = torch.where(given, torch.where(some, torch.gather(log_all, 1, at)[:, 0], -math.inf), 0.0).float()
    out = dict(logp=logp, entropy=entropy, norm=torch.stack([m[:, 0], log_sum], 1))
    if s["k"]:
        best = torch.sort(x, dim=1, descending=True, stable=True).indices[:, : s["k"]]
        masked = torch.gather(x, 1, best) == -math.inf
        out["top_ids"] = torch.where(masked, -1, best).to(torch.int32)
        out["top_logp"] = torch.where(masked, -math.inf, torch.gather(log_all, 1, best)).float()
    return out


def _score_back_plain(s):
    x, t, _ = _below(s)
    log_p = t - s["norm"][:, 1:]
    masked = x == -math.inf
    p = torch.where(masked, 0.0, torch.exp(log_p))
    given = (s["ids"] >= 0) & (s["ids"] < x.shape[1])
    at = torch.where(given, s["ids"], 0).long()[:, None]
    given = given & ~torch.gather(masked, 1, at)[:, 0]
    g = torch.where(given, s["dlogp"], 0.0)
    out = -p * (g[:, None] + s["dentropy"][:, None] * (log_p + s["entropy"][:, None]))
    out = torch.where(masked, 0.0, out)
    out.scatter_add_(1, at, g[:, None])
    return (out / s["temperature"]).to(s["logits"].dtype)


def _act(a, kind):
    """(act(a), act'(a))"""
    if kind == "relu":
        return a.clamp(min=0), (a > 0).to(a.dtype)
    if kind == "silu":
        q = 1.0 / (1.0 + torch.exp(-a))
        return a * q, q * (1.0 + a * (1.0 - q))
    q = 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5)))
    return a * q, q + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))


def _ffn_plain(s):
    slots, width = s["x"].shape
    inner, ends, kind = s["inner"], s["ends"], s["x"].dtype
    y = torch.zeros(slots, width, device="cuda")
    pre = torch.zeros(slots, 2 * inner, device="cuda")
    for e in range(s["experts"]):
        lo, hi = ends[e], ends[e + 1]
        if lo < hi:
            pre[lo:hi] = s["x"][lo:hi].float() @ s["w_in"][e].float().T
            h = _act(pre[lo:hi, :inner], s["act"])[0] * pre[lo:hi, inner:]
            y[lo:hi] = h @ s["w_out"][e].float().T
    return dict(y=y.to(kind), pre=pre.to(kind))


def _ffn_back_plain(s):
    inner, ends, kind = s["inner"], s["ends"], s["x"].dtype
    dx = torch.zeros(s["x"].shape, device="cuda")
    dw_in, dw_out = torch.zeros(s["w_in"].shape, device="cuda"), torch.zeros(s["w_out"].shape, device="cuda")
    for e in range(s["experts"]):
        lo, hi = ends[e], ends[e + 1]
        if lo < hi:
            x, dy, pre = (s[name][lo:hi].float() for name in ("x", "dy", "pre"))
            a, b = pre[:, :inner], pre[:, inner:]
            v, slope = _act(a, s["act"])
            dh = dy @ s["w_out"][e].float()
            dpre = torch.cat([dh * b * slope, dh * v], 1)
            dx[lo:hi] = dpre @ s["w_in"][e].float()
            dw_in[e] = dpre.T @ x
            dw_out[e] = dy.T @ (v * b)
    return dict(dx=dx.to(kind), dw_in=dw_in.to(kind), dw_out=dw_out.to(kind))


M32 = 0xFFFFFFFF
DROP = 0x44524F50  # "DROP"


def _philox(block, key):
    """Philox4x32-10 (Salmon et al., SC'11) of the counters (block lo, block hi, DROP, 0): words [blocks, 4]."""
    c = [block & M32, block >> 32, torch.full_like(block, DROP), torch.zeros_like(block)]
    k0, k1 = key & M32, (key >> 32) & M32
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & M32) ^ c[1] ^ k0, b & M32, ((a >> 32) & M32) ^ c[3] ^ k1, a & M32]
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    return torch.stack(c, 1)


def _kept(s):
    count = s["x"].numel()
    words = _philox(torch.arange((count + 3) // 4, device="cuda"), s["key"])
    return (words.view(-1)[:count] >= math.floor(s["p"] * 2.0**32)).view_as(s["x"])


def _dropout_plain(s):
    out = torch.where(_kept(s), s["x"].float() * (1.0 / (1.0 - s["p"])), 0.0)
    if s["residual"]:
        out = out + s["added"].float()
    return out.to(s["x"].dtype)


# ---------------------------------------------------------------------------------------------- one pass


def run(state):
    s = state
    if own:
        from paper_2609_27209_gb300 import erc

        if s["op"] == "score":
            if s["way"] == "backward":
                return dict(dlogits=erc.erc_score_rows_backward(
                    s["logits"], s["ids"], s["norm"], dlogp=s["dlogp"], entropy=s["entropy"], dentropy=s["dentropy"],
                    temperature=s["temperature"]))
            logp, entropy, norm, top_ids, top_logp = erc.erc_score_rows(s["logits"], s["ids"], k=s["k"],
                                                                        temperature=s["temperature"])
            out = dict(logp=logp, entropy=entropy, norm=norm)
            if s["k"]:
                out.update(top_ids=top_ids, top_logp=top_logp)
            return out
        if s["op"] == "ffn":
            act = dict(silu=erc.ERC_ACT_SILU, gelu=erc.ERC_ACT_GELU, relu=erc.ERC_ACT_RELU)[s["act"]]
            if s["way"] == "backward":
                dx, dw_in, dw_out = erc.erc_expert_ffn_backward(s["dy"], s["x"], s["pre"], s["offsets"], s["w_in"],
                                                                s["w_out"], act=act)
                return dict(dx=dx, dw_in=dw_in, dw_out=dw_out)
            y, pre = erc.erc_expert_ffn(s["x"], s["offsets"], s["w_in"], s["w_out"], act=act, keep=s["way"] == "train")
            return dict(y=y, pre=pre) if s["way"] == "train" else dict(y=y)
        return dict(out=erc.erc_dropout(s["x"], s["p"], s["key"], residual=s.get("added")))
    if s["op"] == "score":
        return dict(dlogits=_score_back_plain(s)) if s["way"] == "backward" else _score_plain(s)
    if s["op"] == "ffn":
        if s["way"] == "backward":
            return _ffn_back_plain(s)
        out = _ffn_plain(s)
        return out if s["way"] == "train" else dict(y=out["y"])
    return dict(out=_dropout_plain(s))


def work(case):
    size = BYTES[case["type"]]
    if case["op"] == "score":
        rows, n = case["rows"], case["n"]
        if case["way"] == "backward":
            return {"bytes": rows * (2 * n * size + 24), "flops": 6 * rows * n}
        return {"bytes": rows * (n * size + 20 + 8 * case["k"]), "flops": 4 * rows * n}
    if case["op"] == "ffn":
        slots, experts, width, inner = case["slots"], case["experts"], case["width"], case["inner"]
        weights = 3 * min(experts, slots) * width * inner
        if case["way"] == "backward":
            moved = slots * (3 * width + 2 * inner) + weights + 3 * experts * width * inner
            return {"bytes": moved * size, "flops": 12 * slots * width * inner}
        moved = slots * (2 * width + (2 * inner if case["way"] == "train" else 0)) + weights
        return {"bytes": moved * size, "flops": 6 * slots * width * inner}
    count = case["rows"] * case["width"]
    return {"bytes": (3 if case["residual"] else 2) * count * size, "flops": 2 * count}


# ---------------------------------------------------------------------------------------------- 64 bits


def _exact_score(s):
    x = s["logits"].double()
    rows, n = x.shape
    x = torch.nan_to_num(x, nan=-math.inf, posinf=math.inf, neginf=-math.inf) / s["temperature"]
    live = torch.isfinite(x.amax(1))
    given = (s["ids"] >= 0) & (s["ids"] < n)
    at = s["ids"].long().clamp(0, n - 1)[:, None]
    log_p = torch.where(live[:, None], x - torch.logsumexp(x, 1, keepdim=True), -math.inf)
    p = log_p.exp()
    entropy = -torch.where(p > 0, p * log_p, 0.0).sum(1)
    if s["way"] == "backward":
        hit = torch.gather(log_p, 1, at)[:, 0]
        g = torch.where(given & (hit > -math.inf), s["dlogp"].double(), 0.0)
        one = torch.zeros_like(p).scatter_(1, at, 1.0)
        pull = torch.where(p > 0, p * (log_p + entropy[:, None]), 0.0)
        return dict(dlogits=(g[:, None] * (one - p) - s["dentropy"].double()[:, None] * pull) / s["temperature"])
    logp = torch.where(given, torch.gather(log_p, 1, at)[:, 0], 0.0)
    top = x.amax(1)
    log_sum = torch.where(live, torch.logsumexp(x, 1) - top, -math.inf)
    out = dict(logp=logp, entropy=entropy, norm=torch.stack([top * s["temperature"], log_sum], 1))
    if s["k"]:
        out["top_ids"] = None
        out["top_logp"] = log_p.topk(s["k"], 1).values
    return out


def _exact_act(a, kind):
    if kind == "relu":
        return torch.where(a > 0, a, 0.0), torch.where(a > 0, 1.0, 0.0)
    if kind == "silu":
        return a / (1 + torch.exp(-a)), (1 + torch.exp(-a) * (1 + a)) / (1 + torch.exp(-a)) ** 2
    cdf = 0.5 * torch.erfc(-a / math.sqrt(2))
    return a * cdf, cdf + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)


def _exact_ffn(s):
    inner, last = s["inner"], s["ends"][-1]
    out = {}
    parts = {name: [] for name in ("y", "pre", "dx", "dw_in", "dw_out")}
    for e, (lo, hi) in enumerate(zip(s["ends"], s["ends"][1:])):
        x, into, back = s["x"][lo:hi].double(), s["w_in"][e].double(), s["w_out"][e].double()
        gate, up = into[:inner], into[inner:]
        if s["way"] != "backward":
            a, b = torch.einsum("sd,fd->sf", x, gate), torch.einsum("sd,fd->sf", x, up)
            parts["pre"].append(torch.cat([a, b], 1))
            parts["y"].append(torch.einsum("sf,df->sd", _exact_act(a, s["act"])[0] * b, back))
            continue
        a, b = s["pre"][lo:hi].double().split(inner, 1)
        dy = s["dy"][lo:hi].double()
        value, slope = _exact_act(a, s["act"])
        dh = torch.einsum("sd,df->sf", dy, back)
        da, db = dh * b * slope, dh * value
        parts["dx"].append(torch.einsum("sf,fd->sd", da, gate) + torch.einsum("sf,fd->sd", db, up))
        parts["dw_in"].append(torch.cat([torch.einsum("sf,sd->fd", da, x), torch.einsum("sf,sd->fd", db, x)]))
        parts["dw_out"].append(torch.einsum("sd,sf->df", dy, value * b))
    for name, values in parts.items():
        if values and name.startswith("dw"):
            out[name] = torch.stack(values)
        elif values:
            out[name] = torch.nn.functional.pad(torch.cat(values), (0, 0, 0, s["slots"] - last))
    if s["way"] == "forward":
        del out["pre"]
    return out


def _exact_kept(count, key, p):
    """Which entries stay, with Philox's rounds on unsigned words, a stretch of counters at a time."""
    least, low, kept = int(p * 2**32), np.uint64(2**32 - 1), np.empty((count + 3) // 4 * 4, dtype=bool)
    for first in range(0, kept.size // 4, 1 << 16):
        here = np.arange(first, min(first + (1 << 16), kept.size // 4), dtype=np.uint64)
        x, y, z, w = here & low, here >> np.uint64(32), np.full_like(here, 0x44524F50), np.zeros_like(here)
        for step in range(10):
            left, right = x * np.uint64(0xD2511F53), z * np.uint64(0xCD9E8D57)
            ka, kb = (key + step * 0x9E3779B9) % 2**32, ((key >> 32) + step * 0xBB67AE85) % 2**32
            x, y, z, w = (right >> np.uint64(32)) ^ y ^ np.uint64(ka), right & low, (left >> np.uint64(32)) ^ w ^ np.uint64(kb), left & low
        kept[4 * first : 4 * (first + here.size)] = (np.stack([x, y, z, w], 1) >= np.uint64(least)).ravel()
    return kept[:count]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "score":
        return _exact_score(s)
    if case["op"] == "ffn":
        return _exact_ffn(s)
    kept = torch.from_numpy(_exact_kept(case["rows"] * case["width"], s["key"].item() % 2**64, case["p"]))
    out = s["x"].double() * kept.to("cuda").view_as(s["x"]) / (1 - s["p"])
    return dict(out=out + s["added"].double() if case["residual"] else out)
