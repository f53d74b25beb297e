"""Timed cases of the routing operators: from the router's logits of a mixture-of-experts layer to
the demand vector the planner reads, and the loss that works against the skew in training.

    route     the choice of top_k experts per token and their weights (nimble_moe_route), as it is
              served: nothing but the choice
    train     the training step of a router: choice, weights, counts and probability sums per
              segment (nimble_moe_route), balance loss (nimble_moe_balance_loss) and the gradient
              of the logits from the gradients of weights and loss (nimble_moe_route_backward)
    demand    the All-to-Allv demand of routed tokens: slots per expert and distinct tokens per
              destination GPU (nimble_moe_counts), and the bytes per commodity that a plan is
              solved for (nimble_moe_traffic)

Sizes are those of the benchmark configurations: 64 to 1024 experts, 2 or 8 per token, 4096 to
16384 tokens per GPU, hidden sizes 4096 and 7168 in bf16, fabrics of 8 to 512 GPUs.

`run` computes the same in plain torch where `own` is false.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ALPHA = 1e-2                # weight of the balance loss


def _route(op, tokens, experts, top_k, dtype, score="softmax", renorm=True, scale=1.0, bias=False,
           padded=0.0, masked=0.0, segments=1, ragged=False):
    return dict(op=op, tokens=tokens, experts=experts, top_k=top_k, dtype=dtype, score=score,
                renorm=renorm, scale=scale, bias=bias, padded=padded, masked=masked,
                segments=segments, ragged=ragged)


def _demand(batch, ranks, tokens, experts, top_k, skew, hidden, way_back=False):
    return dict(op="demand", batch=batch, ranks=ranks, tokens=tokens, experts=experts, top_k=top_k,
                skew=skew, hidden=hidden, way_back=way_back)


def listed():
    return [
        # one token of one sequence being generated, 64 experts
        dict(_route("route", 1, 64, 2, "f32"), name="route_1x64"),
        # a decoding batch on a model of 256 experts that balances by a bias on the choice
        dict(_route("route", 96, 256, 8, "bf16", score="sigmoid", scale=2.5, bias=True),
             name="route_96x256_sigmoid"),
        # a prompt on one GPU of the 512-GPU fabric: 1024 experts
        dict(_route("route", 16384, 1024, 8, "bf16"), name="route_16384x1024"),
        # a training step on one GPU of the two-node fabric: 64 experts, top-2
        dict(_route("train", 4096, 64, 2, "f32"), name="train_4096x64"),
        # one GPU of the 16-node fabric, eight packed sequences of unequal lengths, a loss each
        dict(_route("train", 8192, 256, 8, "bf16", score="sigmoid", scale=2.5, bias=True,
                    segments=8, ragged=True), name="train_8192x256_packed"),
        # a padded batch, a count of experts that fills no power of two, some of them switched off
        dict(_route("train", 30011, 160, 6, "f16", renorm=False, scale=16.0, padded=0.2,
                    masked=0.1, segments=61, ragged=True), name="train_30011x160_padded"),
        # one GPU of the 512-GPU fabric
        dict(_route("train", 16384, 1024, 8, "f32"), name="train_16384x1024"),
        # every source of the 128-GPU fabric at once, as the model of the whole fabric sees it
        dict(_route("train", 1 << 20, 256, 8, "bf16", segments=128), name="train_1048576x256"),
        # the demand of one layer on two nodes
        dict(_demand(1, 16, 4096, 64, 2, 1.2, 4096), name="demand_2x8"),
        # 61 MoE layers of a one-node model in one call
        dict(_demand(61, 8, 8192, 64, 2, 1.0, 7168), name="demand_61_layers_1x8"),
        # the way back of an odd fabric: 7 nodes of 6 GPUs
        dict(_demand(3, 42, 5001, 252, 5, 1.4, 7168, way_back=True), name="demand_7x6_back"),
        # the largest fabric: 512 sources, 1024 experts, top-8
        dict(_demand(1, 512, 16384, 1024, 8, 1.6, 7168), name="demand_64x8"),
    ]


def _log_int(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over the logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["route", "train", "train", "demand"])
    if op == "demand":
        ranks = rng.choice([4, 6, 8, 16, 42, 64, 128, 192, 512])
        per = rng.choice([1, 2, 4, 6, 8])
        experts = min(ranks * per, 1024 // ranks * ranks)
        top_k = rng.randint(1, min(8, experts))
        tokens = _log_int(rng, 1, 16384)
        batch = _log_int(rng, 1, max(1, min(256, (1 << 22) // (ranks * tokens))))
        return _demand(batch, ranks, tokens, experts, top_k, 0.8 + 0.8 * rng.random(),
                       rng.choice([4096, 7168]), rng.random() < 0.3)
    experts = rng.choice([8, 16, 60, 64, 96, 128, 160, 256, 256, 384, 512, 1000, 1024])
    top_k = rng.randint(1, min(8, experts))
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    score = rng.choice(["softmax", "softmax", "sigmoid"])
    if op == "route":
        return _route(op, _log_int(rng, 1, 65536), experts, top_k, dtype, score,
                      rng.random() < 0.6, rng.choice([1.0, 2.5]), rng.random() < 0.4,
                      rng.choice([0.0, 0.0, 0.3]), rng.choice([0.0, 0.1]))
    tokens = _log_int(rng, 16, min(1 << 18, (1 << 26) // experts))
    return _route(op, tokens, experts, top_k, dtype, score, rng.random() < 0.6,
                  rng.choice([1.0, 2.5]), rng.random() < 0.4, rng.choice([0.0, 0.0, 0.3]),
                  rng.choice([0.0, 0.1]), _log_int(rng, 1, min(256, tokens)), rng.random() < 0.5)


def _segments(case, rng):
    """Row offsets of the segments: equal ones that cover every row, or ragged ones (some empty)
    that leave a few rows behind the last."""
    T, S = case["tokens"], case["segments"]
    if not case["ragged"]:
        return np.array([T * s // S for s in range(S + 1)], dtype=np.int32)
    cut = np.sort(rng.integers(0, T - T // 50 + 1, S - 1))
    return np.r_[0, cut, T - T // 50].astype(np.int32)


def _popularity(n, s, gen):
    """log of Zipf(s) weights of n experts in a random order."""
    order = torch.randperm(n, generator=gen, device=DEVICE).float() + 1.0
    return -s * torch.log(order)


def _chosen(rows, k, logw, gen):
    """k distinct experts per row, drawn with Zipf weights, the first drawn first."""
    out = torch.empty((rows, k), dtype=torch.int32, device=DEVICE)
    step = max(1, (1 << 26) // logw.numel())
    for a in range(0, rows, step):
        n = min(step, rows - a)
        u = torch.rand((n, logw.numel()), generator=gen, device=DEVICE).clamp_(min=1e-12)
        noise = u.log_().neg_().log_().neg_()
        out[a:a + n] = noise.add_(logw).topk(k, dim=1).indices.int()
    return out


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    rng = np.random.default_rng(int(seed))
    if case["op"] == "demand":
        B, R, T, E, k = (case[n] for n in ("batch", "ranks", "tokens", "experts", "top_k"))
        index = torch.cat([_chosen(R * T, k, _popularity(E, case["skew"], gen), gen)
                           for _ in range(B)])
        seg = torch.arange(B * R + 1, dtype=torch.int32, device=DEVICE) * T
        place = torch.arange(E, dtype=torch.int32, device=DEVICE) // (E // R)
        return dict(case=case, index=index, seg=seg, place=place,
                    counts=torch.zeros((B * R, E), dtype=torch.int32, device=DEVICE),
                    rank_tokens=torch.zeros((B * R, R), dtype=torch.int32, device=DEVICE),
                    traffic=torch.zeros((B, R * (R - 1)), dtype=torch.float64, device=DEVICE))
    T, E, k, S = (case[n] for n in ("tokens", "experts", "top_k", "segments"))
    dt = DTYPES[case["dtype"]]
    x = torch.randn((T, E), generator=gen, device=DEVICE)
    pop = _popularity(E, 1.0, gen)
    x += pop - pop.mean()
    if case["masked"]:
        off = torch.rand((T, E), generator=gen, device=DEVICE) < case["masked"]
        off[::101] = True                       # a row that its mask leaves without experts
        x.masked_fill_(off, -math.inf)
    x = x.to(dt)
    bias = (-0.5 * (pop - pop.mean())).contiguous() if case["bias"] else None
    keep = None
    if case["padded"]:
        keep = (torch.rand(T, generator=gen, device=DEVICE) >= case["padded"]).to(torch.uint8)
    seg = _segments(case, rng)
    state = dict(case=case, x=x, bias=bias, keep=keep,
                 index=torch.full((T, k), -1, dtype=torch.int32, device=DEVICE),
                 weight=torch.zeros((T, k), device=DEVICE))
    if case["op"] == "train":
        # a mean over the tokens; in f16 with the loss scaled, so that gradients stay in its range
        unit = 1.0 if dt == torch.float16 else 1.0 / T
        state.update(
            seg=torch.as_tensor(seg).to(DEVICE),
            grad_weight=torch.randn((T, k), generator=gen, device=DEVICE) * unit,
            grad_loss=torch.rand(S, generator=gen, device=DEVICE) * (unit * T / S),
            counts=torch.zeros((S, E), dtype=torch.int32, device=DEVICE),
            routed=torch.zeros(S, dtype=torch.int32, device=DEVICE),
            prob_sum=torch.zeros((S, E), device=DEVICE),
            loss=torch.zeros(S, device=DEVICE),
            grad_logits=torch.zeros((T, E), dtype=dt, device=DEVICE))
    return state


# ---- the framework's calls ------------------------------------------------------------------

def _own_run(st):
    from paper_2604_00317_amd import binding as B
    case = st["case"]
    if case["op"] == "demand":
        B.nimble_moe_counts(st["index"], case["experts"], st["counts"], d_expert_rank=st["place"],
                            d_rank_tokens=st["rank_tokens"], d_seg_ptr=st["seg"])
        B.nimble_moe_traffic(case["batch"], st["rank_tokens"], 2 * case["hidden"], st["traffic"],
                             way_back=case["way_back"])
        return dict(counts=st["counts"], rank_tokens=st["rank_tokens"], traffic=st["traffic"])
    form = dict(sigmoid=case["score"] == "sigmoid", renorm=case["renorm"], scale=case["scale"],
                d_keep=st["keep"])
    if case["op"] == "route":
        B.nimble_moe_route(st["x"], st["index"], st["weight"], d_bias=st["bias"], **form)
        return dict(index=st["index"], weight=st["weight"])
    sums = dict(d_counts=st["counts"], d_routed=st["routed"])
    B.nimble_moe_route(st["x"], st["index"], st["weight"], d_bias=st["bias"],
                       d_prob_sum=st["prob_sum"], d_seg_ptr=st["seg"], **sums, **form)
    B.nimble_moe_balance_loss(st["counts"], st["routed"], st["prob_sum"], case["top_k"], ALPHA,
                              st["loss"])
    B.nimble_moe_route_backward(st["x"], st["index"], st["weight"], st["grad_logits"],
                                d_grad_weight=st["grad_weight"], alpha=ALPHA,
                                d_grad_loss=st["grad_loss"], d_seg_ptr=st["seg"], **sums, **form)
    return {n: st[n] for n in _TRAINED}


_TRAINED = ("index", "weight", "counts", "routed", "prob_sum", "loss", "grad_logits")


# ---- the plain form -------------------------------------------------------------------------

def _plain_choice(x, bias, live, k):
    """The k largest keys per row in falling order, ties to the lowest index; -1 where there is none."""
    key = x + (0.0 if bias is None else bias)
    key = key.masked_fill((x == -math.inf) | ~live[:, None], -math.inf)
    val, idx = torch.sort(key, dim=1, descending=True, stable=True)
    return torch.where(val[:, :k] > -math.inf, idx[:, :k], -1)


def _plain_scores(x, ok, case):
    """(log of the score of every expert, log of the row's sum, probabilities); rows without a
    choice: probabilities 0, sum 1."""
    ls = x if case["score"] == "softmax" else -torch.log1p(torch.exp(-x.abs())) + x.clamp(max=0.0)
    stat = torch.where(ok, torch.logsumexp(ls, 1), 0.0)
    prob = torch.where(ok[:, None], torch.exp(ls - stat[:, None]), 0.0)
    return ls, stat, prob


def _plain_weights(ls, stat, idx, case):
    have = idx >= 0
    chosen = torch.gather(ls, 1, idx.clamp(min=0)).masked_fill(~have, -math.inf)
    if case["renorm"]:
        w = torch.softmax(chosen, 1)
    elif case["score"] == "softmax":
        w = torch.exp(chosen - stat[:, None])
    else:
        w = torch.exp(chosen)
    return torch.where(have, w, 0.0) * case["scale"]


def _plain_run(st):
    case = st["case"]
    if case["op"] == "demand":
        return _plain_demand(st)
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    x = st["x"].float()
    rows = torch.arange(T, device=x.device)
    live = torch.ones(T, dtype=torch.bool, device=x.device)
    if st["keep"] is not None:
        live = st["keep"] != 0
    if case["op"] == "train":
        live = live & (rows >= st["seg"][0]) & (rows < st["seg"][-1])
    idx = _plain_choice(x, st["bias"], live, k)
    ok = idx[:, 0] >= 0
    ls, stat, prob = _plain_scores(x, ok, case)
    weight = _plain_weights(ls, stat, idx, case)
    out = dict(index=idx.int(), weight=weight)
    if case["op"] == "route":
        return out
    S, ends = case["segments"], st["seg"].long()
    seg_of = torch.bucketize(rows, ends[1:], right=True).clamp(max=S - 1)
    have = idx >= 0
    slot = (seg_of[:, None] * E + idx)[have]
    counts = torch.zeros(S * E, dtype=torch.int64, device=x.device)
    counts = counts.scatter_add_(0, slot, torch.ones_like(slot)).view(S, E)
    if T % S == 0 and not case["ragged"]:
        prob_sum = prob.view(S, T // S, E).sum(1, dtype=torch.float64)
    else:
        covered = T - T // 50 if case["ragged"] else T
        prob_sum = torch.segment_reduce(prob[:covered].double(), "sum", offsets=ends, axis=0,
                                        initial=0.0)
    routed = torch.zeros(S, dtype=torch.int64, device=x.device).scatter_add_(0, seg_of, ok.long())
    n = routed.clamp(min=1).double()
    loss = ALPHA * E / k * (counts * prob_sum).sum(1) / n ** 2
    # backward
    coef = (st["grad_loss"].double() * ALPHA * E / k / n ** 2)[:, None] * counts
    c = coef.float()[seg_of]
    g = torch.where(have, st["grad_weight"], 0.0)
    wg = (weight * g).sum(1, keepdim=True)
    a = weight * (g - wg / case["scale"]) if case["renorm"] else weight * g
    rest = (prob * c).sum(1, keepdim=True)
    if case["score"] == "softmax":
        dx = prob * (c - rest - (0.0 if case["renorm"] else wg))
    else:
        dx = prob * torch.sigmoid(-x) * (c - rest)
        a = a * torch.sigmoid(-torch.gather(x, 1, idx.clamp(min=0)))
    dx.scatter_add_(1, idx.clamp(min=0), torch.where(have, a, 0.0))
    return dict(out, counts=counts.int(), routed=routed.int(),
                prob_sum=prob_sum.float(), loss=loss.float(), grad_logits=dx.to(st["x"].dtype))


def _plain_demand(st):
    case = st["case"]
    B, R, E, k = (case[n] for n in ("batch", "ranks", "experts", "top_k"))
    idx = st["index"].long()
    src = torch.arange(idx.shape[0], device=idx.device)[:, None] // case["tokens"]
    counts = torch.zeros(B * R * E, dtype=torch.int32, device=idx.device)
    counts.scatter_add_(0, (src * E + idx).view(-1),
                        torch.ones(idx.numel(), dtype=torch.int32, device=idx.device))
    dst = st["place"].long()[idx]
    before = torch.ones((k, k), dtype=torch.bool, device=idx.device).tril(-1)
    first = ~((dst[:, :, None] == dst[:, None, :]) & before).any(2)
    at = (src * R + dst)[first]
    tokens = torch.zeros(B * R * R, dtype=torch.int32, device=idx.device)
    tokens.scatter_add_(0, at, torch.ones_like(at, dtype=torch.int32))
    tokens = tokens.view(B, R, R)
    pairs = (tokens.transpose(1, 2) if case["way_back"] else tokens)
    away = ~torch.eye(R, dtype=torch.bool, device=idx.device)
    traffic = pairs[:, away].double() * (2 * case["hidden"])
    return dict(counts=counts.view(B * R, E), rank_tokens=tokens.view(B * R, R), traffic=traffic)


def run(state):
    if own:
        return _own_run(state)
    return _plain_run(state)


# ---- in 64 bits -----------------------------------------------------------------------------

def _exact_demand(case, st):
    B, R, T, E = (case[n] for n in ("batch", "ranks", "tokens", "experts"))
    index = st["index"].cpu().numpy()
    counts = np.empty((B * R, E), dtype=np.int32)
    tokens = np.empty((B * R, R), dtype=np.int32)
    for s in range(B * R):
        part = index[s * T:(s + 1) * T]
        counts[s] = np.bincount(part.ravel(), minlength=E)
        hit = np.zeros((T, R), dtype=bool)
        hit[np.arange(T)[:, None], part // (E // R)] = True
        tokens[s] = hit.sum(0)
    traffic = np.empty((B, R * (R - 1)))
    for b in range(B):
        m = tokens[b * R:(b + 1) * R].astype(np.float64)
        m = m.T if case["way_back"] else m
        traffic[b] = m[~np.eye(R, dtype=bool)] * (2.0 * case["hidden"])
    return dict(counts=torch.as_tensor(counts), rank_tokens=torch.as_tensor(tokens),
                traffic=torch.as_tensor(traffic))


def _logit64(x):
    """log of the logistic function."""
    return np.where(x > 0, -np.log1p(np.exp(-np.abs(x))), x - np.log1p(np.exp(-np.abs(x))))


def exact(case, seed):
    """The definition in 64 bits, a segment at a time."""
    if case["op"] != "demand" and case["tokens"] * case["experts"] > 1 << 25:
        return None
    st = prepare(case, seed)
    if case["op"] == "demand":
        return _exact_demand(case, st)
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    train = case["op"] == "train"
    x32 = st["x"].float().cpu().numpy()
    key = x32 if st["bias"] is None else x32 + st["bias"].cpu().numpy()[None, :]
    live = np.ones(T, dtype=bool) if st["keep"] is None else st["keep"].cpu().numpy() != 0
    ends = st["seg"].cpu().numpy() if train else np.array([0, T])
    S = len(ends) - 1
    f = {n: st[n].double().cpu().numpy() for n in ("grad_weight", "grad_loss") if n in st}
    out = dict(index=np.full((T, k), -1, dtype=np.int32), weight=np.zeros((T, k)))
    if train:
        out.update(counts=np.zeros((S, E), dtype=np.int32),
                   routed=np.zeros(S, dtype=np.int32), prob_sum=np.zeros((S, E)),
                   loss=np.zeros(S), grad_logits=np.zeros((T, E)))
    for s in range(S):
        rows = np.arange(ends[s], ends[s + 1])
        rows = rows[live[rows]]
        rows = rows[np.isfinite(x32[rows]).any(1)]
        if not rows.size:
            continue
        x = x32[rows].astype(np.float64)
        kk = np.where(np.isfinite(x32[rows]), key[rows], -np.inf)
        pick = np.argsort(-kk, axis=1, kind="stable")[:, :k]
        there = np.take_along_axis(kk, pick, 1) > -np.inf
        soft = case["score"] == "softmax"
        with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
            u = x if soft else np.where(np.isfinite(x), _logit64(x), -np.inf)
        top = u.max(1, keepdims=True)
        total = top + np.log(np.exp(u - top).sum(1, keepdims=True))
        p = np.exp(u - total)
        up = np.where(there, np.take_along_axis(u, pick, 1), -np.inf)
        if case["renorm"]:
            q = np.exp(up - up.max(1, keepdims=True))
            q /= q.sum(1, keepdims=True)
        else:
            q = np.exp(up - total) if soft else np.exp(up)
        w = q * case["scale"]
        out["index"][rows] = np.where(there, pick, -1)
        out["weight"][rows] = w
        if not train:
            continue
        cnt = np.bincount(pick[there], minlength=E)
        out["counts"][s], out["routed"][s], out["prob_sum"][s] = cnt, len(rows), p.sum(0)
        unit = ALPHA * E / k / len(rows) ** 2
        out["loss"][s] = unit * (cnt * p.sum(0)).sum()
        # the Jacobian of the probabilities, then of the weights of the chosen
        dp = f["grad_loss"][s] * unit * cnt
        dw = np.where(there, f["grad_weight"][rows], 0.0) * case["scale"]
        if case["renorm"]:
            du_pick = q * (dw - (q * dw).sum(1, keepdims=True))
        else:
            du_pick = q * dw
        du = p * (dp - (p * dp).sum(1, keepdims=True))
        if soft and not case["renorm"]:
            du -= p * du_pick.sum(1, keepdims=True)
        np.put_along_axis(du, pick, np.take_along_axis(du, pick, 1) + np.where(there, du_pick, 0.0), 1)
        slope = 1.0 if soft else np.exp(_logit64(np.where(np.isfinite(x), -x, 0.0)))
        out["grad_logits"][rows] = np.where(np.isfinite(x), du * slope, 0.0)
    return {n: torch.as_tensor(v) for n, v in out.items()}


def work(case):
    if case["op"] == "demand":
        B, R, T, E, k = (case[n] for n in ("batch", "ranks", "tokens", "experts", "top_k"))
        n = B * R * T
        return dict(bytes=n * k * 4 + E * 4 + B * R * (E + R) * 4 + B * R * (R - 1) * 8,
                    flops=n * (2 * k + k * (k - 1) // 2))
    T, E, k, S = (case[n] for n in ("tokens", "experts", "top_k", "segments"))
    z = DTYPES[case["dtype"]].itemsize
    size = T * E * z + T * k * 8 + (E * 4 if case["bias"] else 0) + (T if case["padded"] else 0)
    ops = T * (5 * E + 4 * k)
    if case["op"] == "train":
        size += T * E * z + T * k * 4 + S * (E * 8 + 16)
        ops += T * (8 * E + 6 * k)
    return dict(bytes=size, flops=ops)
