"""Performance cases of the operators for layers of experts and for clipped gradients, beside plain torch forms of each.

A layer of experts sends each of T tokens to K of E experts.  K-FAC on such a layer keeps a pair of factors for every expert, built
from that expert's tokens alone, so the tokens are brought into the experts' order first:

  sort           expert (T, K) -> offsets (E + 1), order (T K), place (T, K): assignment i = t K + k goes to row place[i], the rows of
                 expert e are offsets[e] .. offsets[e + 1] - 1 with assignments ascending, order[row] = i, -1 behind the last row.  An
                 expert outside 0 .. E - 1 is no assignment: its place is -1.
  dispatch       xs[place[t, k]] = x[t]                                 rows behind the last one stay as they are
  dispatch_back  dx[t] = sum_k dxs[place[t, k]]                         the gradient of dispatch
  combine        y[t] = sum_k weights[t, k] ys[place[t, k]]
  combine_back   dys[place[t, k]] = weights[t, k] dy[t],  dweights[t, k] = <dy[t], ys[place[t, k]]>
  factor         F_e = (1 / R_e) sum_r a_r a_r^T over the R_e rows of expert e, a_r = [row; 1] with a bias; 0 for no rows; with `decay`
                 S_e <- decay S_e + (1 - decay) F_e instead, S_e as it was for no rows
  clip           norm = sqrt(sum of g^2 over all tensors), out = g min(1, max_norm / norm)
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DECAY = 0.95
ALIGN = 128                                # elements: where a bucket of gradients begins each tensor


def listed():
    return [
        # One step of generation for two dozen sequences: launches and host work decide.
        {"name": "sort_step", "kind": "sort", "tokens": 24, "choices": 2, "experts": 16, "skew": 0.5, "drop": 0.0},
        # A training batch over many small experts, some tokens beyond the experts' capacity.
        {"name": "sort_batch", "kind": "sort", "tokens": 65536, "choices": 8, "experts": 256, "skew": 0.5, "drop": 0.05},
        # A single token on its way to its experts.
        {"name": "dispatch_token_bf16", "kind": "dispatch", "tokens": 1, "choices": 8, "experts": 64, "dim": 2048, "dtype": "bf16", "skew": 0.5, "drop": 0.0},
        # A batch's tokens brought into the experts' order.
        {"name": "dispatch_batch_bf16", "kind": "dispatch", "tokens": 16384, "choices": 4, "experts": 64, "dim": 2048, "dtype": "bf16", "skew": 0.5, "drop": 0.0},
        # Results of few experts of an odd width, in full precision, some assignments dropped.
        {"name": "combine_odd_f32", "kind": "combine", "tokens": 3001, "choices": 3, "experts": 13, "dim": 1001, "dtype": "f32", "skew": 1.0, "drop": 0.1},
        # The gradient of a small batch's dispatch.
        {"name": "dispatch_back_f16", "kind": "dispatch_back", "tokens": 4096, "choices": 2, "experts": 8, "dim": 1024, "dtype": "f16", "skew": 0.5, "drop": 0.0},
        # The gradient of a batch's weighted sum: the experts' output gradients, which the factors G come from, and the router's.
        {"name": "combine_back_bf16", "kind": "combine_back", "tokens": 16384, "choices": 4, "experts": 64, "dim": 2048, "dtype": "bf16", "skew": 0.5, "drop": 0.02},
        # A first test: a few small experts with biases in full precision.
        {"name": "factor_small_f32", "kind": "factor", "rows": 1024, "experts": 8, "dim": 256, "dtype": "f32", "bias": True, "ema": False, "skew": 0.5, "drop": 0.0},
        # Experts of a width that is no multiple of anything, very unequal, some without a token.
        {"name": "factor_ragged_f16", "kind": "factor", "rows": 5000, "experts": 19, "dim": 577, "dtype": "f16", "bias": True, "ema": False, "skew": 2.0, "drop": 0.05},
        # A training batch's running averages.
        {"name": "factor_batch_bf16", "kind": "factor", "rows": 65536, "experts": 32, "dim": 2048, "dtype": "bf16", "bias": False, "ema": True, "skew": 0.5, "drop": 0.0},
        # The gradients of a small model, each tensor where the last one ends.
        {"name": "clip_small_f32", "kind": "clip", "tensors": 41, "elements": 300001, "dtype": "f32", "aligned": False},
        # The gradients of a language model in one bucket.
        {"name": "clip_model_bf16", "kind": "clip", "tensors": 291, "elements": 500000000, "dtype": "bf16", "aligned": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["sort", "dispatch", "dispatch_back", "combine", "combine_back", "factor", "factor", "clip"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind == "clip":
        elements = _log(rng, 1000, 250000000)
        return {"kind": kind, "tensors": min(_log(rng, 1, 400), elements), "elements": elements, "dtype": dtype, "aligned": rng.random() < 0.5}
    routing = {"skew": round(rng.uniform(0, 2), 2), "drop": rng.choice([0.0, round(rng.uniform(0, 0.2), 2)])}
    experts = _log(rng, 2, 256)
    choices = rng.randint(1, min(8, experts))
    if kind == "sort":
        return {"kind": kind, "tokens": _log(rng, 1, 65536), "choices": choices, "experts": experts, **routing}
    if kind == "factor":
        dim = _log(rng, 32, 2048)
        dim = dim // 8 * 8 if rng.random() < 0.5 else dim
        experts = min(experts, max(2, 32 * 2048 ** 2 // dim ** 2))
        return {"kind": kind, "rows": _log(rng, 1, 65536), "experts": experts, "dim": dim, "dtype": dtype, "bias": rng.random() < 0.5,
                "ema": rng.random() < 0.5, **routing}
    dim = _log(rng, 32, 4096)
    dim = dim // 8 * 8 if rng.random() < 0.5 else dim
    tokens = min(_log(rng, 1, 65536), 16384 * 4 * 1024 // (choices * dim))      # (half the largest listed case's elements)
    return {"kind": kind, "tokens": max(1, tokens), "choices": choices, "experts": experts, "dim": dim, "dtype": dtype, **routing}


def _routing(case, tokens, choices, g):
    """(expert, weights): each token's `choices` best experts by unequal scores, some of them dropped, and their softmax."""
    E = case["experts"]
    liking = torch.randn(E, generator=g, device="cuda") * case["skew"]
    noise = -torch.log(-torch.log(torch.rand((tokens, E), generator=g, device="cuda").clamp(1e-20, 1 - 1e-7)))
    top, expert = (liking + noise).topk(choices, dim=1)
    expert = expert.to(torch.int32)
    if case["drop"]:
        expert[torch.rand((tokens, choices), generator=g, device="cuda") < case["drop"]] = -1
    return expert.contiguous(), torch.softmax(top, dim=1).contiguous()


def _sorted(expert, experts):
    """The plain form of sort."""
    flat = expert.reshape(-1).to(torch.int64)
    there = (flat >= 0) & (flat < experts)
    key = torch.where(there, flat, experts)
    count = torch.zeros(experts + 1, dtype=torch.int64, device=flat.device).index_add_(0, key, torch.ones_like(key))
    offsets = torch.cat([count.new_zeros(1), count[:experts].cumsum(0)])
    by_expert = torch.argsort(key, stable=True)
    row = torch.arange(flat.numel(), device=flat.device)
    place = torch.empty_like(row)
    place[by_expert] = row
    place = torch.where(there, place, -1)
    order = torch.where(row < offsets[experts], by_expert, -1)
    return offsets.to(torch.int32), order.to(torch.int32), place.to(torch.int32).reshape(expert.shape)


def _rows(case, g, n, dim, scale=1.0):
    return (torch.randn((n, dim), generator=g, device="cuda") * scale).to(DTYPES[case["dtype"]])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]
    s = {"kind": kind}
    if kind == "clip":
        sizes = _sizes(case)
        step = ALIGN if case["aligned"] else 1
        at = [0]
        for n in sizes:
            at.append(at[-1] + -(-n // step) * step)
        flat = torch.randn(at[-1], generator=g, device="cuda", dtype=torch.float32).mul_(1e-2)
        s["flat"] = flat.to(DTYPES[case["dtype"]])
        for a, n, b in zip(at, sizes, at[1:]):
            s["flat"][a + n:b] = 0                                   # between the bucket's tensors
        s["out"] = torch.zeros_like(s["flat"])
        s["max_norm"] = 0.3 * 1e-2 * math.sqrt(sum(sizes))           # gradients about three times the norm wanted
        if own:
            from paper_1811_12019_amd import binding as kb
            s["batch"] = kb.GradBatch([s["flat"][a:a + n] for a, n in zip(at, sizes)], [s["out"][a:a + n] for a, n in zip(at, sizes)])
        return s
    if kind == "factor":
        R, E, dim = case["rows"], case["experts"], case["dim"]
        expert, _ = _routing(case, R, 1, g)
        s["offsets"] = _sorted(expert, E)[0]
        s["bounds"] = s["offsets"].tolist()
        s["x"] = _rows(case, g, R, dim).clamp_(min=0)
        d = dim + int(case["bias"])
        s["bias"], s["ema"] = case["bias"], case["ema"]
        if case["ema"]:
            s["F"] = torch.randn((E, d, d), generator=g, device="cuda").mul_(1e-2)
            s["F"].add_(s["F"].transpose(1, 2).clone()).add_(torch.eye(d, device="cuda"))
        else:
            s["F"] = torch.zeros((E, d, d), device="cuda")
        if own:
            from paper_1811_12019_amd import binding as kb
            s["plan"] = kb.ExpertFactors(R, E, dim, s["x"].dtype, has_bias=case["bias"])
        return s
    T, K, E = case["tokens"], case["choices"], case["experts"]
    s["expert"], s["weights"] = _routing(case, T, K, g)
    s["experts"] = E
    if kind == "sort":
        s["offsets"] = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
        s["order"] = torch.zeros(T * K, dtype=torch.int32, device="cuda")
        s["place"] = torch.zeros((T, K), dtype=torch.int32, device="cuda")
    else:
        s["offsets"], s["order"], s["place"] = _sorted(s["expert"], E)
        dim = case["dim"]
        rows, tokens = (T * K, dim), (T, dim)
        dtype = DTYPES[case["dtype"]]
        if kind == "dispatch":
            s["x"], s["xs"] = _rows(case, g, *tokens), torch.zeros(rows, dtype=dtype, device="cuda")
        else:
            s["ys"] = _rows(case, g, *rows)
            s["y"] = torch.zeros(tokens, dtype=dtype, device="cuda")
        if kind == "combine_back":
            s["dy"] = _rows(case, g, *tokens, scale=0.1)
            s["dys"], s["dweights"] = torch.zeros(rows, dtype=dtype, device="cuda"), torch.zeros((T, K), device="cuda")
    if own:
        from paper_1811_12019_amd import binding as kb
        s["route"] = kb.ExpertRoute(T, K, E, offsets=s["offsets"], order=s["order"], place=s["place"])
    return s


def _sizes(case):
    """The tensors' sizes: few large ones and many small ones, odd ones among them, `elements` in all."""
    n, total = case["tensors"], case["elements"]
    share = [1.0 / (1 + i % 7) ** 2 for i in range(n)]
    whole = sum(share)
    sizes = [max(1, int((total - n) * v / whole)) for v in share]
    sizes[0] += total - sum(sizes)
    return sizes


def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    from paper_1811_12019_amd import binding as kb
    kind = s["kind"]
    if kind == "sort":
        kb.kfac_expert_sort(s["route"], s["expert"])
        return {"offsets": s["offsets"], "order": s["order"], "place": s["place"]}
    if kind == "dispatch":
        kb.kfac_expert_dispatch(s["route"], s["x"], s["xs"])
        return s["xs"]
    if kind == "dispatch_back":
        kb.kfac_expert_combine(s["route"], s["ys"], None, s["y"])
        return s["y"]
    if kind == "combine":
        kb.kfac_expert_combine(s["route"], s["ys"], s["weights"], s["y"])
        return s["y"]
    if kind == "combine_back":
        kb.kfac_expert_combine_backward(s["route"], s["dy"], s["ys"], s["weights"], s["dys"], s["dweights"])
        return {"dys": s["dys"], "dweights": s["dweights"]}
    if kind == "factor":
        if s["ema"]:
            kb.kfac_expert_factor(s["plan"], s["x"], s["offsets"], running=s["F"], decay=DECAY)
        else:
            kb.kfac_expert_factor(s["plan"], s["x"], s["offsets"], out=s["F"])
        return s["F"]
    norm = kb.kfac_grad_clip_batched(s["batch"], s["max_norm"])
    return {"norm": norm, "out": s["out"]}


def _plain(s):
    kind = s["kind"]
    if kind == "sort":
        s["offsets"], s["order"], s["place"] = _sorted(s["expert"], s["experts"])
        return {"offsets": s["offsets"], "order": s["order"], "place": s["place"]}
    if kind == "dispatch":
        token = s["order"].clamp(min=0) // s["place"].shape[1]
        s["xs"] = torch.where((s["order"] >= 0)[:, None], s["x"][token], s["xs"])
        return s["xs"]
    if kind in ("combine", "dispatch_back"):
        there = (s["place"] >= 0)[:, :, None]
        terms = torch.where(there, s["ys"][s["place"].clamp(min=0)].float(), 0)
        if kind == "combine":
            terms = torch.where(there, terms * s["weights"][:, :, None], 0)
        return terms.sum(1).to(s["ys"].dtype)
    if kind == "combine_back":
        there = s["place"] >= 0
        dy = s["dy"].float()
        rows = s["order"].clamp(min=0)
        dys = dy[rows // s["place"].shape[1]] * s["weights"].reshape(-1)[rows][:, None]
        s["dys"] = torch.where((s["order"] >= 0)[:, None], dys.to(s["dys"].dtype), s["dys"])
        dots = (s["ys"][s["place"].clamp(min=0)].float() * dy[:, None, :]).sum(2)
        return {"dys": s["dys"], "dweights": torch.where(there, dots, 0)}
    if kind == "factor":
        fresh = torch.stack([_mean_square(s["x"][a:b], s["bias"]) for a, b in zip(s["bounds"], s["bounds"][1:])])
        if not s["ema"]:
            return fresh
        there = (s["offsets"][1:] > s["offsets"][:-1])[:, None, None]
        s["F"] = torch.where(there, DECAY * s["F"] + (1 - DECAY) * fresh, s["F"])
        return s["F"]
    norm = s["flat"].double().square().sum().sqrt().float()
    scale = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)
    return {"norm": norm, "out": (s["flat"].float() * scale).to(s["flat"].dtype)}


def _mean_square(rows, bias):
    a = rows.float()
    if bias:
        a = torch.cat([a, a.new_ones((a.shape[0], 1))], dim=1)
    return a.t().matmul(a) / max(1, a.shape[0])


def work(case):
    size = 4 if case.get("dtype", "f32") == "f32" else 2
    kind = case["kind"]
    if kind == "clip":
        return {"bytes": 2 * case["elements"] * size + 4, "flops": 3 * case["elements"]}
    if kind == "factor":
        d, keep = case["dim"] + int(case["bias"]), 1 - case["drop"]
        out = 4 * case["experts"] * d * d * (2 if case["ema"] else 1)
        return {"bytes": keep * case["rows"] * case["dim"] * size + out, "flops": keep * case["rows"] * d * (d + 1)}
    T, K = case["tokens"], case["choices"]
    if kind == "sort":
        return {"bytes": 4 * (3 * T * K + case["experts"] + 1), "flops": 0}
    rows = (1 - case["drop"]) * T * K * case["dim"]
    one = T * case["dim"]
    if kind == "combine_back":
        return {"bytes": size * (one + 2 * rows) + 12 * T * K, "flops": 3 * rows}
    weights = 4 * T * K if kind == "combine" else 0
    return {"bytes": size * (one + rows) + 4 * T * K + weights, "flops": 0 if kind == "dispatch" else (2 if kind == "combine" else 1) * rows}


def exact(case, seed):
    kind = case["kind"]
    if kind == "sort":
        return None
    s = prepare(case, seed)
    if kind == "clip":
        g = s["flat"].to(torch.float64)
        norm = torch.linalg.vector_norm(g)
        return {"norm": norm, "out": g.mul_(min(1.0, s["max_norm"] / float(norm)))}
    if kind == "factor":
        new = torch.zeros_like(s["F"], dtype=torch.float64)
        for e, (a, b) in enumerate(zip(s["bounds"], s["bounds"][1:])):
            if b == a:
                new[e] = s["F"][e] if s["ema"] else 0
                continue
            x = s["x"][a:b].double()
            d = x.shape[1]
            new[e, :d, :d] = torch.mm(x.t().contiguous(), x) / (b - a)
            if s["bias"]:
                new[e, d, :d] = new[e, :d, d] = x.mean(0)
                new[e, d, d] = 1
            if s["ema"]:
                new[e] = s["F"][e].double() * DECAY + new[e] * (1 - DECAY)
        return new
    T, K = s["place"].shape
    rows = torch.nonzero(s["order"] >= 0).reshape(-1)
    token, choice = s["order"][rows].long() // K, s["order"][rows].long() % K
    weights = s["weights"].double()[token, choice]
    if kind == "dispatch":
        xs = torch.zeros(s["xs"].shape, dtype=torch.float64, device="cuda")
        xs[rows] = s["x"].double()[token]
        return xs
    if kind == "combine_back":
        dys = torch.zeros(s["dys"].shape, dtype=torch.float64, device="cuda")
        dweights = torch.zeros((T, K), dtype=torch.float64, device="cuda")
        dy = s["dy"].double()[token]
        dys[rows] = dy * weights[:, None]
        dweights[token, choice] = torch.linalg.vecdot(dy, s["ys"].double()[rows])
        return {"dys": dys, "dweights": dweights}
    y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
    terms = s["ys"].double()[rows]
    return y.index_add_(0, token, terms * weights[:, None] if kind == "combine" else terms)
