"""Cases for the operators of an expert layer: routing, the product in 8-bit integers, and the exchange of rows.

An expert layer sends every token to a few of many weight matrices ("experts"). Three operators make it up, next to the
AllToAllv that moves rows between ranks:

  route     scores of T tokens for E experts, the choice of the top k, their weights, and the layout of the rows in
            expert order (which row of the exchanged buffer belongs to which token); backward: gradient of the scores
  product   y = x W^T with W in 8-bit integers and a scale for each output channel, x quantised within the call with a
            scale for each token; one weight matrix, or one for each expert over rows that are gathered in expert order
  exchange  dispatch: rows in expert order from tokens; combine: the weighted sum of a token's rows; and both gradients

`own` selects between the plain form (elementary torch operations in 32 bits) and the framework's kernels.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
GAP = 1e-6  # smallest distance between two keys on which a choice may hang (32-bit scores are good to about 1e-7)


# ---------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one new token of a served sequence: sigmoid scores, a bias for balance, 4 of 8 groups, renormalised weights
        dict(name="route_one_token", op="route", T=1, E=256, k=8, score="sigmoid", bias=True, groups=8, top_groups=4, renorm=True, scale=2.5, dtype="fp32", pad=0),
        # a small decode batch with padded places, odd sizes, softmax scores as they are
        dict(name="route_decode_batch", op="route", T=61, E=60, k=4, score="softmax", bias=False, groups=1, top_groups=1, renorm=False, scale=1.0, dtype="bf16", pad=5),
        # a long prompt, or many at once
        dict(name="route_prompt", op="route", T=16384, E=256, k=8, score="sigmoid", bias=True, groups=8, top_groups=4, renorm=True, scale=2.5, dtype="bf16", pad=0),
        # a training step's gradient of the scores
        dict(name="route_grad_training", op="route_grad", T=32768, E=128, k=8, score="softmax", bias=False, groups=1, top_groups=1, renorm=True, scale=1.0, dtype="bf16", pad=0),
        # one new token through a dense layer: the weights are read once, and that is the time
        dict(name="product_one_token", op="product", T=1, K=4096, N=8192, E=0, k=0, dtype="bf16"),
        # a prompt of odd length through a layer of odd width
        dict(name="product_ragged", op="product", T=997, K=2064, N=4104, E=0, k=0, dtype="fp16"),
        # the largest: a batch of prompts through a square layer
        dict(name="product_prompts", op="product", T=8192, K=8192, N=8192, E=0, k=0, dtype="bf16"),
        # a decode batch over 64 experts: a few rows for each, all the weights
        dict(name="product_experts_decode", op="product", T=64, K=4096, N=2048, E=64, k=8, dtype="bf16"),
        # prompts over 64 experts: about a thousand rows for each, unevenly
        dict(name="product_experts_prompts", op="product", T=8192, K=4096, N=2048, E=64, k=8, dtype="bf16"),
        # a decode batch's rows come back to their tokens
        dict(name="combine_decode", op="combine", T=32, H=4096, E=64, k=8, dtype="bf16", pad=0),
        # prompts' rows go out in expert order
        dict(name="dispatch_prompts", op="dispatch", T=8192, H=4096, E=64, k=8, dtype="bf16", pad=0),
        # a training step: gradients of the experts' rows and of the weights, odd sizes
        dict(name="combine_grad_training", op="combine_grad", T=4099, H=2056, E=60, k=6, dtype="bf16", pad=3),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["route", "route", "route_grad", "product", "product", "product", "dispatch", "dispatch_grad", "combine", "combine_grad"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("route", "route_grad"):
        groups = rng.choice([1, 1, 4, 8])
        E = groups * rng.randint(max(2, 8 // groups), 384 // groups)
        top_groups = groups if groups == 1 else rng.randint(2, groups // 2 + 1)
        k = rng.randint(1, min(8, E // groups * top_groups))
        score = rng.choice(["softmax", "sigmoid"])
        T = _log(rng, 1, 32768 * 128 // max(E, 128))
        return dict(op=op, T=T, E=E, k=k, score=score, bias=score == "sigmoid", groups=groups, top_groups=top_groups,
                    renorm=rng.random() < 0.6, scale=rng.choice([1.0, 2.5]), dtype=dtype, pad=rng.choice([0, 0, T // 7]))
    if op == "product":
        T, K, N = _log(rng, 1, 8192), 16 * _log(rng, 8, 512), 8 * _log(rng, 16, 1024)
        if rng.random() < 0.5:
            return dict(op=op, T=T, K=K, N=N, E=0, k=0, dtype=dtype)
        E, k = rng.choice([8, 16, 60, 64, 128]), rng.randint(1, 8)
        while E * N * K > 64 * 4096 * 2048:
            N, K = max(128, N // 16 * 8), max(128, K // 32 * 16)
        while T * k * N * K > 8192 * 8 * 4096 * 2048:
            T = max(1, T // 2)
        return dict(op=op, T=T, K=K, N=N, E=E, k=k, dtype=dtype)
    E = rng.choice([8, 16, 60, 64, 128, 256])
    T, k, H = _log(rng, 1, 8192), rng.randint(1, 8), rng.choice([1, 8]) * _log(rng, 32, 512)
    return dict(op=op, T=T, H=H, E=E, k=k, dtype=dtype, pad=rng.choice([0, 0, T // 7]))


# ---------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _exact_keys(logits, bias, case):
    """Keys of the choice in 64 bits, experts of the groups that are not chosen at -inf, and the smallest distance that the choice hangs on."""
    x = logits.double()
    key = torch.sigmoid(x) if case["score"] == "sigmoid" else x
    if bias is not None:
        key = key + bias.double()
    T, E = x.shape
    gap = torch.full((T,), math.inf, dtype=torch.float64, device=x.device)
    G = case["groups"]
    if G > 1:
        per = key.view(T, G, E // G)
        n = min(2 if case["score"] == "sigmoid" else 1, E // G)
        gs, order = per.topk(n, dim=-1).values.sum(-1).sort(dim=-1, descending=True, stable=True)
        gap = torch.minimum(gap, (gs[:, :-1] - gs[:, 1:]).amin(-1))
        keep = torch.zeros(T, G, dtype=torch.bool, device=x.device).scatter_(1, order[:, : case["top_groups"]], True)
        key = key.masked_fill(~keep.repeat_interleave(E // G, dim=1), -math.inf)
    top = key.topk(min(case["k"] + 1, E), dim=-1).values
    if top.shape[1] > 1:
        d = top[:, :-1] - top[:, 1:]
        gap = torch.minimum(gap, torch.where(torch.isnan(d), math.inf, d).amin(-1))
    return key, gap


def _logits(case, seed):
    """Scores before the softmax or sigmoid: some experts are more popular than others. Where the choice goes by 32-bit
    scores, rows in which it hangs on less than their rounding are drawn again: who wins there is no property of the operator."""
    g = _gen(seed)
    T, E, dt = case["T"], case["E"], DTYPES[case["dtype"]]
    popular = 0.5 * torch.randn(E, device="cuda", generator=g)
    logits = (torch.randn(T, E, device="cuda", generator=g) + popular).to(dt)
    bias = None
    if case["bias"]:  # a balance bias moves in steps of 0.001, against the popularity
        bias = (-50 * popular + 20 * torch.randn(E, device="cuda", generator=g)).round() * 0.001
    if case["score"] == "sigmoid":
        for _ in range(20):
            bad = (_exact_keys(logits, bias, case)[1] < GAP).nonzero().flatten()
            if bad.numel() == 0:
                break
            logits[bad] = (torch.randn(bad.numel(), E, device="cuda", generator=g) + popular).to(dt)
    mask = None
    if case.get("pad", 0):
        mask = torch.ones(T, dtype=torch.uint8, device="cuda")
        mask[T - case["pad"]:] = 0
    return logits, bias, mask


def _route_case(case):
    """The routing in front of a product or an exchange: plain softmax, top k, renormalised."""
    return dict(T=case["T"], E=case["E"], k=case["k"], score="softmax", bias=False, groups=1, top_groups=1, renorm=True, scale=1.0,
                dtype="fp32", pad=case.get("pad", 0))


def _rand(g, shape, dt, scale=1.0):
    return (torch.randn(shape, device="cuda", generator=g) * scale).to(dt)


def _weights_i8(g, shape):
    """Weights as they are stored: 8-bit integers with a scale for each output channel."""
    w = (torch.randn(shape, device="cuda", generator=g) * 36).round_().clamp_(-127, 127).to(torch.int8)
    s = (0.5 + torch.rand(shape[:-1], device="cuda", generator=g)) * (0.02 / 36)
    return w, s


def _inputs(case, seed):
    op, dt = case["op"], DTYPES.get(case["dtype"])
    if op in ("route", "route_grad"):
        logits, bias, mask = _logits(case, seed)
        s = dict(logits=logits, bias=bias, mask=mask)
        if op == "route_grad":
            s["routing"] = _plain_route(case, logits, bias, mask)
            s["dweights"] = torch.randn(case["T"], case["k"], device="cuda", generator=_gen(seed + 1))
        return s
    g = _gen(seed + 1)
    s = {}
    if case["E"]:
        rc = _route_case(case)
        s["routing"] = _plain_route(rc, *_logits(rc, seed))
    if op == "product":
        T, K, N, E = case["T"], case["K"], case["N"], case["E"]
        s["x"] = _rand(g, (T, K), dt)
        s["w"], s["ws"] = _weights_i8(g, (E, N, K) if E else (N, K))
        return s
    T, H = case["T"], case["H"]
    if op == "dispatch":
        s["x"] = _rand(g, (T, H), dt)
    else:
        s["rows"] = _rand(g, (T * case["k"], H), dt)
        if op == "combine_grad":
            s["dy"] = _rand(g, (T, H), dt, 0.05)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op = case["op"]
    if own:
        from paper_2608_00358_b200 import experts as ex
        if op in ("route", "route_grad"):
            s["router"] = ex.Router(case["E"], case["k"], score=case["score"], groups=case["groups"], top_groups=case["top_groups"],
                                    group_best=2 if case["score"] == "sigmoid" else 1, renormalise=case["renorm"], scale=case["scale"])
            s["out"] = s["router"].outputs(case["T"])
        if "routing" in s:
            r = s["routing"]
            s["plan"] = ex.Routing(*r)
        if op == "product":
            s["linear"] = ex.Int8Linear(s["w"], s["ws"])
            s["y"] = torch.empty(case["T"] * max(case["k"], 1), case["N"], dtype=s["x"].dtype, device="cuda")
        if op in ("dispatch", "combine_grad"):
            s["rows_out"] = torch.empty(case["T"] * case["k"], case["H"], dtype=DTYPES[case["dtype"]], device="cuda")
    elif op == "product" and case["E"]:
        s["offsets_host"] = s["routing"][3].tolist()  # the plain form calls torch once for each expert
    return s


# ---------------------------------------------------------------------------------------------------- plain forms
def _plain_scores(case, logits):
    x = logits.float()
    if case["score"] == "sigmoid":
        return 1 / (1 + torch.exp(-x))
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _plain_layout(ids, E):
    """Rows in expert order, tokens in order within an expert; a place without an expert (-1) has no row."""
    flat = ids.flatten().long()
    n = flat.numel()
    counts = torch.zeros(E + 1, dtype=torch.int64, device=ids.device).scatter_add_(0, torch.where(flat < 0, E, flat), torch.ones_like(flat))
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=ids.device)
    offsets[1:] = counts[:E].cumsum(0)
    order = torch.where(flat < 0, E, flat).sort(stable=True).indices
    at = torch.arange(n, device=ids.device)
    slots = torch.empty_like(flat)
    slots[order] = at
    slots = torch.where(flat < 0, -1, slots)
    source = torch.where(at < offsets[E], order, -1)
    return counts[:E], offsets.int(), slots.int().view(ids.shape), source.int()


def _plain_route(case, logits, bias, mask):
    T, E, G, k = case["T"], case["E"], case["groups"], case["k"]
    s = _plain_scores(case, logits)
    key = s if bias is None else s + bias
    if case["score"] == "softmax":
        key = logits.float()  # the softmax keeps the order of its arguments: no choice hangs on how it was rounded
    if G > 1:
        n = min(2 if case["score"] == "sigmoid" else 1, E // G)
        best = key.view(T, G, E // G).sort(dim=-1, descending=True, stable=True).values[..., :n].sum(-1)
        order = best.sort(dim=-1, descending=True, stable=True).indices[:, : case["top_groups"]]
        keep = torch.zeros(T, G, dtype=torch.bool, device=key.device).scatter_(1, order, True)
        key = torch.where(keep.repeat_interleave(E // G, dim=1), key, -math.inf)
    ids = key.sort(dim=-1, descending=True, stable=True).indices[:, :k]
    w = s.gather(1, ids)
    if case["renorm"]:
        w = w / w.sum(-1, keepdim=True)
    w = w * case["scale"]
    ids = ids.int()
    if mask is not None:
        ids = torch.where(mask[:, None] != 0, ids, -1)
        w = torch.where(mask[:, None] != 0, w, 0.0)
    counts, offsets, slots, source = _plain_layout(ids, E)
    return ids, w, counts, offsets, slots, source


def _plain_route_grad(case, logits, mask, routing, dweights):
    s = _plain_scores(case, logits)
    ids = routing[0].clamp(min=0).long()
    live = routing[0] >= 0
    dw = torch.where(live, dweights, 0.0) * case["scale"]
    c = s.gather(1, ids)
    if case["renorm"]:
        total = c.sum(-1, keepdim=True)
        dw = (dw - (dw * c).sum(-1, keepdim=True) / total) / total
    if case["score"] == "sigmoid":
        d = torch.zeros_like(s).scatter_add_(1, ids, torch.where(live, dw * c * (1 - c), 0.0))
    else:
        g = torch.zeros_like(s).scatter_add_(1, ids, torch.where(live, dw, 0.0))
        d = s * (g - (g * s).sum(-1, keepdim=True))
    if mask is not None:
        d = torch.where(mask[:, None] != 0, d, 0.0)
    return d.to(logits.dtype)


def _plain_quantise(x):
    x = x.float()
    amax = x.abs().amax(-1, keepdim=True)
    q = torch.round(x * torch.where(amax > 0, 127 / amax, 0.0)).clamp(-127, 127)
    return q, amax / 127


def _plain_product(s):
    q, sx = _plain_quantise(s["x"])
    if "offsets_host" not in s:
        return ((q @ s["w"].float().t()) * sx * s["ws"]).to(s["x"].dtype)
    off, token = s["offsets_host"], (s["routing"][5] // s["case"]["k"]).long()
    y = torch.empty(token.numel(), s["w"].shape[1], dtype=s["x"].dtype, device=q.device)
    for e in range(len(off) - 1):
        if off[e + 1] > off[e]:
            t = token[off[e]: off[e + 1]]
            y[off[e]: off[e + 1]] = ((q[t] @ s["w"][e].float().t()) * sx[t] * s["ws"][e]).to(y.dtype)
    return y


def _plain_exchange(s):
    case, (ids, w, _, _, slots, source) = s["case"], s["routing"]
    T, k = slots.shape
    at, live = slots.clamp(min=0).long(), (slots >= 0)
    op = case["op"]
    if op == "dispatch":
        return torch.where((source >= 0)[:, None], s["x"][source.clamp(min=0).long() // k], 0.0).to(s["x"].dtype)
    rows = s["rows"]
    got = torch.where(live[..., None], rows[at.flatten()].view(T, k, -1).float(), 0.0)
    if op == "dispatch_grad":
        return got.sum(1).to(rows.dtype)
    if op == "combine":
        return (got * w[..., None]).sum(1).to(rows.dtype)
    dw = (got * s["dy"].float()[:, None]).sum(-1)
    src = source.clamp(min=0).long()
    drows = torch.where((source >= 0)[:, None], w.flatten()[src][:, None] * s["dy"].float()[src // k], 0.0).to(rows.dtype)
    return drows, dw


# ---------------------------------------------------------------------------------------------------- one pass
def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if own:
        from paper_2608_00358_b200 import experts as ex
        if op == "route":
            r = s["router"].route(s["logits"], bias=s["bias"], token_mask=s["mask"], out=s["out"])
            return r.ids, r.weights, r.counts, r.offsets, r.slots, r.source
        if op == "route_grad":
            return s["router"].backward(s["logits"], s["plan"], s["dweights"], bias=s["bias"], token_mask=s["mask"])
        if op == "product":
            return s["linear"](s["x"], routing=s.get("plan"), out=s["y"])
        if op == "dispatch":
            return ex.dispatch(s["x"], s["plan"], out=s["rows_out"])
        if op == "dispatch_grad":
            return ex.dispatch_backward(s["rows"], s["plan"])
        if op == "combine":
            return ex.combine(s["rows"], s["plan"])
        return ex.combine_backward(s["dy"], s["rows"], s["plan"], out=s["rows_out"])
    if op == "route":
        return _plain_route(case, s["logits"], s["bias"], s["mask"])
    if op == "route_grad":
        return _plain_route_grad(case, s["logits"], s["mask"], s["routing"], s["dweights"])
    if op == "product":
        return _plain_product(s)
    return _plain_exchange(s)


def work(case):
    op, T, E, k = case["op"], case["T"], case["E"], case["k"]
    es = BYTES[case["dtype"]]
    if op == "route":  # scores in; ids, weights, slots, source, counts and offsets out
        return dict(bytes=T * E * es + T * k * 16 + E * (16 if case["bias"] else 12), flops=6 * T * E)
    if op == "route_grad":
        return dict(bytes=2 * T * E * es + T * k * 8, flops=8 * T * E)
    if op == "product":
        K, N = case["K"], case["N"]
        rows = T * max(k, 1)
        used = E * (1 - (1 - 1 / E) ** rows) if E else 1  # an expert without rows need not be read
        return dict(bytes=int(T * K * es + used * N * (K + 4) + rows * N * es + (rows * 4 if E else 0)), flops=2 * rows * K * N)
    H, n = case["H"], T * k
    if op == "dispatch":
        return dict(bytes=(T + n) * H * es + n * 4, flops=T * H)
    if op == "combine":
        return dict(bytes=(T + n) * H * es + n * 8, flops=2 * n * H)
    if op == "dispatch_grad":
        return dict(bytes=(T + n) * H * es + n * 4, flops=n * H)
    return dict(bytes=(T + 2 * n) * H * es + n * 12, flops=3 * n * H)


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _exact_route(case, logits, bias, mask):
    T, E, k = case["T"], case["E"], case["k"]
    key = _exact_keys(logits, bias, case)[0]
    ids = torch.empty(T, k, dtype=torch.int64, device=key.device)
    key = key.clone()
    for j in range(k):  # the first of the largest, k times over
        ids[:, j] = (key == key.amax(-1, keepdim=True)).int().argmax(-1)
        key.scatter_(1, ids[:, j: j + 1], -math.inf)
    x = logits.double()
    s = torch.sigmoid(x) if case["score"] == "sigmoid" else torch.softmax(x, -1)
    w = s.gather(1, ids)
    if case["renorm"]:
        w = w / w.sum(-1, keepdim=True)
    w = w * case["scale"]
    if mask is not None:
        ids[mask == 0] = -1
        w[mask == 0] = 0
    flat = ids.flatten().cpu().numpy()
    source = np.concatenate([np.nonzero(flat == e)[0] for e in range(E)] + [np.full(int((flat < 0).sum()), -1)])
    slots = np.full(flat.shape, -1)
    n = int((flat >= 0).sum())
    slots[source[:n]] = np.arange(n)
    counts = np.array([(flat == e).sum() for e in range(E)], dtype=np.int64)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    as_i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
    return ids.int(), w, torch.from_numpy(counts).cuda(), as_i32(offsets), as_i32(slots).view(T, k), as_i32(source)


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "route":
        return _exact_route(case, s["logits"], s["bias"], s["mask"])
    if op == "route_grad":
        x = s["logits"].double().requires_grad_()
        p = torch.sigmoid(x) if case["score"] == "sigmoid" else torch.softmax(x, -1)
        ids = s["routing"][0].long()
        w = p.gather(1, ids.clamp(min=0))
        if case["renorm"]:
            w = w / w.sum(-1, keepdim=True)
        (w * case["scale"] * s["dweights"].double() * (ids >= 0)).sum().backward()
        return x.grad
    if op == "product":
        x = s["x"].double()
        amax = x.abs().amax(-1, keepdim=True)
        q = torch.round(x * 127 / amax.clamp(min=1e-300)).clamp(-127, 127)
        sx = amax / 127
        if not case["E"]:
            return (q @ s["w"].double().t()) * sx * s["ws"].double()
        ids = s["routing"][0].flatten()
        y = torch.zeros(ids.numel(), case["N"], dtype=torch.float64, device="cuda")
        at = 0
        for e in range(case["E"]):
            t = (ids == e).nonzero().flatten() // case["k"]
            y[at: at + t.numel()] = (q[t] @ s["w"][e].double().t()) * sx[t] * s["ws"][e].double()
            at += t.numel()
        return y
    ids, w, _, _, slots, _ = s["routing"]
    T, k = slots.shape
    t, j = (slots >= 0).nonzero(as_tuple=True)
    at = slots[t, j].long()
    if op == "dispatch":
        y = torch.zeros(T * k, case["H"], dtype=torch.float64, device="cuda")
        y[at] = s["x"].double()[t]
        return y
    rows = s["rows"].double()
    y = torch.zeros(T, case["H"], dtype=torch.float64, device="cuda")
    if op in ("combine", "dispatch_grad"):
        f = w.double() if op == "combine" else torch.ones_like(w, dtype=torch.float64)
        for c in range(k):
            here = slots[:, c] >= 0
            y[here] += f[here, c, None] * rows[slots[here, c].long()]
        return y
    dy = s["dy"].double()
    drows = torch.zeros_like(rows)
    drows[at] = w.double()[t, j, None] * dy[t]
    dw = torch.zeros(T, k, dtype=torch.float64, device="cuda")
    dw[t, j] = (dy[t] * rows[at]).sum(-1)
    return drows, dw
