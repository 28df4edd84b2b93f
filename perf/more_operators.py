"""Cases for an expert layer in 4-bit floating point, and for what stands between its two products in training.

  round      rows to 4-bit floating point in small blocks with a scale each, and back to the values that they stand for
  product    y = x W^T with W in such blocks, x quantised within the call; one weight matrix, or one for each expert over
             rows that are gathered in expert order
  layer      a whole expert layer for a few tokens: the chosen experts' gated products and their weighted sum. The
             weights are in 4 bits, the activations are not rounded: with few tokens the weights are what is read
  activate   the gated activation of rows in expert order with dropout, whose mask comes from a counter-based generator
             and is never stored; backward: gradient of the gate's and of the other half

Formats. "nvfp4": blocks of 16, s = e4m3(max|x| / (6 g)) with a 32-bit scale g for the whole matrix, step d = s g.
"mxfp4": blocks of 32, d = 2^e with the least whole e at which nothing saturates. q = e2m1(x / d), ties to even.

`own` selects between the plain form (elementary torch operations in 32 bits) and the framework's kernels.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
BLOCK = {"nvfp4": 16, "mxfp4": 32}


# ---------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a decode batch's rows on their way out in a quarter of the bytes
        dict(name="round_decode", op="round", M=48, K=4096, E=0, k=0, format="nvfp4", dtype="bf16"),
        # a prompt of odd length and width
        dict(name="round_ragged", op="round", M=1999, K=2057, E=0, k=0, format="mxfp4", dtype="fp32"),
        # prompts' rows in expert order, each token read once and written to four places
        dict(name="round_prompts_to_experts", op="round", M=8192, K=4096, E=64, k=4, format="nvfp4", dtype="bf16"),
        # one new token through a dense layer: the weights are read once, and that is the time
        dict(name="product_one_token", op="product", T=1, K=4096, N=8192, E=0, k=0, format="nvfp4", dtype="bf16", bias=False),
        # a prompt of odd length through a layer of odd width, with a bias
        dict(name="product_ragged", op="product", T=997, K=2064, N=4104, E=0, k=0, format="mxfp4", dtype="fp16", bias=True),
        # the largest: a batch of prompts through a square layer
        dict(name="product_prompts", op="product", T=8192, K=8192, N=8192, E=0, k=0, format="nvfp4", dtype="bf16", bias=False),
        # prompts over 64 experts, about a thousand rows for each, unevenly
        dict(name="product_experts_prompts", op="product", T=8192, K=4096, N=2048, E=64, k=8, format="nvfp4", dtype="bf16", bias=False),
        # one new token through 8 of 64 experts
        dict(name="layer_one_token", op="layer", T=1, H=4096, I=2048, E=64, k=8, format="nvfp4", dtype="bf16"),
        # a decode batch, odd sizes
        dict(name="layer_decode_batch", op="layer", T=19, H=2056, I=1416, E=60, k=4, format="mxfp4", dtype="bf16"),
        # a small training step of odd sizes, some rows behind the last expert's
        dict(name="activate_ragged", op="activate", M=1003, I=1410, p=0.1, act="gelu", pad=21, dtype="fp32"),
        # training: rows in expert order of a long batch
        dict(name="activate_training", op="activate", M=32768, I=2048, p=0.1, act="silu", pad=0, dtype="bf16"),
        # their gradient
        dict(name="activate_grad_training", op="activate_grad", M=32768, I=2048, p=0.1, act="silu", pad=0, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["round", "round", "product", "product", "product", "layer", "layer", "activate", "activate_grad"])
    dtype, fmt = rng.choice(["bf16", "bf16", "fp16", "fp32"]), rng.choice(["nvfp4", "nvfp4", "mxfp4"])
    if op == "round":
        K = rng.choice([1, 1, 8, 32]) * _log(rng, 64, 256)
        k = rng.choice([0, 0, rng.randint(1, 4)])
        return dict(op=op, M=_log(rng, 1, 8192), K=K, E=rng.choice([8, 60, 128]) if k else 0, k=k, format=fmt, dtype=dtype)
    if op == "product":
        T, K, N = _log(rng, 1, 8192), rng.choice([1, 8, 8, 32, 32]) * _log(rng, 64, 256), rng.choice([1, 8, 8]) * _log(rng, 32, 1024)
        bias = rng.random() < 0.3
        if rng.random() < 0.5:
            return dict(op=op, T=T, K=K, N=N, E=0, k=0, format=fmt, dtype=dtype, bias=bias)
        E, k = rng.choice([8, 16, 60, 64, 128]), rng.randint(1, 8)
        while E * N * K > 64 * 4096 * 2048:
            N, K = max(128, N // 16 * 8), max(128, K // 32 * 16)
        while T * k * N * K > 8192 * 8 * 4096 * 2048:
            T = max(1, T // 2)
        return dict(op=op, T=T, K=K, N=N, E=E, k=k, format=fmt, dtype=dtype, bias=bias)
    if op == "layer":
        E, k = rng.choice([8, 16, 60, 64]), rng.randint(1, 8)
        return dict(op=op, T=_log(rng, 1, 48), H=8 * _log(rng, 32, 512), I=rng.choice([1, 8, 16]) * _log(rng, 100, 128), E=E, k=k, format=fmt, dtype=dtype)
    M, I = _log(rng, 1, 32768), rng.choice([1, 8, 16]) * _log(rng, 64, 128)
    return dict(op=op, M=M, I=I, p=rng.choice([0.0, 0.1, 0.25]), act=rng.choice(["silu", "silu", "gelu", "relu"]), pad=rng.choice([0, 0, M // 9]),
                dtype="bf16" if dtype == "fp32" and M * I > 1 << 24 else dtype)


# ---------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rand(g, shape, dt, scale=1.0):
    """Activations: normal, with a few columns that are much larger than the others."""
    x = torch.randn(shape, device="cuda", generator=g)
    x *= scale * torch.where(torch.rand(shape[-1], device="cuda", generator=g) < 0.01, 8.0, 1.0)
    return x.to(dt)


def _routing(g, T, E, k):
    """Some experts are more popular than others; weights are a softmax over the chosen. (ids, weights, counts, offsets, slots, source)"""
    score = torch.randn(T, E, device="cuda", generator=g) + 0.5 * torch.randn(E, device="cuda", generator=g)
    top = score.topk(k, dim=-1)
    ids, weights = top.indices.int(), torch.softmax(top.values, -1)
    flat = top.indices.flatten()
    source = flat.sort(stable=True).indices
    slots = torch.empty_like(source)
    slots[source] = torch.arange(T * k, device="cuda")
    counts = torch.bincount(flat, minlength=E)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0)
    return ids, weights, counts, offsets, slots.int().view(T, k), source.int()


# Of 256 elements of a normal matrix whose blocks' largest map to 6: how many have each magnitude
_OFTEN = (31, 59, 51, 38, 38, 20, 13, 6)


def _weights_fp4(g, shape, fmt):
    """Weights as they are stored: two codes to a byte (the earlier in the low half), a byte for each block's scale, and a 32-bit scale for
    each matrix."""
    *lead, K = shape
    table = torch.tensor([c for c, often in enumerate(_OFTEN) for _ in range(often)], dtype=torch.uint8, device="cuda")
    rows = int(math.prod(lead))
    codes = torch.empty((rows, (K + 1) // 2), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // max(K, 1))
    for r in range(0, rows, step):
        n = min(step, rows - r) * ((K + 1) // 2)
        a, b, sign = (torch.randint(256, (n,), device="cuda", generator=g, dtype=torch.int32) for _ in range(3))
        byte = table[a] | (table[b] << 4) | ((sign & 1) << 3).to(torch.uint8) | ((sign & 2) << 6).to(torch.uint8)
        codes[r: r + step] = byte.view(-1, codes.shape[1])
    if K % 2:
        codes[:, -1] &= 15
    blocks = (K + BLOCK[fmt] - 1) // BLOCK[fmt]
    if fmt == "nvfp4":  # the matrix's largest block has the largest scale; most are a few binades below
        scales = torch.randint(104, 122, (rows, blocks), device="cuda", generator=g, dtype=torch.int32).to(torch.uint8)
    else:
        scales = torch.randint(119, 122, (rows, blocks), device="cuda", generator=g, dtype=torch.int32).to(torch.uint8)
    matrices = shape[0] if len(shape) == 3 else 1
    wide = (0.5 + torch.rand(matrices, device="cuda", generator=g)) * (2.0 ** -14 if fmt == "nvfp4" else 1.0)
    if fmt == "mxfp4":
        wide.fill_(1.0)
    return codes.view(*lead, -1), scales.view(*lead, blocks), wide


def _inputs(case, seed):
    op, dt, g = case["op"], DTYPES[case["dtype"]], _gen(seed)
    s = {}
    if op == "round":
        s["x"] = _rand(g, (case["M"], case["K"]), dt)
        s["wide"] = torch.tensor(2.0 ** -6 if case["M"] % 2 else 0.0173, dtype=torch.float32, device="cuda")
        if case["k"]:
            s["routing"] = _routing(g, case["M"], case["E"], case["k"])
    elif op == "product":
        T, K, N, E, fmt = case["T"], case["K"], case["N"], case["E"], case["format"]
        s["x"] = _rand(g, (T, K), dt)
        s["wide"] = torch.tensor(0.0173, dtype=torch.float32, device="cuda")
        s["w"] = _weights_fp4(g, (E, N, K) if E else (N, K), fmt)
        s["bias"] = torch.randn((max(E, 1), N), device="cuda", generator=g) if case["bias"] else None
        if E:
            s["routing"] = _routing(g, T, E, case["k"])
    elif op == "layer":
        T, H, I, E, fmt = case["T"], case["H"], case["I"], case["E"], case["format"]
        s["x"] = _rand(g, (T, H), dt)
        s["up"], s["down"] = _weights_fp4(g, (E, 2 * I, H), fmt), _weights_fp4(g, (E, H, I), fmt)
        s["routing"] = _routing(g, T, E, case["k"])
    else:
        M, I = case["M"], case["I"]
        s["rows"] = (1.5 * torch.randn((M, 2 * I), device="cuda", generator=g)).to(dt)
        s["seed"] = torch.randint(-(1 << 62), 1 << 62, (2,), device="cuda", generator=g)  # the generator's key, and which call of the step it is
        s["offsets"] = torch.tensor([0, M // 3, M - case["pad"]], dtype=torch.int32, device="cuda")
        if op == "activate_grad":
            s["dy"] = (0.05 * torch.randn((M, I), device="cuda", generator=g)).to(dt)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op = case["op"]
    if own:
        from paper_2608_00358_b200 import experts as ex
        from paper_2608_00358_b200 import fp4
        if "routing" in s:
            s["plan"] = ex.Routing(*s["routing"])
        if "wide" in s:
            s["wide"] = float(s["wide"])
        if op == "product":
            s["linear"] = fp4.Fp4Linear(*s["w"], K=case["K"], format=case["format"], bias=s["bias"], x_scale=s["wide"])
        if op == "layer":
            up, down = (fp4.Fp4Linear(*s[n], K=case[K], format=case["format"]) for n, K in (("up", "H"), ("down", "I")))
            s["layer"] = fp4.FewTokens(up, down, act="silu")
        return s
    if "wide" in s:
        s["six"] = 6 * s["wide"]
    if "routing" in s and op != "round":
        s["offsets_host"] = s["routing"][3].tolist()  # the plain form calls torch once for each expert
    return s


# ---------------------------------------------------------------------------------------------------- plain forms
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _blocks(x, n):
    """x in blocks of n along its rows, with zeros behind the last element."""
    K = x.shape[-1]
    if K % n:
        x = torch.nn.functional.pad(x, (0, n - K % n))
    return x.view(*x.shape[:-1], -1, n)


def _two_to(e):
    """2^e in 32 bits, e from -126 to 127."""
    return ((e + 127) << 23).view(torch.float32)


def _steps(x, fmt, wide, six):
    """The step of each block of x [.., blocks, n]."""
    top = x.abs().amax(-1, keepdim=True)
    if fmt == "nvfp4":
        return (top / six).clamp(max=448.0).to(torch.float8_e4m3fn).float() * wide
    m, e = torch.frexp(top)
    return _two_to(torch.where(m > 0.75, e - 2, e - 3).clamp(-126, 127))


def _plain_round(x, fmt, wide, six):
    """The values that the 4-bit form of x stands for, in 32 bits."""
    b = _blocks(x.float(), BLOCK[fmt])
    d = _steps(b, fmt, wide, six)
    a = b.abs() / d  # (a block of zeros has no quotient: its elements compare false below and stay 0)
    code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int())
    v = torch.tensor(_LEVELS, device=x.device)[torch.where(d > 0, code, 0)] * d
    return torch.where(b < 0, -v, v).flatten(-2)[..., : x.shape[-1]]


def _plain_weights(w, fmt, K, e=None):
    """A matrix of weights in 32 bits."""
    codes, scales, wide = w
    if e is not None:
        codes, scales, wide = codes[e], scales[e], wide[e]
    pair = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)[..., :K].int()
    v = torch.tensor(_LEVELS + tuple(-x for x in _LEVELS), device=codes.device)[pair]
    d = scales.view(torch.float8_e4m3fn).float() * wide if fmt == "nvfp4" else _two_to(scales.int() - 127)
    return (_blocks(v, BLOCK[fmt]) * d[..., None]).flatten(-2)[..., :K]


def _plain_product(s):
    case = s["case"]
    fmt, K = case["format"], case["K"]
    q = _plain_round(s["x"], fmt, s["wide"], s["six"])
    if not case["E"]:
        y = q @ _plain_weights(s["w"], fmt, K).t()
        return (y if s["bias"] is None else y + s["bias"]).to(s["x"].dtype)
    off, token = s["offsets_host"], (s["routing"][5] // case["k"]).long()
    y = torch.empty(token.numel(), case["N"], dtype=s["x"].dtype, device=q.device)
    for e in range(case["E"]):
        if off[e + 1] > off[e]:
            o = q[token[off[e]: off[e + 1]]] @ _plain_weights(s["w"], fmt, K, e).t()
            y[off[e]: off[e + 1]] = (o if s["bias"] is None else o + s["bias"][e]).to(y.dtype)
    return y


def _plain_layer(s):
    case, off = s["case"], s["offsets_host"]
    fmt, H, I, k = case["format"], case["H"], case["I"], case["k"]
    _, weights, _, _, slots, source = s["routing"]
    x, token = s["x"].float(), (source // k).long()
    rows = torch.empty(token.numel(), H, device=x.device)
    for e in range(case["E"]):
        if off[e + 1] > off[e]:
            u = x[token[off[e]: off[e + 1]]] @ _plain_weights(s["up"], fmt, H, e).t()
            h = u[:, :I] / (1 + torch.exp(-u[:, :I])) * u[:, I:]
            rows[off[e]: off[e + 1]] = h @ _plain_weights(s["down"], fmt, I, e).t()
    return (rows[slots.long()] * weights[..., None]).sum(1).to(s["x"].dtype)


def _mul_hilo(a, m):
    """High and low half of the 64-bit products of unsigned 32-bit numbers (held in 64-bit integers) with a constant."""
    p = a * (m & 0xFFFF)
    q = a * (m >> 16)  # both below 2^48
    lo = p + ((q & 0xFFFF) << 16)
    return ((q >> 16) + (lo >> 32)) & 0xFFFFFFFF, lo & 0xFFFFFFFF


def _keep(M, I, p, seed):
    """Which elements of [M, I] stay: word i % 4 of Philox-4x32-10 (Salmon and others, 2011) at counter (i // 4, seed[1]) and key seed[0], where
    i = row * I + column; kept from p * 2^32 on."""
    at = torch.arange((M * I + 3) // 4, device=seed.device)
    half = 0xFFFFFFFF
    c = [at & half, at >> 32, (seed[1] & half).expand_as(at), ((seed[1] >> 32) & half).expand_as(at)]
    k0, k1 = seed[0] & half, (seed[0] >> 32) & half
    for _ in range(10):
        h0, l0 = _mul_hilo(c[0], 0xD2511F53)
        h1, l1 = _mul_hilo(c[2], 0xCD9E8D57)
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & half, (k1 + 0xBB67AE85) & half
    return (torch.stack(c, -1).flatten()[: M * I] >= round(p * 2.0 ** 32)).view(M, I)


def _act(g, act):
    """The activation and its derivative."""
    if act == "silu":
        sig = 1 / (1 + torch.exp(-g))
        return g * sig, sig * (1 + g * (1 - sig))
    if act == "gelu":
        phi = 0.5 * (1 + torch.erf(g * 0.5 ** 0.5))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) * (0.5 / math.pi) ** 0.5
    on = (g > 0).to(g.dtype)
    return g * on, on


def _factors(case, s, dt):
    """What dropout multiplies an element with; rows behind the last expert's have 0."""
    M, I = case["M"], case["I"]
    f = torch.full((M, I), 1.0 / (1.0 - case["p"]), dtype=dt, device=s["rows"].device)
    if case["p"] > 0:
        f = torch.where(_keep(M, I, case["p"], s["seed"]), f, 0.0)
    return torch.where((torch.arange(M, device=f.device) < s["offsets"][-1])[:, None], f, 0.0)


def _activate(case, s, dt):
    x, I = s["rows"].to(dt), case["I"]
    a, da = _act(x[:, :I], case["act"])
    f = _factors(case, s, dt)
    if case["op"] == "activate":
        return a * x[:, I:] * f
    dy = s["dy"].to(dt) * f
    return torch.cat((dy * x[:, I:] * da, dy * a), 1)


# ---------------------------------------------------------------------------------------------------- one pass
def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if own:
        from paper_2608_00358_b200 import activation as ac
        from paper_2608_00358_b200 import fp4
        if op == "round":
            return fp4.quantize_rows(s["x"], format=case["format"], scale=s["wide"], routing=s.get("plan")).dequantize(s["x"].dtype)
        if op == "product":
            return s["linear"](s["x"], routing=s.get("plan"))
        if op == "layer":
            return s["layer"](s["x"], s["plan"])
        if op == "activate":
            return ac.activate(s["rows"], act=case["act"], p=case["p"], seed=s["seed"], offsets=s["offsets"])
        return ac.activate_backward(s["dy"], s["rows"], act=case["act"], p=case["p"], seed=s["seed"], offsets=s["offsets"])
    if op == "round":
        v = _plain_round(s["x"], case["format"], s["wide"], s["six"]).to(s["x"].dtype)
        return v[(s["routing"][5] // case["k"]).long()] if case["k"] else v
    if op == "product":
        return _plain_product(s)
    if op == "layer":
        return _plain_layer(s)
    return _activate(case, s, torch.float32).to(s["rows"].dtype)


def work(case):
    op, es = case["op"], BYTES[case["dtype"]]
    if op == "round":  # rows in; the values out
        n = case["M"] * max(case["k"], 1)
        return dict(bytes=(case["M"] + n) * case["K"] * es + n * 4, flops=4 * case["M"] * case["K"])
    if op in ("activate", "activate_grad"):
        n = case["M"] * case["I"]
        return dict(bytes=(3 if op == "activate" else 5) * n * es, flops=(60 if case["p"] else 10) * n)
    E, k, T = case["E"], case["k"], case["T"]
    each = 0.5 + 1 / BLOCK[case["format"]]  # bytes of a weight
    rows = T * max(k, 1)
    used = E * (1 - (1 - k / E) ** T) if E else 1  # an expert without rows need not be read
    if op == "layer":
        weights = 3 * case["H"] * case["I"]
        return dict(bytes=int(used * weights * each + 2 * T * case["H"] * es + rows * 8), flops=2 * rows * weights)
    K, N = case["K"], case["N"]
    return dict(bytes=int(T * K * es + used * N * K * each + rows * N * es + (rows * 4 if E else 0)), flops=2 * rows * K * N)


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _exact_two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_e4m3(v):
    """The nearest number of 1 + 3 bits from 2^-6 on, multiple of 2^-9 below, at most 448; ties to even."""
    v = v.clamp(max=448.0)
    step = _exact_two_to(torch.frexp(v).exponent.clamp(min=-5) - 4)
    return torch.round(v / step) * step


def _exact_round(x, fmt, wide):
    b = _blocks(x.double(), BLOCK[fmt])
    top = b.abs().amax(-1, keepdim=True)
    if fmt == "nvfp4":
        d = _exact_e4m3(top / (6 * wide.double())) * wide.double()
    else:
        e = torch.ceil(torch.log2((top / 6).clamp(min=1e-30)))
        e = torch.where(top > 6 * _exact_two_to(e), e + 1, torch.where(top <= 6 * _exact_two_to(e - 1), e - 1, e))  # log2 may be off at a border
        d = torch.where(top > 0, _exact_two_to(e), 0.0)
    a = torch.where(d > 0, b.abs() / d, 0.0).clamp(max=6.0)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return (torch.sign(b) * torch.round(a / step) * step * d).flatten(-2)[..., : x.shape[-1]]


def _exact_weights(w, fmt, K, e=None):
    codes, scales, wide = (t if e is None else t[e] for t in w)
    v = torch.stack((codes.long() % 16, codes.long() // 16), -1).flatten(-2)[..., :K]
    m, two = (v % 2).double(), (v % 8 // 2).double()
    v = torch.where(v >= 8, -1.0, 1.0) * torch.where(two == 0, 0.5 * m, (1 + 0.5 * m) * _exact_two_to(two - 1))
    c = scales.long()
    if fmt == "nvfp4":
        d = torch.where(c < 8, (c % 8).double() / 512, (1 + (c % 8).double() / 8) * _exact_two_to(c // 8 - 7)) * wide.double()
    else:
        d = _exact_two_to(c - 127)
    return v * d.repeat_interleave(BLOCK[fmt], -1)[..., :K]


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op in ("activate", "activate_grad"):
        I = case["I"]
        x = s["rows"].double().requires_grad_()
        g, u = x[:, :I], x[:, I:]
        a = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu}[case["act"]](g)
        y = a * u * _factors(case, s, torch.float64)
        if op == "activate":
            return y.detach()
        y.backward(s["dy"].double())
        return x.grad
    fmt, k = case["format"], case["k"]
    if op == "round":
        v = _exact_round(s["x"], fmt, s["wide"])
        return v[s["routing"][5].long() // k] if k else v
    if op == "product":
        q, K = _exact_round(s["x"], fmt, s["wide"]), case["K"]
        if not case["E"]:
            y = q @ _exact_weights(s["w"], fmt, K).t()
            return y if s["bias"] is None else y + s["bias"].double()
        ids = s["routing"][0].flatten()
        y, at = torch.zeros(ids.numel(), case["N"], dtype=torch.float64, device="cuda"), 0
        for e in range(case["E"]):
            t = (ids == e).nonzero().flatten() // k
            if t.numel():
                y[at: at + t.numel()] = q[t] @ _exact_weights(s["w"], fmt, K, e).t() + (0.0 if s["bias"] is None else s["bias"][e].double())
            at += t.numel()
        return y
    H, I = case["H"], case["I"]
    ids, weights = s["routing"][:2]
    x, y = s["x"].double(), torch.zeros(case["T"], H, dtype=torch.float64, device="cuda")
    for e in range(case["E"]):
        t, j = (ids == e).nonzero(as_tuple=True)
        if t.numel():
            u = x[t] @ _exact_weights(s["up"], fmt, H, e).t()
            o = (torch.nn.functional.silu(u[:, :I]) * u[:, I:]) @ _exact_weights(s["down"], fmt, I, e).t()
            y.index_add_(0, t, o * weights[t, j, None].double())
    return y
