"""What stands beside the sparse product in a layer with compressed weights, as a program that serves such layers calls it:
the product with 4-bit weights (`quant_plan_create`, `QuantPlan.execute`), the root-mean-square norm that makes its
operand (`norm`), the gated activation between two of them (`gate`), and the feed-forward block of all three.

Activations are features x tokens, as B and C of `Plan.execute`; "features" is that order in memory (a row holds one
feature of all tokens), "tokens" the other one (a row holds one token).  A case is

  kind      "product", "norm", "gate" or "block"
  product   rows, cols (M and K), group (weights to a scale), zeros (zero points, else 8), tokens (N), type (of B and C;
            "int8": B in codes with a scale for each token, C in bfloat16), order
  norm      cols (K), tokens, type, order, residual (an addend, its sum is written), codes (int8 output with scales)
  gate      cols (F), tokens, type, order, act, codes
  block     cols (K), inner (F), group, tokens, type: norm, product with 2 F rows, gate, product with K rows, int8 between

Codes are returned as the values that they stand for.
"""
import math

import torch

own = False

TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
EPS = 1e-6


def _product(name, rows, cols, group, zeros, tokens, type, order):
    return dict(name=name, kind="product", rows=rows, cols=cols, group=group, zeros=zeros, tokens=tokens, type=type, order=order)


def _norm(name, cols, tokens, type, order, residual, codes):
    return dict(name=name, kind="norm", cols=cols, tokens=tokens, type=type, order=order, residual=residual, codes=codes)


def _gate(name, cols, tokens, type, order, act, codes):
    return dict(name=name, kind="gate", cols=cols, tokens=tokens, type=type, order=order, act=act, codes=codes)


def _block(name, cols, inner, group, tokens, type):
    return dict(name=name, kind="block", cols=cols, inner=inner, group=group, tokens=tokens, type=type)


def listed():
    return [
        # the smallest configuration's layer, one token: a call is launch latency
        _product("product_smallest", 256, 256, 32, False, 1, "float32", "features"),
        # token-by-token decoding of a square layer
        _product("product_one_token", 4096, 4096, 128, False, 1, "bfloat16", "tokens"),
        # the two feed-forward projections: a small batch in codes, and a batch in the sparse product's own layout
        _product("product_codes", 1024, 4096, 128, True, 16, "int8", "tokens"),
        _product("product_columns", 4096, 1024, 64, True, 32, "float32", "features"),
        # nothing is a multiple of anything
        _product("product_ragged", 3001, 2511, 64, True, 200, "float16", "tokens"),
        # a prompt
        _product("product_prompt", 8192, 8192, 128, False, 512, "bfloat16", "tokens"),
        # before a product: one token, a batch in the sparse product's layout, a prompt in codes
        _norm("norm_one_token", 4096, 1, "bfloat16", "tokens", True, False),
        _norm("norm_columns", 1024, 128, "float32", "features", True, False),
        _norm("norm_codes", 8192, 2048, "bfloat16", "tokens", True, True),
        # between two products: a small batch, a prompt
        _gate("gate_batch", 4096, 16, "float16", "tokens", "silu", False),
        _gate("gate_prompt", 16384, 2048, "bfloat16", "tokens", "silu", False),
        # the block they make, a few tokens
        _block("block_few_tokens", 4096, 8192, 128, 8, "bfloat16"),
    ]


MOST_FLOPS = 2 * 8192 * 8192 * 512
MOST_BYTES = 6 * 16384 * 2048


def draw(rng):
    def size(lo, hi):
        x = math.exp(rng.uniform(math.log(lo), math.log(hi)))
        step = rng.choice((1, 1, 2, 64, 128)) if x >= 128 else 1
        return int(min(hi, max(lo, round(x / step) * step)))

    while True:
        kind = rng.choice(("product", "product", "product", "norm", "norm", "gate", "block"))
        order = rng.choice(("features", "tokens"))
        floats = rng.choice(("float32", "float16", "bfloat16"))
        short = rng.choice(("float16", "bfloat16"))
        if kind == "product":
            case = _product("", size(64, 16384), size(64, 16384), rng.choice((32, 64, 128, 128, 256)), rng.random() < 0.5,
                            size(1, 512), rng.choice((floats, "int8")), order)
            case["order"] = "tokens" if case["type"] == "int8" else order
        elif kind == "norm":
            codes = rng.random() < 0.5
            case = _norm("", size(64, 16384), size(1, 4096), short if codes else floats, order, rng.random() < 0.7, codes)
        elif kind == "gate":
            codes = rng.random() < 0.5
            case = _gate("", size(64, 16384), size(1, 4096), short if codes else floats, order,
                         rng.choice(("silu", "silu", "gelu", "relu")), codes)
        else:
            case = _block("", size(256, 8192), size(256, 16384), rng.choice((64, 128)), size(1, 256), short)
        del case["name"]
        w = work(case)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return case


def _weights(rows, cols, group, zeros, g):
    """Normal weights in 4 bits: codes (two in a byte, the even column in the low half), a scale and a zero point a group."""
    groups, std = -(-cols // group), cols ** -0.5
    w = torch.zeros((rows, groups * group), device="cuda")
    w[:, :cols] = torch.randn((rows, cols), device="cuda", generator=g) * std
    w = w.view(rows, groups, group)
    if zeros:
        lo, hi = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
        scales = ((hi - lo) / 15).clamp(min=1e-8)
        points = torch.round(-lo / scales).clamp(0, 15)
    else:
        scales = (w.abs().amax(2) / 7).clamp(min=1e-8)
        points = torch.full_like(scales, 8)
    q = torch.round(w / scales[:, :, None] + points[:, :, None]).clamp(0, 15).to(torch.uint8).view(rows, groups * group)
    q = q[:, :cols + cols % 2].contiguous()
    return dict(rows=rows, cols=cols, group=group, codes=q[:, ::2] | (q[:, 1::2] << 4), scales=scales, points=points.to(torch.uint8), zeros=zeros)


def _acts(rows, tokens, order, g, spread=0.5):
    """Activations: normal, some features larger than others, as (rows, tokens) in the order given."""
    x = torch.randn((tokens, rows), device="cuda", generator=g) * torch.exp(spread * torch.randn((rows,), device="cuda", generator=g))
    return x.t() if order == "tokens" else x.t().contiguous()


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed + 1_000_003)
    kind, tokens, order = case["kind"], case["tokens"], case.get("order", "tokens")
    state = dict(case=case)
    if kind == "product":
        state["W"] = _weights(case["rows"], case["cols"], case["group"], case["zeros"], g)
        B = _acts(case["cols"], tokens, order, g)
        if case["type"] == "int8":
            state["scales"] = B.abs().amax(0) / 127
            state["B"] = torch.round(B / state["scales"]).to(torch.int8)
        else:
            state["B"] = B.to(TYPES[case["type"]])
    elif kind == "gate":
        state["a"] = (2 * _acts(case["cols"], tokens, order, g)).to(TYPES[case["type"]])
        state["b"] = _acts(case["cols"], tokens, order, g).to(TYPES[case["type"]])
    else:
        T = TYPES[case["type"]]
        state["x"] = _acts(case["cols"], tokens, order, g).to(T)
        state["r"] = (4 * _acts(case["cols"], tokens, order, g)).to(T)
        state["w"] = (1 + 0.2 * torch.randn((case["cols"],), device="cuda", generator=g)).to(T)
        if kind == "block":
            state["up"] = _weights(2 * case["inner"], case["cols"], case["group"], False, g)
            state["down"] = _weights(case["cols"], case["inner"], case["group"], False, g)
    return state


def _plan(W):
    import paper_2506_15174_amd as spmm
    return spmm.quant_plan_create(W["rows"], W["cols"], W["codes"], W["scales"], W["points"] if W["zeros"] else None, group=W["group"])


def prepare(case, seed):
    state = _inputs(case, seed)
    if own:
        for key in ("W", "up", "down"):
            if key in state:
                state["plan_" + key] = _plan(state[key])
    return state


def _dense(W):
    """The 4-bit weights in 32 bits."""
    q = torch.stack((W["codes"] & 15, W["codes"] >> 4), 2).view(W["rows"], -1)[:, :W["cols"]].float()
    of = torch.arange(W["cols"], device="cuda") // W["group"]
    return (q - W["points"].float()[:, of]) * W["scales"][:, of]


def _acted(x, act):
    if act == "silu":
        return x / (1 + torch.exp(-x))
    if act == "gelu":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    return x.clamp(min=0)


def _coded(p, size):
    """Codes of the values p x size (a token's factor) and the tokens' scales; rounding is by p alone."""
    most = p.abs().amax(0)
    codes = torch.round(p * torch.where(most > 0, 127 / most, 0))
    return codes, most * size / 127


def _normed(x, r, w, codes):
    """(the sum in x's type, the normed values in 32 bits or codes, scales)"""
    t = x if r is None else (x.float() + r.float()).to(x.dtype)
    v = t.float()
    size = 1 / torch.sqrt((v.double() * v.double()).mean(0) + EPS).float()
    if codes:
        return t, *_coded(v * w.float()[:, None], size)
    return t, v * size * w.float()[:, None], None


def _values(codes, scales, T):
    return torch.mul(codes, scales, out=torch.empty_like(codes, dtype=T))


def _run_own(state):
    import paper_2506_15174_amd as spmm
    case = state["case"]
    kind = case["kind"]
    if kind == "product":
        if case["type"] == "int8":
            return state["plan_W"].execute(state["B"], scales=state["scales"], dtype=torch.bfloat16)
        return state["plan_W"].execute(state["B"])
    if kind == "norm":
        y = spmm.norm(state["x"], state["w"], EPS, residual=state["r"] if case["residual"] else None, dtype=torch.int8 if case["codes"] else None)
        out = _values(y.out, y.scales, state["x"].dtype) if case["codes"] else y.out
        return dict(y=out, total=y.total) if case["residual"] else dict(y=out)
    if kind == "gate":
        y = spmm.gate(state["a"], state["b"], act=case["act"], dtype=torch.int8 if case["codes"] else None)
        return _values(y.out, y.scales, state["a"].dtype) if case["codes"] else y.out
    y = spmm.norm(state["x"], state["w"], EPS, residual=state["r"], dtype=torch.int8)
    h = state["plan_up"].execute(y.out, scales=y.scales, dtype=state["x"].dtype)
    z = spmm.gate(h[:case["inner"]], h[case["inner"]:], dtype=torch.int8)
    return dict(y=state["plan_down"].execute(z.out, scales=z.scales, dtype=state["x"].dtype), total=y.total)


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    kind = case["kind"]
    if kind == "product":
        B = state["B"].float()
        C = _dense(state["W"]) @ B
        if case["type"] == "int8":
            return (C * state["scales"]).to(torch.bfloat16)
        return C.to(state["B"].dtype)
    if kind == "norm":
        t, y, scales = _normed(state["x"], state["r"] if case["residual"] else None, state["w"], case["codes"])
        out = y.to(t.dtype) if scales is None else _values(y, scales, t.dtype)
        return dict(y=out, total=t) if case["residual"] else dict(y=out)
    if kind == "gate":
        p = _acted(state["a"].float(), case["act"]) * state["b"].float()
        return _values(*_coded(p, 1.0), state["a"].dtype) if case["codes"] else p.to(state["a"].dtype)
    T = state["x"].dtype
    t, codes, scales = _normed(state["x"], state["r"], state["w"], True)
    h = (_dense(state["up"]) @ codes * scales).to(T).float()
    codes, scales = _coded(_acted(h[:case["inner"]], "silu") * h[case["inner"]:], 1.0)
    return dict(y=(_dense(state["down"]) @ codes * scales).to(T), total=t)


def work(case):
    kind, N, size = case["kind"], case["tokens"], 4 if case["type"] == "float32" else 2

    def weights(rows, cols, zeros):
        return rows * (cols / 2 + (4.5 if zeros else 4) * -(-cols // case["group"]))

    if kind == "product":
        M, K = case["rows"], case["cols"]
        B = K * N + 4 * N if case["type"] == "int8" else K * N * size
        return {"bytes": weights(M, K, case["zeros"]) + B + M * N * size, "flops": 2 * M * K * N}
    K = case["cols"]
    if kind == "norm":
        return {"bytes": K * N * ((3 if case["residual"] else 1) * size + (1 if case["codes"] else size)) + size * K, "flops": 4 * K * N}
    if kind == "gate":
        return {"bytes": K * N * (2 * size + (1 if case["codes"] else size)), "flops": 6 * K * N}
    F = case["inner"]
    return {"bytes": weights(2 * F, K, False) + weights(K, F, False) + 4 * K * N * size + size * K, "flops": 6 * F * K * N}


def _exact_product(W, B):
    """sum over groups of scale x (sum of (code - zero point) x B), in 64 bits."""
    C = torch.zeros((W["rows"], B.shape[1]), dtype=torch.float64, device="cuda")
    for n, k in enumerate(range(0, W["cols"], W["group"])):
        k1 = min(W["cols"], k + W["group"])
        at = torch.arange(k, k1, device="cuda")
        q = (W["codes"][:, at // 2].int() >> (4 * (at % 2)).int()) & 15
        C += W["scales"][:, n, None].double() * ((q - W["points"][:, n, None].int()).double() @ B[k:k1])
    return C


def _exact_acted(x, act):
    if act == "silu":
        return x * torch.sigmoid(x)
    return torch.relu(x) if act == "relu" else torch.nn.functional.gelu(x, approximate="tanh")


def _exact_values(p, size):
    """The values that 8-bit codes of p x size stand for, and the codes' step."""
    step = p.abs().amax(0) / 127
    return torch.round(p / step.clamp(min=1e-300)) * step * size


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "product":
        B = s["B"].double()
        return _exact_product(s["W"], B * s["scales"].double() if case["type"] == "int8" else B)
    if kind == "gate":
        p = _exact_acted(s["a"].double(), case["act"]) * s["b"].double()
        return _exact_values(p, 1.0) if case["codes"] else p
    t = s["x"].double()
    if kind == "block" or case["residual"]:
        t = (t + s["r"].double()).to(s["x"].dtype).double()
    size = (t.square().mean(0) + EPS).rsqrt()
    p = t * s["w"].double()[:, None]
    if kind == "norm":
        y = _exact_values(p, size) if case["codes"] else p * size
        return dict(y=y, total=t) if case["residual"] else dict(y=y)
    h = _exact_product(s["up"], _exact_values(p, size)).to(s["x"].dtype).double()
    z = _exact_values(_exact_acted(h[:case["inner"]], "silu") * h[case["inner"]:], 1.0)
    return dict(y=_exact_product(s["down"], z), total=t)
