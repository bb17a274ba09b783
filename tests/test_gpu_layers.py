"""The operators beside the sparse product on the GPU, against plain implementations in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2506_15174_amd as spmm
from layers_reference import HALF_STEP, SMALLEST, TYPES, act64, as64, codes_of, placed, summed, weights

pytestmark = pytest.mark.gpu

FLOATS = ("float32", "float16", "bfloat16")


@pytest.fixture(autouse=True)
def gpu():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    spmm.load()


def plan_of(M, K, group, seed, **kw):
    codes, scales, zeros, W = weights(M, K, group, seed, **kw)
    return spmm.quant_plan_create(M, K, codes, scales, zeros, group=group), W


def product_bound(W, B, type, out, C):
    """A sum of up to 128 columns of a group takes one rounding of at most a step (2^-23, as sums in matrix instructions may be cut off)
    for each product, three times as many for B in three parts; then one for each of at most ceil(K / 32) groups and of 16 waves and ranges, one for a
    token's scale; the output's own half step."""
    terms = {"float32": 384, "float16": 128, "bfloat16": 128, "int8": 0}[type] + W.shape[1] / 32 + 18
    return terms * 2.0 ** -23 * (np.abs(W) @ np.abs(B)) * 1.01 + HALF_STEP[out] * np.abs(C) + SMALLEST[out]


def check_product(M, K, N, group, type, order, seed, out=None, c_order=None, whole=False, zeros=True, pad=0, offset=0, c_pad=0):
    plan, W = plan_of(M, K, group, seed, zeros=zeros, whole=whole)
    rng = np.random.default_rng(seed + 1)
    scales = None
    if type == "int8":
        B = rng.integers(-127, 128, (K, N))
        s = (2.0 ** rng.integers(-3, 3, N) if whole else rng.uniform(0.01, 0.1, N)).astype(np.float32)
        scales = torch.from_numpy(s).cuda()
        d = placed(B, type, order, pad, offset)
        B64 = as64(d) * s
    else:
        d = placed(rng.integers(-4, 5, (K, N)) if whole else rng.standard_normal((K, N)), type, order, pad, offset)
        B64 = as64(d)
    want = W @ B64
    c_order, out = c_order or order, out or ("float32" if type == "int8" or whole else type)
    C = placed(np.zeros((M, N)), out, c_order, c_pad, offset)
    memory = torch.as_strided(C, ((N if c_order == "tokens" else M) * C.stride(1 if c_order == "tokens" else 0) - c_pad,), (1,), C.storage_offset())
    memory.fill_(float("nan"))
    assert plan.execute(d, C, scales=scales) is C
    got = as64(C)
    if whole:
        assert np.array_equal(got, want)
    else:
        err = np.abs(got - want)
        assert (err <= product_bound(W, B64, type, out, want)).all(), "largest error %.3g" % np.nanmax(err)
    assert int(memory.isnan().sum()) == memory.numel() - M * N, "elements beside C were written"
    made = plan.execute(d, scales=scales, dtype=TYPES[out])
    assert made.dtype == TYPES[out] and torch.equal(made, C)


@pytest.mark.parametrize("type", FLOATS + ("int8",))
@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("N", [1, 3, 16, 17, 40, 70, 130])
def test_whole_numbers_are_exact(type, group, N):
    """Every product and sum is a whole number times a power of two: any mistake of place shows."""
    check_product(45, 391, N, group, type, "tokens", N + group, whole=True)
    if type != "int8":
        check_product(45, 391, N, group, type, "features", N + group + 1, whole=True)


@pytest.mark.parametrize("type", FLOATS + ("int8",))
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K", [(8200, 520), (16500, 260), (70, 2200), (8200, 2200), (16500, 1290)])
def test_whole_numbers_are_exact_in_every_shape_of_workgroup(type, group, M, K):
    """Rows and columns for which waves have one, two or four tiles of rows, and one or several blocks of columns."""
    for N in (1, 2, 7, 16, 33, 100):
        check_product(M, K, N, group, type, "tokens", N + group, whole=True)
        if type != "int8":
            check_product(M, K, N, group, type, "features", N + group + 1, whole=True)


@pytest.mark.parametrize("type", ["float16", "bfloat16", "int8"])
@pytest.mark.parametrize("group,zeros", [(32, True), (32, False), (64, True), (64, False), (128, True), (128, False)])
@pytest.mark.parametrize("N", [2040, 1001, 500])
def test_whole_numbers_are_exact_in_prompts(type, group, zeros, N):
    """Teams of eight, four and two waves (the token counts); fewer blocks of columns than teams, as many, and more."""
    for n, K in enumerate((100, 390, 650, 1300)):
        check_product(4090 - 16 * n, K, N, group, type, "features" if n % 2 and type != "int8" else "tokens", N + group, whole=True, zeros=zeros)


@pytest.mark.parametrize("type", FLOATS + ("int8",))
@pytest.mark.parametrize("M,K,N,group", [(1, 1, 1, 32), (1, 1, 5, 64), (5, 2, 1, 128), (16, 128, 16, 32), (17, 33, 2, 32), (33, 129, 33, 128), (64, 65, 64, 64),
                                         (100, 1000, 1, 128), (300, 257, 129, 384), (31, 4100, 7, 128), (48, 640, 300, 1024), (2100, 96, 8, 64), (130, 2048, 513, 64)])
def test_odd_sizes(type, M, K, N, group):
    for order in ("tokens", "features") if type != "int8" else ("tokens",):
        check_product(M, K, N, group, type, order, M + K + N)


@pytest.mark.parametrize("type", FLOATS + ("int8",))
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("M,K,N", [(1024, 4096, 16), (4096, 1024, 1), (512, 2048, 128)])
def test_layers_sizes(type, zeros, M, K, N):
    check_product(M, K, N, 128, type, "tokens", K, zeros=zeros)
    check_product(M, K, N, 64, type, "tokens" if type == "int8" else "features", K, zeros=zeros)


@pytest.mark.parametrize("type", FLOATS + ("int8",))
@pytest.mark.parametrize("out", FLOATS)
@pytest.mark.parametrize("c_order", ["tokens", "features"])
@pytest.mark.parametrize("N", [1, 6, 45])
def test_strides_offsets_and_output_types(type, out, c_order, N):
    for pad, offset in ((1, 1), (3, 0), (8, 8), (5, 3)):
        check_product(50, 300, N, 64, type, "tokens", 7 + pad, out=out, c_order=c_order, pad=pad, offset=offset, c_pad=pad)
        if type != "int8":
            check_product(50, 300, N, 64, type, "features", 8 + pad, out=out, c_order=c_order, pad=pad, offset=offset, c_pad=pad)


@pytest.mark.parametrize("type", FLOATS)
@pytest.mark.parametrize("N", [1, 5, 20])
def test_infinities_and_nan_go_where_the_sum_says(type, N):
    """Each in one token: that token's elements are what the plain sum gives, others are untouched by it."""
    M, K = 40, 200
    plan, W = plan_of(M, K, 64, 3)
    B = np.random.default_rng(4).standard_normal((K, N))
    B[7, 0] = np.inf
    if N > 1:
        B[150, 1] = np.nan
    if N > 2:
        B[3, 2], B[199, 2] = -np.inf, np.inf
    for order in ("tokens", "features"):
        d = placed(B, type, order)
        with np.errstate(invalid="ignore"):
            want = (W[:, :, None] * as64(d)[None]).sum(1)
        got = as64(plan.execute(d, dtype=torch.float32))
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
        assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
        fine = np.isfinite(want)
        assert np.allclose(got[fine], want[fine], rtol=0, atol=1e-3)


def test_large_and_small_values_of_32_bits():
    """Parts are cut off, not rounded up: values next to the largest stay finite; values down to 2^-100 keep their 24 bits."""
    M, K = 16, 96
    q = np.full((M, K // 2), 0x99, np.uint8)   # weights of 1
    for big in (np.float32(3.4e38), np.float32(1.9999999) * np.float32(2.0 ** -100), np.float32(np.pi)):
        B = np.zeros((K, 4), np.float32)
        B[5] = [big, -big, big, 0]
        for n in (1, 4):
            C = spmm.quant_plan_create(M, K, q, np.ones((M, 1), np.float32)).execute(torch.from_numpy(B[:, :n].copy()).cuda())
            assert np.array_equal(C.cpu().numpy(), np.repeat(B[5:6, :n], M, 0))


def test_nothing_to_do():
    for M, K, N in ((0, 5, 3), (4, 0, 3), (0, 0, 1)):
        plan = spmm.quant_plan_create(M, K, np.zeros((M, (K + 1) // 2), np.uint8), np.zeros((M, -(-K // 128)), np.float32))
        C = plan.execute(torch.ones((K, N), device="cuda"))
        assert C.shape == (M, N) and (C == 0).all()
        assert plan.describe() == {"M": M, "K": K, "group": 128, "device_bytes": 0}


@pytest.mark.parametrize("type", FLOATS + ("int8",))
@pytest.mark.parametrize("M,N", [(70, 300), (4090, 1000), (20, 17)])
def test_no_columns_and_many_tokens(type, M, N):
    plan = spmm.quant_plan_create(M, 0, np.zeros((M, 0), np.uint8), np.zeros((M, 0), np.float32))
    B = torch.zeros((0, N), dtype=TYPES[type], device="cuda")
    C = torch.full((M, N), 7.0, device="cuda")
    plan.execute(B, C=C, scales=torch.ones(N, device="cuda") if type == "int8" else None)
    assert (C == 0).all()


def test_plans_from_tensors_of_every_kind():
    codes, scales, zeros, W = weights(20, 70, 32, 5, whole=True)
    B = torch.randint(-3, 4, (70, 9)).float()
    want = torch.from_numpy(W @ B.double().numpy()).float()
    for put in (lambda a: a, torch.from_numpy, lambda a: torch.from_numpy(a).cuda()):
        for type in (torch.float32, torch.float16, torch.bfloat16):
            s = put(scales)
            plan = spmm.quant_plan_create(20, 70, put(codes), s.to(type) if torch.is_tensor(s) else s, put(zeros), group=32)
            assert torch.equal(plan.execute(B.cuda()).cpu(), want)


# ---- norm -----------------------------------------------------------------------------------------------------

def norm_case(K, N, type, order, seed, residual=True, pad=0, offset=0, w_type="float32", spread=1.0):
    rng = np.random.default_rng(seed)
    x = placed(rng.standard_normal((K, N)) * np.exp(spread * rng.standard_normal((K, 1))), type, order, pad, offset)
    r = placed(3 * rng.standard_normal((K, N)), type, order, pad, offset) if residual else None
    w = torch.from_numpy(1 + 0.3 * rng.standard_normal(K)).to(TYPES[w_type]).cuda()
    return x, r, w


def check_norm(x, r, w, eps, type, out_type, **kw):
    K, N = x.shape
    t = summed(x.cpu(), None if r is None else r.cpu())   # (x may be written: total=x)
    y = spmm.norm(x, w, eps, residual=r, dtype=TYPES[out_type], **kw)
    if r is not None or "total" in kw:
        assert torch.equal(y.total.cpu(), t) and y.total.dtype == t.dtype
    else:
        assert y.total is None
    t64, w64 = as64(t), as64(w)[:, None]
    f = 1 / np.sqrt((t64 ** 2).mean(0) + eps)
    # squares of one sign: a chain of at most K / 16 + 256 roundings, halved by the root; then a handful of single ones
    rel = ((K / 16 + 256) / 2 + 8) * 2.0 ** -24
    if out_type == "int8":
        codes, most = codes_of(t.float().numpy() * w.float().cpu().numpy()[:, None])
        assert np.array_equal(y.out.cpu().numpy(), codes)
        assert y.out.stride(0) == 1 or K == 1
        assert np.allclose(as64(y.scales), most * f / 127, rtol=rel, atol=SMALLEST["float32"])
    else:
        want = t64 * f * w64
        assert (np.abs(as64(y.out) - want) <= (rel + HALF_STEP[out_type]) * np.abs(want) * 1.01 + SMALLEST[out_type]).all()
        assert y.scales is None
    return y


@pytest.mark.parametrize("type", FLOATS)
@pytest.mark.parametrize("out", FLOATS + ("int8",))
@pytest.mark.parametrize("order", ["tokens", "features"])
@pytest.mark.parametrize("K,N", [(1, 1), (7, 1), (1, 9), (64, 3), (256, 16), (1000, 17), (4096, 1), (4100, 33), (513, 260)])
def test_norm(type, out, order, K, N):
    for residual in (False, True):
        x, r, w = norm_case(K, N, type, order, K + N, residual, w_type=type if K % 2 else "float32")
        check_norm(x, r, w, 1e-6, type, out)


@pytest.mark.parametrize("type", FLOATS)
@pytest.mark.parametrize("K,N,order", [(16384, 5, "tokens"), (16384, 5, "features"), (20001, 2, "tokens"), (8192, 300, "tokens"), (2048, 1024, "features"), (70000, 3, "tokens"),
                                       (70000, 1, "features"), (50, 5000, "tokens"), (50, 5000, "features"), (300, 66000, "tokens")])
def test_norm_long(type, K, N, order):
    x, r, w = norm_case(K, N, type, order, 1)
    check_norm(x, r, w, 1e-5, type, type)
    check_norm(x, r, w, 1e-5, type, "int8")


@pytest.mark.parametrize("type", FLOATS)
@pytest.mark.parametrize("order", ["tokens", "features"])
@pytest.mark.parametrize("pad,offset", [(1, 1), (3, 0), (8, 8), (5, 3)])
@pytest.mark.parametrize("K,N", [(300, 1), (300, 37), (40, 300), (4000, 5)])
def test_norm_strides_and_sums_in_place(type, order, pad, offset, K, N):
    for out in (type, "int8"):
        for which in ("x", "r", "new"):
            x, r, w = norm_case(K, N, type, order, 2, pad=pad, offset=offset)
            target = {"x": x, "r": r, "new": placed(np.zeros((K, N)), type, order, pad, offset)}[which]
            keep = as64(r if which == "x" else x)
            y = check_norm(x, r, w, 1e-6, type, out, total=target)
            assert y.total is target and np.array_equal(as64(r if which == "x" else x), keep)
            # outputs that are handed in, and what lies beside them
            x, r, w = norm_case(K, N, type, order, 2, pad=pad, offset=offset)
            o = placed(np.zeros((K, N)), out, "tokens" if out == "int8" else order, pad, offset)
            s = torch.full((N,), 9.0, device="cuda") if out == "int8" else None
            z = check_norm(x, r, w, 1e-6, type, out, out=o, scales=s)
            assert z.out is o and torch.equal(o, y.out) and (s is None or z.scales is s)
            rows = torch.as_strided(o, (N, o.stride(1)) if o.stride(0) == 1 and N > 1 else (K, o.stride(0)), (max(o.stride()), 1), o.storage_offset()) if K > 1 and N > 1 else None
            if rows is not None and pad:
                beside = rows[:-1, (K if o.stride(0) == 1 else N):]
                assert (beside == 77).all() if out == "int8" else beside.isnan().all()


@pytest.mark.parametrize("order", ["tokens", "features"])
@pytest.mark.parametrize("K,N", [(40, 6), (5000, 6)])
def test_norm_of_zeros_infinities_and_nan(order, K, N):
    x, _, w = norm_case(K, N, "float32", order, 3, residual=False)
    x[:, 0] = 0
    x[3, 1] = float("inf")
    x[K - 1, 2] = float("nan")
    x[:, 3] *= 2.0 ** -130
    x[5, 4] = float("-inf")
    y = spmm.norm(x, w, 1e-6, dtype=torch.int8)
    codes, scales = y.out.cpu(), y.scales.cpu()
    assert (codes[:, [0, 1, 2, 4]] == 0).all() and scales[0] == 0 and scales[[1, 2, 4]].isnan().all()
    want, _ = codes_of((x[:, [3, 5]] * w[:, None]).cpu().numpy())
    assert np.array_equal(codes[:, [3, 5]].numpy(), want) and (codes[:, 3].abs() == 127).any()
    z = as64(spmm.norm(x, w, 1e-6).out)
    assert (z[:, 0] == 0).all() and np.isnan(z[3, 1]) and np.isnan(z[:, 2]).all() and np.isnan(z[5, 4]) and np.isfinite(z[:, [3, 5]]).all()
    assert (z[[0, 1, 2, 4], 1] == 0).all()
    nothing = spmm.norm(torch.zeros((8, 2), device="cuda"), torch.ones(8, device="cuda"), 0.0)   # 0 / 0
    assert nothing.out.isnan().all()


# ---- gate -----------------------------------------------------------------------------------------------------

def act_error(x, act):
    """Relative: the exponential's argument is rounded (gelu: its cubic too) and its error grows with its magnitude; then a handful of single roundings."""
    if act == "relu":
        return np.full_like(x, 2.0 ** -24)
    u = np.abs(x) if act == "silu" else 2 * np.sqrt(2 / np.pi) * np.abs(x + 0.044715 * x ** 3)
    return (np.minimum(u, 110) * (1 if act == "silu" else 8) + 12) * 2.0 ** -24


def check_gate(a, b, act, type, out_type, **kw):
    F, N = a.shape
    a64 = as64(a)
    want = act64(a64, act) * (1.0 if b is None else as64(b))
    y = spmm.gate(a, b, act, dtype=TYPES[out_type], **kw)
    # below 2^-126 the exponential may be infinite and the quotient 0
    err = act_error(a64, act) * np.abs(want) + 2.0 ** -120 * (1.0 if b is None else np.abs(as64(b)))
    if out_type == "int8":
        most = np.abs(want).max(0)
        scales = as64(y.scales)
        # P / 127 is rounded once more than P: 2^-24
        assert (np.abs(scales - most / 127) <= (act_error(a64, act).max(0) + 2.0 ** -24) * most / 127 * 1.01 + 2.0 ** -120).all()
        assert (np.abs(as64(y.out) * scales - want) <= 0.5001 * scales + err + act_error(a64, act).max(0) * most).all()
        assert int(y.out.abs().max()) <= 127
    else:
        assert (np.abs(as64(y.out) - want) <= err + HALF_STEP[out_type] * np.abs(want) * 1.01 + SMALLEST[out_type]).all()
        assert y.scales is None
    return y


@pytest.mark.parametrize("type", FLOATS)
@pytest.mark.parametrize("out", FLOATS + ("int8",))
@pytest.mark.parametrize("order", ["tokens", "features"])
@pytest.mark.parametrize("F,N", [(1, 1), (9, 1), (1, 5), (256, 16), (1000, 17), (4096, 1), (4100, 33), (513, 260)])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_gate(type, out, order, F, N, act):
    rng = np.random.default_rng(F + N)
    a, b = placed(4 * rng.standard_normal((F, N)), type, order), placed(rng.standard_normal((F, N)), type, order)
    check_gate(a, b, act, type, out)
    check_gate(a, None, act, type, out)


@pytest.mark.parametrize("type", FLOATS)
@pytest.mark.parametrize("order", ["tokens", "features"])
@pytest.mark.parametrize("F,N", [(300, 1), (300, 37), (20000, 3), (64, 3000)])
def test_gate_halves_of_one_tensor_strides_and_what_lies_beside(type, order, F, N):
    rng = np.random.default_rng(5)
    for pad, offset in ((0, 0), (1, 1), (8, 8)):
        h = placed(rng.standard_normal((2 * F, N)), type, order, pad, offset)
        for out in (type, "int8"):
            y = check_gate(h[:F], h[F:], "silu", type, out)
            o = placed(np.zeros((F, N)), out, "tokens" if out == "int8" else order, pad, offset)
            z = check_gate(h[:F], h[F:], "silu", type, out, out=o)
            assert z.out is o and torch.equal(o, y.out)
            if pad and N > 1:
                rows = torch.as_strided(o, (N, o.stride(1)) if o.stride(0) == 1 else (F, o.stride(0)), (max(o.stride()), 1), o.storage_offset())
                beside = rows[:-1, (F if o.stride(0) == 1 else N):]
                assert (beside == 77).all() if out == "int8" else beside.isnan().all()


@pytest.mark.parametrize("order", ["tokens", "features"])
def test_gate_of_large_values_infinities_and_nan(order):
    v = np.array([0.0, -0.0, 90.0, -90.0, 1e4, -1e4, 6e4, -6e4, 1e-30, -1e-30, np.inf, -np.inf, np.nan])
    a = placed(np.repeat(v[:, None], 3, 1), "float32", order)
    silu, gelu, relu = (as64(spmm.gate(a, act=act).out)[:, 0] for act in ("silu", "gelu", "relu"))
    for got in (silu, gelu, relu):
        assert got[10] == np.inf and np.isnan(got[12]) and got[2] == 90 and got[4] == 1e4 and (got[[0, 1]] == 0).all() and got[6] == 6e4
    for got in (silu, gelu):
        assert (np.abs(got[[3, 5, 7]]) < 1e-30).all() and np.allclose(got[[8, 9]], [5e-31, -5e-31], rtol=1e-6)
    assert (relu[[3, 5, 7, 9, 11]] == 0).all()


# ---- the operators together, streams and graphs ---------------------------------------------------------------

def block(plans, x, r, w, F, short):
    y = spmm.norm(x, w, 1e-6, residual=r, dtype=torch.int8)
    h = plans[0].execute(y.out, scales=y.scales, dtype=short)
    z = spmm.gate(h[:F], h[F:], dtype=torch.int8)
    return plans[1].execute(z.out, scales=z.scales, dtype=short), y.total


@pytest.mark.parametrize("type", ["bfloat16", "float16"])
@pytest.mark.parametrize("N", [1, 5, 48])
def test_feed_forward_block_in_codes(type, N):
    D, F = 320, 700
    up, W1 = plan_of(2 * F, D, 64, 1, zeros=False)
    down, W2 = plan_of(D, F, 128, 2)
    x, r, w = norm_case(D, N, type, "tokens", 3, w_type=type)
    y, total = block((up, down), x, r, w, F, TYPES[type])
    t = summed(x.cpu(), r.cpu())
    assert torch.equal(total.cpu(), t)
    t64 = as64(t)
    n = t64 / np.sqrt((t64 ** 2).mean(0) + 1e-6) * as64(w)[:, None]

    def coded(p):
        step = np.abs(p).max(0) / 127
        return np.rint(p / step) * step

    def rounded(p):
        return as64(torch.from_numpy(p).to(TYPES[type]))

    h = rounded(W1 @ coded(n))
    g = coded(act64(h[:F], "silu") * h[F:])
    want = W2 @ g
    # a code next to a border may be the neighbour's: a step of its token, for few; h may round to the neighbour: its half step twice
    step = np.abs(g).max(0) / 127
    bound = 2 * HALF_STEP[type] * (np.abs(W2) @ np.abs(g)) + HALF_STEP[type] * np.abs(want) + 4 * np.abs(W2).max() * step
    assert (np.abs(as64(y) - want) <= bound).all()


def test_feed_forward_block_on_pruned_weights():
    """The norm and the gate in the sparse product's own layout, float32 (features, tokens)."""
    from workloads import generators as gen
    a, b = gen.uniform_positions(512, 256, 0.8, 1), gen.uniform_positions(256, 512, 0.8, 2)
    plans = [spmm.plan_create(c.M, c.K, c.row_ptr, c.col_idx, c.vals) for c in (a, b)]
    dense = []
    for c in (a, b):
        W = np.zeros((c.M, c.K))
        W[np.repeat(np.arange(c.M), np.diff(c.row_ptr)), c.col_idx] = c.vals
        dense.append(W)
    for N in (1, 32, 50):
        x, r, w = norm_case(256, N, "float32", "features", 4)
        y = spmm.norm(x, w, 1e-6, residual=r)
        got = as64(plans[1].execute(spmm.gate(plans[0].execute(y.out), act="gelu").out))
        t = as64(summed(x.cpu(), r.cpu()))
        n = t / np.sqrt((t ** 2).mean(0) + 1e-6) * as64(w)[:, None]
        want = dense[1] @ act64(dense[0] @ n, "gelu")
        S = np.abs(dense[1]) @ (1.2 * np.abs(dense[0]) @ np.abs(n))   # (the activation's slope is at most 1.13)
        assert (np.abs(got - want) <= 2e-5 * S).all()


@pytest.mark.parametrize("N", [1, 12, 40])
def test_streams_and_graphs(N):
    """A side stream, and two graphs of one plan replayed in turn with eager calls between them."""
    D, F = 256, 384
    plans = [plan_of(2 * F, D, 64, 1)[0], plan_of(D, F, 64, 2)[0]]
    inputs = [norm_case(D, N, "bfloat16", "tokens", s) for s in (1, 2)]
    wants = [[o.clone() for o in block(plans, *i, F, torch.bfloat16)] for i in inputs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graphs, outs = [], []
    with torch.cuda.stream(side):
        for i, want in zip(inputs, wants):
            for got, w in zip(block(plans, *i, F, torch.bfloat16), want):
                assert torch.equal(got, w)
    y = spmm.norm(*inputs[0][:1], inputs[0][2], 1e-6, stream=side)
    z = plans[0].execute(y.out, stream=side)
    spmm.gate(z, stream=side)
    side.synchronize()
    assert torch.equal(y.out, spmm.norm(*inputs[0][:1], inputs[0][2], 1e-6).out) and torch.equal(z, plans[0].execute(y.out))
    torch.cuda.synchronize()
    for i in inputs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(block(plans, *i, F, torch.bfloat16))
        graphs.append(graph)
    for _ in range(4):
        for k in (0, 1):
            for o in outs[k]:
                o.fill_(float("nan"))
        graphs[0].replay()
        graphs[1].replay()
        eager = block(plans, *inputs[0], F, torch.bfloat16)
        torch.cuda.synchronize()
        for k in (0, 1):
            for o, w in zip(outs[k], wants[k]):
                assert torch.equal(o, w)
        assert torch.equal(eager[0], wants[0][0])


@pytest.mark.parametrize("type", FLOATS)
@pytest.mark.parametrize("D,N", [(1024, 128), (3000, 270), (5000, 2)])
def test_rows_of_features_in_graphs(type, D, N):
    """Norm and gate with a feature a row of memory: two graphs replayed in turn with eager calls on other sizes between them."""
    inputs = [norm_case(D, N, type, "features", s) for s in (1, 2)]
    other = norm_case(700, 400, type, "features", 3)

    def calls(x, r, w):
        n, c = spmm.norm(x, w, residual=r), spmm.norm(x, w, dtype=torch.int8)
        g = spmm.gate(n.out, x, dtype=torch.int8)
        return [n.out, n.total, c.out, c.scales, g.out, g.scales]

    wants = [[o.clone() for o in calls(*i)] for i in inputs]
    calls(*other)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in inputs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(calls(*i))
        graphs.append(graph)
    for _ in range(4):
        for out in outs:
            for o in out:
                o.fill_(77)
        graphs[1].replay()
        calls(*other)
        graphs[0].replay()
        eager = calls(*inputs[0])
        torch.cuda.synchronize()
        for out, want in zip(outs + [eager], wants + wants[:1]):
            for o, w in zip(out, want):
                assert torch.equal(o, w)


def test_the_benchmarks_blocks():
    """Both blocks of the benchmark run, again with the same bits, and on one residual."""
    import bench
    from workloads import generators as gen
    for tokens in (1, 24):
        passes, plans = bench.block_passes(torch, spmm, gen, 128, 320, tokens)
        (y, t), (z, u) = passes["codes"](), passes["pruned"]()
        assert y.shape == z.shape == t.shape == u.shape == (128, tokens)
        assert y.isfinite().all() and z.isfinite().all() and y.float().std() > 0 and z.std() > 0
        # the sum of two values rounded to bf16, rounded: three half steps
        assert ((t.float() - u).abs() <= 3 * 2.0 ** -8 * 1.01 * (u.abs() + 8)).all()
        for name, want in (("codes", y), ("pruned", z)):
            assert torch.equal(passes[name]()[0], want)
        for plan in plans:
            plan.destroy()


@pytest.mark.parametrize("order", ["tokens", "features"])
@pytest.mark.parametrize("K,N", [(48, 3), (48, 40), (300, 8), (2, 100)])
def test_offsets_past_32_bits(order, K, N):
    """Rows of memory that lie 2^32 elements apart, first to last: the same bits as from rows that lie together."""
    rows, row = (N, K) if order == "tokens" else (K, N)
    ld = max(row, 2 ** 32 // (rows - 1) + 1)

    def apart(like):
        far = torch.empty(((rows - 1) * ld + row,), dtype=like.dtype, device="cuda").as_strided((rows, row), (ld, 1))
        far.copy_(like if order == "features" else like.t())
        return far if order == "features" else far.t()

    x = torch.randn((K, N), device="cuda").bfloat16()
    near = x if order == "features" else x.t().contiguous().t()
    far, w = apart(x), torch.ones(K, device="cuda")
    plan, _ = plan_of(50, K, 64, 3)
    assert torch.equal(plan.execute(far), plan.execute(near))
    out = apart(torch.zeros_like(x))
    n, m = spmm.norm(far, w, residual=near, out=out), spmm.norm(near, w, residual=near)
    assert n.out is out and torch.equal(out, m.out) and torch.equal(n.total, m.total)
    for dtype in (torch.bfloat16, torch.int8):
        g, h = spmm.gate(far, near, dtype=dtype), spmm.gate(near, near, dtype=dtype)
        assert torch.equal(g.out, h.out) and (dtype != torch.int8 or torch.equal(g.scales, h.scales))
    if order == "tokens":
        q = torch.randint(-127, 128, (K, N), dtype=torch.int8, device="cuda")
        s = torch.rand(N, device="cuda")
        assert torch.equal(plan.execute(apart(q), scales=s), plan.execute(q.t().contiguous().t(), scales=s))


def test_the_same_inputs_give_the_same_bits():
    for M, K, N in ((300, 4096, 1), (300, 4096, 9), (64, 8192, 64)):
        plan, _ = plan_of(M, K, 128, 5)
        B = torch.randn((K, N), device="cuda")
        first = plan.execute(B)
        for _ in range(5):
            torch.randn(1 << 20, device="cuda")
            assert torch.equal(plan.execute(B), first)


# ---- refusals -------------------------------------------------------------------------------------------------

def test_what_the_product_refuses():
    plan, _ = plan_of(6, 10, 32, 1)
    B = torch.ones((10, 4), device="cuda")
    q, s = torch.ones((4, 10), dtype=torch.int8, device="cuda").t(), torch.ones(4, device="cuda")
    for bad in (B.cpu(), B.double(), B.long(), B[0], B[None], B[:9], torch.ones((20, 8), device="cuda")[::2, ::2], B[:, :1].expand(10, 4), torch.ones((10, 4), device="cuda").to_sparse()):
        with pytest.raises(ValueError, match="B "):
            plan.execute(bad)
    C = torch.empty((6, 4), device="cuda")
    for bad in (C.cpu(), C.double(), q[:6], C[:5], C[0], torch.empty((12, 8), device="cuda")[::2, ::2]):
        with pytest.raises(ValueError, match="C "):
            plan.execute(B, bad)
    for kw in (dict(scales=s), dict(dtype=torch.int8), dict(dtype=torch.float64), dict(C=C, dtype=torch.float16)):
        with pytest.raises(ValueError):
            plan.execute(B, **kw)
    for scales in (None, s.cpu(), s.half(), s[:3], torch.ones((1, 4), device="cuda"), torch.ones(8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="scales"):
            plan.execute(q, scales=scales)
    with pytest.raises(ValueError, match="one token a row"):
        plan.execute(q.contiguous(), scales=s)
    for bad in (np.ones((10, 4), np.float32), 3, None):
        with pytest.raises(TypeError):
            plan.execute(bad)
    with pytest.raises(TypeError):
        plan.execute(B, dtype="float32")
    with pytest.raises(spmm.SpmmError) as err:
        plan.execute(torch.empty((10, 0), device="cuda"))
    assert err.value.status == spmm.binding.SPMM_ERR_INVALID_ARG
    both = torch.ones((10, 4), device="cuda")
    with pytest.raises(spmm.SpmmError) as err:
        plan.execute(both, both[:6])
    assert err.value.status == spmm.binding.SPMM_ERR_INVALID_ARG
    assert not plan.execute(B.clone().requires_grad_()).requires_grad
    plan.destroy()
    plan.destroy()
    with pytest.raises(spmm.SpmmError):
        plan.execute(B)


def test_the_product_refuses_an_output_over_its_scales():
    plan, _ = plan_of(6, 10, 32, 1)
    q, memory = torch.ones((4, 10), dtype=torch.int8, device="cuda").t(), torch.ones(64, device="cuda")
    for at in (0, 20, 23):
        with pytest.raises(spmm.SpmmError) as err:
            plan.execute(q, C=memory[:24].view(6, 4), scales=memory[at:at + 4])
        assert err.value.status == spmm.binding.SPMM_ERR_INVALID_ARG
    assert plan.execute(q, C=memory[:24].view(6, 4), scales=memory[24:28]).isfinite().all()


def test_what_norm_and_gate_refuse():
    x, w = torch.ones((10, 4), device="cuda"), torch.ones(10, device="cuda")
    for bad in (x.cpu(), x.double(), x.to(torch.int8), x[0], torch.ones((20, 8), device="cuda")[::2, ::2], x[:, :1].expand(10, 4), x[:0], x[:, :0]):
        with pytest.raises(ValueError):
            spmm.norm(bad, w)
        with pytest.raises(ValueError):
            spmm.gate(bad)
    for bad in (w.cpu(), w.double(), w[:9], x, torch.ones(20, device="cuda")[::2]):
        with pytest.raises(ValueError, match="weight"):
            spmm.norm(x, bad)
    for bad in (x.half(), x[:9], x.cpu()):
        for call in (lambda: spmm.norm(x, w, residual=bad), lambda: spmm.norm(x, w, total=bad), lambda: spmm.gate(x, bad)):
            with pytest.raises(ValueError):
                call()
    for bad in (x.cpu(), x[:9], x.double()):
        for call in (lambda: spmm.norm(x, w, out=bad), lambda: spmm.gate(x, out=bad)):
            with pytest.raises(ValueError, match="out"):
                call()
    s = torch.ones(4, device="cuda")
    for kw in (dict(scales=s), dict(dtype=torch.int8, scales=s[:3]), dict(dtype=torch.float64), dict(dtype=torch.int8, out=torch.empty_like(x))):
        with pytest.raises(ValueError):
            spmm.norm(x, w, **kw)
        with pytest.raises(ValueError):
            spmm.gate(x, **kw)
    with pytest.raises(ValueError):
        spmm.gate(x, act="tanh")
    turned = torch.ones((4, 10), device="cuda").t()
    invalid, unsupported = spmm.binding.SPMM_ERR_INVALID_ARG, spmm.binding.SPMM_ERR_UNSUPPORTED
    for status, call in ((unsupported, lambda: spmm.norm(x, w, residual=turned)), (unsupported, lambda: spmm.norm(x, w, out=turned)), (unsupported, lambda: spmm.norm(x, w, total=turned)),
                         (unsupported, lambda: spmm.gate(x, turned)), (unsupported, lambda: spmm.gate(x, out=torch.empty((10, 4), dtype=torch.int8, device="cuda"))),
                         (invalid, lambda: spmm.norm(x, w, out=x)), (invalid, lambda: spmm.gate(x, out=x)), (invalid, lambda: spmm.norm(x, w, -1.0)),
                         (invalid, lambda: spmm.norm(x, w, float("nan"))), (invalid, lambda: spmm.norm(x[:9], w[:9], total=x[1:]))):
        with pytest.raises(spmm.SpmmError) as err:
            call()
        assert err.value.status == status
    for call in (lambda: spmm.norm(3, w), lambda: spmm.norm(x, None), lambda: spmm.gate(None), lambda: spmm.norm(x, w, dtype=3)):
        with pytest.raises(TypeError):
            call()
