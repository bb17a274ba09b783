"""The operators beside the sparse product on the GPU: values at the borders of what the header defines, in every path."""
import numpy as np
import pytest
import torch

import paper_2506_15174_amd as spmm
from layers_reference import HALF_STEP, TYPES, as64, placed, weights

pytestmark = pytest.mark.gpu

FLOATS = ("float32", "float16", "bfloat16")
# features, tokens, order in memory: one wave a token, one workgroup of 256 or 1024, long rows; rows of features in one launch and in two
ROWS_PATHS = [(40, 6, "tokens"), (2000, 3, "tokens"), (4100, 3, "tokens"), (8000, 600, "tokens"), (16000, 3, "tokens"), (33000, 3, "tokens"), (70000, 2, "tokens"),
              (40, 6, "features"), (1024, 128, "features"), (4096, 6, "features"), (5000, 6, "features"), (3000, 270, "features")]


@pytest.fixture(autouse=True)
def gpu():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    spmm.load()


@pytest.mark.parametrize("type", FLOATS)
@pytest.mark.parametrize("K,N,order", ROWS_PATHS)
def test_codes_of_a_token_of_zeros_without_eps(type, K, N, order):
    """P is 0: codes and scale are 0 whatever eps is; so they are where the weights make it 0."""
    x = placed(np.random.default_rng(K).standard_normal((K, N)), type, order)
    x[:, 0] = 0
    w = torch.ones(K, device="cuda")
    for eps in (0.0, 1e-6):
        y = spmm.norm(x, w, eps, dtype=torch.int8)
        assert y.scales[0] == 0 and (y.out[:, 0] == 0).all() and y.scales.isfinite().all() and (y.scales[1:] > 0).all()
        n = spmm.norm(x, torch.zeros_like(w), eps, dtype=torch.int8)
        assert (n.scales == 0).all() and (n.out == 0).all()
    g = spmm.gate(x, x, dtype=torch.int8)
    assert g.scales[0] == 0 and (g.out[:, 0] == 0).all() and (g.scales[1:] > 0).all()


# ---- sizes at which a launch takes a second axis ----------------------------------------------------------------

@pytest.mark.parametrize("type,N", [("float32", 2 ** 29 + 77), ("bfloat16", 2 ** 30 + 77)])
def test_more_tokens_by_features_than_one_axis_of_a_launch_has(type, N):
    """2^24 tiles side by side: windows of tokens are as from a call on the window alone, which goes in one launch, and the rest is written.

    The statistics of the two need not have the same bits: one of the two squares may be added in one rounding with its product (t_0^2 + t_1^2 as a multiply-add) or in two.  Each
    side's factor has at most two roundings in the sum, one in the mean and one with eps, all four halved by the root, then one in the root and one in the quotient: 4 half
    steps.  A scale has two more, its product with P and the division by 127, and a value of the output two, its products with t and the weight: 6 on each side, 12 between them, and twice the output's own."""
    near = dict(rtol=12 * 2.0 ** -24 * 1.01, atol=0)
    a, w = torch.empty((2, N), dtype=TYPES[type], device="cuda"), torch.tensor([1.5, -0.75], device="cuda")
    for k in range(2):
        a[k].uniform_(0.5, 2.0)
    y = spmm.norm(a, w, dtype=torch.int8)
    windows = [0, 2 ** 25 - 700, 2 ** 26 - 700, N // 2 - 333, N - 2000]
    for n in windows:
        z = spmm.norm(a[:, n:n + 2000], w, dtype=torch.int8)
        assert torch.equal(y.out[:, n:n + 2000], z.out) and torch.allclose(y.scales[n:n + 2000].double(), z.scales.double(), **near)
    assert y.scales.min() > 0 and y.scales.max() < 1
    for n in range(0, N, 2 ** 27):
        assert (y.out[:, n:n + 2 ** 27].abs().amax(0) == 127).all()
    del y, z
    y = spmm.norm(a, w)
    for n in windows:
        z = spmm.norm(a[:, n:n + 2000], w)
        assert torch.allclose(y.out[:, n:n + 2000].double(), z.out.double(), rtol=(12 * 2.0 ** -24 + (2 * HALF_STEP[type] if type != "float32" else 0)) * 1.01, atol=0)
    # r lies in 1/2 .. 2: no value of the output is 0
    for n in range(0, N, 2 ** 27):
        assert (y.out[0, n:n + 2 ** 27] > 0.3).all() and (y.out[1, n:n + 2 ** 27] < -0.1).all()
    del y
    y = spmm.gate(a, act="relu", dtype=torch.int8)
    for n in windows:
        z = spmm.gate(a[:, n:n + 2000], act="relu", dtype=torch.int8)
        assert torch.equal(y.out[:, n:n + 2000], z.out) and torch.equal(y.scales[n:n + 2000], z.scales)
    assert y.scales.min() > 0


# ---- one token ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("K", [1, 7, 300, 5000])
def test_one_token_in_columns_with_gaps_and_without(K):
    """Any of the tensors may be a column of a wider matrix, the sum too.  With gaps the squares are added up in another order: a chain of at most K / 16 + 256 roundings on each side,
    halved by the root, then eight single ones."""
    near = dict(rtol=2 * ((K / 16 + 256) / 2 + 8) * 2.0 ** -24, atol=0)
    rng = np.random.default_rng(K)
    values = [torch.from_numpy(rng.standard_normal((K, 1))).float().cuda() for _ in range(2)]
    w = torch.ones(K, device="cuda")
    want = spmm.norm(values[0], w, residual=values[1])
    codes = spmm.norm(values[0], w, residual=values[1], dtype=torch.int8)
    for gaps in range(16):
        def column(n, value=None):
            t = torch.full((K, 4), 7.0, device="cuda")[:, 1:2] if gaps >> n & 1 else torch.full((K, 1), 7.0, device="cuda")
            return t if value is None else t.copy_(value)
        x, r = column(0, values[0]), column(1, values[1])
        y = spmm.norm(x, w, residual=r, total=column(2), out=column(3))
        assert torch.equal(y.total, want.total) and torch.allclose(y.out, want.out, **near)
        z = spmm.norm(x, w, residual=r, total=column(2), dtype=torch.int8)
        assert torch.equal(z.total, want.total) and torch.equal(z.out, codes.out) and torch.allclose(z.scales, codes.scales, **near)
        assert torch.equal(spmm.gate(x, r, out=column(3)).out, spmm.gate(values[0], values[1]).out)


# ---- outputs between the rows of inputs ----------------------------------------------------------------------------

def beside(type, order, sizes, N):
    """Tensors of sizes[i] features x N side by side in the rows of one piece of memory, and what the rows hold behind them."""
    if order == "tokens":
        memory = torch.full((N, sum(sizes) + 3), 7.0, dtype=TYPES[type], device="cuda")
        at = [sum(sizes[:i]) for i in range(len(sizes))]
        return [memory[:, a:a + s].t() for a, s in zip(at, sizes)], memory[:, sum(sizes):]
    rows = max(sizes)
    memory = torch.full((rows, len(sizes) * N + 3), 7.0, dtype=TYPES[type], device="cuda")
    return [memory[:s, i * N:(i + 1) * N] for i, s in enumerate(sizes)], memory[:, len(sizes) * N:]


@pytest.mark.parametrize("type", FLOATS)
@pytest.mark.parametrize("order", ["tokens", "features"])
@pytest.mark.parametrize("M,K,N", [(50, 300, 3), (50, 300, 20), (300, 500, 150), (2100, 300, 600)])
def test_outputs_between_the_rows_of_inputs(type, order, M, K, N):
    """B and C, and x, residual, sum and output, in one piece of memory; what lies between stays."""
    codes, scales, zeros, _ = weights(M, K, 64, K + N)
    plan = spmm.quant_plan_create(M, K, codes, scales, zeros, group=64)
    a, r = (torch.from_numpy(np.random.default_rng(s).standard_normal((K, N))).to(TYPES[type]).cuda() for s in (1, 2))
    w = torch.ones(K, device="cuda")
    (B, C), rest = beside(type, order, (K, M), N)
    assert torch.equal(plan.execute(B.copy_(a), C), plan.execute(a if order == "features" else a.t().contiguous().t())) and torch.equal(B, a) and (rest == 7).all()
    (x, y, t, o), rest = beside(type, order, (K,) * 4, N)
    got, want = spmm.norm(x.copy_(a), w, residual=y.copy_(r), total=t, out=o), spmm.norm(x.clone(), w, residual=y.clone())
    assert torch.equal(got.out, want.out) and torch.equal(got.total, want.total) and torch.equal(x, a) and torch.equal(y, r) and (rest == 7).all()
    o.fill_(7)
    assert torch.equal(spmm.gate(x, y, out=o).out, spmm.gate(x.clone(), y.clone()).out) and torch.equal(x, a) and torch.equal(y, r) and torch.equal(t, want.total) and (rest == 7).all()


# ---- views that torch has not made yet -----------------------------------------------------------------------------

def test_views_whose_negation_is_still_to_be_made():
    """Their memory holds the other sign: refused wherever a tensor goes in or out, taken once they are made."""
    codes, scales, _, W = weights(6, 10, 32, 1, zeros=False)
    plan = spmm.quant_plan_create(6, 10, codes, scales, group=32)
    part = torch.randn((10, 1, 2), device="cuda")
    lazy = torch.view_as_complex(part).conj().imag
    assert lazy.is_neg() and lazy.shape == (10, 1)
    x, w = torch.randn((10, 1), device="cuda"), torch.ones(10, device="cuda")
    out = torch.view_as_complex(torch.zeros((6, 1, 2), device="cuda")).conj().imag
    one = torch.view_as_complex(torch.ones((1, 2), device="cuda")).conj().imag
    q = torch.ones((10, 1), dtype=torch.int8, device="cuda")
    for call in (lambda: plan.execute(lazy), lambda: plan.execute(x, out), lambda: plan.execute(q, scales=one), lambda: spmm.norm(lazy, w), lambda: spmm.norm(x, w, residual=lazy),
                 lambda: spmm.norm(x, w, total=lazy), lambda: spmm.norm(x, w, out=lazy), lambda: spmm.norm(x[:1], one), lambda: spmm.norm(x, w, dtype=torch.int8, scales=one),
                 lambda: spmm.gate(lazy), lambda: spmm.gate(x, lazy), lambda: spmm.gate(x, out=lazy), lambda: spmm.gate(x, dtype=torch.int8, scales=one)):
        with pytest.raises(ValueError, match="negation"):
            call()
    made = lazy.resolve_neg()
    assert torch.equal(made, -part[:, :, 1]) and torch.equal(plan.execute(made), plan.execute(-part[:, :, 1]))
    assert torch.equal(spmm.norm(made, w).out, spmm.norm((-part[:, :, 1]).contiguous(), w).out)


# ---- the norm's statistics -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("type", FLOATS)
@pytest.mark.parametrize("K,N,order,step", [(8000, 3, "tokens", 512), (16000, 3, "tokens", 512), (30000, 3, "tokens", 512), (70000, 2, "tokens", 512), (8000, 600, "tokens", 512),
                                            (1024, 128, "features", 16), (1024, 128, "features", 32), (4096, 6, "features", 64), (5000, 270, "features", 128), (8192, 270, "features", 128)])
def test_what_waves_leave_is_not_lost_beside_a_large_square(type, K, N, order, step):
    """One square of 2^24 and single ones in other waves' or tiles' shares, 2^24 + 15 where there are 16 waves: in fp32 none of the ones would move the sum.

    The sum is exact then.  The mean is rounded (a half step, halved by the root), the root, the quotient, the product with t: 3.5 half steps of fp32; a scale has the division by
    127 besides."""
    x = torch.zeros((K, N), dtype=torch.float64)
    ones = torch.arange(step, min(K, 16 * step if order == "tokens" or step < 100 else K), step)
    for n in range(N):
        x[ones[: max(1, len(ones) - n % 3)], n] = 1.0
    x[0] = 4096.0
    d = placed(x.numpy(), type, order)
    w = torch.ones(K, device="cuda")
    f = 1 / np.sqrt((x.numpy() ** 2).mean(0))
    y = spmm.norm(d, w, 0.0, dtype=torch.float32)
    assert (np.abs(as64(y.out) - x.numpy() * f) <= 3.5 * 2.0 ** -24 * 1.01 * x.numpy() * f).all()
    z = spmm.norm(d, w, 0.0, dtype=torch.int8)
    assert (np.abs(as64(z.scales) - 4096 * f / 127) <= 4.5 * 2.0 ** -24 * 1.01 * 4096 * f / 127).all()


# ---- the gate's activation -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("order", ["tokens", "features"])
def test_silu_is_as_exact_for_large_arguments(order):
    """In half steps of fp32 (2^-24), relative: the exponential's instruction 2, what its argument's rounding left 1 (and less than 0.1 for all that is neglected of it), the product with x 1, the sum
    1 + e 1, the reciprocal's instruction 2, the quotient 1, the product with b 1: 9.1.  Below 2^-126 an exponential may count as 0."""
    F, N = 4096, 16
    rng = np.random.default_rng(11)
    a = placed(rng.uniform(-100, 100, (F, N)) * rng.uniform(0, 1, (1, N)), "float32", order)
    b = placed(rng.uniform(0.5, 2, (F, N)), "float32", order)
    a64, b64 = as64(a), as64(b)
    want = a64 * np.exp(np.minimum(a64, 0)) / (1 + np.exp(-np.abs(a64)))
    for second in (None, b):
        w = want if second is None else want * b64
        got = as64(spmm.gate(a, second).out)
        assert (np.abs(got - w) <= 9.1 * 2.0 ** -24 * np.abs(w) + 2.0 ** -126 * 128 * 2).all()
    y = spmm.gate(a, b, dtype=torch.int8)
    most = np.abs(want * b64).max(0)
    # P, and its division by 127
    assert (np.abs(as64(y.scales) - most / 127) <= 10.1 * 2.0 ** -24 * most / 127).all()


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_small_results_of_the_gate(act):
    """x exp(x) at -86, where 1 + exp(86) would have a reciprocal below the normal numbers.  The instruction for the exponential gives 0 for results below 2^-126, as exp(-87.5) = 1.0e-38 is (2^-126 is
    1.18e-38): there the result is off by all of itself, |x| exp(x), which is less than |x| 2^-126."""
    x = np.array([[-80.0], [-86.0], [-87.5]]) if act == "silu" else np.array([[-9.0], [-10.0], [-10.3]])
    got = as64(spmm.gate(placed(x, "float32", "features"), act=act).out)
    x = as64(placed(x, "float32", "features", device="cpu"))
    u = x if act == "silu" else 2 * np.sqrt(2 / np.pi) * (x + 0.044715 * x ** 3)
    want = x * np.exp(u) / (1 + np.exp(u))
    # gelu's u has four roundings of its own, of at most |u| 2^-24 each (its constants' among them), and an error of u is one of the result
    rel = 9.1 * 2.0 ** -24 + (0 if act == "silu" else 5 * np.abs(u) * 2.0 ** -24)
    assert (np.abs(got - want) <= rel * np.abs(want) + np.where(np.exp(u) < 2.0 ** -126, np.abs(x) * 2.0 ** -126, 0)).all()
