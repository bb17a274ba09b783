"""The product with 4-bit weights, the norm and the gate on the GPU in the paths of many tokens and many rows: each with padded and offset rows, every order and type of output, infinities and NaN, values
that are no whole numbers, and more tokens than one launch has."""
import numpy as np
import pytest
import torch

import paper_2506_15174_amd as spmm
from layers_reference import TYPES, as64, placed, weights
from test_gpu_layers import check_product, plan_of

pytestmark = pytest.mark.gpu

FLOATS = ("float32", "float16", "bfloat16")


@pytest.fixture(autouse=True)
def gpu():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    spmm.load()


# ---- fp32 in three parts ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("K,group", [(1024, 128), (1100, 64), (1100, 32), (2100, 128)])
@pytest.mark.parametrize("M", [40, 300, 600, 1100, 8200, 16400])
def test_all_24_bits_of_a_value_arrive(M, K, group):
    """One value a token, in another column for each, times a weight that is a power of two: the three parts add up to the value, so every bit of the result is known.  Rows and tokens for every
    shape of wave, up to 16 tokens read along the rows, in one launch and in two."""
    rng = np.random.default_rng(M + K)
    q = rng.choice(np.array([0, 4, 6, 7, 8, 9, 10, 12], np.uint8), (M, K + K % 2))   # less 8: powers of two and 0
    scales = (2.0 ** rng.integers(-3, 4, (M, -(-K // group)))).astype(np.float32)
    plan = spmm.quant_plan_create(M, K, q[:, ::2] | (q[:, 1::2] << 4), scales, group=group)
    W = torch.from_numpy((q[:, :K].astype(np.float32) - 8) * scales[:, np.arange(K) // group]).cuda()
    for N in (1, 2, 4, 16, 17, 32, 130, 600):
        value = (rng.integers(2 ** 23, 2 ** 24, N) | 1).astype(np.float32) * 2.0 ** rng.integers(-40, 20, N).astype(np.float32) * rng.choice((-1, 1), N).astype(np.float32)
        for last in (False, True):
            # (columns of all blocks; then the last block's only)
            column = rng.integers(K - (K - 1) % 128 - 1 if last else 0, K, N)
            B = np.zeros((K, N), np.float32)
            B[column, np.arange(N)] = value
            want = W[:, torch.from_numpy(column).cuda()] * torch.from_numpy(value.astype(np.float32)).cuda()
            for order in ("tokens", "features"):
                assert torch.equal(plan.execute(placed(B, "float32", order)), want), (N, order, last)


# ---- many tokens ---------------------------------------------------------------------------------------------------

# rows, columns, tokens: waves of one and two tiles of rows by two of tokens; fp32's four by four and two by four; teams of two, four and eight
MANY = [(300, 700, 40), (1100, 520, 600), (620, 391, 600), (2100, 650, 130)]
TEAMS = [(4090, 391, 500), (4080, 650, 1001), (4070, 300, 2040)]


@pytest.mark.parametrize("type", FLOATS + ("int8",))
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True), (256, True)])
@pytest.mark.parametrize("M,K,N", MANY + TEAMS)
def test_values_in_paths_of_many_tokens(type, group, zeros, M, K, N):
    check_product(M, K, N, group, type, "tokens", M + group, zeros=zeros)
    if type != "int8":
        check_product(M, K, N, group, type, "features", M + group, zeros=zeros)


@pytest.mark.parametrize("type", FLOATS + ("int8",))
@pytest.mark.parametrize("out", FLOATS)
@pytest.mark.parametrize("c_order", ["tokens", "features"])
@pytest.mark.parametrize("M,K,N", MANY[:2] + TEAMS[:2])
def test_strides_offsets_and_outputs_in_paths_of_many_tokens(type, out, c_order, M, K, N):
    for pad, offset in ((1, 1), (5, 3)):
        check_product(M, K, N, 64, type, "tokens", 7 + pad, out=out, c_order=c_order, pad=pad, offset=offset, c_pad=pad)
        if type != "int8":
            check_product(M, K, N, 64, type, "features", 8 + pad, out=out, c_order=c_order, pad=pad, offset=offset, c_pad=pad)


@pytest.mark.parametrize("type", FLOATS + ("int8",))
@pytest.mark.parametrize("M,K,N", [(300, 1, 200), (5, 31, 300), (2000, 33, 300), (20, 129, 1000), (1, 1, 5000), (1, 5000, 100)])
def test_odd_sizes_of_many_tokens(type, M, K, N):
    for order in ("tokens", "features") if type != "int8" else ("tokens",):
        check_product(M, K, N, 32, type, order, M + K)


@pytest.mark.parametrize("type", FLOATS)
@pytest.mark.parametrize("order", ["tokens", "features"])
@pytest.mark.parametrize("M,K,N", MANY + TEAMS)
def test_infinities_and_nan_in_paths_of_many_tokens(type, order, M, K, N):
    """Each in one token, of the first, a middle and the last tile: its elements are what the plain sum gives, and no other token sees it."""
    plan, W = plan_of(M, K, 64, 3)
    B = np.random.default_rng(4).standard_normal((K, N))
    special = {0: {7: np.inf}, 5: {K - 1: np.nan}, N // 2: {3: -np.inf, K - 2: np.inf}, N - 1: {K // 2: -np.inf}}
    clean = as64(plan.execute(placed(B, type, order), dtype=torch.float32))
    for n, values in special.items():
        for k, v in values.items():
            B[k, n] = v
    d = placed(B, type, order)
    got, B64 = as64(plan.execute(d, dtype=torch.float32)), as64(d)
    others = np.setdiff1d(np.arange(N), list(special))
    assert np.array_equal(got[:, others], clean[:, others])
    for n in special:
        with np.errstate(invalid="ignore"):
            want = (W * B64[:, n]).sum(1)
        assert np.array_equal(np.isnan(got[:, n]), np.isnan(want)) and not np.isfinite(got[:, n][~np.isfinite(want)]).any()
        inf = np.isinf(want)
        assert np.array_equal(got[inf, n], want[inf])


# ---- more than one launch has --------------------------------------------------------------------------------------

@pytest.mark.parametrize("type,order", [("int8", "tokens"), ("float16", "tokens"), ("float16", "features"), ("float32", "features")])
def test_products_of_more_tokens_than_a_launch_has(type, order):
    """65528 tiles of 16 tokens go at a time; all is in whole numbers, so every column is known."""
    M, K, N = 20, 32, 65528 * 16 + 37
    codes, scales, zeros, W = weights(M, K, 32, 5, whole=True)
    plan = spmm.quant_plan_create(M, K, codes, scales, zeros, group=32)
    B = torch.randint(-4, 5, (N, K) if order == "tokens" else (K, N), device="cuda").to(TYPES[type])
    B = B.t() if order == "tokens" else B
    s = (2.0 ** torch.randint(-3, 4, (N,), device="cuda")) if type == "int8" else None
    for c_order in ("tokens", "features"):
        C = torch.full((N, M) if c_order == "tokens" else (M, N), float("nan"), device="cuda")
        C = C.t() if c_order == "tokens" else C
        plan.execute(B, C, scales=s)
        for n in range(0, N, 2 ** 18):
            want = torch.from_numpy(W).cuda() @ B[:, n:n + 2 ** 18].double()
            assert torch.equal(C[:, n:n + 2 ** 18].double(), want if s is None else want * s[n:n + 2 ** 18].double())


@pytest.mark.parametrize("K,N", [(8, 4 * 2 ** 20 + 5), (520, 2 ** 20 + 3)])
@pytest.mark.parametrize("out", ["bfloat16", "int8"])
def test_norms_of_more_tokens_than_a_row_of_workgroups_has(K, N, out):
    """Four tokens a workgroup, or one, and more than 2^20 workgroups: the tokens on either side of the border as in a call of their own, and all of them written."""
    x = torch.empty((N, K), dtype=torch.bfloat16, device="cuda").uniform_(0.5, 2).t()
    w = torch.ones(K, device="cuda")
    y = spmm.norm(x, w, dtype=TYPES[out])
    border = 2 ** 20 * (4 if K <= 512 else 1)
    for n in (0, border - 100, N - 50):
        z = spmm.norm(x[:, n:n + 200], w, dtype=TYPES[out])
        assert torch.equal(y.out[:, n:n + 200], z.out) and (out != "int8" or torch.equal(y.scales[n:n + 200], z.scales))
    # of values in 1/2 .. 2 none is below a quarter of the largest
    for n in range(0, N, 2 ** 18):
        part = y.out[:, n:n + 2 ** 18].float()
        assert ((part >= (31 if out == "int8" else 0.24)) & (part <= 127)).all()


def test_gates_of_more_elements_than_a_row_of_workgroups_has():
    """2^31 elements and some, in one piece and in short rows with gaps."""
    a = torch.empty((2 ** 20 + 3, 2050), dtype=torch.bfloat16, device="cuda").normal_()
    for part in (a[:, :2048].reshape(-1, 2048), a[:, :2048]):
        x = part.t()
        out = torch.full((x.shape[1], x.shape[0]), float("nan"), dtype=torch.bfloat16, device="cuda").t()
        spmm.gate(x, act="relu", out=out)
        for n in range(0, x.shape[1], 2 ** 17):
            assert torch.equal(out[:, n:n + 2 ** 17], x[:, n:n + 2 ** 17].clamp(min=0))
