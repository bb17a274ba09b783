"""Plain implementations in 64 bits of the operators beside the sparse product, and their inputs (numpy)."""
import numpy as np
import torch

TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16, "int8": torch.int8}
HALF_STEP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
SMALLEST = {"float32": 2.0 ** -149, "float16": 2.0 ** -24, "bfloat16": 2.0 ** -133}


def weights(M, K, group, seed, zeros=True, whole=False):
    """(codes in bytes, scales, zeros or None, W in 64 bits); whole: scales are powers of two."""
    rng = np.random.default_rng(seed)
    groups = -(-K // group)
    q = rng.integers(0, 16, (M, K + K % 2), dtype=np.uint8)
    codes = q[:, ::2] | (q[:, 1::2] << 4)   # (the high half behind an odd last column holds anything)
    scales = 2.0 ** rng.integers(-2, 3, (M, groups)) if whole else rng.uniform(0.001, 0.1, (M, groups)) * rng.choice((-1, 1), (M, groups))
    scales = scales.astype(np.float32)
    z = rng.integers(0, 16, (M, groups), dtype=np.uint8) if zeros else None
    of = np.arange(K) // group
    W = (q[:, :K].astype(np.float64) - (z[:, of] if zeros else 8)) * scales[:, of].astype(np.float64) if K else np.zeros((M, 0))
    return codes, scales, z, W


def placed(a, type, order, pad=0, offset=0, device="cuda"):
    """The 2-D array on the device in the order given, rows of memory `pad` elements longer than needed, and starting `offset` elements into its memory."""
    a = torch.as_tensor(np.ascontiguousarray(a)).to(TYPES[type])
    rows, cols = a.shape
    if order == "tokens":
        return placed(a.t().numpy() if type != "bfloat16" else a.t().float().numpy(), type, "features", pad, offset, device).t()
    ld = cols + pad
    memory = torch.empty(offset + rows * ld, dtype=TYPES[type])
    if type == "int8":
        memory.fill_(77)
    else:
        memory.fill_(float("nan"))
    view = memory.to(device)[offset:].view(rows, ld)[:, :cols]
    view.copy_(a)
    return view


def as64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def act64(x, act):
    with np.errstate(over="ignore"):
        if act == "silu":
            return x / (1 + np.exp(-x))
        if act == "gelu":
            return x / (1 + np.exp(-2 * np.sqrt(2 / np.pi) * (x + 0.044715 * x ** 3)))   # (1 + tanh(u)) / 2
    return np.maximum(x, 0)


def summed(x, r):
    """x + r in 32 bits, rounded to their type (torch tensors on the host)."""
    return x if r is None else (x.float() + r.float()).to(x.dtype)


def codes_of(p):
    """Codes and the largest magnitude of a token's fp32 values p (features, tokens), as the header defines them."""
    most = np.abs(p).max(axis=0)
    up = np.where(most < np.float32(2.0 ** -100), np.float32(2.0 ** 100), np.float32(1))
    with np.errstate(divide="ignore", invalid="ignore"):
        steps = np.where(most > 0, np.float32(127) / (most * up), np.float32(0)).astype(np.float32)
    return np.rint(p * up * steps).astype(np.int8), most
