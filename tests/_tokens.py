"""Plain implementations in 64 bits of what the token operators compute, and the bounds their results are held to."""
import numpy as np
import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a step, relative
U32 = 2.0 ** -24


def stored(dtype, ref):
    """What storing ref in dtype may be off by: half a step, which is UNIT relative to a normal number, and for float16, whose steps below 2^-14 are all
    2^-24, 2^-25 there."""
    return UNIT[dtype] * ref.abs() + (2.0 ** -25 if dtype == torch.float16 else 0.0)


def philox(counter, key):
    """Philox4x32-10 of one counter (four words) or arrays of them."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k0, k1 = (int(k) for k in key)
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def factors(rows, width, p, seed, offset):
    """What dropout multiplies [rows, width] by, float64."""
    thr = round(p * 65536)
    groups = -(-width // 8)
    col, row = np.meshgrid(np.arange(groups), np.arange(rows))
    o = offset % (1 << 64)
    words = philox((col, row, np.full_like(col, o & 0xFFFFFFFF, dtype=np.uint64), np.full_like(col, o >> 32, dtype=np.uint64)), (seed & 0xFFFFFFFF, seed >> 32))
    u = np.stack([x for w in words for x in (w & np.uint64(0xFFFF), w >> np.uint64(16))], -1).reshape(rows, groups * 8)[:, :width]
    return torch.from_numpy((u >= thr).astype(np.float64) * (65536.0 / (65536 - thr) if thr < 65536 else 0.0))


def rows_at(values, stride, offset=0):
    """The 2-D tensor on the GPU with rows `stride` elements apart, `offset` elements into its memory; what lies between is NaN."""
    n, C = values.shape
    buf = torch.full((max(1, n) * stride + offset,), float("nan"), dtype=values.dtype, device="cuda")
    v = buf[offset:].as_strided((n, C), (stride, 1))
    v.copy_(values)
    return v


def close(got, ref, bound, what=""):
    """|got - ref| <= bound, element by element; NaN nowhere that ref is not."""
    got, bad = got.double(), None
    err = (got - ref).abs()
    bad = ~(err <= bound)
    if bad.any():
        i = tuple(int(x) for x in torch.nonzero(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {float(got[i])!r}, expected {float(ref[i])!r} within {float(torch.as_tensor(bound).expand_as(err)[i]):.3e}")
