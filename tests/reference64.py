"""Plain 64-bit forms of the operators on blocks of 128 and on experts, for the tests.  No code of the library."""
import numpy as np
import torch

F8 = torch.float8_e4m3fn


def decode(q):
    """E4M3 bytes (any device) as float64"""
    return q.cpu().contiguous().view(F8).to(torch.float64).numpy()


def spread(s, n, axis, block=128):
    return np.repeat(s, block, axis=axis).take(np.arange(n), axis=axis)


def quant_block(x, br, bc):
    """float32 [rows x cols] in blocks of br x bc: codes (uint8) and scales (float32), step by step as the definition rounds"""
    x = np.asarray(x, np.float32)
    rows, cols = x.shape
    r, c = -(-rows // br), -(-cols // bc)
    wide = np.zeros((r * br, c * bc), np.float32)
    wide[:rows, :cols] = np.abs(x)
    amax = wide.reshape(r, br, c, bc).max(axis=(1, 3))
    with np.errstate(divide="ignore", over="ignore", under="ignore"):
        s = np.where(amax > 0, amax / np.float32(448.0), np.float32(1.0)).astype(np.float32)
        inv = np.minimum(np.float32(1.0) / s, np.finfo(np.float32).max).astype(np.float32)
        y = x * spread(spread(inv, rows, 0, br), cols, 1, bc)
    q = torch.from_numpy(np.clip(y, -448.0, 448.0).astype(np.float32)).to(F8).view(torch.uint8).numpy()
    return q, s


def mx_values(q, e):
    """codes with an exponent byte per 32 columns (None: 1) as float64"""
    v = decode(q)
    return v if e is None else v * np.exp2(np.repeat(e.cpu().numpy().astype(np.float64) - 127.0, 32, axis=1))


def plan(experts, n_experts, multiple, rows):
    """(row_of, source, offsets) as lists, assignment by assignment"""
    lists = [[] for _ in range(n_experts)]
    for a, e in enumerate(np.asarray(experts).reshape(-1).tolist()):
        if 0 <= e < n_experts:
            lists[e].append(a)
    source, offsets = [], []
    for mine in lists:
        offsets.append(len(source))
        source += mine + [-1] * (-len(mine) % multiple)
    source += [-1] * (rows - len(source))
    row_of = [-1] * np.asarray(experts).size
    for r, a in enumerate(source):
        if a >= 0:
            row_of[a] = r
    return row_of, source, offsets + [rows]
