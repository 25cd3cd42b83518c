"""What the tests of ttf_rotate, ttf_cache_append and ttf_attend share: inputs, the definitions in 64 bits written plainly
from include/ttf.h, and the error that the kernels' arithmetic may make."""
import math

import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def axis_of(j, axes, sections, cyclic):
    if axes == 1:
        return 0
    if cyclic:
        a = j % axes
        return a if a > 0 and j // axes < sections[a] else 0
    for a in range(axes):
        if j < sum(sections[:a + 1]):
            return a
    raise AssertionError


def rotate_ref(x, positions, freq, weight=None, eps=1e-6, rot_dim=None, interleaved=False, sections=None, cyclic=False, factor=1.0):
    """x [rows, heads, D] (any dtype, CPU) -> (result in 64 bits, bound on the error of an fp32 evaluation rounded once)"""
    dt, x = x.dtype, x.double()
    rows, heads, D = x.shape
    rot = D if rot_dim is None else rot_dim
    positions = positions.reshape(rows, -1)
    axes = positions.shape[1]
    y = x
    if weight is not None:
        y = x * weight.double() / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    z, size = y.clone(), y.abs()
    for j in range(rot // 2):
        u, v = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        a = positions[:, axis_of(j, axes, sections, cyclic)].double() * freq[j].double()
        c, s = factor * torch.cos(a)[:, None], factor * torch.sin(a)[:, None]
        z[:, :, u], z[:, :, v] = y[:, :, u] * c - y[:, :, v] * s, y[:, :, v] * c + y[:, :, u] * s
        both = abs(factor) * (y[:, :, u].abs() + y[:, :, v].abs())
        size[:, :, u] = size[:, :, v] = both
    # fp32: the sum of D squares is off by at most D half steps, root, division and products by a step each; the turn is
    # rounded once (pi half steps of the angle) and its cosine and sine are within two steps
    return z, z.abs() * half_step(dt) + size * (D + 24) * 2.0 ** -24


def attend_ref(q, k_cache, v_cache, start, length, table, scale, causal=True, window=0, out=None):
    """Token by token and head by head (CPU tensors; start, length and table are lists).  Returns the result in 64 bits and a
    bound on the kernels' error: bf16 weights where the dtype is bf16, fp32 scores and sums, one rounding."""
    dt = q.dtype
    rows, heads, D = q.shape
    pages, page, hk, _ = k_cache.shape
    group = heads // hk
    res = torch.zeros((rows, heads, D), dtype=torch.float64) if out is None else out.double().clone()
    tol = torch.zeros((rows, heads, D), dtype=torch.float64)
    weights = half_step(dt) if dt == torch.bfloat16 else 0.0
    for b in range(len(length)):
        n = start[b + 1] - start[b]
        if n == 0:
            continue
        slots = [(table[b][s // page], s % page) for s in range(length[b])]
        ids = torch.tensor([g for g, _ in slots], dtype=torch.long)
        rws = torch.tensor([r for _, r in slots], dtype=torch.long)
        k, v = k_cache[ids, rws].double(), v_cache[ids, rws].double()          # [length, hk, D]
        for i in range(n):
            c = length[b] - n + i
            hi = 0 if c < 0 else (c + 1 if causal else length[b])
            lo = max(0, c - window + 1) if window else 0
            row = start[b] + i
            if hi <= lo:
                res[row] = 0
                continue
            for h in range(hk):
                hs = slice(h * group, (h + 1) * group)
                t = (q[row, hs].double() @ k[lo:hi, h].T) * scale
                p = torch.softmax(t, -1)
                res[row, hs] = p @ v[lo:hi, h]
                most = (q[row, hs].double().abs() @ k[lo:hi, h].abs().T).amax(-1) * abs(scale)
                # a score is off by (D + 4) steps of the sum of its terms' sizes (tensor cores truncate: steps, not half
                # steps), which moves a weight and the sum of all of them by that much; sums of n terms; exp2 within 2 steps
                rel = weights + 2.0 ** -23 * (2 * (D + 4) * most + (hi - lo) + 64)
                tol[row, hs] = rel[:, None] * (p @ v[lo:hi, h].abs())
    return res, tol + res.abs() * half_step(dt)


def spread_pages(lengths, page, generator, spare=2, fill=-1):
    """a table with the pages of all sequences in random order -> (table as lists, number of pages)"""
    used = [-(-n // page) for n in lengths]
    ids = torch.randperm(sum(used) + spare, generator=generator).tolist()
    width = max(1, max(used))
    table, at = [], 0
    for u in used:
        table.append(ids[at:at + u] + [fill] * (width - u))
        at += u
    return table, sum(used) + spare


def starts(new):
    s = [0]
    for n in new:
        s.append(s[-1] + n)
    return s


def ints(x, device="cuda"):
    return torch.tensor(x, dtype=torch.int32, device=device)


def worst(got, ref, tol):
    """largest error as a multiple of what is allowed"""
    d = (got.double() - ref).abs()
    assert torch.isfinite(got.double()).all()
    return float(torch.where(d == 0, torch.zeros_like(d), d / tol.clamp(min=1e-300)).max()) if d.numel() else 0.0
