"""The paged cache's operators in 64 bits, from their definitions, on the CPU; a pool as plain position-major data."""
import math

import torch


def frequencies(rot, theta=10000.0, scaling="none", factor=1.0, trained_pos=0, low=1.0, high=4.0):
    out = []
    for j in range(rot // 2):
        base = theta * factor ** (rot / (rot - 2)) if scaling == "base" else theta
        f = base ** (-2.0 * j / rot)
        if scaling == "linear":
            f /= factor
        if scaling == "bands":
            w = min(max((trained_pos * f / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            f = f * w + f * (1.0 - w) / factor
        out.append(f)
    return torch.tensor(out, dtype=torch.float64)


def rotate(x, pos, rot, pairing="half", magnitude=1.0, inverse=False, **freq):
    """x [n][heads][hd] in 64 bits, pair by pair"""
    y = x.double().clone()
    angle = pos.double()[:, None] * frequencies(rot, **freq)
    for j in range(rot // 2):
        a, b = (j, j + rot // 2) if pairing == "half" else (2 * j, 2 * j + 1)
        c, s = magnitude * torch.cos(angle[:, j])[:, None], magnitude * torch.sin(angle[:, j])[:, None]
        if inverse:
            s = -s
        u, w = x[..., a].double(), x[..., b].double()
        y[..., a], y[..., b] = u * c - w * s, w * c + u * s
    return y


def places(dtype, hd, ps):
    """element of a block where position p, feature i keeps its key and its value: two [ps][hd] index tensors"""
    k, v = torch.empty(ps, hd, dtype=torch.int64), torch.empty(ps, hd, dtype=torch.int64)
    for p in range(ps):
        for i in range(hd):
            if dtype == torch.float32:
                k[p, i], v[p, i] = p * hd + i, ps * hd + p * hd + i
            else:
                q, r = divmod(p, 32)
                k[p, i] = q * 64 * hd + (((r // 16 * (hd // 32) + i // 32) * 4 + i % 32 // 8) * 16 + r % 16) * 8 + i % 8
                v[p, i] = q * 64 * hd + 32 * hd + ((i // 16 * 4 + r % 16 // 4) * 16 + i % 16) * 8 + r // 16 * 4 + r % 4
    return k, v


def read_pool(pool, n_layers, n_pages, hkv, hd, ps):
    """[2][layer][page][hkv][ps][hd] of a flat pool on the CPU"""
    k, v = places(pool.dtype, hd, ps)
    b = pool.view(n_layers, n_pages, hkv, 2 * ps * hd)
    return torch.stack([b[..., k], b[..., v]])


def write_pool(kv, dtype):
    """the flat pool of [2][layer][page][hkv][ps][hd]"""
    _, n_layers, n_pages, hkv, ps, hd = kv.shape
    k, v = places(dtype, hd, ps)
    b = torch.empty(n_layers, n_pages, hkv, 2 * ps * hd, dtype=dtype)
    b[..., k.flatten()] = kv[0].to(dtype).flatten(-2)
    b[..., v.flatten()] = kv[1].to(dtype).flatten(-2)
    return b.flatten()


def attend(q, kv, seqs, pages, window, scale):
    """q [n][hq][hd]; kv [2][page][hkv][ps][hd] (one layer); seqs: (rows, positions) of each sequence; pages: its page numbers, lists.
    Returns the output, sum_j p_j |v_j| (what errors of the probabilities are measured against) and max_j sum_i |q_i k_ji| scale."""
    n, hq, hd = q.shape
    n_pages, hkv, ps = kv.shape[1], kv.shape[2], kv.shape[3]
    out, size, dots = torch.zeros(n, hq, hd, dtype=torch.float64), torch.zeros(n, hq, hd, dtype=torch.float64), torch.zeros(n, hq, 1).double()
    row = 0
    for (rows, length), table in zip(seqs, pages):
        for j in range(rows):
            p = length - rows + j
            lo = max(0, p - window + 1) if window else 0
            seen = [x for x in range(lo, p + 1) if 0 <= table[x // ps] < n_pages]
            if seen:
                pg, at = torch.tensor([table[x // ps] for x in seen]), torch.tensor([x % ps for x in seen])
                for h in range(hq):
                    g = h // (hq // hkv)
                    k, v = kv[0, pg, g, at].double(), kv[1, pg, g, at].double()
                    x = (k @ q[row, h].double()) * scale
                    w = torch.softmax(x, 0)
                    out[row, h], size[row, h] = w @ v, w @ v.abs()
                    dots[row, h] = (k.abs() @ q[row, h].double().abs()).max() * scale
            row += 1
    return out, size, dots
