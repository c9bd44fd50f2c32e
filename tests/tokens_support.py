"""Helpers for the tests of filtered sampling and tree acceptance: the definitions in 64 bits,
row by row, and calls of the binding on host data."""
import ctypes
import math

import numpy as np
import torch

from paper_2505_14260_gb300 import msd

# A product for each kernel that msd_linear4 has, with scales and zeros staged and (where such sizes exist) not, and the sizes
# of large models' layers: type, group, m, k, o, zeros; few, rows and outputs of a CTA, staged (msd_test_linear4_shape).
LINEAR4 = [
    ("bf16", 32, 1, 98776, 134, True, 0, 16, 128, 0),
    ("bf16", 32, 11, 2040, 132, True, 0, 16, 128, 1),
    ("bf16", 32, 1, 37984, 3053, True, 0, 16, 256, 0),
    ("bf16", 32, 10, 1192, 4911, True, 0, 16, 256, 1),
    ("bf16", 32, 19, 88664, 138, True, 0, 32, 128, 0),
    ("bf16", 32, 19, 1088, 132, True, 0, 32, 128, 1),
    ("bf16", 32, 21, 4160, 24002, True, 0, 32, 256, 0),
    ("bf16", 32, 17, 1048, 6680, True, 0, 32, 256, 1),
    ("bf16", 32, 33, 65504, 143, True, 0, 64, 128, 0),
    ("bf16", 32, 38, 1056, 130, True, 0, 64, 128, 1),
    ("bf16", 32, 907, 22280, 147, True, 0, 64, 256, 0),
    ("bf16", 32, 36, 1032, 6374, True, 0, 64, 256, 1),
    ("bf16", 32, 765, 23968, 132, True, 0, 128, 128, 0),
    ("bf16", 32, 741, 1936, 135, True, 0, 128, 128, 1),
    ("bf16", 32, 1, 1032, 131, True, 1, 8, 32, 1),
    ("bf16", 32, 9, 1032, 131, True, 1, 16, 32, 1),
    ("bf16", 64, 11, 3488, 137, True, 0, 16, 128, 1),
    ("bf16", 64, 2, 78256, 2949, True, 0, 16, 256, 0),
    ("bf16", 64, 9, 1912, 4928, True, 0, 16, 256, 1),
    ("bf16", 64, 22, 1056, 131, True, 0, 32, 128, 1),
    ("bf16", 64, 19, 49936, 4611, True, 0, 32, 256, 0),
    ("bf16", 64, 18, 1160, 4639, False, 0, 32, 256, 1),
    ("bf16", 64, 51, 130072, 140, True, 0, 64, 128, 0),
    ("bf16", 64, 36, 1040, 141, True, 0, 64, 128, 1),
    ("bf16", 64, 947, 65336, 142, False, 0, 64, 256, 0),
    ("bf16", 64, 40, 1840, 6082, True, 0, 64, 256, 1),
    ("bf16", 64, 912, 32664, 130, True, 0, 128, 128, 0),
    ("bf16", 64, 453, 1656, 144, True, 0, 128, 128, 1),
    ("bf16", 64, 1, 1136, 136, True, 1, 8, 32, 1),
    ("bf16", 64, 10, 1088, 136, True, 1, 16, 32, 1),
    ("bf16", 128, 9, 4824, 136, True, 0, 16, 128, 1),
    ("bf16", 128, 13, 2280, 5127, True, 0, 16, 256, 1),
    ("bf16", 128, 20, 1088, 142, True, 0, 32, 128, 1),
    ("bf16", 128, 19, 1224, 6067, True, 0, 32, 256, 1),
    ("bf16", 128, 37, 1056, 132, False, 0, 64, 128, 1),
    ("bf16", 128, 145, 11104, 10036, True, 0, 64, 256, 0),
    ("bf16", 128, 35, 1568, 6462, True, 0, 64, 256, 1),
    ("bf16", 128, 468, 89184, 139, True, 0, 128, 128, 0),
    ("bf16", 128, 458, 1760, 135, True, 0, 128, 128, 1),
    ("bf16", 128, 1, 1088, 131, True, 1, 8, 32, 1),
    ("bf16", 128, 15, 1056, 131, True, 1, 16, 32, 1),
    ("f32", 32, 1, 78688, 131, True, 0, 16, 128, 0),
    ("f32", 32, 11, 1040, 136, True, 0, 16, 128, 1),
    ("f32", 32, 4, 26648, 3010, True, 0, 16, 256, 0),
    ("f32", 32, 9, 1568, 1944, False, 0, 16, 256, 1),
    ("f32", 32, 20, 77088, 133, True, 0, 32, 128, 0),
    ("f32", 32, 19, 1048, 138, True, 0, 32, 128, 1),
    ("f32", 32, 355, 31688, 130, True, 0, 32, 256, 0),
    ("f32", 32, 473, 1576, 132, True, 0, 32, 256, 1),
    ("f32", 32, 1, 1056, 131, True, 1, 8, 32, 1),
    ("f32", 64, 2, 113936, 1944, True, 0, 16, 128, 0),
    ("f32", 64, 9, 1064, 132, True, 0, 16, 128, 1),
    ("f32", 64, 1, 41664, 3877, True, 0, 16, 256, 0),
    ("f32", 64, 10, 1544, 1984, True, 0, 16, 256, 1),
    ("f32", 64, 228, 118032, 139, True, 0, 32, 128, 0),
    ("f32", 64, 19, 1040, 140, True, 0, 32, 128, 1),
    ("f32", 64, 355, 64776, 131, True, 0, 32, 256, 0),
    ("f32", 64, 595, 1216, 140, True, 0, 32, 256, 1),
    ("f32", 64, 2, 1072, 131, True, 1, 8, 32, 1),
    ("f32", 128, 10, 1056, 137, True, 0, 16, 128, 1),
    ("f32", 128, 12, 1728, 2004, True, 0, 16, 256, 1),
    ("f32", 128, 751, 78096, 301, True, 0, 32, 128, 0),
    ("f32", 128, 20, 1088, 133, True, 0, 32, 128, 1),
    ("f32", 128, 249, 110280, 149, True, 0, 32, 256, 0),
    ("f32", 128, 242, 1608, 144, False, 0, 32, 256, 1),
    ("f32", 128, 3, 1088, 133, True, 1, 8, 32, 1),
    ("bf16", 64, 645, 4096, 11008, True, 0, 128, 128, 1),
    ("bf16", 32, 645, 11008, 4096, False, 0, 128, 128, 0),
    ("bf16", 32, 60, 4096, 11008, False, 0, 64, 256, 1),
    ("bf16", 128, 645, 11008, 11008, True, 0, 128, 128, 0),
    ("bf16", 128, 60, 13824, 32000, True, 0, 64, 256, 0),
    ("f32", 32, 16, 5120, 32000, False, 0, 16, 256, 0),
    ("f32", 32, 16, 5120, 32000, True, 0, 16, 256, 0),
    ("f32", 64, 60, 4096, 11008, True, 0, 32, 256, 1),
    ("f32", 128, 200, 11008, 4096, False, 0, 32, 256, 1),
]


def linear4_shape(dtype, group, m, k, o, zeros, codes=1 << 20):
    """How msd_linear4 launches a product whose codes lie at this address."""
    a = 1 << 20                       # (an address that nothing reads)
    w, out = msd.msd_weight4(codes, a, a if zeros else None, o, k, group), msd.msd_linear4_shape()
    assert msd.lib().msd_test_linear4_shape(msd.MSD_BF16 if dtype == "bf16" else msd.MSD_F32, m, ctypes.byref(w), ctypes.byref(out)) == msd.MSD_OK
    return out


class Row:
    """What the settings (t, k, p, m; None: off) leave of one row of logits: weights in id order."""

    def __init__(self, x, t=None, k=None, p=None, m=None):
        x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
        self.w = np.zeros(x.size)
        order = np.lexsort((np.arange(x.size), -x))
        order = order[x[order] > -np.inf]
        if order.size == 0:
            return
        t, m = 1.0 if t is None else float(t), 0.0 if m is None else float(m)
        p = 1.0 if p is None else float(p)
        if not t >= 2.0 ** -100 or m > 1 or p <= 0:
            order = order[:1]
        t = min(max(t, 2.0 ** -100), 2.0 ** 100) if t == t else 1.0
        with np.errstate(invalid="ignore", over="ignore"):
            w = np.where(x[order] == x[order[0]], 1.0, np.exp((x[order] - x[order[0]]) / t))
        n = order.size
        if k is not None and k > 0:
            n = min(n, int(k))
        if p < 1:
            mass = np.cumsum(w[:n])
            n = int(np.searchsorted(mass, p * mass[-1])) + 1
        if m > 0:
            n = min(n, max(1, int(np.sum(w >= m))))
        self.w[order[:n]] = w[:n]

    def draw(self, u):
        mass = np.cumsum(self.w)
        if not mass[-1] > 0:
            return -1
        u = min(max(float(u), 0.0), 1 - 2.0 ** -24) if u == u else 0.0
        return int(np.searchsorted(mass, u * mass[-1], side="right"))


def host(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def settings(n, **given):
    """Filter of values or lists, and rows' settings for Row."""
    types = dict(temperature=torch.float32, top_k=torch.int32, top_p=torch.float32, min_p=torch.float32)
    dev = {name: torch.tensor(v if isinstance(v, (list, tuple)) else [v] * n, dtype=types[name], device="cuda")
           for name, v in given.items() if v is not None}
    short = dict(temperature="t", top_k="k", top_p="p", min_p="m")
    vals = {name: v.cpu().numpy() for name, v in dev.items()}
    return msd.Filter(**dev), [{short[name]: v[i] for name, v in vals.items()} for i in range(n)]


def check_sample(x, u, want_probs=True, **given):
    """msd.sample on x [rows, vocab] (a GPU tensor, any row stride) against Row."""
    rows, vocab = x.shape
    f, each = settings(rows, **given)
    tokens = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    logp = torch.full((rows,), 7.0, device="cuda")
    probs = torch.full((rows, vocab + 3), 7.0, device="cuda")[:, :vocab] if want_probs else None
    msd.sample(x, u, f if given else None, tokens, logp=logp, probs=probs)
    torch.cuda.synchronize()
    xs, us, ts, ls = host(x), host(u), tokens.cpu().numpy(), logp.cpu().numpy()
    ps = None if probs is None else probs.double().cpu().numpy()
    for i in range(rows):
        r = Row(xs[i], **each[i])
        total = r.w.sum()
        t = r.draw(us[i])
        assert ts[i] == t, (i, each[i], ts[i], t)
        if t < 0:
            assert ls[i] == -math.inf
        else:
            want = math.log(r.w[t] / total)
            # one rounding to fp32; the weights' 2^-44 in the sum
            assert abs(float(ls[i]) - want) <= 2.0 ** -24 * abs(want) + vocab * 2.0 ** -44 + 1e-12, (i, ls[i], want)
        if ps is not None:
            share = r.w / total if total > 0 else r.w
            assert ((ps[i] > 0) == (share > 1e-37)).all() or (np.abs((ps[i] > 0) * 1.0 - (share > 0)) * share).max() <= 1e-36, i
            # exp2f 2^-22, its argument's rest, the total's reciprocal and two products 2^-24 each
            assert (np.abs(ps[i] - share) <= 2.0 ** -21 * share + 1e-37).all(), (i, np.abs(ps[i] - share).max())
    return tokens


def check_accept(x, counts, tokens, parent, u, nodes, n_nodes=None, children=None, **given):
    """msd.accept against a walk with Row. tokens, parent: per sequence lists of up to `nodes`."""
    n, depth, k = len(counts), u.shape[1] - 1, u.shape[2] - 1
    f, each = settings(n, **given)
    starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")  # noqa: E731
    b = msd.Batch(torch.arange(n, dtype=torch.int32, device="cuda"), i32(starts), int(starts[-1]))
    tree = msd.Tree(n, nodes)
    for i in range(n):
        c = len(tokens[i])
        tree.tokens[i * nodes:i * nodes + c] = i32(tokens[i])
        tree.parent[i * nodes:i * nodes + c] = i32(parent[i])
    if n_nodes is not None:
        tree.n_nodes.copy_(i32(n_nodes))
    path = torch.full((n, depth + 1), -7, dtype=torch.int32, device="cuda")
    length, bonus = torch.full((n,), -7, dtype=torch.int32, device="cuda"), torch.full((n,), -7, dtype=torch.int32, device="cuda")
    msd.accept(x, b, tree, u, f if given else None, path, length, bonus)
    torch.cuda.synchronize()
    xs, us = host(x), host(u).astype(np.float64)
    for i in range(n):
        live = min(counts[i], nodes, n_nodes[i] if n_nodes is not None else nodes)
        want, got = [], None
        if live > 0:
            want, at = [0], 0
            while got is None:
                d = len(want) - 1
                r = Row(xs[starts[i] + at], **each[i])
                kids = [j for j in range(at + 1, live) if parent[i][j] == at][:k] if d < depth else []
                nxt = None
                for c, j in enumerate(kids):
                    t = tokens[i][j]
                    if 0 <= t < r.w.size:
                        if us[i, d, c] * r.w.sum() < r.w[t]:
                            nxt = j
                            break
                        r.w[t] = 0.0
                if nxt is None:
                    got = r.draw(us[i, d, k])
                else:
                    at = nxt
                    want.append(at)
        a = len(want) - 1 if want else 0
        assert path[i].tolist() == want + [-1] * (depth + 1 - len(want)), (i, path[i].tolist(), want)
        assert int(length[i]) == a and int(bonus[i]) == (-1 if got is None else got), (i, int(bonus[i]), got)
    return path, length, bonus
