"""Helpers for the paged cache's tests: pools with scattered pages, plain 64-bit forms, and
the bounds that the kernels' results are held to."""
import math

import torch

from paper_2505_14260_gb300 import msd

U = 2.0 ** -24                # half a unit in the last place of fp32, relative


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def starts(counts):
    return i32([0] + torch.tensor(counts, dtype=torch.int64).cumsum(0).tolist())


def batch(seqs, counts):
    return msd.Batch(i32(seqs), starts(counts), sum(counts))


def pool(lens, *, seed=0, dtype="bf16", layers=1, heads=4, kv_heads=2, head_dim=64, page=16, spare=4, extra_seqs=0,
         extra_pages=2, stale=float("nan"), **more):
    """A pool whose sequences have the given lengths, on pages in no order; K and V are
    normal, `stale` in every slot that no sequence holds."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    need = [-(-x // page) for x in lens]
    total, room = sum(need) + spare, max(need + [1]) + extra_pages
    order = torch.randperm(total, generator=g, device="cuda")[: sum(need)].to(torch.int32)
    table = torch.full((len(lens) + extra_seqs, room), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    kv = torch.randn(layers, total, 2, kv_heads, page, head_dim, generator=g, device="cuda").to(dt)
    held = torch.zeros(total, dtype=torch.bool, device="cuda")
    held[order.long()] = True
    kv[:, ~held] = stale
    for i, x in enumerate(lens):
        if x % page:
            kv[:, table[i, need[i] - 1].long(), :, :, x % page:] = stale
    p = msd.Pages(dtype=dtype, layers=layers, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page_size=page,
                  n_pages=total, max_seqs=len(lens) + extra_seqs, max_pages=room, kv=kv, table=table,
                  lens=i32(list(lens) + [0] * extra_seqs), refs=torch.zeros(total, dtype=torch.int32, device="cuda"),
                  **more)
    p.restore()
    return p


def tokens(p, layer, seq):
    """K and V of a sequence, [len, kv_heads, head_dim] each, in 64 bits."""
    n, page = int(p.lens[seq]), p.cfg.page_size
    ids = p.table[seq, : -(-n // page)].long()
    x = p.kv[layer, ids].double().permute(1, 0, 3, 2, 4).reshape(2, -1, p.cfg.n_kv_heads, p.cfg.head_dim)
    return x[0, :n], x[1, :n]


def random_tree(n_seqs, nodes, seed, valid=None):
    """msd.Tree of random trees and the [n, N, N] ancestor-or-self matrix."""
    r = torch.Generator().manual_seed(seed)
    t = msd.Tree(n_seqs, nodes)
    see = torch.zeros(n_seqs, nodes, nodes, dtype=torch.bool)
    depth = torch.zeros(n_seqs, nodes, dtype=torch.int64)
    for b in range(n_seqs):
        see[b, 0, 0] = True
        for i in range(1, nodes):
            p = int(torch.randint(max(0, i - 12), i, (1,), generator=r))
            see[b, i] = see[b, p]
            see[b, i, i] = True
            depth[b, i] = depth[b, p] + 1
    words = torch.zeros(n_seqs, nodes, t.W, dtype=torch.int64)
    for j in range(nodes):
        bit = torch.where(see[:, :, j], torch.tensor(1 << (j % 64) if j % 64 < 63 else -(1 << 63)), 0)
        words[:, :, j // 64] |= bit
    t.mask.copy_(words.reshape(-1))
    t.depth.copy_(depth.reshape(-1))
    if valid is not None:
        t.n_nodes.copy_(i32(valid))
        for b, v in enumerate(valid):
            see[b, v:] = False
    return t, see.cuda(), depth.cuda()


def visible(L, rows, window, sinks, see=None, depth=None):
    """[rows, L + rows]: which slots each row sees."""
    S = L + rows
    place = torch.arange(S, device="cuda")
    if see is None:
        ok = torch.ones(rows, S, dtype=torch.bool, device="cuda").tril(L)
    else:
        place = torch.cat([place[:L], L + depth[:rows]])
        ok = torch.cat([see[:rows].any(1, keepdim=True).expand(rows, L), see[:rows, :rows]], 1)
    if window:
        ok = ok & ((place[L:, None] - place[None] < window) | (place < sinks)[None])
    return ok


def attend(q, k, v, ok):
    """softmax(q k / sqrt(d)) v over the visible slots, in 64 bits; the sums run over the
    visible keys alone. q [R, H, d], k and v [S, K, d], ok [R, S]."""
    R, H, d = q.shape
    G = H // k.shape[1]
    out = torch.zeros(R, H, d, dtype=torch.float64, device=q.device)
    lse = torch.full((R, H), -math.inf, dtype=torch.float64, device=q.device)
    for r in range(R):
        at = ok[r].nonzero()[:, 0]
        if at.numel() == 0:
            continue
        kk, vv = k[at].repeat_interleave(G, 1), v[at].repeat_interleave(G, 1)
        z = torch.einsum("hd,shd->hs", q[r].double(), kk) / math.sqrt(d)
        lse[r] = torch.logsumexp(z, 1)
        out[r] = torch.einsum("hs,shd->hd", torch.softmax(z, 1), vv)
    return out, lse


def bounds(q, k, v, ref, lse, dtype):
    """Absolute bounds of out and lse, elementwise. A score is a sum of d products with at most
    d + 2 roundings: off by e <= (d + 2) u sum |q k| / sqrt(d) (the tensor core's fp32 sums
    truncate and drop bits of the smaller terms: 8 u a term). Weights are off by a factor of
    1 +- (2 e + 2^-21) (the exponential and its argument), sums of S of them by S u (their error grows like
    sqrt(S); S u bounds it). bf16: weights are rounded to 8 bits (2^-9), and the result."""
    d, S = q.shape[-1], k.shape[0]
    fin_k, fin_v = torch.nan_to_num(k, 0, 0, 0), torch.nan_to_num(v, 0, 0, 0)
    e = (d + 2) * (U if dtype == "f32" else 8 * U) * d ** 0.5 * float(q.double().abs().max()) * float(fin_k.abs().max())
    weight = 2 * e + 2.0 ** -21 + S * U + (2.0 ** -9 if dtype == "bf16" else 0.0)
    out = weight * float(fin_v.abs().max()) + (2.0 ** -8 if dtype == "bf16" else 4 * U) * ref.abs()
    return out, 2 * e + 2.0 ** -20 + S * U + 4 * U * lse.abs()


def typical(q, k, dtype):
    """What the 2-norm of a result's error stays below, relative to the result's: roundings are
    independent, so a score of size z is off by some u z (here 16 u (8 + z), for the largest), and with
    bf16 each weight and each result by at most 2^-9 relative: sqrt(2) 2^-9, twice that here."""
    G = q.shape[1] // k.shape[1]
    kk = torch.nan_to_num(k, 0, 0, 0).repeat_interleave(G, 1)
    z = float((torch.einsum("rhd,shd->rhs", q.double(), kk) / q.shape[-1] ** 0.5).abs().max())
    return 16 * U * (8 + z) * (4 if dtype == "bf16" else 1) + (2.0 ** -7.5 if dtype == "bf16" else 0.0)
