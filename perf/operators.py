"""Operator cases of the paged cache: what a program that serves many multimodal
requests from one pool of cache pages does between its projections, through the
public binding (Pages of paper_2505_14260_gb300.msd).

Kinds of case
  attention  the rows at the end of each sequence (one token, a chunk of a prompt,
             or a drafted tree) against the sequence's pages: grouped heads, a
             window with first tokens that stay visible, log-sum-exp.
  rope       positions of text, images and video on three axes (time, height,
             width), the rotation of q and k by them, and K and V into the pages.
             With `decode` the rows are a drafted tree's, at positions in hand.
  fork       sequences that another one's pages are shared with (several answers
             about one image), after the last round's were freed. `deep`: copies.
  evict      a long sequence cut to its first tokens and its newest ones in a fork
             of it, the other pages freed.
  step       a decode step's cache work: fork, room for the tree's rows, rotation
             and K/V of every layer, then only the accepted path stays.

A pool's pages are in no order, and what no sequence holds is NaN, as fresh memory
may be. Widths are those of this repository's workloads (4 heads of 64, 16 of 64,
32 and 40 of 128) and generic grouped ones. Plain forms run in 32 bits on padded
batches; positions are whole numbers, whose angles are reduced as such.
"""
import math
import random

import torch

own = False

NEVER = -1                    # a table entry that holds no page


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _case(kind, dtype, n, heads, kv_heads, hd, page, **more):
    return dict(kind=kind, dtype=dtype, n=n, heads=heads, kv_heads=kv_heads, hd=hd, page=page, **more)


def _attn(dtype, n, heads, kv_heads, hd, page, prefix, rows, tree=False, window=0, sinks=0):
    return _case("attention", dtype, n, heads, kv_heads, hd, page, prefix=prefix, rows=rows, tree=tree,
                 window=window, sinks=sinks)


def _rope(dtype, src, n, heads, kv_heads, hd, page, text, images, t, h, w, step, turns, rot, decode=False):
    return _case("rope", dtype, n, heads, kv_heads, hd, page, src=src, text=text, images=images, t=t, h=h, w=w,
                 step=step, turns=turns, rot=rot, decode=decode)


def listed():
    return [
        # the tiny reference model's tree behind its prompt, fp32: the smallest call
        dict(_attn("f32", 1, 4, 4, 64, 16, 96, 16, tree=True), name="attn_tiny_tree_f32"),
        # fp32 chunks of two prompts with odd lengths at a small width, two query heads to a KV head
        dict(_attn("f32", 2, 16, 8, 64, 32, 77, 333), name="attn_chunk_f32"),
        # one token each of 64 requests whose lengths go from tens to thousands
        dict(_attn("bf16", 64, 32, 8, 128, 16, 8191, 1), name="attn_decode_ragged64"),
        # the 60-node tree of a 7B request behind a long multimodal prefix (5 x 576 + 512)
        dict(_attn("bf16", 1, 32, 32, 128, 64, 3392, 60, tree=True), name="attn_tree_7b_long"),
        # one token behind a very long context
        dict(_attn("bf16", 1, 32, 8, 128, 32, 131071, 1), name="attn_decode_128k"),
        # a long video prompt through a layer with a window and four first tokens
        dict(_attn("bf16", 1, 32, 8, 128, 64, 0, 8192, window=2048, sinks=4), name="attn_prompt_window"),
        # ragged chunks of two prompts behind what is cached of them
        dict(_attn("bf16", 2, 32, 8, 128, 64, 4096, 4096), name="attn_chunk_ragged"),
        # a drafted tree's 60 rows of one layer, from the projection's fp32 output
        dict(_rope("bf16", "f32", 1, 32, 32, 128, 64, 60, 0, 1, 1, 1, 1, False, 128, decode=True), name="rope_tree_7b"),
        # 16 prompts, each with two images of 24 x 24 tokens and a ragged text
        dict(_rope("bf16", "bf16", 16, 32, 8, 128, 64, 512, 2, 1, 24, 24, 1, True, 128), name="rope_prompts16"),
        # eight answers each about eight prompts, 32 layers
        dict(_case("fork", "bf16", 8, 32, 8, 128, 16, layers=32, prefix=1221, fan=8, deep=False), name="pages_fork64"),
        # sixteen long sequences cut to 4 + 1023 tokens, 8 layers
        dict(_case("evict", "bf16", 16, 32, 8, 128, 64, layers=8, prefix=4001, first=4, newest=1023), name="pages_evict16"),
        # the cache work of a batch of 16 decode steps, 4 layers
        dict(_case("step", "bf16", 16, 32, 8, 128, 32, layers=4, prefix=700, rows=60, path=7), name="pages_step16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_WIDTHS = [(4, 4, 64), (16, 16, 64), (16, 4, 64), (32, 32, 128), (32, 8, 128), (40, 40, 128), (28, 4, 128), (8, 1, 64)]
_LARGEST = 5.2e11             # flops of a drawn attention at most (the largest listed: 5.3e11)
_MOST_SCORES = 2.2e9          # scores of its padded plain form at most


def _draw_attention(rng):
    f32 = rng.random() < 0.2
    heads, kv_heads, hd = rng.choice(_WIDTHS[:3] if f32 else _WIDTHS)
    shape = rng.choice(["one", "one", "tree", "tree", "chunk", "chunk"])
    n = rng.choice([1, 1, 2, 3, _log_int(rng, 4, 64)])
    prefix = _log_int(rng, 1, 1000 if f32 else 60000 if n < 4 else 6000) - 1
    rows = 1 if shape == "one" else rng.randint(2, 140) if shape == "tree" else _log_int(rng, 2, 400 if f32 else 4000)
    window = rng.choice([0, 0, _log_int(rng, 1, 4096)])
    return _attn("f32" if f32 else "bf16", n, heads, kv_heads, hd, rng.choice([16, 32, 64, 128]), prefix, rows,
                 tree=shape == "tree", window=window, sinks=rng.choice([0, 1, 4, 37]) if window else 0)


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "rope", "rope", "fork", "evict", "step"])
    heads, kv_heads, hd = rng.choice(_WIDTHS)
    page = rng.choice([16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "rope":
        rot = rng.choice([hd, hd, hd // 2])
        if rng.random() < 0.4:
            return _rope(dtype, rng.choice([dtype, "f32"]), rng.randint(1, 16), heads, kv_heads, hd, page,
                         rng.randint(1, 140), 0, 1, 1, 1, 1, rng.random() < 0.5, rot, decode=True)
        video = rng.random() < 0.4
        return _rope(dtype, rng.choice([dtype, "f32"]), rng.choice([1, 2, 5, 16]), heads, kv_heads, hd, page,
                     _log_int(rng, 2, 600), rng.randint(0, 3), rng.randint(2, 6) if video else 1,
                     rng.randint(1, 24), rng.randint(1, 24), rng.randint(1, 5), rng.random() < 0.5, rot)
    if kind == "fork":
        return _case(kind, dtype, rng.randint(1, 8), heads, kv_heads, hd, page, layers=rng.choice([1, 4, 16]),
                     prefix=_log_int(rng, 1, 2000), fan=rng.randint(1, 6), deep=rng.random() < 0.3)
    if kind == "evict":
        prefix = _log_int(rng, 2, 4000)
        return _case(kind, dtype, rng.randint(1, 16), heads, kv_heads, hd, page, layers=rng.randint(1, 4), prefix=prefix,
                     first=rng.randint(0, min(9, prefix - 1)), newest=rng.randint(0, min(1200, prefix)))
    if kind == "step":
        rows = rng.randint(1, 130)
        return _case(kind, dtype, rng.randint(1, 16), heads, kv_heads, hd, page, layers=rng.randint(1, 4),
                     prefix=_log_int(rng, 1, 2000), rows=rows, path=rng.randint(1, min(9, rows)))
    c = _draw_attention(rng)
    if _scores(c) <= _MOST_SCORES and work(c)["flops"] <= _LARGEST:
        return c
    return draw(rng)


def _spread(top, lo, i):
    """Ragged sizes: sequence 0 has the largest, the others spread over the logarithm."""
    lo = min(lo, top)
    return top if i == 0 or top <= 1 else int(round(max(lo, 1) * (top / max(lo, 1)) ** (((i * 37 + 11) % 64) / 63)))


def _kept(c):
    return min(c["prefix"], c["first"] + c["newest"])


def _rows(c):
    """Rows of each sequence in the call."""
    if c["kind"] == "rope" and not c["decode"]:
        return [_spread(c["text"], 2, i) + c["images"] * c["t"] * c["h"] * c["w"] for i in range(c["n"])]
    if c["kind"] == "rope":
        return [c["text"]] * c["n"]
    if c["kind"] == "attention" and not c["tree"] and c["rows"] > 1:
        return [_spread(c["rows"], 2, i) for i in range(c["n"])]
    return [c.get("rows", 0)] * c["n"]


def _prefixes(c):
    """Tokens of each sequence before the call's rows."""
    if c["kind"] == "rope":
        return [641 if c["decode"] else 0] * c["n"]
    return [_spread(c["prefix"], 16, i) for i in range(c["n"])]


def _scores(c):
    return c["n"] * c["heads"] * max(_rows(c)) * (max(_prefixes(c)) + max(_rows(c)))


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(counts):
    return _i32([0] + torch.tensor(counts).cumsum(0).tolist())


def _sections(c):
    """Frequencies that turn by time, height and width: a quarter and halves of the rest
    one after another; where they take turns, height and width end before the last ones."""
    half = c.get("rot", c["hd"]) // 2
    side = half * 5 // 16 if c.get("turns") else half * 3 // 8
    return [half - 2 * side, side, side]


def _rotates(c):
    return dict(rot=c.get("rot", c["hd"]), sections=_sections(c), turns=c.get("turns", False), base=10000.0)


def prepare(case, seed):
    c = dict(case)
    dt, dev = _dtype(c["dtype"]), "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 7919 + 3)
    pick = random.Random(seed * 31 + 7)
    n, page, layers = c["n"], c["page"], c.get("layers", 1)
    rows, before = _rows(c), _prefixes(c)
    held = [a + b for a, b in zip(before, rows)] if c["kind"] in ("attention", "rope") else before
    need = [-(-x // page) for x in held]
    room = -(-(max(held) + max(rows)) // page) + 1
    fan = c["fan"] if c["kind"] == "fork" else 1 if c["kind"] in ("evict", "step") else 0
    spare = {"fork": (room if c.get("deep") else 1) * n * fan, "evict": n * (room + 1),
             "step": n * (-(-max(rows) // page) + 2)}.get(c["kind"], 0)
    total = sum(need) + spare + 3
    seqs = n * (1 + fan) + 1
    s = {"c": c, "pages_total": total, "room": room}

    # the pool: pages in no order, NaN in what no sequence holds
    order = torch.randperm(sum(need) + 3, generator=g, device=dev)[: sum(need)].to(torch.int32)
    table = torch.full((seqs, room), NEVER, dtype=torch.int32, device=dev)
    lens = torch.zeros(seqs, dtype=torch.int32, device=dev)
    at = 0
    for i in range(n):
        table[i, : need[i]] = order[at:at + need[i]]
        at += need[i]
    lens[:n] = _i32(held)
    refs = torch.zeros(total, dtype=torch.int32, device=dev)
    refs[order.long()] = 1
    kv = torch.empty(layers, total, 2, c["kv_heads"], page, c["hd"], device=dev, dtype=dt)
    kv.normal_(generator=g)
    kv[:, :, 0] += torch.randn(c["kv_heads"], 1, c["hd"], generator=g, device=dev).to(dt)     # keys have a mean
    kv[:, refs == 0] = float("nan")
    for i in range(n):
        if held[i] % page:
            kv[:, table[i, need[i] - 1].long(), :, :, held[i] % page:] = float("nan")
    s.update(table=table, lens=lens, refs=refs, kv=kv)

    # the rows of a call
    T, H, K, hd = sum(rows), c["heads"], c["kv_heads"], c["hd"]
    s["seqs"] = _i32([i if fan == 0 else n + i for i in range(n)])
    s["row_start"] = _starts(rows)
    if c["kind"] == "attention":
        s["q"] = (1.5 * torch.randn(T, H, hd, generator=g, device=dev)).to(dt)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(T, H, device=dev)
    if c["kind"] in ("rope", "step"):
        src = _dtype(c.get("src", "f32"))
        s["qkv"] = torch.randn(T, (H + 2 * K) * hd, generator=g, device=dev).to(src)
        s["q_out"] = torch.empty(T, H, hd, device=dev, dtype=dt)
        if c["kind"] == "rope" and not c["decode"]:
            spans, starts, size = [], [0], c["t"] * c["h"] * c["w"]
            for i in range(n):
                text, first = rows[i] - c["images"] * size, min(8, max(1, _spread(c["text"], 2, i) - 1))
                gap = max(0, (text - first) // (c["images"] + 1))
                spans += [[first + k * (size + gap), c["t"], c["h"], c["w"], c["step"]] for k in range(c["images"])]
                starts.append(len(spans))
            s["spans"], s["span_start"] = _i32(spans or [[0, 0, 0, 0, 0]]), _i32(starts)
            s["pos"] = torch.empty(3, T, dtype=torch.int32, device=dev)
            s["next"] = torch.empty(n, dtype=torch.int32, device=dev)
        else:
            depth = [0] + [pick.randint(1, 6) for _ in range(max(rows) - 1)]
            s["pos"] = torch.cat([p + _i32(depth) for p in before]).to(torch.int32)[None]      # one for all axes
    if c.get("tree"):
        N, W = max(rows), -(-max(rows) // 64)
        masks, depths = [], []
        for _ in range(n):
            parent, depth, mask = [-1], [0], [1]
            for i in range(1, N):
                p = pick.choice([j for j in range(i) if depth[j] < 8])
                depth.append(depth[p] + 1)
                mask.append(mask[p] | 1 << i)
            depths += depth
            masks += [[m >> 64 * w & (1 << 64) - 1 for w in range(W)] for m in mask]
        words = torch.tensor([[x - (1 << 64) if x >> 63 else x for x in m] for m in masks], device=dev)
        s["mask"], s["depth"] = words.view(n, N, W), _i32(depths).view(n, N)
        s["nodes"] = _i32([max(1, N - i % 3) for i in range(n)])            # some trees are a node or two short
    if c["kind"] == "fork":
        s["src"] = _i32([i for i in range(n) for _ in range(fan)])
        s["dst"] = _i32([n + k for k in range(n * fan)])
    elif fan:
        s["src"], s["dst"] = _i32(list(range(n))), s["seqs"]
    if c["kind"] == "evict":
        width = max(_kept({**c, "prefix": p}) for p in before)
        keep = [list(range(p)) if p <= c["first"] + c["newest"] else
                list(range(c["first"])) + list(range(p - c["newest"], p)) for p in before]
        s["n_keep"] = _i32([len(k) for k in keep])
        s["keep"] = _i32([k + [-1] * (max(width, 1) - len(k)) for k in keep])
        s["row_start"] = _starts(before)
    if c["kind"] == "step":
        keep = [[0] + sorted(pick.sample(range(1, c["rows"]), pick.randint(0, c["path"] - 1))) for _ in range(n)]
        s["n_keep"] = _i32([len(k) for k in keep])
        s["keep"] = _i32([k + [-1] * (c["path"] - len(k)) for k in keep])
    if own:
        from paper_2505_14260_gb300 import msd
        r = _rotates(c)
        s["pages"] = msd.Pages(dtype=c["dtype"], layers=layers, heads=H, kv_heads=K, head_dim=hd, page_size=page,
                               n_pages=total, max_seqs=seqs, max_pages=room, rot_dim=r["rot"],
                               rot_sections=r["sections"], rot_interleaved=r["turns"], rope_base=r["base"],
                               kv=kv, table=table, lens=lens, refs=refs)
        s["pages"].restore()
        s["batch"] = msd.Batch(s["seqs"], s["row_start"], int(s["row_start"][-1]))
        if c.get("tree"):
            t = s["tree"] = msd.Tree(n, max(rows))
            t.mask.copy_(s["mask"].reshape(-1))
            t.depth.copy_(s["depth"].reshape(-1))
            t.n_nodes.copy_(s["nodes"])
    torch.cuda.synchronize()
    return s


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------
def _owner(row_start, total):
    """(sequence, row within it) of each row."""
    t = torch.arange(total, device=row_start.device)
    i = torch.searchsorted(row_start[1:].long(), t, right=True)
    return i, t - row_start.long()[i]


def _plain_attention(s):
    c = s["c"]
    n, K, hd, page = c["n"], c["kv_heads"], c["hd"], c["page"]
    G, T = c["heads"] // K, s["q"].shape[0]
    R, S = max(_rows(c)), max(_rows(c)) + max(_prefixes(c))
    starts = s["row_start"].long()
    counts, lens = starts[1:] - starts[:-1], s["lens"].long()[s["seqs"].long()]
    base = lens - counts
    # keys and values of every sequence, padded to the longest
    slot = torch.arange(S, device="cuda")
    held = slot[None] < lens[:, None]
    pid = s["table"][s["seqs"].long()].long()[:, (slot // page).clamp(max=s["room"] - 1)].clamp(min=0)
    layer = s["kv"][0]
    k = torch.where(held[..., None, None], layer[pid, 0, :, slot % page].float(), 0.0)      # [n, S, K, hd]
    v = torch.where(held[..., None, None], layer[pid, 1, :, slot % page].float(), 0.0)
    r = torch.arange(R, device="cuda")
    q = s["q"][(starts[:-1, None] + r).clamp(max=T - 1)].float().view(n, R, K, G, hd)
    # what each row sees
    node = slot[None] - base[:, None]                                                       # row number of a key
    if c["tree"]:
        j = node.clamp(0, R - 1)
        words = s["mask"][torch.arange(n, device="cuda")[:, None, None], r[None, :, None], (j // 64)[:, None]]
        child = (words >> (j % 64)[:, None]) & 1 == 1
        depth = s["depth"].long()
        place_q = base[:, None] + depth
        place_k = torch.where(node >= 0, base[:, None] + depth.gather(1, j), slot[None])
        live = r[None] < s["nodes"][:, None]
    else:
        child = node[:, None] <= r[None, :, None]
        place_q, place_k = base[:, None] + r[None], slot[None].expand(n, S)
        live = r[None] < counts[:, None]
    sees = live[..., None] & held[:, None] & ((node < 0)[:, None] | child)
    if c["window"]:
        sees &= (place_q[..., None] - place_k[:, None] < c["window"]) | (place_k < c["sinks"])[:, None]
    sees = sees[:, None, None]                                                              # [n, 1, 1, R, S]
    z = torch.matmul(q.permute(0, 2, 3, 1, 4), k.permute(0, 2, 3, 1)[:, :, None]) * hd ** -0.5   # [n, K, G, R, S]
    z = z.masked_fill_(~sees, float("-inf"))
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z.sub_(torch.where(m.isfinite(), m, 0.0)))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v.permute(0, 2, 1, 3)[:, :, None]) / torch.where(total > 0, total, 1.0)
    lse = (m + torch.log(total))[..., 0]
    i, at = _owner(s["row_start"], T)
    out = o.permute(0, 3, 1, 2, 4).reshape(n, R, c["heads"], hd)[i, at].to(_dtype(c["dtype"]))
    return {"out": out, "lse": lse.permute(0, 3, 1, 2).reshape(n, R, c["heads"])[i, at]}


def _plain_positions(s):
    c = s["c"]
    T = s["pos"].shape[1]
    i, r = _owner(s["row_start"], T)
    size = c["t"] * c["h"] * c["w"]
    ahead = max((c["t"] - 1) * c["step"] + 1, c["h"], c["w"])
    last = (s["row_start"][1:] - s["row_start"][:-1]).long()
    if not c["images"]:
        return r.to(torch.int32).expand(3, T), last.to(torch.int32)
    first = s["spans"][:, 0].long().view(c["n"], c["images"])[i]                            # [T, images]
    done = (first + size <= r[:, None]).sum(1)
    inside = (first <= r[:, None]) & (r[:, None] < first + size)
    p = r - done * (size - ahead)
    k = (inside * (r[:, None] - first)).sum(1)                                              # place in the span
    p, k, one = p - k, k, inside.any(1)
    at = torch.stack([k // (c["h"] * c["w"]) * c["step"], k // c["w"] % c["h"], k % c["w"]])
    return torch.where(one, p + at, p).to(torch.int32), (last - c["images"] * (size - ahead)).to(torch.int32)


def _plain_rotate(x, pos, r):
    """x [T, heads, hd] in fp32, pos [1 or 3, T]. An angle in turns is a product mod 1:
    whole numbers mod 2^64."""
    half = r["rot"] // 2
    if not half:
        return x
    i = torch.arange(half, device=x.device)
    a, b, d = r["sections"]
    if r["turns"]:
        axis = torch.where((i % 3 == 1) & (i < 3 * b), 1, torch.where((i % 3 == 2) & (i < 3 * d), 2, 0))
    else:
        axis = (i >= a).long() + (i >= a + b).long()
    turn = (torch.pow(r["base"], -2.0 * i.double() / r["rot"]) / (2 * math.pi) * 2.0 ** 64).to(torch.int64)
    p = pos.long().expand(3, -1)[axis].T                                                    # [T, half]
    angle = ((p * turn) >> 32).float() * (2 * math.pi / 2.0 ** 32)
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    u, w = x[..., :half], x[..., half:2 * half]
    return torch.cat([u * cos - w * sin, w * cos + u * sin, x[..., 2 * half:]], -1)


def _plain_append(s, layer, pos):
    """K and V rotated into the last slots of their sequences; q rotated."""
    c = s["c"]
    T, H, K, hd, page = s["qkv"].shape[0], c["heads"], c["kv_heads"], c["hd"], c["page"]
    x = s["qkv"].float().view(T, H + 2 * K, hd)
    turned = _plain_rotate(x[:, :H + K], pos, _rotates(c))
    i, r = _owner(s["row_start"], T)
    starts, seq = s["row_start"].long(), s["seqs"].long()[i]
    slot = s["lens"].long()[seq] - (starts[1:] - starts[:-1])[i] + r
    pid = s["table"].long()[seq, slot // page]
    dt = _dtype(c["dtype"])
    s["kv"][layer][pid, 0, :, slot % page] = turned[:, H:].to(dt)
    s["kv"][layer][pid, 1, :, slot % page] = x[:, H + K:].to(dt)
    return turned[:, :H].to(dt)


def _plain_free(s, seqs):
    seqs = seqs.long()
    rows = s["table"][seqs]
    held = rows >= 0
    s["refs"].scatter_add_(0, rows[held].long(), torch.full_like(rows[held], -1))
    s["table"][seqs] = NEVER
    s["lens"][seqs] = 0


def _take(s, wanted):
    """The lowest free pages, in the order of `wanted` (a mask); 0 refs before this call."""
    free = (s["refs"] == 0).nonzero()[:, 0].to(torch.int32)
    rank = torch.cumsum(wanted.reshape(-1).long(), 0).view(wanted.shape) - 1
    return torch.where(wanted, free[rank.clamp(0, free.numel() - 1)], NEVER)


def _plain_fork(s, src, dst, deep):
    src, dst, page = src.long(), dst.long(), s["c"]["page"]
    lens = s["lens"][src]
    k = torch.arange(s["room"], device="cuda")
    held, whole = k[None] * page < lens[:, None], (k[None] + 1) * page <= lens[:, None]
    fresh = held if deep else held & ~whole
    rows = s["table"][src]
    new = _take(s, fresh)
    s["table"][dst] = torch.where(fresh, new, rows)
    s["lens"][dst] = lens
    shared = rows[held & ~fresh].long()
    s["refs"].scatter_add_(0, shared, torch.ones_like(shared, dtype=torch.int32))
    s["refs"][new[fresh].long()] = 1
    # tokens below the length, not the rest of the page
    some = (torch.arange(page, device="cuda") < (lens[:, None] - k[None] * page)[..., None])[fresh]
    to, of = new[fresh].long(), rows[fresh].long()
    s["kv"][:, to] = torch.where(some[:, None, None, :, None], s["kv"][:, of], s["kv"][:, to])


def _plain_reserve(s, seqs, row_start):
    seqs, page = seqs.long(), s["c"]["page"]
    add = row_start[1:] - row_start[:-1]
    before, after = s["lens"][seqs], s["lens"][seqs] + add
    k = torch.arange(s["room"], device="cuda")[None]
    fresh = (k >= ((before + page - 1) // page)[:, None]) & (k * page < after[:, None])
    new = _take(s, fresh)
    s["table"][seqs] = torch.where(fresh, new, s["table"][seqs])
    s["refs"][new[fresh].long()] = 1
    s["lens"][seqs] = after


def _plain_compact(s, seqs, row_start, keep, n_keep):
    seqs, page = seqs.long(), s["c"]["page"]
    base = s["lens"][seqs].long() - (row_start[1:] - row_start[:-1]).long()
    after, width = base + n_keep.long(), keep.shape[1]
    j = torch.arange(width, device="cuda")[None]
    live = j < n_keep[:, None]
    moved = live & (keep != j)
    still = torch.where(moved.any(1), moved.long().argmax(1), n_keep.long())
    first = (base + still) // page                                                          # first page that changes
    k = torch.arange(s["room"], device="cuda")[None]
    rows = s["table"][seqs]
    held = rows >= 0
    stays = k * page < after[:, None]
    shared = held & (s["refs"][rows.clamp(min=0).long()] > 1)
    fresh = stays & (k >= first[:, None]) & shared
    new = _take(s, fresh)
    gone = rows[held & (fresh | ~stays)].long()
    now = torch.where(fresh, new, torch.where(stays, rows, NEVER))
    # every token of a page that changes: from its old place to its new one
    slot = torch.arange(s["room"] * page, device="cuda")[None]
    t = slot - base[:, None]
    source = torch.where(t < 0, slot, base[:, None] + keep.long().gather(1, t.clamp(0, width - 1)))
    some = (slot < after[:, None]) & (slot // page >= first[:, None])
    i = torch.arange(seqs.numel(), device="cuda")[:, None].expand_as(some)[some]
    source, to = source[some], slot.expand_as(some)[some]
    of = rows[i, source // page].long()
    values = s["kv"][:, of, :, :, source % page]
    s["kv"][:, now[i, to // page].long(), :, :, to % page] = values
    s["refs"].scatter_add_(0, gone, torch.full_like(gone, -1, dtype=torch.int32))
    s["refs"][new[fresh].long()] = 1
    s["table"][seqs] = now
    s["lens"][seqs] = after.to(torch.int32)


def _state(s):
    return {"table": s["table"], "lens": s["lens"], "refs": s["refs"], "kv": s["kv"]}


def _append_layers(s):
    c = s["c"]
    return [_plain_append(s, layer, s["pos"]) for layer in range(c["layers"])][-1]


def _run_plain(s):
    c = s["c"]
    if c["kind"] == "attention":
        return _plain_attention(s)
    if c["kind"] == "rope":
        if c["decode"]:
            return {"q": _plain_append(s, 0, s["pos"]), "kv": s["kv"]}
        pos, after = _plain_positions(s)
        return {"pos": pos, "next": after, "q": _plain_append(s, 0, pos), "kv": s["kv"]}
    _plain_free(s, s["dst"])
    _plain_fork(s, s["src"], s["dst"], c.get("deep", False))
    if c["kind"] == "fork":
        return _state(s)
    more = {}
    if c["kind"] == "step":
        _plain_reserve(s, s["seqs"], s["row_start"])
        more["q"] = _append_layers(s)
    _plain_compact(s, s["seqs"], s["row_start"], s["keep"], s["n_keep"])
    return {**_state(s), **more}


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _split(s):
    c = s["c"]
    H, K, hd = c["heads"], c["kv_heads"], c["hd"]
    q, k, v = s["qkv"].split([H * hd, K * hd, K * hd], 1)
    return q, k, v


def _append_own(s, layer, pos):
    q, k, v = _split(s)
    return s["pages"].rope_append(layer, s["batch"], q, k, v, pos, s["q_out"])


def run(state):
    s, c = state, state["c"]
    if not own:
        return _run_plain(s)
    pages = s["pages"]
    if c["kind"] == "attention":
        pages.attention(0, s["batch"], s["q"], s["out"], lse=s["lse"], tree=s.get("tree"), window=c["window"],
                        sinks=c["sinks"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["kind"] == "rope":
        if c["decode"]:
            return {"q": _append_own(s, 0, s["pos"]), "kv": s["kv"]}
        pages.positions(s["batch"], s["span_start"], s["spans"], s["pos"], s["next"])
        return {"pos": s["pos"], "next": s["next"], "q": _append_own(s, 0, s["pos"]), "kv": s["kv"]}
    pages.free(s["dst"])
    pages.fork(s["src"], s["dst"], deep=c.get("deep", False))
    if c["kind"] == "fork":
        return _state(s)
    more = {}
    if c["kind"] == "step":
        pages.reserve(s["batch"])
        more["q"] = [_append_own(s, layer, s["pos"]) for layer in range(c["layers"])][-1]
    pages.compact(s["batch"], s["keep"], s["n_keep"])
    return {**_state(s), **more}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def _seen(L, rows, window, sinks):
    """(row, key) pairs and keys that some row of a chunk sees."""
    if not window:
        return sum(L + r + 1 for r in range(rows)), L + rows
    pairs = sum(min(L + r + 1, window) + min(sinks, max(0, L + r + 1 - window)) for r in range(rows))
    return pairs, min(L + rows, window + rows - 1 + sinks)


def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    hd, H, K, page = c["hd"], c["heads"], c["kv_heads"], c["page"]
    rows, before, layers = _rows(c), _prefixes(c), c.get("layers", 1)
    token = 2 * K * hd * size
    if c["kind"] == "attention":
        nbytes = flops = 0
        for L, r in zip(before, rows):
            if c["tree"]:       # a row sees the prefix and a path; every node is on some path
                pairs, keys = _seen(L + 1, 1, c["window"], c["sinks"])
                pairs, keys = (pairs - 1) * r + 5 * r, keys - 1 + r
            else:
                pairs, keys = _seen(L, r, c["window"], c["sinks"])
            nbytes += keys * token + 2 * r * H * hd * size + 4 * r * H + 4 * (keys // page + 1)
            flops += 4 * hd * H * pairs
        return {"bytes": nbytes, "flops": flops}
    T = sum(rows)
    src = 4 if c.get("src", "f32") == "f32" else 2
    append = T * ((H + 2 * K) * hd * (src + size) + 12)
    turning = 6 * T * (H + K) * c.get("rot", hd) // 2
    if c["kind"] == "rope":
        return {"bytes": append, "flops": turning}
    pages = sum(-(-p // page) for p in before)
    if c["kind"] == "fork":
        tokens = sum(c["fan"] * (p if c["deep"] else p % page) for p in before)
        return {"bytes": 2 * tokens * token * layers + 16 * c["fan"] * pages, "flops": 0}
    if c["kind"] == "evict":
        # what is kept, where anything is dropped (the source keeps its own pages), else the fork's last page
        tokens = sum(_kept({**c, "prefix": p}) if p > c["first"] + c["newest"] else p % page for p in before)
        return {"bytes": 2 * tokens * token * layers + 16 * pages, "flops": 0}
    tokens = sum(p % page for p in before) + c["n"] * (c["path"] - 1) // 2
    return {"bytes": layers * (append + 2 * tokens * token) + 16 * pages, "flops": layers * turning}


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------
def _exact_attention(s):
    c = s["c"]
    K, hd, page = c["kv_heads"], c["hd"], c["page"]
    G = c["heads"] // K
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(out.shape[:2], float("-inf"), dtype=torch.float64, device="cuda")
    starts, lens = s["row_start"].tolist(), s["lens"].tolist()
    for i, seq in enumerate(s["seqs"].tolist()):
        a, b, S = starts[i], starts[i + 1], lens[seq]
        R, L = b - a, S - (b - a)
        pids = s["table"][seq, : -(-S // page)].long()
        place = torch.arange(S, device="cuda")
        see = torch.ones(R, S, dtype=torch.bool, device="cuda")
        if c["tree"]:
            place = torch.cat([place[:L], L + s["depth"][i, :R].long()])
            words = s["mask"][i, :R].view(R, -1, 1)
            see[:, L:] = (((words >> torch.arange(64, device="cuda")) & 1) == 1).reshape(R, -1)[:, :R]
            see[s["nodes"].tolist()[i]:] = False
        else:
            see = see.tril(L)
        if c["window"]:
            near = place[L:, None] - place[None] < c["window"]
            see &= near | (place < c["sinks"])[None]
        for h in range(K):
            k = s["kv"][0, pids, 0, h].reshape(-1, hd)[:S].double()
            v = s["kv"][0, pids, 1, h].reshape(-1, hd)[:S].double()
            for top in range(0, R, 1024):
                rows = slice(top, min(top + 1024, R))
                q = s["q"][a:b][rows, h * G:(h + 1) * G].double()
                z = torch.einsum("rgd,sd->rgs", q, k) / math.sqrt(hd)
                z = torch.where(see[rows, None], z, float("-inf"))
                e = torch.logsumexp(z, -1)
                p = torch.exp(z - torch.where(e.isfinite(), e, 0.0)[..., None])
                at = slice(a + rows.start, a + rows.stop)
                out[at, h * G:(h + 1) * G] = torch.einsum("rgs,sd->rgd", p, v)
                lse[at, h * G:(h + 1) * G] = e
    return {"out": out, "lse": lse}


def _exact_positions(c, rows):
    """Token by token, on the host."""
    columns, after, size = [], [], c["t"] * c["h"] * c["w"]
    for i, total in enumerate(rows):
        text, first = total - c["images"] * size, min(8, max(1, _spread(c["text"], 2, i) - 1))
        gap = max(0, (text - first) // (c["images"] + 1))
        begins = {first + k * (size + gap) for k in range(c["images"])}
        p, r = 0, 0
        while r < total:
            if r in begins:
                columns += [(p + a * c["step"], p + b, p + d) for a in range(c["t"]) for b in range(c["h"])
                            for d in range(c["w"])]
                p, r = p + max((c["t"] - 1) * c["step"] + 1, c["h"], c["w"]), r + size
            else:
                columns.append((p, p, p))
                p, r = p + 1, r + 1
        after.append(p)
    return torch.tensor(columns, dtype=torch.float64, device="cuda").T, after


def _exact_turn(s, pos):
    """The rotated heads as complex numbers in polar form."""
    c = s["c"]
    rot, H, K, hd = c.get("rot", c["hd"]), c["heads"], c["kv_heads"], c["hd"]
    x = s["qkv"].double().view(-1, H + 2 * K, hd).clone()
    half = rot // 2
    a, b, d = _sections(c)
    axis = [0] * a + [1] * b + [2] * d
    if c.get("turns"):
        axis = [0] * half
        for i in range(b):
            axis[3 * i + 1] = 1
        for i in range(d):
            axis[3 * i + 2] = 2
    for i in range(half):
        angle = pos[axis[i] if len(pos) > 1 else 0].double() * 10000.0 ** (-2 * i / rot)
        z = torch.complex(x[:, :H + K, i], x[:, :H + K, i + half]) * torch.polar(torch.ones_like(angle), angle)[:, None]
        x[:, :H + K, i], x[:, :H + K, i + half] = z.real, z.imag
    return x[:, :H], x[:, H:H + K], x[:, H + K:]


def _exact_store(s, layer, k, v, kv):
    page, at = s["c"]["page"], 0
    starts = s["row_start"].tolist()
    for i, seq in enumerate(s["seqs"].tolist()):
        rows = starts[i + 1] - starts[i]
        slot = torch.arange(s["lens"][seq].item() - rows, s["lens"][seq].item(), device="cuda")
        pid = s["table"][seq].long()[slot // page]
        kv[layer, pid, 0, :, slot % page] = k[at:at + rows]
        kv[layer, pid, 1, :, slot % page] = v[at:at + rows]
        at += rows


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["kind"] == "attention":
        return _exact_attention(s)
    if c["kind"] == "rope":
        pos = s["pos"] if c["decode"] else _exact_positions(c, _rows(c))[0]
        q, k, v = _exact_turn(s, pos)
        kv = s["kv"].double()
        _exact_store(s, 0, k, v, kv)
        return {"pos": None, "next": None, "q": q, "kv": kv} if not c["decode"] else {"q": q, "kv": kv}
    if c["kind"] == "step":
        q, _, _ = _exact_turn(s, s["pos"])
        return {"table": None, "lens": None, "refs": None, "kv": None, "q": q}
    return None                      # page ids and copies: no computed numbers
