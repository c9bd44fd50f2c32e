"""Operator cases of a decode step outside attention: products with 4-bit weights, and the
way from logits to tokens, through the public binding (paper_2505_14260_gb300.msd).

Kinds of case
  linear    y = x W^T, W in 4-bit codes with a scale (and a zero) for each group of a row:
            one token, a few drafts, a drafted tree, a prompt. x bf16 or fp32, y fp32.
  quantize  such a W from a bf16 or fp32 matrix: codes, scales, zeros, and the values that
            the codes stand for.
  sample    a token for each row of logits from a given uniform, at the row's temperature,
            top-k, top-p and min-p, with its log-probability; with `probs` the whole
            distribution that is left.
  accept    speculative sampling over the drafted trees of a batch of requests, each with
            its own settings: the accepted path, its length and the next token.

Widths are those of this repository's workloads (hidden 256, 4096 and 5120, ffn 688, 11008
and 13824, vocabularies of 1024 and 32000) and generic ones. Products and quantisation are
computed in 32 bits in the plain forms; what decides on a token is in 64, since a uniform
may lie next to a border of two tokens' masses.
"""
import math
import random

import numpy as np
import torch

own = False


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _linear(m, k, o, group, zeros, x):
    return dict(kind="linear", m=m, k=k, o=o, group=group, zeros=zeros, x=x)


def _quantize(k, o, group, zeros, w):
    return dict(kind="quantize", k=k, o=o, group=group, zeros=zeros, w=w)


def _sample(rows, vocab, x, t, k, p, min_p, masked=0.0, probs=False):
    """t, k, p, min_p: the largest settings of the rows; `masked`: share of tokens at -inf."""
    return dict(kind="sample", rows=rows, vocab=vocab, x=x, t=t, k=k, p=p, min_p=min_p, masked=masked, probs=probs)


def _accept(n, nodes, depth, children, vocab, x, t, k, p, min_p):
    return dict(kind="accept", n=n, nodes=nodes, depth=depth, children=children, vocab=vocab, x=x, t=t, k=k, p=p,
                min_p=min_p)


def listed():
    return [
        # one token of one request through a 7B attention projection: the smallest product
        dict(_linear(1, 4096, 4096, 128, False, "bf16"), name="linear_token_7b"),
        # a pass of the draft: ten frontier rows through a 7B down projection, finer groups with zeros
        dict(_linear(10, 11008, 4096, 64, True, "bf16"), name="linear_drafts_7b_down"),
        # a 7B request's tree of 60 nodes through an up projection
        dict(_linear(60, 4096, 11008, 128, True, "bf16"), name="linear_tree_7b_up"),
        # the head of a 13B model for 16 requests, activations kept in fp32
        dict(_linear(16, 5120, 32000, 32, False, "f32"), name="linear_head_13b_f32"),
        # a multimodal prompt of ragged length (576 + 69 tokens) through an up projection
        dict(_linear(645, 4096, 11008, 128, False, "bf16"), name="linear_prompt_7b"),
        # one 7B attention projection brought to 4 bits
        dict(_quantize(4096, 4096, 128, False, "bf16"), name="quantize_7b"),
        # a 13B head from fp32 masters, the finest groups, with zeros
        dict(_quantize(5120, 32000, 32, True, "f32"), name="quantize_head_13b_f32"),
        # the next token of one request, usual settings: the smallest draw
        dict(_sample(1, 32000, "f32", 0.7, 50, 0.9, 0.0), name="sample_one"),
        # 64 requests over a large odd vocabulary, a tenth of it ruled out by a grammar, bf16 logits
        dict(_sample(64, 100003, "bf16", 1.2, 0, 0.95, 0.0, masked=0.1), name="sample_batch64_bf16"),
        # the distributions of a tree's 60 rows, as drafting from them or a loss on them wants them
        dict(_sample(60, 32000, "f32", 1.0, 2000, 0.99, 0.001, probs=True), name="sample_probs_tree"),
        # a 7B request's drafted tree of 60 nodes
        dict(_accept(1, 60, 6, 10, 32000, "f32", 1.0, 0, 0.9, 0.0), name="accept_tree_7b"),
        # 16 requests with a tree each
        dict(_accept(16, 60, 6, 10, 32000, "f32", 0.8, 200, 0.95, 0.02), name="accept_batch16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST_FLOPS = 5.81e10         # as the largest listed product
_MOST_BYTES = 1.4e9           # as the largest listed quantisation
_MOST_LOGITS = 2.6e7          # as the largest listed batch of trees


def _draw_settings(rng):
    return dict(t=rng.choice([0.3, 0.7, 1.0, 1.7]), k=rng.choice([0, 0, 1, 40, 1000]),
                p=rng.choice([1.0, 0.5, 0.9, 0.99]), min_p=rng.choice([0.0, 0.0, 0.05, 0.3]))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "quantize", "sample", "sample", "accept", "accept"])
    x = rng.choice(["bf16", "f32"])
    if kind in ("linear", "quantize"):
        k = rng.choice([256, 688, 4096, 5120, 11008, 13824, 8 * _log_int(rng, 1, 1800)])
        o = rng.choice([256, 688, 4096, 5120, 11008, 13824, _log_int(rng, 1, 32000)])
        group, zeros = rng.choice([32, 64, 128]), rng.random() < 0.5
        c = _quantize(k, o, group, zeros, x)
        if kind == "linear":
            c = _linear(rng.choice([1, 1, rng.randint(2, 16), rng.randint(17, 130), _log_int(rng, 2, 2000)]), k, o,
                        group, zeros, x)
    elif kind == "sample":
        vocab = rng.choice([1024, 32000, _log_int(rng, 2, 150000)])
        rows = rng.choice([1, rng.randint(2, 64), _log_int(rng, 2, 960)])
        c = _sample(rows, vocab, x, masked=rng.choice([0.0, 0.0, 0.3]), probs=rng.random() < 0.3, **_draw_settings(rng))
    else:
        c = _accept(_log_int(rng, 1, 16), rng.choice([16, 60, rng.randint(1, 130)]), rng.randint(1, 9), rng.randint(1, 16),
                    rng.choice([1024, 32000, _log_int(rng, 40, 60000)]), x, **_draw_settings(rng))
    w = work(c)
    logits = c.get("rows", c.get("n", 0) * c.get("nodes", 0)) * c.get("vocab", 0)
    return c if w["flops"] <= _MOST_FLOPS and w["bytes"] <= _MOST_BYTES and logits <= _MOST_LOGITS else draw(rng)


_SIZE = {"bf16": 2, "f32": 4}


def _groups(c):
    return -(-c["k"] // c["group"])


def work(c):
    if c["kind"] in ("linear", "quantize"):
        weight = c["o"] * (c["k"] / 2 + _groups(c) * (3 if c["zeros"] else 2))
        if c["kind"] == "linear":
            return {"bytes": weight + c["m"] * (c["k"] * _SIZE[c["x"]] + 4 * c["o"]), "flops": 2.0 * c["m"] * c["k"] * c["o"]}
        return {"bytes": weight + 2 * c["o"] * c["k"] * _SIZE[c["w"]], "flops": 4.0 * c["o"] * c["k"]}
    if c["kind"] == "sample":
        n = c["rows"] * c["vocab"]
        return {"bytes": n * (_SIZE[c["x"]] + (4 if c["probs"] else 0)) + 28 * c["rows"], "flops": 4.0 * n}
    rows = sum(_nodes(c))
    return {"bytes": rows * (c["vocab"] * _SIZE[c["x"]] + 8) + 4 * c["n"] * (c["depth"] + 1) * (c["children"] + 2),
            "flops": 4.0 * rows * c["vocab"]}


def _nodes(c):
    """Trees of a batch are ragged: the first is whole, the others have fewer nodes."""
    return [max(1, c["nodes"] - (i * 7) % max(1, c["nodes"] // 3)) for i in range(c["n"])]


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _inputs_linear(c, g):
    o, k, G = c["o"], c["k"], _groups(c)
    rand = dict(generator=g, device="cuda")
    codes = torch.empty(o, k // 2, dtype=torch.uint8, device="cuda")
    for at in range(0, o, 8192):                                   # in parts: fp32 stand-ins of a large matrix
        n = torch.randn(min(8192, o - at), k, **rand).mul_(2.4).round_().add_(8).clamp_(0, 15).to(torch.uint8)
        codes[at:at + n.shape[0]] = n[:, 0::2] | (n[:, 1::2] << 4)
    scales = (0.006 * (0.5 + torch.rand(o, G, **rand))).bfloat16()
    zeros = torch.randint(5, 11, (o, G), dtype=torch.uint8, **rand) if c["zeros"] else None
    # a few channels of a decoder's activations are much larger than the others
    x = torch.randn(c["m"], k, **rand) * torch.where(torch.rand(k, **rand) < 0.01, 20.0, 1.0)
    return dict(codes=codes, scales=scales, zeros=zeros, x=x.to(_dtype(c["x"])))


def _inputs_quantize(c, g):
    w = torch.randn(c["o"], c["k"], generator=g, device="cuda").mul_(0.02)
    w[:, :: 97] *= 6.0
    return dict(w=w.to(_dtype(c["w"])))


def _logits(rows, vocab, g):
    """A bulk of unlikely tokens and some hundred likely ones, as a trained head gives."""
    x = torch.randn(rows, vocab, generator=g, device="cuda").mul_(2.0)
    n = min(300, vocab)
    at = torch.randint(0, vocab, (rows, n), generator=g, device="cuda")
    peak = 13.0 - 1.6 * torch.log1p(torch.arange(n, device="cuda").float())
    return x.scatter_reduce_(1, at, peak + torch.randn(rows, n, generator=g, device="cuda"), "amax")   # an id may come twice


def _settings(c, n):
    """Row 0 has the case's settings, the others go down from them; every fifth row of a batch is greedy."""
    i = torch.arange(n, device="cuda")
    t = c["t"] * (1 - 0.1 * (i % 4).float())
    t[i % 5 == 4] = 0.0
    s = {"temperature": t}
    if c["k"]:
        s["top_k"] = (c["k"] - (i % 3) * (c["k"] // 4)).to(torch.int32)
    if c["p"] < 1:
        s["top_p"] = c["p"] * (1 - 0.05 * (i % 3).float())
    if c["min_p"]:
        s["min_p"] = c["min_p"] * (1 + 0.25 * (i % 2).float())
    return s


def _inputs_sample(c, g):
    x = _logits(c["rows"], c["vocab"], g)
    if c["masked"]:
        out = torch.rand(x.shape, generator=g, device="cuda") < c["masked"]
        out[:, 0] = False                                          # something is left of a small vocabulary
        x.masked_fill_(out, -math.inf)
    return dict(logits=x.to(_dtype(c["x"])), u=torch.rand(c["rows"], generator=g, device="cuda"),
                settings=_settings(c, c["rows"]))


def _inputs_accept(c, seed, g):
    counts, N, n = _nodes(c), c["nodes"], c["n"]
    starts = np.concatenate([[0], np.cumsum(counts)])
    logits = _logits(int(starts[-1]), c["vocab"], g).to(_dtype(c["x"]))
    r = random.Random(seed)
    parent, depth = np.full((n, N), -1, np.int32), np.zeros((n, N), np.int32)
    ordinal, see = np.zeros((n, N), np.int64), np.zeros((n, N, N), bool)
    for b in range(n):
        born = np.zeros(N, np.int64)
        see[b, 0, 0] = True
        for j in range(1, N):
            open_ = [i for i in range(max(0, j - 24), j) if depth[b, i] < c["depth"] and born[i] < c["children"]]
            p = r.choice(open_[:4]) if open_ else 0
            parent[b, j], depth[b, j], ordinal[b, j] = p, depth[b, p] + 1, born[p]
            born[p] += 1
            see[b, j] = see[b, p]
            see[b, j, j] = True
    # a child's token: the parent's likeliest ones in turn, as a draft that is near its target proposes
    width = min(max(c["children"], int(ordinal.max()) + 1), c["vocab"])
    best = torch.topk(logits.float(), width).indices.cpu().numpy()
    tokens = np.zeros((n, N), np.int32)
    for b in range(n):
        for j in range(1, counts[b]):
            tokens[b, j] = best[starts[b] + parent[b, j], ordinal[b, j] % width]
    words = -(-N // 64)
    bits = np.zeros((n, N, words * 64), np.uint64)
    bits[:, :, :N] = see
    mask = (bits.reshape(n, N, words, 64) << np.arange(64, dtype=np.uint64)).sum(-1, dtype=np.uint64).view(np.int64)
    u = torch.rand(n, c["depth"] + 1, c["children"] + 1, generator=g, device="cuda")
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    return dict(logits=logits, u=u, settings=_settings(c, n), tokens=dev(tokens), parent=dev(parent), depth=dev(depth),
                mask=dev(mask), counts=dev(np.array(counts, np.int32)), starts=dev(starts.astype(np.int32)),
                seqs=torch.arange(n, dtype=torch.int32, device="cuda"))


def _inputs(c, seed):
    g = _gen(seed)
    if c["kind"] == "accept":
        return _inputs_accept(c, seed, g)
    return {"linear": _inputs_linear, "quantize": _inputs_quantize, "sample": _inputs_sample}[c["kind"]](c, g)


def prepare(case, seed):
    c, s = case, dict(_inputs(case, seed), c=case)
    new = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    if c["kind"] == "linear":
        s["y"] = new(c["m"], c["o"])
    elif c["kind"] == "quantize":
        s.update(codes=new(c["o"], c["k"] // 2, dtype=torch.uint8), scales=new(c["o"], _groups(c), dtype=torch.bfloat16),
                 zeros=new(c["o"], _groups(c), dtype=torch.uint8) if c["zeros"] else None, values=torch.empty_like(s["w"]))
    elif c["kind"] == "sample":
        s.update(tokens=new(c["rows"], dtype=torch.int32), logp=new(c["rows"]),
                 probs=new(c["rows"], c["vocab"]) if c["probs"] else None)
    else:
        s.update(path=new(c["n"], c["depth"] + 1, dtype=torch.int32), accept_len=new(c["n"], dtype=torch.int32),
                 bonus=new(c["n"], dtype=torch.int32))
    if own:
        from paper_2505_14260_gb300 import msd
        s["msd"] = msd
        if c["kind"] == "linear":
            s["weight"] = msd.Weight4(s["codes"], s["scales"], s["zeros"], group=c["group"])
        elif c["kind"] == "quantize":
            s["weight"] = msd.Weight4(s["codes"], s["scales"], s["zeros"], group=c["group"])
        else:
            s["filter"] = msd.Filter(**s["settings"])
        if c["kind"] == "accept":
            s["batch"] = msd.Batch(s["seqs"], s["starts"], s["logits"].shape[0])
            tree = s["tree"] = msd.Tree(c["n"], c["nodes"])
            for name, of in (("tokens", "tokens"), ("parent", "parent"), ("depth", "depth"), ("mask", "mask"),
                             ("n_nodes", "counts")):
                getattr(tree, name).copy_(s[of].reshape(-1))
    return s


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------
def _spread(t, c):
    """A group's values for each element of its rows."""
    return t.float().repeat_interleave(c["group"], 1)[:, :c["k"]]


def _codes(packed):
    return torch.stack([packed & 15, packed >> 4], -1).view(packed.shape[0], -1)


def _plain_linear(s):
    c = s["c"]
    zero = _spread(s["zeros"], c) if c["zeros"] else 8.0
    return s["x"].float() @ (_spread(s["scales"], c) * (_codes(s["codes"]).float() - zero)).T


def _plain_quantize(s):
    """Quotients in 64 bits: in 32 some fall on a border of two codes that they only lie next to."""
    c, w, G = s["c"], s["w"], _groups(s["c"])
    short = G * c["group"] - c["k"]
    w = torch.nn.functional.pad(w.float(), (0, short)).view(c["o"], G, c["group"])
    if c["zeros"]:
        lo, hi = w.amin(-1).clamp(max=0), w.amax(-1).clamp(min=0)
        scales = ((hi.double() - lo.double()) / 15)
    else:
        scales = w.abs().amax(-1).double() / 7
    scales = _to_bf16(scales)
    step = torch.where(scales > 0, scales.double(), 1.0)
    zero = torch.round(-lo.double() / step).clamp(0, 15) if c["zeros"] else torch.full_like(step, 8.0)
    q = torch.round(w.double() / step[..., None]).add_(zero[..., None]).clamp_(0, 15)
    values = (scales.float()[..., None] * (q.float() - zero.float()[..., None])).view(c["o"], -1)[:, :c["k"]]
    q = q.view(c["o"], -1)[:, :c["k"]].to(torch.uint8)
    return {"codes": q[:, 0::2] | (q[:, 1::2] << 4), "scales": scales.contiguous(),
            "zeros": zero.to(torch.uint8) if c["zeros"] else None, "values": values.to(s["w"].dtype)}


def _to_bf16(x):
    """64 bits to bf16 in one rounding: the fp32 value is rounded to odd first."""
    f = x.float()
    bits = f.view(torch.int32)
    off = (f.double() != x) & (bits & 1 == 0)
    return (bits + torch.where(off, torch.where(f.double() < x, 1, -1), 0).int()).view(torch.float32).bfloat16()


def _weights(x, settings, row):
    """exp((x - max) / T) of each row's kept tokens, in id order and 64 bits, 0 elsewhere."""
    at = lambda name, off: settings[name][row].double()[:, None] if name in settings else off  # noqa: E731
    x = x.double()
    top = x.amax(1, keepdim=True)
    T = at("temperature", 1.0)
    w = torch.exp((x - top) / torch.where(T > 0, T, 1.0))
    del x
    order = torch.sort(torch.where(w > 0, w, 0.0), dim=1, descending=True, stable=True)
    rank = torch.arange(w.shape[1], device=w.device)[None]
    k = at("top_k", 0.0)
    sorted_ = order.values * ((rank < k) | (k <= 0) if "top_k" in settings else True)
    before = torch.cumsum(sorted_, 1) - sorted_
    p = at("top_p", 1.0)
    kept = (before < p * sorted_.sum(1, keepdim=True)) | (p >= 1) if "top_p" in settings else sorted_ > 0
    kept = kept & (sorted_ >= at("min_p", 0.0)) & ((T > 0) | (rank == 0)) | (rank == 0)
    return torch.zeros_like(w).scatter_(1, order.indices, torch.where(kept, sorted_, 0.0))


def _draw_token(w, u):
    """The smallest id whose cumulative mass exceeds u of the whole."""
    mass = torch.cumsum(w, 1)
    return (mass <= u.double()[:, None] * mass[:, -1:]).sum(1)


def _plain_sample(s):
    w = _weights(s["logits"], s["settings"], slice(None))
    t = _draw_token(w, s["u"])
    total = w.sum(1, keepdim=True)
    out = {"tokens": t.int(), "logp": torch.log(w.gather(1, t[:, None]) / total)[:, 0].float()}
    if s["probs"] is not None:
        out["probs"] = (w / total).float()
    return out


def _plain_accept(s):
    c = s["c"]
    n, N, D, k = c["n"], c["nodes"], c["depth"], c["children"]
    node = torch.arange(N, device="cuda")
    live = node[None] < s["counts"][:, None]
    owner = torch.repeat_interleave(torch.arange(n, device="cuda"), s["counts"].long(), output_size=s["logits"].shape[0])
    w = _weights(s["logits"], s["settings"], owner)
    parent, depth, tokens = s["parent"].long().clamp(min=0), s["depth"].long(), s["tokens"].long()
    above = s["starts"][:-1, None].long() + torch.where(live, parent, 0)
    # [b, j, i]: child i of the same parent comes before j
    elder = (parent[:, :, None] == parent[:, None]) & (node[:, None] > node) & (node > 0) & (live[:, :, None] & live[:, None])
    ordinal = elder.sum(2)
    again = (elder & (tokens[:, :, None] == tokens[:, None])).any(2)
    tried = live & (node > 0) & (ordinal < k) & (depth <= D)
    mass = torch.where(tried & ~again, w[above, tokens], 0.0)
    left = w.sum(1)[above] - (elder.double() @ mass[..., None])[..., 0]
    u = s["u"].double()
    b = torch.arange(n, device="cuda")[:, None]
    taken = tried & (u[b, (depth - 1).clamp(0, D), ordinal.clamp(max=k)] * left < mass)
    taken &= ~(elder & taken[:, None]).any(2)                       # the first child that is accepted
    see = ((s["mask"].view(n, N, -1, 1) >> torch.arange(64, device="cuda")) & 1).view(n, N, -1)[..., :N].bool()
    on = (~see | (taken | (node == 0))[:, None]).all(2) & live     # all of a node's ancestors and itself
    length = on.sum(1) - 1
    path = torch.full((n, D + 2), -1, dtype=torch.int32, device="cuda")
    path.scatter_(1, torch.where(on, depth, D + 1), torch.where(on, node[None], -1).int())
    path[:, D + 1] = -1
    last = path.gather(1, length[:, None]).long()
    rest = w[(s["starts"][:-1, None].long() + last)[:, 0]]
    gone = tried & (parent == last)                                 # rejected children; a column behind the ids for the others
    rest = torch.cat([rest, rest[:, :1]], 1).scatter_(1, torch.where(gone, tokens, c["vocab"]), 0.0)[:, :-1]
    bonus = _draw_token(rest, s["u"][b[:, 0], length, torch.full_like(length, k)])
    return {"path": path[:, :D + 1].contiguous(), "accept_len": length.int(), "bonus": bonus.int()}


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(state):
    s, c = state, state["c"]
    if c["kind"] == "linear":
        return s["weight"].linear(s["x"], s["y"]) if own else _plain_linear(s)
    if c["kind"] == "quantize":
        if own:
            s["weight"].quantize(s["w"], values=s["values"])
            return {n: s[n] for n in ("codes", "scales", "zeros", "values")}
        return _plain_quantize(s)
    if c["kind"] == "sample":
        if own:
            s["msd"].sample(s["logits"], s["u"], s["filter"], s["tokens"], logp=s["logp"], probs=s["probs"])
            return {n: s[n] for n in ("tokens", "logp", "probs") if s[n] is not None}
        return _plain_sample(s)
    if own:
        s["msd"].accept(s["logits"], s["batch"], s["tree"], s["u"], s["filter"], s["path"], s["accept_len"], s["bonus"])
        return {n: s[n] for n in ("path", "accept_len", "bonus")}
    return _plain_accept(s)


# ---------------------------------------------------------------------------
# From the definitions, in 64 bits
# ---------------------------------------------------------------------------
def _exact_linear(c, s):
    x, out = s["x"].double(), torch.empty(c["m"], c["o"], dtype=torch.float64, device="cuda")
    for at in range(0, c["o"], 2048):
        part = slice(at, min(at + 2048, c["o"]))
        code = torch.empty(part.stop - at, c["k"], dtype=torch.float64, device="cuda")
        code[:, 0::2], code[:, 1::2] = (s["codes"][part] % 16).double(), (s["codes"][part] // 16).double()
        total = torch.zeros(c["m"], part.stop - at, dtype=torch.float64, device="cuda")
        for g in range(_groups(c)):
            at_k = slice(g * c["group"], min((g + 1) * c["group"], c["k"]))
            zero = s["zeros"][part, g].double()[:, None] if c["zeros"] else 8.0
            total += (x[:, at_k] @ (code[:, at_k] - zero).T) * s["scales"][part, g].double()[None]
        out[:, part] = total
    return out


def _exact_quantize(c, s):
    w = s["w"].float().cpu().numpy().astype(np.float64)
    G = _groups(c)
    codes, scales = np.zeros(w.shape, np.uint8), np.zeros((c["o"], G), np.float64)
    zeros, values = np.full((c["o"], G), 8.0), np.zeros(w.shape)
    for g in range(G):
        part = w[:, g * c["group"]:(g + 1) * c["group"]]
        span = np.maximum(part.max(1), 0) - np.minimum(part.min(1), 0) if c["zeros"] else np.abs(part).max(1)
        wide = span / (15 if c["zeros"] else 7)
        e = np.floor(np.log2(np.where(wide > 0, wide, 1.0))) - 7          # 8 significant bits
        sc = np.rint(wide / 2.0 ** e) * 2.0 ** e
        div = np.where(sc > 0, sc, 1.0)
        if c["zeros"]:
            zeros[:, g] = np.clip(np.rint(-np.minimum(part.min(1), 0) / div), 0, 15)
        q = np.clip(np.rint(part / div[:, None]) + zeros[:, g, None], 0, 15)
        codes[:, g * c["group"]:(g + 1) * c["group"]] = q
        values[:, g * c["group"]:(g + 1) * c["group"]] = sc[:, None] * (q - zeros[:, g, None])
        scales[:, g] = sc
    return {"codes": codes[:, 0::2] + 16 * codes[:, 1::2], "scales": scales,
            "zeros": zeros.astype(np.uint8) if c["zeros"] else None, "values": values}


class _Row:
    """The filtered distribution of one row of logits, by sorting."""

    def __init__(self, x, settings, i):
        x = x.astype(np.float64)
        T, k = settings.get("temperature"), settings.get("top_k")
        p, m = settings.get("top_p"), settings.get("min_p")
        T = 1.0 if T is None else float(T[i])
        order = np.lexsort((np.arange(x.size), -x))
        order = order[x[order] > -np.inf]
        if T <= 0:
            order = order[:1]
        w = np.exp((x[order] - x[order[0]]) / (T if T > 0 else 1.0))
        if k is not None and int(k[i]) > 0:
            order, w = order[:int(k[i])], w[:int(k[i])]
        most = len(w)
        if p is not None and float(p[i]) < 1:
            mass = np.cumsum(w)
            most = int(np.searchsorted(mass, float(p[i]) * mass[-1])) + 1   # the shortest prefix that reaches p
        if m is not None:
            most = min(most, int(np.sum(w >= float(m[i]))))
        most = max(most, 1)
        self.w = np.zeros(x.size)
        self.w[order[:most]] = w[:most]

    def draw(self, u):
        mass = np.cumsum(self.w)
        return int(np.searchsorted(mass, u * mass[-1], side="right"))


def _host(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _exact_sample(c, s):
    x, u, settings = _host(s["logits"]), _host(s["u"]).astype(np.float64), {k: _host(v) for k, v in s["settings"].items()}
    tokens, logp = np.zeros(c["rows"], np.int32), np.zeros(c["rows"])
    probs = np.zeros(x.shape) if c["probs"] else None
    for i in range(c["rows"]):
        r = _Row(x[i], settings, i)
        tokens[i] = r.draw(u[i])
        logp[i] = np.log(r.w[tokens[i]] / r.w.sum())
        if probs is not None:
            probs[i] = r.w / r.w.sum()
    return dict(tokens=tokens, logp=logp, **({} if probs is None else {"probs": probs}))


def _exact_accept(c, s):
    h = {n: _host(s[n]) for n in ("logits", "u", "tokens", "parent", "counts", "starts")}
    settings = {k: _host(v) for k, v in s["settings"].items()}
    u, D, k = h["u"].astype(np.float64), c["depth"], c["children"]
    path, length = np.full((c["n"], D + 1), -1, np.int32), np.zeros(c["n"], np.int32)
    bonus = np.zeros(c["n"], np.int32)
    for b in range(c["n"]):
        at, d = 0, 0
        path[b, 0] = 0
        while True:
            r = _Row(h["logits"][h["starts"][b] + at], settings, b)
            kids = [j for j in range(1, h["counts"][b]) if h["parent"][b, j] == at][:k] if d < D else []
            nxt = None
            for i, j in enumerate(kids):
                t = h["tokens"][b, j]
                if u[b, d, i] * r.w.sum() < r.w[t]:
                    nxt = j
                    break
                r.w[t] = 0.0
            if nxt is None:
                length[b], bonus[b] = d, r.draw(u[b, d, k])
                break
            at, d = nxt, d + 1
            path[b, d] = at
    return {"path": path, "accept_len": length, "bonus": bonus}


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    return {"linear": _exact_linear, "quantize": _exact_quantize, "sample": _exact_sample,
            "accept": _exact_accept}[c["kind"]](c, s)
