"""Several questions about one image, decoded from one pool of cache pages.

    python examples/shared_image.py [--questions 4] [--tokens 24] [--dtype bf16]

A small decoder of random weights (grouped heads, one layer with a window) whose cache is a
Pages pool, driven as a serving program drives its own model:

1. the prompt, text and a 24 x 24 image, runs once: positions on three axes, K and V into
   the pages, attention of the prompt's rows;
2. every question is a fork of it: the image's pages are shared, not copied;
3. the questions' texts, of different lengths, run as one ragged batch;
4. the answers are decoded twice, on forks of their own: token by token, and with a tree of
   drafts a pass that is verified at once and of which the accepted path stays. The drafts
   here are the first decode's tokens, wrong now and then, with random siblings: what counts
   is that both decodes give the same tokens while the second takes fewer passes.
"""
from __future__ import annotations

import argparse
import ctypes
import os
import random
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2505_14260_gb300 import msd  # noqa: E402

HIDDEN, LAYERS, HEADS, KV_HEADS, HEAD_DIM, FFN, VOCAB = 512, 3, 8, 2, 64, 1024, 1000
GRID = 24                     # the image's tokens: GRID x GRID
WINDOW, SINKS = 200, 4        # of the middle layer


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def batch(seqs, counts):
    starts = [0]
    for c in counts:
        starts.append(starts[-1] + c)
    return msd.Batch(i32(seqs), i32(starts), starts[-1])


def linear(x, w):
    """x @ w.T in fp32: the library's GEMM for bf16 weights."""
    if w.dtype == torch.float32:
        return x.float() @ w.T
    x, y = x.to(w.dtype).contiguous(), torch.empty(x.shape[0], w.shape[0], device="cuda")
    st = msd.lib().msd_linear_noalloc(x.data_ptr(), x.stride(0), x.shape[0], x.shape[1], w.data_ptr(), w.shape[0],
                                      y.data_ptr(), y.stride(0), 0,
                                      ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    if st != msd.MSD_OK:
        raise msd.MsdError(st, "msd_linear_noalloc", "")
    return y


def norm(x):
    return x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6)


class Decoder:
    def __init__(self, pages, dtype, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        mat = lambda o, i: (torch.randn(o, i, generator=g, device="cuda") * i ** -0.5).to(dtype)  # noqa: E731
        self.pages, self.dtype = pages, dtype
        self.embed = torch.randn(VOCAB, HIDDEN, generator=g, device="cuda")
        width = (HEADS + 2 * KV_HEADS) * HEAD_DIM
        self.layers = [dict(qkv=mat(width, HIDDEN), o=mat(HIDDEN, HEADS * HEAD_DIM), up=mat(2 * FFN, HIDDEN),
                            down=mat(HIDDEN, FFN)) for _ in range(LAYERS)]
        self.head = mat(VOCAB, HIDDEN)

    def forward(self, b, x, pos, tree=None):
        """Rows x of the batch (their slots reserved) through the layers; the logits."""
        for i, w in enumerate(self.layers):
            q, k, v = linear(norm(x), w["qkv"]).split([HEADS * HEAD_DIM, KV_HEADS * HEAD_DIM, KV_HEADS * HEAD_DIM], 1)
            turned = torch.empty(b.rows, HEADS, HEAD_DIM, device="cuda", dtype=self.dtype)
            self.pages.rope_append(i, b, q, k, v, pos, turned)
            seen = torch.empty_like(turned)
            narrow = dict(window=WINDOW, sinks=SINKS) if i == 1 else {}
            self.pages.attention(i, b, turned, seen, tree=tree, **narrow)
            x = x + linear(seen.view(b.rows, -1), w["o"])
            gate, up = linear(norm(x), w["up"]).chunk(2, 1)
            x = x + linear(torch.nn.functional.silu(gate) * up, w["down"])
        return linear(norm(x), self.head)


def draft_tree(n, want, nodes, rng, root):
    """Tokens and a msd.Tree for n sequences: a chain of the wanted tokens, some of them wrong,
    and random siblings. Depths and ancestor masks follow from the parents."""
    tree = msd.Tree(n, nodes)
    tokens, depths, masks, parents = [], [], [], []
    for s in range(n):
        parent, depth, mask, toks, tip = [-1], [0], [1], [root[s]], 0
        for i in range(1, nodes):
            chain = i % 2 == 1 and depth[tip] < len(want[s])
            p = tip if chain else rng.randrange(i)
            right = chain and rng.random() < 0.85
            toks.append(want[s][depth[p]] if right else rng.randrange(VOCAB))
            parent.append(p)
            depth.append(depth[p] + 1)
            mask.append(mask[p] | 1 << i)
            tip = i if chain else tip
        tokens.append(toks)
        parents.append(parent)
        depths += depth
        masks += [m - (1 << 64) if m >> 63 else m for m in mask]
    tree.depth.copy_(i32(depths))
    tree.mask.copy_(torch.tensor(masks))
    return tree, tokens, parents


def run(questions=4, tokens=24, dtype="bf16", nodes=16, seed=0, say=print):
    rng = random.Random(seed)
    page, seqs = 16, 1 + 3 * questions
    pages = msd.Pages(dtype=dtype, layers=LAYERS, heads=HEADS, kv_heads=KV_HEADS, head_dim=HEAD_DIM, page_size=page,
                      n_pages=64 + questions * 24, max_seqs=seqs, max_pages=64, rot_sections=(8, 12, 12))
    model = Decoder(pages, pages.dtype, seed)

    # 1. the shared prompt: 8 text tokens, the image, 5 text tokens
    rows, image = 8 + GRID * GRID + 5, GRID * GRID
    b = batch([0], [rows])
    pages.reserve(b)
    pos, after = torch.empty(3, rows, dtype=torch.int32, device="cuda"), i32([0])
    pages.positions(b, i32([0, 1]), i32([[8, 1, GRID, GRID, 1]]), pos, after)
    text = model.embed[torch.tensor([rng.randrange(VOCAB) for _ in range(13)], device="cuda")]
    pixels = torch.randn(image, HIDDEN, generator=torch.Generator(device="cuda").manual_seed(seed + 1), device="cuda")
    model.forward(b, torch.cat([text[:8], pixels, text[8:]]), pos)
    shared = int((pages.refs > 0).sum())

    # 2., 3. a fork for each question, the questions' texts in one batch
    asked = list(range(1, 1 + questions))
    pages.fork(i32([0] * questions), i32(asked))
    texts = [[rng.randrange(VOCAB) for _ in range(3 + 5 * k)] for k in range(questions)]
    b = batch(asked, [len(t) for t in texts])
    pages.reserve(b)
    pos = torch.empty(3, b.rows, dtype=torch.int32, device="cuda")
    place = i32([0] * questions)                  # the next token's position of each question
    pages.positions(b, None, None, pos, place, first=after.expand(questions).contiguous())
    logits = model.forward(b, model.embed[torch.tensor(sum(texts, []), device="cuda")], pos)
    last = b.row_start[1:].long() - 1
    first = logits[last].argmax(1)
    say(f"{questions} questions: {int((pages.refs > 0).sum())} pages, {shared} of them the prompt's; "
        f"without sharing {sum(-(-int(n) // page) for n in pages.lens[1:1 + questions])}")

    # 4. token by token
    plain = [questions + s for s in asked]
    pages.fork(i32(asked), i32(plain))
    got, token, at = [[int(t)] for t in first], first, place.clone()
    b = batch(plain, [1] * questions)
    for _ in range(tokens):
        pages.reserve(b)
        token = model.forward(b, model.embed[token], at[None]).argmax(1)
        at += 1
        for s, t in enumerate(token.tolist()):
            got[s].append(t)
    pages.free(i32(plain))

    # with a tree a pass
    drafted = [2 * questions + s for s in asked]
    pages.fork(i32(asked), i32(drafted))
    fast, at, passes = [[int(t)] for t in first], place.clone(), 0
    while min(len(f) for f in fast) <= tokens:
        b = batch(drafted, [nodes] * questions)
        pages.reserve(b)
        want = [got[s][len(fast[s]):] for s in range(questions)]
        tree, toks, parents = draft_tree(questions, want, nodes, rng, [f[-1] for f in fast])
        pos = (at[:, None] + tree.depth.view(questions, nodes)).view(1, -1)
        best = model.forward(b, model.embed[torch.tensor(sum(toks, []), device="cuda")], pos, tree).argmax(1)
        best, keep = best.view(questions, nodes).tolist(), []
        for s in range(questions):                # follow the child that the target agrees with
            path, more = [0], True
            while more:
                node = path[-1]
                more = next((i for i in range(1, nodes) if parents[s][i] == node and toks[s][i] == best[s][node]), None)
                if more:
                    path.append(more)
            keep.append(path)
            fast[s] += [best[s][n] for n in path]
        n_keep = i32([len(k) for k in keep])
        pages.compact(b, i32([k + [-1] * (nodes - len(k)) for k in keep]), n_keep)
        at += n_keep
        passes += 1
    same = [f[: tokens + 1] == g for f, g in zip(fast, got)]
    pages.free(i32(drafted + asked + [0]))
    torch.cuda.synchronize()
    say(f"{tokens} tokens each: {tokens} passes of one token, {passes} of a tree of {nodes}; "
        f"same tokens: {sum(same)} of {questions}; pages left in use: {int((pages.refs > 0).sum())}")
    return got, fast, passes, pages


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--questions", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=24)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = ap.parse_args()
    run(a.questions, a.tokens, a.dtype)


if __name__ == "__main__":
    main()
