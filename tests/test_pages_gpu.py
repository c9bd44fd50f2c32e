"""The pool's page operations against a model of them on the host, rotary positions and the
rotation with K/V into the pages against 64-bit forms, and what they refuse."""
import math
import random

import pytest
import torch

from paper_2505_14260_gb300 import build, msd
from tests.pages_support import batch, i32, pool, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


class Model:
    """What the pool should hold: page ids, counts and a token's value per slot."""

    def __init__(self, n_pages, max_seqs, page):
        self.refs, self.page = [0] * n_pages, page
        self.pages = [[] for _ in range(max_seqs)]
        self.toks = [[] for _ in range(max_seqs)]

    def take(self, n):
        free = [i for i, r in enumerate(self.refs) if r == 0][:n]
        if len(free) < n:
            raise MemoryError
        return free

    def reserve(self, seqs, counts):
        need = [-(-(len(self.toks[s]) + c) // self.page) - len(self.pages[s]) for s, c in zip(seqs, counts)]
        ids = self.take(sum(need))
        for s, c, n in zip(seqs, counts, need):
            for _ in range(n):
                self.pages[s].append(ids.pop(0))
                self.refs[self.pages[s][-1]] = 1
            self.toks[s] += [None] * c

    def fork(self, src, dst, deep):
        own = [len(self.pages[s]) if deep else int(len(self.toks[s]) % self.page > 0) for s in src]
        ids = self.take(sum(own))
        for s, d, n in zip(src, dst, own):
            keep = len(self.pages[s]) - n
            self.pages[d] = self.pages[s][:keep] + [ids.pop(0) for _ in range(n)]
            for p in self.pages[d]:
                self.refs[p] += 1
            self.toks[d] = list(self.toks[s])

    def compact(self, seqs, counts, keep):
        plans, need = [], 0
        for s, c, k in zip(seqs, counts, keep):
            base = len(self.toks[s]) - c
            still = next((j for j, x in enumerate(k) if x != j), len(k))
            first, now = (base + still) // self.page, -(-(base + len(k)) // self.page)
            shared = [x for x in range(first, now) if self.refs[self.pages[s][x]] > 1]
            plans.append((base, now, shared))
            need += len(shared)
        ids, gone = self.take(need), []
        for (s, k), (base, now, shared) in zip(zip(seqs, keep), plans):
            toks = self.toks[s]
            self.toks[s] = toks[:base] + [toks[base + j] for j in k]
            gone += self.pages[s][now:] + [self.pages[s][x] for x in shared]
            self.pages[s] = self.pages[s][:now]
            for x in shared:
                self.pages[s][x] = ids.pop(0)
                self.refs[self.pages[s][x]] = 1
        for p in gone:
            self.refs[p] -= 1

    def free(self, seqs):
        for s in seqs:
            for p in self.pages[s]:
                self.refs[p] -= 1
            self.pages[s], self.toks[s] = [], []


def fill(p, m, counter):
    """New tokens (None) get values of their own, in the pool and in the model."""
    for s, toks in enumerate(m.toks):
        for t, x in enumerate(toks):
            if x is None:
                toks[t] = next(counter)
                slot = p.kv[:, m.pages[s][t // m.page], :, :, t % m.page]
                slot.copy_(value(p, toks[t]))


def value(p, x):
    c = p.cfg
    base = torch.arange(c.n_layers * 2 * c.n_kv_heads, device="cuda").view(c.n_layers, 2, c.n_kv_heads, 1)
    at = torch.arange(c.head_dim, device="cuda")
    return ((x * 7 + base * 3 + at) % 199).to(p.dtype)


def compare(p, m):
    torch.cuda.synchronize()
    assert p.refs.tolist() == m.refs
    assert p.lens.tolist() == [len(t) for t in m.toks]
    for s, ids in enumerate(m.pages):
        assert p.table[s].tolist() == ids + [-1] * (p.cfg.max_pages - len(ids)), s
        for t, x in enumerate(m.toks[s]):
            assert torch.equal(p.kv[:, ids[t // m.page], :, :, t % m.page], value(p, x).expand(-1, -1, -1, -1)), (s, t)


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("dtype,head_dim,page,kv_heads", [("bf16", 64, 16, 1), ("f32", 128, 32, 2), ("bf16", 128, 16, 3)])
def test_random_programs(seed, dtype, head_dim, page, kv_heads):
    """Sequences of operations on small pools, some of which run out of pages."""
    r = random.Random(seed)
    n_pages, max_seqs = r.choice([13, 40, 70]), 7
    p = msd.Pages(dtype=dtype, layers=2, heads=kv_heads, kv_heads=kv_heads, head_dim=head_dim, page_size=page,
                  n_pages=n_pages, max_seqs=max_seqs, max_pages=9)
    p.kv.zero_()
    m, counter, full = Model(n_pages, max_seqs, page), iter(range(10 ** 6)), 0
    for _ in range(25):
        op = r.choice(["reserve", "reserve", "fork", "compact", "compact", "free"])
        seqs = r.sample(range(max_seqs), r.randint(1, 4))
        try:
            if op == "reserve":
                counts = [min(r.choice([0, 1, 5, page, 40]), 9 * page - len(m.toks[s])) for s in seqs]
                p.reserve(batch(seqs, counts))
                m.reserve(seqs, counts)
            elif op == "fork":
                dst = [s for s in range(max_seqs) if not m.toks[s]][:3]
                src = [s for s in range(max_seqs) if s not in dst]
                if not dst or not src:
                    continue
                src, deep = [r.choice(src) for _ in dst], r.random() < 0.3
                p.fork(i32(src), i32(dst), deep=deep)
                m.fork(src, dst, deep)
            elif op == "compact":
                counts = [r.randint(0, len(m.toks[s])) for s in seqs]
                keep = [sorted(r.sample(range(c), r.randint(0, c))) for c in counts]
                if r.random() < 0.3:
                    keep = [list(range(len(k))) for k in keep]
                width = max(1, max(len(k) for k in keep))
                rows = i32([k + [-1] * (width - len(k)) for k in keep])
                ident = all(k == list(range(len(k))) for k in keep) and r.random() < 0.5
                p.compact(batch(seqs, counts), None if ident else rows, i32([len(k) for k in keep]))
                m.compact(seqs, counts, keep)
            else:
                p.free(i32(seqs))
                m.free(seqs)
        except MemoryError:                        # the pool reports it with its next call
            torch.cuda.synchronize()
            full += 1
            with pytest.raises(msd.MsdError) as e:
                p.free(i32([0]))
            assert e.value.status == msd.MSD_ERR_CAPACITY
        fill(p, m, counter)
        compare(p, m)


def test_a_large_pool_and_a_long_list():
    """More pages than one pass of the bitmap scan takes, more sequences than a CTA has threads."""
    n, page = 1500, 16
    p = msd.Pages(dtype="bf16", layers=1, heads=1, kv_heads=1, head_dim=64, page_size=page, n_pages=300000,
                  max_seqs=n + 1, max_pages=200000)
    counts = [2_100_000] + [(i * 29) % 70 for i in range(n - 1)]
    order = list(range(n - 1, -1, -1))
    b = batch(order, counts)
    p.reserve(b)
    need = [-(-c // page) for c in counts]
    at = 0
    for s, k in zip(order, need):
        assert p.table[s, :k].tolist() == list(range(at, at + k))
        at += k
    assert int(p.refs.sum()) == at and p.lens[order[0]] == counts[0]
    p.fork(i32([order[0]]), i32([n]))
    torch.cuda.synchronize()
    assert torch.equal(p.table[n], p.table[order[0]]) and int(p.refs.max()) == 2
    p.free(i32(order))
    torch.cuda.synchronize()
    assert p.refs.nonzero()[:, 0].tolist() == list(range(need[0])) and int(p.refs.max()) == 1
    p.free(i32([n, n]))
    torch.cuda.synchronize()
    assert int(p.refs.abs().sum()) == 0 and (p.table == -1).all()
    del p
    torch.cuda.empty_cache()


def test_calls_that_cannot_be_carried_out_change_nothing():
    p = pool([20, 40, 33], extra_seqs=3, spare=3)
    before = [t.clone() for t in (p.table, p.lens, p.refs, p.kv.nan_to_num())]

    def reported(status, call):
        call()
        torch.cuda.synchronize()
        with pytest.raises(msd.MsdError) as e:
            p.free(i32([5]))
        assert e.value.status == status
        p.free(i32([5]))                                          # the next call runs
        torch.cuda.synchronize()
        for a, b in zip(before, (p.table, p.lens, p.refs, p.kv.nan_to_num())):
            assert torch.equal(a, b)
    D, C = msd.MSD_ERR_DEVICE, msd.MSD_ERR_CAPACITY
    room = p.cfg.max_pages * 16
    reported(D, lambda: p.reserve(batch([0, 9], [1, 1])))
    reported(D, lambda: p.reserve(batch([0, 0], [1, 1])))
    reported(D, lambda: p.reserve(batch([0, 1], [1, room])))
    reported(D, lambda: p.reserve(msd.Batch(i32([0, 1]), i32([0, 3, 1]), 1)))
    reported(C, lambda: p.reserve(batch([0, 1, 4], [1, 1, 16 * 4])))
    reported(D, lambda: p.fork(i32([0]), i32([1])))               # in use
    reported(D, lambda: p.fork(i32([0, 0]), i32([3, 3])))
    reported(D, lambda: p.fork(i32([0, 3]), i32([3, 4])))         # copies what is being made
    reported(D, lambda: p.fork(i32([0]), i32([-1])))
    reported(C, lambda: p.fork(i32([0, 1, 2]), i32([3, 4, 5]), deep=True))
    for keep, n_keep in [([[0, 0]], [2]), ([[1, 0]], [2]), ([[0, 5]], [2]), ([[-1, 1]], [2]), ([[0, 1]], [3]), ([[0, 1]], [-1])]:
        reported(D, lambda: p.compact(batch([1], [5]), i32(keep), i32(n_keep)))
    reported(D, lambda: p.compact(batch([0, 0], [5, 5]), None, i32([1, 1])))
    reported(D, lambda: p.compact(batch([0], [21]), None, i32([1])))
    reported(D, lambda: p.free(i32([77])))


def test_restore_counts_shared_pages_and_reports_bad_tables():
    p = pool([64, 40], extra_seqs=1)
    p.table[2, :2] = p.table[0, :2]
    p.lens[2] = 32
    p.restore()
    torch.cuda.synchronize()
    assert p.refs[p.table[0, :4].long()].tolist() == [2, 2, 1, 1] and int(p.refs.sum()) == 9
    assert (p.table[2, 2:] == -1).all()
    p.table[2, 1] = p.cfg.n_pages
    p.restore()
    torch.cuda.synchronize()
    with pytest.raises(msd.MsdError):
        p.restore()
    p.table[2, 1] = p.table[0, 1]
    p.lens[2] = 30                                                # its second page is half full, and sequence 0's
    p.restore()
    torch.cuda.synchronize()
    with pytest.raises(msd.MsdError):
        p.restore()
    p.lens[2] = -4
    p.restore()
    torch.cuda.synchronize()
    with pytest.raises(msd.MsdError):
        p.restore()
    assert int(p.lens[2]) == 0


# ---------------------------------------------------------------------------
# Positions
# ---------------------------------------------------------------------------
def positions(rows, spans, first):
    out, p, r, at = [], first, 0, {s[0]: s for s in spans}
    while r < rows:
        if r in at:
            _, t, h, w, step = at[r]
            out += [(p + a * step, p + b, p + c) for a in range(t) for b in range(h) for c in range(w)]
            p, r = p + max((t - 1) * step + 1, h, w), r + t * h * w
        else:
            out.append((p, p, p))
            p, r = p + 1, r + 1
    return out, p


@pytest.mark.parametrize("many", [False, True])
def test_positions(many):
    p = pool([1] * 6)
    r = random.Random(many)
    rows = [1, 700, 33, 0, 5000, 12]
    spans = [[], [(3, 1, 24, 24, 1), (600, 4, 2, 3, 7)], [(0, 3, 2, 2, 5), (12, 1, 1, 1, 1), (13, 2, 5, 2, 9)], [], [], [(0, 2, 2, 3, 1)]]
    at = 0
    while many and at < 4900:                                     # more spans than one tile of them
        t, h, w = r.randint(1, 2), r.randint(1, 3), r.randint(1, 3)
        spans[4].append((at, t, h, w, r.randint(1, 4)))
        at += t * h * w + r.randint(0, 3)
    first = [0, 5, -3, 9, 1 << 20, 7]
    T = sum(rows)
    pos, nxt = torch.full((3, T + 5), 99, dtype=torch.int32, device="cuda"), i32([0] * 6)
    flat = [list(s) for ss in spans for s in ss]
    b = batch(list(range(6)), rows)
    p.positions(b, starts([len(s) for s in spans]), i32(flat), pos, nxt, first=i32(first))
    ref = [positions(n, s, f) for n, s, f in zip(rows, spans, first)]
    assert pos[:, :T].T.tolist() == [list(x) for rr, _ in ref for x in rr]
    assert nxt.tolist() == [x for _, x in ref] and (pos[:, T:] == 99).all()
    p.positions(b, None, None, pos)
    assert pos[:, :T].T.tolist() == [[x] * 3 for n in rows for x in range(n)]


def test_lengths_past_the_table_are_reported_and_bound_nothing():
    p = pool([20, 40], extra_seqs=1)
    for call in (lambda: p.free(i32([0])), lambda: p.reserve(batch([0], [1])), lambda: p.fork(i32([0]), i32([2])),
                 lambda: p.compact(batch([0], [1]), None, i32([1]))):
        for bad in (-7, p.cfg.max_pages * 16 + 1, 2 ** 31 - 1):
            p.lens[0] = bad
            table, refs = p.table.clone(), p.refs.clone()
            call()
            torch.cuda.synchronize()
            with pytest.raises(msd.MsdError) as e:
                p.free(i32([2]))
            assert e.value.status == msd.MSD_ERR_DEVICE
            assert torch.equal(p.table, table) and torch.equal(p.refs, refs)


def test_spans_out_of_place_are_reported():
    p = pool([1])
    pos, b = torch.zeros(3, 30, dtype=torch.int32, device="cuda"), batch([0], [30])
    for spans in [[[25, 1, 2, 3, 1]], [[-1, 1, 2, 2, 1]], [[0, 0, 2, 2, 1]], [[0, 1, 2, 2, 0]], [[0, 1, 2, 3, 1], [5, 1, 1, 1, 1]],
                  [[0, 1 << 30, 1 << 30, 4, 1]], [[9, 1, 1, 1, 1], [3, 1, 1, 1, 1]], None]:
        p.positions(b, i32([0, 2]) if spans is None else starts([len(spans)]), i32(spans or [[0, 1, 1, 1, 1]]), pos)
        torch.cuda.synchronize()
        with pytest.raises(msd.MsdError) as e:
            p.restore()
        assert e.value.status == msd.MSD_ERR_DEVICE


# ---------------------------------------------------------------------------
# Rotation and append
# ---------------------------------------------------------------------------
def rotate(x, pos, rot, sections, turns, base):
    """x [T, heads, hd] in 64 bits; pos [3, T] whole numbers. Angles are reduced mod 2 pi from
    exact fractions of a turn (Python's whole numbers)."""
    half = rot // 2
    x = x.clone()
    for i in range(half):
        if turns:
            axis = 1 if i % 3 == 1 and i < 3 * sections[1] else 2 if i % 3 == 2 and i < 3 * sections[2] else 0
        else:
            axis = int(i >= sections[0]) + int(i >= sections[0] + sections[1])
        angle = pos[axis].double() * float(base) ** (-2.0 * i / rot)
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        u, w = x[:, :, i].clone(), x[:, :, i + half].clone()
        x[:, :, i], x[:, :, i + half] = u * c - w * s, w * c + u * s
    return x


@pytest.mark.parametrize("dtype,src", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("heads,kv_heads,hd,rot,sections,turns", [
    (4, 2, 64, 64, (8, 12, 12), False), (4, 4, 128, 128, (24, 20, 20), True), (7, 1, 128, 64, (16, 8, 8), False),
    (40, 40, 128, 128, (64, 0, 0), False), (2, 1, 64, 40, (10, 5, 5), True), (2, 2, 64, 6, (1, 1, 1), True),
    (3, 1, 64, 0, (0, 0, 0), False)])
def test_rope_append(dtype, src, heads, kv_heads, hd, rot, sections, turns):
    """Rows of ragged sequences, at positions up to 2^24 (an fp64 angle there is off by at most
    2^24 2^-53 2 pi = 1e-8), as parts of wide rows, into the second layer; nothing else of
    the pool changes."""
    lens, counts = [70, 16, 33, 5], [9, 16, 0, 1]
    p = pool(lens, dtype=dtype, layers=2, heads=heads, kv_heads=kv_heads, head_dim=hd, rot_dim=rot, rot_sections=sections,
             rot_interleaved=turns, stale=3.0, extra_seqs=1)
    T, g = sum(counts), torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(T, (heads + 2 * kv_heads) * hd + 64, generator=g, device="cuda")
    x = x if src == "f32" else x.bfloat16()
    q, k, v = x[:, 64:].split([heads * hd, kv_heads * hd, kv_heads * hd], 1)
    pos = torch.randint(-100, 1 << 24, (3, T), generator=g, device="cuda", dtype=torch.int32)
    pos[:, 0] = 0
    out = torch.zeros(T, heads, hd, device="cuda", dtype=p.dtype)
    before = p.kv.clone()
    seqs = [0, 1, 2, 3]
    p.rope_append(1, batch(seqs, counts), q, k, v, pos, out)
    full = x[:, 64:].double().view(T, heads + 2 * kv_heads, hd)
    ref = rotate(full[:, :heads + kv_heads], pos, rot, sections, turns, 10000.0)
    # an angle is off by 2^-25 of half a turn (its 32 bits as a float) and the 64-bit one by 1e-8; sine and
    # cosine, two products and a sum: 5 roundings of |u| + |w|; then the cache's type
    mag = 2 * full.abs().amax(-1, keepdim=True)
    def close(a, b, m):
        tol = m * (math.pi * 2.0 ** -25 + 2e-8 + 5 * 2.0 ** -24) + (b.abs() * 2.0 ** -8 if dtype == "bf16" else 0)
        assert bool(((a.double() - b).abs() <= tol).all())
    close(out, ref[:, :heads], mag[:, :heads])
    at = 0
    want = before.double()
    for s, n in zip(seqs, counts):
        for t in range(n):
            slot = lens[s] - n + t
            page = int(p.table[s, slot // 16])
            close(p.kv[1, page, 0, :, slot % 16], ref[at, heads:], mag[at, heads:heads + kv_heads])
            assert torch.equal(p.kv[1, page, 1, :, slot % 16].double(), full[at, heads + kv_heads:].to(p.dtype).double())
            want[1, page, :, :, slot % 16] = p.kv[1, page, :, :, slot % 16].double()
            at += 1
    assert torch.equal(p.kv.double(), want)
    one = torch.zeros_like(out)                                   # one position for all axes
    p.rope_append(1, batch(seqs, counts), q, k, v, pos[:1].contiguous(), one)
    close(one, rotate(full[:, :heads], pos[:1].expand(3, -1), rot, sections, turns, 10000.0), mag[:, :heads])


def test_positions_past_what_floats_hold():
    """Positions near 2^31: a rotation by p equals rotations by p - d and d in turn."""
    p = pool([2], dtype="f32", heads=1, kv_heads=1, rot_sections=(32, 0, 0))
    x = torch.randn(1, 64, device="cuda")
    kv = torch.zeros(1, 64, device="cuda")
    b, big, d = batch([0], [1]), 2147483000, 123457

    def turn(y, at):
        out = torch.zeros(1, 1, 64, device="cuda")
        p.rope_append(0, b, y, kv, kv, i32([[at]]), out)
        return out[0]
    once, twice = turn(x, big), turn(turn(x, big - d), d)
    assert float((once - twice).abs().max()) <= 3 * 2 * float(x.abs().max()) * (math.pi * 2.0 ** -25 + 5 * 2.0 ** -24)
    back = turn(turn(x, big), -big)
    assert float((back - x).abs().max()) <= 3 * 2 * float(x.abs().max()) * (math.pi * 2.0 ** -25 + 5 * 2.0 ** -24)


def test_rows_without_a_slot_are_skipped_and_reported():
    p = pool([20, 3], extra_seqs=1, stale=0.0)
    x, out = torch.randn(6, 4 * 64, device="cuda").bfloat16(), torch.zeros(6, 4, 64, device="cuda", dtype=torch.bfloat16)
    before = p.kv.clone()
    for b in [batch([1, 5], [1, 5]), batch([2, 1], [5, 1])]:
        p.rope_append(0, b, x, x[:, :128], x[:, 128:], torch.zeros(1, 6, dtype=torch.int32, device="cuda"), out)
        torch.cuda.synchronize()
        with pytest.raises(msd.MsdError):
            p.restore()
    changed = (p.kv != before).flatten(2).any(-1)[0]
    assert set(changed.nonzero()[:, 0].tolist()) <= set(p.table[1, :1].tolist())


def test_refusals():
    p = pool([20], dtype="bf16")
    b = batch([0], [2])
    x, out = torch.randn(2, 4 * 64, device="cuda"), torch.zeros(2, 4, 64, device="cuda", dtype=torch.bfloat16)
    pos = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    good = [p.ptr, 0, b.c(), x.data_ptr(), 256, x.data_ptr(), 256, x.data_ptr(), 256, msd.MSD_F32, pos.data_ptr(), 0,
            out.data_ptr(), 256, msd._stream(None)]
    L = msd.lib()
    assert L.msd_rope_append(*good) == msd.MSD_OK
    for at, v in [(1, -1), (1, 1), (2, None), (3, None), (3, x.data_ptr() + 4), (4, 255), (4, 258), (6, 64), (8, 127), (9, 5),
                  (10, None), (11, 1), (12, None), (12, out.data_ptr() + 2), (13, 250), (13, 260)]:
        args = list(good)
        args[at] = v
        assert L.msd_rope_append(*args) == msd.MSD_ERR_INVALID, (at, v)
    with pytest.raises(ValueError):
        p.rope_append(0, b, x, x[:, :128].bfloat16(), x[:, :128], pos, out)
    with pytest.raises(ValueError):
        p.rope_append(0, b, x[:1], x[:, :128], x[:, :128], pos, out)
    with pytest.raises(ValueError):
        p.fork(i32([0]), torch.tensor([1], device="cuda"))
    S = msd._stream(None)
    assert L.msd_pages_fork(p.ptr, 0, p.lens.data_ptr(), p.lens.data_ptr(), 0, S) == msd.MSD_ERR_INVALID
    assert L.msd_pages_free(p.ptr, 9, p.lens.data_ptr(), S) == msd.MSD_ERR_INVALID
    assert L.msd_pages_free(p.ptr, 1, None, S) == msd.MSD_ERR_INVALID
    assert L.msd_pages_compact(p.ptr, b.c(), None, 0, None, S) == msd.MSD_ERR_INVALID
    assert L.msd_rope_positions(p.ptr, b.c(), None, None, 0, None, pos.data_ptr(), 1, None, S) == msd.MSD_ERR_INVALID
    assert L.msd_pages_destroy(None) == msd.MSD_OK and L.msd_pages_last_error(None) == b"null pool"
