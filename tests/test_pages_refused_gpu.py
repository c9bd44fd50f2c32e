"""What the paged cache does when a call cannot be carried out, is given lists or tables that are wrong, or
meets sizes at its limits: nothing that other sequences hold changes, and the caller is told."""
import pytest
import torch

from paper_2505_14260_gb300 import build, msd
from tests.pages_support import attend, batch, bounds, i32, pool, random_tree, tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def state(p):
    return [t.clone() for t in (p.table, p.lens, p.refs, p.kv.nan_to_num())]


def same(p, before):
    return all(torch.equal(a, b) for a, b in zip(before, (p.table, p.lens, p.refs, p.kv.nan_to_num())))


def reported(p, status):
    """The next call reports an earlier one's error and does nothing."""
    torch.cuda.synchronize()
    with pytest.raises(msd.MsdError) as e:
        p.restore()
    assert e.value.status == status


# ---------------------------------------------------------------------------
# Calls queued behind one that could not be carried out
# ---------------------------------------------------------------------------
def step(p, seqs, rows):
    """A pass of a model over new rows, as it is queued: room, rotation and K/V, attention, then the first two
    rows of each stay. Returns what it writes beside the pool."""
    g = torch.Generator(device="cuda").manual_seed(5)
    n = len(seqs) * rows
    x = torch.randn(n, 8 * 64, generator=g, device="cuda").to(p.dtype)
    q, out = (torch.full((n, 4, 64), 7.0, device="cuda", dtype=p.dtype) for _ in range(2))
    lse, pos = torch.full((n, 4), 7.0, device="cuda"), i32([list(range(n))])
    b, n_keep = batch(seqs, [rows] * len(seqs)), i32([2] * len(seqs))

    def run():
        p.reserve(b)
        p.rope_append(0, b, x[:, :256], x[:, 256:384], x[:, 384:], pos, q)
        p.attention(0, b, q, out, lse=lse)
        p.compact(b, None, n_keep)
    return run, (q, out, lse)


def shared_pool(dtype="bf16"):
    """Sequences 0 and 1 share four full pages, 2 holds six of its own; one page is free."""
    p = pool([64, 96], dtype=dtype, extra_seqs=3, spare=1, extra_pages=8)
    p.fork(i32([0]), i32([2]))
    torch.cuda.synchronize()
    return p


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("graph", [False, True])
def test_calls_behind_a_failed_reserve_change_nothing(dtype, graph):
    """Too few pages, then the rest of the pass before the host can know of it: nothing changes, not even the
    outputs; after the error has been reported and pages are free, the same calls run."""
    p = shared_pool(dtype)
    run, outs = step(p, [0, 2], 20)                  # four pages; one is free
    one, src, dst = i32([1]), i32([0]), i32([3])
    before = state(p)
    if graph:
        recorded = torch.cuda.CUDAGraph()
        with torch.cuda.graph(recorded):
            run()
        for _ in range(3):
            recorded.replay()
    else:
        torch.cuda._sleep(40_000_000)                # what follows is queued before any of it runs
        run()
        p.free(one)
        p.fork(src, dst)
    torch.cuda.synchronize()
    assert same(p, before)
    assert all((t == 7).all() for t in outs)
    reported(p, msd.MSD_ERR_CAPACITY)
    p.free(one)
    recorded.replay() if graph else run()
    torch.cuda.synchronize()
    assert p.lens.tolist() == [66, 0, 66, 0, 0] and not any((t == 7).all() for t in outs)
    assert torch.equal(p.table[0, :4], p.table[2, :4]) and p.table[0, 4] != p.table[2, 4]
    p.restore()                                      # nothing is pending


@pytest.mark.parametrize("fail", ["fork", "compact", "free"])
def test_calls_behind_other_failed_operations_change_nothing(fail):
    p = shared_pool()
    p.free(i32([1]))
    run, outs = step(p, [0, 2], 20)
    zero, two, pair, five = i32([0]), i32([2]), i32([0, 77]), batch([0], [5])
    keep = i32([[1, 0]])
    before = state(p)
    torch.cuda._sleep(40_000_000)                    # what follows is queued before any of it runs
    if fail == "fork":
        p.fork(zero, two)                            # in use
    elif fail == "compact":
        p.compact(five, keep, two)
    else:
        p.free(pair)
    run()
    torch.cuda.synchronize()
    assert same(p, before) and all((t == 7).all() for t in outs)
    reported(p, msd.MSD_ERR_DEVICE)
    run()
    torch.cuda.synchronize()
    assert p.lens.tolist() == [66, 0, 66, 0, 0]


def test_an_error_that_the_host_has_not_seen_is_not_cleared_with_an_earlier_one():
    """The host is told of an attention's error while a reserve that will fail is still queued: what it queues
    then waits for the reserve's own error to be reported."""
    p = shared_pool()
    x, one, told = torch.zeros(1, 4, 64, device="cuda", dtype=p.dtype), batch([4], [1]), torch.cuda.Event()
    b, n_keep = batch([0, 2], [20, 20]), i32([2, 2])
    before = state(p)
    torch.cuda._sleep(40_000_000)
    p.attention(0, one, x, x)                        # a row of a sequence without tokens
    told.record()
    torch.cuda._sleep(100_000_000)
    p.reserve(b)
    told.synchronize()
    with pytest.raises(msd.MsdError) as e:
        p.restore()
    assert e.value.status == msd.MSD_ERR_DEVICE
    p.compact(b, None, n_keep)
    torch.cuda.synchronize()
    assert same(p, before)
    reported(p, msd.MSD_ERR_CAPACITY)
    p.free(one.seqs)


@pytest.mark.parametrize("bad", [False, True])
def test_a_refusal_that_another_error_hides_is_reported_too(bad):
    """An attention's error and a reserve's (too few pages, or a bad list: the attention's own kind) before the host
    looks: the first report is the attention's, and nothing runs until the second."""
    p = shared_pool()
    x, one = torch.zeros(1, 4, 64, device="cuda", dtype=p.dtype), batch([4], [1])
    b, twice, last, n_keep = batch([0, 2], [20, 20]), batch([0, 0], [1, 1]), batch([0], [20]), i32([2])
    before = state(p)
    torch.cuda._sleep(40_000_000)
    p.attention(0, one, x, x)                        # a row of a sequence without tokens
    p.reserve(twice if bad else b)
    torch.cuda.synchronize()
    torch.cuda._sleep(40_000_000)
    with pytest.raises(msd.MsdError) as e:
        p.compact(last, None, n_keep)
    assert e.value.status == msd.MSD_ERR_DEVICE
    p.compact(last, None, n_keep)                    # queued before the reserve's error has come up
    torch.cuda.synchronize()
    assert same(p, before)
    reported(p, msd.MSD_ERR_DEVICE if bad else msd.MSD_ERR_CAPACITY)
    p.compact(last, None, n_keep)                    # runs
    torch.cuda.synchronize()
    assert p.lens.tolist() == [46, 96, 64, 0, 0]


def test_an_error_met_while_recording_is_reported_again():
    """A call that is being recorded reports the error but cannot take note of it: nothing runs then."""
    p = shared_pool()
    p.reserve(batch([0], [40]))
    torch.cuda.synchronize()
    x = torch.ones(1, device="cuda")
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        x.add_(1)
        for _ in range(2):
            with pytest.raises(msd.MsdError):
                p.restore()
    reported(p, msd.MSD_ERR_CAPACITY)
    p.reserve(batch([0], [16]))
    torch.cuda.synchronize()
    assert int(p.lens[0]) == 80


# ---------------------------------------------------------------------------
# Pages that several sequences hold, pages that are none
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_on_shared_pages_are_not_written(dtype):
    """Rows appended without room of their own lie on the fork's pages too: skipped and reported."""
    p = shared_pool(dtype)
    before = state(p)
    q = torch.full((20, 4, 64), 7.0, device="cuda", dtype=p.dtype)
    g = torch.randn(20, 512, device="cuda").to(p.dtype)
    p.rope_append(0, batch([0], [20]), g[:, :256], g[:, 256:384], g[:, 384:], i32([list(range(20))]), q)
    torch.cuda.synchronize()
    assert same(p, before) and not (q == 7).any()
    reported(p, msd.MSD_ERR_DEVICE)
    p.free(i32([2]))                                 # now they are its own
    p.rope_append(0, batch([0], [20]), g[:, :256], g[:, 256:384], g[:, 384:], i32([list(range(20))]), q)
    p.restore()
    torch.cuda.synchronize()
    p.restore()
    _, v = tokens(p, 0, 0)
    assert torch.equal(v[44:], g[:, 384:].double().view(20, 2, 64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("entry", [-1, 1 << 20])
def test_an_entry_that_is_no_page_is_read_as_zeros_and_reported(dtype, page, entry):
    """In the middle of a sequence, and its last page: K and V there count as zeros, in both types; other
    sequences are as they were."""
    p = pool([5 * page + 3, 3 * page, 2 * page], dtype=dtype, page=page, heads=4, kv_heads=2)
    counts = [40, 9, 1]
    kv = [tokens(p, 0, s) for s in range(3)]
    for s, k in ((0, 1), (0, 5), (1, 2)):
        p.table[s, k] = entry
        for x in kv[s]:
            x[k * page:(k + 1) * page] = 0
    for window, sinks in ((0, 0), (4 * page, 3)):
        q = torch.randn(sum(counts), 4, 64, device="cuda").to(p.dtype)
        out, lse = torch.full_like(q, 7.0), torch.zeros(sum(counts), 4, device="cuda")
        p.attention(0, batch([0, 1, 2], counts), q, out, lse=lse, window=window, sinks=sinks)
        reported(p, msd.MSD_ERR_DEVICE)
        at = 0
        for (k, v), n in zip(kv, counts):
            place = torch.arange(k.shape[0], device="cuda")
            ok = place[None] <= place[-n:, None]
            if window:
                ok &= (place[-n:, None] - place[None] < window) | (place < sinks)[None]
            ref, rl = attend(q[at:at + n], k, v, ok)
            bo, bl = bounds(q[at:at + n], k, v, ref, rl, dtype)
            assert bool(((out[at:at + n].double() - ref).abs() <= bo).all())
            assert bool(((lse[at:at + n].double() - rl).abs() <= bl).all())
            at += n


# ---------------------------------------------------------------------------
# Lists that are refused whole
# ---------------------------------------------------------------------------
def test_free_takes_a_list_whole_or_not_at_all():
    p = pool([20, 40, 33], extra_seqs=2)
    for bad in ([0, 77], [77, 0, 1], [1, -1, 2]):
        before = state(p)
        p.free(i32(bad))
        reported(p, msd.MSD_ERR_DEVICE)
        assert same(p, before)
    for length in (-7, p.cfg.max_pages * 16 + 1):
        keep = int(p.lens[1])
        p.lens[1] = length
        before = state(p)
        p.free(i32([0, 1, 2]))
        reported(p, msd.MSD_ERR_DEVICE)
        assert same(p, before)
        p.lens[1] = keep
    p.free(i32([2, 0, 4, 2, 0]))
    torch.cuda.synchronize()
    assert p.lens.tolist() == [0, 40, 0, 0, 0] and int(p.refs.sum()) == 3
    p.restore()


def test_free_of_a_long_list():
    n = 4000
    p = msd.Pages(dtype="bf16", layers=1, heads=1, kv_heads=1, head_dim=64, page_size=16, n_pages=3 * n, max_seqs=n,
                  max_pages=3)
    b = batch(list(range(n)), [1 + i % 48 for i in range(n)])
    p.reserve(b)
    torch.cuda.synchronize()
    before = state(p)
    p.free(i32(list(range(n - 1)) + [n]))
    reported(p, msd.MSD_ERR_DEVICE)
    assert same(p, before)
    p.free(b.seqs)
    torch.cuda.synchronize()
    assert not p.refs.any() and not p.lens.any() and (p.table == -1).all()


def test_page_counts_past_32_bits_are_refused():
    """Rows that would need 32 x 2^26 pages, more than 32 bits count: refused, nothing grows. (20 GB of tables.)"""
    p = msd.Pages(dtype="bf16", layers=1, heads=1, kv_heads=1, head_dim=64, page_size=16, n_pages=40, max_seqs=33,
                  max_pages=1 << 26)
    p.reserve(batch([32], [5]))
    for n in (32, 31):
        b = msd.Batch(i32(list(range(n))), torch.zeros(n + 1, dtype=torch.int32, device="cuda"), 0)
        # every sequence asks for 2^30 rows: the boundaries wrap, their differences do not
        b.row_start.copy_(((torch.arange(n + 1) << 30) & 0xffffffff).to(torch.int64).to(torch.int32))
        p.reserve(b)
        reported(p, msd.MSD_ERR_CAPACITY)
        assert p.lens.tolist() == [0] * 32 + [5] and int(p.refs.sum()) == 1
    p.reserve(batch([0, 1], [30, 17]))
    torch.cuda.synchronize()
    assert p.lens[:2].tolist() == [30, 17] and int(p.refs.sum()) == 5
    del p
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------
# Values that are not finite in a long prompt
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("window,sinks", [(0, 0), (4096, 2)])
def test_a_long_prompt_with_values_that_are_not_finite(window, sinks):
    """Some entries of V: the rows that see them have them in their columns, everything else is what it is
    without them, to the bit, and the launch ends by itself (no wait runs out)."""
    n = 131072
    p = pool([n], heads=8, kv_heads=1, head_dim=128, page=128, stale=0.0)
    q = torch.randn(n, 8, 128, device="cuda").to(p.dtype)
    b, want, got = batch([0], [n]), torch.empty_like(q), torch.empty_like(q)
    p.attention(0, b, q, want, window=window, sinks=sinks)
    for slot, col, value in ((5, 3, float("nan")), (70000, 40, float("inf")), (n - 9, 100, -float("inf"))):
        p.kv[0, p.table[0, slot // 128].long(), 1, 0, slot % 128, col] = value
        want[slot:slot + window if window else n, :, col] = value
    p.attention(0, b, q, got, window=window, sinks=sinks)
    torch.cuda.synchronize()
    p.restore()                                      # nothing to report
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())


# ---------------------------------------------------------------------------
# Limits
# ---------------------------------------------------------------------------
def test_compaction_of_a_pool_of_many_layers():
    """More (layer, K or V) pairs than a launch's y extent; shared pages are replaced in every layer."""
    layers = 65535
    p = msd.Pages(dtype="bf16", layers=layers, heads=1, kv_heads=1, head_dim=128, page_size=16, n_pages=4, max_seqs=2,
                  max_pages=3)
    p.reserve(batch([0], [32]))
    p.kv.view(layers, -1).copy_(torch.arange(layers, device="cuda")[:, None].remainder(251))
    p.kv[:, :, :, :, 16 - 3:] += 1000
    p.fork(i32([0]), i32([1]))
    p.compact(batch([0], [3]), None, i32([1]))
    p.compact(batch([1], [20]), i32([[0, 18]]), i32([2]))
    torch.cuda.synchronize()
    assert p.lens.tolist() == [30, 14] and int(p.refs.sum()) == 3
    for seq, slot, value in ((0, 12, 0), (0, 13, 1000), (0, 28, 0), (0, 29, 1000), (1, 11, 0), (1, 12, 0), (1, 13, 1000)):
        page = p.kv[:, p.table[seq, slot // 16].long(), :, 0, slot % 16].float()
        assert torch.equal(page, (torch.arange(layers, device="cuda") % 251 + value)[:, None, None].to(p.dtype).float().expand_as(page))
    del p
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_depths_that_no_tree_has_are_reported(dtype):
    """A window goes by depths: one outside 0 .. tree_nodes - 1 is told, and taken as the nearest that is inside."""
    p = pool([300, 40], dtype=dtype)
    t, _, _ = random_tree(2, 20, 3)
    q = torch.randn(40, 4, 64, device="cuda").to(p.dtype)
    b, got = batch([0, 1], [20, 20]), []
    for bad, inside in ((10 ** 6, 19), (-3, 0)):
        for value in (bad, inside):
            t.depth.view(2, 20)[0, 7] = value
            out, lse = torch.empty_like(q), torch.empty(40, 4, device="cuda")
            p.attention(0, b, q, out, lse=lse, tree=t, window=30, sinks=2)
            if value == bad:
                reported(p, msd.MSD_ERR_DEVICE)
            got.append((out, lse))
        torch.cuda.synchronize()
        p.restore()
        for x, y in zip(got[-2], got[-1]):
            assert torch.equal(x, y)
    t.n_nodes[1] = 12
    t.depth.view(2, 20)[1, 12:] = -9                 # past the tree's nodes: of no account
    p.attention(0, b, q, out, lse=lse, tree=t, window=30, sinks=2)
    torch.cuda.synchronize()
    p.restore()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sequences_past_one_launch_take_the_tiles_of_the_whole_call(dtype):
    """The 513th of 513 single tokens is computed as it is by itself, to the bit."""
    lens = [1 + i % 30 for i in range(512)] + [60000]
    p = pool(lens, dtype=dtype, heads=8, kv_heads=2, head_dim=128)
    q = torch.randn(513, 8, 128, device="cuda").to(p.dtype)
    out, lse = torch.empty_like(q), torch.empty(513, 8, device="cuda")
    p.attention(0, batch(list(range(513)), [1] * 513), q, out, lse=lse)
    one, l1 = torch.empty_like(q[:1]), torch.empty(1, 8, device="cuda")
    p.attention(0, batch([512], [1]), q[512:], one, lse=l1)
    torch.cuda.synchronize()
    assert torch.equal(out[512:], one) and torch.equal(lse[512:], l1)
