"""Products with 4-bit weights (msd_linear4) and their codes (msd_quantize4) against plain
64-bit forms: one row to many, odd sizes, every group, short last groups, zeros, both types,
strides, accumulation, streams, graphs, values that are not finite, and refusals."""
import math

import numpy as np
import pytest
import torch

from paper_2505_14260_gb300 import build, msd
from tests.tokens_support import LINEAR4, linear4_shape

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def weight(o, k, group, zeros, seed=0):
    g, n = gen(seed), -(-k // group)
    codes = torch.randint(0, 256, (o, k // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = (0.01 + 0.05 * torch.rand(o, n, generator=g, device="cuda")).bfloat16()
    z = torch.randint(0, 16, (o, n), generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    return msd.Weight4(codes, scales, z, group)


def values(w):
    """The weight's values in 64 bits."""
    c = torch.stack([w.codes & 15, w.codes >> 4], -1).view(w.o, w.k).double()
    wide = lambda t: t.double().repeat_interleave(w.group, 1)[:, :w.k]  # noqa: E731
    return wide(w.scales) * (c - (8.0 if w.zeros is None else wide(w.zeros)))


def check(w, x, y, before=None):
    """Any order of fp32 sums of k terms is off by k units of 2^-24 of the terms' magnitudes at
    most, twice that where additions truncate; the typical size: a group's terms add up in 8 steps
    or fewer on the tensor cores and the at most few hundred groups like a random walk."""
    v = values(w)
    ref = x.double() @ v.T + (0 if before is None else before.double())
    room = x.double().abs() @ v.abs().T + (0 if before is None else before.double().abs())
    err = (y.double() - ref).abs()
    assert bool((err <= (w.k + 16) * 2.0 ** -23 * room + 1e-36).all()), float((err / room.clamp(min=1e-30)).max())
    assert float(err.norm()) <= 2.0 ** -19 * float(ref.norm().clamp(min=1e-30)) + 2.0 ** -21 * float(room.norm()), \
        float(err.norm() / ref.norm())


def run(m, k, o, group=128, zeros=False, dtype=torch.bfloat16, seed=0, accumulate=False):
    w = weight(o, k, group, zeros, seed)
    x = torch.randn(m, k, generator=gen(seed + 1), device="cuda").to(dtype)
    y = torch.randn(m, o, generator=gen(seed + 2), device="cuda") if accumulate else torch.full((m, o), math.nan, device="cuda")
    before = y.clone() if accumulate else None
    assert w.linear(x, y, accumulate=accumulate) is y
    torch.cuda.synchronize()
    check(w, x, y, before)


TYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 2, 3, 7, 8, 9, 16, 17, 60, 64, 65, 130])
def test_rows(m, group, zeros, dtype):
    run(m, 1024, 200, group, zeros, dtype, seed=m)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k", [8, 16, 24, 32, 40, 64, 96, 120, 128, 136, 160, 256, 688, 1000, 1056, 4096, 11008, 13824])
@pytest.mark.parametrize("m", [1, 12, 70])
def test_inner_sizes(m, k, dtype):
    for group, zeros in ((128, False), (64, True), (32, True)):
        run(m, k, 77, group, zeros, dtype, seed=k)


@pytest.mark.parametrize("m", [1, 5, 33, 140])
@pytest.mark.parametrize("o", [1, 2, 15, 16, 17, 63, 127, 128, 129, 1000, 4096, 32000])
def test_outputs(m, o):
    run(m, 512, o, 64, True, seed=o)
    run(m, 416, o, 128, False, torch.float32, seed=o)


@pytest.mark.parametrize("m", [1, 9, 60, 300])
def test_accumulate(m):
    run(m, 768, 300, 128, True, accumulate=True)
    run(m, 768, 300, 32, False, torch.float32, accumulate=True)


@pytest.mark.parametrize("m", [500, 1025, 2100])
def test_many_rows(m):
    run(m, 1056, 530, 128, True)
    run(m, 1000, 130, 32, False, torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 3, 8, 12, 16, 30])
def test_few_rows_of_long_ones(m, group, dtype):
    """Few rows on either side of the choice between the kernels; codes that tensor copies take and ones they do not."""
    for k, o, zeros in ((11000, 150, True), (9984, 300, False), (11008, 40, True), (2048, 9000, True), (1000, 20000, False)):
        run(m, k, o, group, zeros, dtype, seed=m + k)


@pytest.mark.parametrize("m,o", [(129, 11008), (150, 12700), (192, 10000), (130, 19456), (256, 9856)])
def test_rows_past_a_block(m, o):
    """Where rows past a multiple of 128 make the fewest CTAs blocks of 64 rows, and beside it."""
    run(m, 256, o, 128, True)


@pytest.mark.parametrize("case", LINEAR4, ids=lambda c: "-".join(str(v) for v in c[:6]))
def test_every_kernel(case):
    """Each kernel that there is, with its scales and zeros staged and read where they are, and the sizes of large layers. Relative to the
    norm of y: a group's sum is rounded (or cut) once for each 16 elements and plane that are added to it, its share of the total once,
    by 2^-24 of the sum on average, alike within a group at worst and at random over the groups; 4 for the rest."""
    dtype, group, m, k, o, zeros, few, rows, outputs, staged = case
    w = weight(o, k, group, zeros, m)
    c = linear4_shape(dtype, group, m, k, o, zeros, w.codes.data_ptr())
    assert (c.few, c.rows, c.outputs, c.staged) == (few, rows, outputs, staged)
    x = torch.randn(m, k, generator=gen(m + 1), device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    y = w.linear(x, torch.full((m, o), math.nan, device="cuda"))
    torch.cuda.synchronize()
    ref = x.double() @ values(w).T
    adds = group // 16 * (3 if dtype == "f32" else 1)
    assert float((y.double() - ref).norm() / ref.norm()) <= 2.0 ** -24 * (adds + (k / group) ** 0.5 + 4)
    assert float((y.double() - ref).abs().max() / ref.abs().max()) <= 2.0 ** -20 * (adds + (k / group) ** 0.5 + 4)


@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("m", [5, 12, 60])
def test_later_planes_of_fp32_x_keep_their_bits(m, group):
    """With sums of their own, or first: errors of 8e-8 of the norm of y where plane after plane made 4.4e-7. The bound lies between."""
    w = weight(300, 2048, group, True, m)
    x = torch.randn(m, 2048, generator=gen(m), device="cuda")
    y = w.linear(x, torch.empty(m, 300, device="cuda")).double()
    ref = x.double() @ values(w).T
    assert float((y - ref).norm() / ref.norm()) <= 2.0 ** -22


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 11, 66, 200])
def test_strides_and_neighbours(m, dtype):
    """Rows of x and y inside wider ones: nothing beside y's rows is written, what lies beside x's is not read."""
    k, o = 352, 45
    w = weight(o, k, 64, True)
    wide = torch.full((m + 2, k + 48), math.nan, device="cuda", dtype=dtype)
    wide[1:-1, 16:16 + k] = torch.randn(m, k, generator=gen(1), device="cuda").to(dtype)
    out = torch.full((m + 2, o + 9), 7.0, device="cuda")
    w.linear(wide[1:-1, 16:16 + k], out[1:-1, 3:3 + o])
    torch.cuda.synchronize()
    check(w, wide[1:-1, 16:16 + k], out[1:-1, 3:3 + o])
    out[1:-1, 3:3 + o] = 7.0
    assert bool((out == 7).all())


def test_codes_at_a_four_byte_address():
    """Weights inside a larger buffer, at an address that only words are aligned to."""
    for k in (1024, 352, 40):
        w = weight(50, k, 32, True)
        raw = torch.zeros(50 * k // 2 + 64, dtype=torch.uint8, device="cuda")
        inside = raw[4:4 + 50 * k // 2].view(50, k // 2)
        inside.copy_(w.codes)
        x = torch.randn(70, k, generator=gen(3), device="cuda").bfloat16()
        for m in (1, 20, 70):
            y = torch.full((m, 50), math.nan, device="cuda")
            w2 = msd.Weight4(inside, w.scales, w.zeros, 32)
            w2.linear(x[:m], y)
            torch.cuda.synchronize()
            check(w, x[:m], y)


def test_fp32_x_is_not_rounded():
    """x whose values need all 24 bits: the products differ from those of x in bf16 or in two parts."""
    w = weight(64, 256, 32, False)
    x = torch.zeros(3, 256, device="cuda")
    x[:, 0], x[:, 1] = 1 + 2.0 ** -23, -1.0
    x[1] *= 2.0 ** 60
    x[2] *= 2.0 ** -60
    y = torch.empty(3, 64, device="cuda")
    w.codes[:, 0] = 0x99                     # code 9 in both: 1 * scale
    w.linear(x, y)
    torch.cuda.synchronize()
    want = w.scales[:, 0].double() * 2.0 ** -23
    for i, f in enumerate((1.0, 2.0 ** 60, 2.0 ** -60)):
        assert torch.equal(y[i].double(), want * f)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m,o", [(8, 300), (12, 300), (12, 20000), (60, 300), (60, 20000)])
def test_fp32_x_is_not_rounded_in_any_kernel(m, o, group):
    """The same of every kernel of fp32 x: rows of one value that needs 24 bits, with another of the opposite sign or not."""
    w = weight(o, 256, group, False)
    w.codes[:, 0] = 0x99
    x = torch.zeros(m, 256, device="cuda")
    x[:, 0] = (1 + 2.0 ** -23) * 2.0 ** torch.arange(m, device="cuda")
    x[::2, 1] = -(2.0 ** torch.arange(0, m, 2, device="cuda"))
    y = torch.empty(m, o, device="cuda")
    w.linear(x, y)
    torch.cuda.synchronize()
    s = w.scales[:, 0].double()
    for i in range(m):
        assert torch.equal(y[i], (s * float(x[i, 0].double() + x[i, 1].double())).float())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m", [2, 10, 66, 200])
def test_the_largest_values(m, group, dtype):
    """Up to 2^117: a group's sum, 128 products with up to 15, stays finite before it is scaled."""
    w = weight(40, 256, group, True)
    x = torch.randn(m, 256, generator=gen(1), device="cuda").sign() * 2.0 ** 117
    x[1::2] = x[1::2].abs()
    x = x.to(dtype)
    y = w.linear(x, torch.empty(m, 40, device="cuda"))
    torch.cuda.synchronize()
    check(w, x, y)


@pytest.mark.parametrize("m,o", [(8, 64), (12, 64), (40, 64), (12, 20000)])
def test_the_smallest_values(m, o):
    """fp32 down to 2^-110 exactly, below it less what lies under bf16's smallest step, 2^-133; bf16 as it is. Scales of 2^100."""
    ones = torch.full((o, 128), 0x99, dtype=torch.uint8, device="cuda")
    w = msd.Weight4(ones, torch.full((o, 8), 2.0 ** 100, dtype=torch.bfloat16, device="cuda"), None, 32)
    v = torch.tensor([(1 + 2.0 ** -23) * 2.0 ** e for e in (-100, -109, -110)] + [2.0 ** -126, 2.0 ** -133, 0.0, -0.0, 0.0], dtype=torch.float64)
    small = torch.tensor([(1 + 2.0 ** -23) * 2.0 ** e for e in (-111, -112, -120, -126, -127, -133, -134, -149)], dtype=torch.float64)
    for values_, room in ((v, 0.0), (small, 2.0 ** -33)):
        x = torch.zeros(m, 256, device="cuda")
        x[:8, 0] = values_.float().cuda()
        y = w.linear(x, torch.empty(m, o, device="cuda")).double().cpu()
        assert bool(((y[:8] - 2.0 ** 100 * values_.float().double()[:, None]).abs() <= room).all())
    x = torch.zeros(m, 256, dtype=torch.bfloat16, device="cuda")
    x[:2, 0] = torch.tensor([2.0 ** -126, 2.0 ** -133], device="cuda").bfloat16()
    y = w.linear(x, torch.empty(m, o, device="cuda")).double()
    assert bool((y[0] == 2.0 ** -26).all()) and bool((y[1] == 2.0 ** -33).all()) and bool((y[2:] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [2, 10, 66, 200])
def test_values_that_are_not_finite(m, dtype):
    """They reach their own rows of y alone; so do the largest finite ones."""
    w = weight(40, 256, 128, True)
    x = torch.randn(m, 256, generator=gen(1), device="cuda").to(dtype)
    clean = torch.empty(m, 40, device="cuda")
    w.linear(x, clean)
    x[1, 5] = math.inf
    if m > 2:
        x[3, 200], x[m - 1, 0] = math.nan, -math.inf
    y = torch.empty(m, 40, device="cuda")
    w.linear(x, y)
    torch.cuda.synchronize()
    bad = torch.zeros(m, dtype=torch.bool)
    bad[1] = True
    if m > 2:
        bad[3] = bad[m - 1] = True
    assert not bool(y[bad.cuda()].isfinite().any())
    assert torch.equal(y[~bad.cuda()], clean[~bad.cuda()])


@pytest.mark.parametrize("m,k,o,group,dtype,chunk", [(1, 5120, 300, 128, torch.bfloat16, 13), (60, 1024, 300, 64, torch.bfloat16, 0),
                                                     (60, 640, 20000, 32, torch.bfloat16, 3), (458, 3520, 135, 128, torch.bfloat16, 7),
                                                     (30, 4096, 300, 64, torch.float32, 2)])
def test_a_wait_that_runs_out(m, k, o, group, dtype, chunk):
    """Codes that never come: after 2 s every role gives up, y is NaN, nothing beside it is written and the next call is as ever."""
    w = weight(o, k, group, True)
    x = torch.randn(m, k, generator=gen(1), device="cuda").to(dtype)
    wide = torch.full((m, o + 3), 7.0, device="cuda")
    start = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start[0].record()
    assert msd.lib().msd_test_linear4_timeout(x.data_ptr(), k, msd.MSD_BF16 if dtype == torch.bfloat16 else msd.MSD_F32, m, w._ref,
                                              wide.data_ptr(), o + 3, chunk, torch.cuda.current_stream().cuda_stream) == msd.MSD_OK
    start[1].record()
    y = w.linear(x, torch.empty(m, o, device="cuda"))
    torch.cuda.synchronize()
    assert bool(wide[:, :o].isnan().all()) and bool((wide[:, o:] == 7).all())
    assert 1900 < start[0].elapsed_time(start[1]) < 3000
    check(w, x, y)


def test_no_rows():
    weight(8, 64, 32, False).linear(torch.empty(0, 64, device="cuda"), torch.empty(0, 8, device="cuda"))


def test_the_same_sums_each_time():
    for m in (1, 16, 60, 300):
        w, x = weight(600, 4096, 128, True), torch.randn(m, 4096, generator=gen(1), device="cuda").bfloat16()
        ys = [w.linear(x, torch.empty(m, 600, device="cuda")) for _ in range(5)]
        assert all(torch.equal(y, ys[0]) for y in ys[1:])


def test_streams_and_graphs():
    w = weight(5000, 2048, 64, True)
    xs = [torch.randn(60, 2048, generator=gen(s), device="cuda").bfloat16() for s in (1, 2)]
    want = [w.linear(x, torch.empty(60, 5000, device="cuda")) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    out = [torch.empty(60, 5000, device="cuda") for _ in xs]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, x, y in zip(streams, xs, out):
            w.linear(x, y, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    for m in (1, 60):
        x, y = xs[0][:m].clone(), torch.empty(m, 5000, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            w.linear(x, y)
        for src in xs:
            x.copy_(src[:m])
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, w.linear(src[:m], torch.empty(m, 5000, device="cuda")))


# -- codes -------------------------------------------------------------------
def plain_codes(w, group, zeros):
    """Quotients in 64 bits (exact enough to tell every border: scales have 8 bits, values 24)."""
    o, k = w.shape
    n = -(-k // group)
    v = torch.nn.functional.pad(w.double().nan_to_num(0.0), (0, n * group - k)).view(o, n, group)
    lo, hi = v.amin(-1).clamp(max=0), v.amax(-1).clamp(min=0)
    wide = (hi - lo) / 15 if zeros else torch.maximum(hi, -lo) / 7
    part, e = np.frexp(wide.cpu().numpy())                 # exact powers of two (the GPU's pow rounds them)
    s = torch.from_numpy(np.ldexp(np.rint(part * 256), e - 8)).cuda()
    s = torch.where(s >= 2.0 ** -126, s, 0.0)
    div = torch.where(s > 0, s, 1.0)
    z = torch.round(-lo / div).clamp(0, 15) if zeros else torch.full_like(s, 8.0)
    z = torch.where(s > 0, z, 0.0 if zeros else 8.0)
    q = torch.where(s[..., None] > 0, torch.round(v / div[..., None]) + z[..., None], z[..., None]).clamp(0, 15)
    out = (s[..., None] * (q - z[..., None])).view(o, -1)[:, :k]
    q = q.view(o, -1)[:, :k].to(torch.uint8)
    return q[:, 0::2] | (q[:, 1::2] << 4), s, z.to(torch.uint8), out


def check_codes(w, group, zeros, with_values=True):
    c, s, z, v = plain_codes(w, group, zeros)
    got = torch.full((w.shape[0], w.shape[1] + 8), 7.0, dtype=w.dtype, device="cuda")[:, :w.shape[1]] if with_values else None
    q = msd.Weight4.of(w, group=group, zeros=zeros)
    if with_values:
        q.quantize(w, values=got)
    torch.cuda.synchronize()
    assert torch.equal(q.scales.double(), s)
    assert q.zeros is None or torch.equal(q.zeros, z)
    assert torch.equal(q.codes, c), int((q.codes != c).sum())
    if with_values:
        assert torch.equal(got, v.to(w.dtype))          # products of 8 and 5 bits: one rounding to bf16, none to fp32


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("o,k", [(1, 8), (3, 24), (2, 32), (17, 40), (5, 136), (64, 256), (33, 688), (130, 1000), (257, 4096)])
def test_codes(o, k, group, zeros, dtype):
    w = (0.02 * torch.randn(o, k, generator=gen(o + k), device="cuda")).to(dtype)
    check_codes(w, group, zeros)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("zeros", [False, True])
def test_codes_of_odd_values(zeros, dtype):
    """Zero groups, one sign, ties of two codes, one large value, tiny and huge ones, NaN."""
    g = gen(4)
    w = torch.randn(12, 256, generator=g, device="cuda")
    w[0] = 0
    w[1] = w[1].abs()
    w[2] = -w[2].abs()
    w[3] = torch.randint(-14, 15, (256,), generator=g, device="cuda") / 2.0
    w[3, ::32] = 7.0                                       # scale 1: every half is a tie
    w[4, 9] = 1000.0
    w[5] *= 1e-37
    w[6] *= 1e-42
    w[7] *= 1e36
    w[8, ::5] = math.nan
    w[9] = 0
    w[9, 100] = -1e-30
    w[10] = 3.0
    w[11, 64:] = 0
    check_codes(w.to(dtype), 32, zeros)
    check_codes(w.to(dtype), 128, zeros)


def test_many_borders():
    """fp32 values around every border of two codes."""
    s = 2.0 ** -7
    base = torch.arange(-15, 16, device="cuda").float().repeat_interleave(3) * (s / 2)
    ulp = torch.tensor([-1, 0, 1], dtype=torch.int32, device="cuda").repeat(31)
    v = (base.view(torch.int32) + ulp).view(torch.float32)
    v = torch.where((base == 0) & (ulp != 0), 1e-9 * ulp, v)
    w = torch.zeros(16, 128, device="cuda")
    w[:, :93] = v * torch.logspace(-8, 7, 16, base=2.0, device="cuda")[:, None]
    w[:, 100] = 7 * s * torch.logspace(-8, 7, 16, base=2.0, device="cuda")
    for zeros in (False, True):
        check_codes(w, 128, zeros)


def test_codes_of_strided_rows():
    wide = torch.randn(20, 320, generator=gen(5), device="cuda")
    check_codes(wide[:, 32:32 + 200], 64, True)
    check_codes(wide.bfloat16()[:, 64:64 + 200], 64, False)
    check_codes(wide[:1, 4:4 + 16], 32, False, with_values=False)


def test_of_beside_another_stream():
    """What the current stream still writes into memory that it has given back does not meet codes made on another stream."""
    w = 0.05 * torch.randn(512, 1024, generator=gen(8), device="cuda")
    want = msd.Weight4.of(w, group=64, zeros=True)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        used = [torch.empty_like(t) for t in (want.codes, want.scales, want.zeros)]
        for _ in range(200):
            for t in used:
                t.fill_(77)
        del used, t
        got = msd.Weight4.of(w, group=64, zeros=True, stream=s)
        torch.cuda.synchronize()
        for a, b in ((got.codes, want.codes), (got.scales, want.scales), (got.zeros, want.zeros)):
            assert torch.equal(a, b)
        del got, a


def test_of_and_linear_together():
    """A projection brought to 4 bits: its products are those of the values it stands for."""
    w = 0.05 * torch.randn(688, 256, generator=gen(6), device="cuda")
    back = torch.empty_like(w)
    q = msd.Weight4.of(w, group=32, zeros=True).quantize(w, values=back)
    assert torch.equal(values(q), back.double())
    assert float((back - w).norm() / w.norm()) < 0.15          # a step of range / 15, uniformly within half of it
    x = torch.randn(5, 256, generator=gen(7), device="cuda")
    y = q.linear(x, torch.empty(5, 688, device="cuda"))
    check(q, x, y)


def test_refusals():
    w = weight(40, 256, 64, False)
    x, y = torch.randn(4, 256, device="cuda"), torch.empty(4, 40, device="cuda")
    for bad in (lambda: w.linear(x.half(), y), lambda: w.linear(x[:, :128], y), lambda: w.linear(x, y.bfloat16()), lambda: w.linear(x, y[:3]),
                lambda: w.linear(x.t(), y), lambda: w.linear(x.cpu(), y), lambda: w.linear(x, y.cpu()),
                lambda: msd.Weight4(w.codes, w.scales[:, :1], None, 64), lambda: msd.Weight4(w.codes, w.scales.float(), None, 64),
                lambda: msd.Weight4(w.codes.int(), w.scales, None, 64), lambda: msd.Weight4(w.codes, w.scales, None, 48),
                lambda: msd.Weight4(w.codes, w.scales, w.codes, 64), lambda: w.quantize(x), lambda: msd.Weight4.of(x.half()),
                lambda: w.quantize(torch.empty(40, 256, device="cuda"), values=torch.empty(40, 256, device="cuda").bfloat16())):
        with pytest.raises(ValueError):
            bad()
    odd = msd.Weight4(torch.zeros(4, 6, dtype=torch.uint8, device="cuda"), torch.ones(4, 1, dtype=torch.bfloat16, device="cuda"), None, 64)
    unaligned = torch.empty(4, 264, device="cuda")
    for bad in (lambda: odd.linear(torch.empty(1, 12, device="cuda"), torch.empty(1, 4, device="cuda")),
                lambda: w.linear(unaligned[:, 1:257], y), lambda: w.linear(torch.empty(4, 257, device="cuda")[:, :256], y),
                lambda: w.quantize(torch.empty(40, 257, device="cuda")[:, :256])):
        with pytest.raises(msd.MsdError):
            bad()
