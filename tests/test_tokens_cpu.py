"""Filtered sampling, tree acceptance and 4-bit products: arguments that are refused before
anything touches a GPU, and the sums behind the fixed-point weights."""
import ctypes
import itertools
import os
import random
import re
import shutil
import subprocess

import pytest
import torch

from paper_2505_14260_gb300 import build, msd
from tests.tokens_support import LINEAR4, linear4_shape

P = ctypes.c_void_p
A = 1 << 20                      # an address that nothing reads: every call here is refused


@pytest.fixture(scope="module")
def lib():
    build.build()
    return msd.lib()


def linear(lib, x=A, ldx=64, xt=msd.MSD_BF16, m=1, codes=A, scales=A, o=8, k=64, group=32, y=A, ldy=8):
    w = msd.msd_weight4(codes, scales, None, o, k, group)
    return lib.msd_linear4(x, ldx, xt, m, ctypes.byref(w), y, ldy, 0, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(ldx=63), dict(ldx=68), dict(xt=2), dict(m=-1), dict(codes=None), dict(scales=None),
                                 dict(o=0), dict(k=0), dict(k=60), dict(k=12, ldx=16), dict(group=16), dict(group=48), dict(y=None),
                                 dict(ldy=7), dict(x=A + 2), dict(x=A + 8), dict(y=A + 2), dict(codes=A + 2), dict(scales=A + 1)], ids=str)
def test_linear4_refuses(lib, bad):
    assert linear(lib, **bad) == msd.MSD_ERR_INVALID


@pytest.mark.parametrize("bad", [dict(k=2**31 - 8, ldx=2**31 - 8), dict(k=2**30 + 8, ldx=2**30 + 8), dict(o=2**31 - 1, ldy=2**31 - 1),
                                 dict(o=2**30 + 1, ldy=2**30 + 1)], ids=str)
def test_weights_whose_indices_would_pass_32_bits(lib, bad):
    """Sizes are rounded up to groups, chunks and tiles in 32 bits."""
    for group in (32, 64, 128):
        assert linear(lib, group=group, **bad) == msd.MSD_ERR_INVALID
        a = dict(o=8, k=64)
        a.update({n: v for n, v in bad.items() if n in a})
        w = msd.msd_weight4(A, A, None, a["o"], a["k"], group)
        assert lib.msd_quantize4(A, a["k"], msd.MSD_F32, ctypes.byref(w), None, 0, None) == msd.MSD_ERR_INVALID


def test_every_kernel_of_a_product_is_among_the_tested_ones(lib):
    """The list that the GPU tests run has each kernel, with scales and zeros staged and not, whatever the times that choose between
    them become; sizes from a token's to long prompts' lead to no other."""
    for dtype, group, m, k, o, zeros, few, rows, outputs, staged in LINEAR4:
        c = linear4_shape(dtype, group, m, k, o, zeros)
        assert (c.few, c.rows, c.outputs, c.staged) == (few, rows, outputs, staged), (dtype, group, m, k, o, zeros)
    tested = {(c[0], c[1], *c[6:]) for c in LINEAR4}
    blocks = {"bf16": [(1, 8, 32), (1, 16, 32), (0, 16, 128), (0, 16, 256), (0, 32, 128), (0, 32, 256), (0, 64, 128), (0, 64, 256), (0, 128, 128)],
              "f32": [(1, 8, 32), (0, 16, 128), (0, 16, 256), (0, 32, 128), (0, 32, 256)]}
    for dtype in blocks:
        for group, b in itertools.product((32, 64, 128), blocks[dtype]):
            assert (dtype, group, *b, 1) in tested, (dtype, group, b)
    rng, rare = random.Random(3), set()
    for _ in range(20000):
        dtype, group = rng.choice(("bf16", "f32")), rng.choice((32, 64, 128))
        m, k, o = int(2 ** rng.uniform(0, 12)), 8 * int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 17))
        c = linear4_shape(dtype, group, m, k, o, rng.random() < 0.5)
        assert c.smem_bytes <= 227 * 1024 and 1 <= c.split <= 8
        assert c.few or c.smem_bytes >= 193 * 1024          # (all of an SM's tensor memory: no second CTA that waits for some fits beside it)
        if (dtype, group, c.few, c.rows, c.outputs, c.staged) not in tested:
            rare.add((dtype, group, c.few, c.rows, c.outputs, c.staged))
    assert all(not staged and not few for _, _, few, _, _, staged in rare) and len(rare) <= 4, rare


def test_the_shape_hook_refuses_bad_arguments(lib):
    w, out = msd.msd_weight4(A, A, None, 8, 64, 32), msd.msd_linear4_shape()
    for dtype, m, weight in ((2, 1, w), (1, 0, w), (1, -1, w), (1, 1, msd.msd_weight4(A, A, None, 8, 60, 32)), (1, 1, msd.msd_weight4(A, A, None, 0, 64, 32))):
        assert lib.msd_test_linear4_shape(dtype, m, ctypes.byref(weight), ctypes.byref(out)) == msd.MSD_ERR_INVALID
    assert lib.msd_test_linear4_shape(1, 1, None, ctypes.byref(out)) == msd.MSD_ERR_INVALID
    assert lib.msd_test_linear4_shape(1, 1, ctypes.byref(w), None) == msd.MSD_ERR_INVALID


def test_the_timeout_hook_refuses_what_it_cannot_hold_back(lib):
    for codes, k, chunk in ((A, 64, -1), (A, 64, 2**31 - 1), (A + 4, 64, 0), (A, 72, 0)):
        w = msd.msd_weight4(codes, A, None, 8, k, 32)
        assert lib.msd_test_linear4_timeout(A, k, 1, 1, ctypes.byref(w), A, 8, chunk, None) == msd.MSD_ERR_INVALID
    assert lib.msd_test_linear4_timeout(A, 64, 1, 1, None, A, 8, 0, None) == msd.MSD_ERR_INVALID


def test_linear4_without_rows_or_weight(lib):
    assert linear(lib, m=0) == msd.MSD_OK
    assert lib.msd_linear4(A, 64, 1, 1, None, A, 8, 0, None) == msd.MSD_ERR_INVALID


@pytest.mark.parametrize("bad", [dict(x=None), dict(ld=63), dict(ld=66), dict(t=3), dict(x=A + 4), dict(v=A + 8), dict(ldv=60), dict(k=20)], ids=str)
def test_quantize4_refuses(lib, bad):
    a = dict(x=A, ld=64, t=msd.MSD_F32, k=64, v=A, ldv=64)
    a.update(bad)
    w = msd.msd_weight4(A, A, None, 8, a["k"], 32)
    assert lib.msd_quantize4(a["x"], a["ld"], a["t"], ctypes.byref(w), a["v"], a["ldv"], None) == msd.MSD_ERR_INVALID


@pytest.mark.parametrize("bad", [dict(x=None), dict(ld=99), dict(t=2), dict(rows=-1), dict(vocab=0), dict(vocab=393217, ld=400000), dict(u=None),
                                 dict(tokens=None), dict(probs=A, ldp=99), dict(x=A + 2), dict(probs=A + 1, ldp=100)], ids=str)
def test_sample_refuses(lib, bad):
    a = dict(x=A, ld=100, t=msd.MSD_F32, rows=2, vocab=100, u=A, tokens=A, probs=None, ldp=0)
    a.update(bad)
    assert lib.msd_sample(a["x"], a["ld"], a["t"], a["rows"], a["vocab"], None, a["u"], a["tokens"], None, a["probs"], a["ldp"],
                          None) == msd.MSD_ERR_INVALID


@pytest.mark.parametrize("bad", [dict(x=None), dict(ld=99), dict(t=5), dict(vocab=0), dict(nodes=0), dict(nodes=1025), dict(u=None), dict(depth=-1),
                                 dict(children=0), dict(children=257), dict(scratch=None), dict(path=None), dict(len_=None), dict(bonus=None),
                                 dict(tokens=None), dict(parent=None), dict(start=None), dict(n=-1), dict(rows=-1)], ids=str)
def test_accept_refuses(lib, bad):
    a = dict(x=A, ld=100, t=msd.MSD_F32, vocab=100, nodes=4, u=A, depth=2, children=3, scratch=A, path=A, len_=A, bonus=A, tokens=A, parent=A,
             start=A, n=2, rows=4)
    a.update(bad)
    b = msd.msd_batch(a["n"], A, a["start"], a["rows"])
    t = msd.msd_tree(a["tokens"], a["parent"], None, None, None)
    assert lib.msd_accept_batch(a["x"], a["ld"], a["t"], a["vocab"], ctypes.byref(b), ctypes.byref(t), a["nodes"], None, a["u"], a["depth"],
                                a["children"], a["scratch"], a["path"], a["len_"], a["bonus"], None) == msd.MSD_ERR_INVALID


@pytest.mark.parametrize("bad", [dict(rows=2**31 - 1), dict(rows=2**30 + 1), dict(n=2**31 - 1), dict(n=2**30 + 1)], ids=str)
def test_trees_whose_indices_would_pass_32_bits(lib, bad):
    """Rows are taken 1024 at a time, sequences halved and 32 at a time, in 32 bits."""
    a = dict(n=2, rows=4)
    a.update(bad)
    b = msd.msd_batch(a["n"], A, A, a["rows"])
    t = msd.msd_tree(A, A, None, None, None)
    assert lib.msd_accept_batch(A, 1, msd.MSD_BF16, 1, ctypes.byref(b), ctypes.byref(t), 4, None, A, 2, 3, A, A, A, A, None) == msd.MSD_ERR_INVALID


def test_nothing_to_do_needs_no_gpu(lib):
    assert lib.msd_sample(None, 0, 0, 0, 100, None, None, None, None, None, 0, None) == msd.MSD_OK
    b, t = msd.msd_batch(0, None, None, 0), msd.msd_tree()
    assert lib.msd_accept_batch(None, 0, 0, 100, ctypes.byref(b), ctypes.byref(t), 4, None, None, 2, 3, None, None, None, None, None) == msd.MSD_OK


def test_the_binding_refuses_host_tensors(lib):
    c, s = torch.zeros(4, 32, dtype=torch.uint8), torch.ones(4, 2, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        msd.Weight4(c, s, None, 32)
    with pytest.raises(ValueError):
        msd.Weight4.of(torch.zeros(4, 64))
    with pytest.raises(ValueError):
        msd.sample(torch.zeros(2, 10), torch.zeros(2), None, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        msd.Filter(temperature=torch.ones(2))
    assert msd.Filter().n is None


# weight_exp.cuh compiled for the host: single operations of fp32 are the same there (no contraction, fmaf exact)
SHIM = """
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#define __device__
#define __forceinline__ inline
struct float2 { float x, y; };
static float2 make_float2(float x, float y) { return {x, y}; }
static unsigned __float_as_uint(float f) { unsigned u; memcpy(&u, &f, 4); return u; }
static float __uint_as_float(unsigned u) { float f; memcpy(&f, &u, 4); return f; }
static float __fmul_rn(float a, float b) { return a * b; }
static float __fdiv_rn(float a, float b) { return a / b; }
"""
MAIN = """
int main() {
    static const msd::ExpTable table;
    const float2 *pairs = reinterpret_cast<const float2 *>(table.pair);
    const float temperatures[] = {1.f, 0.7f, 0.05f, 1e-3f, 3.f, 30.f, 1e4f, 0x1p-100f, 0x1p100f};
    double worst = 0;
    uint64_t seed = 1;
    for (float t : temperatures) {
        const float log2e = 1.44269504088896340736f, rest = (float)(1.44269504088896340736 - (double)log2e);
        msd::RowScale r;
        r.c_hi = __fdiv_rn(log2e, t);
        r.c_lo = __fdiv_rn(fmaf(-r.c_hi, t, log2e) + rest, t);
        for (int i = 0; i < 200000; ++i) {
            seed = seed * 6364136223846793005ull + 1442695040888963407ull;
            const double spread = 33.0 * (double)(seed >> 40) / (1 << 24);
            seed = seed * 6364136223846793005ull + 1442695040888963407ull;
            r.top = (float)(((double)(seed >> 40) / (1 << 24) - 0.5) * 60.0 * (t < 100.f ? t : 100.f));
            const float x = i % 16 == 0 ? r.top : (float)(r.top - spread * t);
            const long double want = ldexpl(expl(((long double)x - (long double)r.top) / (long double)t), msd::WEIGHT_BITS);
            const unsigned long long w = msd::weight_of(msd::exponent_of(x, r), pairs);
            if (i % 16 == 0 && w != 1ull << msd::WEIGHT_BITS) return puts("the largest is not 2^44"), 1;
            const double off = (double)fabsl((long double)w - want);
            if (off > worst) worst = off;
        }
    }
    printf("%.4f\\n", worst);
    return 0;
}
"""


def test_weights_are_exponentials_to_a_unit_or_two(tmp_path):
    """2^44 exp((logit - max) / T) of 1.8 million logits at 9 temperatures against long double: half a unit for rounding to an integer,
    and what the exponent (a pair of fp32 values) and the series leave, which weight_exp.cuh puts below another one and a half."""
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    text = open(os.path.join(os.path.dirname(msd.__file__), "csrc", "weight_exp.cuh")).read()
    text = re.sub(r'#pragma once|#include "common.cuh"', "", text)
    src = tmp_path / "weights.cpp"
    src.write_text(SHIM + text + MAIN)
    subprocess.run(["g++", "-O1", "-std=c++17", "-ffp-contract=off", str(src), "-o", str(tmp_path / "weights")], check=True)
    out = subprocess.run([str(tmp_path / "weights")], check=True, capture_output=True, text=True).stdout
    assert float(out) <= 2.0, out
