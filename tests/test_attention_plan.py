"""How attention calls are divided (csrc/attention_plan.h, compiled here for the host): the form that a shape runs, grids and workspaces
within their bounds at any sizes."""
import ctypes as C
import os
import random
import subprocess

import pytest

from paper_2408_06995_amd import binding as B

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2408_06995_amd", "csrc")

PROGRAM = r"""
#include <stdio.h>
#include "attention_plan.h"
using namespace fpq;
int main()
{
    long long b, hk, g, lq, lk, d;
    int type, causal;
    while (scanf("%lld %lld %lld %lld %lld %lld %d %d", &b, &hk, &g, &lq, &lk, &d, &type, &causal) == 8) {
        const AttentionPlan p = plan_attention(b, hk, g, lq, lk, d, type, causal);
        const Strides s = packed_strides(hk, lk, d);
        printf("%d %d %d %d %d %d %d %d %d %d %d %lld %lld %lld\n", p.q_pad, p.by_keys, p.waves, p.blocks, p.splits, p.q_waves, p.q_blocks, p.q_splits, p.k_waves, p.k_blocks, p.k_splits,
               (long long)s.b, (long long)s.t, (long long)s.h);
    }
    return 0;
}
"""
FP32, BF16 = 0, 1


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src, out = str(d / "plan.cpp"), str(d / "plan")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, src, "-o", out])

    def ask(calls):
        lines = subprocess.run([out], input="\n".join(" ".join(map(str, c)) for c in calls), capture_output=True, text=True, check=True).stdout.splitlines()
        names = "q_pad by_keys waves blocks splits q_waves q_blocks q_splits k_waves k_blocks k_splits stride_b stride_t stride_h".split()
        return [dict(zip(names, map(int, l.split()))) for l in lines]
    return ask


@pytest.mark.parametrize("call,expected", [
    # samples, key heads, heads of a group, queries, keys, dimension, type, causal
    ((16, 8, 4, 1, 4096, 128, BF16, 1), dict(by_keys=1, blocks=1, splits=4)),                   # single tokens over a long cache
    ((16, 8, 4, 1, 4096, 128, FP32, 1), dict(by_keys=1, blocks=1, splits=4)),
    ((1, 8, 1, 64, 64, 160, FP32, 0), dict(by_keys=1, blocks=1, splits=1)),                     # the smallest self-attention
    ((8, 8, 1, 4096, 77, 40, FP32, 0), dict(by_keys=0, waves=4, blocks=32, splits=1)),          # cross-attention
    ((4, 8, 1, 4096, 4096, 40, BF16, 0), dict(by_keys=0, waves=4, blocks=32, splits=1, q_splits=1, k_splits=1)),
    ((2, 8, 1, 1024, 1024, 80, FP32, 0), dict(by_keys=0, waves=4, blocks=8, splits=4, k_splits=2)),
    ((4, 4, 4, 1999, 1999, 128, BF16, 1), dict(by_keys=0, waves=4, q_pad=2048, splits=1, k_splits=4)),
    ((32, 8, 4, 32768, 32768, 128, FP32, 1), dict(by_keys=0, splits=1, q_splits=1, k_splits=1)),      # so many blocks balance by themselves
    ((1, 8, 1, 100, 100, 40, BF16, 0), dict(by_keys=1, q_waves=2, k_waves=2)),
])
def test_the_form_that_a_shape_runs(plan, call, expected):
    got = plan([call])[0]
    assert {k: got[k] for k in expected} == expected, got


def shapes(n):
    rng = random.Random(5)
    log = lambda lo, hi: int(round(2.0 ** rng.uniform(lo, hi)))
    out = []
    while len(out) < n:
        c = (log(0, 9), log(0, 6), rng.choice([1, 1, 2, 4, 7, 16]), log(0, 20), log(0, 20), rng.choice([8, 40, 64, 80, 96, 128, 160, rng.randint(1, 160)]),
             rng.choice([FP32, BF16]), rng.choice([0, 1]))
        if c[0] * c[1] * c[2] * (c[3] + 128) <= 2 ** 31:
            out.append(c)
    return out


def test_every_row_has_a_block_and_parts_are_few(plan):
    calls = shapes(4000)
    for c, p in zip(calls, plan(calls)):
        b, hk, g, lq, lk, d, type_, causal = c
        few = 32 if type_ == BF16 else 64
        assert p["blocks"] * (few if p["by_keys"] else 32 * p["waves"]) >= g * (lq if p["by_keys"] else p["q_pad"]), c
        assert lq <= p["q_pad"] <= 1.1 * lq and p["q_blocks"] * 32 * p["q_waves"] >= g * p["q_pad"] and p["k_blocks"] * 32 * p["k_waves"] >= lk, c
        for blocks, splits, most in ((p["blocks"], p["splits"], 1024), (p["q_blocks"], p["q_splits"], 1024), (p["k_blocks"], p["k_splits"], 1024 if type_ == FP32 else 2048)):
            assert 1 <= splits <= 32 and (splits == 1 or b * hk * blocks * splits <= most), c


def sizes(c):
    a = B.fpq_attention_args_t(type=c[6], causal=c[7], batch=c[0], kv_heads=c[1], q_heads=c[1] * c[2], q_len=c[3], kv_len=c[4], head_dim=c[5], scale=1.0)
    return B.lib().fpq_attention_workspace_size(C.byref(a)), B.lib().fpq_attention_backward_workspace_size(C.byref(a))


def test_workspaces_do_not_grow_with_parts():
    """Beyond the packed tensors and the rows' statistics, what is stated has a bound."""
    up = lambda n: -(-n // 256) * 256
    for c in shapes(4000) + [(1, 8, 4, 32768, 32768, 128, FP32, 0), (1, 8, 1, 16384, 16384, 128, FP32, 1), (1, 8, 4, 32768, 32768, 128, BF16, 1)]:
        b, hk, g, lq, lk, d, type_, _ = c
        row = -(-d // 8) * 8 * (6 if type_ == FP32 else 2)
        rows, keys = up(b * hk * g * lq * row), up(b * hk * lk * row)
        forward, backward = sizes(c)
        assert forward <= 2 * keys + 85e6, c
        assert backward <= 2 * keys + 2 * rows + b * hk * g * -(-lq // 32) * 256 + 420e6, c


@pytest.mark.parametrize("heads,keys,dim", [(4, 1 << 29, 8), (64, 1 << 30, 160), (2, (1 << 30) - 1, 5), (3, 7, 33)])
def test_strides_of_packed_keys(plan, heads, keys, dim):
    """heads x keys past 2^31 and past 2^32."""
    p, cols = plan([(2, heads, 1, 1, keys, dim, FP32, 0)])[0], -(-dim // 8) * 8
    assert (p["stride_b"], p["stride_t"], p["stride_h"]) == (heads * keys * cols, cols, keys * cols)
