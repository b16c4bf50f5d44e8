"""The kernels that the GPU tests of the microscaled products reach, from recorded launches (no GPU)."""
import os
import random

import pytest

from paper_2402_04925_amd import _abi
from tests import mx_launches, test_gpu_mx_routes as t

if not os.path.exists(_abi.LIB_PATH):
    from paper_2402_04925_amd import build
    build.build()


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("recorder"))
    return lambda calls: mx_launches.record(calls, d)


def reached(record, calls):
    return {mx_launches.instance(p) for p in record(calls)}


# rows: 1 to 16, to 32 and to 64 of them, each in whole and (16-bit outputs) in half tiles; tiles: six shapes (the gated
# product five), each with and without K split
@pytest.mark.parametrize("op,dtypes,each", [("gemm", t.DTS, 2 * 3 + 6 * 2), ("mlp", ["fp16"], 3 + 6 * 2), ("gated", ["fp16"], 3 + 5 * 2)])
def test_every_kernel_is_tested(record, op, dtypes, each):
    for dt in dtypes:
        for fmt in t.FMTS:
            got = reached(record, [(op, fmt, dt, *s) for s in t.ROUTES])
            assert len(got) == each, sorted(got)


def test_random_products_run_on_tested_kernels(record):
    rng = random.Random(1)
    size = lambda lo, hi, step: max(step, round(lo * (hi / lo) ** rng.random() / step) * step)
    ops = [("gemm", "fp16"), ("gemm", "bf16"), ("mlp", "fp16"), ("gated", "fp16")]
    calls = []
    for _ in range(4000):
        step = rng.choice([8, 8, 128])
        op, dt = rng.choice(ops)
        calls.append((op, rng.choice(t.FMTS), dt, size(1, rng.choice([64, 4096]), 1), size(8, 32768, step), size(8, 32768, step)))
    tested = reached(record, [(op, fmt, dt, *s) for op, dt in ops for fmt in t.FMTS for s in t.ROUTES])
    assert reached(record, calls) <= tested


def test_reductions_follow_splits(record):
    """Recorded as (product, reduction); every other product is one launch."""
    for p in record([("gemm", fmt, dt, *s) for fmt in t.FMTS for dt in t.DTS for s in t.ROUTES]):
        assert len(p) == 1 or len(p) == 2 and p[1][0].startswith("k_mx_reduce")
