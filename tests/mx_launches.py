"""The kernels that a microscaled product launches, without a GPU: libtpdq.so on the
stand-ins of launch_recorder.cpp, in a process of its own (as tests/launches.py).

A call is (op, fmt, dtype, M, N, K): op "gemm", "mlp" or "gated", of the MLP the first
product (its second has 8 outputs, which are left out)."""
from __future__ import annotations

import ctypes
import json
import os
import subprocess
import sys

from tests import launches

ROOT = launches.ROOT
X_AT, WS_AT, Y_AT, W_AT = (i << 44 for i in range(1, 5))
ANY_WS = (1 << 43) - 1


def record(calls, tmpdir):
    """[(launches of the product as (kernel with its template arguments, workgroups, threads))]"""
    launches.record([], tmpdir)  # builds the stand-ins
    r = subprocess.run([sys.executable, "-c", "from tests import mx_launches; mx_launches._serve()"], cwd=ROOT,
                       input=json.dumps({"so": os.path.join(tmpdir, "recorder.so"), "calls": calls}), capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return [[tuple(l) for l in c] for c in json.loads(r.stdout)]


def instance(product):
    """What a product is computed by: its kernel's instantiation, and whether K was split over workgroups."""
    return product[0][0], len(product) > 1


def _call(abi, lib, op, fmt, dtype, M, N, K):
    up = lambda a, b: -(-a // b)
    X = abi.Mx(X_AT, up(K, 128) * (64 if fmt == abi.MX_FP4 else 128), X_AT + (1 << 43), up(K, 512) * 16, M, K, fmt, abi.MX_ROWS)
    tiled = lambda i, R, K: abi.Mx(W_AT + (i << 41), up(K, 128) * 2048, W_AT + (i << 41) + (1 << 40), up(K, 512) * 512, R, K,
                                   abi.MX_FP4, abi.MX_TILED)
    b = ctypes.byref
    dt = abi.BF16 if dtype == "bf16" else abi.FP16
    if op == "gemm":
        st = lib.tpdq_mx_gemm(b(X), b(tiled(0, N, K)), dt, Y_AT, N, WS_AT, ANY_WS, None)
    else:
        gate = b(tiled(1, N, K)) if op == "gated" else None
        st = lib.tpdq_mx_mlp_shard(b(X), gate, b(tiled(0, N, K)), b(tiled(2, 8, N)), dt, Y_AT, WS_AT, ANY_WS, None)
    assert st == abi.OK, (op, fmt, dtype, M, N, K, lib.tpdq_last_error())
    done = [(l["kernel"], l["grid"][0], l["block"]) for l in json.loads(lib._recorder.recorder_take().decode())]
    if op != "gemm":  # the second product, and its reduction where it is split
        second = 1 if "k_mx_reduce" not in done[-1][0] or "true>" in done[-1][0].replace(" ", "") else 2
        done = done[:-second]
    return done


def _serve():
    req = json.load(sys.stdin)
    rec = ctypes.CDLL(req["so"], mode=ctypes.RTLD_GLOBAL)
    rec.recorder_take.restype = ctypes.c_char_p
    from paper_2402_04925_amd import _abi
    lib = _abi._declare(ctypes.CDLL(os.path.join(ROOT, "paper_2402_04925_amd", "libtpdq.so")))
    lib._recorder = rec
    print(json.dumps([_call(_abi, lib, *c) for c in req["calls"]]))
