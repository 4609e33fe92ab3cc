"""The 8-bit linear without a GPU: the refusals of its C ABI, which kernel and which split over K it runs, and the oracle's
own pins.  No call here reaches a kernel launch."""
import ctypes
import os
import re
import shutil
import subprocess
from fractions import Fraction

import numpy as np
import pytest

import w8_cases
from oracle import hadamard, quant, w8
from paper_2606_02823_amd import qift
from test_kernel_resources import kernels

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_02823_amd", "csrc")
OK, E_NULL, E_SHAPE, E_SPEC, E_FORMAT, E_ALIGN, E_WS = 0, -1, -2, -3, -4, -6, -8
A = 0x10000       # a 16-byte aligned fake device address (never dereferenced)
MIS = 0x10008


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(qift.LIB_PATH):
        pytest.skip("libqift.so not built")
    return qift.lib()


def test_every_declared_symbol_is_exported(L):
    text = open(os.path.join(ROOT, "include", "qift_w8.h")).read()
    names = set(re.findall(r"\b(qift_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert names == set(qift.W8_EXPORTS)
    for n in names:
        assert hasattr(L, n), n
    assert ctypes.sizeof(qift.W8C) == 32


def test_quantizers_refuse(L):
    def wq(W=A, N=4, K=256, block=64, flags=0, lv=A, sc=A):
        return L.qift_quantize_weights8(W, N, qift.HadamardSpec(K, block, flags), lv, sc, None)

    def aq(x=A, M=4, K=256, block=64, flags=0, q=A, sc=A):
        return L.qift_rotate_quant_act8(x, M, qift.HadamardSpec(K, block, flags), q, sc, None)

    for f in (wq, aq):
        for kw in ({"K": 0}, {"K": 96}, {"K": 65536}):
            assert f(**kw) == E_SHAPE, kw
        for kw in ({"block": 0}, {"block": 3}, {"block": 1}, {"block": 512}, {"block": 16384, "K": 16384}):
            assert f(**kw) == E_SPEC, kw
    for kw in ({"W": None}, {"lv": None}, {"sc": None}):
        assert wq(**kw) == E_NULL
    for kw in ({"x": None}, {"q": None}, {"sc": None}):
        assert aq(**kw) == E_NULL
    assert wq(N=0) == wq(K=16384 + 64) == wq(N=2 ** 23) == wq(N=2 ** 24, K=64) == E_SHAPE
    assert aq(M=0) == aq(M=2 ** 31) == aq(M=2 ** 23) == E_SHAPE
    assert wq(block=8192, K=8192) == E_SPEC and wq(flags=qift.SPEC_BF16) == E_SPEC
    for flags in (1 << 17, qift.clip_flags(0, 4), qift.clip_flags(5, 4), qift.clip_flags(4, 17), -1):
        assert aq(flags=flags) == E_SPEC
    for kw in ({"W": MIS}, {"lv": MIS}, {"sc": MIS}):
        assert wq(**kw) == E_ALIGN
    for kw in ({"x": MIS}, {"q": MIS}, {"sc": MIS}):
        assert aq(**kw) == E_ALIGN


def test_linear_refuses(L):
    def f(N=512, K=256, lv=A, sw=A, q=A, sx=A, M=4, dt=0, out=A, acc=None, ws=None, nb=0):
        w = qift.W8C(N, K, lv, sw)
        return L.qift_w8a8_linear(ctypes.byref(w), q, sx, M, dt, out, acc, ws, nb, None)

    assert L.qift_w8a8_linear(None, A, A, 4, 0, A, None, None, 0, None) == E_NULL
    for kw in ({"lv": None}, {"sw": None}, {"q": None}, {"sx": None}, {"out": None}):
        assert f(**kw) == E_NULL
    for dt in (-1, 3):
        assert f(dt=dt) == E_FORMAT
    for kw in ({"N": 0}, {"N": 2 ** 31}, {"K": 0}, {"K": 32}, {"K": 131072 + 64}, {"M": 0}, {"M": -1}, {"M": 2 ** 31},
               {"N": 2 ** 24, "M": 2 ** 12}):
        assert f(**kw) == E_SHAPE, kw
    for kw in ({"lv": MIS}, {"sw": MIS}, {"q": MIS}, {"sx": MIS}, {"out": MIS}, {"acc": MIS}):
        assert f(**kw) == E_ALIGN, kw
    need = L.qift_w8a8_workspace_bytes(ctypes.byref(qift.W8C(4096, 14336, A, A)), 300)
    assert need > 0
    big = {"N": 4096, "K": 14336, "M": 300}
    assert f(**big, ws=A, nb=need - 1) == E_WS and f(**big, ws=None, nb=need) == E_WS
    assert f(**big, ws=MIS, nb=need) == E_ALIGN


def test_workspace_query_of_unsupported_shapes(L):
    q = lambda N, K, M: L.qift_w8a8_workspace_bytes(ctypes.byref(qift.W8C(N, K, A, A)), M)  # noqa: E731
    assert q(0, 256, 100) == q(512, 100, 100) == q(512, 256, 0) == q(512, 1 << 20, 100) == 0
    assert q(4096, 4096, 1) == 0
    assert L.qift_w8a8_workspace_bytes(None, 4) == 0


PROBE = """
#include <cstdio>
#include "qift_w8_route.h"
using namespace qift::route;
int main() {
  long N, M, K;
  while (std::scanf("%ld %ld %ld", &N, &M, &K) == 3) {
    const W8Plan p = w8_plan(N, M, K, true), u = w8_plan(N, M, K, false);
    std::printf("%d %d %d %d %zu %d %d\\n", p.rows, p.bn, p.bm, p.parts, w8_workspace(p, N, M), u.parts, u.rows ? u.rows : u.bm);
  }
}
"""


def test_plan_limits(tmp_path):
    """Every part has a step at least, the parts' sums fit the query, and the second launch's grid has its limit."""
    cxx = shutil.which("g++") or shutil.which("clang++") or "/opt/rocm/llvm/bin/clang++"
    (tmp_path / "probe.cpp").write_text(PROBE)
    subprocess.run([cxx, "-std=c++17", "-I", CSRC, str(tmp_path / "probe.cpp"), "-o", str(tmp_path / "probe")], check=True)
    sizes = [(N, M, K) for N in (1, 63, 64, 129, 1024, 4096, 4099, 28672, 131072) for M in (1, 17, 24, 64, 65, 128, 333, 1024, 4096, 70000)
             for K in (64, 128, 256, 1088, 4096, 14336, 131072)]
    out = subprocess.run([str(tmp_path / "probe")], input="".join("%d %d %d\n" % s for s in sizes), text=True,
                         capture_output=True, check=True).stdout.splitlines()
    seen = set()
    for (N, M, K), line in zip(sizes, out):
        rows, bn, bm, parts, ws, unsplit, kind = (int(v) for v in line.split())
        assert unsplit == 1 and kind > 0
        assert 1 <= parts <= (K + 127) // 128
        if rows:
            assert rows % 4 == 0 and 4 <= rows <= (32 if M <= 16 else 64) and M <= 32 and parts == 1
        else:
            assert (bn, bm) in ((128, 32), (128, 64), (256, 128), (256, 256)) and (bm > 32 or M <= 32)
        assert ws == (0 if parts == 1 else parts * M * ((N + 3) // 4 * 4) * 4) and (parts == 1 or M <= 65535)
        seen.add((-(-rows // 16) * 16, bm, parts > 1))
    assert {(16, 0, False), (32, 0, False), (64, 0, False), (0, 32, False), (0, 64, True), (0, 128, False), (0, 256, False)} <= seen


@pytest.mark.parametrize("name,count", [("k_w8_rows", 18), ("k_w8_gemm", 16), ("k_w8_sum", 3)])
def test_no_spills(name, count):
    ks = {k: v for k, v in kernels(qift.LIB_PATH).items() if f"{len(name)}{name}I" in k}
    assert len(ks) == count
    assert not {k for k, v in ks.items() if v[".vgpr_spill_count"] or v[".private_segment_fixed_size"]}
    if name == "k_w8_gemm":   # the large tiles: a workgroup to a CU; the others leave room for two
        assert all(v[".group_segment_fixed_size"] <= (81920 if "ILi1E" in k else 163840) for k, v in ks.items())


WAITS = """
#include <cstdio>
#include "qift_waits.h"
using namespace qift::waits;
int main() {
  int NS, L;
  while (std::scanf("%d %d", &NS, &L) == 2) std::printf("%d %d %d\\n", w8_first(L), w8_prologue(NS, L), w8_handover(NS, L));
}
"""


def test_counted_waits(tmp_path):
    """The loads sent in the tiled product's order: where a step hands its buffer over, the next step's have all landed, and what
    goes into a buffer goes there after every wave has passed the barrier behind its last read of it."""
    cxx = shutil.which("g++") or shutil.which("clang++") or "/opt/rocm/llvm/bin/clang++"
    (tmp_path / "probe.cpp").write_text(WAITS)
    subprocess.run([cxx, "-std=c++17", "-I", CSRC, str(tmp_path / "probe.cpp"), "-o", str(tmp_path / "probe")], check=True)
    cases = [(3, 5), (3, 3), (3, 6), (2, 8)]
    out = subprocess.run([str(tmp_path / "probe")], input="".join("%d %d\n" % c for c in cases), text=True, capture_output=True,
                         check=True).stdout.splitlines()
    for (NS, L), line in zip(cases, out):
        first, prologue, handover = (int(v) for v in line.split())
        for steps in range(1, 12):
            sent, landed, done = [], 0, -1

            def send(k, n):
                assert k - NS <= done, (NS, L, k)                    # the step whose buffer this was has handed it over
                sent.extend([k] * n)

            for k in range(NS - 1):
                send(k, L)
            send(NS - 1, first)
            landed = max(landed, len(sent) - prologue)
            for k in range(-(-steps // NS) * NS):
                assert sent[:landed].count(k) == L, (NS, L, k)       # step k's tiles are there when it reads them
                send(k + NS - 1, L - first)
                landed = max(landed, len(sent) - handover)
                assert sent[:landed].count(k + 1) == L
                done = k
                send(k + NS, first)
            assert 0 <= handover <= prologue < 64


def test_oracle_codes_are_the_rationals():
    rng = np.random.default_rng(3)
    X = np.concatenate([rng.normal(0, 1, (3, 16)), rng.integers(-254, 255, (4, 16)) * 0.5, np.zeros((1, 16))])
    X[4, 0] = 127.0   # halves of whole steps: exact ties
    for clip in ((1, 1), (9, 10), (1, 16)):
        q = w8.codes(X, clip)
        for m in range(len(X)):
            a = max(abs(Fraction(float(v))) for v in X[m])
            for k in range(16):
                if a == 0:
                    assert q[m, k] == 0
                    continue
                r = 127 * clip[1] * abs(Fraction(float(X[m, k]))) / (clip[0] * a)
                want = min(round(r), 127)   # Fraction rounds half to even
                assert q[m, k] == (-want if X[m, k] < 0 else want)


def test_oracle_scales_and_error_bound():
    """|X - s sqrt(b) q| is at most half a step (no clipping), and quantized weights are within half a stored step."""
    rng = np.random.default_rng(4)
    x = rng.normal(0, 1, (3, 256)).astype(np.float16)
    q, s = w8.act_quant8(x, 64)
    X = hadamard.rotate_act_units(x, 64) * 2.0 ** -24
    step = s.astype(np.float64)[:, None] * 8.0
    assert np.all(np.abs(X - step * q) <= step * (0.5 + 127 * 2.0 ** -24)) and np.abs(q).max() == 127
    W = hadamard.rotate_weights(rng.normal(0, 0.02, (5, 256)), 64)
    L, sw = w8.quantize_weights8(W)
    d = sw.astype(np.float64)[:, None]
    assert np.all(np.abs(W - d * L) <= d * (0.5 + 127 * 2.0 ** -11))
    assert np.array_equal(w8.epilogue(np.array([[3]]), np.array([0.5]), np.array([2.0])), [[np.float32(3.0)]])
    assert quant.rne(np.array([2.5]))[0] == 2


KERNEL = """
#include <cstdio>
#include "qift_w8_route.h"
using namespace qift::route;
int main() {
  long N, M, K;
  while (std::scanf("%ld %ld %ld", &N, &M, &K) == 3) {
    const W8Plan p = w8_plan(N, M, K, true);
    if (!p.rows) std::printf("%dx%d:%d\\n", p.bn, p.bm, p.parts);
    else if (M <= 16) std::printf("rows %dx1x%d:1\\n", p.rows > 16 ? 2 : 1, p.rows <= 16 && w8_eight_waves(p, N, K) ? 8 : 4);
    else std::printf("rows %dx2x4:1\\n", p.rows > 32 ? 4 : p.rows > 16 ? 2 : 1);
  }
}
"""


def test_each_kernel_has_its_sizes(tmp_path):
    """The sizes that the GPU tests run take the kernels that they are there for: every rows kernel, every tile uncut and cut, the
    tiles with ragged sides and with K of an odd number of 64s among the uncut ones."""
    cxx = shutil.which("g++") or shutil.which("clang++") or "/opt/rocm/llvm/bin/clang++"
    (tmp_path / "probe.cpp").write_text(KERNEL)
    subprocess.run([cxx, "-std=c++17", "-I", CSRC, str(tmp_path / "probe.cpp"), "-o", str(tmp_path / "probe")], check=True)
    out = subprocess.run([str(tmp_path / "probe")], input="".join(f"{N} {M} {K}\n" for M, N, K, _, _ in w8_cases.CASES), text=True,
                         capture_output=True, check=True).stdout.splitlines()
    assert len(out) == len(w8_cases.CASES)
    for (M, N, K, name, parts), got in zip(w8_cases.CASES, out):
        assert got == f"{name}:{parts}", (M, N, K)
    for rows in w8_cases.ROWS:
        assert any(c[3] == "rows " + rows for c in w8_cases.CASES), rows
    for tile in w8_cases.TILES:
        bn, bm = (int(v) for v in tile.split("x"))
        whole, cut = ([c for c in w8_cases.CASES if c[3] == tile and (c[4] > 1) == split] for split in (False, True))
        assert whole and cut, tile
        assert any(c[1] % bn and c[0] % bm for c in whole) and any(c[1] % bn and c[0] % bm for c in cut), tile
        assert any(c[2] % 128 == 64 for c in whole), tile


def test_workspace_of_several_numbers_of_tokens(L):
    """The largest step's need is not enough for every smaller one; that of all of them is."""
    w = object.__new__(qift.W8)
    w.c = qift.W8C(4096, 11008, A, A)
    w._ref = ctypes.byref(w.c)
    each = [qift.w8a8_workspace_bytes(w, M) for M in range(1, 513)]
    assert each[511] < max(each) and qift.w8a8_workspace_bytes(w, range(1, 513)) == max(each)
    assert qift.w8a8_workspace_bytes(w, [333]) == each[332] and qift.w8a8_workspace_bytes(w, ()) == 0
