"""A serving step's calls without a GPU: the arithmetic of csrc/qift_step.h (a program compiled from that header), the
refusals of the C ABI, and the oracle's own pins.  No call here reaches a kernel launch."""
import ctypes
import os
import re
import shutil
import subprocess
from fractions import Fraction

import numpy as np
import pytest

from oracle import step as ostep
from paper_2606_02823_amd import qift
from test_kernel_resources import kernels

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_02823_amd", "csrc")
OK, E_NULL, E_SHAPE, E_SPEC, E_FORMAT, E_ALIGN = 0, -1, -2, -3, -4, -6
A, B_ = 0x10000, 0x20000   # aligned fake device addresses (never dereferenced)
MIS = 0x10008
I31 = 2 ** 31 - 1

PROBE = r"""
#include <cstdio>
#include <cstring>
#include "qift_step.h"
using namespace qift;
int main() {
  char what[16];
  while (std::scanf("%15s", what) == 1) {
    if (!std::strcmp(what, "ask")) {
      int len, n, page, width;
      std::scanf("%d %d %d %d", &len, &n, &width, &page);
      const step::Ask a = step::ask(len, n, (long long)width * page, pages::make_div((unsigned)page));
      std::printf("%d %d %d %d %d %d\n", a.len, a.n, a.held, a.need, (int)a.fits, (int)a.bad);
    } else if (!std::strcmp(what, "taken")) {
      int len, n, page, width, start, base, rows, depth;
      std::scanf("%d %d %d %d %d %d %d %d", &len, &n, &width, &page, &start, &base, &rows, &depth);
      const step::Ask a = step::ask(len, n, (long long)width * page, pages::make_div((unsigned)page));
      std::printf("%d\n", (int)step::taken(a, start, base, rows, depth));
    } else if (!std::strcmp(what, "slot")) {
      int entry, at, page;
      std::scanf("%d %d %d", &entry, &at, &page);
      std::printf("%d\n", step::slot_of(entry, (unsigned)at, (unsigned)page));
    } else if (!std::strcmp(what, "head")) {
      int h, q, k;
      std::scanf("%d %d %d", &h, &q, &k);
      const step::Head a = step::head_of(h, q, k);
      std::printf("%d %d %d\n", a.own, (int)a.have, (int)a.key);
    } else {
      int count, at, s[257];
      std::scanf("%d %d", &count, &at);
      for (int i = 0; i <= count; ++i) std::scanf("%d", s + i);
      std::printf("%d\n", step::find(s, count, at));
    }
  }
}
"""


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(qift.LIB_PATH):
        pytest.skip("libqift.so not built")
    return qift.lib()


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("clang++") or "/opt/rocm/llvm/bin/clang++"
    d = tmp_path_factory.mktemp("step")
    (d / "probe.cpp").write_text(PROBE)
    subprocess.run([cxx, "-std=c++17", "-I", CSRC, str(d / "probe.cpp"), "-o", str(d / "probe")], check=True)

    def ask(lines):
        out = subprocess.run([str(d / "probe")], input="\n".join(lines) + "\n", text=True, capture_output=True, check=True).stdout
        return [[int(v) for v in line.split()] for line in out.splitlines()]
    return ask


def test_what_a_sequence_asks_for(probe):
    cases = [(len_, n, width, page) for page in (16, 48, 128) for width in (1, 3, I31 // page)
             for len_ in (-5, 0, 1, page - 1, page, page + 1, 3 * page, width * page, I31) for n in (-1, 0, 1, 17, page, I31)]
    for (len_, n, width, page), got in zip(cases, probe([f"ask {a} {b} {c} {d}" for a, b, c, d in cases])):
        room = width * page
        have, new = min(max(len_, 0), room), max(n, 0)
        fits = 0 <= len_ <= room and have + new <= room
        need = -(-(have + new) // page) - -(-have // page) if fits else 0
        bad = n < 0 or not 0 <= len_ <= room or (new > 0 and not fits)
        assert got == [have, new, -(-have // page), need, fits, bad], (len_, n, width, page)


def test_slots_and_search(probe):
    cases = [(-1, 0, 16), (0, 15, 16), (5, 3, 48), (I31 // 16, 15, 16), (I31 // 16 + 1, 0, 16), (I31, 127, 128), (-(2 ** 31), 3, 256)]
    for (e, at, page), got in zip(cases, probe([f"slot {a} {b} {c}" for a, b, c in cases])):
        s = e * page + at
        assert got == [s if e >= 0 and s <= I31 else -1]
    rng = np.random.default_rng(2)
    lines, want = [], []
    for _ in range(200):
        n = rng.integers(0, 3, 256) * rng.integers(0, 9, 256)
        s = np.concatenate([[0], np.cumsum(n)])
        if s[-1] == 0:
            continue
        at = int(rng.integers(0, s[-1]))
        lines.append(f"find 256 {at} " + " ".join(map(str, s)))
        want.append([int(np.searchsorted(s, at, side="right")) - 1])
    assert probe(lines) == want


def test_heads_of_a_wave(probe):
    """Every head that a wave touches is one that is there, without query or key heads too."""
    cases = [(h, q, k) for q, k in ((1, 0), (0, 1), (5, 0), (0, 4), (3, 1), (32, 8), (7, 0), (0, 6)) for h in range(-(-(q + k) // 16) * 16)]
    for (h, q, k), (own, have, key) in zip(cases, probe([f"head {a} {b} {c}" for a, b, c in cases])):
        assert 0 <= own < (k if key else q) and have == (h < q + k)
        if have:
            assert (bool(key), own) == ((h >= q), h - q if h >= q else h)


def test_every_declared_symbol_is_exported(L):
    text = open(os.path.join(ROOT, "include", "qift_step.h")).read()
    names = set(re.findall(r"\b(qift_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert names == set(qift.STEP_EXPORTS)
    for n in names:
        assert hasattr(L, n), n
    assert ctypes.sizeof(qift.HeadRopeC) == 16 + 3 * 8
    assert not set(qift.STEP_EXPORTS) & set(qift.EXPORTS + qift.PAGES_EXPORTS + qift.W8_EXPORTS)


def test_plan_refusals(L):
    def f(lens=A, counts=A, B=4, table=A, width=8, page=64, free=A, depth=A, cap=100, rows=7, starts=A, lo=B_, slots=A, pos=A,
          do=B_):
        return L.qift_kv4_plan_step(lens, counts, B, table, width, page, free, depth, cap, rows, starts, lo, slots, pos, do, None)

    for kw in ({"B": -1}, {"B": 65536}, {"width": 0}, {"page": 0}, {"page": 24}, {"page": -16}, {"width": 2 ** 25}, {"cap": -1},
               {"cap": 2 ** 31}, {"rows": -1}, {"rows": 2 ** 31}, {"lo": A}, {"do": A}):
        assert f(**kw) == E_SHAPE, kw
    for kw in ({"lens": None}, {"counts": None}, {"table": None}, {"free": None}, {"depth": None}, {"starts": None}, {"lo": None},
               {"slots": None}, {"pos": None}, {"do": None}):
        assert f(**kw) == E_NULL, kw
    for name in ("lens", "counts", "table", "free", "depth", "starts", "lo", "slots", "pos", "do"):
        assert f(**{name: 0x10002}) == E_ALIGN, name


def test_release_refusals(L):
    def f(lens=A, done=A, B=4, table=A, width=8, page=64, free=A, depth=A, cap=100, lo=B_, do=B_):
        return L.qift_kv4_release(lens, done, B, table, width, page, free, depth, cap, lo, do, None)

    for kw in ({"B": -1}, {"B": 65536}, {"width": 0}, {"page": 24}, {"width": 2 ** 25}, {"cap": -1}, {"lo": A}, {"do": A}):
        assert f(**kw) == E_SHAPE, kw
    for kw in ({"lens": None}, {"done": None}, {"table": None}, {"free": None}, {"depth": None}, {"lo": None}, {"do": None}):
        assert f(**kw) == E_NULL, kw
    for name in ("lens", "done", "table", "free", "depth", "lo", "do"):
        assert f(**{name: 0x10002}) == E_ALIGN, name


def test_rope_refusals(L):
    def f(head=128, rot=128, pairs=0, eps=1e-5, freq=A, qw=None, kw=None, q=A, qs=4096, k=B_, ks=1024, dt=0, pos=A, rows=3, Hq=32,
          Hkv=8, qo=A, qos=4096, ko=B_, kos=1024):
        r = qift.HeadRopeC(head, rot, pairs, eps, freq, qw, kw)
        return L.qift_head_norm_rope(ctypes.byref(r), q, qs, k, ks, dt, pos, rows, Hq, Hkv, qo, qos, ko, kos, None)

    assert L.qift_head_norm_rope(None, A, 4096, A, 1024, 0, A, 3, 32, 8, A, 4096, A, 1024, None) == E_NULL
    assert f(dt=2) == f(dt=-1) == E_FORMAT
    for kw in ({"head": 64}, {"rot": -8}, {"rot": 12}, {"rot": 136}, {"rows": -1}, {"Hq": -1}, {"Hkv": -1}, {"Hq": 0, "Hkv": 0},
               {"Hq": 65536}, {"qs": 4088}, {"ks": 1016}, {"qos": 4088}, {"kos": 1016}, {"qs": 2 ** 31}, {"rows": 2 ** 26},
               {"rows": 2 ** 23}, {"qos": 4104}, {"kos": 2048}, {"qo": B_}, {"ko": A}, {"qo": 0x40000, "ko": 0x40000}):
        assert f(**kw) == E_SHAPE, kw
    for kw in ({"pairs": 2}, {"pairs": -1}, {"eps": 0.0}, {"eps": 2.0 ** -81}, {"eps": -1e-5}, {"eps": float("inf")}, {"eps": float("nan")}):
        assert f(**kw) == E_SPEC, kw
    for kw in ({"freq": None}, {"q": None}, {"k": None}, {"pos": None}, {"qo": None}, {"ko": None}):
        assert f(**kw) == E_NULL, kw
    for kw in ({"freq": MIS}, {"qw": MIS}, {"kw": MIS}, {"q": MIS}, {"k": MIS}, {"qo": MIS}, {"ko": MIS}, {"pos": 0x10002},
               {"qs": 4100, "qos": 4100}, {"ks": 1028, "kos": 1028}, {"qo": 0x40000, "qos": 4100}, {"ko": 0x40000, "kos": 1028}):
        assert f(**kw) == E_ALIGN, kw
    assert f(rows=0) == OK and f(rows=0, q=None, pos=None) == OK


@pytest.mark.parametrize("name,count", [("k_plan", 1), ("k_release", 1), ("k_rope", 12)])
def test_no_spills(name, count):
    ks = {k: v for k, v in kernels(qift.LIB_PATH).items() if f"{len(name)}{name}" in k}
    assert len(ks) == count
    assert not {k for k, v in ks.items() if v[".vgpr_spill_count"] or v[".private_segment_fixed_size"]}


def test_oracle_plan():
    """One short step by hand, and what a whole run of steps and releases keeps: no page twice, every token in its place."""
    table = np.array([[7, -1, -1], [9, 4, -1]], np.int32)
    free = np.array([1, 2, 3, 0, 0], np.int32)
    got = ostep.plan(np.array([16, 20]), np.array([2, 13]), table, free, 3, 16, 20)
    assert list(got[0]) == [0, 2, 15] and list(got[1]) == [18, 33] and got[2].tolist() == [[7, 3, -1], [9, 4, 2]]
    assert list(got[3][:5]) == [48, 49, 68, 69, 70] and got[3][14] == 32 and list(got[3][15:]) == [-1] * 5
    assert list(got[4][:3]) == [16, 17, 20] and got[5] == 1 and got[6] is False
    rng = np.random.default_rng(1)
    B, width, page, pages = 6, 5, 16, 20
    lens, table, free, depth = np.zeros(B, np.int32), np.full((B, width), -1, np.int32), np.arange(pages, dtype=np.int32), pages
    for _ in range(60):
        counts = rng.integers(0, 12, B).astype(np.int32)
        starts, lens, table, slots, pos, depth, bad = ostep.plan(lens, counts, table, free, depth, page, 80)
        live = [int(p) for b in range(B) for p in table[b, :-(-int(lens[b]) // page)]]
        assert sorted(live + [int(p) for p in free[:depth]]) == list(range(pages))
        done = (rng.random(B) < 0.2) | (lens > 60)
        lens, free, depth, bad = ostep.release(lens, done.astype(np.int32), table, free, depth, page)
        assert not bad


def test_oracle_plan_where_pages_run_out():
    """A sequence that needs no page takes none, whatever those before it asked for; no page is lost or had twice."""
    table, free = np.array([[-1] * 10, [6] + [-1] * 9], np.int32), np.arange(5, dtype=np.int32)
    got = ostep.plan(np.array([0, 1]), np.array([160, 1]), table, free, 5, 16, 170)
    assert list(got[1]) == [0, 2] and got[3][160] == 97 and got[5] == 5 and got[6]
    rng = np.random.default_rng(3)
    B, width, page, pages, short = 8, 5, 16, 14, 0
    lens, table, free, depth = np.zeros(B, np.int32), np.full((B, width), -1, np.int32), np.arange(pages, dtype=np.int32), pages
    for _ in range(200):
        counts = rng.integers(0, 20, B).astype(np.int32)
        _, lens, table, _, _, depth, bad = ostep.plan(lens, counts, table, free, depth, page, 100)
        short += bad
        live = [int(p) for b in range(B) for p in table[b, :-(-int(lens[b]) // page)]]
        assert sorted(live + [int(p) for p in free[:depth]]) == list(range(pages))
        done = (rng.random(B) < 0.1) | (lens > 60)
        lens, free, depth, bad = ostep.release(lens, done.astype(np.int32), table, free, depth, page)
        assert not bad
    assert 20 < short < 200


def test_pages_taken_up_to_a_sequence(probe):
    """The largest of these over the sequences is what the oracle takes."""
    rng = np.random.default_rng(8)
    lines, want, sizes = [], [], []
    for _ in range(60):
        B, width, page = int(rng.integers(1, 9)), 5, 16
        lens, counts = rng.integers(0, 70, B), rng.integers(0, 30, B)
        rows, depth = int(rng.integers(0, counts.sum() + 2)), int(rng.integers(0, 20))
        start = base = 0
        for n, c in zip(lens, counts):
            lines.append(f"taken {n} {c} {width} {page} {start} {base} {rows} {depth}")
            start += int(c)
            base += -(-(n + c) // page) - -(-n // page) if n + c <= width * page else 0
        sizes.append(B)
        want.append(depth - ostep.plan(lens, counts, np.zeros((B, width), np.int32), np.zeros(depth, np.int32), depth, page, rows)[5])
    got = iter(v for v, in probe(lines))
    assert [max(next(got) for _ in range(n)) for n in sizes] == want


def test_oracle_rotation():
    """It keeps the length of each pair, positions add up, and position 0 leaves the normed head as it is."""
    rng = np.random.default_rng(5)
    x, w = rng.normal(0, 2, (4, 3, 128)), rng.normal(1, 0.1, 128)
    freq = (1e4 ** (-np.arange(48) / 48)).astype(np.float32)
    for pairs in (False, True):
        y, _ = ostep.head_norm_rope(x, w, 1e-6, freq, np.array([0, 5, 1000, -1]), 96, pairs)
        n = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + np.float64(np.float32(1e-6))) * w
        assert np.allclose(y[0], n[0], rtol=1e-14) and np.all(y[3] == 0)
        assert np.allclose((y[1:3] ** 2).sum(-1), (n[1:3] ** 2).sum(-1)) and np.array_equal(y[1, :, 96:], n[1, :, 96:])
        z, _ = ostep.head_norm_rope(y[1:2], None, 1e-6, freq, np.array([995]), 96, pairs)
        direct, _ = ostep.head_norm_rope(x[1:2], w, 1e-6, freq, np.array([1000]), 96, pairs)
        assert np.allclose(z, direct, atol=1e-12)


def _apart(call, sizes, outputs):
    """call with every array in a place of its own, then each output laid over each other array, at its first entry and at its last."""
    at, place = 0x100000, {}
    for name, n in sizes.items():
        place[name] = at
        at += 4 * n + 4096
    for out in outputs:
        for name in sizes:
            if name == out:
                continue
            for move in (place[name], place[name] + 4 * (sizes[name] - 1), place[name] - 4 * (sizes[out] - 1)):
                assert call({**place, out: move}) == E_SHAPE, (out, name, move - place[name])


def test_outputs_lie_apart(L):
    """Every workgroup reads the inputs afresh and nothing orders the outputs: no output may overlap another array."""
    B, width, cap, rows = 300, 3, 70, 900

    def plan(p):
        return L.qift_kv4_plan_step(p["lens"], p["counts"], B, p["table"], width, 16, p["free"], p["depth"], cap, rows, p["starts"],
                                    p["lens_out"], p["slots"], p["positions"], p["free_out"], None)

    def release(p):
        return L.qift_kv4_release(p["lens"], p["done"], B, p["table"], width, 16, p["free"], p["depth"], cap, p["lens_out"],
                                  p["free_out"], None)

    _apart(plan, {"lens": B, "counts": B, "table": B * width, "free": cap, "depth": 1, "starts": B + 1, "lens_out": B, "slots": rows,
                     "positions": rows, "free_out": 1}, ("table", "starts", "lens_out", "slots", "positions", "free_out"))
    _apart(release, {"lens": B, "done": B, "table": B * width, "free": cap, "depth": 1, "lens_out": B, "free_out": 1},
           ("free", "lens_out", "free_out"))


TURN = r"""
#include <cstdio>
#include "qift_step.h"
int main() {
  int position;
  float freq, s, c;
  while (std::scanf("%d %a", &position, &freq) == 2) {
    qift::step::turn(position, freq, s, c);
    std::printf("%a %a\n", (double)s, (double)c);
  }
}
"""
PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798")


def exact_turn(position, freq):
    """Sine and cosine of position * freq to 70 digits and more of the angle."""
    x = position * Fraction(float(freq))
    r = x - 2 * PI * round(x / (2 * PI))
    r = Fraction(round(r * 2 ** 200), 2 ** 200)
    term, s, c = Fraction(1), Fraction(0), Fraction(0)
    for k in range(40):
        part = term if k % 4 < 2 else -term
        if k % 2:
            s += part
        else:
            c += part
        term = Fraction(round(term * r * 2 ** 200), 2 ** 200) / (k + 1)
    return float(s), float(c)


def test_sine_and_cosine_of_every_angle(tmp_path):
    """Within 2^-22 for every angle below 2^40, whether or not fp64 holds it; NaN from there on and for frequencies that are no number."""
    cxx = shutil.which("g++") or shutil.which("clang++") or "/opt/rocm/llvm/bin/clang++"
    (tmp_path / "probe.cpp").write_text(TURN)
    subprocess.run([cxx, "-std=c++17", "-I", CSRC, str(tmp_path / "probe.cpp"), "-o", str(tmp_path / "probe")], check=True)
    rng = np.random.default_rng(17)
    cases = [(p, np.float32(f)) for p in (0, 1, 7, 100000, 2 ** 24 + 1, 2 ** 28, 1639311774, 2142287670, I31)
             for f in (0.0, 1e-38, 1e-3, 0.1, 1.0, 2.6565, 96.7, 100.7, -100.7, 511.0, 1e6, 1e9, 9.8e8, 1e12, 1e30, np.inf, np.nan)]
    cases += [(int(p), np.float32(np.exp(f))) for p, f in zip(rng.integers(0, I31, 3000), rng.uniform(-12, 6.2, 3000))]
    # angles beside the borders of the quadrants: position 1, and far ones
    for n in list(range(1, 40)) + [int(v) for v in rng.integers(1, 2 ** 33, 400)]:
        p = int(rng.integers(1, I31))
        cases += [(1, np.nextafter(np.float32(n * float(PI) / 4), np.float32(side))) for side in (0, 1e30)]
        cases += [(p, np.float32(n * float(PI) / 4 / p))]
    out = subprocess.run([str(tmp_path / "probe")], input="".join(f"{p} {float(f).hex()}\n" for p, f in cases), text=True,
                         capture_output=True, check=True).stdout.splitlines()
    assert len(out) == len(cases)
    for (p, f), line in zip(cases, out):
        s, c = (float.fromhex(v) for v in line.split())
        if not np.isfinite(f) or p * abs(Fraction(float(f))) >= 2 ** 40:
            assert np.isnan(s) and np.isnan(c), (p, f)
        else:
            want = exact_turn(p, f)
            assert abs(s - want[0]) <= 2.0 ** -22 and abs(c - want[1]) <= 2.0 ** -22, (p, f)


def test_rope_launches_have_fewer_than_2_32_threads(L):
    """Workgroups of four waves, a wave to each row here: 2^26 - 3 rows and more would round up to 2^32 threads."""
    r = qift.HeadRopeC(128, 128, 0, 1e-5, A, None, None)
    for rows in (2 ** 26 - 3, 2 ** 26 - 1):
        for Hq in (1, 4):
            assert L.qift_head_norm_rope(ctypes.byref(r), A, 512, None, 0, 0, A, rows, Hq, 0, A, 512, None, 0, None) == E_SHAPE


VIEWS = r"""
#include <cstdio>
#include "qift_step.h"
int main() {
  long v[8];
  for (;;) {
    for (long& x : v)
      if (std::scanf("%ld", &x) != 1) return 0;
    using qift::step::View;
    std::printf("%d\n", (int)qift::step::overlap(View{(unsigned long)v[0], v[1], v[2], v[3]}, View{(unsigned long)v[4], v[5], v[6], v[7]}));
  }
}
"""


def test_views_that_share_memory(tmp_path):
    """Against the bytes one by one: any strides, interleaved rows of one stride, ends that touch, single rows, none."""
    cxx = shutil.which("g++") or shutil.which("clang++") or "/opt/rocm/llvm/bin/clang++"
    (tmp_path / "probe.cpp").write_text(VIEWS)
    subprocess.run([cxx, "-std=c++17", "-I", CSRC, str(tmp_path / "probe.cpp"), "-o", str(tmp_path / "probe")], check=True)
    rng = np.random.default_rng(11)
    cases = []
    for i in range(20000):
        view = []
        for _ in range(2):
            size = int(rng.integers(0, 6))
            view.append([int(rng.integers(1000, 1060)), size + int(rng.integers(0, 9)) + (size == 0), size, int(rng.integers(0, 7))])
        if i % 2:
            view[1][1] = view[0][1] = max(view[0][1], view[1][1])     # one stride
        cases.append(view)
    out = subprocess.run([str(tmp_path / "probe")], input="\n".join(" ".join(map(str, a + b)) for a, b in cases), text=True,
                         capture_output=True, check=True).stdout.split()
    assert len(out) == len(cases)
    seen = [0, 0]
    for (a, b), got in zip(cases, out):
        sets = [{at + r * stride + i for r in range(rows) for i in range(size)} for at, stride, size, rows in (a, b)]
        assert int(got) == bool(sets[0] & sets[1]), (a, b)
        seen[int(got)] += 1
    assert min(seen) > 3000


def test_rope_outputs_lie_apart(L):
    """Waves take their heads in any order: an output is its own input with its stride, or shares nothing with any array."""
    r = qift.HeadRopeC(128, 128, 0, 1e-5, 0x1000, 0x1400, 0x1800)
    rows, s = 40, 48 * 128      # q, k and v of 32 + 8 + 8 heads stacked
    big = 0x1000000

    def f(q=big, qs=s, k=big + 2 * 32 * 128, ks=s, pos=0x2000, qo=2 * big, qos=32 * 128, ko=3 * big, kos=8 * 128):
        return L.qift_head_norm_rope(ctypes.byref(r), q, qs, k, ks, 0, pos, rows, 32, 8, qo, qos, ko, kos, None)

    row, head = 2 * s, 256
    for kw in ({"qo": big + head, "qos": s}, {"qo": big - head, "qos": s}, {"qo": big + row, "qos": s}, {"qo": big + row, "qos": 2 * s},
               {"qo": big + 39 * row}, {"ko": big + 31 * head, "kos": s}, {"ko": big + 33 * head, "kos": s}, {"ko": big + 5 * row + 39 * head},
               {"ko": big, "kos": s}, {"qo": 2 * big, "ko": 2 * big + 31 * head, "qos": s, "kos": s}, {"ko": 2 * big + 39 * 32 * head},
               {"qo": 0x2000}, {"qo": 0x2000 + 144}, {"ko": 0x1000}, {"ko": 0x1400 + 240}, {"ko": 0x1800}):
        assert f(**kw) == E_SHAPE, kw
