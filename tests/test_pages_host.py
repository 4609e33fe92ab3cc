"""The paged KV4 cache without a GPU: the index arithmetic of csrc/qift_pages.h (a program compiled from that header),
the refusals of the C ABI, and the oracle's own pins.

No call here reaches a kernel launch: every argument set fails validation or has nothing to do.
"""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

from oracle import kv4 as okv4, pages as opages
from paper_2606_02823_amd import qift

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_02823_amd", "csrc")
OK, E_NULL, E_SHAPE, E_FORMAT, E_ALIGN, E_WS = 0, -1, -2, -4, -6, -8
A = 0x10000       # a 16-byte aligned fake device address (never dereferenced)
MIS = 0x10008

PROBE = r"""
#include <cstdio>
#include <cstring>
#include "qift_pages.h"
using namespace qift::pages;
int main() {
  char what[16];
  while (std::scanf("%15s", what) == 1) {
    if (!std::strcmp(what, "div")) {
      unsigned d, x;
      std::scanf("%u %u", &d, &x);
      std::printf("%u\n", quotient(x, make_div(d)));
    } else if (!std::strcmp(what, "slot")) {
      unsigned slot, page, Hkv, head;
      std::scanf("%u %u %u %u", &slot, &page, &Hkv, &head);
      std::printf("%u\n", slot_row(slot, make_div(page), Hkv, head));
    } else if (!std::strcmp(what, "token")) {
      unsigned t, entry, Hkv, head, page;
      std::scanf("%u %u %u %u %u", &t, &entry, &Hkv, &head, &page);
      const Div d = make_div(page / 16);
      std::printf("%u %u\n", table_index(t, d), token_row(t, entry, Hkv, head, d));
    } else if (!std::strcmp(what, "seq")) {
      int s0, s1, len, rows, most_nodes; long long most;
      std::scanf("%d %d %d %d %d %lld", &s0, &s1, &len, &rows, &most_nodes, &most);
      const Seq q = sequence(s0, s1, len, rows, most_nodes, most);
      std::printf("%d %d %d %d %d\n", q.row0, q.n, q.len, q.ctx, (int)q.bad);
    } else if (!std::strcmp(what, "last")) {
      int n, len, masked, block_rows, block; unsigned G;
      std::scanf("%d %d %d %u %d %d", &n, &len, &masked, &G, &block_rows, &block);
      std::printf("%d\n", last_token(sequence(0, n, len, n, 256, 1 << 28), masked, make_div(G), block_rows, block));
    } else if (!std::strcmp(what, "chain")) {
      int t0, ctx, node;
      std::scanf("%d %d %d", &t0, &ctx, &node);
      std::printf("%llu\n", (unsigned long long)chain_bits(t0, ctx, node));
    } else if (!std::strcmp(what, "tree")) {
      int d0; unsigned long long w0, w1;
      std::scanf("%d %llu %llu", &d0, &w0, &w1);
      std::printf("%llu\n", (unsigned long long)tree_bits(d0, w0, w1));
    } else if (!std::strcmp(what, "plan")) {
      long long B, len; int Hkv, G, nodes;
      std::scanf("%lld %d %d %d %lld", &B, &Hkv, &G, &nodes, &len);
      const Plan p = plan(B, Hkv, G, nodes, len);
      std::printf("%d %d %d %lld\n", p.rt, p.blocks, p.shares, (long long)records(p, B, Hkv));
    } else if (!std::strcmp(what, "used")) {
      long long W; int n;
      std::scanf("%lld %d", &W, &n);
      std::printf("%d\n", used_shares(W, n));
    } else if (!std::strcmp(what, "share")) {
      long long W; int n, i;
      std::scanf("%lld %d %d", &W, &n, &i);
      std::printf("%lld %lld\n", (long long)first_slot(W, n, i), (long long)first_slot(W, n, i + 1));
    } else if (!std::strcmp(what, "slots")) {
      int len;
      std::scanf("%d", &len);
      std::printf("%d %d\n", rounds_of(len), slots_of(len));
    } else if (!std::strcmp(what, "place")) {
      int g, shares, blocks;
      std::scanf("%d %d %d", &g, &shares, &blocks);
      const Place p = place(g, shares, blocks);
      std::printf("%d %d\n", p.share, p.block);
    } else if (!std::strcmp(what, "round")) {
      int slot;
      std::scanf("%d", &slot);
      std::printf("%d\n", round_at(slot));
    }
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("clang++") or "/opt/rocm/llvm/bin/clang++"
    d = tmp_path_factory.mktemp("pages")
    (d / "probe.cpp").write_text(PROBE)
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wno-unused-result", "-Xlinker", "-O1", "-I", CSRC, str(d / "probe.cpp"), "-o",
                    str(d / "probe")], check=True)

    def run(lines):
        out = subprocess.run([str(d / "probe")], input="".join(" ".join(map(str, x)) + "\n" for x in lines), text=True,
                             capture_output=True, check=True).stdout.splitlines()
        assert len(out) == len(lines)
        return [[int(v) for v in o.split()] for o in out]
    return run


def test_division_by_a_multiplier(ask):
    rng = np.random.default_rng(3)
    top = 2 ** 31 - 1
    ds = [1, 2, 3, 4, 5, 7, 16, 48, 63, 64, 65, 1000, 2 ** 20 - 1, 2 ** 20, 2 ** 30, 2 ** 30 + 1, top]
    ds += [int(v) for v in rng.integers(1, top, 40)]
    lines = []
    for d in ds:
        xs = {0, 1, d - 1, d, d + 1, 2 * d - 1, top, top - 1, top // d * d, top // d * d - 1}
        lines += [("div", d, x) for x in sorted(x for x in xs if 0 <= x <= top)]
        lines += [("div", d, int(x)) for x in rng.integers(0, top, 50)]
    for (_, d, x), (got,) in zip(lines, ask(lines)):
        assert got == x // d, (d, x)


def test_rows_stay_in_the_cache(ask):
    # every slot, and every token of a table entry that names a page, falls on its own row of [pages][Hkv][page]
    for pages, page, Hkv in ((3, 16, 1), (5, 48, 8), (2, 256, 3), (7, 64, 2)):
        lines, want = [], []
        for slot in range(pages * page):
            for head in range(Hkv):
                lines.append(("slot", slot, page, Hkv, head))
                want.append((slot // page * Hkv + head) * page + slot % page)
        got = [g[0] for g in ask(lines)]
        assert got == want and sorted(got) == list(range(pages * Hkv * page))
    # the largest pools: the last row below 2^31
    for pages, page, Hkv in (((2 ** 31 - 1) // 16, 16, 1), ((2 ** 31 - 1) // (64 * 8), 64, 8), (1, 2 ** 31 - 16, 1)):
        last = pages * page - 1
        assert ask([("slot", last, page, Hkv, Hkv - 1)])[0][0] == pages * page * Hkv - 1
    rng = np.random.default_rng(4)
    lines, want = [], []
    for _ in range(4000):
        page, Hkv = 16 * int(rng.integers(1, 40)), int(rng.integers(1, 40))
        t, entry, head = int(rng.integers(0, 2 ** 28)), int(rng.integers(0, 2 ** 31 // (page * Hkv))), int(rng.integers(0, Hkv))
        lines.append(("token", t, entry, Hkv, head, page))
        want.append([t // page, (entry * Hkv + head) * page + t % page])
    got = ask(lines)
    assert got == want and max(g[1] for g in got) < 2 ** 31


def test_any_device_data_gives_counts_in_range(ask):
    rng = np.random.default_rng(5)
    odd = [-2 ** 31, -1, 0, 1, 2, 63, 64, 100, 101, 2 ** 28, 2 ** 31 - 1]
    lines = []
    for _ in range(3000):
        s0, s1, ln = (int(rng.choice(odd)) for _ in range(3))
        lines.append(("seq", s0, s1, ln, int(rng.choice([1, 5, 100])), int(rng.choice([1, 7, 256])),
                      int(rng.choice([1, 16, 1000, 2 ** 28 - 1]))))
    for (_, s0, s1, ln, rows, nodes, most), (row0, n, length, ctx, bad) in zip(lines, ask(lines)):
        assert 0 <= row0 and 0 <= n <= nodes and row0 + n <= rows
        assert 0 <= length <= most and ctx == max(0, length - n)
        good = 0 <= s0 <= s1 <= rows and s1 - s0 <= nodes and 0 <= ln <= most
        assert bad == (not good)
        if good:
            assert (row0, n, length) == (s0, s1 - s0, ln)


def test_seen_bits(ask):
    rng = np.random.default_rng(6)
    lines, want = [], []
    for _ in range(2000):
        t0 = 64 * int(rng.integers(0, 8))
        n, ctx = int(rng.integers(1, 257)), int(rng.integers(0, 400))
        node = int(rng.integers(0, n))
        lines.append(("chain", t0, ctx, node))
        want.append(sum(1 << i for i in range(64) if t0 + i <= ctx + node))
        mask = rng.integers(0, 2, n).astype(bool)
        words = [int(w) & (2 ** 64 - 1) for w in opages.pack_mask(mask[None], 256)[0]] + [0]
        d0 = t0 - ctx
        k = max(d0, 0) >> 6
        w = [words[i] if i < 5 else 0 for i in (k, k + 1)]
        lines.append(("tree", d0, *w))
        want.append(sum(1 << i for i in range(64) if d0 + i < 0 or (d0 + i < n and mask[d0 + i])))
    assert [g[0] for g in ask(lines)] == want


def test_last_token_of_a_block_of_rows(ask):
    lines, want = [], []
    for n in (1, 2, 5, 37, 64, 256):
        for G in (1, 3, 4, 8):
            for length in (n, n + 1, n + 700):
                for br in (16, 32, 64):
                    for block in range(-(-n * G // br)):
                        top = min(n - 1, ((block + 1) * br - 1) // G)
                        lines += [("last", n, length, 0, G, br, block), ("last", n, length, 1, G, br, block)]
                        want += [length - n + top + 1, length]
    assert [g[0] for g in ask(lines)] == want


def test_plan_covers_every_row(ask):
    rng = np.random.default_rng(7)
    lines = []
    for _ in range(3000):
        lines.append(("plan", int(np.exp(rng.uniform(0, 11))), int(np.exp(rng.uniform(0, 5))), int(rng.integers(1, 65)),
                      int(rng.integers(1, 257)), int(np.exp(rng.uniform(0, 19.4)))))
    for (_, B, Hkv, G, nodes, length), (rt, blocks, shares, records) in zip(lines, ask(lines)):
        assert rt in (1, 2, 4) and blocks * 16 * rt >= nodes * G > (blocks - 1) * 16 * rt
        assert 0 <= shares <= B * Hkv * (-(-length // 256) + 2) and (B <= 512 or shares == 0)
        assert records == (shares + B * Hkv if shares else 0)


def test_every_block_of_every_share_has_one_workgroup(ask):
    """Also where fewer shares are used than the launch was made for; and no XCD (every eighth workgroup) has more than
    its part."""
    rng = np.random.default_rng(12)
    for _ in range(60):
        blocks = int(np.exp(rng.uniform(0, 6.9)))
        planned = max(1, 512 // blocks)
        used = planned if rng.integers(0, 2) else int(rng.integers(0, planned + 1))
        groups = (planned * blocks + 7) // 8 * 8
        got = ask([("place", g, used, blocks) for g in range(groups)])
        at = [(g, s, k) for g, (s, k) in enumerate(got) if s < used]
        assert all(s >= 0 and 0 <= k < blocks for _, s, k in at)
        assert sorted((s, k) for _, s, k in at) == [(s, k) for s in range(used) for k in range(blocks)]
        assert max([sum(g % 8 == x for g, _, _ in at) for x in range(8)]) == -(-used * blocks // 8)


def test_shares_cover_every_round_once(ask):
    """The runs of units that the shares take, as the kernel walks them: every round once and in order, the records'
    numbers different and inside the workspace, and the shares of a unit that have rounds of it next to each other (the
    partial records of a unit are joined from its first share to its last)."""
    rng = np.random.default_rng(11)
    for _ in range(80):
        B, Hkv = int(rng.integers(1, 9)), int(rng.integers(1, 9))
        lens = rng.integers(0, 256 * 30, B) * rng.integers(0, 2, B) // rng.choice([1, 1, 8])
        nodes = rng.integers(0, 2, B)                                     # sequences without nodes have no slots
        slots = np.array([g[1] for g in ask([("slots", int(t)) for t in lens])]) * nodes
        rounds = np.array([g[0] for g in ask([("slots", int(t)) for t in lens])]) * nodes
        assert (rounds[nodes > 0] == np.maximum(1, -(-lens[nodes > 0] // 256))).all()
        W = int(slots.sum()) * Hkv
        asked = int(rng.integers(1, 120))
        if W == 0:
            continue
        n = ask([("used", W, asked)])[0][0]
        assert n == min(W, asked)
        bounds = ask([("share", W, n, i) for i in range(n)])
        assert bounds[0][0] == 0 and all(lo < hi for lo, hi in bounds) and bounds[-1][1] == W
        assert all(a[1] == b[0] for a, b in zip(bounds, bounds[1:]))
        at_slot = [g[0] for g in ask([("round", i) for i in range(int(slots.max()) + 1)])]
        numbers = set()
        for b in range(B):
            for kv in range(Hkv):
                at, k, u = int(slots[:b].sum()) * Hkv + kv * int(slots[b]), int(slots[b]), b * Hkv + kv
                took, next_round = [], 0
                for i, (lo, hi) in enumerate(bounds):
                    lo, hi = max(lo, at), min(hi, at + k)
                    if lo >= hi or at_slot[hi - at] == at_slot[lo - at]:
                        continue
                    assert at_slot[lo - at] == next_round
                    next_round = at_slot[hi - at]
                    took.append(i)
                    assert 0 <= i + u < n + B * Hkv and i + u not in numbers
                    numbers.add(i + u)
                assert next_round == rounds[b] and took == list(range(took[0], took[-1] + 1) if took else [])


# ---- the C ABI ---------------------------------------------------------------------------------------------------


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(qift.LIB_PATH):
        pytest.skip("libqift.so not built")
    return qift.lib()


def pool(pages=10, page=64, Hkv=8, head_dim=128, reserved=0, **kw):
    ptr = dict(k_codes=A, k_scales=A, k_zeros=A, v_codes=A, v_scales=A, v_zeros=A)
    ptr.update(kw)
    return ctypes.byref(qift.KV4PagesC(pages, page, Hkv, head_dim, reserved, *ptr.values()))


BAD_POOLS = [dict(pages=0), dict(page=0), dict(page=8), dict(page=72), dict(page=-16), dict(Hkv=0), dict(Hkv=65536),
             dict(head_dim=64), dict(reserved=1), dict(pages=2 ** 31), dict(pages=2 ** 22 + 1), dict(pages=2 ** 62)]


def test_every_declared_symbol_is_exported(L):
    text = open(os.path.join(ROOT, "include", "qift_pages.h")).read()
    names = set(re.findall(r"\b(qift_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert names == set(qift.PAGES_EXPORTS)
    for n in names:
        assert hasattr(L, n), n
    assert ctypes.sizeof(qift.KV4PagesC) == 8 + 4 * 4 + 6 * 8
    assert not set(qift.PAGES_EXPORTS) & set(qift.EXPORTS)


def test_append_refusals(L):
    def f(cache=pool(), k=A, v=A, ks=1024, vs=1024, dt=0, slots=A, n=4, kv=None, vv=None):
        return L.qift_kv4_append(cache, k, v, ks, vs, dt, slots, n, kv, vv, None)
    assert f(cache=None) == E_NULL
    for bad in BAD_POOLS:
        assert f(cache=pool(**bad)) == E_SHAPE, bad
    assert f(dt=2) == E_FORMAT and f(dt=-1) == E_FORMAT
    for kw in (dict(n=-1), dict(n=2 ** 31), dict(ks=1023), dict(vs=0), dict(ks=-1024), dict(vs=2 ** 31),
               dict(cache=pool(pages=1, page=16, Hkv=65535), n=2 ** 20, ks=65535 * 128, vs=65535 * 128)):
        assert f(**kw) == E_SHAPE, kw
    # workgroups of 256 threads along one axis of a launch: fewer than 2^32 threads
    assert f(n=2 ** 24, k=None) == E_SHAPE and f(n=2 ** 24 - 16, k=None) == E_NULL
    for kw in (dict(k=None), dict(v=None), dict(slots=None), dict(kv=A), dict(vv=A), dict(cache=pool(v_zeros=None))):
        assert f(**kw) == E_NULL, kw
    for kw in (dict(k=MIS), dict(v=MIS), dict(ks=1028), dict(vs=1030), dict(slots=A + 2), dict(kv=MIS, vv=A),
               dict(kv=A, vv=MIS), dict(cache=pool(k_codes=MIS)), dict(cache=pool(v_scales=MIS))):
        assert f(**kw) == E_ALIGN, kw
    assert f(n=0, k=None, v=None, slots=None) == OK     # nothing to do


def test_read_refusals(L):
    def f(cache=pool(), slots=A, n=4, dt=0, kv=A, vv=A):
        return L.qift_kv4_read(cache, slots, n, dt, kv, vv, None)
    assert f(cache=None) == E_NULL
    for bad in BAD_POOLS:
        assert f(cache=pool(**bad)) == E_SHAPE, bad
    assert f(dt=3) == E_FORMAT
    assert f(n=-1) == E_SHAPE and f(n=2 ** 31) == E_SHAPE
    assert f(n=2 ** 30, slots=None) == E_SHAPE and f(n=2 ** 30 - 64, slots=None) == E_NULL
    for kw in (dict(slots=None), dict(kv=None), dict(vv=None), dict(cache=pool(k_scales=None))):
        assert f(**kw) == E_NULL, kw
    for kw in (dict(slots=A + 1), dict(kv=MIS), dict(vv=MIS), dict(cache=pool(k_zeros=MIS))):
        assert f(**kw) == E_ALIGN, kw
    assert f(n=0, slots=None, kv=None, vv=None) == OK


def test_tree_refusals(L):
    ws = L.qift_kv4_attention_tree_workspace_bytes

    def f(cache=pool(), q=A, qs=4096, dt=0, rows=5, table=A, tp=100, starts=A, lens=A, B=2, Hq=32, nodes=8, length=3000,
          vis=None, out=A, work=A, size=1 << 40):
        return L.qift_kv4_attention_tree(cache, q, qs, dt, rows, table, tp, starts, lens, B, Hq, nodes, length, vis, out, work,
                                         size, None)
    assert f(cache=None) == E_NULL
    for bad in BAD_POOLS:
        assert f(cache=pool(**bad)) == E_SHAPE, bad
    assert f(dt=2) == E_FORMAT
    for kw in (dict(B=-1), dict(B=65536), dict(Hq=0), dict(Hq=12), dict(Hq=8 * 65, qs=8 * 65 * 128), dict(nodes=0),
               dict(nodes=257), dict(length=0), dict(length=2 ** 28), dict(rows=-1), dict(rows=2 ** 31), dict(tp=0), dict(qs=4095),
               dict(qs=2 ** 31)):
        assert f(**kw) == E_SHAPE, kw
    # (512 workgroups to a sequence and KV head)
    big = dict(cache=pool(Hkv=1), Hq=64, qs=64 * 128, nodes=256, length=256)
    assert f(B=2 ** 15, q=None, **big) == E_SHAPE and f(B=2 ** 15 - 16, q=None, **big) == E_NULL
    for kw in (dict(q=None), dict(table=None), dict(starts=None), dict(lens=None), dict(out=None), dict(cache=pool(k_codes=None))):
        assert f(**kw) == E_NULL, kw
    for kw in (dict(q=MIS), dict(qs=4100), dict(out=MIS), dict(table=A + 2), dict(starts=A + 1), dict(lens=A + 2), dict(vis=A + 4),
               dict(work=MIS), dict(cache=pool(v_codes=MIS))):
        assert f(**kw) == E_ALIGN, kw
    need = ws(2, 32, 8, 128, 8, 3000)
    assert need > 2 * 8 * 8 and (need - 2 * 8 * 8) % (8 * 4 * 130 * 4) == 0   # records of rows, then a pair per unit
    assert f(work=None) == E_WS and f(size=need - 1) == E_WS and f(size=0) == E_WS
    assert f(B=0, q=None, table=None, starts=None, lens=None, out=None, work=None) == OK
    assert f(rows=0, q=None, out=None) == OK
    # the query: 0 for what is not supported and for sequences of one chunk
    assert ws(1, 32, 8, 64, 8, 1000) == 0 and ws(1, 30, 8, 128, 8, 1000) == 0 and ws(1, 32, 8, 128, 300, 1000) == 0
    assert ws(1, 32, 8, 128, 8, 256) == 0 and ws(0, 32, 8, 128, 8, 1000) == 0


def test_binding_refuses_before_any_call():
    import torch
    with pytest.raises(TypeError):
        qift.KV4Pages(*(qift.KV4(torch.zeros(2, 8, 16, 64, dtype=torch.uint8), torch.zeros(2, 8, 16), torch.zeros(2, 8, 16))
                        for _ in range(2)))
    with pytest.raises(TypeError):
        qift._rows(torch.zeros(3, 8, 128, dtype=torch.float16), 0, torch.float16, (3, 8, 128), "k")


# ---- the oracle ---------------------------------------------------------------------------------------------------


def test_oracle_quantizer_is_kv4s_on_fp16():
    rng = np.random.default_rng(8)
    x = rng.normal(0, 1, (300, 128)).astype(np.float16)
    x[::7] = 0
    for a, b in zip(opages.quantize(x.astype(np.float32)), okv4.kv4_quant(x)):
        assert np.array_equal(a, b)


def test_oracle_attention_is_kv4s_for_one_token():
    rng = np.random.default_rng(9)
    q = rng.normal(0, 1, (1, 8, 128))
    k, v = rng.normal(0, 1, (2, 50, 2, 128)).astype(np.float32)
    got = opages.attention(q, k, v, opages.chain(1, 50))
    assert np.allclose(got, okv4.attention_decode(q, k[None], v[None]), rtol=1e-12)
    # a tree whose mask is the lower triangle is the chain; a row that sees nothing gives 0
    q = rng.normal(0, 1, (5, 8, 128))
    a = opages.attention(q, k, v, opages.chain(5, 50))
    assert np.array_equal(a, opages.attention(q, k, v, opages.tree(np.tril(np.ones((5, 5), dtype=bool)), 50)))
    none = opages.attention(q, k[:5], v[:5], opages.tree(np.zeros((5, 5), dtype=bool), 5))
    assert not none.any()


def test_oracle_append_then_read():
    rng = np.random.default_rng(10)
    pages, page, Hkv = 4, 16, 2
    empty = (np.zeros((pages, Hkv, page, 128), np.uint8), np.zeros((pages, Hkv, page), np.float32),
             np.zeros((pages, Hkv, page), np.uint8))
    x = rng.normal(0, 1, (6, Hkv, 128)).astype(np.float32)
    slots = [0, 63, -1, 17, 64, 40]
    *after, values = opages.append(*empty, x, slots)
    assert np.array_equal(opages.read(*after, slots), values)
    assert not values[2].any() and not values[4].any()                 # padding, and past the pool
    assert (after[1] != 0).sum() == 4 * Hkv
    assert np.abs(values[0] - x[0]).max() <= after[1].max() * 4        # within the clipped range's steps


def test_nodes_that_are_left_out_do_not_move_the_others(ask):
    """A sequence with more nodes than the launch was made for, or than there are rows: the first ones stand where the
    starts and the length put them, and the tokens of the others, which come behind, are cut off.  A sequence whose first
    row is none has no rows at all."""
    rng = np.random.default_rng(13)
    lines = [("seq", 0, 3, 400, 3, 2, 1000), ("seq", 0, 3, 400, 2, 256, 1000), ("seq", 0, 5, 3, 5, 2, 1000),
             ("seq", -4, 3, 400, 5, 256, 1000), ("seq", 6, 9, 400, 5, 256, 1000), ("seq", 0, 2 ** 31 - 1, 400, 5, 256, 1000)]
    got = ask(lines)
    assert got[:2] == [[0, 2, 399, 397, 1]] * 2 and got[2] == [0, 2, 2, 0, 1]
    assert got[3][1] == got[4][1] == 0 and got[5] == [0, 5, 5, 0, 1]
    lines = []
    for _ in range(3000):
        rows = int(rng.integers(1, 40))
        s0 = int(rng.integers(0, rows + 1))
        lines.append(("seq", s0, s0 + int(rng.integers(0, 60)), int(rng.integers(0, 200)), rows, int(rng.integers(1, 50)), 150))
    for (_, s0, s1, ln, rows, most_nodes, most), (row0, n, length, ctx, bad) in zip(lines, ask(lines)):
        nodes, ln = s1 - s0, min(ln, most)
        assert row0 == s0 and n == min(nodes, rows - s0, most_nodes)
        assert ctx == max(0, ln - nodes)
        assert length == (ln if n == nodes else min(ln, ctx + n))


def test_workspace_covers_every_smaller_call(L):
    """A workspace of the queried size serves every call whose sequences, nodes and lengths are at most the queried ones, and
    the query grows with each of them; a call itself asks for what its own plan needs, which may be less."""
    ws = L.qift_kv4_attention_tree_workspace_bytes

    def enough(B, Hq, Hkv, nodes, length, size):   # (misaligned queries are refused after the size, and nothing is launched)
        st = L.qift_kv4_attention_tree(pool(Hkv=Hkv), MIS, Hq * 128, 0, 5, A, 100, A, A, B, Hq, nodes, length, None, A, A, size, None)
        assert st in (E_ALIGN, E_WS)
        return st == E_ALIGN
    # the server of 16 sequences whose largest step is 64 nodes over 8192 tokens
    most = ws(16, 32, 8, 128, 64, 8192)
    assert most > 0
    for nodes in range(1, 65):
        assert enough(16, 32, 8, nodes, 8192, most), nodes
    rng = np.random.default_rng(14)
    for _ in range(300):
        Hkv, G = int(rng.choice([1, 2, 4, 8, 32])), int(rng.choice([1, 2, 3, 4, 8, 64]))
        B, nodes, length = int(np.exp(rng.uniform(0, 7))), int(rng.integers(1, 257)), int(np.exp(rng.uniform(0, 12)))
        size = ws(B, Hkv * G, Hkv, 128, nodes, length)
        assert size < 26e6
        for _ in range(12):
            b, n, t = int(rng.integers(1, B + 1)), int(rng.integers(1, nodes + 1)), int(rng.integers(1, length + 1))
            assert enough(b, Hkv * G, Hkv, n, t, size), (B, Hkv, G, nodes, length, b, n, t)
            assert ws(b, Hkv * G, Hkv, 128, n, t) <= size
    # no call of one round of tokens needs any
    assert ws(600, 32, 8, 128, 256, 256) == 0 and enough(600, 32, 8, 256, 256, 0)


def test_binding_refuses_a_stream_of_another_device():
    """Kernels are launched on the cache's device: a stream of another one would run them there, on memory it may not reach."""
    from types import SimpleNamespace

    def call(*args):
        raise AssertionError("the call must not be reached")
    with pytest.raises(ValueError, match="stream"):
        qift._run(0, call, (), SimpleNamespace(device_index=1, cuda_stream=0))


def test_plan_has_row_tiles_that_the_kernel_is_built_for(ask):
    lines = [("plan", B, Hkv, G, nodes, length) for B in (1, 7, 600) for Hkv in (1, 8) for G in (1, 3, 4, 64) for nodes in (1, 4, 5, 16, 17, 256)
             for length in (1, 257, 5000)]
    for (_, _, _, G, nodes, _), (rt, blocks, *_) in zip(lines, ask(lines)):
        assert rt == (1 if nodes * G <= 16 else 2) and blocks == -(-nodes * G // (16 * rt))
