"""A serving step around the paged cache on the GPU: plans and releases (whole numbers: equal to the oracle's), and the norms
and rotation of heads.

Rotation against fp64, for |a| + |b| of a value's pair (its own size where it is not rotated), with u = 2^-24: the sum of
squares takes 8 fused steps in a lane and 4 joins, the mean one more, at most 13 u, half of that in the root; the reciprocal root
is within 2 u, its product with the weight and with the value u each: 11 u of the normed value; sine and cosine are
within 4 u (u for the reduced angle, at most pi / 4, and 3 u for the sums), the two products and the sum of a rotation within
2 u of |a| + |b|: 17 u (|a| + |b|) < 2^-19 (|a| + |b|), and half a step of the output's type, 2^-11 or 2^-8 of
the value, for fp16 at least 2^-25.
"""
import numpy as np
import pytest
import torch

from oracle import linear as olin, pages as opages, step as ostep, w8

pytestmark = pytest.mark.gpu

HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
I31 = 2 ** 31 - 1


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_02823_amd import qift
    qift.lib()
    return qift


def dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


class Server:
    """Tables of B sequences with the given lengths in pages of a pool, in any order, and what is free."""

    def __init__(self, rng, lens, width, page, spare):
        self.page = page
        self.lens = np.asarray(lens, np.int32)
        held = -(-np.clip(self.lens, 0, width * page) // page)
        pages = rng.permutation(int(held.sum()) + spare).astype(np.int32)
        self.table = np.full((len(lens), width), -1, np.int32)
        at = 0
        for b, h in enumerate(held):
            self.table[b, :h] = pages[at:at + h]
            at += h
        self.depth = spare
        self.free = np.concatenate([pages[at:], np.full(at + 3, -1, np.int32)])


def check_plan(Q, s, counts, rows, depth=None):
    depth = s.depth if depth is None else depth
    want = ostep.plan(s.lens, counts, s.table, s.free, depth, s.page, rows)
    table, free = dev(s.table), dev(s.free)
    Q.device_error()
    got = Q.kv4_plan_step(dev(s.lens), dev(counts), table, free, dev([depth]), s.page, rows)
    bits = Q.device_error()
    for name, w in (("starts", want[0]), ("lens", want[1]), ("slots", want[3]), ("positions", want[4])):
        assert np.array_equal(getattr(got, name).cpu().numpy(), w), name
    assert np.array_equal(table.cpu().numpy(), want[2]) and int(got.free_count) == want[5]
    assert np.array_equal(free.cpu().numpy(), s.free)
    assert bits == (Q.DEVERR_INDEX if want[6] else 0)
    return want


@pytest.mark.parametrize("page", [16, 48, 64, 256])
@pytest.mark.parametrize("B,n,width,pad", [(1, 1, 4, 0), (3, 1, 9, 2), (61, 1, 40, 3), (255, 3, 7, 0), (256, 2, 5, 1), (257, 40, 6, 9),
                                           (1000, 5, 3, 100), (4, 3000, 300, 7)])
def test_plans(Q, B, n, width, pad, page):
    rng = np.random.default_rng(B + n + page)
    counts = rng.integers(0, 2 * n + 1, B)
    counts[rng.random(B) < 0.1] = 0
    lens = np.minimum(rng.integers(0, width * page + 1, B), np.maximum(0, width * page - counts))
    lens[rng.random(B) < 0.2] = 0
    counts = np.minimum(counts, width * page - lens)
    s = Server(rng, lens, width, page, int((counts // page + 1).sum()) + 2)
    want = check_plan(Q, s, counts, int(counts.sum()) + pad)
    assert not want[6]


def test_plan_of_a_long_prompt_and_of_nothing(Q):
    rng = np.random.default_rng(2)
    s = Server(rng, [70, 0, 5], 4200, 16, 8500)
    check_plan(Q, s, np.array([1, 65536, 0]), 65600)
    check_plan(Q, s, np.array([0, 0, 0]), 5)
    check_plan(Q, s, np.array([0, 0, 0]), 0)
    s = Server(rng, [], 3, 16, 4)
    check_plan(Q, s, np.array([], np.int32), 6)


@pytest.mark.parametrize("B", [3, 300, 900])
def test_plans_that_leave_sequences_out(Q, B):
    """Too few pages, rows or places in a table row, at any point of the order."""
    rng = np.random.default_rng(B)
    width, page = 5, 16
    lens = rng.integers(0, 60, B)
    counts = rng.integers(0, 30, B)
    s = Server(rng, lens, width, page, 4 * B)
    assert np.any(lens + counts > width * page) or B == 3
    total = int(counts.sum())
    for rows in (total, total - 1, total // 2, 7, 0):
        for depth in (4 * B, B // 2, 1, 0):
            check_plan(Q, s, counts, rows, depth)


def test_plans_where_pages_run_out(Q):
    """Sequences that need no page behind ones that found too few: the stack keeps what nobody took."""
    rng = np.random.default_rng(21)
    s = Server(rng, [0, 1], 10, 16, 5)
    want = check_plan(Q, s, np.array([160, 1]), 170)
    assert want[5] == 5 and list(want[1]) == [0, 2]
    for B in (7, 256, 600):
        s = Server(rng, rng.integers(0, 60, B), 5, 16, 3 * B)
        counts = rng.integers(0, 20, B)
        for depth in (B // 2, 2, 0):
            want = check_plan(Q, s, counts, int(counts.sum()), depth)
            assert 0 <= want[5] <= depth and (want[6] or depth > 0)


def test_plan_with_numbers_out_of_range(Q):
    rng = np.random.default_rng(7)
    width, page = 4, 32
    for _ in range(6):
        s = Server(rng, rng.integers(0, 100, 40), width, page, 90)
        counts = rng.integers(0, 40, 40)
        check_plan(Q, s, counts, 900)
        s.lens[[3, 9]] = -5, I31
        counts[[4, 11]] = -9, I31
        check_plan(Q, s, counts, 900)
        check_plan(Q, s, counts, 900, depth=-3)
        check_plan(Q, s, counts, 900, depth=10 ** 6)
        s.lens[[3, 9]], counts[[4, 11]] = 0, 1
        s.free[s.depth - 2], s.free[s.depth - 5] = -4, I31
        s.table[7, 0], s.table[8, 0] = -1, 2 ** 30
        check_plan(Q, s, counts, 900)


def test_plan_writes_only_its_outputs(Q):
    rng = np.random.default_rng(4)
    B, width, page, rows = 300, 6, 16, 700
    s = Server(rng, rng.integers(0, 50, B), width, page, 700)
    counts = rng.integers(0, 4, B)
    sizes, pad = (B + 1, B, rows, rows, 1), 16
    room = torch.full((sum(sizes) + pad * 6,), 12345, dtype=torch.int32, device="cuda")
    at, views, keep = pad, [], torch.ones_like(room, dtype=torch.bool)
    for n in sizes:
        views.append(room[at:at + n])
        keep[at:at + n] = False
        at += n + pad
    out = Q.KV4Plan(*views)
    want = ostep.plan(s.lens, counts, s.table, s.free, s.depth, page, rows)
    assert Q.kv4_plan_step(dev(s.lens), dev(counts), dev(s.table), dev(s.free), dev([s.depth]), page, rows, out=out) is out
    assert np.array_equal(out.slots.cpu().numpy(), want[3]) and np.array_equal(out.starts.cpu().numpy(), want[0])
    assert torch.all(room[keep] == 12345)


def check_release(Q, s, done, depth=None):
    depth = s.depth if depth is None else depth
    want = ostep.release(s.lens, done, s.table, s.free, depth, s.page)
    free, table = dev(s.free), dev(s.table)
    Q.device_error()
    lens, count = Q.kv4_release(dev(s.lens), dev(done), table, free, dev([depth]), s.page)
    assert Q.device_error() == (Q.DEVERR_INDEX if want[3] else 0)
    assert np.array_equal(lens.cpu().numpy(), want[0]) and np.array_equal(free.cpu().numpy(), want[1]) and int(count) == want[2]
    assert np.array_equal(table.cpu().numpy(), s.table)


@pytest.mark.parametrize("B,width,page", [(1, 1, 16), (5, 300, 16), (64, 20, 64), (256, 3, 48), (700, 9, 16)])
def test_releases(Q, B, width, page):
    rng = np.random.default_rng(B)
    s = Server(rng, rng.integers(0, width * page + 1, B), width, page, 6)
    for share in (0.0, 0.3, 1.0):
        check_release(Q, s, (rng.random(B) < share) * rng.integers(1, 5, B))
    check_release(Q, s, np.ones(B, np.int64), depth=len(s.free) - 1)     # no room for all
    s.lens[0] = -1
    check_release(Q, s, np.ones(B, np.int64))
    s.lens[0], s.table[B - 1] = I31, -2
    check_release(Q, s, np.ones(B, np.int64), depth=-1)
    check_release(Q, Server(rng, [], 3, 16, 4), np.array([], np.int64))


def test_a_servers_run(Q):
    """Steps and releases in turn, each from the tensors of the one before, two sets of outputs in turn in one captured graph."""
    rng = np.random.default_rng(12)
    B, width, page, rows, pages = 40, 12, 16, 400, 300
    lens, table = np.zeros(B, np.int32), np.full((B, width), -1, np.int32)
    free, depth = rng.permutation(pages).astype(np.int32), pages
    t_lens, t_table, t_free, t_depth = dev(lens), dev(table), dev(free), dev([depth])
    counts, done = dev(np.zeros(B)), dev(np.zeros(B))
    plan = Q.kv4_plan_step(t_lens, counts, t_table, t_free, t_depth, page, rows)
    back = Q.kv4_release(plan.lens, done, t_table, t_free, plan.free_count, page)

    def step():
        Q.kv4_plan_step(t_lens, counts, t_table, t_free, t_depth, page, rows, out=plan)
        Q.kv4_release(plan.lens, done, t_table, t_free, plan.free_count, page, out=back)
        t_lens.copy_(back[0])
        t_depth.copy_(back[1])

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(25):
        n = np.minimum(rng.integers(0, 15, B), width * page - lens)
        over = ((rng.random(B) < 0.1) | (lens > width * page - 20)).astype(np.int32)
        counts.copy_(dev(n))
        done.copy_(dev(over))
        g.replay() if i % 3 else step()
        starts, lens, table, slots, pos, depth, bad = ostep.plan(lens, n, table, free, depth, page, rows)
        lens, free, depth, bad2 = ostep.release(lens, over, table, free, depth, page)
        assert np.array_equal(plan.slots.cpu().numpy(), slots) and np.array_equal(t_lens.cpu().numpy(), lens)
        assert np.array_equal(t_table.cpu().numpy(), table) and int(t_depth) == depth
        assert np.array_equal(t_free.cpu().numpy()[:depth], free[:depth])


# ---- norms and rotation


def heads_of(rng, rows, heads, dtype):
    x = rng.normal(0, 1, (rows, heads, 128)) * np.exp(rng.normal(0, 1, (rows, heads, 1)))
    x[:, :, rng.integers(0, 128, 3)] *= 20
    if rows > 2 and heads:
        x[1, 0] = 0.0
        x[2, -1] *= 1e-6
    return torch.from_numpy(x).to(dtype)


def check_rope(y, x, weight, eps, freq, pos, rot, pairs):
    dtype = x.dtype
    ref, scale = ostep.head_norm_rope(x.double().numpy(), None if weight is None else weight.double().numpy(), eps, freq, pos, rot, pairs)
    half = HALF[dtype] * np.abs(ref)
    if dtype is torch.float16:
        half = np.maximum(half, 2.0 ** -25)
    off = np.abs(y.double().cpu().numpy() - ref) - (half * (1 + 2.0 ** -19) + 2.0 ** -19 * scale)
    assert y.dtype is dtype and np.all(off <= 0), float(off.max())


def frequencies(rot, theta=5e5):
    half = rot // 2
    return (theta ** (-np.arange(half) / max(half, 1))).astype(np.float32)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rot,pairs", [(128, False), (128, True), (64, False), (96, False), (96, True), (8, False), (8, True), (120, False),
                                       (0, False), (0, True)])
@pytest.mark.parametrize("rows,Hq,Hkv,norms", [(1, 32, 8, 3), (7, 3, 1, 1), (5, 1, 1, 0), (130, 8, 2, 2), (9, 0, 4, 3), (4, 5, 0, 1)])
def test_heads(Q, rows, Hq, Hkv, norms, rot, pairs, dtype):
    rng = np.random.default_rng(rows + Hq + rot + pairs)
    q, k = heads_of(rng, rows, Hq, dtype), heads_of(rng, rows, Hkv, dtype)
    wq, wk = (torch.from_numpy(rng.normal(1, 0.3, 128)).to(dtype) if norms & bit else None for bit in (1, 2))
    freq = frequencies(rot)
    pos = rng.integers(0, 100000, rows)
    if rows > 3:
        pos[3] = -1
    rope = Q.HeadRope(dev(freq, torch.float32), rot, pairs, None if wq is None else wq.cuda(), None if wk is None else wk.cuda(), 1e-6)
    yq, yk = Q.head_norm_rope(rope, q.cuda(), k.cuda(), dev(pos))
    check_rope(yq, q, wq, 1e-6, freq, pos, rot, pairs)
    check_rope(yk, k, wk, 1e-6, freq, pos, rot, pairs)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("rows,Hq,Hkv", [(1400, 32, 8), (4100, 5, 2), (1030, 32, 32)])
def test_many_rows(Q, rows, Hq, Hkv, pairs, dtype):
    """Rows enough for several heads to a lane, from stacked q|k|v rows, written into stacked rows in place and elsewhere."""
    rng = np.random.default_rng(rows)
    qkv = heads_of(rng, rows, Hq + 2 * Hkv, dtype)
    wq, wk = (torch.from_numpy(rng.normal(1, 0.3, 128)).to(dtype) for _ in range(2))
    freq = frequencies(128)
    pos = rng.integers(0, 1 << 20, rows)
    pos[rows // 2], pos[-1] = -1, I31
    rope = Q.HeadRope(dev(freq, torch.float32), 128, pairs, wq.cuda(), wk.cuda(), 1e-5)
    stacked = qkv.cuda()
    q, k = stacked[:, :Hq], stacked[:, Hq:Hq + Hkv]
    yq, yk = Q.head_norm_rope(rope, q, k, dev(pos))
    check_rope(yq, qkv[:, :Hq], wq, 1e-5, freq, pos, 128, pairs)
    check_rope(yk, qkv[:, Hq:Hq + Hkv], wk, 1e-5, freq, pos, 128, pairs)
    got = Q.head_norm_rope(rope, q, k, dev(pos), out=(q, k))
    assert got[0] is q and torch.equal(q, yq) and torch.equal(k, yk)
    assert torch.equal(stacked[:, Hq + Hkv:].cpu(), qkv[:, Hq + Hkv:])       # the values are left


@pytest.mark.parametrize("position", [0, 1, 2 ** 20 + 1, 2 ** 24 + 1, 2 ** 29 - 1, I31])
def test_far_positions(Q, position):
    rng = np.random.default_rng(3)
    q, k = heads_of(rng, 3, 4, torch.bfloat16), heads_of(rng, 3, 4, torch.bfloat16)
    freq = frequencies(128, 1e4)
    pos = np.array([position, max(position - 1, 0), position // 3])
    rope = Q.HeadRope(dev(freq, torch.float32))
    yq, yk = Q.head_norm_rope(rope, q.cuda(), k.cuda(), dev(pos))
    check_rope(yq, q, None, 1.0, freq, pos, 128, False)
    check_rope(yk, k, None, 1.0, freq, pos, 128, False)


def test_rope_writes_only_its_rows(Q):
    rng = np.random.default_rng(8)
    q, k = heads_of(rng, 6, 3, torch.float16), heads_of(rng, 6, 2, torch.float16)
    rope = Q.HeadRope(dev(frequencies(64), torch.float32), 64)
    pos = dev([4, -1, 0, 9, 7, 3])
    room = torch.full((8, 9, 128), 5.0, dtype=torch.float16, device="cuda")
    qo, ko = room[1:7, 1:4], room[1:7, 6:8]
    Q.head_norm_rope(rope, q.cuda(), k.cuda(), pos, out=(qo, ko))
    yq, yk = Q.head_norm_rope(rope, q.cuda(), k.cuda(), pos)
    assert torch.equal(qo, yq) and torch.equal(ko, yk)
    keep = torch.ones_like(room, dtype=torch.bool)
    keep[1:7, 1:4] = keep[1:7, 6:8] = False
    assert torch.all(room[keep] == 5)


def test_step_binding_refuses(Q):
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    with pytest.raises(ValueError):
        Q.kv4_plan_step(i(3), i(4), i(4, 2), i(9), i(1), 16, 4)
    with pytest.raises(TypeError):
        Q.kv4_plan_step(i(4).long(), i(4), i(4, 2), i(9), i(1), 16, 4)
    with pytest.raises(Q.QiftError):
        Q.kv4_plan_step(i(4), i(4), i(4, 2), i(9), i(1), 20, 4)
    lens = i(4)
    with pytest.raises(Q.QiftError):
        Q.kv4_release(lens, i(4), i(4, 2), i(9), i(1), 16, out=(lens, i(1)))
    f = torch.zeros(64, device="cuda")
    h = torch.zeros((2, 4, 128), dtype=torch.float16, device="cuda")
    with pytest.raises(ValueError):
        Q.HeadRope(f, 64)
    with pytest.raises(TypeError):
        Q.HeadRope(f, 128, q_weight=torch.zeros(128, device="cuda"))
    with pytest.raises(TypeError):
        Q.head_norm_rope(Q.HeadRope(f, q_weight=torch.zeros(128, dtype=torch.bfloat16, device="cuda")), h, h, i(2))
    with pytest.raises(ValueError):
        Q.head_norm_rope(Q.HeadRope(f), h, h, i(3))
    with pytest.raises(ValueError):
        Q.head_norm_rope(Q.HeadRope(f), h.transpose(0, 1), h, i(4))
    with pytest.raises(Q.QiftError):
        Q.head_norm_rope(Q.HeadRope(torch.zeros(50, device="cuda"), 100), h, h, i(2))


# ---- together


def test_a_step_of_a_layer(Q):
    """Three steps of a small layer's attention: 8-bit q|k|v projection, plan, norms and rotation, append, attention, a sequence
    that ends.  Codes, sums and slots are the oracle's; the attention is checked against fp64 on the cache that the GPU
    holds (its keys being what head_norm_rope gave, checked on its own)."""
    rng = np.random.default_rng(21)
    B, Hq, Hkv, K, page, width, pages = 3, 4, 2, 256, 16, 6, 14
    N = (Hq + 2 * Hkv) * 128
    w = Q.quantize_weights8(dev(rng.normal(0, 0.05, (N, K)), torch.float32), 256)
    wq, wk = (torch.from_numpy(rng.normal(1, 0.2, 128)).half().cuda() for _ in range(2))
    freq = frequencies(128)
    rope = Q.HeadRope(dev(freq, torch.float32), 128, False, wq, wk)
    cache = Q.KV4Pages.empty(pages, page, Hkv)
    lens, table = dev(np.zeros(B)), dev(np.full((B, width), -1))
    free, depth = dev(rng.permutation(pages)), dev([pages])
    history = [[] for _ in range(B)]     # the slots of each sequence
    Q.device_error()
    for counts in ([20, 1, 7], [1, 1, 1], [1, 30, 2]):
        total = sum(counts)
        rows = total + 2
        x = torch.from_numpy(rng.normal(0, 1, (rows, K))).half()
        act = Q.rotate_quant_act8(x.cuda(), 256)
        codes, s_x = w8.act_quant8(x.numpy(), 256)
        assert np.array_equal(act.q.cpu().numpy(), codes)
        qkv = Q.linear(w, act, workspace=Q.w8a8_workspace(w, rows))
        want = w8.epilogue(olin.int_dot(w.levels.cpu().numpy(), codes), s_x, w.scales.cpu().numpy())
        assert torch.equal(qkv.cpu(), torch.from_numpy(want).half())
        p = Q.kv4_plan_step(lens, dev(counts), table, free, depth, page, rows)
        q, k, v = (t.unflatten(1, (-1, 128)) for t in qkv.split([Hq * 128, Hkv * 128, Hkv * 128], dim=1))
        before = q.cpu().clone()
        Q.head_norm_rope(rope, q, k, p.positions, out=(q, k))
        check_rope(q, before, wq.cpu(), 1e-5, freq, p.positions.cpu().numpy(), 128, False)
        Q.kv4_append(cache, k, v, p.slots)
        out = Q.kv4_attention_tree(q, cache, table, p.starts, p.lens, max_nodes=32, max_len=width * page)
        slots, starts = p.slots.cpu().numpy(), p.starts.cpu().numpy()
        assert np.all(slots[total:] == -1)
        for b in range(B):
            history[b] += slots[starts[b]:starts[b + 1]].tolist()
            assert len(history[b]) == int(p.lens[b])
            kh, vh = (t.float().cpu().numpy() for t in Q.kv4_read(cache, dev(history[b]), dtype=torch.float32))
            mine = q[starts[b]:starts[b + 1]].float().cpu().numpy()
            ref = opages.attention(mine, kh, vh, opages.chain(counts[b], len(history[b])))
            S = np.abs(np.linalg.norm(mine, axis=-1)).max() * np.linalg.norm(kh, axis=-1).max() / np.sqrt(128)
            tol = 2.0 ** -11 * np.abs(ref) + (2 * (S + 16) + 15) * 2.0 ** -21 * np.abs(vh).max() + 2.0 ** -25
            assert np.all(np.abs(out[starts[b]:starts[b + 1]].float().cpu().numpy() - ref) <= tol)
        lens, depth = Q.kv4_release(p.lens, dev([0, counts[1] == 30, 0]), table, free, p.free_count, page)
    assert Q.device_error() == 0
    held = [int(e) for b in (0, 2) for e in table.cpu()[b, :-(-int(lens[b]) // page)]]
    assert int(lens[1]) == 0 and sorted(held + free.cpu()[:int(depth)].tolist()) == list(range(pages))


def test_a_captured_decode_step(Q):
    """A decode step of 8-bit projection, plan, norms and rotation, append and attention in one graph, replayed over growing
    sequences with eager steps between: every replay gives what the eager step on a copy of the same state gives."""
    rng = np.random.default_rng(33)
    B, Hq, Hkv, K, page, width, pages = 5, 8, 2, 512, 16, 4, 24
    N = (Hq + 2 * Hkv) * 128
    w = Q.quantize_weights8(dev(rng.normal(0, 0.05, (N, K)), torch.float32), 512)
    wq, wk = (torch.from_numpy(rng.normal(1, 0.2, 128)).half().cuda() for _ in range(2))
    rope = Q.HeadRope(dev(frequencies(96), torch.float32), 96, True, wq, wk)
    work = Q.kv4_attention_tree_workspace(B, Hq, Hkv, 1, width * page)
    x, counts = torch.zeros((B, K), dtype=torch.float16, device="cuda"), dev(np.ones(B))
    ws = Q.w8a8_workspace(w, B)

    class State:
        def __init__(self):
            self.cache = Q.KV4Pages.empty(pages, page, Hkv)
            self.lens, self.table = dev(np.zeros(B)), dev(np.full((B, width), -1))
            self.free, self.depth = dev(np.arange(pages)), dev([pages])

        def step(self):
            act = Q.rotate_quant_act8(x, 512)
            qkv = Q.linear(w, act, workspace=ws)
            q, k, v = (t.unflatten(1, (-1, 128)) for t in qkv.split([Hq * 128, Hkv * 128, Hkv * 128], dim=1))
            p = Q.kv4_plan_step(self.lens, counts, self.table, self.free, self.depth, page, B)
            Q.head_norm_rope(rope, q, k, p.positions, out=(q, k))
            Q.kv4_append(self.cache, k, v, p.slots)
            out = Q.kv4_attention_tree(q, self.cache, self.table, p.starts, p.lens, max_nodes=1, max_len=width * page, workspace=work)
            self.lens.copy_(p.lens)
            self.depth.copy_(p.free_count)
            return out

    a, b = State(), State()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        State().step()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = a.step()
    for i in range(20):
        x.copy_(torch.from_numpy(rng.normal(0, 1, (B, K))))
        counts.copy_(dev(rng.integers(0, 2, B)))
        g.replay()
        want = b.step()
        torch.cuda.synchronize()
        rows = int(counts.sum())
        assert torch.equal(out[:rows], want[:rows]) and torch.equal(a.lens, b.lens) and torch.equal(a.table, b.table)
        assert torch.equal(a.cache.k.codes, b.cache.k.codes) and torch.equal(a.cache.v.scales, b.cache.v.scales)


def test_other_streams(Q):
    """Each call on a stream given to it, several at once on several streams, and on a stream that is current."""
    rng = np.random.default_rng(5)
    rope = Q.HeadRope(dev(frequencies(128), torch.float32))
    streams, results = [torch.cuda.Stream() for _ in range(3)], []
    cases = []
    for _ in range(3):
        q, k = heads_of(rng, 900, 8, torch.float16).cuda(), heads_of(rng, 900, 2, torch.float16).cuda()
        srv = Server(rng, rng.integers(0, 50, 300), 6, 16, 900)
        cases.append((q, k, dev(rng.integers(0, 1000, 900)), [dev(t) for t in (srv.lens, rng.integers(0, 4, 300), srv.table, srv.free)],
                      dev([srv.depth])))
    torch.cuda.synchronize()
    for s, (q, k, pos, (lens, counts, table, free), depth) in zip(streams, cases):
        y = Q.head_norm_rope(rope, q, k, pos, stream=s)
        p = Q.kv4_plan_step(lens, counts, table, free, depth, 16, 1000, stream=s)
        r = Q.kv4_release(p.lens, torch.zeros_like(counts), table, free, p.free_count, 16, stream=s)
        results.append((y, p, r))
    torch.cuda.synchronize()
    for (y, p, r), (q, k, pos, (lens, counts, table, free), depth) in zip(results, cases):
        y2 = Q.head_norm_rope(rope, q, k, pos)
        assert torch.equal(y[0], y2[0]) and torch.equal(y[1], y2[1])
        p2 = Q.kv4_plan_step(lens, counts, table, free, depth, 16, 1000)    # the pages taken are the same again
        assert torch.equal(p.starts, p2.starts) and torch.equal(p.positions, p2.positions) and torch.equal(p.lens, p2.lens)
        assert torch.equal(p.slots, p2.slots) and torch.equal(p.free_count, p2.free_count)
        assert torch.equal(r[0], p.lens) and torch.equal(r[1], p.free_count)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_large_frequencies(Q, dtype, pairs):
    """Angles that fp64 does not hold, up to 2^40; NaN in the pairs past that and nowhere else."""
    rng = np.random.default_rng(31)
    pos = np.array([0, 1, 1000, 100000, 523018516, 1639311774, 2142287670, I31])
    q, k = heads_of(rng, len(pos), 3, dtype), heads_of(rng, len(pos), 2, dtype)
    freq = np.exp(rng.uniform(-8, 6.2, 64)).astype(np.float32)
    freq[:4] = 2.6565, 96.7, -511.9, 0.0
    rope = Q.HeadRope(dev(freq, torch.float32), 128, pairs)
    yq, yk = Q.head_norm_rope(rope, q.cuda(), k.cuda(), dev(pos))
    check_rope(yq, q, None, 1.0, freq, pos, 128, pairs)
    check_rope(yk, k, None, 1.0, freq, pos, 128, pairs)
    wide = freq.copy()
    wide[5], wide[9], wide[12], wide[13] = 1e9, np.inf, np.nan, 1e30
    y = Q.head_norm_rope(Q.HeadRope(dev(wide, torch.float32), 128, pairs), q.cuda(), k.cuda(), dev(pos))[0]
    with np.errstate(invalid="ignore"):
        lost = ~(np.abs(pos[:, None].astype(np.float64) * wide.astype(np.float64)[None, :]) < 2.0 ** 40)   # (none beside the border)
    values = np.zeros((len(pos), 128), bool)
    i = np.arange(64)
    for at in ((2 * i, 2 * i + 1) if pairs else (i, i + 64)):
        values[:, at] = lost
    gone = torch.from_numpy(values)[:, None, :].expand(-1, 3, -1)
    assert torch.equal(torch.isnan(y.cpu()), gone)
    same = np.abs(freq - wide) == 0
    keep = np.zeros(128, bool)
    for at in ((2 * i, 2 * i + 1) if pairs else (i, i + 64)):
        keep[at] = same
    assert torch.equal(y.cpu()[:, :, torch.from_numpy(keep)], yq.cpu()[:, :, torch.from_numpy(keep)])


def test_a_step_that_leaves_a_sequence_out(Q):
    """The others' outputs are those of a step without it; its rows are told by their positions, and it by its length."""
    rng = np.random.default_rng(41)
    B, Hq, Hkv, page, width, out_at = 5, 8, 2, 16, 6, 2
    cached, counts = np.array([40, 3, 33, 0, 70]), np.array([2, 1, 30, 5, 1])
    s = Server(rng, cached, width, page, 6)
    counts[out_at] = width * page - cached[out_at] + 1      # one more than its row of the table holds
    rows = int(counts.sum()) + 3
    rope = Q.HeadRope(dev(frequencies(128), torch.float32))
    n = len(s.free) * page
    fill = [torch.from_numpy(rng.normal(0, 1, (n, Hkv, 128))).half().cuda() for _ in range(2)]
    new = [torch.from_numpy(rng.normal(0, 1, (rows, h, 128))).half().cuda() for h in (Hq, Hkv, Hkv)]
    results = []
    for without in (False, True):
        cache = Q.KV4Pages.empty(len(s.free), page, Hkv)
        Q.kv4_append(cache, *fill, dev(np.arange(n)))
        table, free = dev(s.table), dev(s.free)
        c = counts.copy()
        c[out_at] = 0 if without else c[out_at]
        Q.device_error()
        p = Q.kv4_plan_step(dev(s.lens), dev(c), table, free, dev([s.depth]), page, rows)
        assert Q.device_error() == (0 if without else Q.DEVERR_INDEX)
        starts, pos, lens = (t.cpu().numpy() for t in (p.starts, p.positions, p.lens))
        # the same tokens, at the rows that the step gives them
        take = np.zeros(rows, np.int64)
        first = np.concatenate([[0], np.cumsum(counts)])
        for b in range(B):
            take[starts[b]:starts[b + 1]] = first[b] + np.arange(c[b])
        q, k, v = (t[torch.from_numpy(take).cuda()].contiguous() for t in new)
        q, k = Q.head_norm_rope(rope, q, k, p.positions)
        Q.kv4_append(cache, k, v, p.slots)
        out = Q.kv4_attention_tree(q, cache, table, p.starts, p.lens, max_nodes=64, max_len=width * page)
        assert Q.device_error() == 0
        served = lens == cached + c
        assert served.tolist() == [b != out_at or without for b in range(B)] and lens[out_at] == cached[out_at]
        for b in range(B):
            assert np.all((pos[starts[b]:starts[b + 1]] >= 0) == served[b])
        results.append([out[starts[b]:starts[b + 1]] for b in range(B) if b != out_at] + [p.free_count, table])
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_steps_on_several_streams(Q):
    """Plan, norms and release of three servers, each on a stream of its own; everything that the calls read is made, and waited
    for, before the first of them, and kept until the last is done."""
    rng = np.random.default_rng(6)
    rope = Q.HeadRope(dev(frequencies(128), torch.float32))
    streams, cases, results = [torch.cuda.Stream() for _ in range(3)], [], []
    for _ in streams:
        q, k = heads_of(rng, 900, 8, torch.float16).cuda(), heads_of(rng, 900, 2, torch.float16).cuda()
        srv = Server(rng, rng.integers(0, 50, 300), 6, 16, 900)
        counts, done = rng.integers(0, 4, 300), rng.integers(0, 2, 300)
        cases.append((srv, counts, done, q, k, [dev(t) for t in (srv.lens, counts, done, srv.table, srv.free, [srv.depth])]))
    torch.cuda.synchronize()
    for s, (_, _, _, q, k, (lens, counts, done, table, free, depth)) in zip(streams, cases):
        p = Q.kv4_plan_step(lens, counts, table, free, depth, 16, 900, stream=s)
        y = Q.head_norm_rope(rope, q, k, p.positions, stream=s)
        r = Q.kv4_release(p.lens, done, table, free, p.free_count, 16, stream=s)
        results.append((p, y, r))
    torch.cuda.synchronize()
    for (p, y, r), (srv, counts, done, q, k, (_, _, _, table, free, _)) in zip(results, cases):
        want = ostep.plan(srv.lens, counts, srv.table, srv.free, srv.depth, 16, 900)
        assert np.array_equal(p.slots.cpu().numpy(), want[3]) and np.array_equal(p.positions.cpu().numpy(), want[4])
        assert np.array_equal(table.cpu().numpy(), want[2])
        back = ostep.release(want[1], done, want[2], srv.free, want[5], 16)
        assert np.array_equal(r[0].cpu().numpy(), back[0]) and np.array_equal(free.cpu().numpy(), back[1]) and int(r[1]) == back[2]
        again = Q.head_norm_rope(rope, q, k, p.positions)
        assert torch.equal(y[0], again[0]) and torch.equal(y[1], again[1])
