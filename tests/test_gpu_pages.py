"""The paged KV4 cache on the GPU against the oracle: what qift_kv4_append writes, what qift_kv4_read gives back and
qift_kv4_attention_tree over the pages.

Codes, scales and zero-points are decided in fp32 in a fixed order on both sides, so they must be equal bit for bit; the
values s (q - z) have one rounding from fp32, which is the same on both sides too.

Attention, per query head, against fp64 on the same cache: |y - ref| <= h |ref| + e, h the half step of the output's type
(fp16 2^-11, bf16 2^-8; and 2^-25 for fp16 outputs below the normal numbers) and e the arithmetic's part:
  scores are sums of 128 exact products in fp32 (the MFMA's sums are within 2^-22 of the sum of |products|, which is at
  most S = |q| |k| / sqrt(128) for the score where zero-points are taken off the codes first; where 64 + z is taken off
  sums of 64 + code, five roundings of partial sums of about 64 |q| s, (5 / 16) 7 |q| s 2^-21, which stays under S of
  keys that fill their codes, |k| about 4 s sqrt(128)); the scale, the factor to powers of two and log2 of the value's scale
  (L the largest |log2 s|) each round once more, as do the logarithm, the exponential and the reciprocal: in all a
  weight is off by at most (S + L) 2^-21 + 2^-21 relative, and the output by twice that times max |v|;
  weights are held to 2^-21, and sums of T / 32 matrix instructions in fp32: (2^-21 + T / 32 * 2^-24) max |v|.
"""
import numpy as np
import pytest
import torch

from oracle import kv4 as okv4, pages as opages

pytestmark = pytest.mark.gpu

HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
NP = {torch.float16: np.float16}


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_02823_amd import qift
    qift.lib()
    return qift


def tensor(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def values(t):
    return t.detach().float().cpu().numpy()


def draw_groups(rng, n, heads, dtype):
    """Keys or values with what the quantizer meets: outliers, one-sided vectors, zeros, tiny ones, ties."""
    x = rng.normal(0, 1, (n * heads, 128))
    x[::5] *= rng.uniform(0.001, 30, (len(x[::5]), 1))
    x[1::7] = np.abs(x[1::7])
    x[2::7] = -np.abs(x[2::7])
    x[3::11] = 0.0
    x[4::13] *= 1e-6
    x[5::17, 3] = 900.0
    x[6::19] = np.round(rng.uniform(-15, 15, (len(x[6::19]), 128))) * 0.5
    if dtype == torch.bfloat16:
        x[7::23] *= 1e-38          # steps among fp32's subnormals
        x[8::29] *= 8e34          # up to 7.2e37, below 2^126
    return torch.from_numpy(x.reshape(n, heads, 128)).to(dtype)


def cache_of(Q, rng, pages, page, Hkv, stale=True):
    """A cache with what an earlier use left in it."""
    side = lambda: Q.KV4(torch.from_numpy(rng.integers(0, 256, (pages, Hkv, page, 64)).astype(np.uint8)).cuda(),  # noqa: E731
                         torch.from_numpy(rng.uniform(0.1, 2, (pages, Hkv, page)).astype(np.float32)).cuda(),
                         torch.from_numpy(rng.integers(0, 16, (pages, Hkv, page)).astype(np.uint8)).cuda())
    return Q.KV4Pages(side(), side())


def unpack(codes):
    c = codes.cpu().numpy()
    return np.stack((c & 15, c >> 4), axis=-1).reshape(*c.shape[:-1], 128)


def host(side):
    return unpack(side.codes), side.scales.cpu().numpy(), side.zeros.cpu().numpy()


def same_cache(side, want):
    codes, scales, zeros = host(side)
    assert np.array_equal(scales.view(np.uint32), want[1].view(np.uint32))
    assert np.array_equal(zeros, want[2])
    assert np.array_equal(codes, want[0])


APPEND = [(1, 8, 64), (2, 1, 16), (3, 3, 48), (15, 8, 16), (16, 2, 32), (17, 32, 128), (61, 5, 64), (130, 8, 256)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("n,Hkv,page", APPEND)
def test_append_then_read(Q, n, Hkv, page, dtype):
    rng = np.random.default_rng(n * 1000 + Hkv)
    pages = -(-n // page) + 3
    cache = cache_of(Q, rng, pages, page, Hkv)
    before = host(cache.k), host(cache.v)
    slots = rng.permutation(pages * page)[:n].astype(np.int32)
    if n > 2:
        slots[-1], slots[n // 2] = -1, -7
    k, v = (draw_groups(rng, n, Hkv, dtype) for _ in range(2))
    # parts of stacked rows: the middle of a wider matrix, 16-byte aligned
    wide = torch.full((n, 64 + 2 * Hkv * 128 + 8), float("nan"), dtype=dtype)
    wide[:, 64:64 + Hkv * 128] = k.reshape(n, -1)
    wide[:, 64 + Hkv * 128:64 + 2 * Hkv * 128] = v.reshape(n, -1)
    wide = wide.cuda()
    kd, vd = wide[:, 64:64 + Hkv * 128].unflatten(1, (Hkv, 128)), wide[:, 64 + Hkv * 128:64 + 2 * Hkv * 128].unflatten(1, (Hkv, 128))
    got = Q.kv4_append(cache, kd, vd, tensor(slots), values=True)
    torch.cuda.synchronize()
    for side, was, x, y in ((cache.k, before[0], k, got[0]), (cache.v, before[1], v, got[1])):
        *want, hat = opages.append(*was, values(x), slots)
        same_cache(side, want)
        ref = torch.from_numpy(hat).to(dtype)
        assert y.dtype == dtype and torch.equal(y.cpu(), ref)
    # reading back gives the same values, in each type; padding zeros
    for out in (torch.float16, torch.bfloat16, torch.float32):
        back = Q.kv4_read(cache, tensor(slots), dtype=out)
        for side, y in ((cache.k, back[0]), (cache.v, back[1])):
            ref = torch.from_numpy(opages.read(*host(side), slots)).to(out)
            assert y.dtype == out and torch.equal(y.cpu(), ref)
    assert Q.device_error() == 0


def test_append_without_values_is_kv4_quant(Q):
    rng = np.random.default_rng(1)
    n, Hkv, page = 40, 4, 16
    cache = cache_of(Q, rng, 3, page, Hkv)
    k, v = (draw_groups(rng, n, Hkv, torch.float16).cuda() for _ in range(2))
    assert Q.kv4_append(cache, k, v, torch.arange(n, dtype=torch.int32, device="cuda")) is None
    for x, side in ((k, cache.k), (v, cache.v)):
        c = Q.kv4_quant(x)
        for name in ("codes", "scales", "zeros"):
            dense = getattr(c, name)                                    # [n, Hkv, ...]
            paged = getattr(side, name).transpose(1, 2).flatten(0, 1)[:n]
            assert torch.equal(paged, dense), name


def test_append_and_read_leave_out_what_is_no_slot(Q):
    rng = np.random.default_rng(2)
    pages, page, Hkv = 2, 16, 2
    cache = cache_of(Q, rng, pages, page, Hkv)
    before = host(cache.k), host(cache.v)
    slots = np.array([3, 32, 2 ** 31 - 1, -2 ** 31, 31], dtype=np.int32)   # 32 slots: 0 .. 31
    k, v = (draw_groups(rng, 5, Hkv, torch.float16) for _ in range(2))
    assert Q.device_error() == 0
    got = Q.kv4_append(cache, k.cuda(), v.cuda(), tensor(slots), values=True)
    assert Q.device_error() == Q.DEVERR_INDEX
    for side, was, x, y in ((cache.k, before[0], k, got[0]), (cache.v, before[1], v, got[1])):
        *want, hat = opages.append(*was, values(x), slots)
        same_cache(side, want)
        assert np.array_equal(values(y), hat.astype(np.float16).astype(np.float32))
    back = Q.kv4_read(cache, tensor(slots), dtype=torch.float32)
    assert Q.device_error() == Q.DEVERR_INDEX
    assert np.array_equal(values(back[0]), opages.read(*host(cache.k), slots))
    # negative slots are padding and no error; one slot read many times is fine
    back = Q.kv4_read(cache, tensor(np.array([-1, 5, 5, 5], dtype=np.int32)))
    assert not back[0][0].any() and torch.equal(back[1][1], back[1][3]) and Q.device_error() == 0


def test_nothing_to_do(Q):
    cache = Q.KV4Pages.empty(2, 16, 2)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    x = torch.empty((0, 2, 128), dtype=torch.float16, device="cuda")
    assert Q.kv4_append(cache, x, x, none, values=True)[0].shape == (0, 2, 128)
    assert Q.kv4_read(cache, none)[1].shape == (0, 2, 128)
    y = Q.kv4_attention_tree(torch.empty((0, 4, 128), dtype=torch.float16, device="cuda"), cache,
                             torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"),
                             torch.zeros(1, dtype=torch.int32, device="cuda"), max_nodes=1, max_len=16)
    assert y.shape == (0, 4, 128)


# ---- attention -------------------------------------------------------------------------------------------------------


def random_tree(rng, n):
    mask = np.eye(n, dtype=bool)
    for i in range(1, n):
        mask[i] |= mask[int(rng.random() ** 1.5 * i)]
    return mask


class Case:
    """Sequences of given (nodes, cached tokens) with random pages, and the attention of their nodes in fp64."""

    def __init__(self, Q, seed, seqs, Hq, Hkv, page, dtype, masks=None, gain=1.0, spare_rows=0, spare_entries=1, kscale=1.0,
                 vscale=None):
        rng = np.random.default_rng(seed)
        self.rng, self.seqs, self.Hq, self.Hkv, self.dtype = rng, seqs, Hq, Hkv, dtype
        counts = [-(-t // page) for _, t in seqs]
        self.pages, self.page = sum(counts) + 2, page
        perm = rng.permutation(self.pages)
        width = max(max(counts), 1) + spare_entries
        self.table = np.full((len(seqs), width), -1, dtype=np.int32)
        self.cache = cache_of(Q, rng, self.pages, page, Hkv)
        at = 0
        self.k, self.v, self.scales = [], [], []
        for b, (_, t) in enumerate(seqs):
            self.table[b, :counts[b]] = perm[at:at + counts[b]]
            at += counts[b]
            if t == 0:
                self.k.append(np.zeros((0, Hkv, 128), np.float32))
                self.v.append(np.zeros((0, Hkv, 128), np.float32))
                self.scales.append(np.zeros((0, Hkv), np.float32))
                continue
            slots = self.slots(b, np.arange(t))
            x = rng.normal(0, kscale, (t, Hkv, 128)) * np.exp(rng.normal(0, 0.5, (t, Hkv, 1)))
            y = rng.normal(0, 1, (t, Hkv, 128)) * np.exp(rng.normal(0, 0.3, (t, Hkv, 1)))
            if vscale is not None:
                y *= vscale
            x[::37, :, 5] = 20.0 * kscale
            y[::41] = 0.0
            Q.kv4_append(self.cache, tensor(x.astype(np.float32), dtype), tensor(y.astype(np.float32), dtype), tensor(slots))
            self.k.append(opages.read(*host(self.cache.k), slots))
            self.v.append(opages.read(*host(self.cache.v), slots))
            self.scales.append(self.cache.v.scales.cpu().numpy()[slots // page, :, slots % page])
        self.rows = sum(n for n, _ in seqs) + spare_rows
        self.starts = np.concatenate([[0], np.cumsum([n for n, _ in seqs])]).astype(np.int32)
        self.lens = np.array([t for _, t in seqs], dtype=np.int32)
        q = rng.normal(0, gain, (self.rows, Hq, 128)) * rng.uniform(0.2, 3, (self.rows, Hq, 1))
        self.q = torch.from_numpy(q).to(dtype)
        self.max_nodes = max(n for n, _ in seqs)
        self.masks = masks

    def slots(self, b, t):
        return (self.table[b, t // self.page] * self.page + t % self.page).astype(np.int32)

    def seen(self, b):
        n, t = self.seqs[b]
        return opages.chain(n, t) if self.masks is None else opages.tree(self.masks[b], t)

    def visible(self, max_nodes):
        if self.masks is None:
            return None
        w = np.zeros((self.rows, -(-max_nodes // 64)), dtype=np.int64)
        for b, m in enumerate(self.masks):
            w[self.starts[b]:self.starts[b + 1]] = opages.pack_mask(m, max_nodes)
        return tensor(w)

    def run(self, Q, max_nodes=None, max_len=None, **kw):
        max_nodes = max_nodes or self.max_nodes
        max_len = max_len or max(1, int(self.lens.max()))
        return Q.kv4_attention_tree(self.q.cuda(), self.cache, tensor(self.table), tensor(self.starts), tensor(self.lens),
                                    max_nodes=max_nodes, max_len=max_len, visible=self.visible(max_nodes), **kw)

    def reference(self, b):
        return opages.attention(values(self.q[self.starts[b]:self.starts[b + 1]]), self.k[b], self.v[b], self.seen(b))

    def check(self, y, label="", only=None):
        y = values(y).astype(np.float64)
        worst = 0.0
        for b, (n, t) in enumerate(self.seqs):
            if only is not None and b not in only:
                continue
            got, ref = y[self.starts[b]:self.starts[b + 1]], self.reference(b)
            if n == 0:
                continue
            q, G = values(self.q[self.starts[b]:self.starts[b + 1]]).astype(np.float64), self.Hq // self.Hkv
            kn = np.linalg.norm(self.k[b].astype(np.float64), axis=-1).max(axis=0) if t else np.zeros(self.Hkv)
            vmax = np.abs(self.v[b]).max(axis=(0, 2)) if t else np.zeros(self.Hkv)
            S = np.linalg.norm(q, axis=-1) * np.repeat(kn, G)[None] / np.sqrt(128.0)
            L = np.abs(np.log2(np.maximum(self.scales[b], 2.0 ** -90))).max() if t else 0.0
            e = (2 * (S + L + 1) * 2.0 ** -21 + 2.0 ** -21 + t / 32 * 2.0 ** -24) * np.repeat(vmax, G)[None]
            if self.dtype == torch.float16:
                e = e + 2.0 ** -25
            limit = HALF[self.dtype] * np.abs(ref) + e[..., None]
            assert np.isfinite(got).all(), (label, b)
            over = np.abs(got - ref) / np.maximum(limit, 1e-300)   # (a limit of 0: equal)
            worst = max(worst, float(over.max()))
            assert over.max() <= 1.0, (label, b, n, t, float(over.max()))
        print(f"{label} worst error {worst:.3f} of the limit", flush=True)


SHAPES = [   # (sequences of (nodes, tokens), Hq, Hkv, page)
    ([(1, 1)], 32, 8, 16),
    ([(1, 2), (1, 63), (1, 64), (1, 65)], 8, 2, 16),
    ([(1, 255), (1, 256), (1, 257), (1, 1000)], 32, 8, 64),
    ([(1, 4097)], 32, 8, 128),
    ([(1, 700), (1, 3)], 4, 4, 48),
    ([(1, 300)], 16, 1, 32),
    ([(1, 520)], 64, 1, 16),
    ([(5, 5), (5, 6), (5, 69)], 32, 32, 16),
    ([(3, 130), (0, 40), (7, 777), (1, 0), (2, 513)], 24, 8, 64),
    ([(17, 17), (33, 1200)], 32, 8, 256),
    ([(64, 64), (37, 2300), (1, 190)], 32, 8, 64),
    ([(65, 400), (63, 63), (128, 129)], 8, 2, 32),
    ([(256, 256), (200, 1100)], 8, 2, 64),
    ([(4, 5000)], 8, 1, 16),
]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("masked", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(f"{n}.{t}" for n, t in s[0]) + f"_h{s[1]}.{s[2]}_p{s[3]}")
def test_attention(Q, shape, masked, dtype):
    seqs, Hq, Hkv, page = shape
    seed = sum((i + 3) * (7 * n + t) for i, (n, t) in enumerate(seqs)) + Hq
    rng = np.random.default_rng(seed + 1)
    masks = [random_tree(rng, n) for n, _ in seqs] if masked else None
    if masked and seqs[-1] == (1, 0):
        masks[-1][:] = False
    c = Case(Q, seed, seqs, Hq, Hkv, page, dtype, masks)
    c.check(c.run(Q), "as sized")
    # a launch made for more nodes and longer sequences gives the same rows
    c.check(c.run(Q, max_nodes=min(256, c.max_nodes + 70), max_len=int(c.lens.max()) + 3000), "roomier")
    assert Q.device_error() == 0


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["fp16", "bf16"])
def test_sharp_scores(Q, dtype):
    """Scores in the hundreds, where a lost bit of a score shows in the result."""
    c = Case(Q, 77, [(9, 900), (1, 300)], 32, 8, 64, dtype, gain=8.0)
    c.check(c.run(Q), "sharp")


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["fp16", "bf16"])
def test_queries_of_every_size(Q, dtype):
    """Rows far below and above 1, some of one value alone and some of one sign, among ordinary ones."""
    rng = np.random.default_rng(7)
    for n, t in ((1, 300), (12, 700), (40, 1500)):
        c = Case(Q, 110 + n, [(n, t)], 16, 4, 64, dtype)
        size = 10.0 ** rng.uniform(-6 if dtype == torch.float16 else -30, 2, (n, 16, 1))
        size[::3] = 1.0
        q = values(c.q) * size
        q[:, 3, 1:] = 0.0
        q[:, 7] = np.abs(q[:, 7])
        q[:, 11] = 0.0
        c.q = torch.from_numpy(q).to(dtype)
        c.check(c.run(Q), f"{n} rows of any size")


@pytest.mark.parametrize("vscale", [1e-6, 3e3])
def test_scale_of_the_values(Q, vscale):
    for dtype in (torch.float16, torch.bfloat16):
        c = Case(Q, 78, [(3, 500)], 16, 4, 32, dtype, vscale=vscale)
        c.check(c.run(Q), f"values x {vscale}")
    c = Case(Q, 79, [(2, 300)], 16, 4, 32, torch.bfloat16, kscale=1e-30, vscale=1e30)
    c.check(c.run(Q), "bf16 far from 1")
    c = Case(Q, 80, [(2, 300)], 16, 4, 32, torch.bfloat16, vscale=1e-20)   # with vectors of zeros, of scale 1, among them
    c.check(c.run(Q), "bf16 tiny")


def test_values_whose_scale_grows_along_the_sequence(Q):
    vs = np.exp(np.linspace(-9, 6, 3000))[:, None, None]
    c = Case(Q, 81, [(2, 3000)], 16, 4, 64, torch.float16, vscale=vs)
    c.check(c.run(Q), "growing")


def test_value_scales_of_every_size_in_one_sequence(Q):
    """Neighbouring tokens' value scales up to 2^166 apart: the large ones decide the sums, all count for the weights."""
    rng = np.random.default_rng(5)
    vs = 10.0 ** rng.choice([-25, -12, 0, 12, 25], size=(1700, 4, 1))
    for nodes in (1, 9):
        c = Case(Q, 93 + nodes, [(nodes, 1700)], 16, 4, 64, torch.bfloat16, vscale=vs)
        c.check(c.run(Q), f"mixed, {nodes} nodes")
        # far scales in the last tokens only: what a wave summed before them stands
        c = Case(Q, 95 + nodes, [(nodes, 1700)], 16, 4, 64, torch.bfloat16, vscale=np.where(np.arange(1700) < 1650, 1.0, 1e-22)[:, None, None])
        c.check(c.run(Q), f"far ones last, {nodes} nodes")


def test_many_sequences_of_any_length(Q):
    """Shares that hold several sequences, ends and beginnings of others, and none of a sequence without nodes; and more
    sequences than are dealt out, a workgroup to each."""
    rng = np.random.default_rng(6)
    lens = [int(t) for t in np.r_[rng.integers(1, 300, 40), 2300, 1, 0, rng.integers(200, 1100, 20), 4000]]
    seqs = [(0 if b % 7 == 3 else min(t, 1 + b % 3), t) for b, t in enumerate(lens)]
    c = Case(Q, 97, seqs, 32, 8, 32, torch.float16)
    c.check(c.run(Q), "ragged")
    seqs = [(min(t, 1 + b % 2), t) for b, t in enumerate(int(t) for t in rng.integers(0, 330, 530))]
    c = Case(Q, 98, seqs, 4, 1, 16, torch.bfloat16)
    c.check(c.run(Q), "a workgroup each")
    c = Case(Q, 99, seqs[:510], 4, 1, 16, torch.bfloat16)
    c.check(c.run(Q), "short, a workgroup each")
    c.check(c.run(Q, max_len=2000), "short, dealt out")
    c = Case(Q, 102, seqs[:400] + [(3, 1700)], 4, 1, 16, torch.float16)
    c.check(c.run(Q), "one long, dealt out")
    assert Q.device_error() == 0


def test_scores_far_from_zero(Q):
    """One seen token is the whole softmax whatever its score: here past -1e31, and past 1e31."""
    only = np.array([[False, True], [False, True]])
    c = Case(Q, 100, [(2, 2)] * 6, 8, 2, 16, torch.bfloat16, [only] * 6)
    rows = lambda x: torch.from_numpy(np.stack([t[1] for t in x for _ in range(2)])).repeat_interleave(4, dim=1)  # noqa: E731
    ref = rows(c.v)
    assert ref.any(dim=-1).all()
    for sign in (-1.0, 1.0):
        c.q = (sign * 1e32 * rows(c.k)).to(torch.bfloat16)          # a score of sign |k|^2 1e32 / sqrt(128)
        y = c.run(Q).float().cpu()
        assert (y - ref).abs().le(ref.abs() * (2.0 ** -8 + 2.0 ** -20)).all(), sign


def test_a_scale_that_is_nan_shows_where_it_is_seen(Q):
    """Node 4 of a chain has a NaN value scale in one KV head: rows 4 and on are NaN in that head's group, no other."""
    for t in (60, 1500):
        c = Case(Q, 101, [(9, t)], 16, 4, 64, torch.float16)
        want = c.run(Q)
        slot = int(c.slots(0, np.array([t - 5]))[0])
        c.cache.v.scales[slot // 64, 2, slot % 64] = float("nan")
        got = c.run(Q)
        assert torch.isnan(got[4:, 8:12]).all()
        keep = torch.ones((9, 16), dtype=torch.bool, device="cuda")
        keep[4:, 8:12] = False
        assert torch.equal(got[keep], want[keep])


def test_rows_that_see_nothing_and_rows_behind_the_last(Q):
    rng = np.random.default_rng(3)
    masks = [random_tree(rng, 6), random_tree(rng, 4), np.zeros((3, 3), dtype=bool)]
    masks[0][2] = False                         # sees nothing: its sequence has no tokens before the nodes
    masks[1][1] = False                         # sees the context alone
    c = Case(Q, 82, [(6, 6), (4, 300), (3, 3)], 32, 8, 16, torch.float16, masks, spare_rows=5)
    out = torch.full((c.rows, 32, 128), 7.0, dtype=torch.float16, device="cuda")
    y = c.run(Q, out=out)
    c.check(y, "empty rows")
    assert not y[2].any() and not y[10:13].any()
    assert (y[13:] == 7.0).all()
    assert Q.device_error() == 0


@pytest.mark.parametrize("seqs", [[(5, 70), (7, 23)], [(5, 2070), (7, 1023)]], ids=["one chunk", "chunks"])
@pytest.mark.parametrize("bad", [float("inf"), float("nan"), -float("inf"), 65504.0])
def test_what_is_not_seen_does_not_count(Q, bad, seqs):
    """Unseen nodes, slots behind a sequence's end and other sequences' pages hold infinities and NaN."""
    rng = np.random.default_rng(4)
    masks = [random_tree(rng, n) for n, _ in seqs]
    for m in masks:
        m[:, 3] = False                          # nobody sees node 3
    c = Case(Q, 83, seqs, 16, 4, 48, torch.float16, masks)
    want = c.run(Q)
    used = np.zeros(c.pages * c.page, dtype=bool)
    for b, (n, t) in enumerate(seqs):
        used[c.slots(b, np.arange(t))] = True
        used[c.slots(b, np.array([t - n + 3]))] = False
    dead = torch.from_numpy(~used.reshape(c.pages, c.page)).cuda()
    for side in (c.cache.k, c.cache.v):
        side.scales.masked_fill_(dead[:, None, :].expand_as(side.scales), bad)
        side.zeros.masked_fill_(dead[:, None, :].expand_as(side.zeros), 255)
    got = c.run(Q)
    assert torch.equal(got, want)
    c.check(got, f"poisoned with {bad}")


def test_a_row_with_nan_keeps_it_to_itself(Q):
    c = Case(Q, 84, [(9, 500)], 16, 4, 64, torch.float16)
    want = c.run(Q)
    c.q[4, 7] = float("nan")
    got = c.run(Q)
    assert torch.isnan(got[4, 7]).all()
    keep = torch.ones((9, 16), dtype=torch.bool, device="cuda")
    keep[4, 7] = False
    assert torch.equal(got[keep], want[keep])


def test_bad_tables_counts_and_lengths(Q):
    """Entries that name no page are not seen, counts and lengths come back into range; the error word says so."""
    c = Case(Q, 85, [(3, 400), (2, 300)], 16, 4, 32, torch.float16)
    good_table = c.table.copy()
    assert Q.device_error() == 0
    for entry in (c.pages, 2 ** 31 - 1, -1, -2 ** 31):
        c.table = good_table.copy()
        c.table[0, 4] = entry                    # tokens 128 .. 159 of sequence 0
        y = c.run(Q)
        assert Q.device_error() == Q.DEVERR_INDEX
        lost = c.seen(0)
        lost[:, 128:160] = False
        ref = opages.attention(values(c.q[:3]), c.k[0], c.v[0], lost)
        assert np.abs(values(y[:3]) - ref).max() <= 2e-3 * np.abs(ref).max()
        c.check(y, "the other sequence", only=(1,))
    c.table = good_table
    # more nodes than the launch was made for: the first ones are served, the others' rows left alone
    out = torch.full((c.rows, 16, 128), 7.0, dtype=torch.float16, device="cuda")
    y = c.run(Q, max_nodes=2, out=out)
    assert Q.device_error() == Q.DEVERR_INDEX
    assert (y[2] == 7.0).all()
    c.check(y, "two nodes", only=(1,))
    # lengths past the limit, or negative
    lens = c.lens.copy()
    for bad in (2 ** 31 - 1, -5):
        c.lens = lens.copy()
        c.lens[0] = bad
        y = c.run(Q, max_len=400)
        assert Q.device_error() == Q.DEVERR_INDEX
        assert bad > 0 or not y[:3].any()        # nothing is cached: nothing to see
        c.check(y, "the other sequence", only=(1,))
    c.lens = lens
    # starts outside the rows
    starts = c.starts.copy()
    for s in ([0, 3, 2 ** 31 - 1], [-4, 3, 5], [0, 5, 3]):
        c.starts = np.array(s, dtype=np.int32)
        c.run(Q)
        assert Q.device_error() == Q.DEVERR_INDEX
    c.starts = starts
    c.check(c.run(Q), "in order again")
    assert Q.device_error() == 0


def test_shared_pages(Q):
    """Two sequences with a common prefix: the same pages in both rows of the table."""
    c = Case(Q, 86, [(2, 400), (2, 400)], 16, 4, 32, torch.float16)
    prefix = 5
    c.table[1, :prefix] = c.table[0, :prefix]
    c.k[1][:160], c.v[1][:160] = c.k[0][:160], c.v[0][:160]
    c.check(c.run(Q), "shared prefix")


def test_strided_queries(Q):
    c = Case(Q, 87, [(4, 200), (1, 90)], 16, 4, 32, torch.bfloat16)
    want = c.run(Q)
    wide = torch.full((c.rows, 5, 16 * 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 2] = c.q.reshape(c.rows, -1).cuda()
    view = wide[:, 2].unflatten(1, (16, 128))
    got = Q.kv4_attention_tree(view, c.cache, tensor(c.table), tensor(c.starts), tensor(c.lens), max_nodes=4, max_len=200)
    assert torch.equal(got, want)


def test_same_call_same_bits(Q):
    c = Case(Q, 88, [(37, 5000), (1, 3000)], 32, 8, 64, torch.float16)
    first = c.run(Q)
    for _ in range(3):
        assert torch.equal(c.run(Q), first)


def test_stale_workspace(Q):
    c = Case(Q, 89, [(9, 3000), (2, 10)], 32, 8, 64, torch.float16)
    ws = Q.kv4_attention_tree_workspace(2, 32, 8, 9, 3000)
    assert ws.numel() > 16
    first = c.run(Q, workspace=ws)
    for fill in (0xFF, 0x7F, 0):
        ws.fill_(fill)
        assert torch.equal(c.run(Q, workspace=ws), first)


def test_refusals_of_the_binding(Q):
    c = Case(Q, 90, [(2, 100)], 16, 4, 32, torch.float16)
    q, t, s, n = c.q.cuda(), tensor(c.table), tensor(c.starts), tensor(c.lens)
    call = lambda q=q, t=t, s=s, n=n, **kw: Q.kv4_attention_tree(q, c.cache, t, s, n, **dict(dict(max_nodes=2, max_len=100), **kw))  # noqa: E731
    for kw, err in ((dict(q=q.float()), TypeError), (dict(q=q[:, :15]), Q.QiftError), (dict(q=q.transpose(1, 2)), ValueError),
                    (dict(q=q.cpu()), TypeError), (dict(t=t.long()), TypeError), (dict(t=t[0]), ValueError), (dict(s=s[:-1]), ValueError),
                    (dict(n=n.long()), TypeError), (dict(visible=torch.zeros(2, 2, dtype=torch.int64, device="cuda")), ValueError),
                    (dict(max_nodes=0), Q.QiftError), (dict(max_nodes=257), Q.QiftError), (dict(max_len=0), Q.QiftError),
                    (dict(out=torch.empty_like(q).float()), TypeError),
                    (dict(max_len=5000, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), Q.QiftError)):
        with pytest.raises(err):
            call(**kw)
    k = torch.zeros((3, 4, 128), dtype=torch.float16, device="cuda")
    slots = torch.zeros(3, dtype=torch.int32, device="cuda")
    for args, err in (((k, k, slots.long()), TypeError), ((k, k[:2], slots), ValueError), ((k, k.bfloat16(), slots), TypeError),
                      ((k.float(), k.float(), slots), TypeError), ((k[:, :3], k[:, :3], slots), ValueError),
                      ((k[:1].expand(3, 4, 128), k, slots), Q.QiftError), ((k, k, slots[:2]), ValueError)):
        with pytest.raises(err):
            Q.kv4_append(c.cache, *args)
    with pytest.raises(TypeError):
        Q.kv4_read(c.cache, slots, dtype=torch.float64)


# ---- together, as a server uses them -----------------------------------------------------------------------------------


def test_prompt_then_drafts_then_acceptance(Q):
    """A prompt is written and attended in chunks; a tree of drafts is appended behind it and verified; the accepted path's
    keys and values are written again behind the prompt, and the next token sees exactly the accepted tokens."""
    rng = np.random.default_rng(5)
    Hq, Hkv, page, dtype = 16, 4, 16, torch.float16
    total, chunk = 100, 40
    cache = Q.KV4Pages.empty(12, page, Hkv)
    table = rng.permutation(12).astype(np.int32)[None, :9]
    slot = lambda t: tensor((table[0, np.asarray(t) // page] * page + np.asarray(t) % page).astype(np.int32))  # noqa: E731
    draw = lambda n: tensor(rng.normal(0, 1, (n, (Hq + 2 * Hkv) * 128)).astype(np.float32), dtype)  # noqa: E731
    part = lambda x: [p.unflatten(1, (-1, 128)) for p in x.split([Hq * 128, Hkv * 128, Hkv * 128], dim=1)]  # noqa: E731

    def step(x, at, mask=None):
        q, k, v = part(x)
        n = len(x)
        vals = Q.kv4_append(cache, k, v, slot(np.arange(at, at + n)), values=True)
        y = Q.kv4_attention_tree(q, cache, tensor(table), tensor(np.array([0, n], np.int32)), tensor(np.array([at + n], np.int32)),
                                 max_nodes=max(n, 1), max_len=9 * page, visible=None if mask is None else tensor(opages.pack_mask(mask, n)))
        everything = slot(np.arange(at + n))
        kk, vv = Q.kv4_read(cache, everything, dtype=torch.float32)
        assert torch.equal(kk[at:].to(dtype), vals[0]) and torch.equal(vv[at:].to(dtype), vals[1])
        seen = opages.chain(n, at + n) if mask is None else opages.tree(mask, at + n)
        ref = opages.attention(values(q), values(kk), values(vv), seen)
        assert np.abs(values(y) - ref).max() <= (2.0 ** -11 + 1e-4) * np.abs(ref).max()
        return k, v

    for at in range(0, total, chunk):
        step(draw(min(chunk, total - at)), at)
    mask = random_tree(rng, 20)
    drafts = draw(20)
    k, v = step(drafts, total, mask)
    path = np.flatnonzero(mask[19])              # the accepted leaf and its ancestors
    keep = torch.from_numpy(path).cuda()
    Q.kv4_append(cache, k[keep], v[keep], slot(np.arange(total, total + len(path))))
    step(draw(1), total + len(path))
    assert Q.device_error() == 0


def test_graph_of_a_decode_step(Q):
    """One captured graph of append and attention serves growing sequences: what it reads on the device changes between
    replays, with eager work between them."""
    rng = np.random.default_rng(6)
    B, Hq, Hkv, page, max_len, dtype = 3, 16, 4, 32, 700, torch.float16
    width = -(-max_len // page)
    lens = np.array([600, 1, 255], dtype=np.int32)
    pool = cache_of(Q, rng, B * width, page, Hkv)
    table = rng.permutation(B * width).astype(np.int32).reshape(B, width)
    for b in range(B):
        t = np.arange(lens[b])
        x, y = (tensor(rng.normal(0, 1, (lens[b], Hkv, 128)).astype(np.float32), dtype) for _ in range(2))
        Q.kv4_append(pool, x, y, tensor((table[b, t // page] * page + t % page).astype(np.int32)))
    qkv = torch.empty((B, (Hq + 2 * Hkv) * 128), dtype=dtype, device="cuda")
    q, k, v = (p.unflatten(1, (-1, 128)) for p in qkv.split([Hq * 128, Hkv * 128, Hkv * 128], dim=1))
    d = dict(slots=torch.empty(B, dtype=torch.int32, device="cuda"), table=tensor(table), lens=torch.empty(B, dtype=torch.int32, device="cuda"),
             starts=torch.arange(B + 1, dtype=torch.int32, device="cuda"))
    out = torch.empty((B, Hq, 128), dtype=dtype, device="cuda")
    ws = Q.kv4_attention_tree_workspace(B, Hq, Hkv, 1, max_len)

    def step():
        Q.kv4_append(pool, k, v, d["slots"])
        Q.kv4_attention_tree(q, pool, d["table"], d["starts"], d["lens"], max_nodes=1, max_len=max_len, out=out, workspace=ws)

    def inputs():
        qkv.copy_(tensor(rng.normal(0, 1, qkv.shape).astype(np.float32), dtype))
        t = lens.copy()
        lens[:] += 1
        d["slots"].copy_(tensor((table[np.arange(B), t // page] * page + t % page).astype(np.int32)))
        d["lens"].copy_(tensor(lens))

    side = torch.cuda.Stream()
    inputs()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        inputs()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.fill_(float("nan"))
        eager = Q.kv4_attention_tree(q, pool, d["table"], d["starts"], d["lens"], max_nodes=1, max_len=max_len)
        assert torch.equal(got, eager)
        for b in range(B):
            t = np.arange(lens[b])
            kk, vv = Q.kv4_read(pool, tensor((table[b, t // page] * page + t % page).astype(np.int32)), dtype=torch.float32)
            ref = opages.attention(values(q[b:b + 1]), values(kk), values(vv), opages.chain(1, lens[b]))
            assert np.abs(values(got[b:b + 1]) - ref).max() <= (2.0 ** -11 + 1e-4) * np.abs(ref).max()
    assert Q.device_error() == 0


def test_two_streams(Q):
    """Calls on two streams at once, each with its own workspace (given, and taken by the call itself)."""
    a = Case(Q, 91, [(5, 3000), (1, 700)], 32, 8, 64, torch.float16)
    b = Case(Q, 92, [(64, 2000)], 32, 8, 64, torch.bfloat16)
    want = a.run(Q), b.run(Q)
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    args = [(c.q.cuda(), c.cache, tensor(c.table), tensor(c.starts), tensor(c.lens)) for c in (a, b)]
    ws = Q.kv4_attention_tree_workspace(2, 32, 8, 5, 3000)
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        got.append((Q.kv4_attention_tree(*args[0], max_nodes=5, max_len=3000, workspace=ws, stream=s),
                    Q.kv4_attention_tree(*args[1], max_nodes=64, max_len=2000, stream=t)))
    torch.cuda.synchronize()
    for x, y in got:
        assert torch.equal(x, want[0]) and torch.equal(y, want[1])


def test_offsets_past_32_bits(Q):
    """A pool whose codes pass 4 GiB on each side, its last pages in use."""
    Hkv, page = 8, 256
    pages = (1 << 32) // (64 * Hkv * page) + 70      # rows past 2^26, code bytes past 2^32
    cache = Q.KV4Pages.empty(pages, page, Hkv)
    rng = np.random.default_rng(7)
    T = 600
    table = np.array([[pages - 1, 0, pages - 2]], dtype=np.int32)
    t = np.arange(T)
    slots = (table[0, t // page].astype(np.int64) * page + t % page).astype(np.int32)
    k, v = (draw_groups(rng, T, Hkv, torch.float16) for _ in range(2))
    Q.kv4_append(cache, k.cuda(), v.cuda(), tensor(slots))
    kk, vv = Q.kv4_read(cache, tensor(slots), dtype=torch.float32)
    for got, x in ((kk, k), (vv, v)):
        q, s, z = opages.quantize(values(x))
        assert np.array_equal(values(got), okv4.kv4_dequant(q, s, z))
    q = tensor(rng.normal(0, 1, (1, 32, 128)).astype(np.float32), torch.float16)
    y = Q.kv4_attention_tree(q, cache, tensor(table), tensor(np.array([0, 1], np.int32)), tensor(np.array([T], np.int32)), max_nodes=1,
                             max_len=T)
    ref = opages.attention(values(q), values(kk), values(vv), opages.chain(1, T))
    assert np.abs(values(y) - ref).max() <= (2.0 ** -11 + 1e-4) * np.abs(ref).max()
