"""The paged KV4 cache at its limits: counts and rows past what a call was made for, scores at the ends of fp32's range,
long sums, and the forms of the calls that take their outputs."""
import numpy as np
import pytest
import torch

from oracle import pages as opages
from test_gpu_pages import HALF, Case, Q, cache_of, draw_groups, host, random_tree, same_cache, tensor, values   # noqa: F401

pytestmark = pytest.mark.gpu


def near(c, got, ref, b, lead=""):
    """Rows of sequence b against fp64, within the limit that test_gpu_pages derives (its own formula, for some rows)."""
    n, t = len(got), c.seqs[b][1]
    q = values(c.q[c.starts[b]:c.starts[b] + n]).astype(np.float64)
    G = c.Hq // c.Hkv
    kn = np.linalg.norm(c.k[b].astype(np.float64), axis=-1).max(axis=0)
    vmax = np.abs(c.v[b]).max(axis=(0, 2))
    S = np.linalg.norm(q, axis=-1) * np.repeat(kn, G)[None] / np.sqrt(128.0)
    L = np.abs(np.log2(np.maximum(c.scales[b], 2.0 ** -90))).max()
    e = (2 * (S + L + 1) * 2.0 ** -21 + 2.0 ** -21 + t / 32 * 2.0 ** -24) * np.repeat(vmax, G)[None]
    if c.dtype == torch.float16:
        e = e + 2.0 ** -25
    over = np.abs(values(got).astype(np.float64) - ref) / (HALF[c.dtype] * np.abs(ref) + e[..., None])
    assert over.max() <= 1.0, (lead, b, float(over.max()))


@pytest.mark.parametrize("masked", [False, True], ids=["chain", "tree"])
def test_first_nodes_of_sequences_with_too_many(Q, masked):  # noqa: F811
    """The nodes that a call was made for keep their places when a sequence has more, or when q has fewer rows than the
    starts say; those left out are neither computed nor seen, and the error word says so."""
    rng = np.random.default_rng(11)
    seqs = [(3, 400), (9, 1300)]
    masks = [random_tree(rng, n) for n, _ in seqs] if masked else None
    c = Case(Q, 120, seqs, 16, 4, 32, torch.float16, masks)
    ref = [c.reference(b) for b in range(2)]
    if masked:                                   # rows that name a node that is left out do not see it
        for m in masks:
            m[:2, 2] = True
    assert Q.device_error() == 0
    out = torch.full((c.rows, 16, 128), 7.0, dtype=torch.float16, device="cuda")
    for most_len in (1300, 5000):
        out.fill_(7.0)
        y = c.run(Q, max_nodes=2, max_len=most_len, out=out)
        assert Q.device_error() == Q.DEVERR_INDEX
        for b in range(2):
            s = c.starts[b]
            near(c, y[s:s + 2], ref[b][:2], b, "two nodes")
            assert (y[s + 2:c.starts[b + 1]] == 7.0).all()
    # two rows fewer than the starts say: the last sequence loses its last two nodes
    visible = c.visible(9)
    if masked:
        for m in masks:
            m[:2, 2] = False
        visible = c.visible(9)
        visible[c.starts[1]:, 0] |= 1 << 7
    y = Q.kv4_attention_tree(c.q[:-2].cuda(), c.cache, tensor(c.table), tensor(c.starts), tensor(c.lens), max_nodes=9, max_len=1300,
                             visible=None if visible is None else visible[:-2].contiguous())
    assert Q.device_error() == Q.DEVERR_INDEX
    near(c, y[:3], ref[0], 0)
    near(c, y[3:], ref[1][:7], 1, "seven rows")
    # a first row that is none: the sequence has no rows
    out.fill_(7.0)
    Q.kv4_attention_tree(c.q.cuda(), c.cache, tensor(c.table), tensor(np.array([-4, 3, 12], dtype=np.int32)), tensor(c.lens),
                         max_nodes=9, max_len=1300, visible=visible, out=out)
    assert Q.device_error() == Q.DEVERR_INDEX
    assert (out[:3] == 7.0).all()


def test_scores_at_the_ends_of_fp32(Q):  # noqa: F811
    """One seen token is the whole softmax while its score is finite in fp32: scores (in powers of two, as the kernel has
    them) between -2^128 and -2^127, and scores whose sum of products before the key's scale is past fp32."""
    only = np.array([[False, True], [False, True]])
    for kscale, top in ((300.0, 2.9e38), (1.0, 5e37), (1e-3, 1e36)):
        c = Case(Q, 121, [(2, 2)] * 6, 8, 2, 16, torch.bfloat16, [only] * 6, kscale=kscale)
        pick = lambda x: torch.from_numpy(np.stack([t[1] for t in x for _ in range(2)])).repeat_interleave(4, dim=1)  # noqa: E731
        key, ref = pick(c.k), pick(c.v)
        norm = (key.double() ** 2).sum(-1, keepdim=True)
        for sign in (-1.0, 1.0):
            # a score of sign * top in powers of two, before log2 of the value's scale (a few)
            c.q = (sign * top * np.sqrt(128.0) / np.log2(np.e) / norm * key).to(torch.bfloat16)
            assert torch.isfinite(c.q.float()).all()
            y = c.run(Q).float().cpu()
            assert (y - ref).abs().le(ref.abs() * (2.0 ** -8 + 2.0 ** -20)).all(), (kscale, sign)


def test_long_sums_keep_their_smallest_parts(Q):  # noqa: F811
    """65536 tokens of one unit in one workgroup (513 sequences, the others empty).  The first 256 have nearly all of the
    weight and the value 0 in half of the dimensions (code = zero-point = 7); what the others add there, code 15, is each
    time about half a step of 64 + code times the weights' sum, and must not be lost or rounded up."""
    T, P, B = 65536, 64, 513
    pages = T // P
    cache = Q.KV4Pages.empty(pages, P, 1)
    k, v = np.full((pages, 1, P, 64), 0x77, np.uint8), np.full((pages, 1, P, 64), 0xFF, np.uint8)
    head = 256 // P
    k[:head, ..., 0] = 0x7F                     # dimension 0: code 15, 8 steps over the zero-point
    k[head:, ..., 0] = 0x77
    v[:head, ..., :32] = 0x77                   # dimensions 0 .. 63: code 7, value 0
    v[head:, ..., 32:] = 0x00                   # dimensions 64 .. 127 of the tail: code 0
    for side, codes in ((cache.k, k), (cache.v, v)):
        side.codes.copy_(tensor(codes))
        side.scales.fill_(1.0)
        side.zeros.fill_(7)
    table = torch.zeros((B, pages), dtype=torch.int32, device="cuda")
    table[0] = torch.arange(pages, dtype=torch.int32, device="cuda")
    starts = torch.ones(B + 1, dtype=torch.int32, device="cuda")
    starts[0] = 0
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    lens[0] = T
    # heads of different weight of the tail: 32 79 w is (i + 0.55) steps of the sum 71 * 64 of a wave
    w = (np.arange(16) * 0.37 + 0.55) * 2.0 ** -11 / (32 * 79)
    q = np.zeros((1, 16, 128))
    q[0, :, 0] = -np.log(w) * np.sqrt(128.0) / 8
    q = torch.from_numpy(q).half()
    y = values(Q.kv4_attention_tree(q.cuda(), cache, table, starts, lens, max_nodes=1, max_len=T)).astype(np.float64)
    assert Q.device_error() == 0
    score = q[0, :, 0].double().numpy() * 8 / np.sqrt(128.0)
    p = np.exp(-score)
    total = 256 + (T - 256) * p
    ref = np.concatenate([np.repeat((8 * (T - 256) * p / total)[:, None], 64, axis=1),
                          np.repeat(((8 * 256 - 7 * (T - 256) * p) / total)[:, None], 64, axis=1)], axis=1)
    # test_gpu_pages' limit: S = score, L = 0, the largest value 8
    limit = HALF[torch.float16] * np.abs(ref) + (2 * (score[:, None] + 1) * 2.0 ** -21 + 2.0 ** -21 + T / 32 * 2.0 ** -24) * 8 + 2.0 ** -25
    over = np.abs(y[0] - ref) / limit
    print("worst error", over[:, :64].max(), over[:, 64:].max(), "of the limit", flush=True)
    assert over.max() <= 1.0


def test_long_sums_of_weights(Q):  # noqa: F811
    """2^20 tokens of one unit in one workgroup: the first 256 have the value 8 and nearly all of the weight, each of the
    others half a step, a little more or less, of what a lane has summed by then (16 tokens of weight 1: 2^-19 a step).  Added one
    by one they would all be lost or all count for a whole step."""
    T, P, B = 1 << 20, 64, 513
    pages = T // P
    cache = Q.KV4Pages.empty(pages, P, 1)
    for side in (cache.k, cache.v):
        side.codes.fill_(0x77)                  # code = zero-point
        side.scales.fill_(1.0)
        side.zeros.fill_(7)
    cache.k.codes[:256 // P, ..., 0] = 0x7F     # dimension 0: code 15, 8 steps over the zero-point
    cache.v.codes[:256 // P] = 0xFF
    table = torch.zeros((B, pages), dtype=torch.int32, device="cuda")
    table[0] = torch.arange(pages, dtype=torch.int32, device="cuda")
    starts = torch.ones(B + 1, dtype=torch.int32, device="cuda")
    starts[0] = 0
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    lens[0] = T
    w = np.repeat([0.45, 0.48, 0.52, 0.55], 4) * 2.0 ** -19
    q = np.zeros((1, 16, 128))
    q[0, :, 0] = -np.log(w) * np.sqrt(128.0) / 8
    q = torch.from_numpy(q).half()
    y = values(Q.kv4_attention_tree(q.cuda(), cache, table, starts, lens, max_nodes=1, max_len=T)).astype(np.float64)
    assert Q.device_error() == 0
    score = q[0, :, 0].double().numpy() * 8 / np.sqrt(128.0)
    ref = (8 * 256 / (256 + (T - 256) * np.exp(-score)))[:, None]
    # half a step, and the sums: 16 roundings within a step of 64 tokens, then one for each of T / 256 steps of a wave; a value
    # sum's T / 64; scores 7 2^-24 S in numerator and denominator; 2^-18 for all that does not grow
    limit = HALF[torch.float16] * ref + (2 * 7 * score[:, None] * 2.0 ** -24 + 2.0 ** -18 + (T / 64 + T / 256) * 2.0 ** -24) * 8
    over = np.abs(y[0] - ref) / limit
    print("worst error", over.max(), "of the limit", flush=True)
    assert over.max() <= 1.0


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["fp16", "bf16"])
def test_many_tokens_against_the_oracle(Q, dtype):  # noqa: F811
    """Enough rows for the reading kernel of four tiles a workgroup, the last of them not full; slots in any order, some of
    none; the outputs given by the caller."""
    rng = np.random.default_rng(21)
    n, Hkv, page = 4133, 8, 48
    pages = -(-n // page) + 2
    cache = cache_of(Q, rng, pages, page, Hkv)
    before = host(cache.k), host(cache.v)
    slots = rng.permutation(pages * page)[:n].astype(np.int32)
    slots[[5, 700, n - 1]] = -1
    k, v = (draw_groups(rng, n, Hkv, dtype) for _ in range(2))
    given = [torch.full((n, Hkv, 128), float("nan"), dtype=dtype, device="cuda") for _ in range(2)]
    got = Q.kv4_append(cache, k.cuda(), v.cuda(), tensor(slots), values=(given[0], given[1]))
    assert got[0] is given[0] and got[1] is given[1]
    for side, was, x, y in ((cache.k, before[0], k, got[0]), (cache.v, before[1], v, got[1])):
        *want, hat = opages.append(*was, values(x), slots)
        same_cache(side, want)
        assert torch.equal(y.cpu(), torch.from_numpy(hat).to(dtype))
    for out in (torch.float16, torch.bfloat16, torch.float32):
        given = [torch.full((n, Hkv, 128), float("nan"), dtype=out, device="cuda") for _ in range(2)]
        back = Q.kv4_read(cache, tensor(slots), dtype=out, out=given)
        assert back[0] is given[0] and back[1] is given[1]
        for side, y in ((cache.k, back[0]), (cache.v, back[1])):
            assert torch.equal(y.cpu(), torch.from_numpy(opages.read(*host(side), slots)).to(out))
    assert Q.device_error() == 0


def test_given_outputs_are_checked(Q):  # noqa: F811
    cache = Q.KV4Pages.empty(2, 16, 4)
    x = torch.zeros((3, 4, 128), dtype=torch.float16, device="cuda")
    slots = torch.arange(3, dtype=torch.int32, device="cuda")
    good = torch.empty_like(x)
    for bad, err in ((good.float(), TypeError), (good[:2], ValueError), (good.cpu(), TypeError), (good.bfloat16(), TypeError),
                     (torch.empty((3, 8, 128), dtype=torch.float16, device="cuda")[:, ::2], ValueError)):
        for pair in ((bad, good), (good, bad)):
            with pytest.raises(err):
                Q.kv4_append(cache, x, x, slots, values=pair)
            with pytest.raises(err):
                Q.kv4_read(cache, slots, out=pair)
    assert not cache.k.scales.any() and Q.device_error() == 0


def test_calls_with_everything_given_allocate_nothing(Q):  # noqa: F811
    c = Case(Q, 122, [(3, 900), (5, 2000)], 16, 4, 32, torch.float16)
    args = [c.q.cuda(), c.cache, tensor(c.table), tensor(c.starts), tensor(c.lens)]
    out = torch.empty_like(args[0])
    ws = Q.kv4_attention_tree_workspace(2, 16, 4, 5, 2000)
    k = torch.randn((8, 4, 128), device="cuda").half()
    pair = torch.empty_like(k), torch.empty_like(k)
    slots = tensor(c.slots(0, np.arange(8)))

    def calls():
        Q.kv4_append(c.cache, k, k, slots, values=pair)
        Q.kv4_read(c.cache, slots, out=pair)
        Q.kv4_attention_tree(*args, max_nodes=5, max_len=2000, out=out, workspace=ws)
    calls()
    torch.cuda.synchronize()
    was = torch.cuda.memory_stats()["allocation.all.allocated"], torch.cuda.mem_get_info()[0]
    for _ in range(3):
        calls()
    torch.cuda.synchronize()
    assert (torch.cuda.memory_stats()["allocation.all.allocated"], torch.cuda.mem_get_info()[0]) == was


def test_steps_of_a_server(Q):  # noqa: F811
    """A chunk of a prompt beside sequences of one token, dealt out and whole; 130 sequences of one token, one of them long; a long
    sequence whose values the whole length weighs."""
    rng = np.random.default_rng(22)
    seqs = [(1, int(t)) for t in rng.integers(1, 900, 15)] + [(256, 700)] + [(1, int(t)) for t in rng.integers(1, 900, 15)]
    c = Case(Q, 123, seqs, 8, 2, 32, torch.bfloat16)
    c.check(c.run(Q), "chunk and tokens")
    c = Case(Q, 126, seqs[12:19], 8, 2, 32, torch.bfloat16)
    c.check(c.run(Q, max_len=2000), "chunk and tokens, dealt out")
    seqs = [(1, int(t)) for t in rng.integers(1, 60, 129)] + [(1, 9000)]
    c = Case(Q, 124, seqs, 32, 8, 16, torch.float16)
    c.check(c.run(Q), "130 users")
    c = Case(Q, 125, [(2, 40000)], 8, 2, 128, torch.float16, gain=0.2)
    c.check(c.run(Q), "40000 tokens")
    assert Q.device_error() == 0
