"""The 8-bit linear on the GPU against the oracle.

Everything here is exact: the codes are decided on the rationals, the sums are integers, and the epilogue's two fp32
products and its one rounding to the outputs' type are the same IEEE operations on both sides.  Only the weight
quantizer's rotation is not exact in fp64: there a level may differ where w / s_w lies within rounding of a half, and a scale
where max|w| / 127 lies within rounding of a halfway point of fp16.
"""
import numpy as np
import pytest
import torch

import w8_cases
from oracle import hadamard, linear as olin, w8

pytestmark = pytest.mark.gpu

OUT = (torch.float16, torch.bfloat16, torch.float32)


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_02823_amd import qift
    qift.lib()
    return qift


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def expect(acc, s_x, s_w, dtype):
    """The outputs bit for bit."""
    return torch.from_numpy(w8.epilogue(acc, s_x, s_w)).to(dtype)


def same(a, b):
    return a.shape == b.shape and a.dtype == b.dtype and torch.equal(a.cpu(), b.cpu())


def tokens(rng, M, K, bf16):
    x = rng.normal(0, 1, (M, K)) * np.exp(rng.normal(0, 1, (M, 1)))
    x[:, rng.integers(0, K, max(1, K // 100))] *= 25.0
    x[M // 2] = 0.0 if M > 1 else x[M // 2]
    if M > 2:
        x[2] = np.round(x[2] * 4) / 4       # few distinct values: exact ties
    if M > 3:
        x[3] = 0.0
        x[3, 0], x[3, min(1, K - 1)] = 127.0, 0.5   # every code a half or near one
    t = torch.from_numpy(x)
    return t.to(torch.bfloat16) if bf16 else t.to(torch.float16)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("M,K,b,clip", [(1, 64, 2, (1, 1)), (5, 64, 64, (9, 10)), (7, 448, 64, (1, 1)), (4, 256, 256, (1, 1)),
                                        (3, 4096, 4096, (1, 1)), (2, 11008, 64, (9, 10)), (2, 14336, 2048, (1, 1)),
                                        (300, 512, 128, (3, 16)), (4, 8192, 8192, (1, 1)), (4, 32768, 4096, (1, 1)),
                                        (300, 8192, 256, (1, 1)), (260, 12288, 4096, (1, 1)), (260, 14336, 2048, (1, 1))])
def test_codes(Q, M, K, b, clip, bf16):
    rng = np.random.default_rng(M * 131 + K + b + bf16)
    x = tokens(rng, M, K, bf16)
    act = Q.rotate_quant_act8(x.cuda(), b, clip)
    q, s = w8.act_quant8(x.float().numpy() if bf16 else x.numpy(), b, clip)
    assert act.sum is None
    assert np.array_equal(act.q.cpu().numpy(), q) and np.array_equal(act.scale.cpu().numpy(), s)


def test_codes_of_far_apart_values(Q):
    """One value of 2^16 times its row's others and more (every exponent difference around the exact decision's cut)."""
    x = torch.zeros((24, 64), dtype=torch.float64)
    for i in range(24):
        x[i, 0], x[i, 3], x[i, 5] = 1.0, 2.0 ** -i, -(2.0 ** -i) / 127 * 63.5
    for dt in (torch.float16, torch.bfloat16):
        t = x.to(dt)
        act = Q.rotate_quant_act8(t.cuda(), 2)
        q, s = w8.act_quant8(t.float().numpy() if dt == torch.bfloat16 else t.numpy(), 2)
        assert np.array_equal(act.q.cpu().numpy(), q) and np.array_equal(act.scale.cpu().numpy(), s)


@pytest.mark.parametrize("N,K,b", [(1, 64, 2), (9, 256, 256), (5, 4096, 4096), (3, 11008, 64), (2, 16384, 2048), (70, 448, 64)])
def test_weights(Q, N, K, b):
    rng = np.random.default_rng(N + K)
    W = (0.02 * rng.standard_t(5, (N, K))).astype(np.float32)
    if N > 2:
        W[1] = 0.0
        W[2] *= 1e-7     # a scale among fp16's subnormals
    w = Q.quantize_weights8(dev(W), b)
    Wr = hadamard.rotate_weights(W.astype(np.float64), b)
    L, s = w8.quantize_weights8(Wr)
    assert np.array_equal(w.scales.cpu().numpy(), s)
    got = w.levels.cpu().numpy().astype(int)
    with np.errstate(divide="ignore", invalid="ignore"):
        u = np.abs(Wr / s.astype(np.float64)[:, None])
        near = np.abs(u - np.floor(u) - 0.5) < 1e-9
    off = got != L
    assert not np.any(off & ~near) and np.abs(got - L).max() <= 1


def operands(rng, N, K, M):
    L, q = (rng.integers(-127, 128, s, dtype=np.int8) for s in ((N, K), (M, K)))
    s_w = (np.exp(rng.normal(-6, 1, N))).astype(np.float16)
    s_x = np.exp(rng.normal(-2, 1, M)).astype(np.float32)
    if N > 3:
        s_w[3] = 0.0
    if M > 2:
        s_x[2] = 0.0
    return L, q, s_w, s_x


# up to 64 tokens: every number of token tiles and of row tiles, whole and cut rows of every kind
ROWS = [(M, N, K) for M in (1, 4, 16, 17, 33, 48, 49, 64) for N, K in ((1, 64), (37, 192), (512, 256), (1027, 448))] + \
       [(M, N, 320) for M in (2, 30, 47, 61) for N in (8200, 9000, 16403)] + [(3, 130, 8192), (64, 70, 131072)] + \
       [(M, N, 1088) for M in (1, 16, 17, 32) for N in (1021, 2045, 3069, 5119, 6142, 7165, 9001, 11003, 13001)]   # 4 to 52 rows to a workgroup


@pytest.mark.parametrize("M,N,K", ROWS)
def test_linear_up_to_64_tokens(Q, M, N, K):
    rng = np.random.default_rng(M * 7 + N * 3 + K)
    L, q, s_w, s_x = operands(rng, N, K, M)
    acc = olin.int_dot(L, q)
    w, act = Q.W8(dev(L), dev(s_w)), Q.QAct(dev(q), dev(s_x))
    ws = Q.w8a8_workspace(w, M)
    for dt in OUT:
        got_acc = torch.full((M, N), -7, dtype=torch.int32, device="cuda")
        assert same(Q.w8a8_linear(w, act, dtype=dt, acc_out=got_acc), expect(acc, s_x, s_w, dt)), dt
        assert same(Q.w8a8_linear(w, act, dtype=dt, workspace=ws), expect(acc, s_x, s_w, dt)), dt
        assert np.array_equal(got_acc.cpu().numpy(), acc)


TILED = [(65, 1, 64), (65, 64, 128), (128, 128, 256), (129, 130, 192), (200, 515, 320), (333, 700, 1088), (70, 4096, 2048),
         (300, 128, 4096), (1000, 66, 4096), (257, 131, 14336), (128, 1024, 131072 // 8)]


@pytest.mark.parametrize("M,N,K", TILED)
def test_linear_tiled(Q, M, N, K):
    """With K cut, where the size is one that is, and along all of it."""
    rng = np.random.default_rng(M + N + K)
    L, q, s_w, s_x = operands(rng, N, K, M)
    acc = olin.int_dot(L, q)
    w, act = Q.W8(dev(L), dev(s_w)), Q.QAct(dev(q), dev(s_x))
    for ws in {None, Q.w8a8_workspace(w, M)}:
        if ws is not None:
            ws.fill_(0x5A)
        for dt in OUT:
            got_acc = torch.full((M, N), -7, dtype=torch.int32, device="cuda")
            out = torch.zeros((M, N), dtype=dt, device="cuda")
            assert Q.w8a8_linear(w, act, out=out, acc_out=got_acc, workspace=ws) is out
            assert same(out, expect(acc, s_x, s_w, dt)), dt
            assert np.array_equal(got_acc.cpu().numpy(), acc)
            assert same(Q.w8a8_linear(w, act, dtype=dt, workspace=ws), out)


# enough tiles of 256 x 256 for the large ones: whole, cut on either side, rows of y at every alignment
@pytest.mark.parametrize("M,N,K", [(4096, 3328, 192), (4000, 3203, 128), (3329, 4098, 64), (3073, 4100, 320), (12800, 1000, 128)])
def test_linear_large_tiles(Q, M, N, K):
    rng = np.random.default_rng(M + N + K)
    L, q, s_w, s_x = operands(rng, N, K, M)
    w, act = Q.W8(dev(L), dev(s_w)), Q.QAct(dev(q), dev(s_x))
    assert Q.w8a8_workspace(w, M) is None
    acc = (q.astype(np.float32) @ L.astype(np.float32).T)   # sums below 2^24: exact
    assert 127 * 127 * K < 2 ** 24
    for dt in OUT:
        got_acc = torch.empty((M, N), dtype=torch.int32, device="cuda") if dt is torch.float16 else None
        assert same(Q.w8a8_linear(w, act, dtype=dt, acc_out=got_acc), expect(acc.astype(np.int64), s_x, s_w, dt)), dt
        if got_acc is not None:
            assert np.array_equal(got_acc.cpu().numpy(), acc.astype(np.int32))


def test_extremes(Q):
    """-128 among the codes, the largest sums, outputs past fp16 and fp32."""
    K = 131072
    for M in (3, 100):
        L, q = np.full((80, K), 127, np.int8), np.full((M, K), 127, np.int8)
        L[1], q[1] = -128, -128
        s_w, s_x = np.full(80, 60000.0, np.float16), np.full(M, 2.0 ** 100, np.float32)
        s_x[0] = 2.0 ** -140
        acc = np.full((M, 80), 127 * 127 * K, np.int64)
        acc[1, :], acc[:, 1] = -128 * 127 * K, -128 * 127 * K
        acc[1, 1] = 128 * 128 * K
        acc32 = acc.astype(np.uint32).view(np.int32).astype(np.int64)   # (128^2 K is 2^31: it wraps)
        w, act = Q.W8(dev(L), dev(s_w)), Q.QAct(dev(q), dev(s_x))
        got = torch.empty((M, 80), dtype=torch.int32, device="cuda")
        for dt in OUT:
            with np.errstate(over="ignore"):
                assert same(Q.w8a8_linear(w, act, dtype=dt, acc_out=got), expect(acc32, s_x, s_w, dt))
            assert np.array_equal(got.cpu().numpy(), acc32)


def test_what_lies_behind_is_left(Q):
    """Outputs inside larger arrays: nothing before or behind them is written."""
    rng = np.random.default_rng(9)
    for M, N, K in ((5, 33, 128), (130, 67, 256), (66, 100, 2048)):
        L, q, s_w, s_x = operands(rng, N, K, M)
        w, act = Q.W8(dev(L), dev(s_w)), Q.QAct(dev(q), dev(s_x))
        for dt in OUT:
            pad = 64
            room = torch.full((2 * pad + M * N,), 7.0, dtype=dt, device="cuda")
            out = room[pad:pad + M * N].view(M, N)
            Q.w8a8_linear(w, act, out=out, workspace=Q.w8a8_workspace(w, M))
            assert same(out, expect(olin.int_dot(L, q), s_x, s_w, dt))
            assert torch.all(room[:pad] == 7) and torch.all(room[pad + M * N:] == 7)


def test_a_captured_linear_is_replayed(Q):
    """Quantizer and linear of both kernels in a graph, on a stream of its own, with new tokens each time."""
    rng = np.random.default_rng(11)
    for M, N, K in ((3, 512, 256), (150, 300, 4096)):
        L, _, s_w, _ = operands(rng, N, K, M)
        w = Q.W8(dev(L), dev(s_w))
        x = torch.zeros((M, K), dtype=torch.float16, device="cuda")
        act, ws = Q.alloc_act8(M, K), Q.w8a8_workspace(w, M)
        y = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")

        def run():
            Q.rotate_quant_act8(x, 64, out=act)
            Q.linear(w, act, out=y, workspace=ws)

        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            run()
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        for i in range(3):
            x.copy_(tokens(rng, M, K, False))
            y.zero_()
            g.replay()
            torch.cuda.synchronize()
            got = y.clone()
            q, s_x = w8.act_quant8(x.cpu().numpy(), 64)
            assert same(got, expect(olin.int_dot(L, q), s_x, s_w, torch.bfloat16))
            y.zero_()
            run()
            assert same(y, got)


def test_binding_refuses(Q):
    w = Q.W8(torch.zeros((8, 64), dtype=torch.int8, device="cuda"), torch.zeros(8, dtype=torch.float16, device="cuda"))
    act = Q.alloc_act8(4, 64)
    with pytest.raises(TypeError):
        Q.rotate_quant_act8(torch.zeros((4, 64), device="cuda"), 64)
    with pytest.raises(TypeError):
        Q.w8a8_linear(w, act, dtype=torch.float64)
    with pytest.raises(ValueError):
        Q.w8a8_linear(w, Q.alloc_act8(4, 128))
    with pytest.raises(ValueError):
        Q.linear(w, act, use_sum=True)
    with pytest.raises(ValueError):
        Q.W8(torch.zeros((8, 64), dtype=torch.int8, device="cuda"), torch.zeros(9, dtype=torch.float16, device="cuda"))
    with pytest.raises(TypeError):
        Q.W8(torch.zeros((8, 64), dtype=torch.int8), torch.zeros(8, dtype=torch.float16, device="cuda"))
    with pytest.raises(Q.QiftError):
        Q.rotate_quant_act8(torch.zeros((4, 96), dtype=torch.float16, device="cuda"), 32)


@pytest.mark.parametrize("M,N,K,kernel,parts", w8_cases.CASES)
def test_linear_of_each_kernel(Q, M, N, K, kernel, parts):
    """Every kernel in every output type, with the sums and without, results inside a larger array whose ends stay as they were.
    (The sums are whole numbers below 2^53 in fp64: exact.)"""
    rng = np.random.default_rng(M + N + K)
    L, q, s_w, s_x = operands(rng, N, K, M)
    acc = (q.astype(np.float64) @ L.astype(np.float64).T).astype(np.int64)
    w, act = Q.W8(dev(L), dev(s_w)), Q.QAct(dev(q), dev(s_x))
    ws = Q.w8a8_workspace(w, M)
    assert ws is not None or parts == 1
    pad = 64
    for dt in OUT:
        want = expect(acc, s_x, s_w, dt)
        got_acc = torch.full((M, N), -7, dtype=torch.int32, device="cuda")
        if ws is not None:
            ws.fill_(0x5A)
        assert same(Q.w8a8_linear(w, act, dtype=dt, acc_out=got_acc, workspace=ws), want), dt
        assert np.array_equal(got_acc.cpu().numpy(), acc)
        room = torch.full((2 * pad + M * N,), 7.0, dtype=dt, device="cuda")
        out = room[pad:pad + M * N].view(M, N)
        Q.w8a8_linear(w, act, out=out, workspace=ws)
        assert same(out, want), dt
        assert torch.all(room[:pad] == 7) and torch.all(room[pad + M * N:] == 7)


def test_one_workspace_for_a_servers_steps(Q):
    """Steps of any size one after the other in the workspace of all sizes, dirty from the step before."""
    rng = np.random.default_rng(23)
    N, K, most = 1027, 8256, 400
    L, q, s_w, s_x = operands(rng, N, K, most)
    w = Q.W8(dev(L), dev(s_w))
    ws = Q.w8a8_workspace(w, range(1, most + 1))
    acc = (q.astype(np.float64) @ L.astype(np.float64).T).astype(np.int64)
    cut = 0
    for M in (1, 400, 33, 130, 17, 333, 64, 399, 250):
        cut += Q.w8a8_workspace_bytes(w, M) > 0
        assert Q.w8a8_workspace_bytes(w, M) <= ws.numel()
        act = Q.QAct(dev(q[:M]), dev(s_x[:M]))
        assert same(Q.w8a8_linear(w, act, workspace=ws), expect(acc[:M], s_x[:M], s_w, torch.float16)), M
    assert cut > 4
