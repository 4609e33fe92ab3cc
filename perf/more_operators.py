"""The operators of a serving step around a paged KV4 cache: what is timed, their plain forms and their values in 64
bits.

Kinds of case (``kind``):
  plan     block table, slots, positions and row starts of a step, from the cached lengths and the numbers of new
           tokens of its sequences and a stack of free pages
  release  the pages of finished sequences put back on the stack
  rope     norms of queries and keys for each head with the position rotation
  linear   the 8-bit linear of fp16 or bf16 tokens: block Hadamard rotation, 8-bit codes with a scale for each
           token, product with 8-bit weights with a scale for each output channel

Linears and heads are those of the LLaMA-3.1-8B (32 / 8 heads, 4096 and 14336 wide) and LLaMA-2-7B (32 / 32 heads,
11008 wide) shapes, the tiny 512 x 256 linear, and an output head of odd width; the head dimension is 128.
"""
import math

import torch

own = False

DEV = "cuda"
D = 128
DTYPE = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # a decode step of 61 users, three rows of padding behind them: latency
        {"name": "plan_decode_61", "kind": "plan", "B": 61, "n": 1, "T": 8192, "page": 64, "pad": 3},
        # prompts of very different length for 2000 sequences
        {"name": "plan_prompts_2000", "kind": "plan", "B": 2000, "n": 64, "T": 4096, "page": 16, "pad": 100},
        # a few of 64 users are done
        {"name": "release_64", "kind": "release", "B": 64, "T": 8192, "page": 64, "every": 9},
        # a third of 3000 sequences end together
        {"name": "release_3000", "kind": "release", "B": 3000, "T": 4096, "page": 16, "every": 3},
        # one user's decode step at a far position: the call's latency
        {"name": "rope_token", "kind": "rope", "rows": 1, "pad": 0, "Hq": 32, "Hkv": 8, "rot": 128, "pairs": 0, "norm": 1,
         "far": 120000, "dtype": "bf16"},
        # a ragged chunk of prompts of a model without grouped heads; neighbouring pairs, half of each head rotated, no norms
        {"name": "rope_chunk_2999", "kind": "rope", "rows": 2999, "pad": 37, "Hq": 32, "Hkv": 32, "rot": 64, "pairs": 1,
         "norm": 0, "far": 4096, "dtype": "fp16"},
        # a batch of prompts: the memory's rate
        {"name": "rope_prompts_16384", "kind": "rope", "rows": 16384, "pad": 0, "Hq": 32, "Hkv": 8, "rot": 128, "pairs": 0,
         "norm": 1, "far": 32768, "dtype": "bf16"},
        # the tiny linear at four tokens: latency
        {"name": "linear_tiny", "kind": "linear", "M": 4, "N": 512, "K": 256, "block": 256, "clip": 0, "dtype": "fp16",
         "out": "fp16"},
        # one token through the stacked q|k|v projection: the weights' bytes
        {"name": "linear_qkv_m1", "kind": "linear", "M": 1, "N": 6144, "K": 4096, "block": 4096, "clip": 0, "dtype": "fp16",
         "out": "fp16"},
        # a step of 61 users through an output head of odd width, 32-bit results
        {"name": "linear_head_m61", "kind": "linear", "M": 61, "N": 32003, "K": 4096, "block": 4096, "clip": 0,
         "dtype": "bf16", "out": "fp32"},
        # a ragged chunk of a prompt through the LLaMA-2-7B down projection
        {"name": "linear_down_m333", "kind": "linear", "M": 333, "N": 4096, "K": 11008, "block": 64, "clip": 1,
         "dtype": "fp16", "out": "fp16"},
        # a batch of prompts through the LLaMA-3.1-8B gate and up projections: the largest, the matrix cores' work
        {"name": "linear_mlp_m4096", "kind": "linear", "M": 4096, "N": 28672, "K": 4096, "block": 4096, "clip": 0,
         "dtype": "bf16", "out": "bf16"},
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], uniform in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["plan", "release", "rope", "rope", "linear", "linear", "linear", "linear"])
    if kind in ("plan", "release"):
        B, T = _log(rng, 1, 4096), _log(rng, 64, 16384)
        case = {"kind": kind, "B": B, "T": T, "page": rng.choice([16, 32, 48, 64, 128, 256])}
        if kind == "release":
            return dict(case, every=rng.randint(1, 12))
        return dict(case, n=rng.choice([1, _log(rng, 2, 16), _log(rng, 1, max(1, min(T // 2, 131072 // B)))]),
                    pad=rng.choice([0, rng.randint(1, 200)]))
    if kind == "rope":
        Hkv, G = rng.choice([(8, 4), (8, 4), (32, 1), (4, 8), (16, 2), (1, 3), (2, 16)])
        rows = _log(rng, 1, 16384 * 40 // (Hkv * G + Hkv) if Hkv * G + Hkv > 40 else 16384)
        return {"kind": kind, "rows": rows, "pad": rng.choice([0, 0, min(rows - 1, rng.randint(1, 9))]), "Hq": Hkv * G,
                "Hkv": Hkv, "rot": rng.choice([128, 128, 128, 64, 96, 32]), "pairs": rng.randint(0, 1),
                "norm": rng.randint(0, 1), "far": _log(rng, 1000, 1 << 20), "dtype": rng.choice(["fp16", "bf16"])}
    K, block = rng.choice([(256, 256), (1024, 1024), (2048, 2048), (4096, 4096), (4096, 4096), (11008, 64), (14336, 2048),
                           (5120, 1024), (448, 64)])
    N = _log(rng, 64, 28672)
    return {"kind": kind, "M": _log(rng, 1, max(1, min(4096, 4096 * 28672 * 4096 // (N * K)))), "N": N, "K": K, "block": block,
            "clip": rng.choice([0, 0, 1]), "dtype": rng.choice(["fp16", "bf16"]),
            "out": rng.choice(["fp16", "bf16", "fp32"])}


# ---- inputs ----------------------------------------------------------------------------------------------------


def _spread(count, most, g):
    """``count`` whole numbers spread over 0 .. most, the same ones for every seed, in an order of the seed's."""
    part = (torch.arange(count, dtype=torch.float64) * 0.6180339887498949 + 0.37) % 1.0
    return (part * (most + 1)).long()[torch.randperm(count, generator=g)]


def _paged(case, seed):
    """A server's tables: (lens, table of the pages that hold them, stack of free pages, its depth, pages)."""
    g = torch.Generator().manual_seed(seed * 23 + 9)
    B, P, T = case["B"], case["page"], case["T"]
    n = case.get("n", 1)
    lens = _spread(B, T, g)   # a step's sequences have anything from nothing to the longest cached
    width = -(-(T + 2 * n) // P)
    held = -(-lens // P)
    used = int(held.sum())
    spare = B * -(-2 * n // P) + B + 5
    perm = torch.randperm(used + spare, generator=g)
    table = torch.full((B, width), -1, dtype=torch.long)
    fill = torch.arange(width)[None, :] < held[:, None]
    table[fill] = perm[:used]
    stack = torch.full((used + spare,), -1, dtype=torch.long)
    stack[:spare] = perm[used:]
    dev = lambda t: t.to(torch.int32).to(DEV)  # noqa: E731
    return dev(lens), dev(table), dev(stack), torch.tensor([spare], dtype=torch.int32, device=DEV), used + spare, g


def prepare(case, seed):
    s = {"case": case, "kept": None}
    if case["kind"] in ("plan", "release"):
        s["lens"], s["table"], s["free"], s["depth"], s["pages"], g = _paged(case, seed)
        if case["kind"] == "plan":
            n = case["n"]
            # one token each, but one sequence in eleven that sits the step out; or any number up to twice the mean
            B = case["B"]
            counts = torch.ones(B, dtype=torch.long) if n == 1 else _spread(B, 2 * n, g)
            counts[10::11] = 0 if n == 1 else counts[10::11]
            s["rows"] = int(counts.sum()) + case["pad"]
            s["counts"] = counts.to(torch.int32).to(DEV)
        else:
            s["done"] = (torch.arange(case["B"]) % case["every"] == 0).to(torch.int32).to(DEV)
        return s
    g = torch.Generator(device=DEV).manual_seed(seed * 29 + 11)
    dt = DTYPE[case["dtype"]]
    if case["kind"] == "rope":
        rows, Hq, Hkv = case["rows"], case["Hq"], case["Hkv"]
        qkv = torch.randn((rows, (Hq + 2 * Hkv) * D), generator=g, device=DEV)
        qkv *= torch.exp(0.4 * torch.randn((rows, 1), generator=g, device=DEV))
        q, k, _ = qkv.to(dt).split([Hq * D, Hkv * D, Hkv * D], dim=1)
        s["q"], s["k"] = q.unflatten(1, (Hq, D)), k.unflatten(1, (Hkv, D))
        s["weights"] = [(1 + 0.3 * torch.randn(D, generator=g, device=DEV)).to(dt) if case["norm"] else None for _ in range(2)]
        pos = torch.randint(0, case["far"], (rows,), generator=g, device=DEV, dtype=torch.int32)
        if case["pad"]:
            pos[-case["pad"]:] = -1
        s["positions"] = pos
        half = case["rot"] // 2
        s["freq"] = (500000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)).float()
        return s
    M, N, K = case["M"], case["N"], case["K"]
    x = torch.randn((M, K), generator=g, device=DEV)
    out = torch.randint(0, K, (max(2, K // 100),), generator=g, device=DEV)
    x[:, out] *= 20.0   # channels with outliers
    s["x"] = x.to(dt)
    s["levels"] = torch.empty((N, K), dtype=torch.int8, device=DEV)
    s["scales"] = torch.empty(N, dtype=torch.float16, device=DEV)
    for i in range(0, N, 8192):   # rotated weights are near Gaussian
        w = 0.02 * torch.randn((min(8192, N - i), K), generator=g, device=DEV)
        sc = (w.abs().amax(1) / 127).half()
        s["scales"][i:i + 8192] = sc
        s["levels"][i:i + 8192] = (w / sc.float()[:, None]).round().clamp(-127, 127).to(torch.int8)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------


def _plain_plan(s):
    P, rows = s["case"]["page"], s["rows"]
    lens, counts, table = s["lens"].long(), s["counts"].long(), s["table"]
    end = torch.cumsum(counts, 0)
    starts = torch.cat((torch.zeros_like(end[:1]), end))
    after = lens + counts
    held, want = (lens + P - 1) // P, (after + P - 1) // P
    top = torch.cumsum(want - held, 0)
    base = top - (want - held)
    j = torch.arange(table.shape[1], device=DEV)
    fresh = (j >= held[:, None]) & (j < want[:, None])
    at = s["depth"].long() - 1 - (base[:, None] + j - held[:, None])
    table.copy_(torch.where(fresh, s["free"][at.clamp(min=0, max=s["free"].numel() - 1)], table))
    r = torch.arange(rows, device=DEV)
    b = torch.searchsorted(end, r, right=True)
    live = b < lens.numel()
    b = b.clamp(max=lens.numel() - 1)
    pos = lens[b] + r - starts[b]
    page = table[b, (pos // P).clamp(max=table.shape[1] - 1)].long()
    gone = torch.full_like(r, -1)
    i32 = lambda t: t.to(torch.int32)  # noqa: E731
    return {"starts": i32(starts), "lens": i32(after), "slots": i32(torch.where(live, page * P + pos % P, gone)),
            "positions": i32(torch.where(live, pos, gone)), "depth": i32(s["depth"] - top[-1]), "table": table}


def _plain_release(s):
    P, table, free = s["case"]["page"], s["table"], s["free"]
    lens, done = s["lens"].long(), s["done"] != 0
    held = torch.where(done, (lens + P - 1) // P, torch.zeros_like(lens))
    top = torch.cumsum(held, 0)
    j = torch.arange(table.shape[1], device=DEV)
    give = j < held[:, None]
    at = s["depth"].long() + (top - held)[:, None] + j
    free[at[give]] = table[give]
    return {"lens": torch.where(done, torch.zeros_like(s["lens"]), s["lens"]), "depth": (s["depth"] + top[-1]).to(torch.int32),
            "free": free}


def _rotate(y, cos, sin, rot, pairs):
    turned, rest = y[..., :rot], y[..., rot:]
    if pairs:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    else:
        a, b = turned[..., :rot // 2], turned[..., rot // 2:]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    return torch.cat((turned, rest), dim=-1)


EPS = 1e-5


def _plain_rope(s):
    case = s["case"]
    angle = s["positions"].double()[:, None, None] * s["freq"].double()   # far positions
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    live = (s["positions"] >= 0)[:, None, None]

    def one(x, w):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
        y = _rotate(y, cos, sin, case["rot"], case["pairs"])
        return torch.where(live, y, torch.zeros_like(y)).to(x.dtype)

    return {"q": one(s["q"], s["weights"][0]), "k": one(s["k"], s["weights"][1])}


def _signs(n, device):
    """The n x n Hadamard matrix of the signs (-1)^popcount(i & j)."""
    i = torch.arange(n, device=device)
    v = i[:, None] & i[None, :]
    v = v ^ (v >> 8)
    v = v ^ (v >> 4)
    v = v ^ (v >> 2)
    v = v ^ (v >> 1)
    return 1.0 - 2.0 * (v & 1).double()


def _clip(case):
    return (9, 10) if case["clip"] else (1, 1)


def _plain_linear(s):
    case = s["case"]
    M, K, b = case["M"], case["K"], case["block"]
    num, den = _clip(case)
    lo = 1 << ((b.bit_length() - 1) // 2)
    # H_b is the Kronecker product of two smaller ones; the sums of fp16 values are exact in 64 bits
    X = torch.matmul(_signs(b // lo, DEV), s["x"].double().view(M * (K // b), b // lo, lo))
    X = torch.matmul(X, _signs(lo, DEV)).view(M, K)
    A = X.abs().amax(1, keepdim=True)
    q = (X.abs() * (127.0 * den) / torch.where(A > 0, A * num, torch.ones_like(A))).round().clamp(max=127) * torch.sign(X)
    s_x = ((A * num) / (den * 127.0 * math.sqrt(b))).float()
    acc = torch.matmul(q.float(), s["levels"].float().t())
    return (acc * s_x * s["scales"].float()).to(DTYPE[case["out"]])


# ---- the framework's calls -------------------------------------------------------------------------------------


def _own(s):
    from paper_2606_02823_amd import qift

    case = s["case"]
    if case["kind"] == "plan":
        p = qift.kv4_plan_step(s["lens"], s["counts"], s["table"], s["free"], s["depth"], page=case["page"], rows=s["rows"])
        return {"starts": p.starts, "lens": p.lens, "slots": p.slots, "positions": p.positions, "depth": p.free_count,
                "table": s["table"]}
    if case["kind"] == "release":
        lens, depth = qift.kv4_release(s["lens"], s["done"], s["table"], s["free"], s["depth"], page=case["page"])
        return {"lens": lens, "depth": depth, "free": s["free"]}
    if case["kind"] == "rope":
        if s["kept"] is None:   # the model's norms and frequencies
            s["kept"] = qift.HeadRope(s["freq"], rot=case["rot"], pairs=bool(case["pairs"]), q_weight=s["weights"][0],
                                      k_weight=s["weights"][1], eps=EPS)
        q, k = qift.head_norm_rope(s["kept"], s["q"], s["k"], s["positions"])
        return {"q": q, "k": k}
    if s["kept"] is None:   # the weights' handle, and the buffers that a server keeps for its steps
        w = qift.W8(s["levels"], s["scales"])
        s["kept"] = (w, qift.alloc_act8(case["M"], case["K"], DEV), qift.w8a8_workspace(w, case["M"]))
    w, act, work = s["kept"]
    qift.rotate_quant_act8(s["x"], case["block"], clip=_clip(case), out=act)
    return qift.w8a8_linear(w, act, dtype=DTYPE[case["out"]], workspace=work)


PLAIN = {"plan": _plain_plan, "release": _plain_release, "rope": _plain_rope, "linear": _plain_linear}


def run(s):
    return _own(s) if own else PLAIN[s["case"]["kind"]](s)


def work(case):
    if case["kind"] == "plan":
        rows = case["B"] * case["n"]
        fresh = case["B"] * max(1, case["n"] // case["page"])
        return {"bytes": 20 * case["B"] + 8 * (rows + case["pad"]) + 8 * fresh, "flops": 0}
    if case["kind"] == "release":
        given = case["B"] / case["every"] * case["T"] / 2 / case["page"]
        return {"bytes": 12 * case["B"] + 8 * given, "flops": 0}
    if case["kind"] == "rope":
        values = (case["rows"] - case["pad"]) * (case["Hq"] + case["Hkv"]) * D
        return {"bytes": 4 * values, "flops": 8 * values}
    M, N, K = case["M"], case["N"], case["K"]
    size = 4 if case["out"] == "fp32" else 2
    return {"bytes": 2 * M * K + N * K + 2 * N + size * M * N, "flops": 2 * M * N * K + M * K * int(math.log2(case["block"]))}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------


def exact(case, seed):
    if case["kind"] in ("plan", "release"):
        return None   # whole numbers
    s = prepare(case, seed)
    if case["kind"] == "rope":
        half, out = case["rot"] // 2, {}
        pos = s["positions"].double().clamp(min=0)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos[:, None] * s["freq"].double()[None, :])
        for name, x, w in (("q", s["q"], s["weights"][0]), ("k", s["k"], s["weights"][1])):
            y = x.double()
            if w is not None:
                y = y / torch.sqrt(torch.einsum("rhd,rhd->rh", y, y)[..., None] / D + EPS) * w.double()
            first = torch.arange(half, device=DEV) * 2 if case["pairs"] else torch.arange(half, device=DEV)
            second = first + (1 if case["pairs"] else half)
            z = torch.complex(y[..., first], y[..., second]) * turn[:, None, :]
            y = y.clone()
            y[..., first], y[..., second] = z.real, z.imag
            y[s["positions"] < 0] = 0
            out[name] = y
        return out
    if case["M"] * case["N"] * case["K"] > 1 << 40:
        return None
    M, K, b = case["M"], case["K"], case["block"]
    num, den = _clip(case)
    X = s["x"].double().view(-1, b)
    h = 1
    while h < b:   # butterflies
        Y = X.view(-1, b // (2 * h), 2, h)
        X = torch.stack((Y[:, :, 0] + Y[:, :, 1], Y[:, :, 0] - Y[:, :, 1]), dim=2).view(-1, b)
        h *= 2
    X = X.view(M, K)
    top = X.abs().max(1, keepdim=True).values
    step = top * num / den / 127
    q = torch.clip(torch.round(X / torch.where(step > 0, step, 1.0)), -127, 127)
    y = torch.empty((M, case["N"]), dtype=torch.float64, device=DEV)
    for i in range(0, case["N"], 4096):
        y[:, i:i + 4096] = (q @ s["levels"][i:i + 4096].double().t()) * s["scales"][i:i + 4096].double()
    return y * (step / math.sqrt(b))
