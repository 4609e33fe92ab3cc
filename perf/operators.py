"""The operators on a paged KV4 cache: what is timed, their plain forms and their values in 64 bits.

Kinds of case (``kind``):
  append  keys and values of new tokens quantized into the slots of a paged 4-bit cache, with the values that
          the cache then stands for
  read    the values of given slots read back from the cache
  tree    attention of each sequence's new tokens (one token, a chain or a tree of drafts, a chunk of a prompt)
          over its pages

A cache is a pool of pages, each of ``page`` tokens: codes [pages, Hkv, page, 64] (two 4-bit codes a byte, value
2i in the low nibble of byte i), scales and zero-points [pages, Hkv, page], for keys and for values.  Slot
p * page + i is token i of page p.  Keys, values and queries are views of stacked q|k|v rows, as the linear
that produces them writes them.  Heads are those of the LLaMA-3.1-8B (32 / 8) and LLaMA-2-7B (32 / 32) shapes,
in drawn cases other groupings too; the head dimension is 128.
"""
import math

import torch

own = False

DEV = "cuda"
D = 128
DTYPE = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # one user's decode step: a single token's keys and values; the call's latency
        {"name": "append_token", "kind": "append", "n": 1, "seqs": 1, "pad": 0, "Hq": 32, "Hkv": 8, "page": 64, "dtype": "fp16"},
        # a decode step of 61 users of a model without grouped heads, three rows of padding behind them
        {"name": "append_step_61", "kind": "append", "n": 64, "seqs": 64, "pad": 3, "Hq": 32, "Hkv": 32, "page": 16,
         "dtype": "bf16"},
        # a batch of seven prompts
        {"name": "append_prompts", "kind": "append", "n": 16384, "seqs": 7, "pad": 37, "Hq": 32, "Hkv": 8, "page": 64,
         "dtype": "fp16"},
        # a short shared prefix of odd length
        {"name": "read_prefix_333", "kind": "read", "n": 333, "seqs": 1, "pad": 0, "Hq": 32, "Hkv": 32, "page": 16,
         "dtype": "fp16"},
        # four long conversations taken up again, for attention in bf16
        {"name": "read_prefix_32768", "kind": "read", "n": 32768, "seqs": 4, "pad": 0, "Hq": 32, "Hkv": 8, "page": 128,
         "dtype": "bf16"},
        # one user, one token, about a thousand cached: latency
        {"name": "decode_b1_t1000", "kind": "tree", "B": 1, "n": 1, "T": 1000, "ragged": 0, "tree": 0, "Hq": 32, "Hkv": 8,
         "page": 64, "dtype": "fp16"},
        # a decode step of 32 users with histories of very different length: the cache's bytes
        {"name": "decode_b32_ragged", "kind": "tree", "B": 32, "n": 1, "T": 8192, "ragged": 1, "tree": 0, "Hq": 32, "Hkv": 8,
         "page": 64, "dtype": "fp16"},
        # four drafted tokens and the last one, 16 users, heads that are not grouped
        {"name": "chain_b16_n5", "kind": "tree", "B": 16, "n": 5, "T": 2048, "ragged": 0, "tree": 0, "Hq": 32, "Hkv": 32,
         "page": 16, "dtype": "bf16"},
        # one user's tree of 64 drafts over a long context
        {"name": "tree_b1_t65536", "kind": "tree", "B": 1, "n": 64, "T": 65536, "ragged": 0, "tree": 1, "Hq": 32, "Hkv": 8,
         "page": 128, "dtype": "fp16"},
        # trees of up to 37 drafts, seven users of different history
        {"name": "tree_b7_n37", "kind": "tree", "B": 7, "n": 37, "T": 2999, "ragged": 1, "tree": 1, "Hq": 32, "Hkv": 8,
         "page": 32, "dtype": "bf16"},
        # trees of 64 drafts for 16 users at a long context: the largest, the matrix cores' work
        {"name": "tree_b16_n64", "kind": "tree", "B": 16, "n": 64, "T": 8192, "ragged": 0, "tree": 1, "Hq": 32, "Hkv": 8,
         "page": 64, "dtype": "fp16"},
        # a chunk of 256 prompt tokens of four users, causal
        {"name": "chunk_b4_n256", "kind": "tree", "B": 4, "n": 256, "T": 2048, "ragged": 1, "tree": 0, "Hq": 32, "Hkv": 8,
         "page": 64, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], uniform in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "append", "read", "tree", "tree", "tree", "tree"])
    Hkv, G = rng.choice([(8, 4), (8, 4), (32, 1), (4, 8), (16, 2), (8, 3), (2, 16)])
    common = {"kind": kind, "Hq": Hkv * G, "Hkv": Hkv, "page": rng.choice([16, 32, 48, 64, 128, 256]),
              "dtype": rng.choice(["fp16", "bf16"])}
    if kind != "tree":
        n = _log(rng, 1, 16384 if Hkv <= 8 else 4096)
        if kind == "read" and rng.random() < 0.25:
            common["dtype"] = "fp32"
        return dict(common, n=n, seqs=_log(rng, 1, min(n, 64)), pad=rng.choice([0, 0, min(n - 1, rng.randint(1, 9))]))
    n = rng.choice([1, 1, _log(rng, 2, 16), _log(rng, 2, 64), _log(rng, 65, 256)])
    T = max(n, _log(rng, 33, 65536))
    # the largest listed case: 16 * 64 * 8192 pairs of tokens, 32 * 8192 cached tokens of 8 heads
    most = min(64, 16 * 64 * 8192 // (n * T), 32 * 8192 * 8 // (T * Hkv))
    return dict(common, B=_log(rng, 1, max(1, most)), n=n, T=T, ragged=rng.randint(0, 1), tree=rng.randint(0, 1))


# ---- inputs ----------------------------------------------------------------------------------------------------


def _nodes(case):
    """New tokens of each sequence."""
    n = case["n"]
    return [n if b == 0 or not case["ragged"] else max(1, n - (b * 5) % (n // 2 + 1)) for b in range(case["B"])]


def _lens(case):
    """Cached tokens of each sequence, the new ones among them: the first has all T."""
    part = [0.0 if b == 0 or not case["ragged"] else 0.97 * ((b * 0.6180339887) % 1.0) for b in range(case["B"])]
    return [max(n, int(round(case["T"] * (1.0 - f)))) for n, f in zip(_nodes(case), part)]


def _quantize(x):
    """(codes 0..15, scales, zero-points) of vectors x [..., 128]: fp32 steps, halves to even.  The quotients in 64
    bits rounded to 32 are the 32-bit quotients; the codes are decided on them."""
    x = x.float()
    c = torch.tensor(0.95, device=x.device)
    hi, lo = x.amax(-1).clamp(min=0) * c, x.amin(-1).clamp(max=0) * c
    s = ((hi - lo).double() / 15.0).float()
    s = torch.where(s == 0, torch.ones_like(s), s)
    z = (-lo.double() / s.double()).float().round().clamp(0, 15)
    q = ((x.double() / s.double()[..., None]).float().round() + z[..., None]).clamp(0, 15)
    return q, s, z


def _pool(case, pages, seed):
    """An empty cache: keys' and values' codes, scales and zero-points, with what an earlier request left there."""
    g = torch.Generator(device=DEV).manual_seed(seed * 7 + 3)
    shape = (pages, case["Hkv"], case["page"])
    return [t for _ in range(2) for t in (
        torch.randint(0, 256, shape + (D // 2,), generator=g, device=DEV, dtype=torch.uint8),
        torch.rand(shape, generator=g, device=DEV) + 0.1,
        torch.randint(0, 16, shape, generator=g, device=DEV, dtype=torch.uint8))]


def _slots(case, seed):
    """(slot of each token, pages of the pool): every sequence's tokens lie in order in pages of its own, from some
    place in its first page on; the pages are scattered over the pool.  The last ``pad`` tokens have none (-1)."""
    g = torch.Generator().manual_seed(seed * 11 + 1)
    n, seqs, P = case["n"], case["seqs"], case["page"]
    run = -(-n // seqs)
    first = torch.randint(0, P, (seqs, 1), generator=g)
    local = first + torch.arange(run)
    each = -(-(run + P - 1) // P)
    perm = torch.randperm(seqs * each + 3, generator=g)
    slots = (perm[torch.arange(seqs)[:, None] * each + local // P] * P + local % P).reshape(-1)[:n]
    if case["pad"]:
        slots[-case["pad"]:] = -1
    return slots.to(torch.int32).to(DEV), int(perm.numel())


def _stacked(case, rows, seed):
    """q|k|v rows of new tokens, and their three parts as views [rows, heads, 128]."""
    g = torch.Generator(device=DEV).manual_seed(seed * 13 + 5)
    Hq, Hkv = case["Hq"], case["Hkv"]
    qkv = torch.randn((rows, (Hq + 2 * Hkv) * D), generator=g, device=DEV)
    qkv *= torch.exp(0.4 * torch.randn((rows, 1), generator=g, device=DEV))
    qkv = qkv.to(DTYPE[case["dtype"]] if case["dtype"] != "fp32" else torch.float16)
    q, k, v = qkv.split([Hq * D, Hkv * D, Hkv * D], dim=1)
    return q.unflatten(1, (Hq, D)), k.unflatten(1, (Hkv, D)), v.unflatten(1, (Hkv, D))


def _ancestors(n, g):
    """Visibility [n, n] of a random tree of n drafts: each sees itself and its ancestors; a parent comes before its
    children, most of them near the root, as a drafter's trees are."""
    see = torch.eye(n, dtype=torch.bool)
    for i in range(1, n):
        see[i] |= see[int(torch.rand((), generator=g) ** 1.5 * i)]
    return see


def prepare(case, seed):
    s = {"case": case, "cache": None, "work": None}
    if case["kind"] != "tree":
        s["slots"], pages = _slots(case, seed)
        s["pool"] = _pool(case, pages, seed)
        if case["kind"] == "append":
            _, s["k"], s["v"] = _stacked(case, case["n"], seed)
        return s
    B, P, Hkv = case["B"], case["page"], case["Hkv"]
    nodes, lens = _nodes(case), _lens(case)
    g = torch.Generator().manual_seed(seed * 17 + 2)
    counts = [-(-t // P) for t in lens]
    perm = torch.randperm(sum(counts) + 2, generator=g)
    # the table's rows have room for T tokens; entries that no token needs are -1
    table = torch.full((B, -(-case["T"] // P)), -1, dtype=torch.int32)
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = perm[at:at + c]
        at += c
    s["table"] = table.to(DEV)
    s["starts"] = torch.tensor([0] + nodes, dtype=torch.int32).cumsum(0).to(torch.int32).to(DEV)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["q"] = _stacked(case, sum(nodes), seed)[0]
    s["visible"] = None
    if case["tree"]:
        words = -(-case["n"] // 64)
        see = torch.zeros((sum(nodes), words * 64), dtype=torch.bool)
        at = 0
        for n in nodes:
            see[at:at + n, :n] = _ancestors(n, g)
            at += n
        bits = see.view(-1, words, 64).long() << torch.arange(64)
        s["visible"] = bits.sum(-1).to(DEV)   # bit 63 is the sign: sums of distinct powers wrap as they should
    # the cache: keys and values quantized page by page
    gd = torch.Generator(device=DEV).manual_seed(seed * 19 + 7)
    pages = int(perm.numel())
    s["pool"] = []
    for spread in (0.5, 0.2):
        x = torch.randn((pages, Hkv, P, D), generator=gd, device=DEV)
        x *= torch.exp(spread * torch.randn((pages, Hkv, P, 1), generator=gd, device=DEV))
        codes = torch.empty((pages, Hkv, P, D // 2), dtype=torch.uint8, device=DEV)
        scales = torch.empty((pages, Hkv, P), device=DEV)
        zeros = torch.empty((pages, Hkv, P), dtype=torch.uint8, device=DEV)
        step = max(1, (1 << 24) // (Hkv * P * D))
        for i in range(0, pages, step):
            c, sc, z = _quantize(x[i:i + step].half())
            c = c.to(torch.uint8)
            codes[i:i + step], scales[i:i + step], zeros[i:i + step] = c[..., 0::2] | (c[..., 1::2] << 4), sc, z.to(torch.uint8)
        s["pool"] += [codes, scales, zeros]
        del x
    # what no token of a sequence has reached yet holds nothing that may be used: the largest values
    tail = [(int(table[b, c - 1]), t - (c - 1) * P) for b, (c, t) in enumerate(zip(counts, lens))]
    for i in (1, 4):
        for page, used in tail:
            s["pool"][i][page, :, used:] = math.inf
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------


def _unpack(codes):
    return torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2)


def _plain_append(s):
    case, out = s["case"], []
    P, heads = case["page"], torch.arange(case["Hkv"], device=DEV)
    slots = s["slots"].long()
    keep = slots >= 0
    page, at = slots[keep] // P, slots[keep] % P
    where = (page[:, None], heads[None, :], at[:, None])
    for x, (codes, scales, zeros) in ((s["k"], s["pool"][:3]), (s["v"], s["pool"][3:])):
        q, sc, z = _quantize(x)
        hat = sc[..., None] * (q - z[..., None]) * keep[:, None, None]
        q = q.to(torch.uint8)
        codes[where] = (q[..., 0::2] | (q[..., 1::2] << 4))[keep]
        scales[where], zeros[where] = sc[keep], z.to(torch.uint8)[keep]
        out.append(hat.to(x.dtype))
    return out


def _plain_read(s):
    case, out = s["case"], []
    P, heads = case["page"], torch.arange(case["Hkv"], device=DEV)
    slots = s["slots"].long()
    keep = slots >= 0
    safe = slots.clamp(min=0)
    where = ((safe // P)[:, None], heads[None, :], (safe % P)[:, None])
    for codes, scales, zeros in (s["pool"][:3], s["pool"][3:]):
        hat = scales[where][..., None] * (_unpack(codes[where]).float() - zeros[where].float()[..., None])
        out.append((hat * keep[:, None, None]).to(DTYPE[case["dtype"]]))
    return out


def _plain_tree(s):
    case = s["case"]
    Hq, Hkv, n, T = case["Hq"], case["Hkv"], case["n"], case["T"]
    G, B = Hq // Hkv, case["B"]
    starts, lens = s["starts"].long(), s["lens"].long()
    count = starts[1:] - starts[:-1]
    node = torch.arange(n, device=DEV)
    row = (starts[:-1, None] + node).clamp(max=s["q"].shape[0] - 1)            # [B, n], rows behind the last doubled
    q = s["q"][row].float().view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    table = s["table"].long().clamp(min=0)
    kv = []
    t = torch.arange(table.shape[1] * case["page"], device=DEV)
    live = t < lens[:, None]                                                    # [B, T]
    for codes, scales, zeros in (s["pool"][:3], s["pool"][3:]):
        sc = scales[table].transpose(1, 2).reshape(B, Hkv, -1)                 # [B, Hkv, T]
        z = zeros[table].transpose(1, 2).reshape(B, Hkv, -1)
        c = _unpack(codes[table].transpose(1, 2).reshape(B, Hkv, -1, D // 2))
        sc = torch.where(live[:, None], sc, torch.zeros_like(sc))
        kv.append(sc[..., None] * (c.float() - z.float()[..., None]))
    ctx = (lens - count)[:, None, None]
    j = t[None, None, :] - ctx                                                  # [B, 1, T]: the node at that place
    if s["visible"] is None:
        bit = j <= node[None, :, None]
    else:
        words = s["visible"][row]                                               # [B, n, words]
        jc = j.clamp(0, words.shape[-1] * 64 - 1).expand(B, n, -1)
        bit = (torch.gather(words, 2, jc >> 6) >> (jc & 63)) & 1 == 1
    see = ((j < 0) | bit) & live[:, None, :]                                    # [B, n, T]
    see = see[:, None, :, None, :].expand(B, Hkv, n, G, -1).reshape(B, Hkv, n * G, -1)
    score = torch.matmul(q, kv[0].transpose(2, 3)) / math.sqrt(D)
    score = score.masked_fill(~see, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    out = torch.matmul(p, kv[1]).view(B, Hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)
    return out[node < count[:, None]].to(s["q"].dtype)


# ---- the framework's calls -------------------------------------------------------------------------------------


def _own(s):
    from paper_2606_02823_amd import qift

    case = s["case"]
    if s["cache"] is None:   # the handle and the workspace that a server makes once
        s["cache"] = qift.KV4Pages(qift.KV4(*s["pool"][:3]), qift.KV4(*s["pool"][3:]))
        if case["kind"] == "tree":
            s["work"] = qift.kv4_attention_tree_workspace(case["B"], case["Hq"], case["Hkv"], case["n"], case["T"], device=DEV)
    if case["kind"] == "append":
        return qift.kv4_append(s["cache"], s["k"], s["v"], s["slots"], values=True)
    if case["kind"] == "read":
        return qift.kv4_read(s["cache"], s["slots"], dtype=DTYPE[case["dtype"]])
    return qift.kv4_attention_tree(s["q"], s["cache"], s["table"], s["starts"], s["lens"], max_nodes=case["n"],
                                   max_len=case["T"], visible=s["visible"], workspace=s["work"])


def run(s):
    if own:
        got = _own(s)
    else:
        got = {"append": _plain_append, "read": _plain_read, "tree": _plain_tree}[s["case"]["kind"]](s)
    if s["case"]["kind"] == "append":
        # the values, and the scales and zero-points of the whole cache after the call
        return {"k": got[0], "v": got[1], "k_scales": s["pool"][1], "v_scales": s["pool"][4], "k_zeros": s["pool"][2],
                "v_zeros": s["pool"][5]}
    return got


def work(case):
    Hq, Hkv = case["Hq"], case["Hkv"]
    size = 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "tree":
        nodes, lens = _nodes(case), _lens(case)
        pairs = sum(n * (t - n) + n * (n + 1) // 2 for n, t in zip(nodes, lens))
        return {"bytes": sum(lens) * Hkv * 138 + 2 * sum(nodes) * Hq * D * 2, "flops": 4 * D * Hq * pairs}
    rows = (case["n"] - case["pad"]) * Hkv
    values = 2 * rows * D
    if case["kind"] == "append":   # in, codes and what goes with them, and the values out again
        return {"bytes": values * 2 + rows * 138 + values * 2, "flops": values * 6}
    return {"bytes": rows * 138 + values * size, "flops": values * 2}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------


def _steps64(x):
    """The quantizer with 64-bit arithmetic, each step rounded to the 32 bits that its definition has."""
    r = lambda t: t.float().double()  # noqa: E731
    x = x.double()
    c = r(torch.tensor(0.95, dtype=torch.float64, device=x.device))
    top, bottom = r(c * torch.relu(x.max(-1).values)), r(-c * torch.relu(-x.min(-1).values))
    s = r(r(top - bottom) / 15)
    s[s == 0] = 1.0
    z = torch.round(r(-bottom / s))
    q = torch.clip(torch.round(r(x / s.unsqueeze(-1))) + z.unsqueeze(-1), 0, 15)
    return q, s, z


def exact(case, seed):
    s = prepare(case, seed)
    P, Hkv = case["page"], case["Hkv"]
    nib = lambda c: torch.stack([(c >> 4 * i) & 15 for i in (0, 1)], -1).reshape(*c.shape[:-1], D).double()  # noqa: E731
    if case["kind"] != "tree":
        slots, out = s["slots"].tolist(), []
        rows = torch.tensor([i for i, t in enumerate(slots) if t >= 0], device=DEV)
        page = torch.tensor([t // P for t in slots if t >= 0], device=DEV)
        at = torch.tensor([t % P for t in slots if t >= 0], device=DEV)
        caches = []
        for i, x in enumerate((s.get("k"), s.get("v"))):
            codes, scales, zeros = s["pool"][3 * i:3 * i + 3]
            full = torch.zeros((len(slots), Hkv, D), dtype=torch.float64, device=DEV)
            if case["kind"] == "append":
                q, sc, z = _steps64(x[rows])
                after = scales.double()
                after[page, :, at] = sc
                caches.append(after)
            else:
                q, sc, z = nib(codes[page, :, at]), scales[page, :, at].double(), zeros[page, :, at].double()
            full[rows] = sc[..., None] * (q - z[..., None])
            out.append(full)
        if case["kind"] == "append":
            return {"k": out[0], "v": out[1], "k_scales": caches[0], "v_scales": caches[1], "k_zeros": None, "v_zeros": None}
        return out
    G, out, at = case["Hq"] // Hkv, [], 0
    for b, (n, t) in enumerate(zip(_nodes(case), _lens(case))):
        page = s["table"][b, :-(-t // P)].long()
        k, v = ((sc[page].double()[..., None] * (nib(c[page]) - z[page].double()[..., None])).transpose(0, 1).reshape(Hkv, -1, D)[:, :t]
                for c, sc, z in (s["pool"][:3], s["pool"][3:]))
        q = s["q"][at:at + n].double()
        see = torch.ones((n, t), dtype=torch.bool, device=DEV)
        if s["visible"] is None:
            see[:, t - n:] = torch.tril(see[:, t - n:])
        else:
            for j in range(n):
                see[:, t - n + j] = (s["visible"][at:at + n, j // 64] >> (j % 64)) & 1 == 1
        got = torch.empty((n, case["Hq"], D), dtype=torch.float64, device=DEV)
        for h in range(Hkv):
            a = torch.einsum("ngd,td->ngt", q[:, h * G:(h + 1) * G], k[h]) / math.sqrt(D)
            a = torch.softmax(a.masked_fill(~see[:, None, :], -math.inf), dim=-1)
            got[:, h * G:(h + 1) * G] = torch.einsum("ngt,td->ngd", a, v[h])
        out.append(got)
        at += n
    return torch.cat(out)
