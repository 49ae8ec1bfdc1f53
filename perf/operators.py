"""The operators around a key/value cache that is kept as DyBit codes, as cases that can be timed and compared.

A decoder that runs on this library's products keeps the keys and values of every token it has seen.  Here they are
stored in pages as signed DyBit codes of 4 or 8 bits with one fp32 scale per token and head.  A case is a dict of plain
values; `kind` says which operator it is:

  norm     RMS norm of every query and key head and the rotation by its token's position, in one pass
  train    the same in a training step: forward, and the gradients of the inputs and of the two weights
  append   new keys and values of a layer encoded into the pages of the cache
  attend   attention of new tokens over the pages: one token a sequence, several, or a whole chunk of a prompt; with
           `groups` over 0, sequences of a group also see a prefix that all of them share, stored once
  pages    whole pages copied to others in all layers: sequences forked, or a scattered pool compacted

The heads of queries, keys and values lie side by side in one row a token, as a fused projection leaves them.
"""
import math
import random

import torch

DEV = "cuda"

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
WIDTH = {"fp32": 4, "fp16": 2, "bf16": 2}


def listed():
    return [
        # one decoding step of a small batch: launches and latency are all there is
        {"name": "norm_step", "kind": "norm", "T": 8, "Hq": 32, "Hkv": 8, "D": 128, "rot": 128, "pairs": "halves", "dtype": "bf16"},
        # a prompt of no even length, a quarter of each head left unrotated, neighbours as pairs
        {"name": "norm_prompt", "kind": "norm", "T": 8191, "Hq": 32, "Hkv": 8, "D": 128, "rot": 96, "pairs": "neighbours", "dtype": "bf16"},
        # a fine-tuning step in 32 bits, as many key heads as query heads, short heads
        {"name": "norm_train", "kind": "train", "T": 4097, "Hq": 16, "Hkv": 16, "D": 64, "rot": 64, "pairs": "halves", "dtype": "fp32"},
        # the new tokens of 64 sequences, one each
        {"name": "append_step", "kind": "append", "T": 64, "Hkv": 8, "D": 128, "k_bits": 8, "v_bits": 8, "page": 64, "dtype": "bf16"},
        # a prompt's keys at 8 bits and values at 4, from this library's 32-bit products
        {"name": "append_prompt", "kind": "append", "T": 16383, "Hkv": 8, "D": 128, "k_bits": 8, "v_bits": 4, "page": 32, "dtype": "fp32"},
        # decoding: 64 sequences of very different lengths, four of the places idle
        {"name": "decode_ragged", "kind": "attend", "B": 64, "n": 1, "lo": 200, "hi": 16384, "idle": 4, "Hq": 32, "Hkv": 8, "D": 128,
         "k_bits": 8, "v_bits": 8, "page": 64, "groups": 0, "plo": 0, "phi": 0, "dtype": "bf16"},
        # decoding: one sequence of 128 Ki tokens, 4-bit cache, queries from 32-bit products
        {"name": "decode_long", "kind": "attend", "B": 1, "n": 1, "lo": 131071, "hi": 131071, "idle": 0, "Hq": 32, "Hkv": 4, "D": 128,
         "k_bits": 4, "v_bits": 4, "page": 128, "groups": 0, "plo": 0, "phi": 0, "dtype": "fp32"},
        # a chunk of the prompts of four sequences behind what is already in the cache
        {"name": "prompt_chunk", "kind": "attend", "B": 4, "n": 2048, "lo": 4096, "hi": 8192, "idle": 0, "Hq": 32, "Hkv": 8, "D": 128,
         "k_bits": 8, "v_bits": 8, "page": 64, "groups": 0, "plo": 0, "phi": 0, "dtype": "bf16"},
        # 64 requests that answer from one document of 32 Ki tokens
        {"name": "prefix_decode", "kind": "attend", "B": 64, "n": 1, "lo": 16, "hi": 1024, "idle": 0, "Hq": 32, "Hkv": 8, "D": 128,
         "k_bits": 8, "v_bits": 8, "page": 64, "groups": 1, "plo": 32768, "phi": 32768, "dtype": "bf16"},
        # four instructions of different lengths shared by seven sequences each, up to four drafted tokens verified at once
        {"name": "prefix_groups", "kind": "attend", "B": 28, "n": 4, "lo": 30, "hi": 300, "idle": 0, "Hq": 24, "Hkv": 8, "D": 64,
         "k_bits": 4, "v_bits": 4, "page": 16, "groups": 4, "plo": 1500, "phi": 6000, "dtype": "fp16"},
        # sixteen sequences forked: the page each of them is in the middle of, in all layers
        {"name": "pages_fork", "kind": "pages", "layers": 24, "pages": 640, "n": 16, "Hkv": 4, "D": 64, "k_bits": 8, "v_bits": 4, "page": 16},
        # a scattered pool compacted: a third of its pages move
        {"name": "pages_compact", "kind": "pages", "layers": 16, "pages": 1536, "n": 511, "Hkv": 8, "D": 128, "k_bits": 8, "v_bits": 8,
         "page": 64},
    ]


# ---- drawn cases -------------------------------------------------------------------------------------------------
def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "train", "append", "attend", "attend", "attend", "attend", "pages"])
    D = rng.choice([64, 128, 128, 256])
    bits = lambda: rng.choice([4, 8])  # noqa: E731
    page = rng.choice([16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    Hkv = rng.choice([1, 2, 4, 8, 8])
    group = rng.choice([1, 2, 3, 4, 5, 7, 8])
    if kind in ("norm", "train"):
        D = rng.choice([64, 80, 96, 128, 128, 256])
        rot = D if rng.random() < 0.6 else 2 * rng.randrange(8, D // 2 + 1)
        T = _log_int(rng, 1, 8192 if kind == "norm" else 4096)
        while T * Hkv * (group + 1) * D > 8192 * 40 * 128 // (1 if kind == "norm" else 2):
            T = T // 2
        return {"kind": kind, "T": max(1, T), "Hq": Hkv * group, "Hkv": Hkv, "D": D, "rot": rot,
                "pairs": rng.choice(["halves", "halves", "neighbours"]), "dtype": dtype}
    if kind == "append":
        T = _log_int(rng, 1, 16384)
        while T * Hkv * D > 1 << 24:
            T = T // 2
        return {"kind": kind, "T": T, "Hkv": Hkv, "D": D, "k_bits": bits(), "v_bits": bits(), "page": page, "dtype": dtype}
    if kind == "pages":
        layers = _log_int(rng, 1, 32)
        pages = _log_int(rng, 64, 4096)
        while layers * pages * Hkv * D * page > 16 * 1536 * 8 * 128 * 64:
            pages = pages // 2
        return {"kind": kind, "layers": layers, "pages": max(8, pages), "n": _log_int(rng, 1, max(2, pages // 3)), "Hkv": Hkv, "D": D,
                "k_bits": bits(), "v_bits": bits(), "page": page}
    form = rng.choice(["decode", "decode", "prefix", "prefix", "draft", "chunk"])
    n = {"decode": 1, "prefix": rng.choice([1, 1, 3]), "draft": rng.randrange(2, 17), "chunk": _log_int(rng, 17, 2048)}[form]
    while True:
        B = _log_int(rng, 1, 96) if form != "chunk" else rng.randrange(1, 5)
        hi = _log_int(rng, 1, 65536) if form != "prefix" else _log_int(rng, 1, 2048)
        if form == "chunk":
            hi = min(8192, n + hi)
        lo = max(1, int(hi * rng.choice([0.02, 0.3, 1.0])))
        groups = rng.randrange(1, min(4, B) + 1) if form == "prefix" else 0
        phi = _log_int(rng, 100, 32768) if groups else 0
        plo = max(1, int(phi * rng.choice([0.2, 1.0]))) if groups else 0
        # padded elements of keys, and scores, that the plain form holds
        if (B * hi + groups * phi) * Hkv * D <= 1 << 30 and B * n * group * Hkv * (hi + phi) <= 1 << 31 and \
                B * n * group * Hkv * (hi + phi) * D <= 1 << 38:
            break
    return {"kind": kind, "B": B, "n": n, "lo": lo, "hi": hi, "idle": 1 if B > 4 and rng.random() < 0.3 else 0, "Hq": Hkv * group,
            "Hkv": Hkv, "D": D, "k_bits": bits(), "v_bits": bits(), "page": page, "groups": groups, "plo": plo, "phi": phi, "dtype": dtype}


# ---- lengths: from the case alone, so that its work is known ------------------------------------------------------
def _lengths(case):
    """(tokens of each sequence, its new tokens among them, sequences of each group, tokens of each group's prefix)."""
    rng = random.Random("%(B)d %(n)d %(lo)d %(hi)d %(groups)d %(phi)d" % case)
    B, n = case["B"], case["n"]
    length = [_log_int(rng, case["lo"], case["hi"]) for _ in range(B)]
    length[rng.randrange(B)] = case["hi"]
    for b in rng.sample(range(B), case["idle"]):
        length[b] = 0
    new = [1 if n == 1 else min(length[b], rng.randrange((n + 1) // 2, n + 1)) for b in range(B)]
    if n > 1 and max(length) >= n:
        new[length.index(max(length))] = n
    g = case["groups"]
    cuts = sorted(rng.sample(range(1, B), g - 1)) if g else []
    sizes = [b - a for a, b in zip([0] + cuts, cuts + [B])] if g else []
    if g and B % g == 0:
        sizes = [B // g] * g
    prefix = [_log_int(rng, case["plo"], case["phi"]) for _ in range(g)]
    return length, new, sizes, prefix


# ---- inputs, made from the seed alone ----------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 7919 + 23)


def _magnitudes(bits):
    """Values of the magnitude codes of a signed format: a fraction below 1, then leading ones as the exponent."""
    m = bits - 1
    out = []
    for c in range(1 << m):
        if c < 1 << (m - 1):
            out.append(c / 2 ** (m - 1))
        elif c == (1 << m) - 1:
            out.append(2.0 ** (m - 1))
        else:
            ones = next(i for i in range(m) if not c & (1 << (m - 1 - i)))
            k = m - ones - 1
            out.append(2.0 ** (ones - 1) * (1 + (c & ((1 << k) - 1)) / 2 ** k))
    return out


def _midpoints(bits):
    v = _magnitudes(bits)
    return [(a + b) / 2 for a, b in zip(v, v[1:])]


def _cache_like(g, pages, Hkv, page, D, bits, spread):
    """Codes and scales of `pages` pages such as an encoder leaves: normal values, channels of different size where `spread`."""
    size = torch.exp(0.5 * torch.randn(Hkv, 1, D, generator=g, device=DEV)) if spread else torch.ones(Hkv, 1, D, device=DEV)
    mid = torch.tensor(_midpoints(bits), device=DEV)
    codes = torch.empty(pages, Hkv, page, D * bits // 8, dtype=torch.uint8, device=DEV)
    scales = torch.empty(pages, Hkv, page, device=DEV)
    step = max(1, (1 << 26) // (Hkv * page * D))
    for p in range(0, pages, step):
        x = torch.randn(min(step, pages - p), Hkv, page, D, generator=g, device=DEV).mul_(size)
        s = x.abs().amax(-1) / 2.0 ** (bits - 2)
        c = torch.bucketize((x / s.unsqueeze(-1)).abs_(), mid, out_int32=True)
        c = torch.where((x < 0) & (c > 0), c | 1 << (bits - 1), c).to(torch.uint8)
        codes[p:p + step] = c if bits == 8 else c[..., 0::2] | c[..., 1::2] << 4
        scales[p:p + step] = s
    return codes, scales


def _tables(g, lengths, page, order):
    """Table of the pages of each sequence, taken from `order` (a shuffled pool); -1 where a sequence has none."""
    counts = [-(-n // page) for n in lengths]
    table = torch.full((len(lengths), max(1, max(counts))), -1, dtype=torch.int32)
    at = 0
    for i, c in enumerate(counts):
        table[i, :c] = order[at:at + c]
        at += c
    return table.to(DEV), order[at:]


def _rotation(rot, positions):
    """Tables of cosines and sines of every position, computed in 64 bits once as a model does."""
    angle = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    return angle.cos().float(), angle.sin().float()


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    st = {"case": case}
    if kind in ("norm", "train"):
        T, Hq, Hkv, D, dt = case["T"], case["Hq"], case["Hkv"], case["D"], DTYPES[case["dtype"]]
        size = torch.exp(0.7 * torch.randn(T, Hq + 2 * Hkv, 1, generator=g, device=DEV))
        qkv = (torch.randn(T, Hq + 2 * Hkv, D, generator=g, device=DEV) * size).to(dt)
        st.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], eps=1e-6)
        st["wq"], st["wk"] = (1 + 0.2 * torch.randn(D, generator=g, device=DEV) for _ in range(2))
        st["cos"], st["sin"] = _rotation(case["rot"], 16384)
        # several sequences side by side, each at a place of its own
        st["positions"] = (torch.arange(T, device=DEV) + torch.randint(0, 4096, (1,), generator=g, device=DEV)) % 16384
        if kind == "train":
            st["gq"], st["gk"] = ((1e-3 * torch.randn(T, H, D, generator=g, device=DEV)).to(dt) for H in (Hq, Hkv))
        return st
    Hkv, D, page, kb, vb = case["Hkv"], case["D"], case["page"], case["k_bits"], case["v_bits"]
    host = random.Random(seed)
    if kind == "append":
        T = case["T"]
        pages = -(-T // page) + 16
        kv = torch.randn(T, 2 * Hkv, D, generator=g, device=DEV) * torch.exp(0.5 * torch.randn(T, 2 * Hkv, 1, generator=g, device=DEV))
        kv = kv.to(DTYPES[case["dtype"]])
        st.update(k=kv[:, :Hkv], v=kv[:, Hkv:], cache=_empty_cache(pages, Hkv, page, D, kb, vb))
        if T <= 256:                                                     # one token of each of T sequences, anywhere in the pool
            st["slots"] = torch.tensor(host.sample(range(pages * page), T), dtype=torch.int64, device=DEV)
        else:                                                            # a prompt: full pages in shuffled order, the last one in part
            order = torch.tensor(host.sample(range(pages), pages), device=DEV)
            at = torch.arange(T, device=DEV)
            st["slots"] = order[at // page] * page + at % page
        return st
    if kind == "pages":
        k = torch.randint(0, 256, (case["layers"], case["pages"], Hkv, page, D * kb // 8), generator=g, device=DEV, dtype=torch.uint8)
        v = torch.randint(0, 256, (case["layers"], case["pages"], Hkv, page, D * vb // 8), generator=g, device=DEV, dtype=torch.uint8)
        ks, vs = (torch.rand(case["layers"], case["pages"], Hkv, page, generator=g, device=DEV) + 0.01 for _ in range(2))
        moved = torch.tensor(host.sample(range(case["pages"]), 2 * case["n"]), dtype=torch.int32, device=DEV)
        st.update(cache=(k, ks, v, vs, kb, vb), src=moved[:case["n"]].contiguous(), dst=moved[case["n"]:].contiguous())
        return st
    length, new, sizes, prefix = _lengths(case)
    counts = [-(-n // page) for n in length + prefix]
    pages = sum(counts) + 8
    order = torch.tensor(host.sample(range(pages), pages), dtype=torch.int32)
    k, ks = _cache_like(g, pages, Hkv, page, D, kb, True)
    v, vs = _cache_like(g, pages, Hkv, page, D, vb, False)
    vs *= torch.exp(0.5 * torch.randn(vs.shape, generator=g, device=DEV))
    as_int = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    st["tables"], order = _tables(g, length, page, order)
    st.update(cache=(k, ks, v, vs, kb, vb), lengths=as_int(length), scale=1.0 / math.sqrt(D))
    T = sum(new)
    qkv = 1.5 * torch.randn(T, case["Hq"] + 2 * Hkv, D, generator=g, device=DEV)
    st["q"] = qkv.to(DTYPES[case["dtype"]])[:, :case["Hq"]]
    st["starts"] = as_int([sum(new[:i]) for i in range(len(new) + 1)])
    if sizes:
        st["prefix"], order = _tables(g, prefix, page, order)
        st["prefix_lengths"] = as_int(prefix)
        st["groups"] = as_int([sum(sizes[:i]) for i in range(len(sizes) + 1)])
        st["largest_group"] = max(sizes)
        st["group_queries"] = max(sum(new[sum(sizes[:i]):sum(sizes[:i + 1])]) for i in range(len(sizes)))
    return st


def _empty_cache(pages, Hkv, page, D, kb, vb):
    return (torch.zeros(pages, Hkv, page, D * kb // 8, dtype=torch.uint8, device=DEV), torch.zeros(pages, Hkv, page, device=DEV),
            torch.zeros(pages, Hkv, page, D * vb // 8, dtype=torch.uint8, device=DEV), torch.zeros(pages, Hkv, page, device=DEV), kb, vb)


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(st):
    return (_run_own if own else _run_plain)(st)


def _run_own(st):
    from paper_2302_12510_amd import binding as B
    case = st["case"]
    kind = case["kind"]
    if kind in ("norm", "train"):
        args = (st["q"], st["k"], st["wq"], st["wk"], st["positions"], st["cos"], st["sin"], st["eps"], case["pairs"] == "neighbours")
        q, k = B.dybit_head_norm_rope(*args)
        if kind == "norm":
            return {"q": q, "k": k}
        dq, dk, dwq, dwk = B.dybit_head_norm_rope_bwd(st["gq"], st["gk"], *args)
        return {"q": q, "k": k, "dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}
    cache = B.KVCache(*st["cache"])
    if kind == "append":
        B.dybit_kv_append(st["k"], st["v"], st["slots"], cache)
        return _buffers(st)
    if kind == "pages":
        B.dybit_kv_copy_pages(cache, st["src"], st["dst"])
        return _buffers(st)
    prefix = None
    if "groups" in st:
        prefix = B.SharedPrefix(st["prefix"], st["prefix_lengths"], st["groups"], st["group_queries"])
    return {"out": B.dybit_kv_attention(st["q"], cache, st["tables"], st["lengths"], st["starts"], max_queries=case["n"],
                                        scale=st["scale"], prefix=prefix)}


def _buffers(st):
    """The cache itself: its codes are whole numbers, which have to be equal, and its scales what they were encoded with."""
    k, ks, v, vs, _, _ = st["cache"]
    return {"k": k, "k_scales": ks, "v": v, "v_scales": vs}


# ---- the plain forms: elementary operations in 32 bits ------------------------------------------------------------
def _run_plain(st):
    case = st["case"]
    kind = case["kind"]
    if kind in ("norm", "train"):
        return _plain_norm(st)
    if kind == "append":
        k, ks, v, vs, kb, vb = st["cache"]
        _plain_append(st["k"], st["slots"], k, ks, kb)
        _plain_append(st["v"], st["slots"], v, vs, vb)
        return _buffers(st)
    if kind == "pages":
        for a in st["cache"][:4]:
            a[:, st["dst"]] = a[:, st["src"]]
        return _buffers(st)
    return _plain_attention(st)


def _halves(x, rot, pairs):
    return (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs == "neighbours" else (x[..., :rot // 2], x[..., rot // 2:rot])


def _rotated(x, cos, sin, rot, pairs):
    a, b = _halves(x, rot, pairs)
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((u, v), -1).flatten(-2) if pairs == "neighbours" else torch.cat((u, v), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_norm(st):
    case = st["case"]
    rot, pairs, dt = case["rot"], case["pairs"], DTYPES[case["dtype"]]
    cos, sin = st["cos"][st["positions"]].unsqueeze(1), st["sin"][st["positions"]].unsqueeze(1)
    out = {}
    for name, w, g in (("q", st["wq"], st.get("gq")), ("k", st["wk"], st.get("gk"))):
        x = st[name].float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + st["eps"])
        n = x * r
        out[name] = _rotated(n * w, cos, sin, rot, pairs).to(dt)
        if g is not None:
            back = _rotated(g.float(), cos, -sin, rot, pairs)            # the transposed rotation
            h = back * w
            out["d" + name] = (r * (h - n * (h * n).mean(-1, keepdim=True))).to(dt)
            out["dw" + name] = (back * n).sum((0, 1))
    return out


def _plain_append(x, slots, codes, scales, bits):
    top = (1 << (bits - 1)) - 1
    mid = torch.tensor(_midpoints(bits), device=DEV)
    x = x.float()
    a = x.abs()
    s = a.amax(-1, keepdim=True)
    s = torch.where(s == 0, torch.ones_like(s), s * 2.0 ** -(bits - 2))
    # the side of a decision point, without rounding: a product of it with 12 leading bits of the scale, and one with the rest
    hi = (s.view(torch.int32) & -4096).view(torch.float32)
    lo = s - hi

    def above(j):                                                        # whether a belongs to a code over j; ties go to the even one
        at = mid[j]
        d = (a - at * hi) - at * lo
        return (d > 0) | ((d == 0) & (j % 2 == 1))
    c = torch.bucketize(a / s, mid, out_int32=True)
    c = c - ((c > 0) & ~above((c - 1).clamp(min=0))).int()
    c = c + ((c < top) & above(c.clamp(max=top - 1))).int()
    c = torch.where((x < 0) & (c > 0), c | (top + 1), c).to(torch.uint8)
    if bits == 4:
        c = c[..., 0::2] | c[..., 1::2] << 4
    page = codes.shape[2]
    codes[slots // page, :, slots % page] = c
    scales[slots // page, :, slots % page] = s.squeeze(-1)


def _decoded(codes, scales, bits, tables):
    """fp32 values [sequence][head][token][D] of the pages in `tables`."""
    t = tables.clamp(min=0)
    c = codes[t]
    if bits == 4:
        c = torch.stack((c & 15, c >> 4), -1).flatten(-2)
    m = _magnitudes(bits)
    x = torch.tensor(m + [-v for v in m], device=DEV)[c.int()]
    x *= scales[t].unsqueeze(-1)
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3)


def _plain_attention(st):
    case = st["case"]
    B, n, Hq, Hkv, D = case["B"], case["n"], case["Hq"], case["Hkv"], case["D"]
    G = Hq // Hkv
    k, ks, v, vs, kb, vb = st["cache"]
    first, count = st["starts"][:-1], st["starts"][1:] - st["starts"][:-1]
    i = torch.arange(n, device=DEV)
    real = i < count[:, None]                                            # [B, n]
    at = (first[:, None] + i).clamp(max=st["q"].shape[0] - 1)
    rows = st["q"].float()[at] * st["scale"]                             # [B, n, Hq, D]
    rows = rows.view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    keys, values = _decoded(k, ks, kb, st["tables"]), _decoded(v, vs, vb, st["tables"])
    token = torch.arange(keys.shape[2], device=DEV)
    seen = (st["lengths"][:, None] - (count[:, None] - 1 - i)).clamp(min=0)
    mask = (token < seen[:, :, None]).repeat_interleave(G, 1).unsqueeze(1)       # [B, 1, n G, L]
    score = torch.where(mask, rows @ keys.transpose(-1, -2), float("-inf"))
    values = torch.where((token < st["lengths"][:, None])[:, None, :, None], values, 0.0)
    top = score.amax(-1, keepdim=True)
    if "groups" in st:
        # a group's queries side by side against its prefix
        starts, S, groups = st["groups"], st["largest_group"], case["groups"]
        group = torch.searchsorted(starts[1:].contiguous(), torch.arange(B, device=DEV, dtype=torch.int32), right=True)
        place = torch.arange(B, device=DEV) - starts[group]
        member = (starts[:-1, None] + torch.arange(S, device=DEV)).clamp(max=B - 1)

        def together(x):
            return x[member].permute(0, 2, 1, 3, 4).reshape(groups, Hkv, S * n * G, x.shape[-1])

        def apart(x):
            return x.view(groups, Hkv, S, n * G, x.shape[-1])[group, :, place]
        pkeys, pvalues = _decoded(k, ks, kb, st["prefix"]), _decoded(v, vs, vb, st["prefix"])
        ptoken = torch.arange(pkeys.shape[2], device=DEV)
        inside = ptoken < st["prefix_lengths"][:, None]
        pscore = torch.where(inside[:, None, None], together(rows) @ pkeys.transpose(-1, -2), float("-inf"))
        pvalues = torch.where(inside[:, None, :, None], pvalues, 0.0)
        top = torch.maximum(top, apart(pscore.amax(-1, keepdim=True)))
    base = torch.where(top == float("-inf"), 0.0, top)
    p = torch.exp(score - base)
    total, out = p.sum(-1, keepdim=True), p @ values
    if "groups" in st:
        p = torch.exp(pscore - together(base))
        total = total + apart(p.sum(-1, keepdim=True))
        out = out + apart(p @ pvalues)
    out = out / torch.where(total == 0, 1.0, total)                      # a query that sees nothing: zeros
    out = out.view(B, Hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B * n, Hq, D).to(DTYPES[case["dtype"]])
    result = torch.empty(st["q"].shape, dtype=out.dtype, device=DEV)
    # a place past a sequence's new tokens is written to a row of its own that is dropped
    spare = torch.where(real, at, st["q"].shape[0]).flatten()
    return {"out": torch.cat((result, result[:1])).index_copy_(0, spare, out)[:-1]}


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    kind, D = case["kind"], case["D"]
    if kind in ("norm", "train"):
        n, e = case["T"] * (case["Hq"] + case["Hkv"]) * D, WIDTH[case["dtype"]]
        tables = 8 * D + case["T"] * 8 + min(case["T"], 16384) * case["rot"] * 4
        if kind == "norm":
            return {"bytes": 2 * n * e + tables, "flops": 8 * n}
        return {"bytes": 4 * n * e + tables + 8 * D, "flops": 22 * n}
    rows = lambda tokens: tokens * case["Hkv"] * (D * (case["k_bits"] + case["v_bits"]) // 8 + 8)  # noqa: E731
    if kind == "append":
        n = 2 * case["T"] * case["Hkv"] * D
        return {"bytes": n * WIDTH[case["dtype"]] + rows(case["T"]) + 8 * case["T"], "flops": 4 * n}
    if kind == "pages":
        return {"bytes": 2 * case["layers"] * case["n"] * rows(case["page"]) + 8 * case["n"], "flops": 0}
    length, new, sizes, prefix = _lengths(case)
    seen = sum(sum(max(0, L - i) for i in range(c)) for L, c in zip(length, new))
    at = 0
    for size, p in zip(sizes, prefix):
        seen += p * sum(new[at:at + size])
        at += size
    return {"bytes": rows(sum(length) + sum(prefix)) + 2 * sum(new) * case["Hq"] * D * WIDTH[case["dtype"]] + 8 * case["B"]
            + 4 * sum(-(-n // case["page"]) for n in length + prefix), "flops": 4 * D * case["Hq"] * seen}


# ---- the same results in 64 bits, from the definitions ------------------------------------------------------------
def _value64(code, bits):
    """Value of sign-magnitude codes: Eq. 1 spelled out with integers."""
    m = bits - 1
    c = (code & ((1 << m) - 1)).to(torch.int64)
    rest = (1 << m) - 1 - c                                               # leading ones of c are leading zeros of this
    k = torch.zeros_like(c)
    for b in range(m):
        k = torch.where(rest >> b > 0, torch.full_like(k, b), k)          # bits behind the first zero
    fraction = c & ((1 << k) - 1)
    big = 2.0 ** (m - k - 2).double() * (1 + fraction.double() / 2.0 ** k.double())
    big = torch.where(rest == 0, torch.full_like(big, 2.0 ** (m - 1)), big)
    value = torch.where(c < 1 << (m - 1), c.double() / 2 ** (m - 1), big)
    return torch.where(code >> m > 0, -value, value)


def _codes64(x, bits):
    """Scales, and codes by distance to the values around, of rows of doubles."""
    m = bits - 1
    every = _value64(torch.arange(1 << m, device=DEV), bits)
    s = x.abs().amax(-1, keepdim=True) / 2.0 ** (m - 1)
    s = torch.where(s == 0, torch.ones_like(s), s)
    upper = torch.searchsorted(every * 1.0, (x.abs() / s).contiguous()).clamp(1, (1 << m) - 1)
    down, up = x.abs() - s * every[upper - 1], s * every[upper] - x.abs()
    c = torch.where((up < down) | ((up == down) & (upper % 2 == 0)), upper, upper - 1)
    return s.squeeze(-1), torch.where((x < 0) & (c > 0), c + (1 << m), c)


def exact(case, seed):
    st = prepare(case, seed)
    kind, D = case["kind"], case["D"]
    if kind in ("norm", "train"):
        return _exact_norm(st)
    if kind == "pages":
        return None
    k, ks, v, vs, kb, vb = st["cache"]
    if kind == "append":
        for x, codes, scales, bits in ((st["k"], k, ks, kb), (st["v"], v, vs, vb)):
            s, c = _codes64(x.double(), bits)
            c = c if bits == 8 else c[..., 0::2] + 16 * c[..., 1::2]
            for h in range(case["Hkv"]):
                where = (st["slots"] // case["page"] * case["Hkv"] + h) * case["page"] + st["slots"] % case["page"]
                codes.view(-1, codes.shape[-1])[where] = c[:, h].to(torch.uint8)
                scales.view(-1)[where] = s[:, h].float()
        return {"k": k, "k_scales": ks.double(), "v": v, "v_scales": vs.double()}
    length, new, sizes, prefix = _lengths(case)

    def read(codes, scales, bits, table, tokens, head):
        pages = table[:-(-tokens // case["page"])].long()
        c = codes[pages, head].flatten(0, 1)[:tokens].to(torch.int32)
        if bits == 4:
            c = torch.stack((c % 16, c // 16), -1).flatten(-2)
        return _value64(c, bits) * scales[pages, head].flatten()[:tokens, None].double()
    group_of = [g for g, size in enumerate(sizes) for _ in range(size)]
    G = case["Hq"] // case["Hkv"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    before, at = {}, 0
    for b in range(case["B"]):
        L, c = length[b], new[b]
        for h in range(case["Hkv"]):
            keys, values = read(k, ks, kb, st["tables"][b], L, h), read(v, vs, vb, st["tables"][b], L, h)
            P = 0
            if sizes:
                g = group_of[b]
                P = prefix[g]
                if (g, h) not in before:
                    before[g, h] = (read(k, ks, kb, st["prefix"][g], P, h), read(v, vs, vb, st["prefix"][g], P, h))
                keys, values = torch.cat((before[g, h][0], keys)), torch.cat((before[g, h][1], values))
            if not keys.shape[0]:
                continue
            q = st["q"][at:at + c, h * G:(h + 1) * G].double().reshape(c * G, D) * st["scale"]
            score = q @ keys.T
            last = P + L - (c - 1 - torch.arange(c, device=DEV)).repeat_interleave(G)
            score = score.masked_fill(torch.arange(P + L, device=DEV) >= last[:, None], float("-inf"))
            out[at:at + c, h * G:(h + 1) * G] = (torch.softmax(score, -1).nan_to_num() @ values).view(c, G, D)
        at += c
    return {"out": out}


def _exact_norm(st):
    case = st["case"]
    rot = case["rot"]
    step = 2 if case["pairs"] == "neighbours" else 1
    first = torch.arange(0, rot, 2, device=DEV) if step == 2 else torch.arange(rot // 2, device=DEV)
    second = first + 1 if step == 2 else first + rot // 2
    turn = torch.complex(st["cos"].double(), st["sin"].double())[st["positions"]][:, None]
    out = {}
    for name, w, g in (("q", st["wq"].double(), st.get("gq")), ("k", st["wk"].double(), st.get("gk"))):
        x = st[name].double()
        rms = (x.pow(2).sum(-1, keepdim=True) / case["D"] + st["eps"]).sqrt()
        y = x / rms * w
        z = torch.complex(y[..., first], y[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
        out[name] = y
        if g is not None:
            b = g.double().clone()
            z = torch.complex(b[..., first], b[..., second]) * turn.conj()
            b[..., first], b[..., second] = z.real, z.imag
            out["dw" + name] = (b * x / rms).sum((0, 1))
            out["d" + name] = b * w / rms - x * (b * w * x).sum(-1, keepdim=True) / (case["D"] * rms ** 3)
    return {n: out[n] for n in ("q", "k", "dq", "dk", "dwq", "dwk") if n in out}
