"""Timed cases of the operators between a layer's qkv and o products: rotary
positions, the paged 4-bit K/V cache and attention over it.

Each case is one call, or one chain of calls, that a serving program makes:

  rope   the q and k heads of a qkv output rotated to their positions
  cache  new K and V rows quantized into their pages, then context rows read back
  attn   attention of each sequence's new rows over its pages
  step   all of it for one layer: rotate, append, attend

The plain forms below compute the same with elementary torch operations in 32
bits (angles in 64).

A batch is B sequences; sequence b has n_b new rows and L_b tokens in the cache,
the new ones included.  Both follow from the case alone (_counts).  q, k and v
are column ranges of one qkv buffer, as the product before them writes it.  K
and V rows are N(0, 1) with per-channel ranges 2^U(0, 3), q is N(0, 1); pages
lie in the cache in random order.
"""
import math

import torch

own = False


# --- cases ------------------------------------------------------------------------

def _rope(name, M, heads, extra, D=128, rot=128, interleaved=False, scaling="none", far=8192):
    return {"name": name, "kind": "rope", "M": M, "heads": heads, "extra": extra, "D": D,
            "rot": rot, "interleaved": interleaved, "scaling": scaling, "far": far}


def _cache(name, B, new, past, read, kvh=8, D=128, G=128, page=64, ragged=True):
    return {"name": name, "kind": "cache", "B": B, "new": new, "len": new + past, "read": read,
            "H": 4 * kvh, "kvh": kvh, "D": D, "G": G, "page": page, "ragged": ragged,
            "mixed": False, "window": 0}


def _attn(name, B, new, length, H, kvh, D=128, G=128, page=64, ragged=False, mixed=False,
          window=0, kind="attn"):
    return {"name": name, "kind": kind, "B": B, "new": new, "len": length, "H": H, "kvh": kvh,
            "D": D, "G": G, "page": page, "ragged": ragged, "mixed": mixed, "window": window}


def listed():
    return [
        # one user's token of a 32 + 8 head layer: latency
        _rope("rope_m1", 1, 40, 8),
        # a ragged prompt, pairs interleaved, half of each head rotated, stretched context
        _rope("rope_m4001_partial", 4001, 72, 8, rot=64, interleaved=True, scaling="bands",
              far=131072),
        # 16 users' tokens enter the cache; the last ones are read back
        _cache("cache_decode_b16", 16, 1, 1000, 16, ragged=False, page=16),
        # prompts enter it, the finest groups; the whole contexts are read back
        _cache("cache_prefill_b8", 8, 4096, 500, 4596, G=32),
        # one user, short context: latency of the whole operator
        _attn("attn_decode_b1_l100", 1, 1, 100, 32, 8, page=16),
        # a serving batch of 64 users with contexts up to 8192 tokens
        _attn("attn_decode_b64_l8192", 64, 1, 8192, 64, 8, ragged=True),
        # one user with a very long context: the split along it
        _attn("attn_decode_b1_l131072", 1, 1, 131072, 32, 8, page=128),
        # drafts of 5 tokens are verified, ungrouped heads of 64 channels, groups of 32
        _attn("attn_draft_b16_mha64", 16, 5, 2000, 12, 12, D=64, G=32, page=32, ragged=True),
        # a chunk of a long prompt
        _attn("attn_chunk_512_l16384", 1, 512, 16384, 64, 8),
        # ragged prompts from empty caches
        _attn("attn_prefill_b4_l2048", 4, 2048, 2048, 32, 8, G=64, ragged=True),
        # the same with a sliding window
        _attn("attn_prefill_b2_window", 2, 3000, 3000, 32, 8, window=1000, ragged=True),
        # a mixed batch: decoding users and one chunk, the whole chain of a layer
        _attn("step_mixed_b9", 9, 256, 4096, 32, 8, mixed=True, ragged=True, kind="step"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "cache", "cache", "attn", "attn", "attn", "attn", "step"])
    D = rng.choice([64, 128, 128])
    kvh = rng.choice([1, 2, 4, 8, 8])
    H = kvh * rng.choice([1, 2, 4, 8, 8])
    if kind == "rope":
        return {"kind": kind, "M": _log(rng, 1, 4096), "heads": H + kvh, "extra": kvh, "D": D,
                "rot": rng.choice([D, D, D // 2, D // 4, D // 2 + 2]),
                "interleaved": rng.random() < 0.5,
                "scaling": rng.choice(["none", "linear", "bands"]), "far": _log(rng, 100, 131072)}
    case = {"kind": kind, "B": _log(rng, 1, 64), "new": 1, "len": 1, "H": H, "kvh": kvh, "D": D,
            "G": rng.choice([g for g in (32, 64, 128, 128) if g <= D]),
            "page": rng.choice([16, 32, 64, 128]), "ragged": rng.random() < 0.7, "mixed": False,
            "window": 0}
    if kind == "cache":
        case["new"] = 1 if rng.random() < 0.4 else _log(rng, 2, 2048)
        case["len"] = case["new"] + _log(rng, 1, 2048)
        case["read"] = _log(rng, 1, case["len"])
        while case["B"] > 1 and case["B"] * case["len"] > 32768:
            case["B"] //= 2
        return case
    case["new"] = 1 if rng.random() < 0.5 else _log(rng, 2, 1024)
    case["len"] = max(case["new"], _log(rng, 8, 32768))
    case["mixed"] = case["new"] > 1 and case["B"] > 1 and rng.random() < 0.4
    if rng.random() < 0.2:
        case["window"] = _log(rng, 16, 4096)
    # no more rows, tokens and scores than the largest listed cases have
    while case["B"] > 1 and (case["B"] * case["len"] > 262144
                             or case["B"] * case["new"] * case["len"] * H > 1 << 28):
        case["B"] = max(1, case["B"] // 2)
    while case["new"] * case["len"] * H > 1 << 28:
        case["new"] = max(1, case["new"] // 2)
    case["mixed"] = case["mixed"] and case["B"] > 1 and case["new"] > 1
    return case


def _counts(case):
    """(n_b, L_b) of every sequence, from the case alone.  Ragged batches spread
    both over (0, 1] of the case's sizes, and from four sequences on the third is
    idle: no rows, no tokens."""
    n, L = [], []
    B = case["B"]
    for b in range(B):
        u, v = (b + 1) * 0.6180339887 % 1.0, (b + 1) * 0.7548776662 % 1.0
        rows = math.ceil(case["new"] * u) if case["ragged"] else case["new"]
        if case["mixed"]:
            rows = 1 if b + 1 < B else case["new"]
        length = math.ceil(case["len"] * v) if case["ragged"] else case["len"]
        if b + 1 == B:  # the largest there is, in every batch
            rows, length = case["new"], case["len"]
        if case["ragged"] and B >= 4 and b == 2:
            rows, length = 0, 0
        n.append(rows)
        L.append(max(rows, length))
    return n, L


def _visible(n, L, window):
    """Sum over the rows of the tokens each sees, and the tokens any of them sees."""
    pairs = tokens = 0
    for rows, length in zip(n, L):
        if not rows:
            continue
        first = length - rows + 1  # tokens up to the first row's position
        w = window if window else length
        full = min(rows, max(0, w - first))  # rows that still see everything before them
        pairs += full * first + full * (full - 1) // 2 + (rows - full) * w
        tokens += min(length, rows - 1 + min(w, first))
    return pairs, tokens


def work(case):
    if case["kind"] == "rope":
        n = case["M"] * case["heads"]
        return {"bytes": 4 * n * case["D"] + 4 * case["M"] + 4 * case["rot"],
                "flops": 3 * n * case["rot"]}
    n, L = _counts(case)
    H, kvh, D, G = case["H"], case["kvh"], case["D"], case["G"]
    M = sum(n)
    row = D // 2 + 4 * (D // G)  # of K or V in the cache, one head
    if case["kind"] == "cache":
        read = sum(min(length, case["read"]) for length in L)
        return {"bytes": 2 * kvh * (M + read) * (2 * D + row), "flops": 0}
    pairs, tokens = _visible(n, L, case["window"])
    w = {"bytes": 2 * kvh * tokens * row + 4 * M * H * D, "flops": 4 * pairs * H * D}
    if case["kind"] == "step":  # q, k and v come in, q and k go out once more, k and v are stored
        w["bytes"] += 2 * M * (H + kvh) * D + 2 * M * (H + kvh) * D + 2 * M * kvh * row
        w["flops"] += 3 * M * (H + kvh) * D
    return w


# --- inputs -----------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _freqs(rot, scaling):
    """Radians per position of the rot / 2 pairs (float64), for base 500000."""
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    f = 500000.0 ** (-2.0 * i / rot)
    if scaling == "linear":
        f = f / 4.0
    elif scaling == "bands":  # long wavelengths slowed 8 times, short ones kept
        turns = 8192.0 * f / (2 * math.pi)
        f = f * (1 / 8 + (1 - 1 / 8) * ((turns - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0))
    return f


def _rows(g, rows, kvh, D):
    """fp16 K or V rows [rows][kvh][D] with per-channel ranges, made in slices."""
    span = torch.exp2(3.0 * torch.rand((kvh, D), generator=g, device="cuda"))
    out = torch.empty((rows, kvh, D), dtype=torch.float16, device="cuda")
    step = max(1, (1 << 26) // (kvh * D))
    for r in range(0, rows, step):
        m = min(step, rows - r)
        out[r:r + m] = torch.randn((m, kvh, D), generator=g, device="cuda") * span
    return out


def _quantized(x, G):
    """(codes uint8 [...][D/2], params fp16 [...][D/G][2]) of fp16 rows [...][D]."""
    v = x.float().unflatten(-1, (-1, G))
    mn, mx = v.amin(dim=-1, keepdim=True), v.amax(dim=-1, keepdim=True)
    s = ((mx - mn) / 15.0).half()
    q = torch.round((v - mn) / torch.where(s > 0, s.float(), 1.0)).clamp(0, 15)
    q = torch.where(s > 0, q, 0.0).to(torch.uint8).flatten(-2)
    return q[..., 0::2] | (q[..., 1::2] << 4), torch.cat([s, mn.half()], dim=-1)


def _values(codes, params):
    """fp32 q * s + mn of codes [...][D/2] and params [...][D/G][2]."""
    q = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).float()
    q = q.unflatten(-1, (params.shape[-2], -1))
    return (q * params[..., 0:1].float() + params[..., 1:2].float()).flatten(-2)


def _pages(codes_rows, params_rows, table, page, pages):
    """A cache [pages][kvh][page][...] that holds rows [B * slots][kvh][...] at the
    table's places."""
    out = []
    for rows in (codes_rows, params_rows):
        kvh = rows.shape[1]
        t = rows.view((-1, page, kvh) + rows.shape[2:]).transpose(1, 2)
        c = torch.zeros((pages,) + t.shape[1:], dtype=rows.dtype, device="cuda")
        c[table.reshape(-1).long()] = t
        out.append(c)
    return out


def _inputs(case, seed):
    g = _gen(seed)
    if case["kind"] == "rope":
        M, D = case["M"], case["D"]
        qkv = torch.randn((M, case["heads"] + case["extra"], D), generator=g, device="cuda").half()
        pos = torch.randint(0, case["far"], (M,), generator=g, device="cuda", dtype=torch.int32)
        return {"x": qkv[:, :case["heads"]], "pos": pos,
                "freqs": _freqs(case["rot"], case["scaling"])}
    n, L = _counts(case)
    B, H, kvh, D, G, page = (case[k] for k in ("B", "H", "kvh", "D", "G", "page"))
    M, width = sum(n), -(-max(max(L), 1) // page)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    starts = [sum(n[:b]) for b in range(B + 1)]
    s = {"row_start": i32(starts), "lens": i32(L), "max_rows": max(n)}
    # each sequence's pages lie anywhere in a cache that has some to spare
    pages = B * width + 3
    s["table"] = torch.randperm(pages, generator=g, device="cuda")[:B * width].view(B, width).int()
    qkv = torch.empty((M, H + 2 * kvh, D), dtype=torch.float16, device="cuda")
    qkv[:, :H] = torch.randn((M, H, D), generator=g, device="cuda")
    qkv[:, H:H + kvh] = _rows(g, M, kvh, D)
    qkv[:, H + kvh:] = _rows(g, M, kvh, D)
    s.update(qkv=qkv, q=qkv[:, :H], k=qkv[:, H:H + kvh], v=qkv[:, H + kvh:])
    for name in ("k", "v"):
        rows = _rows(g, B * width * page, kvh, D)
        parts = [_quantized(rows[r:r + (1 << 16)], G) for r in range(0, rows.shape[0], 1 << 16)]
        s[name + "_codes"], s[name + "_params"] = _pages(
            torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts]), s["table"], page,
            pages)
    # the position of every new row
    rep = torch.repeat_interleave
    count = i32(n).long()
    row = torch.arange(M, device="cuda")
    s["seq"] = rep(torch.arange(B, device="cuda"), count, output_size=M)
    s["pos"] = (s["lens"].long()[s["seq"]] - count[s["seq"]] + row
                - s["row_start"].long()[s["seq"]]).int()
    if case["kind"] == "cache":
        back = [min(length, case["read"]) for length in L]
        s["back_start"] = i32([sum(back[:b]) for b in range(B + 1)])
        s["back_rows"], s["back_max"] = sum(back), max(back)
        s["k_back"], s["v_back"] = (torch.empty((sum(back), kvh, D), dtype=torch.float16,
                                                device="cuda") for _ in "kv")
    else:
        s["out"] = torch.empty((M, H, D), dtype=torch.float16, device="cuda")
        if case["kind"] == "step":
            s["freqs"] = _freqs(D, "none")
            s["qk"] = torch.empty((M, H + kvh, D), dtype=torch.float16, device="cuda")
    return s


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    if case["kind"] == "rope":
        s["out"] = torch.empty((case["M"], case["heads"], case["D"]), dtype=torch.float16,
                               device="cuda")
    return s


# --- one pass ---------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2410_12168_amd as comet

    case = s["case"]
    kind = case["kind"]
    if kind == "rope":
        return comet.rope(s["x"], s["pos"], s["freqs"], interleaved=case["interleaved"],
                          out=s["out"])
    if "handles" not in s:  # a program makes these once, and the workspace with them
        cache = comet.KV4Cache(s["k_codes"], s["k_params"], s["v_codes"], s["v_params"])
        s["handles"] = (cache, comet.KV4Batch(s["row_start"], s["lens"], s["table"],
                                              s["qkv"].shape[0], s["max_rows"]))
        if kind == "cache":
            s["back"] = comet.KV4Batch(s["back_start"], s["lens"], s["table"], s["back_rows"],
                                       s["back_max"])
        else:
            s["work"] = comet.kv4_attention_workspace(s["q"], *s["handles"])
    cache, batch = s["handles"]
    if kind == "cache":
        comet.kv4_append(cache, batch, s["k"], s["v"])
        return comet.kv4_gather(cache, s["back"], k_out=s["k_back"], v_out=s["v_back"])
    q = s["q"]
    if kind == "step":
        H = case["H"]
        qk = comet.rope(s["qkv"][:, :H + case["kvh"]], s["pos"], s["freqs"], out=s["qk"])
        q = qk[:, :H]
        comet.kv4_append(cache, batch, qk[:, H:], s["v"])
    out = comet.kv4_attention(q, cache, batch, window=case["window"], out=s["out"],
                              workspace=s["work"])
    return (out, qk) if kind == "step" else out


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "rope":
        return _plain_rope(s["x"], s["pos"], s["freqs"], case["rot"], case["interleaved"])
    if kind == "cache":
        _plain_append(s, s["k"], s["v"])
        return _plain_gather(s, "k"), _plain_gather(s, "v")
    if kind == "attn":
        return _plain_attention(s, s["q"])
    H, kvh = case["H"], case["kvh"]
    qk = _plain_rope(s["qkv"][:, :H + kvh], s["pos"], s["freqs"], case["D"], False)
    _plain_append(s, qk[:, H:], s["v"])
    return _plain_attention(s, qk[:, :H]), qk


def _plain_rope(x, pos, freqs, rot, interleaved):
    angle = (pos.double()[:, None] * freqs)[:, None]
    c, sn = torch.cos(angle).float(), torch.sin(angle).float()
    v = x.float()
    if interleaved:
        a, b = v[..., 0:rot:2], v[..., 1:rot:2]
        r = torch.stack([a * c - b * sn, b * c + a * sn], dim=-1).flatten(-2)
    else:
        a, b = v[..., :rot // 2], v[..., rot // 2:rot]
        r = torch.cat([a * c - b * sn, b * c + a * sn], dim=-1)
    return torch.cat([r, v[..., rot:]], dim=-1).half()


def _places(s, seq, pos):
    """(page, slot) of tokens `pos` of sequences `seq`."""
    page = s["case"]["page"]
    return s["table"].long()[seq, pos // page], pos % page


def _plain_append(s, k, v):
    pages, slots = _places(s, s["seq"], s["pos"].long())
    for name, rows in (("k", k), ("v", v)):
        codes, params = _quantized(rows, s["case"]["G"])
        s[name + "_codes"][pages, :, slots] = codes
        s[name + "_params"][pages, :, slots] = params


def _plain_gather(s, name):
    start = s["back_start"].long()
    count = start[1:] - start[:-1]
    total = s["back_rows"]
    seq = torch.repeat_interleave(torch.arange(count.shape[0], device="cuda"), count,
                                  output_size=total)
    pos = s["lens"].long()[seq] - count[seq] + torch.arange(total, device="cuda") - start[seq]
    pages, slots = _places(s, seq, pos)
    return _values(s[name + "_codes"][pages, :, slots], s[name + "_params"][pages, :, slots]).half()


def _plain_attention(s, q):
    """Every sequence padded to the longest: rows [B][kvh][n R][D] against tokens
    [B][kvh][L][D]."""
    case = s["case"]
    B, H, kvh, D = (case[k] for k in ("B", "H", "kvh", "D"))
    R, n = H // kvh, s["max_rows"]
    start, lens = s["row_start"].long(), s["lens"].long()
    count = start[1:] - start[:-1]
    rows = start[:-1, None] + torch.arange(n, device="cuda")
    live = torch.arange(n, device="cuda") < count[:, None]
    qp = q.float()[rows.clamp(max=q.shape[0] - 1)]  # [B][n][H][D]
    qp = qp.view(B, n, kvh, R, D).permute(0, 2, 1, 3, 4).reshape(B, kvh, n * R, D)

    def tokens(name):
        c = s[name + "_codes"][s["table"].long()].transpose(1, 2).flatten(2, 3)
        p = s[name + "_params"][s["table"].long()].transpose(1, 2).flatten(2, 3)
        return _values(c, p)

    k = tokens("k")
    x = torch.matmul(qp, k.transpose(2, 3).contiguous()) * D ** -0.5
    del k
    at = (lens - count)[:, None] + torch.arange(n, device="cuda")  # [B][n]
    j = torch.arange(x.shape[-1], device="cuda")
    seen = (j <= at[..., None]) & (j < lens[:, None, None])
    if case["window"]:
        seen = seen & (j > at[..., None] - case["window"])
    seen = seen.repeat_interleave(R, dim=1)[:, None]  # [B][1][n R][L]
    x = x.masked_fill_(~seen, -math.inf)
    x = (x - x.amax(dim=-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = x.sum(dim=-1, keepdim=True)
    o = torch.matmul(x, tokens("v")) / torch.where(total > 0, total, 1.0)
    o = o.view(B, kvh, n, R, D).permute(0, 2, 1, 3, 4).reshape(B, n, H, D)
    return o[live].half()


# --- the same from the definitions, in 64 bits --------------------------------------

def _exact_rotate(x, pos, freqs, rot, interleaved):
    """Pairs as complex numbers, turned by exp(i pos f)."""
    y = x.double().clone()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       torch.outer(pos.double(), freqs))[:, None]
    even = torch.arange(0, rot, 2, device="cuda") if interleaved else torch.arange(rot // 2,
                                                                                   device="cuda")
    odd = even + (1 if interleaved else rot // 2)
    z = torch.complex(y[..., even], y[..., odd]) * turn
    y[..., even], y[..., odd] = z.real, z.imag
    return y


def _exact_group(x, G):
    """What fp16 rows become in the cache, in 64 bits: fp16 scale and offset, codes 0 .. 15."""
    v = x.double().reshape(-1, G)
    low = v.min(dim=1).values[:, None]
    step = ((v.max(dim=1).values[:, None] - low).float() / 15.0).half().double()
    code = torch.where(step > 0, ((v - low) / step.clamp(min=2.0 ** -24)).round().clamp(max=15.0),
                       torch.zeros_like(v))
    return (code * step + low).reshape(x.shape)


def _exact_cached(s, name, b, length):
    """fp64 [length][kvh][D] of sequence b's tokens."""
    page = s["case"]["page"]
    codes, params = s[name + "_codes"], s[name + "_params"].double()
    out = []
    for t in range(0, -(-length // page)):
        p = int(s["table"][b, t])
        c = codes[p].int()
        q = torch.empty(c.shape[:-1] + (2 * c.shape[-1],), dtype=torch.float64, device="cuda")
        q[..., 0::2], q[..., 1::2] = (c % 16).double(), (c // 16).double()
        g = q.reshape(q.shape[:-1] + (-1, s["case"]["G"]))
        g = g * params[p][..., :1] + params[p][..., 1:]
        out.append(g.reshape(q.shape).transpose(0, 1))
    return torch.cat(out)[:length]


def exact(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    if case["kind"] == "rope":
        return _exact_rotate(s["x"], s["pos"], s["freqs"], case["rot"], case["interleaved"])
    n, L = _counts(case)
    H, kvh, D, G = (case[k] for k in ("H", "kvh", "D", "G"))
    k_new, v_new, q, qk = s["k"], s["v"], s["q"].double(), None
    stored = case["kind"] != "attn"
    if case["kind"] == "step":
        qk = _exact_rotate(s["qkv"][:, :H + kvh], s["pos"], s["freqs"], D, False)
        # q and k are kept in fp16 between the calls
        q, k_new = qk[:, :H].half().double(), qk[:, H:].half()
    outs, at = ([], []) if case["kind"] == "cache" else [], 0
    for b, (rows, length) in enumerate(zip(n, L)):
        if not length:
            continue
        k, v = _exact_cached(s, "k", b, length), _exact_cached(s, "v", b, length)
        if stored and rows:
            k[length - rows:] = _exact_group(k_new[at:at + rows], G)
            v[length - rows:] = _exact_group(v_new[at:at + rows], G)
        if case["kind"] == "cache":
            back = min(length, case["read"])
            outs[0].append(k[length - back:])
            outs[1].append(v[length - back:])
        elif rows:
            o = torch.empty((rows, H, D), dtype=torch.float64, device="cuda")
            i = torch.arange(length - rows, length, device="cuda")[:, None]
            j = torch.arange(length, device="cuda")[None]
            hidden = (j > i) | (j <= i - (case["window"] or length))
            for h in range(H):
                x = q[at:at + rows, h] @ k[:, h * kvh // H].t() / math.sqrt(D)
                x[hidden] = -math.inf
                o[:, h] = torch.softmax(x, dim=1) @ v[:, h * kvh // H]
            outs.append(o)
        at += rows
    if case["kind"] == "cache":
        return torch.cat(outs[0]), torch.cat(outs[1])
    return (torch.cat(outs), qk) if case["kind"] == "step" else torch.cat(outs)
