"""Decoding with 4-bit weights and a 4-bit cache: what is measured.

Three operators, each with its listed cases and its range of drawn ones:
  "product"  few rows times an N:M sparse (N = M: dense) weight in 4 bits with
             a scale for every 32 kept rows of a column,
             C = act(alpha * A*B + bias) * mul + residual
  "append"   new keys and values written into a paged cache, of 16- or 32-bit
             values or of 4 bits, with norms of every query and key head and
             rotary positions in the same pass; the 4-bit cache's new rows are
             read back as the values they stand for
  "attend"   attention of one new token per sequence over the 4-bit cache

Four bits are a sign and one of the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6,
times a power of two that 32 values share (of a weight, 32 kept rows of one
column; in the cache, 32 dimensions of a row): the smallest with which the
largest magnitude is at most 7.  Values go to the nearest magnitude, ties to
the one with an even code.

`run` computes the plain form in 32 bits (what is rounded to 4 bits in 64, for
the values next to a border), or, where `own` is set, calls the library.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
LEVELS = ((32, 32), (32, 32), (16, 32), (12, 32), (8, 32), (4, 32), (4, 16), (2, 4))
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-6

# what the largest listed case of each operator costs: no drawn case costs more
MAX_KEPT = 4096 * 11008
MAX_ROWS = 64
MAX_APPEND = 4001 * 8 * 128
MAX_ATTEND = 128 * 8192 * 8 * 128


def _product(name, m, k, n, N, M, V, dtype, out, bias, act, mul, residual):
    return dict(name=name, op="product", m=m, k=k, n=n, N=N, M=M, V=V, dtype=dtype, out=out, bias=bias, act=act,
                mul=mul, residual=residual)


def _append(name, tokens, prompt, heads, group, dim, page, rot, interleaved, norm, dtype, cache):
    return dict(name=name, op="append", tokens=tokens, prompt=prompt, heads=heads, group=group, dim=dim, page=page,
                rot=rot, interleaved=interleaved, norm=norm, dtype=dtype, cache=cache)


def _attend(name, batch, length, ragged, heads, group, dim, page, window, dtype):
    return dict(name=name, op="attend", batch=batch, length=length, ragged=ragged, heads=heads, group=group, dim=dim,
                page=page, window=window, dtype=dtype)


def listed():
    return [
        # decoding one sequence: one token through a sparse layer, added to the residual stream; latency counts
        _product("one_sparse", 1, 8192, 8192, 4, 32, 64, "bf16", "bf16", False, "none", False, True),
        # the same token through a dense gate projection: the matrix-vector product proper
        _product("one_dense_gate", 1, 4096, 11008, 32, 32, 32, "bf16", "bf16", False, "silu", True, False),
        # an odd batch through an MLP up-projection, bias and GELU fused
        _product("batch_13_gelu", 13, 4096, 11008, 8, 32, 32, "f16", "f16", True, "gelu", False, False),
        # the largest batch that is still decoding, down-projection at 50 % with a 32-bit result
        _product("batch_64_down", 64, 11008, 4096, 16, 32, 32, "bf16", "f32", False, "none", False, True),
        # one new token of each of 64 sequences, heads normalised, 16-bit cache; latency counts
        _append("norm_64", 64, False, 8, 4, 128, 16, 128, False, "both", "bf16", "bf16"),
        # a prompt of odd length, heads normalised, straight from 32-bit projections into a 16-bit cache
        _append("norm_prompt_4001", 4001, True, 8, 4, 128, 16, 128, False, "both", "f32", "bf16"),
        # one new token of each of 64 sequences into the 4-bit cache; latency counts
        _append("four_bit_64", 64, False, 8, 4, 128, 16, 128, False, "both", "bf16", "4bit"),
        # a prompt of odd length into the 4-bit cache
        _append("four_bit_prompt_4001", 4001, True, 8, 4, 128, 16, 128, False, "both", "bf16", "4bit"),
        # the start of a conversation: latency counts
        _attend("attend_1_short", 1, 77, False, 8, 4, 128, 16, 0, "bf16"),
        # 48 sequences of lengths from none to 5000 in one batch
        _attend("attend_48_ragged", 48, 5000, True, 8, 8, 128, 16, 0, "f16"),
        # one long document: the work has to be split over its length
        _attend("attend_1_long", 1, 131071, False, 8, 8, 128, 64, 0, "bf16"),
        # a full serving batch (the largest)
        _attend("attend_128_8192", 128, 8192, False, 8, 4, 128, 16, 0, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_product(rng):
    while True:
        N, M = rng.choice(LEVELS)
        V = rng.choice((16, 32, 32, 32, 64, 64, 128))
        m = _log(rng, 1, MAX_ROWS)
        k = max(1, _log(rng, 256, 11008) // 32) * 32
        n = max(1, _log(rng, 256, 11008) // V) * V
        if n * (k // M) * N <= MAX_KEPT and k * n <= 2 * MAX_KEPT and m * n * (k // M) * N <= MAX_ROWS * MAX_KEPT // 2:
            break
    dtype = rng.choice(("bf16", "bf16", "f16"))
    return dict(op="product", m=m, k=k, n=n, N=N, M=M, V=V, dtype=dtype, out=rng.choice((dtype, dtype, "f32")),
                bias=rng.random() < 0.5, act=rng.choice(("none", "relu", "gelu", "silu")), mul=rng.random() < 0.3,
                residual=rng.random() < 0.5)


def _draw_heads(rng):
    heads = rng.choice((1, 2, 4, 5, 8, 8, 16, 32))
    group = rng.choice((1, 2, 3, 4, 4, 7, 8, 16))
    dim = rng.choice((64, 80, 96, 128, 128, 128, 256))
    return heads, group, dim, rng.choice((8, 16, 16, 16, 24, 32, 64))


def _draw_append(rng):
    while True:
        heads, group, dim, page = _draw_heads(rng)
        tokens = _log(rng, 1, 8192)
        if tokens * heads * dim <= MAX_APPEND and tokens * heads * group * dim <= 4 * MAX_APPEND:
            break
    cache = rng.choice(("4bit", "4bit", "4bit", "bf16", "f16", "f32"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32")) if cache == "4bit" else rng.choice((cache, "f32"))
    norm = rng.choice(("both", "both", "both", "q", "k") + (("none",) if cache == "4bit" else ()))
    return dict(op="append", tokens=tokens, prompt=rng.random() < 0.5, heads=heads, group=group, dim=dim, page=page,
                rot=rng.choice((dim, dim, dim // 2, 0)), interleaved=rng.random() < 0.3, norm=norm, dtype=dtype,
                cache=cache)


def _draw_attend(rng):
    while True:
        heads, group, dim, page = _draw_heads(rng)
        batch, length = _log(rng, 1, 256), _log(rng, 1, 131072)
        if batch * length * heads * dim <= MAX_ATTEND and batch * length * heads * dim * group <= 4 * MAX_ATTEND:
            break
    return dict(op="attend", batch=batch, length=length, ragged=rng.random() < 0.6, heads=heads, group=group, dim=dim,
                page=page, window=rng.choice((0, 0, 0, _log(rng, 1, 8192))), dtype=rng.choice(("bf16", "bf16", "f16", "f32")))


def draw(rng):
    return rng.choice((_draw_product, _draw_append, _draw_attend))(rng)


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)


# ---- four bits -------------------------------------------------------------

def _quantised(x):
    """Codes (0 to 15) and exponents of x's groups of 32 along its last
    dimension (the last group may be shorter): x is near the code's magnitude,
    negative from 8 on, times 2 ** exponent."""
    length = x.shape[-1]
    groups = -(-length // 32)
    full = torch.nn.functional.pad(x, (0, groups * 32 - length)).unflatten(-1, (groups, 32))
    mantissa, power = torch.frexp(full.abs().amax(-1))          # mantissa in [0.5, 1); 7 is 0.875 * 2 ** 3
    power = (power - 3 + (mantissa > 0.875).int()).clamp(-125, 125)
    y = torch.ldexp(full, -power[..., None])
    mag = y.abs()
    code = ((mag > 0.25).to(torch.uint8) + (mag >= 0.75) + (mag > 1.25) + (mag >= 1.75) + (mag > 2.5) + (mag >= 3.5)
            + (mag > 5))
    code = torch.where(y < 0, code + 8, code)
    return code.flatten(-2)[..., :length].contiguous(), power.to(torch.int16)


def _values(code, power, dtype=torch.float32):
    """What codes (one a byte) and exponents of groups of 32 along the last dimension stand for."""
    table = torch.tensor(MAGNITUDES + tuple(-x for x in MAGNITUDES), dtype=dtype, device=code.device)
    scale = torch.ldexp(torch.ones((), dtype=dtype, device=code.device), power.int())
    x = torch.index_select(table, 0, code.flatten().int()).view(code.shape)
    return x * scale.repeat_interleave(32, dim=-1)[..., :code.shape[-1]]


# ---- inputs ----------------------------------------------------------------

def _product_inputs(case, seed):
    gen = _generator(seed)
    m, k, n, N, M, V = (case[x] for x in ("m", "k", "n", "N", "M", "V"))
    dtype, out = TYPES[case["dtype"]], TYPES[case["out"]]
    w, q = (k // M) * N, n // V
    keep = torch.rand(k // M, q, M, generator=gen, device="cuda").argsort(-1)[..., :N].sort(-1).values
    # a column's kept rows in a row here: groups of 32 along them
    code, power = _quantised(_randn(gen, n, w, scale=0.02))
    return {
        "A": _randn(gen, m, k, dtype=dtype),
        "codes": code.T.contiguous(),                               # w x n
        "scales": (power.T + 127).to(torch.uint8).contiguous(),     # groups x n: 2 ** (byte - 127)
        "idx": keep.permute(0, 2, 1).reshape(w, q).to(torch.uint8).contiguous(),
        "bias": _randn(gen, n) if case["bias"] else None,
        "mul": _randn(gen, m, n, dtype=out) if case["mul"] else None,
        "residual": _randn(gen, m, n, dtype=out) if case["residual"] else None,
    }


def _rotation(case, positions):
    """cos and sin of the rotary angles, positions x rot/2."""
    half = case["rot"] // 2
    rate = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / max(half, 1))
    angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * rate
    return angle.cos().float(), angle.sin().float()


def _append_inputs(case, seed):
    gen = _generator(seed)
    T, H, G, D, S = (case[x] for x in ("tokens", "heads", "group", "dim", "page"))
    dtype = TYPES[case["dtype"]]
    if case["prompt"]:      # one sequence: T positions in a row after an odd start
        start = 37
        wide = (start + T + S - 1) // S
        pages = wide + 3
        table = torch.randperm(pages, generator=gen, device="cuda")[:wide][None].int()
        seq = torch.zeros(T, dtype=torch.int32, device="cuda")
        pos = torch.arange(start, start + T, device="cuda", dtype=torch.int32)
    else:                   # T sequences, one token each: the pages that are written stand alone
        pages = T + 3
        pos = torch.randint(0, 4096, (T,), generator=gen, device="cuda").int()
        wide = (4096 + S - 1) // S
        last = torch.randperm(pages, generator=gen, device="cuda")[:T]
        table = last[:, None].expand(T, wide).int().contiguous()
        seq = torch.randperm(T, generator=gen, device="cuda").int()
    cos, sin = _rotation(case, int(start + T) if case["prompt"] else 4096)
    # queries, keys and values as one projection writes them: slices of one row a token
    qkv = _randn(gen, T, (G + 2) * H * D, dtype=dtype)
    q_norm, k_norm = (1 + 0.1 * torch.randn(D, generator=gen, device="cuda") for _ in range(2))
    s = {
        "q": qkv[:, :G * H * D].view(T, G * H, D), "k": qkv[:, G * H * D:(G + 1) * H * D].view(T, H, D),
        "v": qkv[:, (G + 1) * H * D:].view(T, H, D),
        "table": table, "seq": seq, "pos": pos, "cos": cos if case["rot"] else None,
        "sin": sin if case["rot"] else None, "pages": pages,
        "q_norm": q_norm if case["norm"] in ("both", "q") else None,
        "k_norm": k_norm if case["norm"] in ("both", "k") else None,
    }
    if case["cache"] != "4bit":
        cache = TYPES[case["cache"]]
        s["k_pages"], s["v_pages"] = (_randn(gen, pages, S, H, D, dtype=cache) for _ in range(2))
    return s


def _lengths(case, seed):
    """The lengths of the sequences, on the host: all of them `length`, or
    from none to `length`, the first one the longest."""
    if not case["ragged"]:
        return [case["length"]] * case["batch"]
    gen = torch.Generator().manual_seed(seed)
    spread = torch.rand(case["batch"], generator=gen).tolist()
    out = [int(math.exp(u * math.log(case["length"] + 1.0))) - 1 if i % 2 else int(u * (case["length"] + 1))
           for i, u in enumerate(spread)]
    out[0] = case["length"]
    return out


def _attend_inputs(case, seed):
    """The queries, the table and the lengths, and the generator that the
    cache's contents come from, page after page."""
    gen = _generator(seed)
    B, H, G, D, S = (case[x] for x in ("batch", "heads", "group", "dim", "page"))
    lengths = _lengths(case, seed)
    need = [(x + S - 1) // S for x in lengths]
    wide = max(1, max(need))
    pages = sum(need) + 1
    # every sequence's pages lie scattered over the cache, which holds no more than they need
    order = torch.randperm(pages - 1, generator=gen, device="cuda").int() + 1
    table = torch.zeros(B, wide, dtype=torch.int32, device="cuda")
    held = torch.arange(wide, device="cuda")[None] < torch.tensor(need, device="cuda")[:, None]
    table[held] = order
    return {"q": _randn(gen, B, G * H, D, dtype=TYPES[case["dtype"]]), "table": table, "pages": pages,
            "lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda")}, gen


def _contents(case, pages, gen):
    """Keys and values of the cache's pages in bf16, some pages at a time:
    (first page, keys, values)."""
    S, H, D = case["page"], case["heads"], case["dim"]
    step = max(1, (1 << 26) // (S * H * D))
    for lo in range(0, pages, step):
        yield lo, *(_randn(gen, min(step, pages - lo), S, H, D, dtype=torch.bfloat16) for _ in range(2))


def _four_bit_cache(case, pages, table):
    """The library's 4-bit cache of that many pages, and the same pages as one sequence."""
    import paper_2503_01253_amd as nm
    S, H, D = case["page"], case["heads"], case["dim"]
    pool = torch.empty(pages, nm.nmspmm_kv4_page_bytes(S, H, D), dtype=torch.uint8, device="cuda")
    row = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    return nm.nmspmm_kv4_cache(pool, table, S, H, D), nm.nmspmm_kv4_cache(pool, row, S, H, D)


def prepare(case, seed):
    if own:
        import paper_2503_01253_amd as nm
    if case["op"] == "product":
        s = _product_inputs(case, seed)
        s["C"] = torch.empty(case["m"], case["n"], dtype=TYPES[case["out"]], device="cuda")
        if own:
            s["weight"] = nm.nmspmm_mx4_pack(s["codes"], s["scales"], s["idx"],
                                             *(case[x] for x in ("n", "k", "N", "M", "V")))
            size = nm.nmspmm_mx4_workspace_bytes(case["m"], s["weight"])
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda") if size > 0 else None
    elif case["op"] == "append":
        s = _append_inputs(case, seed)
        s["q_out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
        if case["cache"] == "4bit":
            s["k_out"], s["v_out"] = (torch.empty(s["k"].shape, device="cuda") for _ in range(2))
            if own:
                s["cache"] = _four_bit_cache(case, s["pages"], s["table"])[0]
            else:       # codes and exponents, as a token's row holds them
                S, H, D = case["page"], case["heads"], case["dim"]
                for x in "kv":
                    s[x + "_codes"] = torch.zeros(s["pages"], S, H, D, dtype=torch.uint8, device="cuda")
                    s[x + "_powers"] = torch.zeros(s["pages"], S, H, -(-D // 32), dtype=torch.int16, device="cuda")
        elif own:
            s["cache"] = nm.nmspmm_kv_cache(s["k_pages"], s["v_pages"], s["table"])
    else:
        s, gen = _attend_inputs(case, seed)
        s["out"] = torch.empty_like(s["q"])
        s["longest"] = case["length"]
        S, H, D, pages = case["page"], case["heads"], case["dim"], s["pages"]
        if own:
            s["cache"], whole = _four_bit_cache(case, pages, s["table"])
            for lo, k, v in _contents(case, pages, gen):
                pos = torch.arange(lo * S, (lo + len(k)) * S, dtype=torch.int32, device="cuda")
                nm.nmspmm_kv4_append(whole, k.view(-1, H, D), v.view(-1, H, D), torch.zeros_like(pos), pos)
            size = nm.nmspmm_kv4_attend_workspace_bytes(s["cache"], H * case["group"], case["length"],
                                                        window=case["window"])
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda") if size > 0 else None
        else:           # two codes a byte
            for x in "kv":
                s[x + "_codes"] = torch.empty(pages, S, H, D // 2, dtype=torch.uint8, device="cuda")
                s[x + "_powers"] = torch.empty(pages, S, H, -(-D // 32), dtype=torch.int16, device="cuda")
            for lo, k, v in _contents(case, pages, gen):
                for x, t in (("k", k), ("v", v)):
                    code, power = _quantised(t.float())
                    s[x + "_codes"][lo:lo + len(t)] = code[..., 0::2] | code[..., 1::2] << 4
                    s[x + "_powers"][lo:lo + len(t)] = power
    s["case"] = dict(case)
    return s


# ---- one pass --------------------------------------------------------------

def _act(x, act):
    if act == "relu":
        return x.clamp_min(0)
    if act == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    if act == "silu":
        return x / (1 + torch.exp(-x))
    return x


def _run_product(s, case):
    alpha = case["M"] / case["N"]
    if own:
        import paper_2503_01253_amd as nm
        return nm.nmspmm_mx4_run(s["A"], s["weight"], s["C"], alpha=alpha, bias=s["bias"], act=case["act"],
                                 mul=s["mul"], residual=s["residual"], workspace=s["workspace"])
    k, n, N, M, V = (case[x] for x in ("k", "n", "N", "M", "V"))
    w = (k // M) * N
    kept = _values(s["codes"].T, s["scales"].T.int() - 127).T       # w x n
    if N == M:
        B = kept
    else:
        at = (torch.arange(w, device="cuda")[:, None] // N * M + s["idx"].int()).repeat_interleave(V, dim=1)
        B = torch.zeros(k, n, device="cuda").scatter_(0, at.long(), kept)
    C = s["A"].float() @ B.contiguous() * alpha
    if s["bias"] is not None:
        C = C + s["bias"]
    C = _act(C, case["act"])
    if s["mul"] is not None:
        C = C * s["mul"].float()
    if s["residual"] is not None:
        C = C + s["residual"].float()
    return C.to(s["C"].dtype)


def _normed(x, weight):
    return x if weight is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.to(x.dtype)


def _rotate(x, cos, sin, interleaved):
    """x (tokens, heads, dim) with its first rot dimensions turned in pairs by
    the angles whose cos and sin (tokens, rot/2) are given."""
    half = cos.shape[-1]
    c, s = cos.to(x.dtype)[:, None], sin.to(x.dtype)[:, None]
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack((a * c - b * s, a * s + b * c), dim=-1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat((a * c - b * s, a * s + b * c), dim=-1)
    return torch.cat((turned, x[..., 2 * half:]), dim=-1)


def _run_append(s, case):
    four = case["cache"] == "4bit"
    if own:
        import paper_2503_01253_amd as nm
        new = dict(cos=s["cos"], sin=s["sin"], q=s["q"], q_out=s["q_out"], interleaved=case["interleaved"],
                   q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS)
        if not four:
            nm.nmspmm_kv_append_norm(s["cache"], s["k"], s["v"], s["seq"], s["pos"], **new)
            return s["k_pages"], s["v_pages"], s["q_out"]
        nm.nmspmm_kv4_append(s["cache"], s["k"], s["v"], s["seq"], s["pos"], **new)
        nm.nmspmm_kv4_read(s["cache"], s["seq"], s["pos"], s["k_out"], s["v_out"])
        return s["k_out"], s["v_out"], s["q_out"]
    pos = s["pos"].long()
    page, slot = s["table"][s["seq"].long(), pos // case["page"]].long(), pos % case["page"]
    # keys that go to 4 bits in 64 bits
    k, q = _normed(s["k"].double() if four else s["k"].float(), s["k_norm"]), _normed(s["q"].float(), s["q_norm"])
    if s["cos"] is not None:
        cos, sin = s["cos"][pos], s["sin"][pos]
        k = _rotate(k, cos, sin, case["interleaved"])
        q = _rotate(q, cos, sin, case["interleaved"])
    s["q_out"].copy_(q)
    if not four:
        s["k_pages"][page, slot] = k.to(s["k_pages"].dtype)
        s["v_pages"][page, slot] = s["v"].to(s["v_pages"].dtype)
        return s["k_pages"], s["v_pages"], s["q_out"]
    for x, t in (("k", k), ("v", s["v"].float())):
        code, power = _quantised(t)
        s[x + "_codes"][page, slot], s[x + "_powers"][page, slot] = code, power
        s[x + "_out"].copy_(_values(s[x + "_codes"][page, slot], s[x + "_powers"][page, slot]))
    return s["k_out"], s["v_out"], s["q_out"]


def _run_attend(s, case):
    if own:
        import paper_2503_01253_amd as nm
        return nm.nmspmm_kv4_attend(s["cache"], s["q"], s["lengths"], s["out"], scale=case["dim"] ** -0.5,
                                    window=case["window"], max_length=s["longest"], workspace=s["workspace"])
    B, H, G, D, S, window = (case[x] for x in ("batch", "heads", "group", "dim", "page", "window"))
    out = torch.empty(B, H, G, D, device="cuda")
    lengths = s["lengths"].long()
    at = torch.arange(s["table"].shape[1] * S, device="cuda")
    keep = at[None] < lengths[:, None]
    if window:
        keep &= at[None] >= lengths[:, None] - window
    q = s["q"].float().view(B, H, G, D) * D ** -0.5
    step = max(1, (1 << 30) // max(1, at.numel() * H * D))      # sequences at a time: 4 GB a copy

    def rows(x, pages):
        byte = s[x + "_codes"][pages]
        code = torch.stack((byte & 15, byte >> 4), dim=-1).flatten(-2)
        return _values(code, s[x + "_powers"][pages]).view(len(pages), -1, H, D)

    for lo in range(0, B, step):
        hi = min(B, lo + step)
        pages, mask = s["table"][lo:hi].long(), keep[lo:hi, None, None]
        score = (q[lo:hi] @ rows("k", pages).permute(0, 2, 3, 1).contiguous()).masked_fill_(~mask, float("-inf"))
        top = score.amax(-1, keepdim=True).clamp_min(-1e30)
        p = torch.exp(score - top)
        total = p.sum(-1, keepdim=True)
        out[lo:hi] = (p @ rows("v", pages).permute(0, 2, 1, 3).contiguous()) / total.clamp_min(1e-30)
    return out.view(B, H * G, D).to(s["q"].dtype)


def run(state):
    case = state["case"]
    return {"product": _run_product, "append": _run_append, "attend": _run_attend}[case["op"]](state, case)


# ---- what a pass cannot do without -----------------------------------------

def _row_bytes(dim):
    """A row of the 4-bit cache: half a byte a dimension, a byte a group of 32."""
    return (dim + 1) // 2 + -(-dim // 32)


def work(case):
    if case["op"] == "product":
        m, k, n, N, M, V = (case[x] for x in ("m", "k", "n", "N", "M", "V"))
        w, q = (k // M) * N, n // V
        rows = m * n * BYTES[case["out"]]
        offsets = 0 if N == M else w * q
        return {"bytes": 2 * m * k + (w * n + 1) // 2 + -(-w // 32) * n + offsets
                + rows * (1 + case["mul"] + case["residual"]) + 4 * n * case["bias"], "flops": 2 * m * n * w}
    heads, group, dim = case["heads"], case["group"], case["dim"]
    if case["op"] == "append":
        T, io = case["tokens"], BYTES[case["dtype"]]
        row = heads * dim * (2 * group + 2) * io + 4 * case["rot"] + 12
        if case["cache"] == "4bit":     # written, read back and handed out in 32 bits
            row += heads * (4 * _row_bytes(dim) + 8 * dim)
        else:
            row += heads * dim * 2 * BYTES[case["cache"]]
        return {"bytes": T * row, "flops": T * heads * (group + 1) * (3 * case["rot"] + 4 * dim)}
    # lengths differ with the seed: those of seed 0 stand for them
    held = [min(x, case["window"]) if case["window"] else x for x in _lengths(case, 0)]
    entries = sum((x + case["page"] - 1) // case["page"] for x in held)
    return {"bytes": 2 * sum(held) * heads * _row_bytes(dim) + 4 * entries + 4 * case["batch"]
            + 2 * case["batch"] * heads * group * dim * BYTES[case["dtype"]],
            "flops": 4 * sum(held) * heads * group * dim}


# ---- the definition in 64 bits ---------------------------------------------

def _nearest(x):
    """x (fp64) rounded to four bits in groups of 32 along its last dimension."""
    out = torch.empty_like(x)
    for lo in range(0, x.shape[-1], 32):
        part = x[..., lo:lo + 32]
        top = part.abs().amax(-1, keepdim=True)
        unit = torch.exp2(torch.floor(torch.log2(top.clamp_min(1e-300))) - 2)
        unit = torch.where(top > 7 * unit, 2 * unit, unit).clamp(2.0 ** -125, 2.0 ** 125)
        mag = (part / unit).abs()
        step = torch.where(mag < 2, 0.5, torch.where(mag < 4, 1.0, 2.0)).double()
        out[..., lo:lo + 32] = torch.copysign((torch.round(mag / step) * step).clamp_max(6) * unit, part)
    return out


def _exact_product(case, seed):
    s = _product_inputs(case, seed)
    k, n, N, M, V = (case[x] for x in ("k", "n", "N", "M", "V"))
    low = (s["codes"] & 7).double()
    # codes 0 to 3 are halves; from 4 on, (2 + the last bit) * 2 ** (code / 2 - 2)
    mag = torch.where(low < 4, low / 2, (2 + low % 2) * torch.exp2(torch.floor(low / 2) - 2))
    values = torch.where(s["codes"] >= 8, -mag, mag)
    for g in range(s["scales"].shape[0]):
        values[32 * g:32 * g + 32] *= torch.exp2(s["scales"][g].double() - 127)
    # window by window: the kept rows of the weight at their places
    rows = s["idx"].view(k // M, N, n // V).long()
    B = torch.zeros(k // M, M, n // V, V, dtype=torch.float64, device="cuda")
    B.scatter_(1, rows[..., None].expand(-1, -1, -1, V), values.view(k // M, N, n // V, V))
    y = s["A"].double().mm(B.view(k, n)).mul_(M).div_(N)
    if s["bias"] is not None:
        y += s["bias"].double()
    if case["act"] == "relu":
        y = torch.where(y > 0, y, torch.zeros_like(y))
    elif case["act"] == "gelu":
        y = y * 0.5 * torch.erfc(-y / math.sqrt(2.0))
    elif case["act"] == "silu":
        y = y * torch.sigmoid(y)
    if s["mul"] is not None:
        y *= s["mul"].double()
    return y if s["residual"] is None else y + s["residual"].double()


def _exact_append(case, seed):
    s = _append_inputs(case, seed)
    pos = s["pos"].long()

    def turned(x, weight):
        x = x.double().clone()
        if weight is not None:
            x = weight.double() * x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS)
        half = case["rot"] // 2
        if half:
            # each pair as a complex number times exp(i angle)
            z = torch.complex(s["cos"].double(), s["sin"].double())[pos][:, None]
            first = slice(0, 2 * half, 2) if case["interleaved"] else slice(0, half)
            second = slice(1, 2 * half, 2) if case["interleaved"] else slice(half, 2 * half)
            y = torch.complex(x[..., first], x[..., second]) * z
            x[..., first], x[..., second] = y.real, y.imag
        return x

    k, v = turned(s["k"], s["k_norm"]), s["v"].double()
    if case["cache"] == "4bit":
        return _nearest(k), _nearest(v), turned(s["q"], s["q_norm"])
    flat = s["table"][s["seq"].long(), torch.div(pos, case["page"], rounding_mode="floor")].long() * case["page"]
    flat = flat + torch.remainder(pos, case["page"])
    pools = []
    for pages, new in ((s["k_pages"], k), (s["v_pages"], v)):
        pool = pages.double()
        pool.view(-1, *pages.shape[2:]).index_copy_(0, flat, new)
        pools.append(pool)
    return pools[0], pools[1], turned(s["q"], s["q_norm"])


def _exact_attend(case, seed):
    s, gen = _attend_inputs(case, seed)
    B, H, G, D, S, window = (case[x] for x in ("batch", "heads", "group", "dim", "page", "window"))
    pools = [torch.empty(s["pages"], S, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for lo, k, v in _contents(case, s["pages"], gen):       # a value of 4 bits is one of bf16
        for pool, t in zip(pools, (k, v)):
            for i in range(0, len(t), 64):
                pool[lo + i:lo + i + 64] = _nearest(t[i:i + 64].double()).bfloat16()
    out = torch.zeros(B, H * G, D, dtype=torch.float64, device="cuda")
    for b, length in enumerate(_lengths(case, seed)):
        first = max(0, length - window) if window else 0
        if first >= length:
            continue
        at = torch.arange(first, length, device="cuda")
        flat = s["table"][b][at // S].long() * S + at % S
        for h in range(H):
            K, V = (pool.view(-1, H, D)[flat, h].double() for pool in pools)
            score = s["q"][b, h * G:(h + 1) * G].double() @ K.T.contiguous() / math.sqrt(D)
            out[b, h * G:(h + 1) * G] = torch.softmax(score, dim=-1) @ V
    return out


def exact(case, seed):
    return {"product": _exact_product, "append": _exact_append, "attend": _exact_attend}[case["op"]](case, seed)
