"""Timed cases of what a serving step does around its paged cache, and of a cache
in 4 bits: pages given to new tokens and taken back, rotary positions, rows
rotated on their way into the pages, the 4-bit pages written, read back and
attended.

Kinds of case
  pages   paged_reserve, then paged_release of the same tokens (drafted tokens
          that are all refused): pages from the pool's free list into the block
          tables, the tokens' offsets, positions and cache rows
  rope    rope: queries and keys turned by their tokens' positions, or, going
          back, a gradient with respect to the turned ones into one with respect
          to the plain ones
  rotate  paged_rope_kv_append: the new tokens' queries turned, their keys turned
          on the way to their pages, their values beside them
  cycle4  paged_kv_append into a 4-bit cache, then paged_kv_read of everything
          the cache holds: what later readers of these tokens will see
  attn4   paged_attn over a 4-bit cache: the new tokens of a ragged batch attend
          to their pages, themselves included

A 4-bit row is e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) with one power of two
per 32 elements: x is stored as e2m1(x / 2^k), k the least integer with
max |x| / 2^k <= 6, and k + 127 in a byte.  A byte of a page holds two elements,
the even one in its low half; a head's tokens lie one after another in a page.

Shapes: videos of up to 256 frames give prefixes of thousands to tens of
thousands of tokens and about 13 event streams of about 42 tokens; 28 query
heads over 4 kv heads of width 128 as in a 7B Omni-LLM.  Scores have a standard
deviation of about 1.5 nats; pages lie in the pool in no order.
"""
import math

import torch

own = False

Q_SIGMA, K_SIGMA, V_SIGMA = 1.5, 1.0, 0.5
HEADS = [(28, 4), (28, 4), (28, 4), (16, 2), (8, 8), (7, 1), (32, 8), (40, 8)]
HALF = {"rot": 128, "inter": False, "scaling": "none", "theta": 1e6, "factor": 1.0, "original": 0}
FAR = {"rot": 128, "inter": False, "scaling": "by_parts", "theta": 1e4, "factor": 8.0, "original": 4096}
PART = {"rot": 64, "inter": True, "scaling": "none", "theta": 1e4, "factor": 1.0, "original": 0}


def listed():
    return [
        # A decode step's tables: one token of each of 32 captions, few of which begin a page.
        {"name": "pages_tokens", "kind": "pages", "page": 16, "S": 32, "n_lo": 1, "n_hi": 1, "len_lo": 1200,
         "len_hi": 16384, "budget": 32},
        # Admission of a large batch of prompts and chunks, more than the step's budget of tokens takes.
        {"name": "pages_prompts", "kind": "pages", "page": 16, "S": 1500, "n_lo": 1, "n_hi": 511, "len_lo": 511,
         "len_hi": 9000, "budget": 300000},
        # The rotation of a decode step alone: the smallest.
        {"name": "rope_tokens", "kind": "rope", "dtype": "bf16", "H_q": 28, "H_kv": 4, "D": 128, "T": 32,
         "pos_hi": 16384, "back": False, **HALF},
        # Training: float32 gradients of a packed batch, half of each head turned, neighbours paired.
        {"name": "rope_grad_f32", "kind": "rope", "dtype": "f32", "H_q": 28, "H_kv": 4, "D": 128, "T": 8001,
         "pos_hi": 8001, "back": True, **PART},
        # Serving: one new token of each of 32 captions.
        {"name": "rotate_tokens", "kind": "rotate", "dtype": "bf16", "H_q": 28, "H_kv": 4, "D": 128, "page": 64,
         "S": 32, "n_lo": 1, "n_hi": 1, "len_lo": 100, "len_hi": 2000, **HALF},
        # Prefill chunks of a long video at positions far beyond the trained length.
        {"name": "rotate_chunks", "kind": "rotate", "dtype": "bf16", "H_q": 28, "H_kv": 4, "D": 128, "page": 64,
         "S": 5, "n_lo": 1999, "n_hi": 4096, "len_lo": 4096, "len_hi": 33000, **FAR},
        # A decode step's tokens into small 4-bit caches, and those read back.
        {"name": "cycle4_tokens", "kind": "cycle4", "dtype": "bf16", "H_q": 32, "H_kv": 8, "D": 64, "page": 16,
         "S": 13, "n_lo": 1, "n_hi": 1, "len_lo": 48, "len_hi": 735},
        # Prefill chunks into a 4-bit cache, and the whole cache as the dense prefix that the event step takes.
        {"name": "cycle4_chunks", "kind": "cycle4", "dtype": "bf16", "H_q": 28, "H_kv": 4, "D": 128, "page": 64,
         "S": 3, "n_lo": 999, "n_hi": 4096, "len_lo": 4096, "len_hi": 16383},
        # One token of one short sequence, a float32 reference run.
        {"name": "attn4_f32_token", "kind": "attn4", "dtype": "f32", "H_q": 4, "H_kv": 1, "D": 64, "page": 16, "S": 1,
         "n_lo": 1, "n_hi": 1, "len_lo": 300, "len_hi": 300, "causal": True},
        # Serving: one new token of each of 32 captions over prefixes of their own lengths.
        {"name": "attn4_tokens", "kind": "attn4", "dtype": "bf16", "H_q": 28, "H_kv": 4, "D": 128, "page": 64, "S": 32,
         "n_lo": 1, "n_hi": 1, "len_lo": 1200, "len_hi": 16384, "causal": True},
        # Drafted tokens of 13 streams, narrow heads, small pages that end anywhere.
        {"name": "attn4_drafts", "kind": "attn4", "dtype": "bf16", "H_q": 32, "H_kv": 8, "D": 64, "page": 16, "S": 13,
         "n_lo": 2, "n_hi": 9, "len_lo": 777, "len_hi": 9001, "causal": True},
        # Chunked prefill of a long video, its last chunk: the largest.
        {"name": "attn4_chunk_32k", "kind": "attn4", "dtype": "bf16", "H_q": 28, "H_kv": 4, "D": 128, "page": 64,
         "S": 1, "n_lo": 2048, "n_hi": 2048, "len_lo": 32768, "len_hi": 32768, "causal": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _turning(rng, D):
    scaling = rng.choice(["none", "none", "linear", "ntk", "by_parts"])
    return {"rot": rng.choice([x for x in (16, 32, 48, 64, 96, 128, 128) if x <= D]), "inter": rng.random() < 0.4,
            "scaling": scaling, "theta": rng.choice([1e4, 5e5, 1e6]),
            "factor": 1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 2.5]),
            "original": rng.choice([2048, 4096, 8192]) if scaling == "by_parts" else 0}


def draw(rng):
    while True:
        kind = rng.choice(["pages", "rope", "rotate", "cycle4", "attn4", "attn4", "attn4", "attn4"])
        D = rng.choice([64, 128, 128])
        H_q, H_kv = rng.choice(HEADS)
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        if kind == "rope":
            case = {"kind": kind, "dtype": dtype, "H_q": H_q, "H_kv": H_kv, "D": D, "T": _log(rng, 1, 20000),
                    "pos_hi": _log(rng, 100, 200000), "back": rng.random() < 0.4, **_turning(rng, D)}
        else:
            S = _log(rng, 1, 2000 if kind == "pages" else 40)
            n_hi = 1 if rng.random() < 0.3 else _log(rng, 1, 4096 if kind == "rotate" else 2048)
            len_hi = max(_log(rng, 17, 33000), n_hi)
            case = {"kind": kind, "page": rng.choice([16, 32, 64, 128, 256]), "S": S, "n_lo": _log(rng, 1, n_hi),
                    "n_hi": n_hi, "len_lo": max(_log(rng, 1, len_hi), n_hi), "len_hi": len_hi}
            if kind == "pages":
                case["budget"] = max(int(rng.uniform(0.5, 1.3) * sum(_sizes(case)[0])), 1)
            else:
                case.update(dtype=dtype, H_q=H_q, H_kv=H_kv, D=D)
            if kind == "rotate":
                case.update(_turning(rng, D))
            if kind == "attn4":
                case["causal"] = rng.random() < 0.8
        if _fits(case):
            return case


def _spread(first, other, count, step):
    """count whole numbers between two, both among them, every step-th after the first and round again."""
    return [first + (other - first) * ((i * step) % count) // (count - 1) for i in range(count)]


def _stride(count):
    return next(x for x in range(max(1, count * 5 // 8), count + 2) if math.gcd(x, count) == 1)


def _sizes(case):
    """(new tokens, length with them) of every sequence."""
    S = case["S"]
    if S == 1:
        return [case["n_hi"]], [case["len_hi"]]
    n = _spread(case["n_hi"], case["n_lo"], S, 1)
    return n, _spread(case["len_lo"], case["len_hi"], S, _stride(S))  # the shortest has the largest chunk


def _pages(length, page):
    return (length + page - 1) // page


def _fits(case):
    """No more work than the largest listed case, in the plain form too, which pads every sequence to the longest."""
    if case["kind"] == "pages":
        return sum(_sizes(case)[0]) <= 400000 and case["S"] * _pages(case["len_hi"], case["page"]) <= 2000000
    w = work(case)
    if w["bytes"] > 3e8 or w["flops"] > (0.9e12 if case["dtype"] == "bf16" else 0.1e12):
        return False
    if case["kind"] == "rope":
        return True
    padded = case["S"] * case["len_hi"]
    if case["kind"] == "attn4":
        return padded <= 600000 and padded * case["n_hi"] * case["H_q"] <= 2 ** 31
    return padded <= 600000 and padded * case["H_kv"] * case["D"] <= 2 ** 29


def work(case):
    if case["kind"] == "pages":
        n, lens = _sizes(case)
        taken = tokens = 0
        for a, t in zip(n, lens):
            if tokens + a > case["budget"]:
                break
            tokens += a
            taken += _pages(t, case["page"]) - _pages(t - a, case["page"])
        # lengths and requests in, offsets out; positions and rows; the entries and free pages, both ways
        return {"bytes": 16 * case["S"] + 12 * tokens + 16 * taken, "flops": 3 * tokens + case["S"]}
    H_q, H_kv, D = case["H_q"], case["H_kv"], case["D"]
    esz = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "rope":
        heads = case["T"] * (H_q + H_kv)
        return {"bytes": heads * 2 * D * esz + 4 * case["T"], "flops": heads * 3 * case["rot"]}
    n, lens = _sizes(case)
    T, total = sum(n), sum(lens)
    dense = 2 * H_kv * D * esz             # one token's keys and values
    row = 2 * H_kv * (D // 2 + D // 32)    # the same in 4 bits
    tables = 4 * sum(_pages(t, case["page"]) for t in lens) + 8 * case["S"]
    if case["kind"] == "rotate":
        new = 4 * sum(_pages(t, case["page"]) - (t - a) // case["page"] for a, t in zip(n, lens))
        return {"bytes": 2 * T * (H_q * D * esz + dense) + new + 16 * case["S"], "flops": T * (H_q + H_kv) * 3 * case["rot"]}
    if case["kind"] == "cycle4":
        return {"bytes": T * (dense + row) + total * (row + dense) + tables, "flops": (T + total) * 2 * H_kv * D}
    seen = sum(a * t - a * (a - 1) // 2 if case["causal"] else a * t for a, t in zip(n, lens))
    return {"bytes": total * row + T * H_q * (2 * D * esz + 4) + tables, "flops": 4 * H_q * D * seen}


def _torch_dtype(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _power(byte):
    """2^(byte - 127) as float32: the byte is the number's exponent field."""
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _quantise4(x):
    """Rows x [..., D] as (bytes of two values [..., D / 2], exponent bytes [..., D / 32]).  Dividing by a power of
    two is exact."""
    x = x.float().unflatten(-1, (-1, 32))
    amax = x.abs().amax(-1)
    m, e = torch.frexp(amax)  # amax = m 2^e, 0.5 <= m < 1; 6 = 0.75 * 2^3
    k = torch.where(m <= 0.75, e - 3, e - 2)
    k = torch.where(amax > 0, k.clamp(-126, 125), torch.zeros_like(k))
    byte = (k + 127).to(torch.uint8)
    y = x * _power(254 - byte)[..., None]
    a = y.abs()  # a tie goes to the neighbour whose code is even
    code = (a > 0.25).to(torch.uint8)
    for tie_up, border in ((True, 0.75), (False, 1.25), (True, 1.75), (False, 2.5), (True, 3.5), (False, 5.0)):
        code += (a >= border) if tie_up else (a > border)
    code = (code + 8 * (y < 0).to(torch.uint8)).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], byte


def _values4(x):
    """The e2m1 values of bytes x [..., D / 2] as float32 [..., D]."""
    code = torch.stack((x & 15, x >> 4), -1).flatten(-2).long()
    mags = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    return torch.tensor(mags + [-v for v in mags], device=x.device)[code]


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _starts(counts):
    """[0, the sums of the first 1, 2, .. counts]"""
    return torch.nn.functional.pad(counts.cumsum(0), (1, 0)).to(torch.int32)


def _normal(g, shape, sigma, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * sigma).to(dtype)


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    st = {"case": case}
    if case["kind"] == "rope":
        shape, dtype = (case["T"], case["H_q"] + 2 * case["H_kv"], case["D"]), _torch_dtype(case["dtype"])
        x = _normal(g, shape, Q_SIGMA, dtype)  # queries, keys and values as one projection leaves them
        st["q"], st["k"] = x[:, :case["H_q"]], x[:, case["H_q"]:case["H_q"] + case["H_kv"]]
        st["pos"] = torch.randint(0, case["pos_hi"], (case["T"],), generator=g, device="cuda", dtype=torch.int32)
        return st
    n, lens = _sizes(case)
    page = case["page"]
    cols, total = _pages(max(lens), page), sum(_pages(t, page) for t in lens) + 8
    st["seq_lens"], st["lens_in"], st["n"] = _i32(lens), _i32(lens) - _i32(n), _i32(n)
    held = st["lens_in"] if case["kind"] == "pages" else st["seq_lens"]
    used = (held + page - 1) // page
    col = torch.arange(cols, device="cuda")
    order = torch.randperm(total, generator=g, device="cuda")
    at = (_starts(used)[:-1, None] + col).clamp(max=total - 1)
    st["table"] = torch.where(col < used[:, None], order[at], -1).to(torch.int32)
    if case["kind"] == "pages":
        left = total - used.sum()  # free pages, a stack
        st["free"] = torch.where(torch.arange(total, device="cuda") < left, order.flip(0), -1).to(torch.int32)
        st["free_n"] = left.to(torch.int32).reshape(1)
        st["free_mid"], st["free_out"] = torch.zeros_like(st["free_n"]), torch.zeros_like(st["free_n"])
        st["cu"] = torch.zeros(case["S"] + 1, dtype=torch.int32, device="cuda")
        st["pos"] = torch.zeros(case["budget"], dtype=torch.int32, device="cuda")
        st["slots"] = torch.zeros(case["budget"], dtype=torch.int64, device="cuda")
        return st
    dtype, H_q, H_kv, D = _torch_dtype(case["dtype"]), case["H_q"], case["H_kv"], case["D"]
    st["T"], st["rows"] = sum(n), sum(lens)
    st["cu"], st["cu_rows"] = _starts(st["n"]), _starts(st["seq_lens"])
    st["lens_out"] = torch.zeros_like(st["seq_lens"])
    for name, sigma in (("k", K_SIGMA), ("v", V_SIGMA)):
        if case["kind"] == "rotate":
            st[name + "_pages"] = _normal(g, (total, page, H_kv, D), sigma, dtype)
        else:
            st[name + "_pages"], st[name + "_scales"] = _quantise4(_normal(g, (total, H_kv, page, D), sigma, dtype))
        if case["kind"] != "attn4":
            st[name + "_new"] = _normal(g, (st["T"], H_kv, D), sigma, dtype)
        if case["kind"] == "cycle4":
            st[name + "_out"] = torch.empty((st["rows"], H_kv, D), dtype=dtype, device="cuda")
    if case["kind"] != "cycle4":
        st["q"] = _normal(g, (st["T"], H_q, D), Q_SIGMA, dtype)
        st["out"] = torch.empty_like(st["q"])
    if case["kind"] == "rotate":  # where a sequence's first key stands
        st["base"] = torch.randint(0, 1000, (case["S"],), generator=g, device="cuda", dtype=torch.int32)
    if case["kind"] == "attn4":
        st["lse"] = torch.empty((st["T"], H_q), dtype=torch.float32, device="cuda")
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        from paper_2607_02963_amd import pdec
        st["pdec"] = pdec
        if case["kind"] in ("rope", "rotate"):
            st["spec"] = pdec.rope_spec(case["D"], rotary_dim=case["rot"], interleaved=case["inter"], theta=case["theta"],
                                        scaling=case["scaling"], factor=case["factor"], original_len=case["original"])
        if case["kind"] == "attn4":
            dims = pdec.paged_dims_of(st["q"], st["k_pages"], st["table"], causal=case["causal"],
                                      max_chunk=case["n_hi"], max_len=case["len_hi"])
            st["workspace"] = torch.empty(max(pdec.paged_workspace_size(dims), 16), dtype=torch.uint8, device="cuda")
    return st


def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    case, pdec = st["case"], st["pdec"]
    kind = case["kind"]
    if kind == "pages":
        pdec.paged_reserve(st["n"], st["lens_in"], st["table"], st["free"], st["free_n"], st["free_mid"],
                           page_size=case["page"], cu_tokens=st["cu"], positions=st["pos"], slots=st["slots"])
        pdec.paged_release(st["lens_in"], st["table"], st["free"], st["free_mid"], st["free_out"],
                           page_size=case["page"])
        return st["cu"], st["pos"], st["slots"], st["table"], st["free"], st["free_mid"], st["free_out"]
    if kind == "rope":
        return pdec.rope(st["q"], st["k"], st["pos"], st["spec"], backward=case["back"])
    if kind == "rotate":
        pdec.paged_rope_kv_append(st["q"], st["k_new"], st["v_new"], st["k_pages"], st["v_pages"], st["table"],
                                  st["cu"], st["lens_in"], st["lens_out"], st["spec"], pos_base=st["base"],
                                  q_out=st["out"])
        return st["out"], st["k_pages"], st["v_pages"], st["lens_out"]
    scales = {"k_scales": st["k_scales"], "v_scales": st["v_scales"]}
    if kind == "attn4":
        return pdec.paged_attn(st["q"], st["k_pages"], st["v_pages"], st["table"], st["cu"], st["seq_lens"],
                               causal=case["causal"], max_chunk=case["n_hi"], max_len=case["len_hi"], out=st["out"],
                               lse=st["lse"], workspace=st["workspace"], **scales)
    pdec.paged_kv_append(st["k_new"], st["v_new"], st["k_pages"], st["v_pages"], st["table"], st["cu"], st["lens_in"],
                         st["lens_out"], **scales)
    pdec.paged_kv_read(st["k_pages"], st["v_pages"], st["table"], st["lens_out"], st["cu_rows"], k_out=st["k_out"],
                       v_out=st["v_out"], **scales)
    return st["k_out"], st["v_out"]


def _owner(cu, count):
    """Sequence of each of count consecutive rows that cu divides, and the row's place in it."""
    n = (cu[1:] - cu[:-1]).long()
    seq = torch.repeat_interleave(torch.arange(len(n), device=cu.device), n, output_size=count)
    return seq, torch.arange(count, device=cu.device) - cu[seq]


def _plain_pages(st):
    case, table, free, page = st["case"], st["table"], st["free"], st["case"]["page"]
    n, lens = st["n"].long(), st["lens_in"].long()
    col = torch.arange(table.shape[1], device="cuda")
    lack = (col >= (lens // page)[:, None]) & (col < ((lens + n + page - 1) // page)[:, None]) & (table < 0)
    fits = (lack.sum(1).cumsum(0) <= st["free_n"]) & (n.cumsum(0) <= case["budget"])
    lack &= fits[:, None]
    rank = lack.flatten().cumsum(0).view(lack.shape) - 1
    table.copy_(torch.where(lack, free[(st["free_n"] - 1 - rank).clamp(min=0)], table))
    torch.sub(st["free_n"], lack.sum(), out=st["free_mid"])
    st["cu"].copy_(_starts(torch.where(fits, n, 0)))
    row = torch.arange(case["budget"], device="cuda")
    seq = torch.searchsorted(st["cu"][1:].long(), row, right=True)
    there = seq < case["S"]  # rows behind the last sequence's are left as they were
    seq = seq.clamp(max=case["S"] - 1)
    pos = lens[seq] + row - st["cu"][seq]
    st["pos"].copy_(torch.where(there, pos, st["pos"]))
    at = (pos // page).clamp(max=table.shape[1] - 1)
    st["slots"].copy_(torch.where(there, table[seq, at].long() * page + pos % page, st["slots"]))
    drop = (col >= ((lens + page - 1) // page)[:, None]) & (table >= 0)
    rank, count = drop.flatten().cumsum(0) - 1, drop.sum()
    to = torch.where(drop.flatten(), st["free_mid"] + count - 1 - rank, len(free))  # one place more than the list has
    free.copy_(torch.cat((free, free[:1])).scatter(0, to, table.flatten())[:-1])
    table.masked_fill_(drop, -1)
    torch.add(st["free_mid"], count, out=st["free_out"])
    return st["cu"], st["pos"], st["slots"], st["table"], st["free"], st["free_mid"], st["free_out"]


def _frequencies(case):
    """The angle of each pair at position 1."""
    R, theta, s = case["rot"], case["theta"], case["factor"]
    if case["scaling"] == "ntk":
        theta *= s ** (R / (R - 2))
    f = [theta ** (-2.0 * i / R) for i in range(R // 2)]
    if case["scaling"] == "linear":
        f = [x / s for x in f]
    if case["scaling"] == "by_parts":  # from 1 to 32 turns over the trained length: from all of the scaling to none
        keep = [min(max((case["original"] * x / (2 * math.pi) - 1.0) / 31.0, 0.0), 1.0) for x in f]
        f = [x * (u + (1 - u) / s) for x, u in zip(f, keep)]
    return torch.tensor(f, dtype=torch.float64, device="cuda")


def _turn(case, x, pos, back=False):
    """Heads x [T, H, D] turned by their positions, rounded once."""
    R = case["rot"]
    angle = pos.double()[:, None] * _frequencies(case)
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if back:
        s = -s
    y = x.float()
    a, b = (y[..., 0:R:2], y[..., 1:R:2]) if case["inter"] else (y[..., :R // 2], y[..., R // 2:R])
    u, v = a * c - b * s, b * c + a * s
    turned = torch.stack((u, v), -1).flatten(-2) if case["inter"] else torch.cat((u, v), -1)
    return torch.cat((turned, y[..., R:]), -1).to(x.dtype)


def _plain_rotate(st):
    case, page = st["case"], st["case"]["page"]
    seq, i = _owner(st["cu"], st["T"])
    t = st["lens_in"][seq] + i
    ids, pos = st["table"][seq, t // page].long(), st["base"][seq] + t
    st["out"].copy_(_turn(case, st["q"], pos))
    st["k_pages"][ids, t % page] = _turn(case, st["k_new"], pos)
    st["v_pages"][ids, t % page] = st["v_new"]
    torch.add(st["lens_in"], st["n"], out=st["lens_out"])
    return st["out"], st["k_pages"], st["v_pages"], st["lens_out"]


def _cached(st, name, seq, t):
    """Cache rows t of sequences seq (index tensors of one shape) as float32 [..., H_kv, D]."""
    page = st["case"]["page"]
    ids, row = st["table"][seq, t // page].long().clamp(min=0), t % page
    x = _values4(st[name + "_pages"][ids, :, row]).unflatten(-1, (-1, 32))
    return (x * _power(st[name + "_scales"][ids, :, row])[..., None]).flatten(-2)


def _plain_attn(st):
    case, q, cu, lens = st["case"], st["q"], st["cu"], st["seq_lens"].long()
    S, H_q, H_kv, D = case["S"], case["H_q"], case["H_kv"], case["D"]
    G, n, L = H_q // H_kv, case["n_hi"], case["len_hi"]
    key = torch.arange(L, device=q.device)
    at = torch.minimum(key[None], lens[:, None] - 1)  # rows past the end repeat the last one and are masked
    every = torch.arange(S, device=q.device)[:, None]
    k = _cached(st, "k", every, at).permute(0, 2, 3, 1).contiguous()  # [S, H_kv, D, L]
    v = _cached(st, "v", every, at).permute(0, 2, 1, 3).contiguous()  # [S, H_kv, L, D]
    i = torch.arange(n, device=q.device)
    x = q[(cu[:-1, None] + i).clamp(max=st["T"] - 1)].float()  # [S, n, H_q, D]
    x = x.view(S, n, H_kv, G, D).permute(0, 2, 1, 3, 4).reshape(S, H_kv, n * G, D)
    last = (lens - st["n"])[:, None] + i if case["causal"] else lens[:, None] - 1 + 0 * i
    last = torch.minimum(last, lens[:, None] - 1)
    hidden = (key > last[..., None])[:, None, :, None]  # [S, 1, n, 1, L]
    sc = ((x @ k) * (1.0 / math.sqrt(D))).view(S, H_kv, n, G, L).masked_fill_(hidden, float("-inf"))
    m = sc.amax(-1, keepdim=True)
    p = sc.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(S, H_kv, n * G, L) @ v).view(S, H_kv, n, G, D) / total
    seq, i = _owner(cu, st["T"])
    st["out"].copy_(o.permute(0, 2, 1, 3, 4)[seq, i].reshape(-1, H_q, D))
    st["lse"].copy_((m + total.log())[..., 0].permute(0, 2, 1, 3)[seq, i].reshape(-1, H_q))
    return st["out"], st["lse"]


def _plain_cycle(st):
    page = st["case"]["page"]
    seq, i = _owner(st["cu"], st["T"])
    t = st["lens_in"][seq] + i
    ids, row = st["table"][seq, t // page].long(), t % page
    for name in "kv":
        x, byte = _quantise4(st[name + "_new"])
        st[name + "_pages"][ids, :, row] = x
        st[name + "_scales"][ids, :, row] = byte
    torch.add(st["lens_in"], st["n"], out=st["lens_out"])
    seq, t = _owner(st["cu_rows"], st["rows"])
    st["k_out"].copy_(_cached(st, "k", seq, t))
    st["v_out"].copy_(_cached(st, "v", seq, t))
    return st["k_out"], st["v_out"]


def _run_plain(st):
    kind = st["case"]["kind"]
    if kind == "rope":
        return tuple(_turn(st["case"], st[name], st["pos"], st["case"]["back"]) for name in "qk")
    return {"pages": _plain_pages, "rotate": _plain_rotate, "cycle4": _plain_cycle, "attn4": _plain_attn}[kind](st)


# ---- the operators' definitions in 64 bits ----

def _power64(k):
    """2^k in float64, from its exponent field."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _binade(x):
    """floor(log2 |x|) of normal float64 values, from their exponent fields."""
    return ((x.view(torch.int64) >> 52) & 2047) - 1023


def _stored(x):
    """What a 4-bit row holds of x [..., D], in float64: rounding to a multiple of 2^-1 of the value's
    binade (2^-1 at the least) after the scale of its 32 elements is taken out."""
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    k = _binade(top) - 2  # top / 2^k lies in [4, 8)
    k = torch.where(top > 6.0 * _power64(k.clamp(min=-900)), k + 1, k)
    k = torch.where(top > 0, k.clamp(-126, 125), torch.zeros_like(k))
    y = x / _power64(k)
    step = _power64(_binade(y.abs().clamp(min=1.0)) - 1)
    return (torch.round(y / step) * step * _power64(k)).flatten(-2)


def _exact_rows(st, name):
    """Every cached row of the batch in float64, sequence after sequence, [rows, H_kv, D]."""
    case, page = st["case"], st["case"]["page"]
    table = st["table"].cpu()
    where = [(table[s, torch.arange(length) // page], torch.arange(length) % page)
             for s, length in enumerate(_sizes(case)[1])]
    ids, row = (torch.cat([w[i] for w in where]).long().cuda() for i in (0, 1))
    b = st[name + "_pages"].permute(0, 2, 1, 3)[ids, row].int()
    code = torch.empty((*b.shape[:-1], case["D"]), dtype=torch.int32, device="cuda")
    code[..., 0::2], code[..., 1::2] = b % 16, b // 16
    e, f = (code >> 1) & 3, (code & 1).double()
    x = torch.where(e == 0, f / 2, (1 + f / 2) * _power64(e - 1))
    x = torch.where(code > 7, -x, x)
    sc = st[name + "_scales"].permute(0, 2, 1, 3)[ids, row].int()
    return x * _power64(sc - 127).repeat_interleave(32, -1)


def _exact_turn(case, x, pos, sign):
    """Pairs as complex numbers times exp(i angle)."""
    import numpy as np
    R, base = case["rot"], np.float64(case["theta"])
    j = np.arange(R // 2)
    if case["scaling"] == "ntk":
        base = base * np.power(case["factor"], R / (R - 2.0))
    f = np.exp(-np.log(base) * (2.0 * j / R)) if R > 2 else np.ones(1)
    if case["scaling"] == "linear":
        f = f / case["factor"]
    if case["scaling"] == "by_parts":
        share = np.clip((f * case["original"] / (2 * np.pi) - 1) / (32 - 1), 0, 1)
        f = share * f + (1 - share) * f / case["factor"]
    angle = sign * pos.double()[:, None, None] * torch.from_numpy(f).cuda()
    y = x.double()
    first = torch.arange(R // 2, device="cuda") * (2 if case["inter"] else 1)
    second = first + (1 if case["inter"] else R // 2)
    z = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.ones_like(angle), angle)
    res = y.clone()
    res[..., first], res[..., second] = z.real, z.imag
    return res


def _exact_pages(case, st):
    n, lens = _sizes(case)
    page, table, free = case["page"], st["table"].tolist(), st["free"].tolist()
    left = st["free_n"].item()
    cu, pos, slots, top = [0], [], [], left
    for s, (a, t) in enumerate(zip(n, lens)):
        want = [c for c in range((t - a) // page, _pages(t, page)) if table[s][c] < 0]
        if len(pos) + a > case["budget"] or len(want) > top:
            break
        for c in want:
            top -= 1
            table[s][c] = free[top]
        pos += range(t - a, t)
        slots += [table[s][i // page] * page + i % page for i in range(t - a, t)]
        cu.append(len(pos))
    cu += [len(pos)] * (len(n) + 1 - len(cu))
    rest = [0] * (case["budget"] - len(pos))
    slots = torch.tensor(slots + rest, dtype=torch.int64, device="cuda")
    # what was given is taken back: the tables and the list are as they were
    return _i32(cu), _i32(pos + rest), slots, st["table"], st["free"], _i32([top]), _i32([left])


def exact(case, seed):
    st = _inputs(case, seed)
    kind = case["kind"]
    if kind == "pages":
        return _exact_pages(case, st)
    if kind == "rope":
        return tuple(_exact_turn(case, st[name], st["pos"], -1 if case["back"] else 1) for name in "qk")
    (n, lens), page = _sizes(case), case["page"]
    if kind == "rotate":
        table = st["table"].tolist()
        at = torch.tensor([table[s][t // page] * page + t % page for s in range(len(n))
                           for t in range(lens[s] - n[s], lens[s])], device="cuda")
        base = st["base"].tolist()
        pos = _i32([base[s] + t for s in range(len(n)) for t in range(lens[s] - n[s], lens[s])])
        res = [_exact_turn(case, st["q"], pos, 1)]
        for name in "kv":
            x = st[name + "_pages"].double()
            new = _exact_turn(case, st["k_new"], pos, 1) if name == "k" else st["v_new"].double()
            x.view(-1, *new.shape[1:])[at] = new
            res.append(x)
        return (*res, _i32(lens))
    k, v = _exact_rows(st, "k"), _exact_rows(st, "v")
    if kind == "cycle4":
        for x, name in ((k, "k"), (v, "v")):
            new, at, row = _stored(st[name + "_new"]), 0, 0
            for a, length in zip(n, lens):
                x[row + length - a:row + length] = new[at:at + a]
                at, row = at + a, row + length
        return k, v
    H_q, H_kv, D = case["H_q"], case["H_kv"], case["D"]
    G, q = H_q // H_kv, st["q"].double()
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device=q.device)
    at = row = 0
    for a, length in zip(n, lens):
        block = max(1, 8192 // G)
        for i in range(0, a, block):
            j = min(a, i + block)
            seen = length - a + j if case["causal"] else length
            key = torch.arange(seen, device=q.device)
            last = torch.arange(i, j, device=q.device) + (length - a) if case["causal"] else None
            for h in range(H_q):
                kk = k[row:row + seen, h // G].t().contiguous()
                z = (q[at + i:at + j, h] @ kk) * D ** -0.5
                if last is not None:
                    z = torch.where(key[None] <= last[:, None], z, torch.full_like(z, -math.inf))
                ls = torch.logsumexp(z, -1)
                out[at + i:at + j, h] = torch.exp(z - ls[:, None]) @ v[row:row + seen, h // G].contiguous()
                lse[at + i:at + j, h] = ls
        at, row = at + a, row + length
    return out, lse
