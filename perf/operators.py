"""Timed cases of the paged-cache operators: a cache held in pages, written as
tokens arrive (as it is, or in 8 bits), attended by chunks of new tokens, read
back to dense rows, and the join of two attention results.

Kinds of case
  attn    paged_attn: the new tokens of a ragged batch of sequences attend to
          their pages, themselves included (append first, then attend)
  append  paged_kv_append: the new tokens' keys and values go to their pages
  cycle   paged_kv_append into an 8-bit cache, then paged_kv_read of everything
          the cache holds: what later readers of these tokens will see
  read    paged_kv_read: pages to dense rows, for the entry points that take a
          dense prefix
  merge   merge_states: attention over a shared prefix and attention over a
          stream's own rows become attention over both

An 8-bit row is e4m3 with one power of two per token and kv head: x is stored
as e4m3(x / 2^k), k the least integer with max |x| / 2^k <= 448, and k + 127 in
a byte.

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


def listed():
    return [
        # The smallest call: one token of one short sequence, a float32 reference run.
        {"name": "attn_f32_token", "kind": "attn", "dtype": "f32", "cache": "f32", "H_q": 4, "H_kv": 1, "D": 64,
         "page": 16, "S": 1, "n_lo": 1, "n_hi": 1, "len_lo": 300, "len_hi": 300, "causal": True},
        # Serving: one new token of each of 32 captions over prefixes of their own lengths, 8-bit cache.
        {"name": "attn_tokens_8bit", "kind": "attn", "dtype": "bf16", "cache": "e4m3", "H_q": 28, "H_kv": 4, "D": 128,
         "page": 64, "S": 32, "n_lo": 1, "n_hi": 1, "len_lo": 1200, "len_hi": 16384, "causal": True},
        # One stream alone over a long video: few rows, one long axis.
        {"name": "attn_token_32k", "kind": "attn", "dtype": "bf16", "cache": "bf16", "H_q": 28, "H_kv": 4, "D": 128,
         "page": 64, "S": 1, "n_lo": 1, "n_hi": 1, "len_lo": 32768, "len_hi": 32768, "causal": True},
        # Drafted tokens of 13 streams, narrow heads, small pages that end anywhere.
        {"name": "attn_drafts", "kind": "attn", "dtype": "bf16", "cache": "bf16", "H_q": 32, "H_kv": 8, "D": 64,
         "page": 16, "S": 13, "n_lo": 2, "n_hi": 9, "len_lo": 777, "len_hi": 9001, "causal": True},
        # The event-parallel step's shared prefix: 32 streams' queries see all of one video's 8-bit pages.
        {"name": "attn_streams_8bit", "kind": "attn", "dtype": "bf16", "cache": "e4m3", "H_q": 28, "H_kv": 4,
         "D": 128, "page": 64, "S": 1, "n_lo": 32, "n_hi": 32, "len_lo": 32768, "len_hi": 32768, "causal": False},
        # Chunked prefill of a long video, its last chunk: the largest.
        {"name": "attn_chunk_32k", "kind": "attn", "dtype": "bf16", "cache": "bf16", "H_q": 28, "H_kv": 4, "D": 128,
         "page": 64, "S": 1, "n_lo": 2048, "n_hi": 2048, "len_lo": 32768, "len_hi": 32768, "causal": True},
        # A batch of odd chunks over an 8-bit cache, first chunks (nothing before them) to late ones.
        {"name": "attn_chunks_8bit", "kind": "attn", "dtype": "bf16", "cache": "e4m3", "H_q": 28, "H_kv": 4, "D": 128,
         "page": 32, "S": 6, "n_lo": 301, "n_hi": 1023, "len_lo": 1023, "len_hi": 12001, "causal": True},
        # The append of a serving step: one token of each of 32 sequences.
        {"name": "append_tokens", "kind": "append", "dtype": "bf16", "cache": "bf16", "H_q": 28, "H_kv": 4, "D": 128,
         "page": 64, "S": 32, "n_lo": 1, "n_hi": 1, "len_lo": 100, "len_hi": 2000},
        # A prefill chunk into an 8-bit cache, and the cache read back.
        {"name": "cycle_chunk", "kind": "cycle", "dtype": "bf16", "cache": "e4m3", "H_q": 28, "H_kv": 4, "D": 128,
         "page": 64, "S": 3, "n_lo": 999, "n_hi": 2048, "len_lo": 2048, "len_hi": 8191},
        # A long video's 8-bit prefix as the dense one that the event-parallel step takes.
        {"name": "read_32k", "kind": "read", "dtype": "bf16", "cache": "e4m3", "H_q": 28, "H_kv": 4, "D": 128,
         "page": 64, "S": 1, "n_lo": 0, "n_hi": 0, "len_lo": 32768, "len_hi": 32768},
        # The join after an event-parallel step: 32 streams of 28 heads.
        {"name": "merge_step", "kind": "merge", "dtype": "bf16", "D": 128, "H_q": 28, "rows": 32},
        # The join after whole branches, float32: 13 x 48 tokens.
        {"name": "merge_branches", "kind": "merge", "dtype": "f32", "D": 128, "H_q": 28, "rows": 624},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["attn", "attn", "attn", "attn", "attn", "append", "cycle", "read", "merge"])
        D = rng.choice([64, 128, 128])
        H_q, H_kv = rng.choice(HEADS)
        if kind == "merge":
            case = {"kind": "merge", "dtype": rng.choice(["bf16", "f32"]), "D": D, "H_q": H_q,
                    "rows": _log(rng, 1, 4000)}
        else:
            dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
            cache = rng.choice([dtype, "e4m3"])
            cache = {"append": dtype, "cycle": "e4m3"}.get(kind, cache)
            S = _log(rng, 1, 40)
            n_hi = 1 if rng.random() < 0.3 else _log(rng, 1, 2048)
            len_hi = max(_log(rng, 17, 33000), n_hi)
            case = {"kind": kind, "dtype": dtype, "cache": cache, "H_q": H_q, "H_kv": H_kv, "D": D,
                    "page": rng.choice([16, 32, 64, 128, 256]), "S": S, "n_lo": _log(rng, 1, n_hi), "n_hi": n_hi,
                    "len_lo": max(_log(rng, 1, len_hi), n_hi), "len_hi": len_hi}
            if kind == "attn":
                case["causal"] = rng.random() < 0.8
            if kind == "read":
                case["n_lo"] = case["n_hi"] = 0
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
    w = work(case)
    if w["bytes"] > 3e8 or w["flops"] > (0.9e12 if case["dtype"] == "bf16" else 0.1e12):
        return False
    if case["kind"] == "merge":
        return True
    padded = case["S"] * case["len_hi"]
    return padded <= 600000 and (case["kind"] != "attn" or padded * case["n_hi"] * case["H_q"] <= 2 ** 31)


def work(case):
    if case["kind"] == "merge":
        rows = case["rows"] * case["H_q"]
        esz = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": rows * (3 * case["D"] * esz + 12), "flops": 3 * rows * case["D"]}
    n, lens = _sizes(case)
    H_q, H_kv, D = case["H_q"], case["H_kv"], case["D"]
    esz = 2 if case["dtype"] == "bf16" else 4
    row = 2 * H_kv * (D + 1 if case["cache"] == "e4m3" else D * esz)  # one token's keys and values in the cache
    dense = 2 * H_kv * D * esz
    tables = 4 * sum(_pages(t, case["page"]) for t in lens) + 8 * case["S"]
    T, total = sum(n), sum(lens)
    if case["kind"] == "append":
        return {"bytes": T * (dense + row), "flops": T * 2 * H_kv * D}
    if case["kind"] == "cycle":
        return {"bytes": T * (dense + row) + total * (row + dense) + tables, "flops": (T + total) * 2 * H_kv * D}
    if case["kind"] == "read":
        return {"bytes": total * (row + dense) + tables, "flops": total * 2 * H_kv * D}
    seen = sum(a * t - a * (a - 1) // 2 if case["causal"] else a * t for a, t in zip(n, lens))
    return {"bytes": total * row + T * H_q * (2 * D * esz + 4) + tables, "flops": 4 * H_q * D * seen}


def _torch_dtype(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _power(byte):
    """2^(byte - 127) as float32: the byte is the number's exponent field."""
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _quantise(x):
    """Rows x [..., D] as (e4m3 values, exponent bytes [...]).  Dividing by a power of two is exact."""
    x = x.float()
    amax = x.abs().amax(-1)
    m, e = torch.frexp(amax)  # amax = m 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
    k = torch.where(m <= 0.875, e - 9, e - 8)
    k = torch.where(amax > 0, k.clamp(-126, 119), torch.zeros_like(k))
    byte = (k + 127).to(torch.uint8)
    return (x * _power(254 - byte)[..., None]).to(torch.float8_e4m3fn), byte


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _starts(counts):
    """[0, the sums of the first 1, 2, .. counts]"""
    return torch.nn.functional.pad(counts.cumsum(0), (1, 0)).to(torch.int32)


def _normal(g, shape, sigma, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * sigma).to(dtype)


def _pool(case, g, pages, sigma):
    """A pool of pages [pages, page, H_kv, D], and an 8-bit one's exponent bytes [pages, H_kv, page]."""
    x = _normal(g, (pages, case["page"], case["H_kv"], case["D"]), sigma, _torch_dtype(case["dtype"]))
    if case["cache"] != "e4m3":
        return x, None
    x, byte = _quantise(x)
    return x, byte.permute(0, 2, 1).contiguous()


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype, H_q, D = _torch_dtype(case["dtype"]), case["H_q"], case["D"]
    st = {"case": case}
    if case["kind"] == "merge":
        shape = (case["rows"], H_q)
        st["out_a"], st["out_b"] = (_normal(g, (*shape, D), V_SIGMA, dtype) for _ in "ab")
        st["lse_a"], st["lse_b"] = (torch.randn(shape, generator=g, device="cuda") * 2 + 6 for _ in "ab")
        return st
    n, lens = _sizes(case)
    H_kv, page = case["H_kv"], case["page"]
    st["T"], st["rows"] = sum(n), sum(lens)
    st["cu"], st["cu_rows"] = _starts(_i32(n)), _starts(_i32(lens))
    st["seq_lens"], st["lens_in"] = _i32(lens), _i32(lens) - _i32(n)
    st["lens_out"] = torch.zeros_like(st["seq_lens"])
    used = (st["seq_lens"] + page - 1) // page
    cols, total = _pages(max(lens), page), sum(_pages(t, page) for t in lens)
    col = torch.arange(cols, device="cuda")
    order = torch.randperm(total + 8, generator=g, device="cuda")
    at = (_starts(used)[:-1, None] + col).clamp(max=total)
    st["table"] = torch.where(col < used[:, None], order[at], -1).to(torch.int32)
    st["k_pages"], st["k_scales"] = _pool(case, g, total + 8, K_SIGMA)
    st["v_pages"], st["v_scales"] = _pool(case, g, total + 8, V_SIGMA)
    if case["kind"] in ("append", "cycle"):
        st["k_new"] = _normal(g, (st["T"], H_kv, D), K_SIGMA, dtype)
        st["v_new"] = _normal(g, (st["T"], H_kv, D), V_SIGMA, dtype)
    if case["kind"] in ("cycle", "read"):
        st["k_out"], st["v_out"] = (torch.empty((st["rows"], H_kv, D), dtype=dtype, device="cuda") for _ in "kv")
    if case["kind"] == "attn":
        st["q"] = _normal(g, (st["T"], H_q, D), Q_SIGMA, dtype)
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty((st["T"], H_q), dtype=torch.float32, device="cuda")
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        from paper_2607_02963_amd import pdec
        st["pdec"] = pdec
        if case["kind"] == "attn":
            dims = pdec.paged_dims_of(st["q"], st["k_pages"], st["table"], causal=case["causal"],
                                      max_chunk=case["n_hi"], max_len=case["len_hi"])
            st["workspace"] = torch.empty(max(pdec.paged_workspace_size(dims), 16), dtype=torch.uint8, device="cuda")
    return st


def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    case, pdec = st["case"], st["pdec"]
    kind = case["kind"]
    if kind == "merge":
        return pdec.merge_states(st["out_a"], st["lse_a"], st["out_b"], st["lse_b"])
    scales = {"k_scales": st["k_scales"], "v_scales": st["v_scales"]}
    if kind == "attn":
        return pdec.paged_attn(st["q"], st["k_pages"], st["v_pages"], st["table"], st["cu"], st["seq_lens"],
                               causal=case["causal"], max_chunk=case["n_hi"], max_len=case["len_hi"], out=st["out"],
                               lse=st["lse"], workspace=st["workspace"], **scales)
    if kind in ("append", "cycle"):
        pdec.paged_kv_append(st["k_new"], st["v_new"], st["k_pages"], st["v_pages"], st["table"], st["cu"],
                             st["lens_in"], st["lens_out"], **scales)
        if kind == "append":
            return st["k_pages"], st["v_pages"], st["lens_out"]
    lens = st["lens_out"] if kind == "cycle" else st["seq_lens"]
    pdec.paged_kv_read(st["k_pages"], st["v_pages"], st["table"], lens, st["cu_rows"], k_out=st["k_out"],
                       v_out=st["v_out"], **scales)
    return st["k_out"], st["v_out"]


def _owner(cu, count):
    """Sequence of each of count consecutive rows that cu divides, and the row's place in it."""
    n = (cu[1:] - cu[:-1]).long()
    seq = torch.repeat_interleave(torch.arange(len(n), device=cu.device), n, output_size=count)
    return seq, torch.arange(count, device=cu.device) - cu[seq]


def _cached(st, name, seq, t):
    """Cache rows t of sequences seq (index tensors of one shape) as float32 [..., H_kv, D]."""
    page = st["case"]["page"]
    ids, row = st["table"][seq, t // page].long().clamp(min=0), t % page
    pages, scales = st[name + "_pages"], st[name + "_scales"]
    if scales is None:
        return pages[ids, row].float()
    x = pages.view(torch.uint8)[ids, row].view(torch.float8_e4m3fn).float()
    return x * _power(scales[ids, :, row])[..., None]


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
    count = (cu[1:] - cu[:-1]).long()
    last = (lens - count)[:, None] + i if case["causal"] else lens[:, None] - 1 + 0 * i
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


def _plain_write(st, name, ids, row):
    new, pages, scales = st[name + "_new"], st[name + "_pages"], st[name + "_scales"]
    if scales is None:
        pages[ids, row] = new
    else:
        x, byte = _quantise(new)
        pages.view(torch.uint8)[ids, row] = x.view(torch.uint8)
        scales[ids, :, row] = byte


def _plain_append(st):
    page = st["case"]["page"]
    seq, i = _owner(st["cu"], st["T"])
    t = st["lens_in"][seq] + i
    ids = st["table"][seq, t // page].long()
    _plain_write(st, "k", ids, t % page)
    _plain_write(st, "v", ids, t % page)
    torch.add(st["lens_in"], st["cu"][1:] - st["cu"][:-1], out=st["lens_out"])


def _plain_read(st):
    seq, t = _owner(st["cu_rows"], st["rows"])
    st["k_out"].copy_(_cached(st, "k", seq, t))
    st["v_out"].copy_(_cached(st, "v", seq, t))
    return st["k_out"], st["v_out"]


def _plain_merge(st):
    la, lb = st["lse_a"], st["lse_b"]
    m = torch.maximum(la, lb)
    wa, wb = torch.exp(la - m), torch.exp(lb - m)
    total = wa + wb
    o = (wa[..., None] * st["out_a"].float() + wb[..., None] * st["out_b"].float()) / total[..., None]
    return o.to(st["out_a"].dtype), m + torch.log(total)


def _run_plain(st):
    kind = st["case"]["kind"]
    if kind == "merge":
        return _plain_merge(st)
    if kind == "attn":
        return _plain_attn(st)
    if kind in ("append", "cycle"):
        _plain_append(st)
        if kind == "append":
            return st["k_pages"], st["v_pages"], st["lens_out"]
    return _plain_read(st)


# ---- the operators' definitions in 64 bits ----

def _power64(k):
    """2^k in float64, from its exponent field."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _binade(x):
    """floor(log2 |x|) of normal float64 values, from their exponent fields."""
    return ((x.view(torch.int64) >> 52) & 2047) - 1023


def _stored(x):
    """What an 8-bit row holds of x [..., D], in float64: rounding to a multiple
    of 2^-3 of the value's binade (2^-9 at the least) after the scale is taken out."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    k = _binade(top) - 8  # top / 2^k lies in [256, 512)
    k = torch.where(top > 448.0 * _power64(k.clamp(min=-900)), k + 1, k)
    k = torch.where(top > 0, k.clamp(-126, 119), torch.zeros_like(k))
    y = x / _power64(k)
    step = _power64(_binade(y.abs().clamp(min=2.0 ** -6)) - 3)
    return torch.round(y / step) * step * _power64(k)


def _exact_rows(st, name):
    """Every cached row of the batch in float64, sequence after sequence."""
    case, page = st["case"], st["case"]["page"]
    table = st["table"].cpu()
    tokens = [torch.arange(length) for length in _sizes(case)[1]]
    where = [table[s, t // page] * page + t % page for s, t in enumerate(tokens)]
    at = torch.cat(where).long().cuda()
    H_kv, D = case["H_kv"], case["D"]
    if case["cache"] == "e4m3":
        b = st[name + "_pages"].view(torch.uint8).reshape(-1, H_kv, D)[at].int()
        e, f = (b >> 3) & 15, (b & 7).double()
        x = torch.where(e == 0, f * 2.0 ** -9, (1 + f / 8) * _power64(e - 7))
        x = torch.where(b > 127, -x, x)
        sc = st[name + "_scales"].permute(0, 2, 1).reshape(-1, H_kv)[at]
        return x * _power64(sc.int() - 127)[..., None]
    return st[name + "_pages"].reshape(-1, H_kv, D)[at].double()


def exact(case, seed):
    st = _inputs(case, seed)
    kind = case["kind"]
    if kind == "merge":
        a, b = st["lse_a"].double(), st["lse_b"].double()
        share = torch.sigmoid(a - b)[..., None]
        out = share * st["out_a"].double() + (1 - share) * st["out_b"].double()
        return out, torch.logaddexp(a, b)
    (n, lens), page = _sizes(case), case["page"]
    if kind == "append":
        table = st["table"].tolist()
        at = torch.tensor([table[s][t // page] * page + t % page for s in range(len(n))
                           for t in range(lens[s] - n[s], lens[s])], device="cuda")
        res = []
        for name in "kv":
            x, new = st[name + "_pages"], st[name + "_new"]
            x = x.double()
            x.view(-1, *new.shape[1:])[at] = new.double()
            res.append(x)
        return (*res, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    k, v = _exact_rows(st, "k"), _exact_rows(st, "v")
    if kind in ("cycle", "read"):
        if kind == "cycle":
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
