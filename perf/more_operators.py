"""Dense attention for serving, over packed prompts and over a paged cache, as measurable cases.

  store   si_store_pages, then si_load_pages: new rows of keys and values enter the pages of a cache, in 16 or 8 bits; they come back as
          the values that are held
  load    si_load_pages: rows of a paged cache for a reader of packed bf16
  decode  si_paged_attention: the newest positions of each request over that request's pages
  prompt  si_prompt_attention: whole prompts, or the next part of them, packed one behind the other

A cache is pages of `page` rows a head, keys and values apart; a request's table says which pages hold its rows.  In 8 bits a row of D values is
D codes (1 sign, 4 exponent and 3 mantissa bits, no infinities, largest 448) and one byte e for the power 2^(e - 127) that they are multiples of.

Sizes are those of the evaluation shapes (64 heads of 128; one compressed row per 4 positions, which all heads share), of groups of heads that
share a head of the cache, of the parity cases (33 heads, heads of 64, ragged lengths), and of a serving loop's calls.
"""
import math

import torch

own = False

DEV = "cuda:0"
NONE, CAUSAL = 0, 1
ALL = 2 ** 31 - 1  # a window of all rows
LARGEST = 448.0
LOWEST, HIGHEST = -64, 63  # exponents of a row's power of two


def _rows(name, op, B, shortest, L, before, H, D, bits, page):
    """B sequences whose new (or wanted) rows number `shortest` to L and start at row `before` of theirs."""
    return {"name": name, "op": op, "B": B, "shortest": shortest, "L": L, "before": before, "H_kv": H, "D": D, "bits": bits, "page": page}


def _decode(name, B, S, shortest, L, H, H_kv, D, bits, page, mask, n_win):
    """S positions of each of B requests, which hold `shortest` to L rows."""
    return {"name": name, "op": "decode", "B": B, "S": S, "shortest": shortest, "L": L, "H": H, "H_kv": H_kv, "D": D, "bits": bits, "page": page,
            "mask": mask, "n_win": n_win}


def _prompt(name, B, shortest, L, before, H, H_kv, D, m, n_win, shared, tail):
    """B sequences of `shortest` to L new positions behind `before` earlier ones, a row of keys and values per m positions; `tail` rows of
    the call belong to no sequence."""
    return {"name": name, "op": "prompt", "B": B, "shortest": shortest, "L": L, "before": before, "H": H, "H_kv": H_kv, "D": D, "m": m, "n_win": n_win,
            "shared": shared, "tail": tail}


def listed():
    return [
        # the newest row of each of 64 requests: the smallest call, latency
        _rows("store_token", "store", 64, 1, 1, 4095, 8, 128, 8, 64),
        # a batch of packed prompts
        _rows("store_prompts", "store", 16, 129, 4001, 0, 8, 128, 8, 64),
        # ragged sequences of five heads of 64 in small pages, read back for a reader of bf16
        _rows("load_ragged", "load", 9, 1, 2047, 37, 5, 64, 8, 16),
        # the cache of one long prompt
        _rows("load_prompt", "load", 1, 65536, 65536, 0, 8, 128, 16, 256),
        # one request with an ordinary context: latency
        _decode("decode_one", 1, 1, 2048, 2048, 64, 8, 128, 16, 64, NONE, ALL),
        # a batch of requests with contexts of different lengths
        _decode("decode_batch", 64, 1, 1025, 8191, 64, 8, 128, 16, 64, NONE, ALL),
        # few requests over long compressed contexts, whose rows all heads share
        _decode("decode_long", 8, 1, 65536, 131072, 64, 1, 128, 8, 256, NONE, ALL),
        # four drafted positions a request to be verified at once, small pages, odd lengths, five heads a group
        _decode("decode_draft", 24, 4, 77, 5003, 40, 8, 64, 8, 16, CAUSAL, ALL),
        # four short prompts: latency
        _prompt("prompt_short", 4, 33, 300, 0, 64, 8, 128, 1, ALL, False, 0),
        # the next parts of many prompts of different lengths, odd head count, rows behind the last sequence
        _prompt("prompt_ragged", 23, 1, 1500, 129, 33, 3, 64, 1, ALL, False, 57),
        # one long prompt
        _prompt("prompt_long", 1, 8192, 8192, 0, 64, 8, 128, 1, ALL, False, 0),
        # a layer that attends to all compressed rows: all heads share them, keys are the values
        _prompt("prompt_compressed", 1, 16384, 16384, 0, 64, 1, 128, 4, ALL, True, 0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["store", "load", "decode", "decode", "prompt", "prompt"])
    D, page, bits = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 64, 256]), rng.choice([8, 16])
    if op in ("store", "load"):
        H = rng.choice([1, 8, 8, rng.randint(1, 16)])
        L = _log_int(rng, 1, 65536 * 8 // (H * (2 if op == "store" else 1)))
        B = max(1, min(_log_int(rng, 1, 64), 32768 * 8 // H // L))
        return _unnamed(_rows("", op, B, rng.randint(1, L), L, rng.choice([0, 0, rng.randint(1, 5000)]), H, D, bits, page))
    H, H_kv = rng.choice([(64, 8), (64, 1), (32, 8), (8, 8), (33, 3), (33, 1), (5, 5), (40, 8)])
    if op == "decode":
        S = rng.choice([1, 1, 1, 2, 4, 7])
        L = _log_int(rng, 100, 131072)
        B = max(1, min(_log_int(rng, 1, 128), 64 * 8192 * 8 // (H_kv * L)))
        return _unnamed(_decode("", B, S, rng.randint(max(S, L // 4), L), L, H, H_kv, D, bits, page, CAUSAL if S > 1 else NONE,
                                rng.choice([ALL, ALL, ALL, 128, 1024])))
    m = rng.choice([1, 1, 1, 2, 4])
    L = _log_int(rng, 16, 6000)
    B = max(1, min(_log_int(rng, 1, 32), 8000 // L))
    before = rng.choice([0, 0, rng.randint(1, 1500)])
    return _unnamed(_prompt("", B, rng.randint(1, L), L, before, H, H_kv, D, m, rng.choice([ALL, ALL, ALL, 128, 1024]), rng.random() < 0.2,
                            rng.choice([0, 0, rng.randint(1, 100)])))


def _unnamed(case):
    return {key: v for key, v in case.items() if key != "name"}


# ---------------------------------------------------------------------------------- inputs
def _spread(case):
    """The sequences' lengths, evenly from the shortest to the longest."""
    B, lo, hi = case["B"], case["shortest"], case["L"]
    return [hi - (hi - lo) * i // max(1, B - 1) for i in range(B)]


def _lengths(gen, case):
    """The same in an order of the seed's."""
    lengths = _spread(case)
    return [lengths[i] for i in torch.randperm(len(lengths), generator=gen, device=DEV).tolist()]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _offsets(lengths):
    return _ints([0] + lengths).cumsum(0, dtype=torch.int32)


def _pages(st, gen, case, rows, filled):
    """Tables of pages in no particular order for sequences that hold `rows` rows, -1 behind, and the pages' arrays.  filled: they hold rows
    of this distribution, otherwise whatever was there."""
    B, H, D, page = case["B"], case["H_kv"], case["D"], case["page"]
    wide = max(1, -(-max(rows) // page))
    used = [-(-r // page) for r in rows]
    n_pages = sum(used) + 3
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    at = torch.arange(wide, device=DEV)[None, :]
    first = (_offsets(used)[:-1, None].long() + at).clamp(max=n_pages - 1)
    st["table"] = torch.where(at < _ints(used)[:, None], order[first], -1).to(torch.int32).contiguous()
    for name in ("K", "V"):
        if case["bits"] == 16:
            x = torch.empty((n_pages, H, page, D), dtype=torch.bfloat16, device=DEV)
            if filled:
                for p in x.split(4096):
                    p.copy_(_keys(gen, p.shape) if name == "K" else _values(gen, p.shape))
            else:
                x.zero_()
            st[name], st[name + "_scales"] = x, None
        else:
            x = torch.empty((n_pages, H, page, D), dtype=torch.uint8, device=DEV)
            e = torch.empty((n_pages, H, page), dtype=torch.uint8, device=DEV)
            if filled:
                for p, q in zip(x.split(4096), e.split(4096)):
                    codes, exponents = _nearest((_keys(gen, p.shape) if name == "K" else _values(gen, p.shape)).to(torch.bfloat16).float())
                    p.copy_(codes)
                    q.copy_(exponents)
            else:
                x.zero_()
                e.fill_(127)
            st[name], st[name + "_scales"] = x, e


def _keys(gen, shape):
    """Rows of different sizes, as keys have them."""
    return torch.randn(shape, generator=gen, device=DEV) * torch.exp(0.3 * torch.randn(shape[:-1] + (1,), generator=gen, device=DEV))


def _values(gen, shape):
    """Components with a mean of their own."""
    return torch.randn(shape, generator=gen, device=DEV) + 0.5 * torch.randn(shape[-1:], generator=gen, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op, B, H_kv, D = case["op"], case["B"], case["H_kv"], case["D"]
    lengths = _lengths(gen, case)
    st = {"case": case, "longest": max(lengths)}
    if op in ("store", "load"):
        N = sum(lengths)
        st["offsets"], st["start"] = _offsets(lengths), _ints([case["before"]] * B)
        _pages(st, gen, case, [case["before"] + n for n in lengths], op == "load")
        if op == "store":
            st["k"], st["v"] = (f(gen, (N, H_kv, D)).to(torch.bfloat16) for f in (_keys, _values))
        st["k_out"], st["v_out"] = (torch.empty((N, H_kv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        return st
    H = case["H"]
    if op == "decode":
        S = case["S"]
        st["lengths"] = _ints(lengths)
        st["first"] = st["lengths"] - S if case["mask"] == CAUSAL else None
        _pages(st, gen, case, lengths, True)
        st["q"] = torch.randn((B, S, H, D), generator=gen, device=DEV).to(torch.bfloat16)
        st["out"] = torch.zeros((B, S, H, D), dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.zeros((B, S, H), dtype=torch.float32, device=DEV)
        # more than si_paged_workspace_bytes of any of these calls
        st["ws"] = torch.empty(4 * (D + 4) * (131072 + 2 * B * S * H), dtype=torch.uint8, device=DEV)
        return st
    rows = [(case["before"] + n) // case["m"] for n in lengths]
    N = sum(lengths) + case["tail"]
    st["longest_rows"] = max(1, max(rows))
    st["q_offsets"], st["k_offsets"], st["first"] = _offsets(lengths), _offsets(rows), _ints([case["before"]] * B)
    st["q"] = torch.randn((N, H, D), generator=gen, device=DEV).to(torch.bfloat16)
    st["k"] = _keys(gen, (max(1, sum(rows)), H_kv, D)).to(torch.bfloat16)
    st["v"] = None if case["shared"] else _values(gen, st["k"].shape).to(torch.bfloat16)
    st["out"] = torch.zeros((N, H, D), dtype=torch.bfloat16, device=DEV)
    st["lse"] = torch.zeros((N, H), dtype=torch.float32, device=DEV)
    return st


# ---------------------------------------------------------------------------------- the pass
def run(state):
    op = state["case"]["op"]
    return (_own if own else _plain)[op](state)


def _power(e):
    """2^e in float32 for whole numbers e, by its bits: exact."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _nearest(x):
    """Codes [.., D] and scale bytes [..] of rows x [.., D] (float32)."""
    fraction, exponent = torch.frexp(x.abs().amax(dim=-1))
    # amax = 2 fraction 2^(exponent - 1): the least e with amax <= 1.75 * 2^(8 + e)
    e = exponent - 9 + (fraction > 0.875).to(exponent.dtype)
    e = torch.where(fraction == 0, torch.full_like(e, LOWEST), e).clamp(LOWEST, HIGHEST)
    y = (x * _power(-e)[..., None]).clamp(-LARGEST, LARGEST)
    return y.to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _held(pages, scales):
    """float32 values of pages [.., rows, D]."""
    if scales is None:
        return pages.float()
    return pages.view(torch.float8_e4m3fn).float() * _power(scales.int() - 127)[..., None]


def _places(offsets, longest, n):
    """Packed rows of every sequence [B, longest], and which of them there are."""
    at = offsets[:-1, None].long() + torch.arange(longest, device=DEV)
    return at.clamp(max=n - 1), at < offsets[1:, None]


def _page_rows(st, which, at, ok):
    """Rows `at` [B, n] of every sequence -> [B, n, H, D] float32, zeros where not ok."""
    page = st["case"]["page"]
    table = st["table"].long()
    p = torch.gather(table, 1, (at // page).clamp(max=table.shape[1] - 1))
    ok = ok & (p >= 0)
    p = p.clamp(min=0)
    scales = st[which + "_scales"]
    rows = _held(st[which][p, :, at % page], None if scales is None else scales[p, :, at % page])
    return torch.where(ok[..., None, None], rows, 0.0)


def _store(st):
    # a row that is stored and read back is what its codes stand for
    if st["case"]["bits"] == 16:
        return {"k": st["k"].clone(), "v": st["v"].clone()}
    return {name: _held(*_nearest(st[name].float())).to(torch.bfloat16) for name in ("k", "v")}


def _load(st):
    case = st["case"]
    places, there = _places(st["offsets"], st["longest"], st["k_out"].shape[0])
    at = st["start"].long()[:, None] + torch.arange(st["longest"], device=DEV)[None, :]
    at = at.expand(case["B"], -1)
    return {"k": _page_rows(st, "K", at, there)[there].to(torch.bfloat16), "v": _page_rows(st, "V", at, there)[there].to(torch.bfloat16)}


def _attend(q, K, V, ok, scale):
    """q [B, S, H, D], K and V [B, T, H_kv, D], ok [B, S, T] -> out [B, S, H, D], lse [B, S, H]."""
    B, S, H, D = q.shape
    H_kv = K.shape[2]
    G = H // H_kv
    x = torch.matmul(q.view(B, S, H_kv, G, D).permute(0, 2, 1, 3, 4).reshape(B, H_kv, S * G, D), K.permute(0, 2, 3, 1).contiguous())
    x = x.mul_(scale).view(B, H_kv, S, G, -1)
    x.masked_fill_(~ok[:, None, :, None, :], -math.inf)
    top = x.amax(dim=4, keepdim=True)
    p = x.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(dim=4, keepdim=True)
    out = torch.matmul(p.view(B, H_kv, S * G, -1), V.permute(0, 2, 1, 3).contiguous()).view(B, H_kv, S, G, D)
    out = out / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + torch.log(total)).squeeze(4)
    return out.permute(0, 2, 1, 3, 4).reshape(B, S, H, D), lse.permute(0, 2, 1, 3).reshape(B, S, H)


def _seen(legal, n_win, T):
    """Rows of T that positions with `legal` [B, S] legal rows see."""
    s = torch.arange(T, device=DEV)
    return (s < legal[..., None]) & (s >= (legal - n_win)[..., None])


def _decoded(st):
    case = st["case"]
    B, S = case["B"], case["S"]
    T = st["longest"]
    held = st["lengths"].long()[:, None]
    legal = held.expand(B, S)
    if case["mask"] == CAUSAL:
        legal = torch.minimum(legal, st["first"].long()[:, None] + torch.arange(S, device=DEV) + 1)
    at = torch.arange(T, device=DEV)[None, :].expand(B, T)
    K, V = (_page_rows(st, which, at, at < held) for which in ("K", "V"))
    out, lse = _attend(st["q"].float(), K, V, _seen(legal, case["n_win"], T), 1.0 / math.sqrt(case["D"]))
    return {"out": out.to(torch.bfloat16), "lse": lse}


def _prompted(st):
    case = st["case"]
    q_at, q_there = _places(st["q_offsets"], st["longest"], st["q"].shape[0])
    k_at, k_there = _places(st["k_offsets"], st["longest_rows"], st["k"].shape[0])
    rows = (st["k_offsets"][1:] - st["k_offsets"][:-1]).long()[:, None]
    position = st["first"].long()[:, None] + torch.arange(st["longest"], device=DEV)
    legal = torch.minimum(rows, (position + 1) // case["m"])
    K = torch.where(k_there[..., None, None], st["k"][k_at].float(), 0.0)
    V = K if st["v"] is None else torch.where(k_there[..., None, None], st["v"][k_at].float(), 0.0)
    o, e = _attend(st["q"][q_at].float(), K, V, _seen(legal, case["n_win"], st["longest_rows"]), 1.0 / math.sqrt(case["D"]))
    out, lse = st["out"].clone(), st["lse"].clone()
    out[q_at[q_there]] = o[q_there].to(torch.bfloat16)
    lse[q_at[q_there]] = e[q_there]
    return {"out": out, "lse": lse}


_plain = {"store": _store, "load": _load, "decode": _decoded, "prompt": _prompted}


def _own_store(st):
    import paper_2605_02568_amd as P
    P.si_store_pages(st["k"], st["v"], st["offsets"], st["start"], st["table"], st["K"], st["V"], st["K_scales"], st["V_scales"])
    return _own_load(st)


def _own_load(st):
    import paper_2605_02568_amd as P
    P.si_load_pages(st["table"], st["K"], st["V"], st["K_scales"], st["V_scales"], st["offsets"], st["start"], st["k_out"], st["v_out"])
    return {"k": st["k_out"], "v": st["v_out"]}


def _own_decode(st):
    import paper_2605_02568_amd as P
    case = st["case"]
    P.si_paged_attention(st["q"], st["table"], st["K"], st["V"], st["K_scales"], st["V_scales"], st["lengths"], st["first"], 1, case["mask"],
                         case["n_win"], 1.0 / math.sqrt(case["D"]), st["out"], st["lse"], st["ws"])
    return {"out": st["out"], "lse": st["lse"]}


def _own_prompt(st):
    import paper_2605_02568_amd as P
    case = st["case"]
    P.si_prompt_attention(st["q"], st["k"], st["v"], st["q_offsets"], st["k_offsets"], st["first"], case["m"], CAUSAL, case["n_win"],
                          1.0 / math.sqrt(case["D"]), st["out"], st["lse"])
    return {"out": st["out"], "lse": st["lse"]}


_own = {"store": _own_store, "load": _own_load, "decode": _own_decode, "prompt": _own_prompt}


# ---------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    op, B, D, H_kv = case["op"], case["B"], case["D"], case["H_kv"]
    lengths = torch.tensor(_spread(case), dtype=torch.float64)
    if op in ("store", "load"):
        values = 2 * float(lengths.sum()) * H_kv
        held = values * (2 * D if case["bits"] == 16 else D + 1)
        if op == "load":
            return {"bytes": held + values * 2 * D, "flops": values * D}
        return {"bytes": 2 * (held + values * 2 * D), "flops": 4 * values * D}
    H, n_win = case["H"], case["n_win"]
    if op == "decode":
        S = case["S"]
        seen = lengths[:, None].expand(B, S)
        if case["mask"] == CAUSAL:
            seen = seen - S + 1 + torch.arange(S, dtype=torch.float64)
        seen = seen.clamp(max=n_win)
        read = float((lengths if n_win == ALL else lengths.clamp(max=n_win + S - 1)).sum())
        row = 2 * D if case["bits"] == 16 else D + 1
        return {"bytes": read * 2 * H_kv * row + B * S * H * (4 * D + 4), "flops": 4 * float(seen.sum()) * H * D}
    m, before = case["m"], case["before"]
    pairs, read = 0.0, 0.0
    for n in _spread(case):
        legal = torch.floor((before + torch.arange(n, dtype=torch.float64) + 1) / m)
        pairs += float(legal.clamp(max=n_win).sum())
        read += float(legal[-1] - (legal[0] - n_win).clamp(min=0))
    return {"bytes": read * H_kv * D * 2 * (1 if case["shared"] else 2) + float(lengths.sum()) * H * (4 * D + 4), "flops": 4 * pairs * H * D}


# ---------------------------------------------------------------------------------- in 64 bits
def _power64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _codes64(codes, scales):
    """By the fields of a code: sign, exponent, mantissa."""
    c = codes.long()
    field, mantissa = (c >> 3) & 15, (c & 7).double()
    size = torch.where(field == 0, mantissa * 2.0 ** -9, (1.0 + mantissa / 8.0) * _power64(field - 7))
    return torch.where(c >= 128, -size, size) * _power64(scales.long() - 127)[..., None]


def _rounded64(x):
    """Rows x [.., D] as 8 bits hold them."""
    top = x.abs().amax(dim=-1, keepdim=True)
    fits = LARGEST * _power64(torch.arange(LOWEST, HIGHEST, device=DEV))  # the largest value of each power but the last
    power = _power64(LOWEST + (top > fits).sum(dim=-1, keepdim=True))
    y = x / power
    size = y.abs().clamp(min=2.0 ** -6)
    step = _power64(torch.frexp(size)[1] - 4)  # 8 steps from a power of two to the next
    return (torch.round(y / step) * step).clamp(-LARGEST, LARGEST) * power


def _rows64(st, which, b, first, n):
    """Rows first .. first + n - 1 of sequence b, [n, H, D], page by page."""
    page = st["case"]["page"]
    parts = []
    for p in range(first // page, -(-(first + n) // page)):
        number = int(st["table"][b, p])
        lo, hi = max(0, first - p * page), min(page, first + n - p * page)
        if st[which + "_scales"] is None:
            rows = st[which][number, :, lo:hi].double()
        else:
            rows = _codes64(st[which][number, :, lo:hi], st[which + "_scales"][number, :, lo:hi])
        parts.append(rows.transpose(0, 1))
    return torch.cat(parts)


def _attend64(q, K, V, legal, n_win, scale):
    """q [n, H, D], K and V [T, H_kv, D], legal [n]."""
    n, H, D = q.shape
    T, H_kv = K.shape[0], K.shape[1]
    out = torch.zeros((n, H, D), dtype=torch.float64, device=DEV)
    lse = torch.full((n, H), -math.inf, dtype=torch.float64, device=DEV)
    if T == 0:
        return out, lse
    step = max(1, (1 << 27) // T)
    s = torch.arange(T, device=DEV)[None, :]
    for h in range(H):
        k, v = K[:, h * H_kv // H].t().contiguous(), V[:, h * H_kv // H].contiguous()
        for i in range(0, n, step):
            few = legal[i:i + step, None]
            x = (q[i:i + step, h].double() @ k) * scale
            x = x.masked_fill((s >= few) | (s < few - n_win), -math.inf)
            e = torch.logsumexp(x, dim=1)
            lse[i:i + step, h] = e
            p = torch.exp(x - torch.where(e == -math.inf, torch.zeros_like(e), e)[:, None])
            out[i:i + step, h] = p @ v
    return out, lse


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "store":
        return {name: st[name].double() if case["bits"] == 16 else _rounded64(st[name].double()) for name in ("k", "v")}
    scale = 1.0 / math.sqrt(case["D"])
    if op == "load":
        at = st["offsets"].tolist()
        return {name: torch.cat([_rows64(st, which, b, case["before"], at[b + 1] - at[b]) for b in range(case["B"])])
                for name, which in (("k", "K"), ("v", "V"))}
    out, lse = st["out"].double(), st["lse"].double()
    if op == "decode":
        for b, n in enumerate(st["lengths"].tolist()):
            legal = torch.full((case["S"],), n, device=DEV)
            if case["mask"] == CAUSAL:
                legal = legal - case["S"] + 1 + torch.arange(case["S"], device=DEV)
            out[b], lse[b] = _attend64(st["q"][b], _rows64(st, "K", b, 0, n), _rows64(st, "V", b, 0, n), legal, case["n_win"], scale)
        return {"out": out, "lse": lse}
    qs, ks = st["q_offsets"].tolist(), st["k_offsets"].tolist()
    for b in range(case["B"]):
        mine = slice(qs[b], qs[b + 1])
        K = st["k"][ks[b]:ks[b + 1]].double()
        V = K if st["v"] is None else st["v"][ks[b]:ks[b + 1]].double()
        legal = (torch.arange(qs[b + 1] - qs[b], device=DEV) + case["before"] + 1) // case["m"]
        out[mine], lse[mine] = _attend64(st["q"][mine], K, V, legal, case["n_win"], scale)
    return {"out": out, "lse": lse}
