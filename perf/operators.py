"""A compressed cache held in 4 bits and bounded in length, as measurable cases.

  store      si_quantize_rows, then si_dequantize_rows: new rows enter the cache; the rows come back as the values the codes stand for
  load       si_dequantize_rows: rows of a 4-bit cache for a reader of bf16
  attention  si_quantized_attention: attention over TopK(t) U Window(t) where the cache is held in 4 bits
  weights    si_accumulate_weights: what every cache row received of the softmax, summed over queries and heads
  evict      si_evict_rows: the rows with the largest weights stay, the arrays that belong to them move together

A row of D values is held as D codes of 4 bits (sign, 2 exponent bits, 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) and one
power of two per 32 values.  Value i of a row is in byte i / 2, in the low half where i is even; a scale byte e stands
for 2^(e - 127).

Sizes are those of the evaluation shapes (64 heads of 128, one compressed row per 4 positions, lists of 512 or 1024, a window
of 128, causal block mask), of the parity cases (few heads, heads of 64, batches, ragged sizes), and of a serving loop's
calls: one new position of each request against that request's rows, of which each has a number of its own.
"""
import math

import torch

own = False

DEV = "cuda:0"
NONE, CAUSAL = 0, 1
BLOCK = 32
VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]  # of the codes 0 .. 7; 8 .. 15 are their negatives
LOWEST, HIGHEST = -13, 13  # exponents of a block's power of two


def _rows(name, op, B, N, D, T):
    return {"name": name, "op": op, "B": B, "N": N, "D": D, "T": T}


def _attention(name, op, B, S, H, D, T, m, k, n_win, mask, ragged):
    return {"name": name, "op": op, "B": B, "S": S, "H": H, "D": D, "T": T, "m": m, "k": k, "n_win": n_win, "mask": mask,
            "ragged": ragged}


def _evict(name, B, T, n_keep, n_sink, n_recent, ragged):
    return {"name": name, "op": "evict", "B": B, "T": T, "n_keep": n_keep, "n_sink": n_sink, "n_recent": n_recent, "ragged": ragged}


def listed():
    return [
        # one new row of each of 32 requests: the smallest call, latency
        _rows("store_token", "store", 32, 1, 128, 4096),
        # the rows of a 1M-position prompt
        _rows("store_prompt", "store", 1, 262144, 128, 262144),
        # a batch of ragged prompts of heads of 64, read back
        _rows("load_batch", "load", 8, 2047, 64, 4099),
        # the rows of a 256k-position prompt read back
        _rows("load_prompt", "load", 1, 65536, 128, 65536),
        # one new position of each of 32 requests against long caches of different lengths
        _attention("attention_decode", "attention", 32, 1, 64, 128, 65536, 4, 1024, 128, NONE, True),
        # a batch of ragged prompts with few heads of 64 and rows that see nothing yet
        _attention("attention_ragged", "attention", 3, 1021, 33, 64, 511, 2, 100, 33, CAUSAL, False),
        # prefill of an ordinary prompt
        _attention("attention_prefill", "attention", 1, 16384, 64, 128, 4096, 4, 512, 128, CAUSAL, False),
        # one new position of each of 32 requests, caches bounded to 8k rows
        _attention("weights_decode", "weights", 32, 1, 64, 128, 8192, 4, 1024, 128, NONE, True),
        # what a prompt's own queries say of its rows
        _attention("weights_prefill", "weights", 1, 8192, 64, 128, 2048, 4, 512, 128, CAUSAL, False),
        # one request's short cache: latency
        _evict("evict_one", 1, 2048, 1536, 4, 128, False),
        # a batch of requests, each with its own number of rows
        _evict("evict_batch", 32, 16411, 12289, 4, 128, True),
        # one request's cache of 1M positions
        _evict("evict_long", 1, 262144, 196608, 4, 128, False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["store", "load", "attention", "attention_decode", "weights", "weights_decode", "evict"])
    if op in ("store", "load"):
        D = rng.choice([32, 64, 128, 128])
        N = _log_int(rng, 1, 262144 if op == "store" else 65536)
        B = max(1, min(_log_int(rng, 1, 64), (262144 if op == "store" else 65536) // N))
        return _drop(_rows("", op, B, N, D, N + rng.randint(0, N)))
    if op == "evict":
        T = _log_int(rng, 100, 262144)
        B = max(1, min(_log_int(rng, 1, 64), 262144 // T))
        n_keep = max(1, int(T * rng.uniform(0.3, 0.95)))
        n_sink = rng.choice([0, 1, 4])
        return _drop(_evict("", B, T, max(n_keep, n_sink + 1), n_sink, rng.randint(0, min(200, n_keep // 2)), rng.random() < 0.5))
    D = rng.choice([64, 128, 128])
    H = rng.choice([64, 64, 32, rng.randint(1, 64)])
    if op.endswith("_decode"):
        B, S, T = _log_int(rng, 1, 128), rng.choice([1, 1, 1, 2, 4]), _log_int(rng, 200, 65536)
        B = max(1, min(B, 2000000 // T))
        return _drop(_attention("", op.split("_")[0], B, S, H, D, T, 4, _log_int(rng, 16, 2048), rng.choice([0, 128, 128, 300]), NONE,
                                rng.random() < 0.5))
    S, m = _log_int(rng, 100, 12000 if op == "attention" else 6000), rng.choice([1, 2, 4, 4])
    B = rng.randint(1, 3) if S < 3000 else 1
    k = _log_int(rng, 16, 512 if S > 4000 else 1024)
    return _drop(_attention("", op, B, S, H, D, max(1, S // m), m, k, rng.choice([0, 64, 128]), CAUSAL, rng.random() < 0.3))


def _drop(case):
    return {key: v for key, v in case.items() if key != "name"}


# ---------------------------------------------------------------------------------- inputs
def _lengths(gen, case):
    """Rows that each request holds, or None: all T."""
    if not case["ragged"]:
        return None
    T = case["T"]
    return torch.randint(max(1, T // 2), T + 1, (case["B"],), generator=gen, device=DEV, dtype=torch.int32)


def _legal(case, lengths):
    """Legal rows of every query [B, S]."""
    B, S, T = case["B"], case["S"], case["T"]
    held = torch.full((B,), T, dtype=torch.int64, device=DEV) if lengths is None else lengths.long()
    legal = held[:, None].expand(B, S)
    if case["mask"] == CAUSAL:
        legal = torch.minimum(legal, ((torch.arange(S, device=DEV) + 1) // case["m"])[None, :])
    return legal


def _lists(gen, case, legal):
    """Index lists as the indexer writes them: distinct legal rows in no particular index order, pads last."""
    B, S, T, k = case["B"], case["S"], case["T"], case["k"]
    out = torch.full((B, S, k), -1, dtype=torch.int32, device=DEV)
    kk = min(k, T)
    step = max(1, (1 << 26) // T)
    for b in range(B):
        for s in range(0, S, step):
            e = min(S, s + step)
            r = torch.rand((e - s, T), generator=gen, device=DEV)
            r.masked_fill_(torch.arange(T, device=DEV)[None, :] >= legal[b, s:e, None], -1.0)
            v, i = torch.topk(r, kk, dim=1)
            out[b, s:e, :kk] = torch.where(v >= 0, i, -1).to(torch.int32)
    return out


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op, B, T = case["op"], case["B"], case["T"]
    st = {"case": case, "table": torch.tensor(VALUES + [-v for v in VALUES], device=DEV)}
    if op in ("store", "load"):
        N, D = case["N"], case["D"]
        st["start"] = torch.randint(0, T - N + 1, (B,), generator=gen, device=DEV, dtype=torch.int32)
        st["codes"] = torch.randint(0, 256, (B, T, D // 2), generator=gen, device=DEV, dtype=torch.uint8)
        st["scales"] = torch.randint(127 - 6, 127 + 3, (B, T, D // BLOCK), generator=gen, device=DEV, dtype=torch.uint8)
        if op == "store":  # rows of different sizes, a few values of a row far larger than the others
            rows = torch.randn((B, N, D), generator=gen, device=DEV)
            rows *= torch.exp(0.5 * torch.randn((B, N, 1), generator=gen, device=DEV))
            rows *= torch.where(torch.rand((D,), generator=gen, device=DEV) < 0.03, 8.0, 1.0)
            st["rows"] = rows.to(torch.bfloat16)
        st["out"] = torch.empty((B, N, D), dtype=torch.bfloat16, device=DEV)
        return st
    if op == "evict":
        st["lengths"] = _lengths(gen, case)
        # a few rows receive most of the softmax, many nothing at all
        w = torch.exp(3.0 * torch.randn((B, T), generator=gen, device=DEV))
        st["weights"] = torch.where(torch.rand((B, T), generator=gen, device=DEV) < 0.3, torch.zeros_like(w), w)
        st["keys"] = torch.randn((B, T, 128), generator=gen, device=DEV).to(torch.bfloat16)
        n = case["n_keep"]
        st["weights_out"] = torch.zeros((B, n), dtype=torch.float32, device=DEV)
        st["keys_out"] = torch.zeros((B, n, 128), dtype=torch.bfloat16, device=DEV)
        st["kept"] = torch.empty((B, n), dtype=torch.int32, device=DEV)
        st["held"] = torch.empty((B,), dtype=torch.int32, device=DEV)
        st["ws"] = torch.empty(B * (T + 65536), dtype=torch.uint8, device=DEV)
        return st
    S, H, D = case["S"], case["H"], case["D"]
    st["lengths"] = _lengths(gen, case)
    legal = _legal(case, st["lengths"])
    st["idx"] = _lists(gen, case, legal)
    st["q"] = torch.randn((B, S, H, D), generator=gen, device=DEV).to(torch.bfloat16)
    codes = torch.empty((B, T, D // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((B, T, D // BLOCK), dtype=torch.uint8, device=DEV)
    for b in range(B):
        c, e = _nearest(torch.randn((T, D), generator=gen, device=DEV).to(torch.bfloat16).float())
        codes[b] = c[:, 0::2] | (c[:, 1::2] << 4)
        scales[b] = e
    st["codes"], st["scales"] = codes, scales
    st["lse"] = torch.empty((B, S, H), dtype=torch.float32, device=DEV)
    if op == "attention":
        st["out"] = torch.empty((B, S, H, D), dtype=torch.float32, device=DEV)
        return st
    st["lse"] = _softmax_parts(st)[2]
    st["weights"] = 0.05 * torch.exp(torch.randn((B, T), generator=gen, device=DEV))
    st["ws"] = torch.empty(8 * B * T, dtype=torch.uint8, device=DEV)
    return st


# ---------------------------------------------------------------------------------- the pass
def run(state):
    op = state["case"]["op"]
    return (_own if own else _plain)[op](state)


def _power(e):
    """2^e in float32 for whole numbers e, by its bits: exact."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _nearest(x):
    """Codes [.., D] and scale bytes [.., D / 32] of x [.., D] (float32)."""
    blocks = x.reshape(*x.shape[:-1], -1, BLOCK)
    fraction, exponent = torch.frexp(blocks.abs().amax(dim=-1))
    # amax = 2 fraction 2^(exponent - 1): the least e with amax <= 7 * 2^e
    e = exponent - 3 + (fraction > 0.875).to(exponent.dtype)
    e = torch.where(fraction == 0, torch.full_like(e, LOWEST), e).clamp(LOWEST, HIGHEST)
    y = (blocks * _power(-e)[..., None]).abs()
    # ties go to the even code
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75).to(torch.uint8) + (y > 1.25).to(torch.uint8) + (y >= 1.75).to(torch.uint8)
            + (y > 2.5).to(torch.uint8) + (y >= 3.5).to(torch.uint8) + (y > 5.0).to(torch.uint8))
    code |= (blocks < 0).to(torch.uint8) << 3
    return code.reshape(x.shape), (e + 127).to(torch.uint8)


def _values(table, codes, scales):
    """float32 values [.., D] of packed codes [.., D / 2] and scale bytes [.., D / 32]."""
    v = table[torch.stack([codes & 15, codes >> 4], dim=-1).int()].flatten(-2)
    blocks = v.reshape(*v.shape[:-1], -1, BLOCK)
    return (blocks * _power(scales.int() - 127)[..., None]).reshape(v.shape)


def _store(st):
    code, e = _nearest(st["rows"].float())
    packed = code[..., 0::2] | (code[..., 1::2] << 4)
    return {"rows": _values(st["table"], packed, e).to(torch.bfloat16)}


def _load(st):
    B, N = st["case"]["B"], st["case"]["N"]
    at = st["start"].long()[:, None] + torch.arange(N, device=DEV)[None, :]
    b = torch.arange(B, device=DEV)[:, None]
    return {"rows": _values(st["table"], st["codes"][b, at], st["scales"][b, at]).to(torch.bfloat16)}


def _softmax_parts(st):
    """Rows [B,S,U,D], weights of the softmax [B,S,H,U], their log sum [B,S,H], row numbers [B,S,U] and which of them count."""
    case = st["case"]
    B, T, n_win = case["B"], case["T"], case["n_win"]
    legal = _legal(case, st["lengths"])[..., None]
    first = (legal - n_win).clamp(min=0)
    lists = st["idx"].long()
    window = first + torch.arange(n_win, device=DEV)
    at = torch.cat([lists.clamp(min=0), window.clamp(max=T - 1)], dim=2)
    ok = torch.cat([(lists >= 0) & ~((lists >= first) & (lists < legal)), window < legal], dim=2)
    b = torch.arange(B, device=DEV)[:, None, None]
    rows = _values(st["table"], st["codes"][b, at], st["scales"][b, at])
    x = torch.matmul(st["q"].float(), rows.transpose(2, 3)) * (1.0 / math.sqrt(case["D"]))
    x = x.masked_fill(~ok[:, :, None, :], -math.inf)
    top = x.amax(dim=3, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(dim=3, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    return rows, p, (top + torch.log(total)).squeeze(3), at, ok


def _attend(st):
    rows, p, lse, _, _ = _softmax_parts(st)
    return {"out": torch.matmul(p, rows), "lse": lse}


def _weigh(st):
    _, p, _, at, ok = _softmax_parts(st)
    (B, S), T = p.shape[:2], st["case"]["T"]
    # what each query gives each row, one place for each; entries that do not count go behind the last row
    given = torch.zeros((B, S, T + 1), device=DEV)
    given.scatter_(2, torch.where(ok, at, T), p.sum(dim=2))
    return {"weights": (st["weights"] + given[:, :, :T].sum(dim=1, dtype=torch.float64)).float()}


def _evicted(st):
    case = st["case"]
    B, T, n = case["B"], case["T"], case["n_keep"]
    s = torch.arange(T, device=DEV)[None, :]
    held = torch.full((B, 1), T, device=DEV) if st["lengths"] is None else st["lengths"].long()[:, None]
    always = (s < case["n_sink"]) | (s >= held - case["n_recent"])
    rank = torch.where(always, math.inf, st["weights"].double())
    rank = torch.where(s < held, rank, -math.inf)
    order = torch.sort(rank, dim=1, descending=True, stable=True)[1][:, :n]
    live = torch.arange(n, device=DEV)[None, :] < held
    at = torch.sort(torch.where(live, order, T), dim=1)[0]
    b = torch.arange(B, device=DEV)[:, None]
    safe = at.clamp(max=T - 1)
    return {"kept": torch.where(live, at, -1).to(torch.int32), "held": held.clamp(max=n).to(torch.int32)[:, 0],
            "weights": torch.where(live, st["weights"][b, safe], st["weights_out"]),
            "keys": torch.where(live[..., None], st["keys"][b, safe], st["keys_out"])}


_plain = {"store": _store, "load": _load, "attention": _attend, "weights": _weigh, "evict": _evicted}


def _own_store(st):
    import paper_2605_02568_amd as P
    P.si_quantize_rows(st["rows"], st["start"], st["codes"], st["scales"])
    P.si_dequantize_rows(st["codes"], st["scales"], st["start"], st["out"])
    return {"rows": st["out"]}


def _own_load(st):
    import paper_2605_02568_amd as P
    P.si_dequantize_rows(st["codes"], st["scales"], st["start"], st["out"])
    return {"rows": st["out"]}


def _own_attend(st):
    import paper_2605_02568_amd as P
    case = st["case"]
    P.si_quantized_attention(st["q"], st["codes"], st["scales"], st["lengths"], st["idx"], case["m"], case["mask"], case["n_win"],
                             1.0 / math.sqrt(case["D"]), st["out"], st["lse"])
    return {"out": st["out"], "lse": st["lse"]}


def _own_weigh(st):
    import paper_2605_02568_amd as P
    case = st["case"]
    weights = st["weights"].clone()  # the call adds in place; every pass starts from the same sums
    P.si_accumulate_weights(st["q"], st["codes"], st["scales"], st["lengths"], st["idx"], case["m"], case["mask"], case["n_win"],
                            1.0 / math.sqrt(case["D"]), st["lse"], weights, st["ws"])
    return {"weights": weights}


def _own_evict(st):
    import paper_2605_02568_amd as P
    case = st["case"]
    P.si_evict_rows(st["weights"], st["lengths"], case["n_keep"], case["n_sink"], case["n_recent"],
                    [(st["weights"], st["weights_out"]), (st["keys"], st["keys_out"])], st["kept"], st["held"], st["ws"])
    return {"kept": st["kept"], "held": st["held"], "weights": st["weights_out"], "keys": st["keys_out"]}


_own = {"store": _own_store, "load": _own_load, "attention": _own_attend, "weights": _own_weigh, "evict": _own_evict}


# ---------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    op, B, T = case["op"], case["B"], case["T"]
    if op in ("store", "load"):
        rows, D = B * case["N"], case["D"]
        held = rows * (D // 2 + D // BLOCK)
        if op == "load":
            return {"bytes": held + rows * D * 2, "flops": rows * D}
        return {"bytes": 2 * rows * D * 2 + 2 * held, "flops": 4 * rows * D}
    share = 0.75 if case["ragged"] else 1.0  # lengths are uniform over T/2 .. T
    if op == "evict":
        n = min(case["n_keep"], share * T)
        return {"bytes": B * (T * share * 4 + case["n_keep"] * 4 + n * 2 * (256 + 4)), "flops": 0}
    S, H, D, k = case["S"], case["H"], case["D"], case["k"]
    t = torch.arange(S, dtype=torch.float64)
    legal = torch.full((S,), share * T, dtype=torch.float64)
    if case["mask"] == CAUSAL:
        legal = torch.minimum(legal, torch.floor((t + 1) / case["m"]))
    win, listed_rows = legal.clamp(max=case["n_win"]), legal.clamp(max=k)
    # rows that the window already holds are listed with the probability that a random legal row is one
    union = B * float((listed_rows + win - listed_rows * win / legal.clamp(min=1)).sum())
    nbytes = B * S * H * D * 2 + min(B * T * share, union) * (D // 2 + D // BLOCK) + B * S * k * 4 + B * S * H * 4
    if op == "weights":
        return {"bytes": nbytes + 2 * min(B * T * share, union) * 4, "flops": 2 * union * H * D}
    return {"bytes": nbytes + B * S * H * D * 4, "flops": 4 * union * H * D}


# ---------------------------------------------------------------------------------- in 64 bits
def _values64(codes, scales):
    """By the fields of a code: sign, exponent, mantissa."""
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).long()
    field, mantissa = (c >> 1) & 3, (c & 1).double()
    size = torch.where(field == 0, 0.5 * mantissa, (1.0 + 0.5 * mantissa) * (1 << (field - 1).clamp(min=0)).double())
    size = torch.where(c >= 8, -size, size)
    return size * _power64(scales.long() - 127).repeat_interleave(BLOCK, dim=-1)


def _power64(e):
    return ((e + 1023) << 52).view(torch.float64)


def exact(case, seed):
    op = case["op"]
    st = prepare(case, seed)
    if op == "store":
        out = []
        for rows in st["rows"].split(1):
            x = rows.double().unflatten(2, (-1, BLOCK))
            top = x.abs().amax(dim=3, keepdim=True)
            fits = 7.0 * _power64(torch.arange(LOWEST, HIGHEST, device=DEV))  # the largest value of each power but the last
            power = _power64(LOWEST + (top > fits).sum(dim=3, keepdim=True))
            y = x / power
            step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
            out.append(((torch.round(y / step) * step).clamp(-6, 6) * power).flatten(2))
        return {"rows": torch.cat(out)}
    if op == "load":
        N = case["N"]
        at = st["start"].tolist()
        return {"rows": torch.stack([_values64(st["codes"][b, s:s + N], st["scales"][b, s:s + N]) for b, s in enumerate(at)])}
    if op == "evict":
        return _evicted64(st)
    B, S, H, D, T, k, n_win = (case[x] for x in ("B", "S", "H", "D", "T", "k", "n_win"))
    legal_of = _legal(case, st["lengths"])
    out = torch.zeros((B, S, H, D), dtype=torch.float64, device=DEV)
    lse = torch.empty((B, S, H), dtype=torch.float64, device=DEV)
    weights = torch.zeros((B, T + 1), dtype=torch.float64, device=DEV)
    step = max(1, (1 << 26) // ((k + n_win) * D))
    for b in range(B):
        cache = _values64(st["codes"][b], st["scales"][b])
        for s in range(0, S, step):
            e = min(S, s + step)
            legal = legal_of[b, s:e, None]
            window = legal - 1 - torch.arange(n_win, device=DEV)[None, :]
            lists = st["idx"][b, s:e].long()
            lists = torch.where((lists >= legal - n_win) & (lists < legal), -1, lists)
            at = torch.cat([lists, window.clamp(min=-1)], dim=1)
            ok = (at >= 0)[:, None, :]
            rows = cache[at.clamp(min=0)]
            x = torch.matmul(st["q"][b, s:e].double(), rows.transpose(1, 2).contiguous()) / math.sqrt(D)
            lse[b, s:e] = torch.logsumexp(x.masked_fill(~ok, -math.inf), dim=2)
            p = torch.where(ok, torch.exp(x - lse[b, s:e, :, None]), 0.0)
            out[b, s:e] = torch.matmul(p, rows)
            # entries that do not count are added behind the last row
            weights[b].index_add_(0, torch.where(at >= 0, at, T).reshape(-1), p.sum(dim=1).reshape(-1))
    if op == "attention":
        return {"out": out, "lse": lse}
    return {"weights": st["weights"].double() + weights[:, :T]}


def _evicted64(st):
    """Row by row of the batch, from the order of the weights alone."""
    case = st["case"]
    T, n = case["T"], case["n_keep"]
    kept = torch.full((case["B"], n), -1, dtype=torch.int32, device=DEV)
    held = torch.empty((case["B"],), dtype=torch.int32, device=DEV)
    weights, keys = st["weights_out"].double(), st["keys_out"].double()
    for b in range(case["B"]):
        length = T if st["lengths"] is None else int(st["lengths"][b])
        first, last = min(case["n_sink"], length), max(0, length - case["n_recent"])
        last = max(last, first)
        room = min(n, length) - first - (length - last)
        middle = torch.argsort(-st["weights"][b, first:last].double(), stable=True)[:room] + first
        at = torch.cat([torch.arange(first, device=DEV), torch.sort(middle)[0], torch.arange(last, length, device=DEV)])
        held[b] = len(at)
        kept[b, :len(at)] = at.to(torch.int32)
        weights[b, :len(at)] = st["weights"][b, at].double()
        keys[b, :len(at)] = st["keys"][b, at].double()
    return {"kept": kept, "held": held, "weights": weights, "keys": keys}
