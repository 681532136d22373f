"""GPU tests of the paged cache and of packed prompts as a server uses them: prompts, rows into pages, next parts, decoding, drafted positions, one after the
other; on side streams, captured and replayed with lengths that grow between replays, by graphs that share a workspace, and two calls at once."""
import numpy as np
import pytest
import torch

import paper_2605_02568_amd as P
from tests import dense_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NONE, CAUSAL = P.SI_MASK_NONE, P.SI_MASK_CAUSAL_BLOCK


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _offsets(lengths):
    return _ints([0] + [int(x) for x in np.cumsum(lengths)])


def _near(got, lse, want, what):
    ro, rl, to, tl = want
    assert np.all(np.abs(R.to64(got) - ro) <= to), what
    assert np.all(np.abs(R.to64(lse) - rl) <= tl), what


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D,H,H_kv,room", [(128, 16, 2, 320), (64, 33, 1, 320), (128, 16, 2, 2048), (64, 33, 1, 1600)])
def test_requests_from_prompt_to_drafted_positions(bits, D, H, H_kv, room):
    g = torch.Generator().manual_seed(bits + D)
    scale, page, wide, n_pages = 1.0 / np.sqrt(D), 16, room // 16, 3 * room // 16 + 10
    parts = [[130, 61, 7], [33, 100, 1]]  # two parts of each prompt
    B = 3
    total = [sum(p) for p in zip(*parts)]
    new = 3 + 2 * 2  # three single positions, two times two drafted ones
    rand = lambda n, h: torch.randn((n, h, D), generator=g).to(torch.bfloat16)  # noqa: E731
    q, k, v = ([rand(n + new, h) for n in total] for h in (H, H_kv, H_kv))
    shape = (n_pages, H_kv, page, D)
    K, V = (torch.zeros(shape, dtype=torch.bfloat16 if bits == 16 else torch.uint8, device=DEV) for _ in range(2))
    scales = [None, None] if bits == 16 else [torch.full(shape[:3], 127, dtype=torch.uint8, device=DEV) for _ in range(2)]
    table = torch.randperm(n_pages, generator=g)[:B * wide].view(B, wide).to(torch.int32).to(DEV)
    held = [0] * B

    def store(lengths):
        rows = [torch.cat([x[b][held[b]:held[b] + n] for b, n in enumerate(lengths)]).to(DEV) for x in (k, v)]
        P.si_store_pages(*rows, _offsets(lengths), _ints(held), table, K, V, *scales)

    def kept(b):  # rows of request b as the cache holds them
        rows = [R.to64(x[b]) for x in (k, v)]
        return rows if bits == 16 else [R.values(*R.quantize(x)) for x in rows]

    for lengths in parts:
        queries = torch.cat([q[b][held[b]:held[b] + n] for b, n in enumerate(lengths)]).to(DEV)
        after = [h + n for h, n in zip(held, lengths)]
        store(lengths)
        if bits == 16:  # the rows of all parts so far come back from the pages
            rows = [torch.empty((sum(after), H_kv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
            P.si_load_pages(table, K, V, *scales, _offsets(after), None, *rows)
        else:
            rows = [torch.cat([x[b][:n] for b, n in enumerate(after)]).to(DEV) for x in (k, v)]
        out, lse = torch.empty_like(queries), torch.empty(queries.shape[:2], device=DEV)
        P.si_prompt_attention(queries, *rows, _offsets(lengths), _offsets(after), _ints(held), 1, CAUSAL, R.ALL, scale, out, lse)
        torch.cuda.synchronize()
        at = 0
        for b, n in enumerate(lengths):
            want = R.attend(R.to64(q[b][held[b]:after[b]]), R.to64(k[b][:after[b]]), R.to64(v[b][:after[b]]), range(held[b], after[b]), 1, 1, R.ALL, scale)
            _near(out[at:at + n], lse[at:at + n], want, (lengths, b))
            at += n
        held = after
    for S in (1, 1, 1, 2, 2):
        store([S] * B)
        first, held = held, [h + S for h in held]
        queries = torch.stack([q[b][first[b]:held[b]] for b in range(B)]).to(DEV)
        out, lse = torch.empty_like(queries), torch.empty(queries.shape[:3], device=DEV)
        ws = torch.empty(P.si_paged_workspace_bytes(B, S, H, H_kv, D), dtype=torch.uint8, device=DEV)
        P.si_paged_attention(queries, table, K, V, *scales, _ints(held), _ints(first), 1, CAUSAL, R.ALL, scale, out, lse, ws)
        torch.cuda.synchronize()
        for b in range(B):
            rows = [x[:held[b]] for x in kept(b)]
            _near(out[b], lse[b], R.attend(R.to64(queries[b]), *rows, range(first[b], held[b]), 1, 1, R.ALL, scale), (S, b))


def _paged_problem(seed, lengths, S, H, H_kv, D, bits, wide=None):
    pages = R.Pages(seed, lengths, H_kv, D, bits, 64, filler=0.0, wide=wide)
    q = torch.randn((len(lengths), S, H, D), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)
    outputs = [torch.empty(q.shape, dtype=torch.bfloat16, device=DEV), torch.empty(q.shape[:3], device=DEV)]
    ws = torch.empty(P.si_paged_workspace_bytes(len(lengths), S, H, H_kv, D), dtype=torch.uint8, device=DEV)
    cache, held = pages.to(DEV), _ints(lengths)

    def call(o, stream=None):
        P.si_paged_attention(q, *cache, held, None, 1, NONE, R.ALL, 0.1, o[0], o[1], ws, stream=stream)

    call.held, call.workspace, call.keep = held, ws, cache
    return call, outputs


def _same(a, b):
    return all(torch.equal(x.view(torch.int16 if x.dtype is torch.bfloat16 else torch.int32), y.view(torch.int16 if y.dtype is torch.bfloat16 else torch.int32))
               for x, y in zip(a, b))


def _fresh(outputs):
    return [torch.full_like(o, -9) for o in outputs]


def _replays(call, outputs, ws=None):
    eager, on_side, captured = _fresh(outputs), _fresh(outputs), _fresh(outputs)
    call(eager, None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(on_side, side)
    side.synchronize()
    assert _same(eager, on_side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(captured, None)
    for replay in range(3):
        for o in captured:
            o.fill_(-9)
        if ws is not None:
            ws.random_(0, 255)  # the workspace carries nothing from call to call
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert _same(eager, captured), f"replay {replay}"
        again = _fresh(outputs)
        call(again, None)
        torch.cuda.synchronize()
        assert _same(eager, again)


@pytest.mark.parametrize("lengths,S,H,H_kv,D,bits", [([3000, 5, 700], 1, 8, 8, 128, 16), ([2000] * 5, 1, 64, 1, 128, 8), ([900, 333], 4, 40, 8, 64, 8), ([100], 1, 8, 2, 64, 16),
                                                         ([1100, 0] + list(range(30, 130)), 1, 8, 4, 64, 16)])
def test_attention_on_a_side_stream_and_replayed(lengths, S, H, H_kv, D, bits):
    call, outputs = _paged_problem(1, lengths, S, H, H_kv, D, bits)
    _replays(call, outputs, call.workspace)


@pytest.mark.parametrize("n,H,H_kv,D", [(700, 64, 8, 128), (150, 8, 2, 64), (2300, 32, 4, 128), (7000, 16, 2, 128)])
def test_prompts_on_a_side_stream_and_replayed(n, H, H_kv, D):
    g = torch.Generator().manual_seed(n)
    q = torch.randn((n, H, D), generator=g).to(torch.bfloat16).to(DEV)
    k, v = (torch.randn((n, H_kv, D), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    off = _ints([0, n // 3, n])
    _replays(lambda o, stream: P.si_prompt_attention(q, k, v, off, off, None, 1, CAUSAL, R.ALL, 0.1, o[0], o[1], stream=stream),
             [torch.empty_like(q), torch.empty((n, H), device=DEV)])


@pytest.mark.parametrize("bits", [16, 8])
def test_rows_on_a_side_stream_and_replayed(bits):
    n, H, D = 777, 5, 128
    g = torch.Generator().manual_seed(n)
    k, v = (torch.randn((n, H, D), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    shape = (60, H, 16, D)
    K, V = (torch.zeros(shape, dtype=torch.bfloat16 if bits == 16 else torch.uint8, device=DEV) for _ in range(2))
    scales = [None, None] if bits == 16 else [torch.zeros(shape[:3], dtype=torch.uint8, device=DEV) for _ in range(2)]
    table = torch.randperm(60, generator=g)[:54].view(2, 27).to(torch.int32).to(DEV)
    off, start = _ints([0, 400, 777]), _ints([3, 11])

    def call(o, stream):
        P.si_store_pages(k, v, off, start, table, K, V, *scales, stream=stream)
        P.si_load_pages(table, K, V, *scales, off, start, o[0], o[1], stream=stream)

    _replays(call, [torch.empty_like(k), torch.empty_like(v)])


def test_a_captured_call_follows_lengths_that_grow():
    """The rows are dealt out on the GPU: a graph captured with short requests serves them when they have become long, and the other way round."""
    call, outputs = _paged_problem(2, [5000, 3000, 64], 1, 16, 2, 128, 16)
    call.held.copy_(_ints([3, 0, 1]))
    captured = _fresh(outputs)
    call(captured)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(captured)
    for lengths in ([3, 0, 1], [5000, 3000, 64], [0, 0, 0], [4097, 31, 33], [128, 2999, 0]):
        call.held.copy_(_ints(lengths))
        graph.replay()
        torch.cuda.synchronize()
        eager = _fresh(outputs)
        call(eager)
        torch.cuda.synchronize()
        assert _same(eager, captured), lengths
        assert bool((captured[0][[n == 0 for n in lengths]] == 0).all())


def test_graphs_that_share_a_workspace():
    problems = [_paged_problem(s, lengths, 1, 16, 2, 128, 16) for s, lengths in ((3, [4000, 100]), (4, [700, 2500]))]
    ws = problems[0][0].workspace
    eager, captured, graphs = [], [], []
    for call, outputs in problems:
        eager.append(_fresh(outputs))
        call(eager[-1])
        torch.cuda.synchronize()
        captured.append(_fresh(outputs))
    for i, (call, outputs) in enumerate(problems):
        q = torch.randn((2, 1, 16, 128), generator=torch.Generator().manual_seed(i + 3)).to(torch.bfloat16).to(DEV)
        graphs.append((torch.cuda.CUDAGraph(), q))
        with torch.cuda.graph(graphs[-1][0]):
            P.si_paged_attention(q, *call.keep, call.held, None, 1, NONE, R.ALL, 0.1, *captured[i], ws)
    for order in ((0, 1), (1, 0), (0, 0), (1, 1)):
        for i in order:
            for o in captured[i]:
                o.fill_(-9)
        for i in order:
            graphs[i][0].replay()
        torch.cuda.synchronize()
        for i in order:
            assert _same(eager[i], captured[i]), order


def test_two_calls_at_once():
    """On two streams, each with a workspace of its own."""
    problems = [_paged_problem(s, lengths, 1, 64, 1, 128, bits) for s, lengths, bits in ((5, [9000, 300], 8), (6, [700, 6500], 16))]
    eager = []
    for call, outputs in problems:
        eager.append(_fresh(outputs))
        call(eager[-1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in problems]
    results = [[_fresh(outputs) for _ in range(5)] for _, outputs in problems]
    torch.cuda.synchronize()
    for i in range(5):
        for (call, _), stream, got in zip(problems, streams, results):
            with torch.cuda.stream(stream):
                call(got[i], stream)
    torch.cuda.synchronize()
    for want, got in zip(eager, results):
        assert all(_same(want, g) for g in got)
