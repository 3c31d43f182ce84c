"""Beam selection and the states behind it, on the GPU, against plain forms in 64 bits.

Scores are float64 values rounded once to float32: half a step, 2^-24 of the value, beside 1e-9 for the sum of 131072 exponentials (1.04e-10 of the sum at most, the
bound of the polynomial, and a few 1e-16 per addition).  Where parent and token are others than the plain form's at that rank, theirs must be as good: the plain
score of the one chosen lies within 2.4e-10 of the score wanted there.  (Let every score be off by e = 1.2e-10 at most: 1.04e-10 of the polynomial, 0.15e-10 of the
rounding to 2^-35 and what the additions lose.  The r best by the kernel's scores and the r best by the plain ones have r-th scores that differ by e at most, and the
plain score of what the kernel chose differs by e from its own.)  So do equal beams, whose rows begin at different places modulo 16 bytes, come in either order;
where they begin at the same place, the order is the plain form's.
"""
import numpy as np
import pytest

from beside_forms import ROW_BAD, beam_select, reorder, softmax_mass

pytestmark = pytest.mark.gpu
NEAR = 2.4e-10


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


@pytest.fixture(scope="module")
def gr():
    from paper_2511_15898_amd import binding
    return binding


def _select(torch, gr, logits, scores, M, T=None, finished=None, eos=-1):
    """A call, run twice; the outputs as arrays."""
    S, K, V = logits.shape
    h = gr.gr_create(S * K, V)
    to = lambda v, t=None: None if v is None else torch.from_numpy(np.ascontiguousarray(v)).cuda()  # noqa: E731
    try:
        args = (h, logits, to(np.asarray(scores, np.float32)), M)
        more = dict(temperature=to(T), finished=to(finished), eos=eos)
        out = [x.clone() for x in gr.gr_beam_select(*args, **more)]
        again = gr.gr_beam_select(*args, **more)
        assert all(torch.equal(a, b) for a, b in zip(out, again))
        return [x.cpu().numpy() for x in out]
    finally:
        gr.gr_destroy(h)


def _plain_score(logits, scores, T, finished, eos, b, v):
    if finished is not None and finished[b]:
        assert v == eos
        return float(scores[b])
    x = logits[b].astype(np.float64)
    return float(scores[b]) + ((x[v] - x.max()) / T - np.log(softmax_mass(x, T).sum()))


def _check(got, logits, scores, M, T=None, finished=None, eos=-1, exact=False):
    best, parent, token, over, status = got
    for s in range(logits.shape[0]):
        want = beam_select(logits[s], scores[s], M, 1.0 if T is None else float(T[s]), None if finished is None else finished[s], eos)
        assert status[s] == 0
        for r in range(M):
            if r >= len(want):
                assert best[s, r] == -np.inf and parent[s, r] == -1 and token[s, r] == -1 and over[s, r] == 0, (s, r)
                continue
            score, b, v = want[r]
            assert abs(float(best[s, r]) - score) <= 2.0 ** -24 * abs(score) + 1e-9, (s, r, best[s, r], score)
            if (parent[s, r], token[s, r]) != (b, v):
                chosen = _plain_score(logits[s], scores[s], 1.0 if T is None else float(T[s]), None if finished is None else finished[s], eos, parent[s, r], token[s, r])
                assert not exact and abs(chosen - score) <= NEAR, (s, r, parent[s, r], token[s, r], chosen, want[r])
            assert over[s, r] == (token[s, r] == eos)
        assert len(set(zip(parent[s, :len(want)].tolist(), token[s, :len(want)].tolist()))) == min(M, len(want))


def _rows(torch, seed, S, K, V, dtype, pad=0, spread=4.0):
    x = (spread * np.random.default_rng(seed).gumbel(size=(S, K, V + pad))).astype(np.float32)
    view = torch.from_numpy(x).cuda().to(getattr(torch, dtype))[:, :, :V]
    return view, view.float().cpu().numpy()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("S,K,V,M,pad", [(1, 1, 1, 1, 0), (1, 1, 3, 8, 1), (2, 3, 5, 16, 0), (1, 4, 255, 4, 0), (3, 2, 1000, 64, 3), (2, 5, 4097, 10, 1), (1, 64, 700, 64, 0),
                                       (1, 64, 9001, 33, 2), (4, 8, 8192, 16, 0), (5, 3, 20001, 6, 7), (1, 4, 32000, 4, 0), (1, 2, 128256, 1, 0), (40, 10, 3001, 20, 0)])
def test_continuations(torch, gr, dtype, S, K, V, M, pad):
    rng = np.random.default_rng(V + M)
    x, ref = _rows(torch, S * V + K, S, K, V, dtype, pad)
    scores = -20.0 * rng.random((S, K)).astype(np.float32)
    T = rng.uniform(0.5, 2.0, S).astype(np.float32) if V % 2 else None
    _check(_select(torch, gr, x, scores, M, T), ref, scores, M, T)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [60, 9001])
def test_finished_unused_and_masked_beams(torch, gr, dtype, V):
    """A finished beam stands beside the others with its score alone; one that is not in use gives nothing, whatever its row holds; a row without an unmasked token neither."""
    S, K, M, eos = 6, 5, 12, 7
    x, ref = _rows(torch, V, S, K, V, dtype, spread=1.0)
    scores = np.full((S, K), -3.0, np.float32) - np.arange(K, dtype=np.float32)
    finished = np.zeros((S, K), np.uint8)
    x, ref = x.clone(), ref.copy()

    def fill(s, b, value):
        x[s, b] = value; ref[s, b] = value
    finished[1, [0, 3]] = 1; fill(1, 3, float("nan"))                       # a finished beam's row is not read
    scores[2, 1:] = -np.inf; fill(2, 2, float("nan"))                      # the first step of a search: one beam
    scores[3] = -np.inf                                                  # nothing in use
    fill(4, 0, -np.inf); finished[4] = [0, 1, 1, 1, 1]                      # only what has ended is left
    finished[5, :] = 1
    _check(_select(torch, gr, x, scores, M, finished=finished, eos=eos), ref, scores, M, finished=finished, eos=eos)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("K,V,M", [(1, 5000, 7), (4, 3000, 20), (64, 2500, 64), (8, 40000, 16)])
def test_ties_go_to_the_lower_beam_and_token(torch, gr, dtype, K, V, M):
    t = getattr(torch, dtype)
    flat = torch.zeros((1, K, V), dtype=t, device="cuda")
    some = flat.clone(); some[:, :, 5::7] = 2.0
    for x in (flat, some):
        scores = np.zeros((1, K), np.float32)
        best, parent, token, over, status = _select(torch, gr, x, scores, M)
        ids = np.arange(V) if x is flat else np.arange(5, V, 7)
        want = [(b, v) for b in range(K) for v in ids[:M]][:M]
        assert [(int(p), int(v)) for p, v in zip(parent[0], token[0])] == want
        _check([best, parent, token, over, status], x.float().cpu().numpy(), scores, M)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_lowest_values_and_rows_far_apart(torch, gr, dtype):
    """The type's lowest value in masked places, rows of nothing else, entries hundreds of temperatures above the rest late in a row, large and tiny temperatures."""
    t = getattr(torch, dtype)
    lowest = float(torch.finfo(t).min)
    V = 20000
    rows = np.random.default_rng(0).standard_normal((1, 6, V)).astype(np.float32)
    rows[0, 1, 100:] = lowest
    rows[0, 2] = lowest
    rows[0, 3, V - 5] = 900.0
    rows[0, 4, :V // 2] = -20000.0
    rows[0, 5, 1::2] = -np.inf
    x = torch.from_numpy(rows).cuda().to(t)
    for T in (1.0, 0.01, 50.0):
        scores = np.array([[-1.0, -2.0, -3.0, -2.5, -1.5, -0.5]], np.float32)
        _check(_select(torch, gr, x, scores, 40, np.array([T], np.float32)), x.float().cpu().numpy(), scores, 40, [np.float32(T)])


def test_bad_sequences(torch, gr):
    S, K, V, M = 8, 3, 3000, 5
    x, ref = _rows(torch, 3, S, K, V, "float32")
    x, ref = x.clone(), ref.copy()
    scores, T = np.full((S, K), -1.0, np.float32), np.ones(S, np.float32)
    x[0, 1, 2999] = float("nan"); x[1, 2, 0] = float("inf"); scores[2, 0] = np.nan; scores[3, 1] = np.inf
    T[4], T[5], T[6] = 0.0, np.nan, -2.0
    got = _select(torch, gr, x, scores, M, T)
    assert (got[4][:7] == ROW_BAD).all() and (got[0][:7] == -np.inf).all() and (got[1][:7] == -1).all() and (got[2][:7] == -1).all() and (got[3][:7] == 0).all()
    _check([v[7:] for v in got], ref[7:], scores[7:], M, T[7:])


def test_a_selection_on_another_stream_and_in_a_graph(torch, gr):
    S, K, V, M = 3, 4, 5000, 8
    x, _ = _rows(torch, 1, S, K, V, "bfloat16")
    x = x.clone()
    scores = torch.zeros((S, K), device="cuda")
    h = gr.gr_create(S * K, V)
    try:
        want = [v.clone() for v in gr.gr_beam_select(h, x, scores, M)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = gr.gr_beam_select(h, x, scores, M, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        out = tuple(torch.empty_like(v) for v in want)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            gr.gr_beam_select(h, x, scores, M, out=out)
        for turn in range(4):
            x.copy_(_rows(torch, 50 + turn, S, K, V, "bfloat16")[0])
            graph.replay()
            torch.cuda.synchronize()
            eager = gr.gr_beam_select(h, x, scores, M)
            assert all(torch.equal(a, b) for a, b in zip(out, eager)), turn
    finally:
        gr.gr_destroy(h)


# ---------------------------------------------------------------- states

def _parents(rng, S, K, kind):
    if kind == "random":
        return rng.integers(0, K, (S, K)).astype(np.int32)
    if kind == "turn":                                                   # every beam takes the next one's
        return ((np.arange(K)[None] + 1 + np.arange(S)[:, None]) % K).astype(np.int32)
    if kind == "one":
        return np.full((S, K), K - 1, np.int32)
    return rng.choice([-1, K, 0, 2 ** 31 - 1, -2 ** 31], (S, K)).astype(np.int32)   # outside: left as they are


def _bytes(torch, rng, shape, dtype):
    size = torch.empty((), dtype=dtype).element_size()
    return torch.from_numpy(rng.integers(0, 256, (*shape[:-1], shape[-1] * size), dtype=np.uint8)).cuda().view(dtype)


def _numpy(state):
    import torch
    flat = state.contiguous()
    return flat.view(torch.uint8).cpu().numpy()


@pytest.mark.parametrize("kind", ["random", "turn", "one", "outside"])
@pytest.mark.parametrize("S,K,O,H,T,D,dtype", [(1, 2, 1, 1, 1, 1, "uint8"), (2, 3, 2, 3, 17, 5, "uint8"), (1, 4, 3, 2, 33, 64, "bfloat16"), (3, 5, 1, 4, 100, 37, "float16"),
                                              (2, 16, 2, 2, 40, 24, "float32"), (1, 17, 1, 3, 9, 31, "bfloat16"), (1, 33, 2, 1, 20, 16, "bfloat16"), (1, 64, 1, 2, 7, 13, "uint8"),
                                              (2, 8, 5, 1, 1, 5001, "float32"), (1, 3, 1, 2, 700, 128, "bfloat16")])
@pytest.mark.parametrize("tokens_first", [False, True])
def test_dense_states(torch, gr, kind, S, K, O, H, T, D, dtype, tokens_first):
    rng = np.random.default_rng(S * K + T + D)
    t = getattr(torch, dtype)
    shape = (O, S * K, T, H, D) if tokens_first else (O, S * K, H, T, D)
    state = _bytes(torch, rng, shape, t)
    if tokens_first:
        state = state.transpose(2, 3)
    parent = _parents(rng, S, K, kind)
    length = rng.integers(0, T + 3, S).astype(np.int32)                     # beyond the end: cut to it
    first = rng.integers(-2, T, S).astype(np.int32)
    for f, l in [(None, None), (first, length), (None, length)]:
        want = reorder(_numpy(state), parent, f, l)
        to = lambda v: None if v is None else torch.from_numpy(v).cuda()  # noqa: E731
        got = gr.gr_beam_reorder(state, to(parent), to(f), to(l))
        assert got is state and np.array_equal(_numpy(state), want)


def _pages(rng, S, K, width, block, length, first, blocks):
    """A table: pages below `first` are the first beam's, the others each beam's own; places beyond the length are no blocks at all."""
    ids = rng.permutation(blocks).tolist()
    table = np.full((S * K, width), -1, np.int32)
    for s in range(S):
        for b in range(K):
            for j in range(-(-int(length[s]) // block)):
                table[s * K + b, j] = table[s * K, j] if b and (j + 1) * block <= first[s] else ids.pop()
    return table


@pytest.mark.parametrize("kind", ["random", "turn"])
@pytest.mark.parametrize("S,K,O,H,block,width,D,dtype", [(1, 2, 1, 1, 1, 3, 16, "uint8"), (2, 4, 2, 2, 16, 5, 64, "bfloat16"), (3, 3, 1, 3, 13, 4, 7, "uint8"), (2, 8, 3, 2, 8, 6, 80, "float16"),
                                                       (1, 16, 2, 1, 32, 3, 128, "bfloat16"), (1, 20, 1, 2, 5, 4, 33, "float32")])
@pytest.mark.parametrize("tokens_first", [False, True])
def test_states_in_pages(torch, gr, kind, S, K, O, H, block, width, D, dtype, tokens_first):
    rng = np.random.default_rng(K * width + D)
    t = getattr(torch, dtype)
    blocks = S * K * width + 2
    state = _bytes(torch, rng, (O, blocks, block, H, D) if tokens_first else (O, blocks, H, block, D), t)
    if tokens_first:
        state = state.transpose(2, 3)
    parent = _parents(rng, S, K, kind)
    length = rng.integers(0, block * width + 1, S).astype(np.int32)
    length[0] = block * width
    first = (length * 0.4).astype(np.int32)
    table = _pages(rng, S, K, width, block, length, first, blocks)
    table[-1, 0] = blocks + 5                                               # no such block: skipped
    to = lambda v: torch.from_numpy(v).cuda()  # noqa: E731
    want = reorder(_numpy(state), parent, first, length, table)
    gr.gr_beam_reorder(state, to(parent), to(first), to(length), to(table))
    assert np.array_equal(_numpy(state), want)


def test_states_in_a_view_leave_what_lies_around_them(torch, gr):
    """A slice of a larger buffer: odd offsets, gaps between heads, tokens and rows."""
    rng = np.random.default_rng(1)
    room = torch.from_numpy(rng.integers(0, 256, (3, 9, 4, 21, 40), dtype=np.uint8)).cuda()
    before = room.cpu().numpy().copy()
    view = room[1:, 2:8, 1:3, 3:20, 5:36]
    parent = np.array([[2, 0, 1], [1, 1, 0]], np.int32)
    gr.gr_beam_reorder(view, torch.from_numpy(parent).cuda(), None, torch.tensor([17, 4], dtype=torch.int32, device="cuda"))
    want = before.copy()
    want[1:, 2:8, 1:3, 3:20, 5:36] = reorder(before[1:, 2:8, 1:3, 3:20, 5:36], parent, None, [17, 4])
    assert np.array_equal(room.cpu().numpy(), want)


def test_states_beyond_32_bits(torch, gr):
    """Rows 3 GB apart."""
    state = torch.zeros((1, 3, 1, 50000, 60000), dtype=torch.uint8, device="cuda")
    for b in range(3):
        state[0, b, 0, -5:] = b + 1
        state[0, b, 0, 25000] = 10 + b
    gr.gr_beam_reorder(state, torch.tensor([[2, 0, 0]], dtype=torch.int32, device="cuda"), torch.tensor([24999], dtype=torch.int32, device="cuda"))
    for b, p in enumerate([2, 0, 0]):
        assert bool((state[0, b, 0, -5:] == p + 1).all()) and bool((state[0, b, 0, 25000] == 10 + p).all()) and int(state[0, b, 0, 24000].max()) == 0
    del state
    torch.cuda.empty_cache()


def test_states_in_a_graph(torch, gr):
    rng = np.random.default_rng(4)
    state = _bytes(torch, rng, (2, 8, 2, 50, 16), torch.bfloat16)
    parent = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    length = torch.zeros(2, dtype=torch.int32, device="cuda")
    gr.gr_beam_reorder(state, parent, None, length)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gr.gr_beam_reorder(state, parent, None, length)
    for turn in range(4):
        p, l = _parents(rng, 2, 4, "random"), rng.integers(0, 51, 2).astype(np.int32)
        parent.copy_(torch.from_numpy(p)); length.copy_(torch.from_numpy(l))
        want = reorder(_numpy(state), p, None, l)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(_numpy(state), want), turn


def test_refusals(torch, gr):
    h = gr.gr_create(8, 100)
    x, scores = torch.zeros((2, 4, 100), device="cuda"), torch.zeros((2, 4), device="cuda")
    state, parent = torch.zeros((1, 8, 1, 4, 4), device="cuda"), torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    try:
        for call in [lambda: gr.gr_beam_select(h, x, scores, 65), lambda: gr.gr_beam_select(h, x, scores, 0), lambda: gr.gr_beam_select(h, x, scores, 4, eos=100),
                     lambda: gr.gr_beam_select(h, x, scores, 4, finished=torch.zeros((2, 4), dtype=torch.uint8, device="cuda")),
                     lambda: gr.gr_beam_select(h, torch.zeros((3, 4, 100), device="cuda"), torch.zeros((3, 4), device="cuda"), 4),
                     lambda: gr.gr_beam_select(h, torch.zeros((1, 1, 101), device="cuda"), torch.zeros((1, 1), device="cuda"), 4),
                     lambda: gr.gr_beam_reorder(torch.zeros((1, 65, 1, 4, 4), device="cuda"), torch.zeros((1, 65), dtype=torch.int32, device="cuda"))]:
            with pytest.raises(gr.GrError) as e:
                call()
            assert e.value.code == gr.GR_EINVAL
        for call in [lambda: gr.gr_beam_select(h, x.double(), scores, 4), lambda: gr.gr_beam_select(h, x.cpu(), scores, 4), lambda: gr.gr_beam_select(h, x, scores[:1], 4),
                     lambda: gr.gr_beam_select(h, x.transpose(0, 1), scores, 4), lambda: gr.gr_beam_select(h, x, scores.double(), 4),
                     lambda: gr.gr_beam_reorder(state[0], parent), lambda: gr.gr_beam_reorder(state, parent[:1]), lambda: gr.gr_beam_reorder(state.transpose(3, 4), parent),
                     lambda: gr.gr_beam_reorder(state[:, :1].expand(1, 8, 1, 4, 4), parent), lambda: gr.gr_beam_reorder(state, parent.long()),
                     lambda: gr.gr_beam_reorder(state, parent, table=torch.zeros((7, 2), dtype=torch.int32, device="cuda"))]:
            with pytest.raises(TypeError):
                call()
    finally:
        gr.gr_destroy(h)


@pytest.mark.parametrize("S,K,V,M,dtype", [(1, 10, 128256, 20, "float32"), (1, 64, 70001, 64, "bfloat16"), (2, 33, 40000, 1, "float16"), (1, 1, 600001, 64, "float32"), (90, 10, 9001, 5, "bfloat16")])
def test_selections_of_many_slices(torch, gr, S, K, V, M, dtype):
    """Hundreds of lists of candidates to a sequence, sequences by the dozen, a row of many tiles."""
    x = torch.from_numpy((3.0 * np.random.default_rng(V).gumbel(size=(S, K, V))).astype(np.float32)).cuda().to(getattr(torch, dtype))
    scores = np.random.default_rng(K).uniform(-6, -4, (S, K)).astype(np.float32)
    got = _select(torch, gr, x, scores, M)
    some = sorted({0, S - 1})
    _check([v[some] for v in got], x[some].float().cpu().numpy(), scores[some], M)


@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_that_rise_and_fall_by_thousands(torch, gr, up, dtype):
    """The largest entry so far lies far above or below what follows: sums are brought to another reference many times, or never."""
    V = 90001
    row = torch.linspace(0.0, 6000.0, V, device="cuda")
    x = torch.stack([row, 0.5 * row, torch.floor(row / 500) * 500]).to(getattr(torch, dtype))[None]
    x = (x if up else x.flip(2)).contiguous()
    scores = np.array([[-3.0, -2.0, -1.0]], np.float32)
    for T in (1.0, 0.05, 700.0):
        _check(_select(torch, gr, x, scores, 12, np.array([T], np.float32)), x.float().cpu().numpy(), scores, 12, [np.float32(T)])


def test_two_handles_on_two_streams(torch, gr):
    """Drafts and selections of two handles at the same time, on streams of their own, for many turns: what they give one after the other."""
    V, turns = 50021, 12
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = [torch.randn((S, K, V), device="cuda", generator=gen) * 3 for S, K in ((3, 4), (1, 8))]
    scores = [torch.zeros(v.shape[:2], device="cuda") for v in x]
    u = [torch.rand((v.shape[0] * v.shape[1], 5), device="cuda", generator=gen) for v in x]
    T = [torch.ones(len(v), device="cuda") for v in u]
    handles = [gr.gr_create(16, V) for _ in x]
    streams = [torch.cuda.Stream() for _ in x]
    try:
        def both(i, stream=None):
            drafts = gr.gr_draft_logits(handles[i], x[i].view(-1, V), T[i], 5, 30, u[i], stream=stream)
            whole = gr.gr_draft_logits(handles[i], x[i].view(-1, V), T[i], 5, 0, u[i], stream=stream)
            return list(drafts) + list(whole) + list(gr.gr_beam_select(handles[i], x[i], scores[i], 6, stream=stream))
        want = [both(i) for i in range(2)]
        torch.cuda.synchronize()
        got = [[both(i, streams[i]) for i in range(2)] for _ in range(turns)]
        torch.cuda.synchronize()
        for turn in got:
            for i in range(2):
                assert all(torch.equal(a, b) for a, b in zip(turn[i], want[i]))
    finally:
        for h in handles:
            gr.gr_destroy(h)


@pytest.mark.parametrize("S,K,V,M", [(1, 1, 1, 1), (2, 3, 5, 8), (3, 2, 130, 30), (7, 12, 1139, 24), (2, 5, 2049, 64), (1, 16, 513, 64), (4, 16, 3100, 17), (2, 64, 300, 50)])
@pytest.mark.parametrize("levels", [1, 3, 40])
def test_few_levels_in_short_rows(torch, gr, S, K, V, M, levels):
    """Rows shorter than a tile whose entries take a few values only, beams of a few scores: most candidates tie with others, within their beam and across."""
    rng = np.random.default_rng(V + levels)
    x = torch.from_numpy(rng.integers(0, levels, (S, K, V)).astype(np.float32)).cuda()
    x[:, :, 1::9] = -float("inf")
    x[:, :, 0] = 0.0
    if K > 1:
        x[:, 1::2] = x[:, :1]                                            # equal beams, at another alignment where V is odd
    scores = rng.integers(-2, 0, (S, K)).astype(np.float32)
    for dtype in (torch.float32, torch.bfloat16):
        y = x.to(dtype)
        _check(_select(torch, gr, y, scores, M), y.float().cpu().numpy(), scores, M, exact=V * y.element_size() % 16 == 0)


def test_scores_beyond_float32(torch, gr):
    """The lowest value at a temperature below 1: the score is one of float64 and -inf in float32, the choice is there."""
    x = torch.full((1, 2, 700), float(torch.finfo(torch.bfloat16).min), dtype=torch.bfloat16, device="cuda")
    x[0, 0, 9] = x[0, 1, 4] = 0.0
    best, parent, token, over, status = _select(torch, gr, x, np.array([[-1.0, -2.0]], np.float32), 5, T=np.array([0.25], np.float32), eos=4)
    assert best.tolist() == [[-1.0, -2.0] + [-np.inf] * 3] and parent.tolist() == [[0, 1, 0, 0, 0]] and token.tolist() == [[9, 4, 0, 1, 2]] and over.tolist() == [[0, 1, 0, 0, 0]]
    assert status.tolist() == [0]
