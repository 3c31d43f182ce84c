"""Block tables, slots and the free list on the GPU against a walk over the requests one by one; and the operators of a decoding loop together."""
import numpy as np
import pytest

from beside_forms import beam_select, page_update

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


@pytest.fixture(scope="module")
def gr():
    from paper_2511_15898_amd import binding
    return binding


def _inputs(rng, lengths, new_lengths, block, width, spare, slots):
    lengths, new_lengths = np.asarray(lengths, np.int32), np.asarray(new_lengths, np.int32)
    R = len(lengths)
    table = np.full((R, width), -1, np.int32)
    held = [min(width, max(0, -(-int(x) // block))) for x in lengths]
    ids = rng.permutation(sum(held) + spare).astype(np.int32)
    at = 0
    for r, n in enumerate(held):
        table[r, :n] = ids[at:at + n]
        at += n
    stack = np.full(len(ids) + 3, -9, np.int32)
    stack[:spare] = ids[at:]
    return dict(lengths=lengths, new_lengths=new_lengths, table=table, free_blocks=stack, free_count=spare, block=block, slots=np.full(slots, -7, np.int64))


def _run(torch, gr, c, **more):
    to = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()  # noqa: E731
    table, stack, slots = to(c["table"]), to(c["free_blocks"]), to(c["slots"])
    out = gr.gr_page_update(to(c["lengths"]), to(c["new_lengths"]), table, stack, to(np.array([c["free_count"]], np.int32)), c["block"], slots, **more)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (*out, slots, table, stack)]


def _check(got, c):
    lengths, count, starts, status, slots, table, stack = page_update(**c)
    assert np.array_equal(got[0], lengths) and int(got[1][0]) == count and np.array_equal(got[2], starts) and np.array_equal(got[3], status)
    assert np.array_equal(got[4], slots) and np.array_equal(got[5], table)
    assert np.array_equal(got[6][:count], stack)
    assert np.array_equal(got[6][max(count, c["free_count"]):], c["free_blocks"][max(count, c["free_count"]):])      # behind the stack: as it was


@pytest.mark.parametrize("R,block,width,grow,shrink,spare", [(1, 16, 4, 1, 0.0, 9), (1, 1, 9, 3, 0.0, 9), (7, 16, 20, 5, 0.3, 50), (64, 13, 30, 40, 0.2, 400), (1000, 16, 40, 9, 0.5, 1000),
                                                            (1025, 32, 12, 1, 0.0, 1100), (300, 128, 20, 900, 0.1, 3000), (5, 7, 4000, 20000, 0.0, 20000), (8192, 16, 10, 17, 0.1, 9000),
                                                            (64, 16, 20, 30, 0.1, 40), (300, 8, 30, 60, 0.3, 0), (6000, 4, 8, 9, 0.4, 100)])
def test_pages(torch, gr, R, block, width, grow, shrink, spare):
    """With room and without: the last cases run out of blocks half way."""
    rng = np.random.default_rng(R + block)
    lengths = rng.integers(0, max(1, width * block - grow), R)
    new = np.where(rng.random(R) < shrink, lengths * rng.choice([0.0, 0.5, 0.9], R), np.minimum(lengths + rng.integers(0, grow + 1, R), width * block)).astype(int)
    c = _inputs(rng, lengths, new, block, width, spare, int(np.maximum(new - lengths, 0).sum()) + 3)
    _check(_run(torch, gr, c), c)


def test_pages_at_their_edges(torch, gr):
    """Whole blocks, nothing new, everything back, no request that fits, lengths that are no lengths, too few slots, entries that are no blocks, no slots at all."""
    rng = np.random.default_rng(3)
    cases = [([16, 32, 0, 15, 17], [17, 32, 16, 16, 17], 4, 9, 40), ([5, 64, 33], [0, 0, 0], 4, 0, 2), ([0, 0], [64, 64], 4, 3, 200), ([10, -1, 70, 10, 10], [20, 5, 3, 65, -2], 4, 9, 90),
             ([1, 1, 1, 40], [5, 9, 2, 10], 4, 9, 7), ([16, 16], [16, 10], 4, 2, 0), ([3, 40], [20, 8], 4, 0, 30)]
    for lengths, new, width, spare, slots in cases:
        c = _inputs(rng, lengths, new, 16, width, spare, slots)
        _check(_run(torch, gr, c), c)
    c = _inputs(rng, [20, 20], [40, 25], 16, 4, 5, 40)
    c["table"][1, 1] = -1
    got = _run(torch, gr, c)
    _check(got, c)
    assert (got[4][20:25] == -1).all()


def test_pages_far_behind_32_bits(torch, gr):
    """Slots are 64-bit numbers: block 2^30 - 1 of 64 tokens."""
    c = _inputs(np.random.default_rng(0), [3], [100], 64, 4, 0, 120)
    c["table"][0, 0] = 5
    c["free_blocks"] = np.array([2 ** 30 - 1, -9], np.int32); c["free_count"] = 1
    got = _run(torch, gr, c)
    _check(got, c)
    assert got[4][61] == (2 ** 30 - 1) * 64 and got[4].max() == (2 ** 30 - 1) * 64 + 35


def test_pages_on_another_stream_and_in_a_graph(torch, gr):
    """A step captured once; the lengths change between the replays, as in a decoding loop with two sets of lengths and counts."""
    rng = np.random.default_rng(8)
    R, block, width = 12, 16, 30
    c = _inputs(rng, rng.integers(1, 100, R), [0] * R, block, width, 200, 64)
    to = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()  # noqa: E731
    old, new, table, stack, slots = (to(c[k]) for k in ("lengths", "new_lengths", "table", "free_blocks", "slots"))
    count = torch.tensor([200], dtype=torch.int32, device="cuda")
    out = tuple(torch.zeros(n, dtype=torch.int32, device="cuda") for n in (R, 1, R + 1, R))
    new.copy_(old)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    gr.gr_page_update(old, new, table, stack, count, block, slots, out, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(out[0], old) and int(out[2].max()) == 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gr.gr_page_update(old, new, table, stack, count, block, slots, out)
        old.copy_(out[0])
        count.copy_(out[1])
    for turn in range(6):
        c.update(lengths=old.cpu().numpy(), table=table.cpu().numpy(), free_blocks=stack.cpu().numpy(), free_count=int(count), slots=slots.cpu().numpy())
        c["new_lengths"] = np.clip(c["lengths"] + rng.integers(-20, 6, R), 0, width * block).astype(np.int32)
        new.copy_(torch.from_numpy(c["new_lengths"]))
        graph.replay()
        torch.cuda.synchronize()
        _check([x.cpu().numpy() for x in (*out, slots, table, stack)], c)


def test_refusals(torch, gr):
    z = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    good = dict(lengths=z(3), new_lengths=z(3), table=z(3, 4), free_blocks=z(5), free_count=z(1), block=16, slots=torch.zeros(4, dtype=torch.int64, device="cuda"))
    gr.gr_page_update(**good)
    for change, kind in [(dict(block=0), gr.GrError), (dict(lengths=z(8193), new_lengths=z(8193), table=z(8193, 1)), gr.GrError), (dict(new_lengths=z(2)), TypeError), (dict(table=z(4, 3).t()), TypeError),
                         (dict(slots=z(4)), TypeError), (dict(free_count=z(2)), TypeError), (dict(lengths=z(3).cpu()), TypeError), (dict(out=(good["lengths"], z(1), z(4), z(3))), gr.GrError),
                         (dict(out=(z(3), good["free_count"], z(4), z(3))), gr.GrError), (dict(table=z(3, 0)), gr.GrError), (dict(free_blocks=z(0)), gr.GrError)]:
        with pytest.raises(kind):
            gr.gr_page_update(**{**good, **change})


def test_a_beam_search_over_pages(torch, gr):
    """The operators as a decoder uses them: pages for every beam's next token, its state written to its slot, the selection, the states behind their parents.  The state of a
    token is the token, so at the end every beam's pages hold the very tokens that a search on the host finds."""
    S, K, V, block, width, steps, prompt, eos = 3, 4, 500, 4, 8, 11, 6, 3
    rng = np.random.default_rng(6)
    model = (3.0 * rng.standard_normal((V, V))).astype(np.float32)              # the next token's logits by the last token alone
    model[:, eos] -= 4.0
    device_model = torch.from_numpy(model).cuda()
    begin = rng.integers(5, V, S)
    h = gr.gr_create(S * K, V)
    try:
        pool = S * K * width
        state = torch.full((1, pool, 1, block, 1), -1, dtype=torch.int32, device="cuda")
        table = torch.full((S * K, width), -1, dtype=torch.int32, device="cuda")
        stack = torch.from_numpy(rng.permutation(pool).astype(np.int32)).cuda()
        sets = [[torch.zeros(S * K, dtype=torch.int32, device="cuda"), torch.tensor([pool], dtype=torch.int32, device="cuda")] for _ in range(2)]
        starts, status = torch.zeros(S * K + 1, dtype=torch.int32, device="cuda"), torch.zeros(S * K, dtype=torch.int32, device="cuda")
        slots = torch.full((S * K * prompt,), -1, dtype=torch.int64, device="cuda")

        def grow(turn, by):
            (old, count), (new, left) = sets[turn % 2], sets[1 - turn % 2]
            gr.gr_page_update(old, old + by, table, stack, count, block, slots, (new, left, starts, status))
            assert int(status.abs().sum()) == 0
            return slots[:S * K * by]
        # the prompt: the same tokens in every beam's own pages
        flat = state.view(-1)
        flat[grow(0, prompt)] = torch.from_numpy(np.repeat(begin, K)).cuda().int().repeat_interleave(prompt)
        last = torch.from_numpy(np.repeat(begin[:, None], K, 1)).cuda()
        scores = torch.full((S, K), -np.inf, device="cuda"); scores[:, 0] = 0.0
        finished = torch.zeros((S, K), dtype=torch.uint8, device="cuda")
        host = [([(0.0, 0)] + [(-np.inf, 0)] * (K - 1), [[int(begin[s])] * prompt for _ in range(K)]) for s in range(S)]
        host_done = np.zeros((S, K), np.uint8)
        for step in range(steps):
            before = scores.cpu().numpy()
            scores, parent, token, finished, st = gr.gr_beam_select(h, device_model[last], scores, K, finished=finished, eos=eos)
            assert int(st.abs().sum()) == 0
            lengths = sets[(1 + step) % 2][0]
            gr.gr_beam_reorder(state, parent, None, lengths[::K].contiguous(), table)
            flat[grow(1 + step, 1)] = token.view(-1)
            last = token.long()
            for s in range(S):
                found = beam_select(np.stack([model[r[-1]] for r in host[s][1]]), before[s], K, finished=host_done[s], eos=eos)
                host[s] = ([(x[0], 0) for x in found], [host[s][1][x[1]] + [x[2]] for x in found])
                host_done[s] = [x[2] == eos for x in found]
        rows, pages = state.view(pool, block).cpu().numpy(), table.cpu().numpy()
        for s in range(S):
            for b in range(K):
                held = rows[pages[s * K + b]].reshape(-1)[:prompt + steps]
                assert held.tolist() == host[s][1][b], (s, b)
            assert np.allclose(scores[s].cpu().numpy(), [x[0] for x in host[s][0]], rtol=2.0 ** -22, atol=1e-9)
        # the sequences end: everything goes back
        (old, count), (new, left) = sets[(1 + steps) % 2], sets[steps % 2]
        gr.gr_page_update(old, torch.zeros_like(old), table, stack, count, block, slots, (new, left, starts, status))
        assert int(left) == pool and sorted(stack.cpu().tolist()) == list(range(pool))
    finally:
        gr.gr_destroy(h)


@pytest.mark.parametrize("R", [6, 700, 8000])
@pytest.mark.parametrize("small", [0, 2, 5])
def test_more_new_tokens_than_32_bits_count(torch, gr, R, small):
    """Requests that ask for 2^30 tokens each: those before the first of them are granted, and no sum wraps round to room."""
    new = np.full(R, 2 ** 30 - 1, np.int32)
    new[:small] = 3
    new[R - 1] = 2
    stack = np.arange(5000, dtype=np.int32)
    c = dict(lengths=np.zeros(R, np.int32), new_lengths=new, table=np.full((R, 1024), -1, np.int32), free_blocks=stack, free_count=5000, block=2 ** 20, slots=np.full(40, -7, np.int64))
    _check(_run(torch, gr, c), c)


@pytest.mark.parametrize("R", [3000, 5000])
def test_many_requests_in_a_graph(torch, gr, R):
    rng = np.random.default_rng(R)
    c = _inputs(rng, rng.integers(1, 100, R), [0] * R, 16, 8, 2 * R, 3 * R)
    c["new_lengths"] = np.clip(c["lengths"] + rng.integers(-20, 4, R), 0, 128).astype(np.int32)
    to = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()  # noqa: E731
    start = {k: to(c[k]) for k in ("table", "free_blocks", "slots")}
    live = {k: v.clone() for k, v in start.items()}
    old, new, count = to(c["lengths"]), to(c["new_lengths"]), torch.tensor([c["free_count"]], dtype=torch.int32, device="cuda")
    out = tuple(torch.zeros(n, dtype=torch.int32, device="cuda") for n in (R, 1, R + 1, R))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gr.gr_page_update(old, new, live["table"], live["free_blocks"], count, 16, live["slots"], out)
    for _ in range(3):
        for k, v in start.items():
            live[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        _check([x.cpu().numpy() for x in (*out, live["slots"], live["table"], live["free_blocks"])], c)
