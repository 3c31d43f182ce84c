"""Drafts drawn on the GPU against a draw in 64 bits, row by row.  A draw may differ only where its uniform lies within 1e-12 of a border of the CDF: both
sides add float64 masses, which are off by a few 1e-16 each, 131072 of them by 3e-11 of the last digit's order at most and by 1e-14 in practice."""
import numpy as np
import pytest

from beside_forms import ROW_BAD, ROW_OK, draft_support, draw, softmax_mass

pytestmark = pytest.mark.gpu
BORDER = 1e-12
LAST = np.float32(1.0 - 2.0 ** -24)


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


@pytest.fixture(scope="module")
def gr():
    from paper_2511_15898_amd import binding
    return binding


def _logits(seed, B, V, kind="heavy"):
    rng = np.random.default_rng(seed)
    x = 4.0 * rng.gumbel(size=(B, V)) if kind == "heavy" else 2.0 * rng.standard_normal((B, V))
    return x.astype(np.float32)


def _uniforms(seed, B, n):
    u = np.random.default_rng(seed).random((B, n)).astype(np.float32)
    u = np.minimum(u, LAST)
    u[0, 0], u[-1, -1] = 0.0, LAST
    return u


def _wide(torch, x, dtype, pad, offset):
    """x on the GPU in rows that lie `pad` entries further apart than they are long and begin `offset` entries into an allocation."""
    B, V = x.shape
    room = torch.full((B * (V + pad) + offset + 8,), 7.0, dtype=dtype, device="cuda")
    view = room[offset:offset + B * (V + pad)].view(B, V + pad)[:, :V]
    view.copy_(torch.from_numpy(x))
    return view


def _check(got, x, k, uniforms, mass_of):
    for b in range(x.shape[0]):
        ids = draft_support(x[b], k)
        for j, (token, near) in enumerate(draw(mass_of(x[b], ids, b), ids, uniforms[b])):
            assert got[b, j] == token or near < BORDER, (b, j, int(got[b, j]), token, near)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("B,V,n,k,pad,offset", [(1, 1, 1, 0, 0, 0), (2, 2, 3, 1, 3, 1), (3, 7, 16, 0, 0, 0), (2, 255, 4, 64, 1, 3), (2, 256, 2, 256, 0, 0), (3, 257, 5, 0, 0, 1),
                                            (2, 300, 4, 256, 5, 7), (5, 1000, 4, 32, 0, 0), (3, 4097, 8, 128, 7, 2), (4, 8192, 2, 65, 0, 0), (2, 20001, 16, 0, 3, 5),
                                            (1, 50021, 4, 1, 0, 1), (1, 128256, 4, 64, 0, 0), (2, 128256, 8, 0, 64, 0), (300, 513, 2, 9, 0, 0)])
def test_drafts_of_logits(torch, gr, dtype, B, V, n, k, pad, offset):
    rng = np.random.default_rng(V + n)
    x = _wide(torch, _logits(B + V, B, V), getattr(torch, dtype), pad, offset)
    T = rng.uniform(0.5, 1.5, B).astype(np.float32)
    u = _uniforms(V, B, n)
    h = gr.gr_create(B, V, max_n=n)
    try:
        drafts, status = gr.gr_draft_logits(h, x, torch.from_numpy(T).cuda(), n, k, torch.from_numpy(u).cuda())
        again, _ = gr.gr_draft_logits(h, x, torch.from_numpy(T).cuda(), n, k, torch.from_numpy(u).cuda())
        assert torch.equal(drafts, again)
        assert int(status.abs().sum()) == ROW_OK
        ref = x.float().cpu().numpy()
        _check(drafts.cpu().numpy(), ref, k, u, lambda row, ids, b: softmax_mass(row[ids], float(T[b])))
    finally:
        gr.gr_destroy(h)


@pytest.mark.parametrize("B,V,n,k,pad,offset", [(1, 1, 2, 0, 0, 0), (2, 5, 16, 3, 0, 1), (4, 256, 4, 0, 0, 0), (2, 257, 4, 0, 3, 1), (3, 3001, 4, 200, 1, 2), (2, 40000, 8, 0, 0, 3),
                                            (1, 128256, 16, 128, 0, 0)])
def test_drafts_of_probabilities(torch, gr, B, V, n, k, pad, offset):
    x = _logits(B * V, B, V, "mild").astype(np.float64)
    q = np.exp(x - x.max(1, keepdims=True))
    if V > 4:
        q[:, :: 3] = 0.0                                            # tokens of no mass are never drawn
    q = (q / q.sum(1, keepdims=True)).astype(np.float32)
    u = _uniforms(V + 1, B, n)
    h = gr.gr_create(B, V, max_n=n)
    try:
        drafts, status = gr.gr_draft(h, _wide(torch, q, torch.float32, pad, offset), n, k, torch.from_numpy(u).cuda())
        drafts = drafts.cpu().numpy()
        assert int(status.abs().sum()) == ROW_OK
        _check(drafts, q, k, u, lambda row, ids, b: row[ids].astype(np.float64))
        assert (np.take_along_axis(q, drafts, 1) > 0).all()
    finally:
        gr.gr_destroy(h)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V", [40, 257, 9000, 70001])
@pytest.mark.parametrize("k", [1, 7, 200, 0])
def test_equal_entries_masks_and_lowest_values(torch, gr, dtype, V, k):
    """Rows of equal entries (the lowest ids are the top k), of few unmasked ones, of the type's lowest value in masked places, far below one token."""
    t = getattr(torch, dtype)
    lowest = float(torch.finfo(t).min)
    rows = np.zeros((6, V), np.float32)
    rows[1] = -np.inf; rows[1, V // 2] = -3.0                          # one token
    rows[2] = lowest; rows[2, 3::11] = 1.0
    rows[3] = lowest                                                # every entry the lowest: as good as any other row of equal ones
    rows[4] = -np.inf; rows[4, 1::5] = np.arange(len(rows[4, 1::5])) % 3
    rows[5] = -30.0; rows[5, V - 1] = 5.0
    x = torch.from_numpy(rows).cuda().to(t)
    u = np.random.default_rng(V).random((6, 9)).astype(np.float32)
    h = gr.gr_create(6, V, max_n=9)
    try:
        drafts, status = gr.gr_draft_logits(h, x, torch.ones(6, device="cuda"), 9, k, torch.from_numpy(u).cuda())
        assert int(status.abs().sum()) == ROW_OK
        _check(drafts.cpu().numpy(), x.float().cpu().numpy(), k, u, lambda row, ids, b: softmax_mass(row[ids], 1.0))
    finally:
        gr.gr_destroy(h)


@pytest.mark.parametrize("V,k", [(50, 8), (50, 0), (9001, 8), (9001, 0)])
def test_bad_rows(torch, gr, V, k):
    """NaN, +inf, all masked, a bad temperature: status and -1, and the rows beside them as ever."""
    x = _logits(5, 9, V)
    for b, bad in enumerate([np.nan, np.inf, None]):
        if bad is None:
            x[b] = -np.inf
        else:
            x[b, V - 1 - b] = bad
    T = np.ones(9, np.float32)
    T[3:7] = [0.0, -1.0, np.nan, np.inf]
    u = _uniforms(3, 9, 3)
    h = gr.gr_create(9, V, max_n=3)
    try:
        drafts, status = gr.gr_draft_logits(h, torch.from_numpy(x).cuda(), torch.from_numpy(T).cuda(), 3, k, torch.from_numpy(u).cuda())
        drafts, status = drafts.cpu().numpy(), status.cpu().numpy()
        assert (status[:7] == ROW_BAD).all() and (drafts[:7] == -1).all() and (status[7:] == ROW_OK).all()
        _check(drafts[7:], x[7:], k, u[7:], lambda row, ids, b: softmax_mass(row[ids], 1.0))
        q = np.full((5, V), 1.0 / V, np.float32)
        q[0, 0] = np.nan; q[1, V - 1] = -1e-6; q[2] = 0.0; q[3] *= 1.01
        drafts, status = gr.gr_draft(h, torch.from_numpy(q).cuda(), 3, k, torch.from_numpy(u[:5].copy()).cuda())
        assert status.tolist() == [ROW_BAD] * 4 + [ROW_OK] and (drafts[:4] == -1).all() and (drafts[4] >= 0).all()
    finally:
        gr.gr_destroy(h)


@pytest.mark.parametrize("tail_mass", [0.0, 1e-3, 0.3])
def test_drafts_lie_in_the_support_that_the_solver_takes(torch, gr, tail_mass):
    from paper_2511_15898_amd import workloads as W
    wl = W.llm_shaped(B=24, V=5000, n=6, k=50, seed_sub=77)
    p, q = (torch.from_numpy(v).cuda() for v in (wl.p, wl.q))
    u = torch.from_numpy(_uniforms(8, 24, 6)).cuda()
    h = gr.gr_create(24, 5000, max_n=6, tail_mass=tail_mass)
    try:
        drafts, status = gr.gr_draft(h, q, 6, 50, u)
        acc, st, token, accepted = gr.gr_solve_verify(h, p, q, 6, 50, 1e-4, drafts, torch.rand(24, device="cuda"))
        assert int(status.abs().sum()) == 0 and bool((token >= 0).all())
        policy = gr.gr_policy_export(h, 24, "cuda")
        for b in range(24):
            ids = policy["order"][b, :int(policy["support"][b])].cpu().numpy()
            mass = np.sort(ids)
            for j, (want, near) in enumerate(draw(wl.q[b, mass].astype(np.float64), mass, u[b].cpu().numpy())):
                assert int(drafts[b, j]) == want or near < BORDER
    finally:
        gr.gr_destroy(h)


def test_drafts_then_verification_of_logits_follow_the_target(torch, gr):
    """The two steps as they are used.  One pair of rows, many times: the emitted tokens are spread as the target says (4.5 standard deviations)."""
    from paper_2511_15898_amd import workloads as W
    B, V, n = 4096, 64, 3
    rng = np.random.default_rng(11)
    t = (2.0 * rng.standard_normal(V)).astype(np.float32)
    d = (t + rng.standard_normal(V)).astype(np.float32)
    tl, dl = (torch.from_numpy(np.repeat(v[None], B, 0)).cuda() for v in (t, d))
    T = torch.ones(B, device="cuda")
    gen = torch.Generator(device="cuda"); gen.manual_seed(5)
    h = gr.gr_create(B, V, max_n=n)
    try:
        drafts, _ = gr.gr_draft_logits(h, dl, T, n, 16, torch.rand((B, n), device="cuda", generator=gen))
        acc, st, token, accepted = gr.gr_solve_logits_verify(h, tl, dl, T, n, 16, 1e-6, drafts, torch.rand(B, device="cuda", generator=gen))
        assert int(st.abs().sum()) == 0
        mass = softmax_mass(t, 1.0); mass /= mass.sum()
        seen = np.bincount(token.cpu().numpy(), minlength=V) / B
        assert (np.abs(seen - mass) <= 4.5 * np.sqrt(mass * (1 - mass) / B) + 1e-9).all()
        assert abs(float(accepted.float().mean()) - float(acc[0])) < 4.5 * 0.5 / np.sqrt(B)
    finally:
        gr.gr_destroy(h)


def test_a_tree_of_paths_drawn_here_is_walked(torch, gr):
    """Paths drawn level by level, each from its own row, then the walk: every draft lies in its support, so no token is -1."""
    S, K, L, V, k = 5, 3, 3, 2000, 40
    gen = torch.Generator(device="cuda"); gen.manual_seed(2)
    target = torch.empty((S, 1, 1, V), device="cuda").exponential_(generator=gen).log_().mul_(-4.0)
    p = torch.softmax(target, -1).expand(S, K, L, V).contiguous()
    q = torch.softmax(0.8 * target + torch.randn((S, 1, 1, V), device="cuda", generator=gen), -1).expand(S, K, L, V).contiguous()
    h = gr.gr_create(S * K, V, max_n=max(K, 3))
    try:
        paths = torch.empty((S, K, L), dtype=torch.int32, device="cuda")
        paths[:, :, 0], _ = gr.gr_draft(h, q[:, 0, 0], K, k, torch.rand((S, K), device="cuda", generator=gen))          # one row, K drafts
        for l in range(1, L):
            one, status = gr.gr_draft(h, q[:, :, l].reshape(S * K, V), 1, k, torch.rand((S * K, 1), device="cuda", generator=gen))
            paths[:, :, l] = one.view(S, K)
            assert int(status.abs().sum()) == 0
        u = np.random.default_rng(4).random((S, L)).astype(np.float32)
        tokens, length, accepted, fallbacks = gr.gr_tree_walk(h, p, q, paths.cpu().numpy(), u, k, 1e-5)
        assert (length >= 1).all() and all((tokens[s, :length[s]] >= 0).all() for s in range(S))
    finally:
        gr.gr_destroy(h)


@pytest.mark.parametrize("V,k", [(3000, 20), (3000, 0)])
def test_drafts_on_another_stream_and_in_a_graph(torch, gr, V, k):
    x = torch.from_numpy(_logits(9, 6, V)).cuda()
    T, u = torch.ones(6, device="cuda"), torch.from_numpy(_uniforms(2, 6, 4)).cuda()
    h = gr.gr_create(6, V)
    try:
        want, _ = gr.gr_draft_logits(h, x, T, 4, k, u)
        want = want.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got, _ = gr.gr_draft_logits(h, x, T, 4, k, u, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)
        drafts, status = torch.empty_like(want), torch.empty(6, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            gr.gr_draft_logits(h, x, T, 4, k, u, drafts, status)
        for turn in range(4):
            x.copy_(torch.from_numpy(_logits(20 + turn, 6, V)))
            drafts.fill_(-5)
            graph.replay()
            torch.cuda.synchronize()
            eager, _ = gr.gr_draft_logits(h, x, T, 4, k, u)
            assert torch.equal(eager, drafts), turn
    finally:
        gr.gr_destroy(h)


def test_drafts_leave_no_policy_and_refuse_what_they_cannot_do(torch, gr):
    h, cut = gr.gr_create(4, 1000, max_n=4), gr.gr_create(4, 1000, max_n=4, tail_mass=0.1)
    x, u, T = torch.zeros((4, 1000), device="cuda"), torch.rand((4, 2), device="cuda"), torch.ones(4, device="cuda")
    q = torch.full((4, 1000), 1e-3, device="cuda")
    try:
        gr.gr_solve(h, q, q, 2, 10, 1e-4)
        gr.gr_draft(h, q, 2, 10, u)
        with pytest.raises(gr.GrError) as e:
            gr.gr_verify(h, torch.zeros((4, 2), dtype=torch.int32, device="cuda"), T)
        assert e.value.code == gr.GR_ESTATE
        for call, code in [(lambda: gr.gr_draft(h, q, 2, 257, u), gr.GR_EUNSUPPORTED), (lambda: gr.gr_draft_logits(cut, x, T, 2, 10, u), gr.GR_EUNSUPPORTED),
                           (lambda: gr.gr_draft(cut, q, 2, 0, u), gr.GR_EUNSUPPORTED), (lambda: gr.gr_draft(h, q, 5, 10, torch.rand((4, 5), device="cuda")), gr.GR_EINVAL),
                           (lambda: gr.gr_draft(h, q.new_zeros((5, 1000)), 1, 10, q.new_zeros((5, 1))), gr.GR_EINVAL)]:
            with pytest.raises(gr.GrError) as e:
                call()
            assert e.value.code == code
        for call in [lambda: gr.gr_draft(h, q.cpu(), 2, 10, u), lambda: gr.gr_draft(h, q.double(), 2, 10, u), lambda: gr.gr_draft(h, q, 3, 10, u), lambda: gr.gr_draft(h, q.t(), 2, 10, u),
                     lambda: gr.gr_draft(h, q[:1].expand(4, 1000), 2, 10, u), lambda: gr.gr_draft_logits(h, x, T[:3], 2, 10, u)]:
            with pytest.raises(TypeError):
                call()
    finally:
        gr.gr_destroy(h); gr.gr_destroy(cut)


# Rows at which the bookkeeping of a pass over a row is at its limits: few or many, short or long, so that they are read by one workgroup of either size or in slices.
SHAPES = [(2, 9001), (1, 49152), (2, 70001), (260, 6000), (515, 5003)]


@pytest.mark.parametrize("B,V", SHAPES + [(1, 300007), (130, 100003)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("k", [3, 256])
@pytest.mark.parametrize("kind", ["rising", "steps", "equal"])
def test_rows_that_keep_more_candidates_than_there_is_room_for(torch, gr, B, V, dtype, k, kind):
    """Rows that rise (every later entry beats the threshold of the first), that rise in steps, and rows of equal entries."""
    i = torch.arange(V, device="cuda", dtype=torch.float32)
    row = {"rising": i * (8.0 / V), "steps": torch.floor(i / 700) % 64, "equal": torch.zeros(V, device="cuda")}[kind]
    x = row.to(getattr(torch, dtype))[None].repeat(B, 1)
    x[B - 1] = x[B - 1].flip(0)                                      # and one that falls
    u = _uniforms(V, B, 4)
    h = gr.gr_create(B, V, max_n=4)
    try:
        drafts, status = gr.gr_draft_logits(h, x, torch.ones(B, device="cuda"), 4, k, torch.from_numpy(u).cuda())
        assert int(status.abs().sum()) == ROW_OK
        drafts, x = drafts.cpu().numpy(), x.float().cpu().numpy()
        some = sorted({0, B // 2, B - 1})
        _check(drafts[some], x[some], k, u[some], lambda row, ids, b: softmax_mass(row[ids], 1.0))
    finally:
        gr.gr_destroy(h)


@pytest.mark.parametrize("B", [1, 300, 600])
@pytest.mark.parametrize("few", [1, 130, 200, 255, 256, 257])
@pytest.mark.parametrize("first", [0, 1283, 5 * 256])
def test_few_unmasked_tokens_close_together(torch, gr, B, few, first):
    """All but `few` entries are masked, and those lie one to a 16-byte chunk in one stretch: fewer than k of 256, or as many, in the hands of few threads."""
    V, k = 20000, 256
    x = torch.full((B, V), -float("inf"), device="cuda")
    at = first + 4 * torch.arange(few, device="cuda")
    x[:, at] = torch.randn((B, few), device="cuda", generator=torch.Generator(device="cuda").manual_seed(few))
    u = _uniforms(few, B, 3)
    h = gr.gr_create(B, V, max_n=3)
    try:
        drafts, status = gr.gr_draft_logits(h, x, torch.ones(B, device="cuda"), 3, k, torch.from_numpy(u).cuda())
        assert int(status.abs().sum()) == ROW_OK
        some = sorted({0, B // 2, B - 1})
        _check(drafts[some].cpu().numpy(), x[some].cpu().numpy(), k, u[some], lambda row, ids, b: softmax_mass(row[ids], 1.0))
    finally:
        gr.gr_destroy(h)


@pytest.mark.parametrize("probs", [True, False])
@pytest.mark.parametrize("B,V,n", [(1, 32768, 16), (2, 65537, 5), (1, 300007, 16), (192, 20011, 3), (256, 5000, 16), (257, 5000, 16), (700, 1025, 2)])
def test_whole_rows_few_and_many_short_and_long(torch, gr, probs, B, V, n):
    x = _logits(V + B, B, V, "mild")
    if probs:
        e = np.exp(x.astype(np.float64))
        x = (e / e.sum(1, keepdims=True)).astype(np.float32)
    u = _uniforms(B, B, n)
    h = gr.gr_create(B, V, max_n=n)
    try:
        cx, cu = torch.from_numpy(x).cuda(), torch.from_numpy(u).cuda()
        drafts, status = gr.gr_draft(h, cx, n, 0, cu) if probs else gr.gr_draft_logits(h, cx, torch.ones(B, device="cuda"), n, 0, cu)
        assert int(status.abs().sum()) == ROW_OK
        some = sorted({0, B // 3, B - 1})
        _check(drafts[some].cpu().numpy(), x[some], 0, u[some],
               (lambda row, ids, b: row[ids].astype(np.float64)) if probs else (lambda row, ids, b: softmax_mass(row[ids], 1.0)))
    finally:
        gr.gr_destroy(h)


@pytest.mark.parametrize("kind,tail_mass", [("float32", 0.0), ("bfloat16", 0.0), ("probs", 0.0), ("probs", 0.2)])
@pytest.mark.parametrize("V", [900, 20011, 100003])
def test_draws_do_not_depend_on_the_rows_beside(torch, gr, kind, tail_mass, V):
    """The same rows alone, in a batch that occupies half the chip, the whole of it, and more: other kernels, the same draws."""
    gen = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((600, V), device="cuda", generator=gen) * 3
    x = torch.softmax(x, 1) if kind == "probs" else x.to(getattr(torch, kind))
    u = torch.rand((600, 7), device="cuda", generator=gen)
    T = torch.rand(600, device="cuda", generator=gen) + 0.5
    h = gr.gr_create(600, V, tail_mass=tail_mass)
    try:
        for k in (1, 40, 256) if tail_mass else (1, 40, 256, 0):
            draw = (lambda n: gr.gr_draft(h, x[:n], 7, k, u[:n])) if kind == "probs" else (lambda n: gr.gr_draft_logits(h, x[:n], T[:n], 7, k, u[:n]))
            drafts, status = draw(600)
            assert int(status.abs().sum()) == ROW_OK
            for n in (2, 130, 200, 256, 300, 512):
                some, status = draw(n)
                assert torch.equal(some, drafts[:n]) and int(status.abs().sum()) == ROW_OK, (k, n)
    finally:
        gr.gr_destroy(h)
