"""Rows, temperatures and scores at the ends of what the calls accept, drafts and beam selections against the plain forms in 64 bits.  Scores and the order of beams are held to what
test_gpu_beam.py derives for them, draws to the border of test_gpu_draft.py: sums of float64 exponentials whose relative error is 1.8e-14 at most (the rounding of a
polynomial's last step included), so borders lie within 4e-14 of the total of where they belong, and 1e-12 leaves room."""
import numpy as np
import pytest

from beside_forms import ROW_BAD, ROW_OK, beam_select, draft_support, draw, softmax_mass
from test_gpu_beam import _check as check_beams, _select as select

pytestmark = pytest.mark.gpu
BORDER = 1e-12


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


@pytest.fixture(scope="module")
def gr():
    from paper_2511_15898_amd import binding
    return binding


def _drafts(torch, gr, x, k, uniforms, T=None):
    """Drafts of x [B, V] on the GPU (probabilities if T is None), as arrays; the call made twice."""
    B, V = x.shape
    n = uniforms.shape[1]
    h = gr.gr_create(B, V, max_n=n)
    u = torch.from_numpy(uniforms).cuda()
    try:
        call = (lambda: gr.gr_draft(h, x, n, k, u)) if T is None else (lambda: gr.gr_draft_logits(h, x, torch.from_numpy(T).cuda(), n, k, u))
        drafts, status = call()
        again, _ = call()
        assert torch.equal(drafts, again)
        return drafts.cpu().numpy(), status.cpu().numpy()
    finally:
        gr.gr_destroy(h)


def _check_drafts(drafts, rows, k, uniforms, T=None, some=None):
    for b in range(len(rows)) if some is None else some:
        ids = draft_support(rows[b], k)
        mass = rows[b, ids].astype(np.float64) if T is None else softmax_mass(rows[b, ids], float(T[b]))
        for j, (token, near) in enumerate(draw(mass, ids, uniforms[b])):
            assert drafts[b, j] == token or near < BORDER, (b, j, int(drafts[b, j]), token, near)


def _uniforms(seed, B, n):
    return np.minimum(np.random.default_rng(seed).random((B, n)).astype(np.float32), np.float32(1.0 - 2.0 ** -24))


@pytest.mark.parametrize("V, many", [(900, 1), (5003, 1), (5003, 8), (40001, 1)])
def test_draws_from_whole_rows_next_to_a_border(torch, gr, V, many):
    """Uniforms that lie between 1.5 and 30 millionths of a millionth of the total from a border of the distribution, which float64 masses tell apart, in rows of heavy tails."""
    rng = np.random.default_rng(V)
    rows, uniforms = [], []
    while len(rows) < 40:
        x = (4.0 * rng.gumbel(size=V)).astype(np.float32)
        cdf = np.cumsum(softmax_mass(x, 1.0).astype(np.longdouble))
        cdf = cdf[:-1] / cdf[-1]
        u = cdf.astype(np.float32)
        far = np.abs(u.astype(np.longdouble) - cdf)
        others = np.minimum(np.diff(cdf, prepend=np.longdouble(-1)), np.diff(cdf, append=np.longdouble(2)))
        near = np.flatnonzero((cdf > 0.05) & (far > 1.5e-12) & (far < 3e-11) & (u < 1) & (others > 1e-10))
        if len(near):
            rows.append(x)
            uniforms.append([u[near[i % len(near)]] for i in range(6)])
    rows, u = np.tile(np.stack(rows), (many, 1)), np.tile(np.array(uniforms, np.float32), (many, 1))
    T = np.ones(len(rows), np.float32)
    drafts, status = _drafts(torch, gr, torch.from_numpy(rows).cuda(), 0, u, T)
    assert (status == ROW_OK).all()
    _check_drafts(drafts, rows, 0, u, T, some=range(40))
    assert many == 1 or (drafts.reshape(many, 40, 6) == drafts[:40]).all()


@pytest.mark.parametrize("T", [7.0e35, 1.0e36, 1.0e37, 2.9e38])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [1003, 40001])
def test_temperatures_next_to_the_largest_float(torch, gr, T, dtype, V):
    """Nothing lies below the lowest entry that such a temperature sets apart, but masked entries, and the places beside a row that begins at no 16-byte boundary, still count nothing."""
    S, K, M = 3, 3, 6
    rng = np.random.default_rng(V)
    x = np.minimum(0.4e36 * rng.gumbel(size=(S, K, V)), 9e36).astype(np.float32)
    x[1] = (x[1] * np.float32(1e-36)).astype(np.float32)                     # ordinary logits: as good as equal
    x[2, :, 3::4] = -np.inf
    x = torch.from_numpy(x).cuda().to(getattr(torch, dtype))
    rows, temps = x.float().cpu().numpy(), np.full(S, T, np.float32)
    scores = rng.uniform(-9.0, -8.0, (S, K)).astype(np.float32)
    check_beams(select(torch, gr, x, scores, M, temps), rows, scores, M, temps)
    u, per_row = _uniforms(V, S * K, 9), np.full(S * K, T, np.float32)
    for k in (0, 100):
        drafts, status = _drafts(torch, gr, x.view(S * K, V), k, u, per_row)
        assert (status == ROW_OK).all()
        _check_drafts(drafts, rows.reshape(S * K, V), k, u, per_row)


@pytest.mark.parametrize("top, T", [(100.0, 1.0e-8), (20.0, 2.48e-9), (10.0, 1.2e-9), (-3.0, 3.0e-10), (1.0, 1.5e-10), (1.0, 1.4e-10)])
def test_temperatures_of_a_thousandth_of_the_last_digit(torch, gr, top, T):
    """The row's largest entry is the float behind the largest one so far, and hundreds of temperatures above it: the sum is brought to it although nothing lies between the two.
    1024 rows, so that each is one workgroup's and the two lie in the hands of one wave, tiles of 4096 entries apart."""
    S, K, V, M = 64, 16, 9000, 3
    x = torch.full((S, K, V), top - 5.0, device="cuda")
    x[:, :, 5] = top
    x[:, ::2, 5 + 4096] = float(np.nextafter(np.float32(top), np.float32(np.inf)))
    x[:, 1::2, 5 + 8192] = float(np.nextafter(np.float32(top), np.float32(np.inf)))
    scores = np.random.default_rng(0).uniform(-9.0, -1.0, (S, K)).astype(np.float32)
    temps = np.full(S, T, np.float32)
    got = select(torch, gr, x, scores, M, temps)
    some = [0, 17, S - 1]
    check_beams([v[some] for v in got], x[some].cpu().numpy(), scores[some], M, temps[some])
    u, per_row = _uniforms(1, S * K, 3), np.full(S * K, T, np.float32)
    for k in (0, 2):
        drafts, status = _drafts(torch, gr, x.view(S * K, V), k, u, per_row)
        assert (status == ROW_OK).all()
        _check_drafts(drafts, x.view(S * K, V).cpu().numpy(), k, u, per_row, some=[0, 1, S * K - 1])


@pytest.mark.parametrize("B, V", [(6, 50), (6, 1001), (6, 9001), (6, 70001), (6, 200003), (200, 9001), (600, 1003)])
@pytest.mark.parametrize("k", [8, 0])
def test_minus_infinity_is_no_probability(torch, gr, B, V, k):
    """At either end of a row, where what lies beside it in its 16 bytes is not the row's, and in the middle; the other entries sum to 1, so nothing else is wrong with it."""
    q = np.random.default_rng(V).random((B, V))
    at = {0: 0, 1: V - 1, 2: V // 2, 4: 1}
    for b, i in at.items():
        q[b, i] = 0.0
    q = (q / q.sum(1, keepdims=True)).astype(np.float32)
    for b, i in at.items():
        q[b, i] = -np.inf
    u = _uniforms(V, B, 3)
    drafts, status = _drafts(torch, gr, torch.from_numpy(q).cuda(), k, u)
    bad = np.zeros(B, bool)
    bad[list(at)] = True
    assert (status[bad] == ROW_BAD).all() and (drafts[bad] == -1).all() and (status[~bad] == ROW_OK).all()
    _check_drafts(drafts, q, k, u, some=[3, 5, B - 1] if B > 6 else [3, 5])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V, k", [(2, 1), (300, 7), (5001, 40), (20011, 256), (100003, 3)])
def test_zeros_of_either_sign_are_equal_logits(torch, gr, dtype, V, k):
    """What a product with a mask leaves: the lower token comes first, whatever the signs, among the drafts' k largest as among the continuations."""
    B = 4
    rng = np.random.default_rng(V)
    x = np.where(rng.random((B, V)) < 0.5, np.float32(-0.0), np.float32(0.0))
    x[0, 0], x[0, 1] = -0.0, 0.0
    x[1, 5::6] = -2.0
    x[2, 3::50] = 1.0
    t = torch.from_numpy(x).cuda().to(getattr(torch, dtype))
    u, T = _uniforms(V, B, 8), np.ones(B, np.float32)
    drafts, status = _drafts(torch, gr, t, k, u, T)
    assert (status == ROW_OK).all()
    _check_drafts(drafts, x, k, u, T)
    M, scores = min(k, 64), np.array([[-1.0, -1.5, -1.25, -1.0]], np.float32)
    check_beams(select(torch, gr, t[None], scores, M), x[None], scores, M, exact=V * t.element_size() % 16 == 0)


@pytest.mark.parametrize("V, k", [(300, 7), (5001, 256), (5001, 300), (20011, 1000)])
def test_the_solver_takes_the_same_tokens_of_equal_zeros(torch, gr, V, k):
    """gr_solve_logits: the k largest draft logits, ties to the lower token, so that the drafts lie in its support."""
    B = 3
    rng = np.random.default_rng(V + k)
    d = np.where(rng.random((B, V)) < 0.5, np.float32(-0.0), np.float32(0.0))
    d[1, rng.permutation(V)[:k // 2]] = 1.0
    target = rng.standard_normal((B, V)).astype(np.float32)
    to = lambda v: torch.from_numpy(v).cuda()  # noqa: E731
    h = gr.gr_create(B, V, max_k=k, max_n=1)
    try:
        acc, status = gr.gr_solve_logits(h, to(target), to(d), torch.ones(B, device="cuda"), 1, k, 1e-4)
        assert bool((status <= 1).all())                                    # equal logits: the truncation may take more variables than there is room for
        for b in range(B):
            taken = gr.gr_policy_export_row(h, b, k, "cuda")["order"].cpu().numpy()
            assert np.array_equal(np.sort(taken), draft_support(d[b], k)), b
    finally:
        gr.gr_destroy(h)


def test_scores_of_zero_tie_whatever_their_sign(torch, gr):
    """Certain continuations, ended beams at 0 and at -0.0: equal scores, so the lower beam comes first."""
    V, M, eos = 40, 5, 7
    x = torch.full((4, 3, V), -float("inf"), device="cuda")
    x[:, :, 9] = 3.0                                                        # the one token, of probability 1
    scores = np.zeros((4, 3), np.float32)
    scores[2, 1] = scores[3, 0] = -0.0
    finished = np.array([[0, 1, 0], [1, 0, 1], [0, 1, 1], [1, 1, 0]], np.uint8)
    best, parent, token, over, status = select(torch, gr, x, scores, M, finished=finished, eos=eos)
    assert status.tolist() == [0] * 4 and (parent == [[0, 1, 2, -1, -1]] * 4).all() and (best[:, :3] == 0).all()
    assert (token[:, :3] == np.where(finished, eos, 9)).all() and (over[:, :3] == finished).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V, rows", [(50, 6), (9001, 6), (70001, 6), (9001, 600)])
def test_logits_up_to_1e37_and_no_further(torch, gr, dtype, V, rows):
    """One border for drafts of every kind and for beams: entries up to it are as good as others, however many, one above it makes the row bad; the lowest value never does."""
    t = getattr(torch, dtype)
    lowest = float(torch.finfo(t).min)
    x = torch.zeros((rows, V), dtype=t, device="cuda")
    x[0] = 9.5e36
    x[1, V - 2] = 1.1e37
    x[2, 0] = 1.0e38
    x[3, 1::2] = 9.9e36; x[3, ::2] = lowest
    x[4] = lowest; x[4, 3] = 2.0e38
    bad = np.zeros(rows, bool)
    bad[[1, 2, 4]] = True
    u, T = _uniforms(V, rows, 2), np.ones(rows, np.float32)
    plain = x.float().cpu().numpy()
    for k in (8, 0):
        drafts, status = _drafts(torch, gr, x, k, u, T)
        assert (status == np.where(bad, ROW_BAD, ROW_OK)).all() and (drafts[bad] == -1).all(), k
        _check_drafts(drafts, plain, k, u, T, some=[0, 3, 5])
    scores = np.full((rows, 1), -1.0, np.float32)
    got = select(torch, gr, x[:, None], scores, 4)
    assert (got[4] == np.where(bad, ROW_BAD, ROW_OK)).all() and (got[1][bad] == -1).all()
    good = [0, 3, 5]
    check_beams([v[good] for v in got], plain[good, None], scores[good], 4)


def test_scores_and_temperatures_up_to_the_largest_float(torch, gr):
    """Positive and finite is all that is asked of a temperature, finite or -inf of a score."""
    big = float(np.finfo(np.float32).max)
    S, K, V, M = 4, 2, 3001, 6
    x = torch.randn((S, K, V), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    rows = x.cpu().numpy()
    scores = np.array([[big, -1.0], [-big, 3.2e38], [-1.0, -2.0], [-1.0, -2.0]], np.float32)
    T = np.array([1.0, 1.0, big, 3.2e38], np.float32)
    finished = np.zeros((S, K), np.uint8)
    finished[0, 0] = finished[1, 0] = 1
    check_beams(select(torch, gr, x, scores, M, T, finished=finished, eos=5), rows, scores, M, T, finished=finished, eos=5)
    u, per_row = _uniforms(3, S * K, 4), np.repeat(T, K)
    for B in (S * K, 600):
        y, v, t = x.view(S * K, V).repeat(B // (S * K), 1), np.tile(u, (B // (S * K), 1)), np.tile(per_row, B // (S * K))
        for k in (0, 30):
            drafts, status = _drafts(torch, gr, y, k, v, t)
            assert (status == ROW_OK).all()
            _check_drafts(drafts, y.cpu().numpy(), k, v, t, some=range(S * K))
    long = torch.randn((2, 200003), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    u = _uniforms(4, 2, 4)
    for k in (0, 30):
        drafts, status = _drafts(torch, gr, long, k, u, T[2:])
        assert (status == ROW_OK).all()
        _check_drafts(drafts, long.cpu().numpy(), k, u, T[2:])
