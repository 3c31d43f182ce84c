"""What the operators beside the verification refuse, at the C entries and without a GPU: the code, and that nothing was launched."""
import pytest

from test_host_paths import recorded  # noqa: F401  (the fixture)

EINVAL, EHIP, EUNSUPPORTED = -1, -4, -5

CALLS = r'''
L = C.c_longlong
class Layout(C.Structure):
    _fields_ = [(n, L) for n in ("outer", "outer_stride", "heads", "head_stride", "row_stride", "tokens", "token_stride", "token_bytes")] + [(n, C.c_int) for n in ("block", "width", "blocks")]
m = buffer(4096)
def draft(h, x=m, stride=100, n=2, k=10, u=m, B=4, V=100, d=m, s=m):
    return lib.gr_draft(h, x, L(stride), n, k, u, B, V, d, s, None)
def draft_logits(h, x=m, dtype=1, stride=100, T=m, n=2, k=10, u=m, B=4, V=100, d=m, s=m):
    return lib.gr_draft_logits(h, x, dtype, L(stride), T, n, k, u, B, V, d, s, None)
def select(h, x=m, dtype=0, stride=100, T=None, scores=m, finished=None, eos=-1, S=2, K=2, V=100, M=4, a=m, b=m, c=m, d=None, s=m):
    return lib.gr_beam_select(h, x, dtype, L(stride), T, scores, finished, eos, S, K, V, M, a, b, c, d, s, None)
def reorder(state=m, parent=m, table=None, S=2, K=2, **more):
    f = dict(outer=1, outer_stride=0, heads=1, head_stride=0, row_stride=64, tokens=4, token_stride=16, token_bytes=16, block=0, width=0, blocks=0)
    f.update(more)
    return lib.gr_beam_reorder(state, C.byref(Layout(**f)), parent, None, None, table, S, K, None)
def pages(old=m, new=m, table=m, stack=m, count=m, R=3, width=4, block=16, pool=8, cap=10, a=None, b=None, c=m, slots=m, s=m):
    return lib.gr_page_update(old, new, table, stack, count, R, width, block, pool, L(cap), a or buffer(8), b or buffer(8), c, slots, s, None)
off = C.c_void_p(C.addressof(m) + 2)
'''


@pytest.mark.parametrize("call, rc", [
    ("draft(h)", 0), ("draft(None)", EINVAL), ("draft(h, x=None)", EINVAL), ("draft(h, u=None)", EINVAL), ("draft(h, stride=99)", EINVAL), ("draft(h, n=0)", EINVAL), ("draft(h, n=4)", EINVAL),
    ("draft(h, B=0)", EINVAL), ("draft(h, B=5)", EINVAL), ("draft(h, V=601, stride=700)", EINVAL), ("draft(h, V=0)", EINVAL), ("draft(h, x=off)", EINVAL),
    ("draft(h, V=600, stride=600, k=257)", EUNSUPPORTED), ("draft(h, V=600, stride=600, k=0)", 0), ("draft(h, V=600, stride=600, k=600)", 0), ("draft(h, V=600, stride=600, k=256)", 0),
    ("draft(cut)", 0), ("draft(cut, V=600, stride=600, k=0)", EUNSUPPORTED), ("draft(cut, k=0)", 0), ("draft_logits(cut)", EUNSUPPORTED), ("draft_logits(h)", 0), ("draft_logits(h, T=None)", EINVAL),
    ("draft_logits(h, dtype=3)", EINVAL), ("draft_logits(h, dtype=-1)", EINVAL), ("draft_logits(h, x=off, dtype=0)", EINVAL), ("draft_logits(h, x=off)", 0),
    ("select(h)", 0), ("select(None)", EINVAL), ("select(h, scores=None)", EINVAL), ("select(h, S=3)", EINVAL), ("select(h, K=0)", EINVAL), ("select(h, S=1, K=65)", EINVAL), ("select(h, M=0)", EINVAL),
    ("select(h, M=65)", EINVAL), ("select(h, S=2147483647, K=3)", EINVAL), ("select(h, V=601, stride=601)", EINVAL), ("select(h, stride=99)", EINVAL), ("select(h, eos=100)", EINVAL),
    ("select(h, eos=-2)", EINVAL), ("select(h, finished=m)", EINVAL), ("select(h, finished=m, eos=0)", 0), ("select(h, dtype=4)", EINVAL), ("select(h, x=off)", EINVAL),
    ("reorder()", 0), ("reorder(state=None)", EINVAL), ("reorder(parent=None)", EINVAL), ("reorder(S=0)", EINVAL), ("reorder(S=65536)", EINVAL), ("reorder(K=65)", EINVAL), ("reorder(K=0)", EINVAL),
    ("reorder(outer=0)", EINVAL), ("reorder(heads=0)", EINVAL), ("reorder(tokens=0)", EINVAL), ("reorder(token_bytes=0)", EINVAL), ("reorder(row_stride=-1)", EINVAL), ("reorder(token_stride=-16)", EINVAL),
    ("reorder(outer=1 << 20, heads=1 << 20)", EINVAL), ("reorder(table=m)", EINVAL), ("reorder(table=m, block=16, width=2, blocks=3)", 0), ("reorder(table=m, block=16, width=2)", EINVAL),
    ("reorder(table=m, block=65536, width=65536, blocks=3)", EINVAL),
    ("pages()", 0), ("pages(old=None)", EINVAL), ("pages(R=0)", EINVAL), ("pages(R=8193)", EINVAL), ("pages(R=8192)", 0), ("pages(width=0)", EINVAL), ("pages(block=0)", EINVAL), ("pages(pool=0)", EINVAL),
    ("pages(cap=-1)", EINVAL), ("pages(cap=1 << 31)", EINVAL), ("pages(cap=0, slots=None)", 0), ("pages(slots=None)", EINVAL), ("pages(a=m)", EINVAL), ("pages(b=m)", EINVAL),
    ("pages(R=8000, width=1 << 20)", EINVAL), ("pages(width=1 << 20, block=1 << 12)", EINVAL)])
def test_a_refused_call_launches_nothing(recorded, call, rc):  # noqa: F811
    r = recorded(CALLS + f"""
h = create(4, 600, 32, 3)
class Config(C.Structure):
    _fields_ = [("max_iter", C.c_int), ("max_T", C.c_int), ("rel_tol", C.c_double), ("flags", C.c_int), ("tail_mass", C.c_double)]
cut = C.c_void_p()
assert lib.gr_create(C.byref(cut), 4, 600, 32, 3, C.byref(Config(0, 0, 0.0, 0, 0.1))) == 0
assert solve(h, 4, 600, 3, 32) == 0
hip.recorded_clear()
result["rc"] = {call}
result["log"] = log()
result["over"] = hip.recorded_over()
result["verify"] = verify(h, 4)
""")
    assert r["rc"] == rc and r["over"] == 0
    assert all(x.startswith("launch ") for x in r["log"]) and bool(r["log"]) == (rc == 0), r["log"]
    assert r["verify"] == (-3 if rc == 0 and call.split("(")[0] in ("draft", "draft_logits", "select") and "(cut" not in call else 0)


@pytest.mark.parametrize("call", ["draft(h)", "draft(h, V=600, stride=600, k=0)", "draft_logits(h)", "select(h)", "reorder()", "pages()"])
def test_a_failed_launch_is_reported_and_leaves_no_error_to_the_next_call(recorded, call):  # noqa: F811
    r = recorded(CALLS + f"""
h = create(4, 600, 32, 3)
hip.recorded_clear()
assert {call} == 0
launches = len(log())
result["seen"] = []
for i in range(launches):
    hip.recorded_clear()
    hip.recorded_fail(b"launch", i)
    rc = {call}
    hip.recorded_clear()
    result["seen"].append([rc, {call}, solve(h, 4, 600, 3, 32), verify(h, 4)])
""")
    assert r["seen"] and all(x == [EHIP, 0, 0, 0] for x in r["seen"]), r["seen"]


@pytest.mark.parametrize("call, launches", [("draft(big, B=1, V=200000, stride=200000)", 2), ("draft(big, B=1, V=200000, stride=200000, k=0)", 2), ("draft_logits(big, B=1, V=200000, stride=200000, k=0)", 2),
                                            ("draft(big, B=1, V=5000, stride=5000)", 1), ("draft(big, B=1, V=5000, stride=5000, k=0)", 1), ("draft(big, B=200, V=200000, stride=200000)", 1),
                                            ("draft(big, B=200, V=200000, stride=200000, k=0)", 1), ("draft_logits(big, B=200, V=200000, stride=200000)", 1), ("select(big)", 2)])
def test_launches_of_few_long_rows_and_of_others(recorded, call, launches):  # noqa: F811
    """A failure of either launch is reported, and the next call is as ever."""
    r = recorded(CALLS + f"""
big = create(200, 200000, 32, 3)
hip.recorded_clear()
assert {call} == 0
result["launches"] = len(log())
result["seen"] = []
for i in range(result["launches"]):
    hip.recorded_clear()
    hip.recorded_fail(b"launch", i)
    rc = {call}
    hip.recorded_clear()
    result["seen"].append([rc, {call}])
""")
    assert r["launches"] == launches and all(x == [EHIP, 0] for x in r["seen"]), r
