"""Layouts of states whose sizes no memory holds, at the C entry and without a GPU: refused, where the products of their sizes wrap round or pass what a launch counts."""
import pytest

from test_beside_refusals import CALLS, EINVAL
from test_host_paths import recorded  # noqa: F401  (the fixture)

HUGE = (1 << 31) - 1


@pytest.mark.parametrize("call, rc", [
    ("reorder(table=m, block=1 << 30, width=1, blocks=3, token_bytes=1 << 34)", EINVAL), ("reorder(table=m, block=4, width=1, blocks=3, token_bytes=1 << 62)", EINVAL),
    ("reorder(table=m, block=4, width=2, blocks=3, token_bytes=1 << 29, token_stride=1 << 29)", EINVAL), ("reorder(table=m, block=4, width=2, blocks=3, token_bytes=(1 << 29) - 1)", 0),
    ("reorder(table=m, block=1, width=1 << 24, blocks=3)", EINVAL), ("reorder(table=m, block=1, width=(1 << 24) - 1, blocks=3)", 0),
    (f"reorder(table=m, block={HUGE}, width=1, blocks=3, token_bytes=1, token_stride=16)", EINVAL), ("reorder(table=m, block=1 << 30, width=1, blocks=3, token_bytes=1, token_stride=16)", 0),
    (f"reorder(tokens={HUGE}, token_bytes={HUGE}, token_stride={HUGE})", EINVAL), (f"reorder(tokens={HUGE}, token_bytes=60, token_stride=60)", 0), (f"reorder(tokens={HUGE}, token_bytes=65, token_stride=65)", EINVAL),
    (f"reorder(tokens=1 << 24, token_bytes=9000, token_stride=10000)", EINVAL), (f"reorder(tokens=(1 << 24) - 1, token_bytes=9000, token_stride=10000)", 0),
    ("reorder(heads=1 << 20, head_stride=1 << 24, tokens=1 << 24, token_bytes=1 << 24, token_stride=1 << 44)", EINVAL),
    (f"reorder(heads={HUGE}, head_stride={HUGE}, tokens=4, token_bytes={HUGE}, token_stride={HUGE} * {HUGE})", EINVAL),
    (f"reorder(outer={HUGE}, outer_stride=1 << 40, tokens=(1 << 24) - 1, token_bytes=9000, token_stride=10000, S=65535)", 0)])
def test_a_layout_beyond_any_memory_is_refused(recorded, call, rc):  # noqa: F811
    r = recorded(CALLS + f"""
result["rc"] = {call}
result["log"] = log()
""")
    assert r["rc"] == rc and [x.split()[0] for x in r["log"]] == ([] if rc else ["launch"]), r
