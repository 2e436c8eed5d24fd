"""The expected committed length (VISPEC_OPT_KV_LEN_HINT) chooses how the shared-prefix attention runs the sequences' own keys."""
import pytest

import gpu_util as gu
from test_gpu_prefix import Case, _binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P,hint,few", [
    (256, 0, False),                  # no expectation: the table's 8192 slots count
    (256, 256, True), (256, 400, True), (256, 3000, False), (256, 100000, False),
    (256, 100, False),                # below the prefix: no expectation of a sequence of this call
    (0, 400, True), (0, 3000, False),
    (0, 2 ** 31 - 1, False), (256, 2 ** 31 - 1, False),
])
def test_the_hint_chooses_the_way_and_leaves_the_result(P, hint, few):
    c = Case(6, 1, 8, 2, P, [100, 3, 0, 1200], 64, seed=14, cap=8192)
    c.device(_binding(), option=(_binding().OPT_KV_LEN_HINT, hint))
    names = gu.kernels_captured(c.call)
    assert any("few_rows_kernel" in n for n in names) == few, names
    assert any("prefix_merge_kernel" in n for n in names) != few, names
    c.call()
    assert c.ctx.status_poll() == 0
    c.check()
    c.ctx.close()


@pytest.mark.parametrize("hint", [300, 5000])
def test_a_hint_given_between_calls_counts_from_the_next_one(hint):
    c = Case(3, 2, 8, 4, 128, [700, 0, 90], 16, seed=15, cap=4096)
    c.device(_binding())
    assert not any("few_rows_kernel" in n for n in gu.kernels_captured(c.call))
    c.call()
    c.ctx.ctx_set_option(_binding().OPT_KV_LEN_HINT, hint)
    c.out.fill_(float("nan"))
    assert any("few_rows_kernel" in n for n in gu.kernels_captured(c.call)) == (hint == 300)
    c.call()
    assert c.ctx.status_poll() == 0
    c.check()
    c.ctx.close()
