"""The two ways in which the shared-prefix attention runs the sequences' own keys: which calls take which, and the edge cases on both.

Values against the CPU oracle in fp64, with the bounds derived in test_gpu_prefix.py.  Every test looks at the names of the kernels that
ran, so that none of them ends up on the other way unseen when the rule between the two changes."""
import math

import numpy as np
import pytest
import torch

import gpu_util as gu
from test_gpu_prefix import Case, E_RANGE, _binding

pytestmark = pytest.mark.gpu

# B, N, Hq, Hkv, room of the table behind the prefix (None: the longest sequence)
SHAPES = {
    "one_row": (3, 1, 4, 4, None),                            # few rows, a warp or more to a unit
    "eight_rows": (3, 4, 4, 2, None),
    "clusters": (3, 1, 4, 2, 1000),                           # few rows, units shared out over a cluster
    "wide_prefix": (40, 1, 16, 2, None),                      # few rows, 320 rows behind the prefix: blocks of 256 and 64
    "ten_rows": (3, 5, 4, 2, None),                           # on the line
}


def _case(shape, P, own, page=16, **kw):
    B, N, Hq, Hkv, room = SHAPES[shape]
    c = Case(B, N, Hq, Hkv, P, own, page, cap=P + room if room else None, **kw)
    c.shape = shape
    return c


def _few(names):
    few, line = (any(k in n for n in names) for k in ("few_rows_kernel", "prefix_merge_kernel"))
    assert few != line, names
    return few


def _call(c):
    """The call, on the way that the shape is for."""
    names = gu.kernels_captured(c.call)
    assert _few(names) == (c.shape != "ten_rows"), names
    c.call()


@pytest.mark.parametrize("early", [0, 1])
@pytest.mark.parametrize("P", [0, 1, 15, 17, 128, 257])
@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_prefixes_short_and_off_the_blocks(shape, P, early):
    c = _case(shape, P, [40, 0, 200], seed=P + 1)
    c.device(_binding(), option=(_binding().OPT_EARLY_PREFETCH, early))
    _call(c)
    assert c.ctx.status_poll() == 0
    c.check()
    c.ctx.close()


@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_lengths_that_do_not_fit(shape):
    for bad in (255, -1, -2 ** 31, 2 ** 31 - 1, "one beyond"):
        c = _case(shape, 256, [100, 60, 0], seed=3)
        want = c.want()
        c.device(_binding())
        c.kvd[1] = c.per * 16 - c.N + 1 if bad == "one beyond" else bad
        _call(c)
        assert c.ctx.status_poll() == E_RANGE
        assert (c.out[1] == 0).all() and (c.lse[1] == -math.inf).all()
        c.check(rows=[b for b in range(c.B) if b != 1], want=want)
        c.ctx.close()
    c = _case(shape, 256, [100, 60, 0], seed=3)
    c.device(_binding())
    c.kvd.fill_(3)                                            # nobody fits
    _call(c)
    assert c.ctx.status_poll() == E_RANGE and (c.out == 0).all() and (c.lse == -math.inf).all()
    c.ctx.close()


@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_entries_outside_the_pool_read_as_zeros(shape):
    for entry in (-1, 2 ** 31 - 1):
        c = _case(shape, 256, [100, 60], seed=4)
        for x in (c.k, c.v):
            x[:, :, 32:48] = 0                                # a shared block, and one of the second sequence's own
            x[1, :, 288:304] = 0
        c.device(_binding())
        c.td[0, 2] = entry
        c.td[1, 18] = entry
        _call(c)
        assert c.ctx.status_poll() == E_RANGE
        c.check()
        c.ctx.close()


@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_masks_that_leave_rows_nothing(shape):
    c = _case(shape, 0, [0, 0, 200], seed=9)
    c.mask[0] = 0                                             # nothing committed, nothing visible: empty rows
    c.mask[1, c.N - 1] = 0
    c.mask[2] = 0                                             # committed keys only
    c.device(_binding())
    _call(c)
    assert c.ctx.status_poll() == 0
    for x in (c.out[0], c.out[1, c.N - 1]):
        assert (x == 0).all()
    for x in (c.lse[0], c.lse[1, :, c.N - 1]):
        assert (x == -math.inf).all()
    c.check()
    c.ctx.close()
    c = _case(shape, 256, [0, 0, 200], seed=10)               # the prefix only; bits at and beyond N are no nodes
    c.mask[:] = 0
    want = c.want()
    c.mask |= np.uint64(0xFFFFFFFFFFFFFFFF) << np.uint64(c.N)
    c.device(_binding())
    _call(c)
    assert c.ctx.status_poll() == 0
    c.check(want=want)
    c.ctx.close()


@pytest.mark.parametrize("value", ["nan", "+inf", "-inf"])
@pytest.mark.parametrize("where", ["tree", "own", "first step", "second step", "last of the prefix"])
@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_a_score_that_is_not_finite(shape, where, value):
    """A key whose one element that is not zero meets a one in every q row: its score is NaN, +inf or -inf in every row that sees it, and
    nothing cancels.  NaN and +inf: out = NaN and lse = -inf in the rows that see it, whatever part of the keys it lies in; -inf: weight
    0.  All other rows keep their values."""
    P = 304                                                   # 19 whole blocks; steps of 128, 128 and 48 keys
    c = _case(shape, P, [140, 33, 10], seed=6)
    b, at = {"tree": (1, P + 33 + c.N - 1), "own": (1, P + 20), "first step": (0, 5), "second step": (0, 130),
             "last of the prefix": (0, P - 1)}[where]
    shared = at < P
    c.q[..., 0] = 0x3F80
    row = np.zeros(128, dtype=np.uint16)
    # the oracle sees it as a weight that is zero in any case: the lowest finite value (NaN and +inf rows are not compared with it)
    row[0] = 0xFF7F
    c.k[slice(None) if shared else b, 0, at] = row
    want = c.want()
    row[0] = {"nan": 0x7FC0, "+inf": 0x7F80, "-inf": 0xFF80}[value]
    c.pools[0][c.table[b, at // 16], 0, at % 16] = row
    c.device(_binding())
    _call(c)
    assert c.ctx.status_poll() == 0
    out, lse = c.out.float().cpu().numpy(), c.lse.cpu().numpy()
    sees = np.zeros((c.B, c.N), dtype=bool)
    if where == "tree":
        sees[1] = (c.mask[1, :, 0] >> np.uint64(c.N - 1)) & np.uint64(1) == 1
    else:
        sees[slice(None) if shared else 1] = True
    assert sees.any()
    G = c.Hq // c.Hkv
    hit = np.zeros((c.B, c.N, c.Hq), dtype=bool)
    if value != "-inf":
        hit[:, :, :G] = sees[:, :, None]
        assert np.isnan(out[hit]).all() and np.isneginf(lse.transpose(0, 2, 1)[hit]).all()
    o, l, a = want
    ok = ~hit
    err = np.abs(out - o)[ok]
    assert (err <= 2.0 ** -8 * (a + np.abs(o))[ok] + 6e-4 * a[ok]).all(), err.max()
    assert (np.abs(lse - l).transpose(0, 2, 1)[ok] <= 5e-4).all()
    c.ctx.close()


@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_captured_calls_follow_lengths_and_table(shape):
    c = _case(shape, 256, [100, 60, 30], seed=12)
    c.device(_binding())
    _call(c)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            for _ in range(3):                                # back to back on one scratch
                c.call()
        for own in ([100, 60, 30], [0, 60, 1], [17, 0, 29]):
            c.kv_len = (256 + np.resize(np.array(own), c.B)).astype(np.int32)
            c.kvd.copy_(torch.from_numpy(c.kv_len))
            c.out.fill_(float("nan"))
            c.lse.fill_(float("nan"))
            graph.replay()
            side.synchronize()
            c.check()
        # the block that a sequence's first own keys lie in, elsewhere
        spare = np.setdiff1d(np.arange(c.pools[0].shape[0]), c.table)[0]
        for d, src in ((c.kd, c.pools[0]), (c.vd, c.pools[1])):
            d[int(spare)] = gu.bf16_dev(src[c.table[1, 16]])
        c.td[1, 16] = int(spare)
        c.out.fill_(float("nan"))
        graph.replay()
        side.synchronize()
        c.check()
    assert c.ctx.status_poll() == 0
    c.ctx.close()


@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_calls_on_two_streams(shape):
    c = _case(shape, 512, [100, 20, 0], seed=8)
    c.device(_binding())
    want = c.want()
    _call(c)
    other, s2 = torch.full_like(c.out, float("nan")), c.ctx.prefix_scratch(c.B, c.N)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(a):
            c.call()
        with torch.cuda.stream(b):
            c.call(lse=False, scratch=s2, out=other)
    torch.cuda.synchronize()
    assert torch.equal(c.out, other) and c.ctx.status_poll() == 0
    c.check(want=want)
    c.ctx.close()
