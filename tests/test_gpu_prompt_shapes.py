"""What the prompt's and the shared prefix's calls take for a tensor of the documented shape: that shape, or neighbouring dimensions of it
joined or split, and not one whose dimensions are merely as many elements in another order."""
import math

import pytest
import torch

import gpu_util as gu
from paper_2509_15235_b200 import synth
from test_gpu_prefix import Case, _binding

pytestmark = pytest.mark.gpu


@pytest.fixture
def prompt():
    b = _binding()
    ctx = b.VerifyContext(2, 1, 4, 2, 128, 128, 2)
    kc, vc = (torch.zeros((2, 2, 128, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kp, vp = (torch.zeros((16, 2, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx.cache_register(0, kc, vc)
    ctx.cache_register_paged(1, kp, vp)
    q, k = (gu.bf16_dev(synth.normal_bf16((6, h, 128), 3 + h)) for h in (4, 2))
    table = torch.arange(16, dtype=torch.int32, device="cuda").view(2, 8)
    cu, kv = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 4, 6], [0, 3]))

    def calls(positions, axes):
        """The three calls that take positions, each giving its rotated q."""
        def rope():
            out = torch.empty_like(q)
            ctx.rope_axes_rows(q, None, positions, axes, out, None)
            return out

        def append():
            out = torch.empty_like(q)
            ctx.kv_append(0, q, k, k, positions, axes, cu, kv, out)
            return out

        def append_paged():
            out = torch.empty_like(q)
            ctx.kv_append_paged(1, q, k, k, positions, axes, cu, kv, table, out)
            return out
        return rope, append, append_paged
    yield b, calls
    assert ctx.status_poll() == 0
    ctx.close()


def test_positions_by_token_are_refused(prompt):
    """[T, n_axes] has as many elements as [n_axes, T]; taken for it, every row would be turned by other rows' positions."""
    b, calls = prompt
    for sections in ((16, 24, 24), (32, 32)):
        n = len(sections)
        pos = torch.arange(n * 6, dtype=torch.int32, device="cuda").view(n, 6)
        good = [f() for f in calls(pos, b.RopeAxes(sections, 1e6))]
        for wrong in (pos.t().contiguous(), pos.t().contiguous().view(6, n, 1), pos.view(-1)[:6].view(1, 6)):
            for f in calls(wrong, b.RopeAxes(sections, 1e6)):
                with pytest.raises(ValueError):
                    f()
        for same in (pos.view(-1), pos.view(n, 1, 6), pos.view(n, 2, 3)):
            for f, want in zip(calls(same, b.RopeAxes(sections, 1e6)), good):
                assert torch.equal(f(), want)
    # one axis: [T], [1, T] and [T, 1] are the same numbers in the same order
    pos = torch.arange(6, dtype=torch.int32, device="cuda")
    good = [f() for f in calls(pos.view(1, 6), b.RopeAxes((64,), 1e6))]
    for same in (pos, pos.view(6, 1)):
        for f, want in zip(calls(same, b.RopeAxes((64,), 1e6)), good):
            assert torch.equal(f(), want)


@pytest.mark.parametrize("N", [1, 5])
def test_prefix_tensors_in_another_order_are_refused(N):
    B, Hq = 3, 8
    c = Case(B, N, Hq, 2, 64, [30, 0, 100], 16, seed=1)
    ctx = c.device(_binding())
    scale = 1 / math.sqrt(128)

    def call(q=c.qd, m=c.md, out=c.out, lse=c.lse, kv=c.kvd):
        ctx.tree_verify_attn_prefix_paged(0, q, kv, c.td, 64, m, scale, c.scratch, out, lse)

    call()
    c.check()
    want = c.out.clone(), c.lse.clone()
    swapped = dict(lse=c.lse.view(B, N, Hq), out=c.out.view(B, Hq, N, 128), m=c.md.view(N, B, 1), q=c.qd.view(B, N, 2 * Hq, 64))
    for name, t in swapped.items():
        if N == 1 and name != "q":                            # the same numbers in the same order
            call(**{name: t})
            continue
        with pytest.raises(ValueError):
            call(**{name: t})
    for same in (dict(lse=c.lse.view(B * Hq, N)), dict(lse=c.lse.view(-1)), dict(out=c.out.view(B * N, Hq, 128)),
                 dict(out=c.out.view(B, N, Hq * 128)), dict(m=c.md.view(B, N)), dict(kv=c.kvd.view(B, 1))):
        c.out.fill_(float("nan"))
        c.lse.fill_(float("nan"))
        call(**same)
        assert torch.equal(c.out, want[0]) and torch.equal(c.lse, want[1])
    assert ctx.status_poll() == 0
    ctx.close()


def test_integers_beyond_the_calls_own_are_refused():
    """2^32 + 64 is not a prefix of 64."""
    c = Case(2, 1, 4, 2, 64, [30, 7], 16, seed=2)
    ctx = c.device(_binding())
    for P in (2 ** 32 + 64, 2 ** 31, -2 ** 31 - 1, 2 ** 64):
        with pytest.raises(OverflowError):
            c.call(prefix=P)
    with pytest.raises(OverflowError):
        ctx.tree_verify_attn_prefix_paged(2 ** 32, c.qd, c.kvd, c.td, 64, c.md, 1.0, c.scratch, c.out, c.lse)
    with pytest.raises(_binding().VispecError):
        c.call(prefix=2 ** 31 - 1)
    c.call()
    c.check()
    assert ctx.status_poll() == 0
    ctx.close()
