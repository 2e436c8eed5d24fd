"""Rotary positions with several axes and the append of new tokens' rows to the cache, against numpy in 64 bits.

A rotated element is formed from an angle rounded to 2^-26 of a turn (1.6 x 2^-24 rad), a sine and a cosine off by at most two
units in the last place (2 x 2^-24 of 1 each), and an fp32 product and sum (2 x 2^-24): 8 x 2^-24 of the pair's |x| + |y| in
all; then it is rounded to bf16 once, half a step (2^-8 of the value)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2509_15235_b200 import synth

pytestmark = pytest.mark.gpu

AXES = {  # D, sections, dealt in turn
    "one": (128, (64,), False), "three": (128, (16, 24, 24), False), "turns": (128, (24, 20, 20), True),
    "two64": (64, (12, 20), False), "four64": (64, (8, 8, 8, 8), True), "uneven": (128, (1, 62, 1), False),
}


def _binding():
    from paper_2509_15235_b200 import binding
    return binding


def _axis_of(sections, interleaved):
    if not interleaved:
        return np.repeat(np.arange(len(sections)), sections)
    left, out = list(sections), []
    for j in range(sum(sections)):
        a = j % len(sections)
        a = a if a and left[a] > 0 else 0
        left[a] -= 1
        out.append(a)
    assert left == [0] * len(sections)
    return np.array(out)


def _rotate(x, positions, sections, interleaved, theta):
    """x [T,H,D] -> (rotated, |x_j| + |x_j+D/2| per element), fp64."""
    T, H, D = x.shape
    half = D // 2
    z = x[..., :half] + 1j * x[..., half:]
    ang = positions[_axis_of(sections, interleaved)].T * float(np.float32(theta)) ** (-2.0 * np.arange(half) / D)
    z = z * np.exp(1j * ang)[:, None]
    size = np.abs(x[..., :half]) + np.abs(x[..., half:])
    return np.concatenate([z.real, z.imag], -1), np.concatenate([size, size], -1)


def _close(got, want, size):
    err = np.abs(got - want)
    slack = size * 8 * 2.0 ** -24
    assert np.isfinite(got).all() and (err <= 2.0 ** -8 * (np.abs(want) + slack) + slack).all(), err.max()


def _draw(T, heads, D, seed, fused):
    """bf16 rows q, k, v on the device and as fp64; fused: slices of one tensor's rows."""
    Hq, Hkv = heads
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((T, Hq + 2 * Hkv, D), generator=g, device="cuda", dtype=torch.bfloat16)
    parts = [x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]]
    return parts if fused else [p.contiguous() for p in parts]


def _np(t):
    return t.detach().double().cpu().numpy()


def _i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("axes", sorted(AXES))
@pytest.mark.parametrize("T,heads", [(1, (4, 4)), (5, (28, 4)), (37, (5, 1)), (700, (16, 2)), (2501, (7, 7))])
@pytest.mark.parametrize("fused", [False, True])
def test_rope_axes_rows(axes, T, heads, fused):
    b = _binding()
    D, sections, inter = AXES[axes]
    ctx = b.VerifyContext(1, 1, *heads, D, 128, 1)
    q, k, _ = _draw(T, heads, D, T, fused)
    pos = np.random.default_rng(T).integers(-50, 40000, size=(len(sections), T))
    ax = b.RopeAxes(sections, 1e6, inter)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    before = _np(q), _np(k)
    ctx.rope_axes_rows(q, k, _i32(pos), ax, qo, ko)
    assert np.array_equal(_np(q), before[0]) and np.array_equal(_np(k), before[1])
    for got, x in ((qo, before[0]), (ko, before[1])):
        _close(_np(got), *_rotate(x, pos, sections, inter, 1e6))
    # in place, and one of the two alone
    ctx.rope_axes_rows(q, None, _i32(pos), ax, q, None)
    assert torch.equal(q, qo) and np.array_equal(_np(k), before[1])
    ctx.rope_axes_rows(None, k, _i32(pos), ax, None, k)
    assert torch.equal(k, ko) and ctx.status_poll() == 0
    ctx.close()


def test_far_positions_and_position_zero():
    """Position 0 is the identity bit for bit; at 2^22 the fp64 part of the angle is still below the fp32 rounding."""
    b = _binding()
    ctx = b.VerifyContext(1, 1, 4, 2, 128, 128, 1)
    q, k, _ = _draw(64, (4, 2), 128, 3, False)
    ax = b.RopeAxes((64,), 1e4)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    ctx.rope_axes_rows(q, k, _i32(np.zeros((1, 64))), ax, qo, ko)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    pos = 2 ** 22 - np.arange(64)[None] * 65537
    ctx.rope_axes_rows(q, k, _i32(pos), ax, qo, ko)
    _close(_np(qo), *_rotate(_np(q), pos, (64,), False, 1e4))
    _close(_np(ko), *_rotate(_np(k), pos, (64,), False, 1e4))
    ctx.close()


def _cache(paged, B, Hkv, S_max, D, seed):
    """(k, v tensors, table or None, view [B,S_max,Hkv,D] of a cache as numpy)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    if not paged:
        k, v = (torch.randn((B, Hkv, S_max, D), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        return k, v, None, lambda t: _np(t).transpose(0, 2, 1, 3)
    rows, major = paged
    per, nb = S_max // rows, B * (S_max // rows) + 3
    shape = (nb, rows, Hkv, D) if major else (nb, Hkv, rows, D)
    k, v = (torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    table = np.random.default_rng(seed).permutation(nb)[:B * per].reshape(B, per)

    def view(t):
        x = _np(t) if major else _np(t).transpose(0, 2, 1, 3)
        return x[table].reshape(B, S_max, Hkv, D)
    return k, v, table, view


def _append(ctx, layer, table, q, k, v, pos, ax, cu, kv_len, q_out, new):
    if table is None:
        ctx.kv_append(layer, q, k, v, pos, ax, cu, kv_len, q_out, new)
    else:
        ctx.kv_append_paged(layer, q, k, v, pos, ax, cu, kv_len, table, q_out, new)


@pytest.mark.parametrize("paged", [None, (16, False), (32, True), (64, False), (128, True)])
@pytest.mark.parametrize("axes", ["one", "three", "turns", "four64"])
@pytest.mark.parametrize("lens,old", [((1, 1, 1), (100, 0, 383)), ((0, 129, 17), (5, 250, 0)), ((384, 0, 0), (0, 384, 7)),
                                      ((300, 255, 384), (84, 1, 0))])
def test_append_places_every_row_and_nothing_else(paged, axes, lens, old):
    b = _binding()
    D, sections, inter = AXES[axes]
    if paged and D != 128:
        pytest.skip("paged pools have head size 128")
    heads, B, S_max, pad = (6, 2), 3, 384, 5
    ctx = b.VerifyContext(B, 1, *heads, D, S_max, 2)
    kc, vc, table, view = _cache(paged, B, heads[1], S_max, D, 11)
    if paged:
        ctx.cache_register_paged(1, kc, vc, paged[1])
    else:
        ctx.cache_register(1, kc, vc)
    cu = np.concatenate([[0], np.cumsum(lens)])
    T = int(cu[-1]) + pad                                     # a batch padded behind its last sequence
    q, k, v = _draw(T, heads, D, 7, True)
    pos = np.random.default_rng(T).integers(0, 30000, size=(len(sections), T))
    ax = b.RopeAxes(sections, 1e4, inter)
    want_k, want_v = view(kc).copy(), view(vc).copy()
    all_k, all_v = kc.clone(), vc.clone()
    q_out = torch.full((T, heads[0], D), 3.0, device="cuda", dtype=torch.bfloat16)
    new = torch.full((B,), -7, device="cuda", dtype=torch.int32)
    tab = None if table is None else _i32(table)
    _append(ctx, 1, tab, q, k, v, _i32(pos), ax, _i32(cu), _i32(old), q_out, new)
    assert ctx.status_poll() == 0
    assert new.tolist() == [o + n for o, n in zip(old, lens)]
    rq, sq = _rotate(_np(q), pos, sections, inter, 1e4)
    rk, sk = _rotate(_np(k), pos, sections, inter, 1e4)
    _close(_np(q_out)[:T - pad], rq[:T - pad], sq[:T - pad])
    assert (_np(q_out)[T - pad:] == 3.0).all()
    got_k, got_v = view(kc), view(vc)
    for i in range(B):
        t, s, n = cu[i], old[i], lens[i]
        _close(got_k[i, s:s + n], rk[t:t + n], sk[t:t + n])
        want_k[i, s:s + n] = got_k[i, s:s + n]
        want_v[i, s:s + n] = _np(v)[t:t + n]
    assert np.array_equal(got_k, want_k) and np.array_equal(got_v, want_v)
    if table is not None:                                     # blocks that the table does not name
        other = np.setdiff1d(np.arange(kc.shape[0]), table)
        assert torch.equal(kc[other], all_k[other]) and torch.equal(vc[other], all_v[other])
    # without a rotation the rows are copies
    _append(ctx, 1, tab, None, k, v, None, None, _i32(cu), _i32(old), None, None)
    for i in range(B):
        t, s, n = cu[i], old[i], lens[i]
        assert np.array_equal(view(kc)[i, s:s + n], _np(k)[t:t + n])
    assert ctx.status_poll() == 0
    ctx.close()


def test_append_matches_the_tree_rows_placement():
    """One axis, every sequence N rows: what vispec_rope_tree_rows places (fp64 products), at most one bf16 step apart."""
    b = _binding()
    B, N, heads, S_max = 2, 9, (4, 2), 256
    ctx = b.VerifyContext(B, N, *heads, 128, S_max, 2)
    caches = [_cache(None, B, heads[1], S_max, 128, 21) for _ in range(2)]
    for l, (kc, vc, _, _) in enumerate(caches):
        ctx.cache_register(l, kc, vc)
    q, k, v = _draw(B * N, heads, 128, 5, False)
    kv_len = _i32([40, 200])
    pos = _i32([[40 + i for i in range(N)], [200 + i for i in range(N)]])
    q2 = q.clone()
    ctx.rope_tree_rows(0, q2.view(B, N, *q.shape[1:]), k.view(B, N, *k.shape[1:]), v.view(B, N, *v.shape[1:]), pos, kv_len, 1e4)
    qo = torch.empty_like(q)
    ctx.kv_append(1, q, k, v, pos.view(1, -1), b.RopeAxes((64,), 1e4), _i32([0, N, 2 * N]), kv_len, qo)
    for got, want in ((qo, q2), (caches[1][0], caches[0][0])):
        step = 2.0 ** -7 * np.maximum(np.abs(_np(want)), np.abs(_np(got))) + 1e-6
        assert (np.abs(_np(got) - _np(want)) <= step).all() and (got != want).float().mean() < 1e-3
    assert torch.equal(caches[0][1], caches[1][1]) and ctx.status_poll() == 0
    ctx.close()


@pytest.mark.parametrize("paged", [None, (16, True)])
def test_append_leaves_alone_what_does_not_fit(paged):
    b = _binding()
    E_RANGE = -4
    heads, B, S_max = (4, 2), 3, 128
    ctx = b.VerifyContext(B, 1, *heads, 128, S_max, 1)
    kc, vc, table, view = _cache(paged, B, heads[1], S_max, 128, 31)
    (ctx.cache_register_paged(0, kc, vc, paged[1]) if paged else ctx.cache_register(0, kc, vc))
    tab = None if table is None else _i32(table)
    q, k, v = _draw(30, heads, 128, 9, False)
    ax, pos = b.RopeAxes((64,), 1e4), _i32(np.arange(30)[None])

    first = kc.clone(), vc.clone()

    def call(cu, old, tab=tab):
        kc.copy_(first[0])                                    # (rows that an earlier call wrote would not show again)
        vc.copy_(first[1])
        k0, v0 = view(kc), view(vc)
        q_out = torch.full_like(q, 3.0)
        new = torch.full((B,), -7, device="cuda", dtype=torch.int32)
        _append(ctx, 0, tab, q, k, v, pos, ax, _i32(cu), _i32(old), q_out, new)
        return (view(kc) != k0).any((2, 3)), (view(vc) != v0).any((2, 3)), _np(q_out), new.tolist(), ctx.status_poll()

    # the middle sequence: one row too many, a negative length
    for bad in (S_max - 9, -1, 2 ** 31 - 1):
        dk, dv, qo, new, st = call([0, 10, 20, 30], [0, bad, S_max - 10])
        assert st == E_RANGE and new == [10, -7, S_max]
        assert not dk[1].any() and not dv[1].any() and dk[0, :10].all() and dk[2, -10:].all()
        assert (qo[10:20] == 3.0).all() and (qo[:10] != 3.0).any(-1).all() and (qo[20:] != 3.0).any(-1).all()
    # ends that are no ends: nothing happens at all
    for cu in ([0, 20, 10, 30], [-1, 10, 20, 30], [0, 10, 20, 31], [0, 10, 20, 2 ** 31 - 1]):
        dk, dv, qo, new, st = call(cu, [0, 0, 0])
        assert st == E_RANGE and new == [-7] * 3 and not dk.any() and not dv.any() and (qo == 3.0).all()
    if paged:
        for entry in (-1, kc.shape[0], 2 ** 31 - 1):
            t2 = np.array(table)
            t2[0, 0] = entry                                  # slots 0..15 of the first sequence
            k0 = first[0]
            _, _, qo, new, st = call([0, 10, 20, 30], [8, 0, 0], _i32(t2))
            assert st == E_RANGE and new == [18, 10, 10] and (qo != 3.0).any(-1).all()
            blk = table[0, 0]
            assert torch.equal(kc[blk], k0[blk]) and not torch.equal(kc[table[0, 1]], k0[table[0, 1]])
    ctx.close()


def test_empty_calls():
    b = _binding()
    ctx = b.VerifyContext(2, 1, 4, 2, 128, 128, 1)
    kc, vc, _, _ = _cache(None, 2, 2, 128, 128, 1)
    ctx.cache_register(0, kc, vc)
    k0 = kc.clone()
    q, k, v = _draw(0, (4, 2), 128, 1, False)
    ax, none = b.RopeAxes((64,), 1e4), _i32(np.zeros((1, 0)))
    ctx.rope_axes_rows(q, k, none, ax, q, k)
    new = torch.full((2,), -7, device="cuda", dtype=torch.int32)
    ctx.kv_append(0, q, k, v, none, ax, _i32([0, 0, 0]), _i32([5, 128]), q, new)
    assert new.tolist() == [5, 128] and torch.equal(kc, k0) and ctx.status_poll() == 0
    ctx.kv_append(0, q, k, v, none, ax, _i32([0]), _i32(np.zeros(0)), q, None)
    assert torch.equal(kc, k0) and ctx.status_poll() == 0
    ctx.close()


def test_captured_append_follows_its_inputs_and_runs_on_its_stream():
    """One graph of a padded decoding step, replayed with other lengths and rows, on a stream of its own."""
    b = _binding()
    heads, B, S_max, T = (4, 2), 4, 128, 16
    ctx = b.VerifyContext(B, 1, *heads, 128, S_max, 1)
    kc, vc, table, view = _cache((16, False), B, heads[1], S_max, 128, 41)
    ctx.cache_register_paged(0, kc, vc)
    q, k, v = _draw(T, heads, 128, 2, False)
    ax, pos, tab = b.RopeAxes((16, 24, 24), 1e6), _i32(np.zeros((3, T))), _i32(table)
    cu, kv_len, new = _i32([0, 1, 2, 3, 4]), _i32([0] * B), _i32([0] * B)
    qo = torch.zeros_like(q)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx.kv_append_paged(0, q, k, v, pos, ax, cu, kv_len, tab, qo, new)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            ctx.kv_append_paged(0, q, k, v, pos, ax, cu, kv_len, tab, qo, new)
        rng = np.random.default_rng(0)
        for lens, old in (([4, 0, 1, 11], [3, 9, 0, 100]), ([1, 1, 1, 1], [7, 127, 20, 0])):
            p = rng.integers(0, 5000, size=(3, T))
            pos.copy_(_i32(p)); cu.copy_(_i32(np.concatenate([[0], np.cumsum(lens)]))); kv_len.copy_(_i32(old))
            k.copy_(torch.randn_like(k))
            graph.replay()
            side.synchronize()
            rk, sk = _rotate(_np(k), p, (16, 24, 24), False, 1e6)
            got, t = view(kc), 0
            for i in range(B):
                _close(got[i, old[i]:old[i] + lens[i]], rk[t:t + lens[i]], sk[t:t + lens[i]])
                t += lens[i]
            assert new.tolist() == [o + n for o, n in zip(old, lens)]
        assert ctx.status_poll() == 0
    ctx.close()


def test_refusals():
    b = _binding()
    E_NULL, E_ALIGN, E_SHAPE, E_RANGE, E_UNSUP, E_UNREG = -1, -2, -3, -4, -5, -9
    ctx = b.VerifyContext(2, 1, 4, 2, 128, 128, 3)
    kc, vc, _, _ = _cache(None, 2, 2, 128, 128, 1)
    ctx.cache_register(0, kc, vc)
    kp, vp, table, _ = _cache((16, False), 2, 2, 128, 128, 1)
    ctx.cache_register_paged(1, kp, vp)
    tab = _i32(table)
    q, k, v = _draw(6, (4, 2), 128, 1, False)
    pos, cu, kv = _i32(np.zeros((1, 6))), _i32([0, 3, 6]), _i32([0, 0])
    ax = b.RopeAxes((64,), 1e4)

    def refused(code, call):
        with pytest.raises(b.VispecError) as e:
            call()
        assert e.value.code == code

    for bad in (b.RopeAxes((63,), 1e4), b.RopeAxes((64, 64), 1e4), b.RopeAxes((0, 64), 1e4), b.RopeAxes((-1, 65), 1e4),
                b.RopeAxes((64,), 1.0), b.RopeAxes((64,), float("nan")), b.RopeAxes((64,), float("inf")),
                b.RopeAxes((4, 56, 4), 1e4, True)):
        p = _i32(np.zeros((len(bad.sections), 6)))
        refused(E_SHAPE, lambda: ctx.rope_axes_rows(q, k, p, bad, q, k))
        refused(E_SHAPE, lambda: ctx.kv_append(0, q, k, v, p, bad, cu, kv, q))
    with pytest.raises(ValueError):
        b.RopeAxes((16,) * 5, 1e4)
    refused(E_NULL, lambda: ctx.rope_axes_rows(q, k, pos, ax, None, k))
    refused(E_NULL, lambda: ctx.rope_axes_rows(q, None, pos, ax, q, k))
    wide = torch.zeros((6, 5, 128), dtype=torch.bfloat16, device="cuda")
    refused(E_SHAPE, lambda: ctx.rope_axes_rows(wide[:, :4], k, pos, ax, wide.view(-1)[:6 * 512].view(6, 4, 128), k))
    refused(E_SHAPE, lambda: ctx.rope_axes_rows(q[:1].expand(6, 4, 128), k, pos, ax, q, k))
    off = torch.zeros(6 * 512 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(6, 4, 128)
    refused(E_ALIGN, lambda: ctx.rope_axes_rows(off, k, pos, ax, q, k))
    odd = torch.zeros((6, 516), dtype=torch.bfloat16, device="cuda")[:, :512].unflatten(1, (4, 128))
    refused(E_ALIGN, lambda: ctx.rope_axes_rows(odd, k, pos, ax, q, k))
    refused(E_SHAPE, lambda: ctx.kv_append(0, q, k, v, pos, ax, cu, kv, q, kv))          # kv_len_out is kv_len
    refused(E_SHAPE, lambda: ctx.kv_append(0, q, k, v, None, None, cu, kv, q))            # q without a rotation
    refused(E_NULL, lambda: ctx.kv_append(0, q, k, v, None, ax, cu, kv, q))
    refused(E_NULL, lambda: ctx.kv_append(0, q, k, v, pos, ax, cu, kv, None))
    refused(E_RANGE, lambda: ctx.kv_append(3, q, k, v, pos, ax, cu, kv, q))
    refused(E_UNREG, lambda: ctx.kv_append(2, q, k, v, pos, ax, cu, kv, q))
    refused(E_UNSUP, lambda: ctx.kv_append(1, q, k, v, pos, ax, cu, kv, q))
    refused(E_UNSUP, lambda: ctx.kv_append_paged(0, q, k, v, pos, ax, cu, kv, tab, q))
    refused(E_SHAPE, lambda: ctx.kv_append(0, q, k, v, pos, ax, _i32([0, 2, 4, 6]), _i32([0, 0, 0]), q))   # B > B_max
    # what the binding itself refuses
    for call in (lambda: ctx.rope_axes_rows(q.float(), k, pos, ax, q, k), lambda: ctx.rope_axes_rows(q.cpu(), k, pos, ax, q, k),
                 lambda: ctx.rope_axes_rows(q, k[:5], pos, ax, q, k), lambda: ctx.rope_axes_rows(q, k, pos[:, :5], ax, q, k),
                 lambda: ctx.rope_axes_rows(q, k, pos.long(), ax, q, k), lambda: ctx.rope_axes_rows(k, k, pos, ax, k, k),
                 lambda: ctx.rope_axes_rows(q.transpose(0, 1).contiguous().transpose(0, 1), k, pos, ax, q, k),
                 lambda: ctx.kv_append(0, q, k, v, pos, ax, cu[:2], kv, q), lambda: ctx.kv_append(0, q, k, v[:, :1], pos, ax, cu, kv, q),
                 lambda: ctx.kv_append_paged(1, q, k, v, pos, ax, cu, kv, tab[:1], q)):
        with pytest.raises((ValueError, TypeError)):
            call()
    with pytest.raises(TypeError):
        ctx.rope_axes_rows(None, None, pos, ax, None, None)
    assert ctx.status_poll() == 0
    ctx.close()


def test_null_context_is_refused():
    lib = _binding().load()
    z = ctypes.c_void_p(0)
    assert lib.vispec_rope_axes_rows(z, z, 0, z, 0, z, 0, None, z, 0, z, 0, z) == -1
    assert lib.vispec_kv_append(z, 0, z, 0, z, 0, z, 0, z, None, z, z, 0, 0, z, 0, z, z) == -1
    assert lib.vispec_kv_append_paged(z, 0, z, 0, z, 0, z, 0, z, None, z, z, z, 0, 0, 0, z, 0, z, z) == -1
