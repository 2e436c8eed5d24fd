"""Attention of a batch that shares a prefix, against the CPU oracle (fp64) on the contiguous caches the pool was cut from.

Tolerances.  A weight is rounded to bf16 before the product with V (at most 2^-8 of it, so at most 2^-8 of A = sum p |v|, which the
oracle gives on |v|), the output once more (2^-8 of it).  Scores are sums of 128 products in fp32: off by at most 128 x 2^-23
of sum |q_i k_i| scale, which is below 20 for the normal inputs here: 3e-4 in the exponent, and so 6e-4 of A (weights and their sum)
at the very most; lse: 3e-4 and the rounding of the sum."""
import ctypes
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2509_15235_b200 import synth

pytestmark = pytest.mark.gpu
NAN = np.uint16(0x7FC0)
E_RANGE = -4
SCALE = 1 / math.sqrt(128)


def _binding():
    from paper_2509_15235_b200 import binding
    return binding


class Case:
    """Contiguous caches whose sequences agree on the first `shared` slots, and the pool and table that hold them."""

    def __init__(self, B, N, Hq, Hkv, P, own, page, major=False, seed=0, cap=None):
        rng = np.random.Generator(np.random.Philox(seed))
        self.B, self.N, self.Hq, self.Hkv, self.P, self.page, self.major = B, N, Hq, Hkv, P, page, major
        self.kv_len = P + np.resize(np.array(own, dtype=np.int32), B)
        need = int(self.kv_len.max()) + N
        self.per = per = max(-(-(cap or need) // page), -(-need // page))
        S = per * page
        self.shared = shared = P // page
        self.q = synth.normal_bf16((B, N, Hq, 128), seed + 1)
        self.k, self.v = (synth.normal_bf16((B, Hkv, S, 128), seed + i) for i in (2, 3))
        for x in (self.k, self.v):
            x[:, :, :shared * page] = x[:1, :, :shared * page]
        parents = np.stack([synth.draw_tree(N, 6, 4, rng) for _ in range(B)])
        self.mask = oracle.tree_mask(parents)[0]
        nb = shared + B * (per - shared) + 2
        perm = rng.permutation(nb)[:nb - 2].astype(np.int32)
        self.table = np.concatenate([np.tile(perm[:shared], (B, 1)), perm[shared:].reshape(B, per - shared)], 1)
        self.pools = []
        for x in (self.k, self.v):
            pool = np.full((nb, Hkv, page, 128), NAN, dtype=np.uint16)
            blocks = x.reshape(B, Hkv, per, page, 128).transpose(0, 2, 1, 3, 4)
            for b in range(B - 1, -1, -1):
                pool[self.table[b]] = blocks[b]
            self.pools.append(pool)
        # rows behind each sequence's last key may hold anything
        for b in range(B):
            for x in self.pools:
                e, r = divmod(int(self.kv_len[b]) + N, page)
                if e < per:
                    x[self.table[b, e], :, r:] = NAN
        # what must not be read: entries behind the last block, and the shared entries of every row but the first
        self.given = self.table.copy()
        for b in range(B):
            self.given[b, -(-(int(self.kv_len[b]) + N) // page):] = 2 ** 30
            if b:
                self.given[b, :shared] = -5

    def device(self, b, layers=1, option=None):
        import gpu_util as gu
        self.ctx = ctx = b.VerifyContext(self.B, self.N, self.Hq, self.Hkv, 128, self.per * self.page, layers)
        pools = [np.ascontiguousarray(x.transpose(0, 2, 1, 3)) if self.major else x for x in self.pools]
        self.kd, self.vd = map(gu.bf16_dev, pools)
        ctx.cache_register_paged(0, self.kd, self.vd, self.major)
        if option:
            ctx.ctx_set_option(*option)
        self.qd, self.md = gu.bf16_dev(self.q), gu.u64_dev(self.mask)
        self.kvd, self.td = gu.i32_dev(self.kv_len), gu.i32_dev(self.given)
        self.scratch = ctx.prefix_scratch(self.B, self.N)
        self.scratch.fill_(0xFF)                              # NaN in every partial that is not written
        self.out = torch.full((self.B, self.N, self.Hq, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((self.B, self.Hq, self.N), float("nan"), dtype=torch.float32, device="cuda")
        return ctx

    def call(self, prefix=None, lse=True, scratch=None, out=None):
        self.ctx.tree_verify_attn_prefix_paged(0, self.qd, self.kvd, self.td, self.P if prefix is None else prefix, self.md, SCALE,
                                               self.scratch if scratch is None else scratch,
                                               self.out if out is None else out, self.lse if lse else None)

    def want(self):
        o, l = oracle.tree_attn(self.q, self.k, self.v, self.kv_len, self.mask, SCALE)
        a, _ = oracle.tree_attn(self.q, self.k, self.v & np.uint16(0x7FFF), self.kv_len, self.mask, SCALE)
        return o, l, a

    def check(self, rows=slice(None), want=None):
        o, l, a = want or self.want()
        got, lse = self.out.float().cpu().numpy(), self.lse.cpu().numpy()
        err = np.abs(got - o)[rows]
        assert (err <= 2.0 ** -8 * (a + np.abs(o))[rows] + 6e-4 * a[rows]).all(), err.max()
        seen = np.isfinite(l[rows])
        assert np.array_equal(np.isfinite(lse[rows]), seen) and (np.abs(lse[rows] - l[rows])[seen] <= 5e-4).all()


CASES = {
    # B, N, Hq, Hkv, P, own
    "decode_gqa": (8, 1, 28, 4, 1300, [46, 354, 1, 0, 127, 128, 129, 300]),
    "decode_mha": (5, 1, 8, 8, 640, [0, 1, 500, 64, 17]),
    "two": (2, 1, 4, 4, 128, [5]),
    "one_sequence": (1, 9, 8, 2, 512, [33]),
    "tree_60": (3, 60, 8, 2, 1111, [354, 46, 0]),                 # prefix blocks of 256, 256, 208 rows; own of 240
    "tree_last_block_short": (5, 15, 8, 2, 900, [100, 3, 250, 0, 60]),   # 300 rows: 256 in two tiles, 44 in alternate steps
    "tree_128": (4, 128, 16, 2, 400, [300, 1200, 0, 5]),          # own rows in four blocks
    "tree_129_rows": (3, 43, 3, 1, 300, [7, 140, 2]),             # own 129 rows: one row in the second tile
    "nothing_shared": (3, 20, 4, 2, 0, [300, 0, 129]),
    "many": (128, 1, 4, 2, 512, [0, 3, 40, 200]),
    "hundreds": (300, 1, 7, 1, 272, [0, 3, 40, 130, 77]),         # prefix rows in nine blocks
    "few_8_rows": (5, 2, 8, 2, 160, [0, 300, 40, 7, 900]),        # 8 rows per sequence and kv head
    "few_9_rows": (5, 3, 6, 2, 160, [0, 300, 40, 7, 900]),
    "few_rows_blocks": (20, 4, 8, 4, 2000, [5, 0, 333]),          # prefix of 160 rows
    # prefix of 560 rows, two blocks of 256 and one of 48 in alternate steps, each cut into as many parts as a whole block
    "few_short_last_block": (80, 1, 28, 4, 2000, [300, 5, 0]),
    "few_wide_last_block": (50, 2, 9, 3, 1500, [30, 5, 0]),       # 300 rows: 256 and 44
    "few_long_own": (3, 1, 4, 2, 4096, [1300, 900, 0]),           # own keys in clusters
    "just_above_few": (3, 17, 2, 2, 500, [5, 200, 64]),
    "many_trees": (40, 8, 8, 8, 256, [10, 60, 0, 300, 5]),
    "long_own": (2, 4, 4, 1, 96, [4000, 2500]),
}


@pytest.mark.parametrize("page,major", [(16, False), (32, True), (64, False), (128, True)])
@pytest.mark.parametrize("name", sorted(CASES))
def test_against_the_oracle(name, page, major):
    c = Case(*CASES[name], page, major, seed=len(name) + page)
    c.device(_binding())
    c.call()
    assert c.ctx.status_poll() == 0
    c.check()
    first = c.out.clone(), c.lse.clone()
    # the same again bit for bit, also without lse and without reading ahead
    c.scratch.fill_(0xFF)
    c.ctx.ctx_set_option(_binding().OPT_EARLY_PREFETCH, 0)
    c.call(lse=False)
    assert torch.equal(c.out, first[0])
    assert c.ctx.status_poll() == 0 and c.ctx.launch_count() in (2, 4)
    c.ctx.close()


@pytest.mark.parametrize("P", [1, 15, 16, 17, 100, 127, 128, 129, 1000])
def test_prefix_lengths_off_the_blocks(P):
    """Slots of a block that the prefix ends within are each sequence's own; any shorter prefix_len is as right."""
    c = Case(3, 11, 8, 2, P, [40, 0, 200], 16, seed=P)
    c.device(_binding())
    want = c.want()
    c.call()
    c.check(want=want)
    c.given[:, :c.shared] = c.table[:, :c.shared]             # now every row's entries are there
    c.td.copy_(torch.from_numpy(c.given))
    for less in (0, P // 2, P):
        c.call(prefix=less)
        assert c.ctx.status_poll() == 0
        c.check(want=want)
    c.ctx.close()


@pytest.mark.parametrize("hint", [0, 400, 3000, 100000])
def test_a_hint_steers_the_way_and_not_the_result(hint):
    """A table with room for far more than the sequences have: the expected length chooses between the ways of reading their own keys."""
    c = Case(6, 1, 8, 2, 256, [100, 3, 0, 1200], 64, seed=14, cap=8192)
    c.device(_binding(), option=(_binding().OPT_KV_LEN_HINT, hint))
    c.call()
    assert c.ctx.status_poll() == 0
    c.check()
    c.ctx.close()


def test_agrees_with_the_call_that_shares_nothing():
    c = Case(4, 60, 28, 4, 1500, [354, 46, 0, 200], 16, True, seed=5)
    c.device(_binding())
    c.call()
    other, lse = torch.empty_like(c.out), torch.empty_like(c.lse)
    c.given[:, :c.shared] = c.table[:, :c.shared]
    table = torch.from_numpy(c.given).cuda()
    c.ctx.tree_verify_attn_paged(0, c.qd, c.kvd, table, c.md, SCALE, other, lse)
    assert c.ctx.status_poll() == 0
    # both round their weights and their output; the weights' roundings differ by the reference that exponents are taken from
    _, _, a = c.want()
    d = np.abs(c.out.float().cpu().numpy() - other.float().cpu().numpy())
    assert (d <= 2.0 ** -7 * (2 * a) + 1e-3 * a).all() and (c.lse - lse).abs().max() <= 1e-3
    c.ctx.close()


def test_masks_that_leave_rows_nothing():
    c = Case(3, 70, 4, 2, 0, [0, 0, 200], 16, seed=9)
    c.mask[0] = 0                                             # nothing committed, nothing visible: empty rows
    c.mask[1, 5:9] = 0
    c.mask[2] = 0                                             # committed keys only
    c.device(_binding())
    c.call()
    assert c.ctx.status_poll() == 0
    out, lse = c.out.float().cpu().numpy(), c.lse.cpu().numpy()
    assert (out[0] == 0).all() and np.isneginf(lse[0]).all()
    assert (out[1, 5:9] == 0).all() and np.isneginf(lse[1, :, 5:9]).all()
    c.check()
    c.ctx.close()
    # bits at and beyond N are no nodes
    c = Case(2, 70, 4, 2, 256, [0, 100], 32, seed=10)
    want = c.want()
    c.mask[:, :, 1] |= np.uint64(0xFFFFFFFFFFFFFFFF) << np.uint64(6)
    c.device(_binding())
    c.call()
    c.check(want=want)
    c.ctx.close()


def test_sequences_that_do_not_fit():
    for bad in (255, -1, -2 ** 31, 2 ** 31 - 1, 640 - 4):     # below the shared slots; kv_len + N beyond the table
        c = Case(3, 5, 4, 2, 256, [100, 60, 0], 16, seed=3, cap=640)
        want = c.want()
        c.device(_binding())
        c.kvd[1] = bad
        c.call()
        assert c.ctx.status_poll() == E_RANGE
        assert (c.out[1] == 0).all() and (c.lse[1] == -math.inf).all()
        c.check(rows=[0, 2], want=want)
        c.ctx.close()
    c = Case(2, 5, 4, 2, 256, [100, 60], 16, seed=3, cap=640)
    c.device(_binding())
    c.kvd.fill_(3)                                            # nobody fits
    c.call()
    assert c.ctx.status_poll() == E_RANGE and (c.out == 0).all() and (c.lse == -math.inf).all()
    c.ctx.close()


def test_table_entries_outside_the_pool_read_as_zeros():
    for entry in (-1, 2 ** 31 - 1):
        c = Case(2, 5, 4, 2, 256, [100, 60], 16, seed=4)
        for x in (c.k, c.v):
            x[:, :, 32:48] = 0                                # a shared block, and one of the second sequence's own
            x[1, :, 288:304] = 0
        c.device(_binding())
        c.td[0, 2] = entry
        c.td[1, 18] = entry
        c.call()
        assert c.ctx.status_poll() == E_RANGE
        c.check()
        c.ctx.close()


@pytest.mark.parametrize("value", [0x7FC0, 0x7F80])
def test_a_key_that_is_not_finite(value):
    """A NaN score, or +inf, makes the rows that may see it NaN and leaves the others as they were."""
    c = Case(3, 6, 4, 2, 300, [140, 33, 10], 16, seed=6)
    want = c.want()
    c.device(_binding())
    import gpu_util as gu
    kp = c.pools[0].copy()
    at = 300 + 33 + 3                                         # tree row 3 of the second sequence, kv head 0
    kp[c.table[1, at // 16], 0, at % 16] = value
    c.kd.copy_(gu.bf16_dev(kp))
    c.call()
    out, lse = c.out.float().cpu().numpy(), c.lse.cpu().numpy()
    sees = (c.mask[1, :, 0] >> np.uint64(3)) & np.uint64(1) == 1
    assert sees.any() and not sees.all()
    if value == 0x7FC0:
        assert np.isnan(out[1, sees, :2]).all() and np.isneginf(lse[1, :2][:, sees]).all()
    assert np.isfinite(out[1, :, 2:]).all() and np.isfinite(out[[0, 2]]).all() and np.isfinite(out[1, ~sees]).all()
    c.check(rows=[0, 2], want=want)
    c.ctx.close()


def test_calls_on_two_streams_with_scratch_of_their_own():
    c = Case(4, 30, 8, 2, 700, [100, 20, 0, 250], 16, seed=8)
    c.device(_binding())
    want = c.want()
    other = torch.full_like(c.out, float("nan"))
    s2 = c.ctx.prefix_scratch(4, 30)
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


def test_captured_calls_follow_lengths_and_table():
    c = Case(4, 8, 8, 2, 512, [100, 20, 0, 250], 16, seed=12)
    c.device(_binding())
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c.call()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            for _ in range(3):                                # back to back on one scratch
                c.call()
        for own in ([100, 20, 0, 250], [0, 0, 0, 0], [7, 250, 130, 1]):
            c.kv_len[:] = 512 + np.array(own)
            c.kvd.copy_(torch.from_numpy(c.kv_len))
            for b in range(4):                                # entries and rows that longer sequences need
                c.given[b, c.shared:] = c.table[b, c.shared:]
            c.td.copy_(torch.from_numpy(c.given))
            import gpu_util as gu
            for d, src in ((c.kd, c.k), (c.vd, c.v)):
                pool = gu.bf16_bits(d)
                blocks = src.reshape(4, 2, c.per, 16, 128).transpose(0, 2, 1, 3, 4)
                for b in range(4):
                    pool[c.table[b, c.shared:]] = blocks[b, c.shared:]
                d.copy_(gu.bf16_dev(pool))
            c.out.fill_(float("nan"))
            graph.replay()
            side.synchronize()
            c.check()
        assert c.ctx.status_poll() == 0
    c.ctx.close()


def test_blocks_beyond_32_bit_offsets():
    """Rows in the last blocks of a pool of more than 2^32 bytes and 2^31 elements, appended and then attended to."""
    b = _binding()
    Hq, Hkv, page, N = 4, 4, 128, 1
    nb = 2 ** 31 // (Hkv * page * 128) + 40
    kp, vp = (torch.empty((nb, Hkv, page, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B, P, own = 2, 256, 140
    ctx = b.VerifyContext(B, N, Hq, Hkv, 128, 512, 1)
    ctx.cache_register_paged(0, kp, vp)
    last = nb - 1
    table = torch.tensor([[last, last - 1, last - 2, last - 3], [last, last - 1, last - 4, last - 5]], dtype=torch.int32, device="cuda")
    k, v = (torch.randn((P + 2 * (own + 1), Hkv, 128), device="cuda").bfloat16() for _ in range(2))
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    ctx.kv_append_paged(0, None, k[:P], v[:P], None, None, i32(0, P, P), i32(0, 0), table)
    ctx.kv_append_paged(0, None, k[P:], v[P:], None, None, i32(0, own + 1, 2 * own + 2), i32(P, P), table)
    q = torch.randn((B, N, Hq, 128), device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty((B, Hq, N), device="cuda")
    mask = torch.ones((B, N, 1), dtype=torch.int64, device="cuda")
    ctx.tree_verify_attn_prefix_paged(0, q, i32(P + own, P + own), table, P, mask, SCALE, ctx.prefix_scratch(B, N), out, lse)
    assert ctx.status_poll() == 0
    for s in range(B):
        rows = torch.cat([torch.arange(P), P + s * (own + 1) + torch.arange(own + 1)]).cuda()
        kk, vv = k[rows].double(), v[rows].double()
        p = torch.softmax(SCALE * torch.einsum("hd,khd->hk", q[s, 0].double(), kk), -1)
        want, a = torch.einsum("hk,khd->hd", p, vv), torch.einsum("hk,khd->hd", p, vv.abs())
        assert ((out[s, 0].double() - want).abs() <= 2.0 ** -8 * (a + want.abs()) + 6e-4 * a).all()
    ctx.close()


def test_a_prompt_from_its_rows_to_a_verified_draft():
    """The operators as they are used: an image prompt rotated by three axes into the pool, the samples' own tokens behind it, the
    tree's rows, the shared-prefix attention, acceptance and commit, and the attention of the next cycle."""
    b = _binding()
    import gpu_util as gu
    B, N, Hq, Hkv, P, page, S = 3, 12, 8, 2, 320, 16, 512
    rng = np.random.default_rng(1)
    ctx = b.VerifyContext(B, N, Hq, Hkv, 128, S, 1)
    per, shared = S // page, P // page
    nb = shared + B * (per - shared)
    perm = rng.permutation(nb).astype(np.int32)
    table = np.concatenate([np.tile(perm[:shared], (B, 1)), perm[shared:].reshape(B, -1)], 1)
    kp, vp = (torch.zeros((nb, page, Hkv, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx.cache_register_paged(0, kp, vp, True)
    td, ax = gu.i32_dev(table), b.RopeAxes((16, 24, 24), 1e6)
    rows = lambda T, H: torch.randn((T, H, 128), device="cuda").bfloat16()
    i32 = gu.i32_dev
    # the prompt, through the first sequence's row of the table; then 5, 0 and 40 tokens of each sample
    pos = np.tile(np.arange(P), (3, 1))
    pos[0, 20:276], pos[1, 20:276], pos[2, 20:276] = 20, 20 + np.arange(256) // 16, 20 + np.arange(256) % 16
    pos[:, 276:] = 36 + np.arange(P - 276)
    start = torch.zeros(B, dtype=torch.int32, device="cuda")
    lens = torch.zeros_like(start)
    ctx.kv_append_paged(0, None, rows(P, Hkv), rows(P, Hkv), i32(pos), ax, i32([0, P, P, P]), start, td, None, lens)
    assert lens.tolist() == [P, 0, 0]
    lens.fill_(P)
    new = torch.zeros_like(lens)
    ctx.kv_append_paged(0, None, rows(45, Hkv), rows(45, Hkv), i32(np.tile(np.arange(45), (3, 1)) + 80), ax, i32([0, 5, 5, 45]), lens,
                        td, None, new)
    assert new.tolist() == [P + 5, P, P + 40]
    parents = np.stack([synth.draw_tree(N, 4, 3, np.random.Generator(np.random.Philox(7))) for _ in range(B)])
    mask = torch.zeros((B, N, 1), dtype=torch.int64, device="cuda")
    scratch = ctx.prefix_scratch(B, N)
    for cycle in range(2):
        ctx.tree_mask_build(i32(parents), mask, None)
        q = rows(B * N, Hq).view(B, N, Hq, 128)
        ctx.rope_tree_rows_paged(0, q, rows(B * N, Hkv).view(B, N, Hkv, 128), rows(B * N, Hkv).view(B, N, Hkv, 128),
                                 (new[:, None] + torch.arange(N, device="cuda")[None]).int().contiguous(), new, td, 1e6)
        out = torch.empty_like(q)
        lse = torch.empty((B, Hq, N), device="cuda")
        ctx.tree_verify_attn_prefix_paged(0, q, new, td, P, mask, SCALE, scratch, out, lse)
        assert ctx.status_poll() == 0

        def flat(pool):
            x = gu.bf16_bits(pool)[table]                     # [B, per, page, Hkv, D]
            return np.ascontiguousarray(x.reshape(B, S, Hkv, 128).transpose(0, 2, 1, 3))
        kv = new.cpu().numpy()
        args = (gu.bf16_bits(q), flat(kp))
        want, want_lse = oracle.tree_attn(*args, flat(vp), kv, gu.u64_host(mask), SCALE)
        a, _ = oracle.tree_attn(*args, flat(vp) & np.uint16(0x7FFF), kv, gu.u64_host(mask), SCALE)
        err = np.abs(out.float().cpu().numpy() - want)
        assert (err <= 2.0 ** -8 * (a + np.abs(want)) + 6e-4 * a).all() and np.abs(lse.cpu().numpy() - want_lse).max() <= 5e-4
        ids = i32(rng.integers(0, 2, size=(B, N)))
        target = i32(rng.integers(0, 2, size=(B, N)))
        path, alen, bonus, after = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((B, N), (B,), (B,), (B,)))
        ctx.accept_commit_paged(0, 1, ids, target, i32(parents), new, td, path, alen, bonus, after)
        assert ctx.status_poll() == 0 and (after == new + alen).all()
        new = after
    ctx.close()


def test_refusals():
    b = _binding()
    E_NULL, E_ALIGN, E_SHAPE, E_UNSUP, E_UNREG, E_WS = -1, -2, -3, -5, -9, -10
    c = Case(2, 3, 4, 2, 64, [10, 20], 16, seed=2)
    ctx = c.device(b, layers=3)
    flat = torch.zeros((2, 2, c.per * 16, 128), dtype=torch.bfloat16, device="cuda")
    ctx.cache_register(1, flat, flat)

    def call(layer=0, q=c.qd, kv=c.kvd, td=c.td, P=64, m=c.md, scale=SCALE, s=c.scratch, out=c.out, lse=c.lse):
        ctx.tree_verify_attn_prefix_paged(layer, q, kv, td, P, m, scale, s, out, lse)

    def refused(code, **kw):
        with pytest.raises(b.VispecError) as e:
            call(**kw)
        assert e.value.code == code

    call()
    refused(E_RANGE, layer=3)
    refused(E_RANGE, layer=-1)
    refused(E_UNREG, layer=2)
    refused(E_UNSUP, layer=1)
    refused(E_RANGE, P=-1)
    refused(E_RANGE, P=c.per * 16 + 1)
    refused(E_UNSUP, scale=0.0)
    refused(E_UNSUP, scale=-1.0)
    refused(E_UNSUP, scale=float("nan"))
    refused(E_WS, s=c.scratch[:-16])
    refused(E_ALIGN, s=c.scratch[4:])
    more = torch.zeros((3, 3, 4, 128), dtype=torch.bfloat16, device="cuda")
    refused(E_SHAPE, q=more, kv=torch.zeros(3, dtype=torch.int32, device="cuda"), td=c.td[:1].expand(3, -1).contiguous(),
            m=c.md[:1].expand(3, -1, -1).contiguous(), out=torch.zeros_like(more), lse=None)
    for kw in (dict(q=c.qd.float()), dict(q=c.qd[:, :, :2]), dict(kv=c.kvd.long()), dict(kv=c.kvd[:1]), dict(td=c.td[:1]), dict(out=c.out[:1]),
               dict(lse=c.lse.double()), dict(m=c.md[:1]), dict(q=c.qd.cpu()), dict(s=c.scratch.float()), dict(lse=c.lse.transpose(1, 2))):
        with pytest.raises((ValueError, TypeError)):
            call(**kw)
    for kw in (dict(q=None), dict(out=None), dict(s=None), dict(kv=None)):
        with pytest.raises(TypeError):
            call(**kw)
    n = ctypes.c_size_t()
    lib = ctx.lib
    assert lib.vispec_prefix_scratch_bytes(ctx.handle, 3, 3, ctypes.byref(n)) == E_SHAPE
    assert lib.vispec_prefix_scratch_bytes(ctx.handle, 2, 0, ctypes.byref(n)) == E_SHAPE
    assert lib.vispec_prefix_scratch_bytes(ctx.handle, 2, 3, None) == E_NULL
    z = ctypes.c_void_p(0)
    assert lib.vispec_tree_verify_attn_prefix_paged(z, 0, z, z, z, 1, 0, z, 1, 1, 1.0, z, 0, z, z, z) == E_NULL
    assert ctx.status_poll() == 0
    ctx.close()
    # more than 8 rows per sequence and kv head: at most 64 sequences
    big = b.VerifyContext(65, 5, 4, 2, 128, 128, 1)
    pool = torch.zeros((8, 2, 16, 128), dtype=torch.bfloat16, device="cuda")
    big.cache_register_paged(0, pool, pool)
    for N, fine in ((5, False), (4, True)):
        q = torch.zeros((65, N, 4, 128), dtype=torch.bfloat16, device="cuda")
        args = (0, q, torch.zeros(65, dtype=torch.int32, device="cuda"), torch.zeros((65, 8), dtype=torch.int32, device="cuda"), 0,
                torch.ones((65, N, 1), dtype=torch.int64, device="cuda"), SCALE, big.prefix_scratch(65, N), q.clone())
        if fine:
            big.tree_verify_attn_prefix_paged(*args)
        else:
            with pytest.raises(b.VispecError) as e:
                big.tree_verify_attn_prefix_paged(*args)
            assert e.value.code == E_UNSUP
    assert big.status_poll() == 0
    big.close()
