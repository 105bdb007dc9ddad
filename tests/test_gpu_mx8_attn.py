"""Attention over the quantised cache against float64, element by element.

Bound: the output is rounded to bf16 (half a step, 2^-8 of |o|) and each probability is rounded to bf16 for
its product with the value (2^-8 of p, so 2^-8 of A = sum p |v| at most); fp32 scores, exponentials and sums
add, relative to p, at most 2^-17 (1 + |score|): scores of up to 128 products accumulate with 2^-17 of
their largest term in the worst case, exp2 and the sums with less.  So |error| <= 2^-8 |o| + 2^-8 (1 + 2^-6) A
+ 2^-17 A (1 + max |score|).  The log-sum-exp: 2^-17 (1 + max |score|).  Everything is checked, nothing sampled.

Where single products are large there is a term of its own.  The 8-bit matrix instruction adds the 16 products of
a 16-dimension group, and the accumulator, after cutting each below 2^-13 of the largest one's power of
two (1.125 beside 2^10 is kept whole, beside 2^11 its eighth is lost, beside 2^14 all of it: measured), so a
score is off by at most E = 17 * 2^-13 * (sum over the 8 groups of their largest |q_i k_i|), each weight by a
factor within 2^(+-2E) after normalisation, and the output by sum p (2^2E - 1) |v| more, the log-sum-exp by E.
"""
import numpy as np
import pytest
import torch

from oracle import mx8
from oracle.numerics import bf16_to_f64
from tests.gpu_helpers import dev, host, log

pytestmark = pytest.mark.gpu

u = pytest.importorskip("paper_2609_32518_amd")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)


def quantised(shape, seed, scale=1.0):
    y = np.random.default_rng(seed).standard_normal(shape) * scale
    return mx8.quantise(y)


def put(codes, scale):
    return torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn), torch.from_numpy(scale).cuda()


class Case:
    """A quantised cache filled with seeded rows, and queries."""

    def __init__(self, B, H, gh, gw, S, R, f0, C, W, seed=1, q_scale=0.1275, guard=0):
        self.a = (f0, C, W)
        T = gh * gw
        slots, N = (S + R) * T, C * T
        self.k, self.v = quantised((B, H, slots, 128), seed), quantised((B, H, slots, 128), seed + 1)
        self.q = quantised((B, N, H, 128), seed + 2, q_scale)
        lo = max(0, f0 - W)
        frames = list(range(min(S, lo))) + list(range(lo, f0 + C))
        self.rows = np.concatenate([(f if f < S else S + (f - S) % R) * T + np.arange(T) for f in frames])
        outside = np.setdiff1d(np.arange(slots), self.rows)
        for codes, scale in (self.k, self.v):                  # rows outside the window hold anything
            codes[:, :, outside], scale[:, :, outside] = 0x7F, 0xFF
        self.geometry = (B, H, gh, gw, S, R)
        self.make()

    def make(self):
        k8, ks = put(*self.k)
        v8, vs = put(*self.v)
        self.cache = u.CacheMX8(*self.geometry, k8=k8, k_scale=ks, v8=v8, v_scale=vs)
        for f in range(self.a[0] + self.a[1]):
            self.cache.advance(f, 1)
        self.q8, self.qs = put(*self.q)

    def expected(self):
        B, N, H = self.q[0].shape[:3]
        o, A = np.empty((B, N, H, 128)), np.empty((B, N, H, 128))
        lse, top = np.empty((B, H, N)), 0.0
        q = mx8.values(*self.q)
        for b in range(B):
            for h in range(H):
                k = mx8.values(self.k[0][b, h, self.rows], self.k[1][b, h, self.rows])
                v = mx8.values(self.v[0][b, h, self.rows], self.v[1][b, h, self.rows])
                o[b, :, h], lse[b, h], A[b, :, h] = mx8.attention(q[b, :, h], k, v)
                top = max(top, float(np.abs(q[b, :, h] @ k.T).max()))
        return o, lse, A, top

    def cut(self):
        """E above, at most, over all queries and keys."""
        q, k = mx8.values(*self.q), mx8.values(self.k[0][:, :, self.rows], self.k[1][:, :, self.rows])
        q, k = (np.abs(t).reshape(t.shape[:-1] + (8, 16)) for t in (q.transpose(0, 2, 1, 3), k))
        # the largest product of a group is at most that of the dimension's largest q and largest k
        return 17 * 2.0 ** -13 * float((q.max(axis=2) * k.max(axis=2)).max(axis=-1).sum(axis=-1).max())

    def check(self, out, lse, want=None, E=0.0):
        o, wl, A, top = want or self.expected()
        got = bf16_to_f64(host(out))
        bound = 2.0 ** -8 * np.abs(o) + 2.0 ** -8 * (1 + 2.0 ** -6) * A + 2.0 ** -17 * A * (1 + top) + A * (4.0 ** E - 1)
        err = np.abs(got - o)
        assert np.isfinite(got).all()
        assert (err <= bound).all(), float((err / bound).max())
        if lse is not None:
            assert np.abs(lse.double().cpu().numpy() - wl).max() <= 2.0 ** -17 * (1 + top) + E

    def run(self, **kw):
        B, N, H = self.q[0].shape[:3]
        lse = torch.full((B, H, N), 9.0, device="cuda")
        out = self.cache.unstep_window_attn_mx8(*self.a, self.q8, self.qs, lse=lse, **kw)
        return out, lse


SHAPES = [  # B, H, gh, gw, S, R, f0, C, W
    (1, 1, 1, 1, 0, 1, 0, 1, 0),            # one key
    (2, 3, 1, 1, 0, 4, 2, 2, 1),            # three keys of two queries
    (1, 2, 1, 1, 2, 70, 100, 1, 63),        # one token, sinks, a tile and two keys
    (2, 3, 1, 1, 0, 600, 900, 1, 599),      # one token over a wrapped ring
    (1, 12, 1, 1, 0, 5000, 5200, 1, 4999),  # one token, many tiles, split
    (1, 1, 1, 1, 1, 3000, 3100, 3, 2000),   # three tokens
    (1, 5, 3, 5, 1, 4, 9, 1, 3), (1, 2, 4, 8, 0, 30, 33, 1, 29), (2, 2, 3, 11, 0, 40, 45, 1, 38),
    (1, 3, 5, 13, 2, 7, 20, 1, 5), (1, 2, 7, 9, 0, 5, 4, 1, 4),
    (1, 2, 8, 16, 0, 12, 30, 2, 9), (1, 1, 16, 16, 0, 3, 2, 1, 2), (2, 5, 17, 23, 2, 8, 17, 2, 5),
    (1, 24, 13, 30, 0, 9, 8, 1, 7), (1, 3, 30, 52, 3, 6, 9, 3, 3),
    (1, 16, 4, 4, 0, 90, 89, 1, 89), (1, 16, 1, 17, 0, 90, 89, 1, 89),     # either side of the few-query kernel
    (1, 130, 4, 5, 0, 80, 79, 1, 79),       # more query tiles than half the chip: one contiguous split of all of them
    (2, 66, 4, 5, 2, 90, 200, 1, 85),       # the same over two runs
    (1, 300, 4, 5, 0, 70, 69, 1, 69)]       # more query tiles than compute units, split


@pytest.mark.parametrize("shape", SHAPES)
def test_every_element(shape):
    c = Case(*shape)
    if shape[1] * shape[0] > 128:                              # the general kernel: work-groups that no tile divides
        assert c.cache.workspace_bytes(*c.a) == 256 * 2 * 256 * 130 * 4
    want = c.expected()
    for split in (True, False):
        log(f"{shape} split={split}")
        c.check(*c.run(use_split=split), want)


# Small chunks in groups of 16 queries: batch, odd sizes, sinks and a wrapped ring, a last group of one, a range of one
# wave, and the first sizes past those (the general kernel)
SMALL = [(3, 3, 1, 18, 0, 23, 22, 1, 22), (2, 5, 3, 7, 2, 9, 30, 1, 8), (1, 2, 17, 23, 1, 4, 9, 1, 3), (1, 24, 1, 33, 0, 6, 5, 2, 4),
         (1, 15, 7, 37, 0, 3, 2, 1, 0), (2, 1, 30, 52, 0, 2, 1, 1, 0), (1, 12, 1, 17, 0, 30, 29, 1, 29), (1, 7, 17, 17, 1, 5, 14, 2, 3),
         (1, 2, 16, 20, 0, 12, 30, 2, 9),
         (1, 1, 28, 27, 1, 6, 12, 1, 4), (2, 3, 1, 259, 0, 9, 8, 1, 8), (1, 4, 16, 16, 0, 17, 16, 1, 16), (1, 5, 1, 20, 2, 300, 400, 1, 250)]


@pytest.mark.parametrize("shape", SMALL)
def test_small_chunks(shape):
    c = Case(*shape)
    want = c.expected()
    guard = torch.full((c.q8.shape[0] + 1,) + tuple(c.q8.shape[1:]), 3.0, device="cuda", dtype=torch.bfloat16)
    for split in (True, False):
        c.check(*c.run(use_split=split, out=guard[:-1]), want)
        assert (guard[-1] == 3.0).all()


@pytest.mark.parametrize("shape", [(1, 2, 8, 16, 0, 5, 4, 1, 4), (1, 2, 16, 20, 0, 12, 30, 2, 9)])
def test_small_chunks_whose_scores_grow_or_vanish(shape):
    """Both kernels: scores that grow by hundreds, then a run of keys whose scores are -infinity, then a NaN key."""
    c = Case(*shape, q_scale=1.0)
    n = len(c.rows)
    q, k = mx8.values(*c.q), mx8.values(*c.k)
    q[..., 0], k[..., 0] = 8.0, 0.0
    k[:, :, c.rows, 0] = np.linspace(-40, 40, n)
    c.q, c.k = mx8.quantise(q), mx8.quantise(k)
    c.make()
    for split in (True, False):
        c.check(*c.run(use_split=split), E=c.cut())
    c = Case(*shape)
    q, k = mx8.values(*c.q), mx8.values(*c.k)
    q[..., 0], k[..., 0] = 2.0 ** 66, 0.0
    k[:, :, c.rows[:n // 2], 0] = -2.0 ** 66
    c.q, c.k = mx8.quantise(q), mx8.quantise(k)
    c.make()
    every, c.rows = c.rows, c.rows[n // 2:]
    c.check(*c.run(), c.expected())
    c.cache.k8.view(torch.uint8)[0, 1, int(every[-1]), 100] = 0x7F
    out, lse = c.run()
    assert torch.isnan(out[:, :, 1]).all() and torch.isnan(lse[:, 1]).all()
    assert torch.isfinite(out[:, :, 0]).all() and torch.isfinite(lse[:, 0]).all()


@pytest.mark.parametrize("shape", [SHAPES[4], SHAPES[12], SHAPES[13]])
def test_scratch_of_any_size(shape):
    """No scratch, too little, a part of it: fewer parts, the same result within the bound."""
    c = Case(*shape)
    want = c.expected()
    need = c.cache.workspace_bytes(*c.a)
    for n in sorted({0, 16, need // 3 // 16 * 16, need}):
        ws = torch.full((n + 64,), 255, dtype=torch.uint8, device="cuda")
        out, lse = c.run(workspace=ws[:n])
        c.check(out, lse, want)
        assert (ws[n:] == 255).all()


@pytest.mark.parametrize("shape,step", [((1, 130, 4, 5, 0, 80, 79, 1, 79), 30.0), ((1, 2, 8, 16, 0, 12, 30, 2, 9), 40.0), ((1, 3, 1, 1, 0, 900, 900, 1, 899), 60.0),
                                        ((2, 1, 16, 17, 0, 8, 9, 2, 5), 25.0)])
def test_scores_that_grow_along_the_keys(shape, step):
    """Later keys score hundreds of units above the first ones: sums and outputs stay finite and right."""
    c = Case(*shape, q_scale=1.0)
    n = len(c.rows)
    q, k = mx8.values(*c.q), mx8.values(*c.k)
    q[..., 0], k[..., 0] = 8.0, 0.0
    k[:, :, c.rows, 0] = np.linspace(-step, step, n)
    c.q, c.k = mx8.quantise(q), mx8.quantise(k)
    c.make()
    for split in (True, False):
        c.check(*c.run(use_split=split), E=c.cut())
    k[:, :, c.rows, 0] = np.linspace(step, -step, n)           # and fall
    c.k = mx8.quantise(k)
    c.make()
    c.check(*c.run(), E=c.cut())


@pytest.mark.parametrize("shape", [(1, 2, 8, 16, 0, 12, 30, 2, 9), (2, 1, 16, 17, 0, 8, 9, 2, 5), (1, 3, 1, 1, 0, 900, 900, 1, 899)])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_that_grow_in_every_dimension(shape, sign):
    """The same spread over the head: equal products, of which none is cut, so the plain bound holds."""
    c = Case(*shape)
    q, k = mx8.values(*c.q), mx8.values(*c.k)
    n = len(c.rows)
    steps = np.repeat(np.arange(-(n // 64), n - n // 64, dtype=np.float64), 16)[:n] * sign
    steps = np.clip(np.round(steps / max(1.0, np.abs(steps).max()) * 7), -7, 7)    # -7 .. 7: exact in e4m3
    q[:], k[:, :, c.rows] = 0.375, steps[:, None]                                  # scores 48 steps: -336 .. 336
    c.q, c.k = mx8.quantise(q), mx8.quantise(k)
    c.make()
    for split in (True, False):
        c.check(*c.run(use_split=split))


def check_without_lse(c, want, E=0.0, **kw):
    """A call without a log-sum may divide by the sum of the rounded weights: p (1 + d), |d| <= 2^-8, above and below,
    so besides the output's own rounding the error is at most 2^-8 (A + |o|) (1 + 2^-7) <= 2^-7 (1 + 2^-7) A, and the
    terms of fp32 and of the 8-bit products as above."""
    o, _, A, top = want
    got = bf16_to_f64(host(c.cache.unstep_window_attn_mx8(*c.a, c.q8, c.qs, **kw)))
    bound = 2.0 ** -8 * np.abs(o) * (1 + 2.0 ** -7) + 2.0 ** -7 * (1 + 2.0 ** -6) * A + 2.0 ** -17 * A * (1 + top) + A * (4.0 ** E - 1)
    assert np.isfinite(got).all()
    assert (np.abs(got - o) <= bound).all(), float((np.abs(got - o) / bound).max())


@pytest.mark.parametrize("shape", [SHAPES[i] for i in (2, 9, 11, 13, 14, 15, 17, 18, 19, 20)] + [(1, 12, 16, 31, 0, 6, 5, 1, 5)])
def test_without_a_log_sum(shape):
    c = Case(*shape)
    want = c.expected()
    for split in (True, False):
        check_without_lse(c, want, use_split=split)


@pytest.mark.parametrize("shape", [(1, 130, 4, 5, 0, 80, 79, 1, 79), (1, 2, 16, 20, 0, 12, 30, 2, 9)])
def test_hard_scores_without_a_log_sum(shape):
    """Scores that grow by hundreds; keys whose scores are -infinity; a NaN query, which leaves every other alone."""
    c = Case(*shape, q_scale=1.0)
    n = len(c.rows)
    q, k = mx8.values(*c.q), mx8.values(*c.k)
    q[..., 0], k[..., 0] = 8.0, 0.0
    k[:, :, c.rows, 0] = np.linspace(-40, 40, n)
    c.q, c.k = mx8.quantise(q), mx8.quantise(k)
    c.make()
    for split in (True, False):
        check_without_lse(c, c.expected(), E=c.cut(), use_split=split)
    c = Case(*shape)
    q, k = mx8.values(*c.q), mx8.values(*c.k)
    q[..., 0], k[..., 0] = 2.0 ** 66, 0.0
    k[:, :, c.rows[:n // 2], 0] = -2.0 ** 66
    c.q, c.k = mx8.quantise(q), mx8.quantise(k)
    c.make()
    c.rows = c.rows[n // 2:]
    check_without_lse(c, c.expected())
    c = Case(*shape)
    o, _, A, top = c.expected()
    c.q8.view(torch.uint8)[0, 3, 1, 77] = 0xFF
    for split in (True, False):
        out = c.cache.unstep_window_attn_mx8(*c.a, c.q8, c.qs, use_split=split)
        assert torch.isnan(out[0, 3, 1]).all()
        got = bf16_to_f64(host(out))
        got[0, 3, 1] = o[0, 3, 1]
        assert (np.abs(got - o) <= 2.0 ** -6 * A + 2.0 ** -17 * A * (1 + top)).all()


def test_equal_keys_give_the_mean():
    c = Case(1, 2, 3, 7, 0, 6, 5, 1, 5)
    c.q = (np.zeros_like(c.q[0]), c.q[1])
    c.make()
    out, lse = c.run()
    c.check(out, lse)
    assert np.abs(lse.cpu().numpy() - np.log(len(c.rows))).max() < 1e-6


def test_large_scales_and_one_head_of_nan():
    """Blocks of very different scales, and a NaN key that spoils its own head only."""
    c = Case(1, 3, 4, 9, 0, 9, 8, 1, 8)
    q, k, v = mx8.values(*c.q), mx8.values(*c.k), mx8.values(*c.v)
    q[..., :32] *= 2.0 ** 40
    k[..., :32] *= 2.0 ** -40
    v *= np.exp2(np.random.default_rng(4).integers(-30, 30, (1, 3, 1, 4)).repeat(32, -1))
    c.q, c.k, c.v = mx8.quantise(q), mx8.quantise(k), mx8.quantise(v)
    c.make()
    want = c.expected()
    c.check(*c.run(), want)
    c.cache.k8.view(torch.uint8)[0, 1, int(c.rows[-1]), 100] = 0x7F
    out, lse = c.run()
    assert torch.isnan(out[0, :, 1]).all() and torch.isnan(lse[0, 1]).all()
    keep = lambda t: t[:, :, [0, 2]]  # noqa: E731
    got = bf16_to_f64(host(out[:, :, [0, 2]].contiguous()))
    assert (np.abs(got - keep(want[0])) <= 2.0 ** -7 * keep(want[2]) + 2.0 ** -17 * keep(want[2]) * (1 + want[3])).all()


@pytest.mark.parametrize("shape,hidden", [((1, 2, 8, 16, 0, 12, 30, 2, 9), 700), ((1, 2, 8, 16, 0, 12, 30, 2, 9), 40), ((1, 3, 1, 1, 0, 900, 900, 1, 899), 300),
                                          ((2, 1, 3, 3, 0, 9, 8, 1, 8), 40), ((1, 5, 1, 1, 0, 5000, 5200, 1, 4999), 2000)])
@pytest.mark.parametrize("where", ["first", "last"])
def test_scores_of_minus_infinity_weigh_nothing(shape, hidden, where):
    """Products that overflow to -infinity for a run of keys: the others' attention, also where a tile, a wave's or
    a work-group's whole share is such keys."""
    c = Case(*shape)
    q, k = mx8.values(*c.q), mx8.values(*c.k)
    gone = c.rows[:hidden] if where == "first" else c.rows[-hidden:]
    q[..., 0], k[..., 0] = 2.0 ** 66, 0.0
    k[:, :, gone, 0] = -2.0 ** 66
    c.q, c.k = mx8.quantise(q), mx8.quantise(k)
    c.make()
    c.rows = np.setdiff1d(c.rows, gone)
    want = c.expected()
    for split in (True, False):
        c.check(*c.run(use_split=split), want)


@pytest.mark.parametrize("shape", [(1, 2, 1, 1, 0, 5000, 5200, 1, 4999), (1, 2, 8, 16, 0, 12, 30, 2, 9)])
@pytest.mark.parametrize("key", [0, 1000, -1])
def test_a_nan_key_reaches_output_and_log_sum(shape, key):
    """In one part of a split range as in the whole one."""
    c = Case(*shape)
    c.cache.k8.view(torch.uint8)[0, 1, int(c.rows[key]), 3] = 0x7F
    for split in (True, False):
        out, lse = c.run(use_split=split)
        assert torch.isnan(out[:, :, 1]).all() and torch.isnan(lse[:, 1]).all()
        assert torch.isfinite(out[:, :, 0]).all() and torch.isfinite(lse[:, 0]).all()


def test_rows_past_two_gigabytes():
    """Offsets past 2^32 bytes: the last head of a cache whose rows lie beyond."""
    H, R, W = 34, 1024 * 1024, 2048
    free = torch.cuda.mem_get_info()[0]
    if free < 24 << 30:
        pytest.skip("needs 24 GiB of device memory")
    c = u.CacheMX8(1, H, 1, 1, 0, R)
    assert c.k8.numel() > 2 ** 32
    f0 = R - 1
    k, v = quantised((1, 1, W + 1, 128), 5), quantised((1, 1, W + 1, 128), 6)
    for dst, sc, (codes, scale) in ((c.k8, c.k_scale, k), (c.v8, c.v_scale, v)):
        dst.view(torch.uint8)[:, -1:, R - W - 1:].copy_(torch.from_numpy(codes))
        sc.fill_(127)
        sc[:, -1:, R - W - 1:].copy_(torch.from_numpy(scale))
    for f in range(0, R, 2048):
        c.advance(f, 2048)
    q = quantised((1, 1, H, 128), 7, 0.1275)
    q8, qs = put(*q)
    out = c.unstep_window_attn_mx8(f0, 1, W, q8, qs)
    o, _, A = mx8.attention(mx8.values(*q)[0, :, -1], mx8.values(k[0][0, 0], k[1][0, 0]), mx8.values(v[0][0, 0], v[1][0, 0]))
    assert (np.abs(bf16_to_f64(host(out))[0, :, -1] - o) <= 2.0 ** -7 * (1 + 2.0 ** -5) * A).all()
    kk, vv = c.unstep_kv_read_mx8(R - 3, 3)
    assert np.array_equal(bf16_to_f64(host(kk))[0, :, -1], mx8.values(k[0][0, 0, -3:], k[1][0, 0, -3:]))
    assert np.array_equal(bf16_to_f64(host(vv))[0, :, -1], mx8.values(v[0][0, 0, -3:], v[1][0, 0, -3:]))


@pytest.mark.parametrize("gh,gw,C,W,S,R,norm", [(1, 1, 1, 40, 0, 48, False), (4, 6, 2, 5, 1, 8, True), (16, 18, 1, 5, 0, 6, False)])
def test_stream_of_steps(gh, gw, C, W, S, R, norm):
    """A clip through unstep_step_mx8: each step equals append + attention bit for bit, its cache equals what
    the appends wrote, and its output is right against float64 over the read-back rows; a repeated step
    overwrites in place and gives the same result."""
    B, H, T = 2, 3, gh * gw
    N = C * T
    a, b = u.CacheMX8(B, H, gh, gw, S, R), u.CacheMX8(B, H, gh, gw, S, R)
    g = torch.Generator(device="cuda").manual_seed(3)
    wq, wk = ((1 + 0.1 * torch.randn(H * 128, device="cuda", generator=g)).bfloat16() for _ in range(2))
    kw = dict(layout="half", q_norm_weight=wq, k_norm_weight=wk) if norm else dict(layout="half")
    held = {}
    for i in range(R // C + 4):
        f0 = i * C
        w = min(W, f0, R - C)
        q, k, v = torch.randn(B, N, 3, H, 128, device="cuda", generator=g).bfloat16().unbind(2)
        cos, sin = u.unstep_rotary_tables(f0, C, gh, gw, dims=(32, 32, 32))
        out = a.unstep_step_mx8(f0, C, w, q, k, v, cos, sin, **kw)
        q8, qs = b.unstep_kv_append_mx8(f0, C, q, k, v, cos, sin, **kw)
        two = b.unstep_window_attn_mx8(f0, C, w, q8, qs)
        assert torch.equal(out.view(torch.int16), two.view(torch.int16))
        assert torch.equal(out.view(torch.int16), a.unstep_step_mx8(f0, C, w, q, k, v, cos, sin, **kw).view(torch.int16))
        for x, y in ((a.k8, b.k8), (a.v8, b.v8), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        for j, (kk, vv) in enumerate(zip(*(t.view(B, C, T, H, 128).unbind(1) for t in a.unstep_kv_read_mx8(f0, C)))):
            held[f0 + j] = (kk.double().cpu().numpy(), vv.double().cpu().numpy())
        lo = max(0, f0 - w)
        frames = list(range(min(S, lo))) + list(range(lo, f0 + C))
        qv = u.unstep_mx8_dequantize(q8, qs).double().cpu().numpy()
        got = out.double().cpu().numpy()
        for bb in range(B):
            for h in range(H):
                ks, vs = (np.concatenate([held[f][t][bb, :, h] for f in frames]) for t in (0, 1))
                o, _, A = mx8.attention(qv[bb, :, h], ks, vs)
                top = np.abs(qv[bb, :, h] @ ks.T).max()
                bound = 2.0 ** -8 * np.abs(o) + 2.0 ** -8 * (1 + 2.0 ** -6) * A + 2.0 ** -17 * A * (1 + top)
                assert (np.abs(got[bb, :, h] - o) <= bound).all()
    assert a.frame_map() == b.frame_map()


def test_step_replayed_from_a_graph():
    """One capture replayed with new inputs, eager work in between; every replay equals an eager twin."""
    B, H, gh, gw, S, R, f0, C, W = 1, 3, 1, 1, 0, 3000, 2999, 1, 2900
    x, y = Case(B, H, gh, gw, S, R, f0 - 1, C, W), Case(B, H, gh, gw, S, R, f0 - 1, C, W)
    n = C * gh * gw
    ws = torch.empty(max(16, x.cache.workspace_bytes(f0, C, W)), dtype=torch.uint8, device="cuda")
    buf = torch.zeros(B, n, 3, H, 128, device="cuda", dtype=torch.bfloat16)
    q8, qs = torch.empty(B, n, H, 128, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), torch.empty(B, n, H, 4, dtype=torch.uint8, device="cuda")
    out = torch.empty(B, n, H, 128, device="cuda", dtype=torch.bfloat16)
    cos, sin = u.unstep_rotary_tables(f0, C, gh, gw, dims=(128, 0, 0))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        x.cache.unstep_step_mx8(f0, C, W, *buf.unbind(2), cos, sin, q8=q8, q_scale=qs, out=out, workspace=ws)
    for r in range(3):
        new = torch.randn(buf.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(r)).bfloat16()
        buf.copy_(new)
        torch.cuda.synchronize()
        g.replay()
        eager = y.cache.unstep_step_mx8(f0, C, W, *new.unbind(2), cos, sin)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), eager.view(torch.int16))


@pytest.mark.parametrize("whole_step", [False, True])
def test_captures_have_scratch_of_their_own(whole_step):
    """Two graphs of one cache, captured without a workspace argument, replayed at once on two streams and after the
    kept scratch has grown and its old memory has gone to another tensor."""
    B, H, gh, gw, S, R, f0, C, W = 1, 4, 1, 1, 0, 5000, 4999, 1, 4000
    c = Case(B, H, gh, gw, S, R, f0, C, W)
    cos, sin = u.unstep_rotary_tables(f0, C, gh, gw, dims=(128, 0, 0))
    qkv = [torch.randn(B, 1, H, 128, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i)).bfloat16() for i in range(3)]

    def call(window):
        if whole_step:
            return c.cache.unstep_step_mx8(f0, C, window, *qkv, cos, sin)
        return c.cache.unstep_window_attn_mx8(f0, C, window, c.q8, c.qs)

    want = {w: call(w).clone() for w in (3000, W)}
    kept = c.cache._ws
    graphs, outs = {}, {}
    for w in want:
        graphs[w] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[w]):
            outs[w] = call(w)
    assert c.cache._ws is kept
    c.cache._ws = None                                         # as when a larger one replaces it
    size = kept.numel()
    del kept
    other = torch.full((size,), 77, dtype=torch.uint8, device="cuda")
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for o in outs.values():
            o.zero_()
        torch.cuda.synchronize()
        for s, w in zip(streams, want):
            with torch.cuda.stream(s):
                graphs[w].replay()
        torch.cuda.synchronize()
        assert (other == 77).all()
        for w in want:
            assert torch.equal(outs[w].view(torch.int16), want[w].view(torch.int16))


def test_streams_and_kept_scratch():
    """A step on a named stream while the program goes on: the same result, and memory that the wrappers
    allocated is not handed out before that stream has used it."""
    c = Case(1, 12, 1, 1, 0, 5000, 5200, 1, 4999)
    want, _ = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(4):
        got.append(c.cache.unstep_window_attn_mx8(*c.a, c.q8, c.qs, stream=side))
        junk = torch.full((1 << 22,), 3.0, device="cuda")
        del junk
    torch.cuda.synchronize()
    for o in got:
        assert torch.equal(o.view(torch.int16), want.view(torch.int16))
