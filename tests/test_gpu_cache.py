"""The KV cache held in 8 bits on the GPU: writes bit for bit, reads bit for bit, attention against float64."""
import math

import numpy as np
import pytest
import torch

from oracle import dam_oracle as orc
from paper_2506_11104_b200 import binding as B
from tests import cache_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def _cu(lengths):
    return [0] + [int(x) for x in np.cumsum(lengths)]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _rows(rng, n, Hkv, d, dtype, spread=1.0):
    """Rows whose channels have sizes of their own."""
    x = rng.standard_normal((n, Hkv, d)) * np.exp(spread * rng.standard_normal((1, Hkv, d)))
    return torch.from_numpy(x).to(torch.float32).to(dtype).to(DEV)


class Pair:
    """A cache on the device and its restatement on the host, written side by side."""

    def __init__(self, lengths, Hkv, d, code, block, dtype, head_major=False):
        self.Hkv, self.d, self.dtype = Hkv, d, dtype
        T = sum(lengths)
        kind = B.CACHE_CODES[code][1]

        def codes():
            if head_major:
                return torch.full((Hkv, T, d), 0x55, dtype=torch.uint8, device=DEV).view(kind).permute(1, 0, 2)
            return torch.full((T, Hkv, d), 0x55, dtype=torch.uint8, device=DEV).view(kind)

        self.cache = B.make_cache(_cu(lengths), Hkv, d, code, block, DEV, codes(), codes())
        self.k, self.v = R.unpack(self.cache, "k"), R.unpack(self.cache, "v")

    def write(self, xk, xv, counts, starts, on_device=True):
        tokens = B.make_shape(_cu(counts), self.Hkv, self.Hkv, self.d, self.dtype, DEV, k_strides=xk.stride()[:2], v_strides=xv.stride()[:2])
        scratch = B.dam_cache_write(xk, xv, tokens, self.cache, _ints(starts) if on_device else None)
        assert B.dam_poll_status(scratch) == 0
        at = 0
        for b, (n, s) in enumerate(zip(counts, starts)):
            for side, x in ((self.k, xk), (self.v, xv)):
                side[b].write(x[at:at + n].cpu().double().numpy(), s)
            at += n

    def check(self):
        for name, want in (("k", self.k), ("v", self.v)):
            for got, w in zip(R.unpack(self.cache, name), want):
                assert np.array_equal(got.scales, w.scales, equal_nan=True)
                assert np.array_equal(got.codes, w.codes)

    def check_read(self, starts, counts):
        tokens = B.make_shape(_cu(counts), self.Hkv, self.Hkv, self.d, self.dtype, DEV)
        K, V, scratch = B.dam_cache_read(self.cache, tokens, _ints(starts))
        assert B.dam_poll_status(scratch) == 0
        for got, side in ((K, self.k), (V, self.v)):
            want = np.concatenate([s.read(p, n) for s, p, n in zip(side, starts, counts)])
            want = torch.from_numpy(want).to(self.dtype)
            assert torch.equal(torch.nan_to_num(got.cpu().float(), nan=1e30), torch.nan_to_num(want.float(), nan=1e30))


FORMS = [(Hkv, d, dtype, code, block) for Hkv, d, dtype, code, block in
         [(2, 128, BF16, "int8", 64), (2, 128, BF16, "e4m3", 64), (3, 64, BF16, "int8", 16), (1, 64, BF16, "e4m3", 128),
          (2, 128, F32, "int8", 128), (1, 128, F32, "e4m3", 16), (2, 64, F32, "int8", 32), (5, 64, F32, "e4m3", 64),
          (1, 128, BF16, "int8", 32), (1, 128, BF16, "e4m3", 128), (1, 64, BF16, "int8", 64)]]


@pytest.mark.parametrize("Hkv,d,dtype,code,block", FORMS)
def test_write_and_read_bit_for_bit(Hkv, d, dtype, code, block):
    """A prompt (ragged, one sequence empty), a chunk that ends and begins inside blocks, single tokens that raise scales."""
    rng = np.random.default_rng(5)
    lengths = [300, 0, 129, 1, 700]
    p = Pair(lengths, Hkv, d, code, block, dtype)
    at = [150, 0, 127, 0, 333]
    p.write(_rows(rng, sum(at), Hkv, d, dtype), _rows(rng, sum(at), Hkv, d, dtype), at, [0] * 5, on_device=False)
    p.check()
    for counts in ([1, 0, 1, 1, 1], [70, 0, 0, 0, 129], [1, 0, 1, 0, 1], [2, 0, 0, 0, 1], [1, 0, 0, 0, 5]):
        gain = 1.3                                            # (later tokens are larger: most of them raise their block's scale)
        xk, xv = _rows(rng, sum(counts), Hkv, d, dtype) * gain, _rows(rng, sum(counts), Hkv, d, dtype) * gain
        p.write(xk, xv, counts, at)
        at = [a + n for a, n in zip(at, counts)]
        p.check()
    p.check_read([0, 0, 0, 0, 0], [a for a in at])
    p.check_read([17, 0, 100, 0, 64], [100, 0, 1, 1, 333])


def test_values_on_the_border_of_two_codes_and_at_the_ends_of_the_range():
    """Quotients of exactly k + 1/2, blocks of zeros, of the smallest and of the largest numbers."""
    d, block = 128, 16
    for dtype in (BF16, F32):
        for code in ("int8", "e4m3"):
            x = torch.zeros(16 * 7, 1, d, dtype=torch.float64)
            x[:16] = (torch.arange(16 * d).view(16, 1, d) % 255 - 127) / 2                # amax 63.5: code k is x = k / 2, and x = k / 4 ties
            x[0, 0, 0] = 63.5
            x[16:32] = torch.randint(-254, 255, (16, 1, d), generator=torch.Generator().manual_seed(1)) / 4
            x[16, 0, 5] = 63.5
            x[48:64] = 1e-38 * torch.randn(16, 1, d, generator=torch.Generator().manual_seed(2), dtype=torch.float64)
            x[64:80] = 3e38 * torch.rand(16, 1, d, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
            x[80:96] = 2.0 ** -133 * (torch.arange(d) % 3 - 1)                             # (bf16's smallest number)
            x[96:112] = torch.linspace(-480, 480, 16 * d, dtype=torch.float64).view(16, 1, d)   # all e4m3 borders: amax rounds up to 512
            x = x.to(torch.float32).to(dtype).to(DEV)
            p = Pair([112], 1, d, code, block, dtype)
            p.write(x, x.flip(2).contiguous(), [112], [0])
            p.check()
            p.check_read([0], [112])


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_block_with_an_infinity_or_a_nan_has_no_scale_until_it_is_begun_anew(code, bad):
    rng = np.random.default_rng(7)
    p = Pair([128], 2, 64, code, 32, BF16)
    x, y = _rows(rng, 100, 2, 64, BF16), _rows(rng, 100, 2, 64, BF16)
    x[40, 1, 3] = bad
    p.write(x, y, [100], [0])
    p.check()
    p.check_read([0], [100])
    assert math.isnan(p.k[0].scales[1, 1]) and np.isfinite(p.k[0].scales[1, 0]) and np.isfinite(p.v[0].scales).all()
    one = _rows(rng, 1, 2, 64, BF16)
    p.write(one, one, [1], [50])                              # a further token of that block: still none
    assert math.isnan(p.k[0].scales[1, 1])
    p.check()
    p.write(x[:32], y[:32], [32], [32])                       # begun anew
    p.check()
    assert np.isfinite(p.k[0].scales).all()
    one[0, 0, 0] = bad                                        # and one that arrives in a block that was fine
    p.write(one, y[:1], [1], [64 + 7])
    p.check()
    p.check_read([0], [72])


def test_rows_with_strides_and_codes_by_head():
    rng = np.random.default_rng(9)
    p = Pair([200, 90], 3, 64, "int8", 64, BF16, head_major=True)
    wide = _rows(rng, 2 * 150, 6, 64, BF16)
    xk, xv = wide[::2, ::2], wide.permute(1, 0, 2).contiguous().permute(1, 0, 2)[150:, 3:]
    p.write(xk, xv, [100, 50], [30, 40])
    p.check()
    # packed rows into strided outputs; what lies between them stays
    out = torch.full((150, 5, 64), 7.0, dtype=BF16, device=DEV)
    tokens = B.make_shape([0, 100, 150], 3, 3, 64, BF16, DEV, k_strides=out.stride()[:2], v_strides=out.stride()[:2])
    other = out.clone()
    B.dam_cache_read(p.cache, tokens, _ints([30, 40]), out[:, 1:], other)
    want = torch.from_numpy(np.concatenate([p.k[0].read(30, 100), p.k[1].read(40, 50)])).to(BF16)
    assert torch.equal(out[:, 1:4].cpu(), want) and (out[:, 0] == 7).all() and (out[:, 4] == 7).all()
    assert (other[:, 3:] == 7).all()


@pytest.mark.parametrize("Hkv,d,dtype,offset", [(1, 64, F32, 4), (3, 128, F32, 0), (64, 128, BF16, 0), (130, 64, BF16, 8), (70, 128, F32, 0)])
def test_reads_of_any_number_of_heads_and_of_rows_off_the_widest_boundary(Hkv, d, dtype, offset):
    """Tokens of a few pieces and tokens that a slot cannot hold; rows that begin 16 bytes behind a 32-byte boundary."""
    rng = np.random.default_rng(15)
    p = _filled(rng, [70, 33], Hkv, d, "int8", 16, dtype)
    tokens = B.make_shape([0, 40, 73], Hkv, Hkv, d, dtype, DEV)
    whole = [torch.full((73 * Hkv * d + 2 * offset + 8,), 5.0, dtype=dtype, device=DEV) for _ in range(2)]
    K, V = (x[offset:offset + 73 * Hkv * d].view(73, Hkv, d) for x in whole)
    _, _, scratch = B.dam_cache_read(p.cache, tokens, _ints([30, 0]), K, V)
    assert B.dam_poll_status(scratch) == 0
    for got, side, x in ((K, p.k, whole[0]), (V, p.v, whole[1])):
        want = torch.from_numpy(np.concatenate([side[0].read(30, 40), side[1].read(0, 33)])).to(dtype)
        assert torch.equal(got.cpu(), want)
        assert (x[:offset] == 5).all() and (x[offset + got.numel():] == 5).all()


def test_ranges_outside_the_capacity_are_refused_alone():
    rng = np.random.default_rng(11)
    p = Pair([64, 64, 64, 64], 1, 64, "e4m3", 16, BF16)
    x = _rows(rng, 40, 1, 64, BF16)
    tokens = B.make_shape([0, 10, 20, 30, 40], 1, 1, 64, BF16, DEV)
    scratch = B.dam_cache_write(x, x, tokens, p.cache, _ints([-1, 55, 54, 2 ** 31 - 1]))
    assert B.dam_poll_status(scratch) == 1
    for side in (p.k, p.v):
        side[2].write(x[20:30].cpu().double().numpy(), 54)
    p.check()
    K, V, scratch = B.dam_cache_read(p.cache, tokens, _ints([-1, 55, 54, 2 ** 31 - 1]))
    assert B.dam_poll_status(scratch) == 1
    assert not K[:20].any() and not K[30:].any() and not V[:20].any()
    assert torch.equal(K[20:30].cpu(), torch.from_numpy(p.k[2].read(54, 10)).to(BF16))
    # an empty range is none, wherever it says it starts
    none = B.make_shape([0, 0, 0, 0, 0], 1, 1, 64, BF16, DEV)
    assert B.dam_poll_status(B.dam_cache_write(x, x, none, p.cache, _ints([-1, 99, 0, 0]))) == 0
    p.check()


def test_many_sequences():
    """More sequences than a search step looks at; most of them short or empty."""
    rng = np.random.default_rng(13)
    lengths = [int(n) for n in rng.integers(0, 40, size=1500)]
    p = Pair(lengths, 1, 64, "int8", 16, BF16)
    counts = [int(rng.integers(0, n + 1)) for n in lengths]
    starts = [int(rng.integers(0, n - c + 1)) // 16 * 16 for n, c in zip(lengths, counts)]
    x = _rows(rng, sum(counts), 1, 64, BF16)
    p.write(x, x.flip(0).contiguous(), counts, starts)
    p.check()
    p.check_read(starts, counts)


# ---- attention ------------------------------------------------------------------------------------------------------


def _filled(rng, lengths, Hkv, d, code, block, dtype, spread=0.5):
    p = Pair(lengths, Hkv, d, code, block, dtype)
    x, y = _rows(rng, sum(lengths), Hkv, d, dtype, spread), _rows(rng, sum(lengths), Hkv, d, dtype, spread)
    tokens = B.make_shape(_cu(lengths), Hkv, Hkv, d, dtype, DEV)
    assert B.dam_poll_status(B.dam_cache_write(x, y, tokens, p.cache)) == 0
    p.k, p.v = R.unpack(p.cache, "k"), R.unpack(p.cache, "v")
    return p


def _check(p, q, positions, O, lse, keep=None, scale=None, heads=None):
    """keep: (sequence, head, position) -> bool [position + 1], or None: every key."""
    Hq, d = q.shape[1], q.shape[2]
    scale = scale or 1.0 / math.sqrt(d)
    got, got_l = O.cpu().double().numpy(), lse.cpu().double().numpy()
    qh = q.cpu().double().numpy()
    G = Hq // p.Hkv
    worst = 0.0
    for b, i in enumerate(positions):
        K, V = p.k[b].values(i + 1), p.v[b].values(i + 1)
        for h in heads or range(Hq):
            kept = np.ones(i + 1, bool) if keep is None else keep(b, h, i)
            want, want_l, A, S, vmax, n = R.attention(qh[b, h], K[:, h // G], V[:, h // G], kept, scale)
            if n == 0:
                assert not got[b, h].any() and got_l[b, h] == -math.inf
                continue
            tol = R.tolerance(want, A, S, vmax, n, q.dtype)
            off = np.abs(got[b, h] - want)
            assert (off <= tol).all(), (b, h, i, float((off / tol).max()))
            worst = max(worst, float((off / tol).max()))
            assert abs(got_l[b, h] - want_l) <= R.lse_tolerance(want_l, d, S, n), (b, h, got_l[b, h], want_l)
    return worst


DECODE = [([1], 4, 1, 64, BF16, "int8", 16), ([1], 8, 8, 128, F32, "e4m3", 128), ([300, 1, 129, 77], 8, 2, 128, BF16, "int8", 64), ([300, 1, 129, 77], 8, 2, 128, BF16, "e4m3", 16),
          ([2000, 500], 4, 1, 64, BF16, "int8", 32), ([1, 2, 15, 16, 17, 127, 128, 129], 8, 8, 64, BF16, "e4m3", 128),
          ([900], 16, 1, 128, BF16, "int8", 64), ([513, 1025], 12, 1, 64, BF16, "e4m3", 64), ([777], 24, 8, 128, BF16, "int8", 128),
          ([640, 333], 8, 2, 128, F32, "int8", 64), ([1500], 6, 2, 64, F32, "e4m3", 16), ([400, 3], 9, 1, 128, F32, "e4m3", 32),
          ([6000], 8, 1, 128, BF16, "e4m3", 64)]


@pytest.mark.parametrize("lengths,Hq,Hkv,d,dtype,code,block", DECODE)
def test_attention_over_every_key(lengths, Hq, Hkv, d, dtype, code, block):
    rng = np.random.default_rng(21)
    p = _filled(rng, lengths, Hkv, d, code, block, dtype)
    q = torch.from_numpy(rng.standard_normal((len(lengths), Hq, d))).float().to(dtype).to(DEV)
    for positions in ([n - 1 for n in lengths], [0] * len(lengths), [n // 2 for n in lengths], [min(n - 1, 127) for n in lengths]):
        O, lse, scratch = B.dam_cache_decode_attention(q, p.cache, _ints(positions))
        assert B.dam_poll_status(scratch) == 0
        _check(p, q, positions, O, lse)


# each way of sharing the keys: a cluster per sequence, a block each (two sizes), the list with the KV heads side by side and one after
# the other; on 148 SMs
SHARED = [([20000, 700, 1], 4, 2, 64, BF16, "int8", 64), ([18000], 8, 1, 128, BF16, "e4m3", 128), ([9000, 17000, 3], 8, 2, 128, F32, "int8", 16),
          ([17, 300, 64, 1, 129, 500, 33] * 29, 2, 1, 64, BF16, "e4m3", 16), ([40, 250, 129, 64, 1] * 40, 16, 4, 128, BF16, "int8", 32),
          ([33, 128, 190] * 100, 6, 3, 64, F32, "e4m3", 64), ([17000, 100], 25, 25, 64, BF16, "int8", 64),
          ([5000] + [1 + 3 * k for k in range(160)], 1, 1, 128, BF16, "e4m3", 64)]


@pytest.mark.parametrize("lengths,Hq,Hkv,d,dtype,code,block", SHARED)
def test_attention_however_the_keys_are_shared(lengths, Hq, Hkv, d, dtype, code, block):
    rng = np.random.default_rng(22)
    p = _filled(rng, lengths, Hkv, d, code, block, dtype)
    q = torch.from_numpy(rng.standard_normal((len(lengths), Hq, d))).float().to(dtype).to(DEV)
    for positions in ([n - 1 for n in lengths], [n * 2 // 3 for n in lengths]):
        O, lse, scratch = B.dam_cache_decode_attention(q, p.cache, _ints(positions))
        assert B.dam_poll_status(scratch) == 0
        _check(p, q, positions, O, lse, heads=sorted({0, Hq // 2, Hq - 1}))
    # a position outside its capacity, in the same form
    positions[-1] = lengths[-1]
    O2, lse2, scratch = B.dam_cache_decode_attention(q, p.cache, _ints(positions))
    assert B.dam_poll_status(scratch) == 1
    assert not O2[-1].any() and torch.isneginf(lse2[-1]).all()
    # (the others' keys may be shared out differently: equal to rounding)
    if len(lengths) > 1:
        _check(p, q, positions[:-1], O2, lse2, heads=[Hq - 1])


def test_attention_over_codes_by_head_and_wide_strides():
    """Head-major codes and codes inside a wider buffer, in every form of the attention."""
    rng = np.random.default_rng(24)
    for lengths, d in (([500, 70], 64), ([500, 70], 128), ([18000], 128), ([60] * 200, 64)):
        T, Hkv, Hq = sum(lengths), 1 if len(lengths) == 200 else 2, 4
        wide = [torch.randint(-127, 128, (T, Hkv + 1, d + 16), dtype=torch.int8, device=DEV) for _ in range(2)]
        major = [torch.randint(-127, 128, (Hkv, T, d), dtype=torch.int8, device=DEV) for _ in range(2)]
        rows = T // 32 + len(lengths)
        scales = [0.01 + 0.02 * torch.rand(rows, Hkv, device=DEV) for _ in range(2)]
        q = torch.from_numpy(rng.standard_normal((len(lengths), Hq, d))).float().to(BF16).to(DEV)
        positions = [n - 1 for n in lengths]
        for codes in ([x[:, 1:, 16:] for x in wide], [x.permute(1, 0, 2) for x in major], [major[0].permute(1, 0, 2), wide[1][:, :Hkv, :d]]):
            p = Pair.__new__(Pair)
            p.Hkv, p.d, p.dtype = Hkv, d, BF16
            p.cache = B.make_cache(_cu(lengths), Hkv, d, "int8", 32, DEV, codes[0], codes[1], scales[0], scales[1])
            p.k, p.v = R.unpack(p.cache, "k"), R.unpack(p.cache, "v")
            O, lse, scratch = B.dam_cache_decode_attention(q, p.cache, _ints(positions))
            assert B.dam_poll_status(scratch) == 0
            _check(p, q, positions, O, lse, heads=[0, Hq - 1])
            blob, keep = _blob(rng, lengths, Hq, 64)
            O, lse, scratch = B.dam_cache_decode_attention(q, p.cache, _ints(positions), blob)
            assert B.dam_poll_status(scratch) == 0
            _check(p, q, positions, O, lse, keep, heads=[0, Hq - 1])


def test_attention_of_many_ragged_sequences():
    """More sequences than a warp has lanes, more shares than chunks and more chunks than shares."""
    rng = np.random.default_rng(23)
    lengths = [int(n) for n in rng.integers(1, 260, size=70)] + [3000]
    p = _filled(rng, lengths, 2, 64, "int8", 16, BF16)
    q = torch.from_numpy(rng.standard_normal((71, 4, 64))).float().to(BF16).to(DEV)
    positions = [n - 1 for n in lengths]
    O, lse, scratch = B.dam_cache_decode_attention(q, p.cache, _ints(positions))
    assert B.dam_poll_status(scratch) == 0
    _check(p, q, positions, O, lse)


def test_attention_does_not_depend_on_what_lies_behind_the_position():
    """NaN codes, infinite and NaN scales behind the last token, and the next sequence's tokens, have no part in the result."""
    rng = np.random.default_rng(25)
    for block in (16, 128):
        p = _filled(rng, [200, 200], 2, 128, "e4m3", block, BF16)
        q = torch.from_numpy(rng.standard_normal((2, 8, 128))).float().to(BF16).to(DEV)
        positions = [100, 33]
        want = B.dam_cache_decode_attention(q, p.cache, _ints(positions))
        for b, i in enumerate(positions):
            t0 = 200 * b
            for codes in (p.cache.k_codes, p.cache.v_codes):
                codes.view(torch.uint8)[t0 + i + 1:t0 + 200] = 0x7F
            for scales in (p.cache.k_scales, p.cache.v_scales):
                row = t0 // block + b
                scales[row + i // block + 1:row + -(-200 // block)] = math.nan
        got = B.dam_cache_decode_attention(q, p.cache, _ints(positions))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_attention_with_scales_of_very_different_sizes():
    """V blocks a factor of 1e12 apart in either order, K blocks that send logits far up: both references move."""
    rng = np.random.default_rng(27)
    for code in ("int8", "e4m3"):
        for order in (1, -1):
            p = Pair([256], 1, 64, code, 16, BF16)
            x = torch.from_numpy(rng.standard_normal((256, 1, 64))).float()
            size = torch.logspace(-6 * order, 6 * order, 16).repeat_interleave(16)[:, None, None]
            grow = torch.linspace(0.1, 30, 256)[:, None, None].flip(0) if order < 0 else torch.linspace(0.1, 30, 256)[:, None, None]
            p.write((x * grow).to(BF16).to(DEV), (x.flip(0) * size).to(BF16).to(DEV), [256], [0])
            q = torch.from_numpy(rng.standard_normal((1, 4, 64))).float().to(BF16).to(DEV)
            O, lse, _ = B.dam_cache_decode_attention(q, p.cache, _ints([255]))
            _check(p, q, [255], O, lse)


def test_queries_of_any_size_and_a_scale_of_its_own():
    rng = np.random.default_rng(29)
    p = _filled(rng, [150], 1, 128, "int8", 64, BF16)
    q = torch.from_numpy(rng.standard_normal((1, 6, 128))).float()
    q[0, 0] *= 1e-30
    q[0, 1] *= 1e30
    q[0, 2] = 0
    q[0, 3, ::2] *= 1e-6                                      # elements far below the row's largest
    q = q.to(BF16).to(DEV)
    for scale in (0.25,):
        O, lse, _ = B.dam_cache_decode_attention(q, p.cache, _ints([149]), softmax_scale=scale)
        _check(p, q, [149], O, lse, scale=scale, heads=[0, 2, 3, 4, 5])
        # logits of 1e30: the largest alone counts
        K, V = p.k[0].values(150)[:, 0], p.v[0].values(150)[:, 0]
        x = K @ q[0, 1].cpu().double().numpy()
        assert np.abs(O[0, 1].cpu().double().numpy() - V[x.argmax()]).max() <= 2.0 ** -7 * np.abs(V[x.argmax()]).max()


def test_a_nan_stays_a_nan():
    rng = np.random.default_rng(31)
    p = _filled(rng, [150, 150], 2, 64, "int8", 64, BF16)
    q = torch.from_numpy(rng.standard_normal((2, 4, 64))).float().to(BF16).to(DEV)
    q[0, 0, 5] = math.nan
    p.cache.v_scales[150 // 64 + 1 + 1, 1] = math.nan         # a V block of sequence 1, KV head 1
    O, lse, _ = B.dam_cache_decode_attention(q, p.cache, _ints([149, 149]))
    assert torch.isnan(O[0, 0]).all() and torch.isnan(lse[0, 0]) and torch.isfinite(O[0, 1:].float()).all()
    assert torch.isnan(O[1, 2:]).all() and torch.isfinite(lse[1]).all() and torch.isfinite(O[1, :2].float()).all()


def _blob(rng, lengths, Hq, pcl, empty_head=None):
    """A blob from planted columns and diagonals, and its masks by the oracle."""
    maps, masks = [], []
    for b, S in enumerate(lengths):
        L = min(S, pcl)
        per = []
        for h in range(Hq):
            P = np.zeros((L, L), np.float32)
            if h != empty_head:
                for c in rng.choice(L, size=min(L, int(rng.integers(0, 6))), replace=False):
                    P[c:, c] = 1
                for r in range(int(rng.integers(0, min(L, 40)))):
                    P[np.arange(r, L), np.arange(0, L - r)] = 1
                P[np.triu_indices(L, 1)] = 0
            maps.append(P.reshape(-1))
            per.append(orc.head_mask_from_probs(P, S, 0.3, 0.8, 0.5, 1e-8))
        masks.append(per)
    shape = B.make_shape(_cu(lengths), Hq, Hq, 64, BF16, DEV)
    blob, _ = B.dam_build_masks_from_scores(torch.from_numpy(np.concatenate(maps)).to(DEV), shape, B.make_rule(pcl, 0.3, 0.8))
    assert B.dam_poll_status(blob) == 0

    def keep(b, h, i):
        hm = masks[b][h]
        return orc.extended_rows(hm.M, hm.D, hm.V, max(i + 1, hm.L), [i])[0, :i + 1].astype(bool)
    return blob, keep


@pytest.mark.parametrize("lengths,Hq,Hkv,d,dtype,code,block,pcl", [
    ([700, 400], 8, 2, 128, BF16, "int8", 64, 128), ([700, 130, 1], 4, 4, 64, BF16, "e4m3", 16, 100),
    ([600], 16, 1, 64, BF16, "int8", 32, 96), ([500, 300], 8, 1, 128, F32, "e4m3", 128, 128), ([640], 10, 1, 64, F32, "int8", 64, 160),
    ([5000], 8, 1, 64, BF16, "e4m3", 64, 2112)])
def test_attention_under_stored_patterns(lengths, Hq, Hkv, d, dtype, code, block, pcl):
    rng = np.random.default_rng(33)
    p = _filled(rng, lengths, Hkv, d, code, block, dtype)
    blob, keep = _blob(rng, lengths, Hq, pcl, empty_head=1)
    q = torch.from_numpy(rng.standard_normal((len(lengths), Hq, d))).float().to(dtype).to(DEV)
    L = min(lengths[0], pcl)
    for at in (0, 5, L - 1, L, L + 1, 2 * L - 1, 2 * L, 10 ** 6):
        positions = [min(n - 1, at) for n in lengths]
        O, lse, scratch = B.dam_cache_decode_attention(q, p.cache, _ints(positions), blob)
        assert B.dam_poll_status(scratch) == 0
        _check(p, q, positions, O, lse, keep)


@pytest.mark.parametrize("num_seqs", [55, 56, 138, 139, 296, 297])
def test_attention_under_patterns_split_over_blocks(num_seqs):
    """Enough sequences for clusters of 8, 4, 2 and 1 blocks (both sides of every boundary on 148 SMs)."""
    rng = np.random.default_rng(num_seqs)
    p = _filled(rng, [200] * num_seqs, 1, 64, "int8", 16, BF16)
    blob, keep = _blob(rng, [200] * num_seqs, 2, 96)
    q = torch.from_numpy(rng.standard_normal((num_seqs, 2, 64))).float().to(BF16).to(DEV)
    positions = [int(x) for x in rng.integers(0, 200, size=num_seqs)]
    O, lse, _ = B.dam_cache_decode_attention(q, p.cache, _ints(positions), blob)
    _check(p, q, positions, O, lse, keep)


def test_a_key_another_head_keeps_has_no_part_in_a_head_that_does_not():
    """Heads of one group, keys of a block without a scale: NaN for the head that keeps one, nothing for the other."""
    rng = np.random.default_rng(35)
    p = _filled(rng, [256], 1, 64, "int8", 16, BF16)
    L = 64
    P = np.zeros((2, L, L), np.float32)
    P[0, 3:, 3] = 1                                           # head 0: column 3 alone
    P[1, 20:, 20] = 1                                         # head 1: column 20, in the next block
    shape = B.make_shape([0, 256], 2, 1, 64, BF16, DEV)
    blob, _ = B.dam_build_masks_from_scores(torch.from_numpy(P.reshape(-1)).to(DEV), shape, B.make_rule(L, 0.3, 0.8))
    p.cache.v_scales[1] = math.nan
    p.cache.k_scales[1] = math.nan
    q = torch.ones(1, 2, 64, dtype=BF16, device=DEV)
    O, lse, _ = B.dam_cache_decode_attention(q, p.cache, _ints([200]), blob)
    assert torch.isfinite(O[0, 0].float()).all() and torch.isfinite(lse[0, 0]) and torch.isnan(O[0, 1]).all()


def test_positions_outside_the_capacity_and_foreign_blobs():
    rng = np.random.default_rng(37)
    p = _filled(rng, [256, 256, 256], 1, 64, "e4m3", 64, BF16)
    q = torch.ones(3, 2, 64, dtype=BF16, device=DEV)
    blob, _ = _blob(rng, [256, 256, 256], 2, 64)
    for mask in (None, blob):
        O, lse, scratch = B.dam_cache_decode_attention(q, p.cache, _ints([100, 256, -1]), mask)
        assert B.dam_poll_status(scratch) == 1
        assert not O[1:].any() and torch.isneginf(lse[1:]).all() and torch.isfinite(lse[0]).all()
    other, _ = _blob(rng, [256, 256], 2, 64)                  # built for another number of sequences
    O, lse, scratch = B.dam_cache_decode_attention(q, p.cache, _ints([100, 100, 100]), other)
    assert B.dam_poll_status(scratch) == 1 and not O.any() and torch.isneginf(lse).all()


def test_a_generation_step_captured_and_replayed_on_another_stream():
    """Write the new token, attend: captured once, replayed with other tokens and positions; two graphs share one scratch."""
    rng = np.random.default_rng(39)
    lengths, Hq, Hkv, d = [300, 500], 8, 2, 128
    p = Pair(lengths, Hkv, d, "int8", 64, BF16)
    x, y = _rows(rng, 450, Hkv, d, BF16), _rows(rng, 450, Hkv, d, BF16)
    p.write(x, y, [150, 300], [0, 0])
    tokens = B.make_shape([0, 1, 2], Hkv, Hkv, d, BF16, DEV)
    q = torch.zeros(2, Hq, d, dtype=BF16, device=DEV)
    k, v = torch.zeros(2, Hkv, d, dtype=BF16, device=DEV), torch.zeros(2, Hkv, d, dtype=BF16, device=DEV)
    pos, O = _ints([150, 300]), torch.zeros(2, Hq, d, dtype=BF16, device=DEV)
    lse = torch.zeros(2, Hq, device=DEV)
    wscr = torch.empty(256, dtype=torch.uint8, device=DEV)
    scratch = torch.empty(B.dam_cache_sizes(p.cache, Hq)[1], dtype=torch.uint8, device=DEV)
    blob, keep = _blob(rng, lengths, Hq, 96)
    side = torch.cuda.Stream()
    graphs = []
    for mask in (None, blob):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            B.dam_cache_write(k, v, tokens, p.cache, pos, wscr)
            B.dam_cache_decode_attention(q, p.cache, pos, mask, O=O, lse=lse, scratch=scratch)
        graphs.append(g)
    torch.cuda.synchronize()
    p.check()                                                 # nothing has run yet
    for step in range(6):
        nk, nv = _rows(rng, 2, Hkv, d, BF16) * (1 + step), _rows(rng, 2, Hkv, d, BF16)
        nq = torch.from_numpy(rng.standard_normal((2, Hq, d))).float().to(BF16)
        positions = [150 + step, 300 + step]
        with torch.cuda.stream(side):
            k.copy_(nk), v.copy_(nv), q.copy_(nq), pos.copy_(_ints(positions))
            graphs[step % 2].replay()
        torch.cuda.synchronize()
        for b in range(2):
            p.k[b].write(nk[b:b + 1].cpu().double().numpy(), positions[b])
            p.v[b].write(nv[b:b + 1].cpu().double().numpy(), positions[b])
        p.check()
        assert B.dam_poll_status(wscr) == 0 and B.dam_poll_status(scratch) == 0
        _check(p, q, positions, O, lse, keep if step % 2 else None)


def test_prompt_chunk_and_generation_together():
    """As a server uses them: a prompt is prefilled and written, its next chunk attends to what the cache gives back, then tokens
    are generated under the same masks; the generation step agrees with the chunk's rows."""
    rng = np.random.default_rng(41)
    S, first, Hq, Hkv, d, pcl = 1024, 512, 8, 2, 128, 256
    K, V = _rows(rng, S, Hkv, d, BF16, 0.3), _rows(rng, S, Hkv, d, BF16, 0.3)
    Q = torch.from_numpy(rng.standard_normal((S, Hq, d))).float().to(BF16).to(DEV)
    blob, keep = _blob(rng, [S], Hq, pcl)
    p = Pair([S], Hkv, d, "int8", 64, BF16)
    p.write(K[:first], V[:first], [first], [0])
    p.write(K[first:], V[first:], [S - first], [first])
    p.check()
    shape = B.make_shape([0, S], Hq, Hkv, d, BF16, DEV)
    Kc, Vc, _ = B.dam_cache_read(p.cache, shape)
    O, lse = torch.zeros_like(Q), torch.zeros(Hq, S, device=DEV)
    scr = B.dam_sparse_attention_rows(Q, Kc, Vc, blob, shape, [(first, S)], O, lse)
    assert B.dam_poll_status(scr) == 0
    for i in (first, 700, S - 1):
        o, l, scratch = B.dam_cache_decode_attention(Q[i:i + 1], p.cache, _ints([i]), blob)
        assert B.dam_poll_status(scratch) == 0
        _check(p, Q[i:i + 1], [i], o, l, keep)
        # the chunk's K and V are the cache's rounded to bf16 (2^-8), its P and O are rounded to bf16 too
        fin = torch.isfinite(l[0])
        assert torch.equal(torch.isfinite(lse[:, i]), fin)
        bound = 4 * 2.0 ** -8 * float(Vc.float().abs().max())
        assert (o[0].float() - O[i].float()).abs().max() <= bound


@pytest.mark.parametrize("d,long", [(128, 4500000), (64, 70000)])
def test_offsets_beyond_32_bits(d, long):
    """A second sequence whose codes begin more than 2^32 bytes into the cache (by its length, or by the stride of a token)."""
    rng = np.random.default_rng(43)
    Hkv, Hq, lengths = (8, 16, [long, 700]) if d == 128 else (1, 2, [long, 700])
    T = sum(lengths)
    if d == 128:
        codes = [torch.zeros(T, Hkv, d, dtype=torch.int8, device=DEV) for _ in range(2)]
    else:                                                     # 64 bytes of every 65536
        codes = [torch.zeros(T, 65536, dtype=torch.int8, device=DEV)[:, None, 128:192] for _ in range(2)]
    assert (long * codes[0].stride(0)) > 2 ** 32
    cache = B.make_cache(_cu(lengths), Hkv, d, "int8", 64, DEV, *codes)
    xs = [_rows(rng, 300 + 500, Hkv, d, BF16) for _ in range(2)]
    tokens = B.make_shape([0, 300, 800], Hkv, Hkv, d, BF16, DEV)
    starts = _ints([long - 300, 0])
    assert B.dam_poll_status(B.dam_cache_write(xs[0], xs[1], tokens, cache, starts)) == 0
    sides = []
    for x, scales in zip(xs, (cache.k_scales, cache.v_scales)):
        tail, head = R.Side(300 + long % 64, Hkv, d, "int8", 64), R.Side(700, Hkv, d, "int8", 64)
        begun = (long - 300) % 64                             # (the block it begins in was begun before, with the scale 0 of the zeros)
        tail = R.Side(begun + 300, Hkv, d, "int8", 64)
        tail.write(x[:300].cpu().double().numpy(), begun)
        head.write(x[300:].cpu().double().numpy(), 0)
        sides.append((tail, head, begun))
    K, V, scratch = B.dam_cache_read(cache, tokens, starts)
    assert B.dam_poll_status(scratch) == 0
    for got, (tail, head, begun) in zip((K, V), sides):
        want = torch.from_numpy(np.concatenate([tail.read(begun, 300), head.read(0, 500)])).to(BF16)
        assert torch.equal(got.cpu(), want)
    p = Pair.__new__(Pair)
    p.Hkv, p.d, p.dtype = Hkv, d, BF16
    p.k, p.v = [sides[0][1]], [sides[1][1]]
    q = torch.from_numpy(rng.standard_normal((2, Hq, d))).float().to(BF16).to(DEV)
    blob, keep = _blob(rng, [100, 100], Hq, 64)
    for mask in (None, blob):
        O, lse, scratch = B.dam_cache_decode_attention(q, cache, _ints([0, 499]), mask)
        assert B.dam_poll_status(scratch) == 0
        _check(p, q[1:], [499], O[1:], lse[1:], mask is not None and (lambda b, h, i: keep(1, h, i)) or None, heads=[0, Hq - 1])
    # the far end of the first sequence, under patterns that reach its last keys only
    L = 64
    P = np.zeros((2, Hq, L, L), np.float32)
    for r in range(40):
        P[:, :, np.arange(r, L), np.arange(0, L - r)] = 1
    shape = B.make_shape([0, 100, 200], Hq, Hkv, d, BF16, DEV)
    blob, _ = B.dam_build_masks_from_scores(torch.from_numpy(P.reshape(-1)).to(DEV), shape, B.make_rule(L, 0.3, 1.0))
    O, lse, scratch = B.dam_cache_decode_attention(q, cache, _ints([long - 1, 499]), blob)
    assert B.dam_poll_status(scratch) == 0
    D, _, cols = B.MaskBlob(blob).pattern_bits(0, 0)
    near = np.flatnonzero(D)
    assert near.max() < 300
    tail_k, tail_v, begun = sides[0][0], sides[1][0], sides[0][2]
    at = sorted(begun + 299 - near)
    Kt, Vt = tail_k.values(begun + 300)[at], tail_v.values(begun + 300)[at]
    Kt, Vt = (np.concatenate([np.zeros((int(cols.sum()), Hkv, d)), x]) for x in (Kt, Vt))   # (the sequence begins with zeros)
    for h in (0, Hq - 1):
        g = h // (Hq // Hkv)
        want, want_l, A, S, vmax, n = R.attention(q[0, h].cpu().double().numpy(), Kt[:, g], Vt[:, g], np.ones(len(Kt), bool), 1 / math.sqrt(d))
        assert (np.abs(O[0, h].cpu().double().numpy() - want) <= R.tolerance(want, A, S, vmax, n, BF16)).all()
        assert abs(float(lse[0, h]) - want_l) <= R.lse_tolerance(want_l, d, S, n)


def test_two_streams_at_once():
    """Two caches, two streams, calls interleaved: what each gets alone."""
    rng = np.random.default_rng(45)
    caches = [_filled(rng, [3000, 40], 2, 128, "int8", 64, BF16), _filled(rng, [700] * 90, 2, 64, "e4m3", 16, BF16)]
    qs = [torch.from_numpy(rng.standard_normal((n, 8, d))).float().to(BF16).to(DEV) for n, d in ((2, 128), (90, 64))]
    pos = [_ints([2999, 39]), _ints([699] * 90)]
    want = [B.dam_cache_decode_attention(q, p.cache, x)[:2] for q, p, x in zip(qs, caches, pos)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k].append(B.dam_cache_decode_attention(qs[k], caches[k].cache, pos[k])[:2])
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(o, want[k][0]) and torch.equal(l, want[k][1]) for o, l in got[k])


def test_calls_without_tokens():
    """No sequence gets a token: nothing is written or read, whatever the starts, and the status says so."""
    rng = np.random.default_rng(46)
    p = _filled(rng, [40, 70], 2, 64, "int8", 16, BF16)
    none = torch.empty(0, 2, 64, dtype=BF16, device=DEV)
    tokens = B.make_shape([0, 0, 0], 2, 2, 64, BF16, DEV)
    for starts in (None, _ints([0, 70]), _ints([-5, 1 << 30])):
        assert B.dam_poll_status(B.dam_cache_write(none, none, tokens, p.cache, starts)) == 0
        K, V, scratch = B.dam_cache_read(p.cache, tokens, starts)
        assert K.shape == V.shape == (0, 2, 64) and B.dam_poll_status(scratch) == 0
    p.check()


def test_a_long_sequence_captured_and_replayed_at_other_positions():
    """The list form and its join, replayed while the positions move over the bounds of the shares."""
    rng = np.random.default_rng(47)
    lengths = [70000, 300]
    p = _filled(rng, lengths, 1, 64, "int8", 64, BF16)
    q = torch.from_numpy(rng.standard_normal((2, 4, 64))).float().to(BF16).to(DEV)
    pos, O, lse = _ints([0, 0]), torch.zeros_like(q), torch.zeros(2, 4, device=DEV)
    scratch = torch.empty(B.dam_cache_sizes(p.cache, 4)[1], dtype=torch.uint8, device=DEV)
    B.dam_cache_decode_attention(q, p.cache, pos, O=O, lse=lse, scratch=scratch)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pos.add_(1)
        B.dam_cache_decode_attention(q, p.cache, pos, O=O, lse=lse, scratch=scratch)
    for at in ([0, 298], [511, 0], [1022, 100], [40000, 7], [69996, 200]):
        pos.copy_(_ints(at))
        for step in range(3):
            g.replay()
            got = O.clone(), lse.clone()
            eager = B.dam_cache_decode_attention(q, p.cache, pos.clone())
            inside = [k for k in range(2) if at[k] + 1 + step < lengths[k]]
            assert B.dam_poll_status(scratch) == (0 if len(inside) == 2 else 1)
            assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])
            if len(inside) == 2:
                _check(p, q, [x + 1 + step for x in at], *got)


def _check_tight(p, q, positions, O, lse, code, keep=None):
    """As _check, with the tolerance that a query's own weights give."""
    Hq, d = q.shape[1], q.shape[2]
    scale, G = 1.0 / math.sqrt(d), Hq // p.Hkv
    got, got_l, qh = O.cpu().double().numpy(), lse.cpu().double().numpy(), q.cpu().double().numpy()
    for b, i in enumerate(positions):
        K, V = p.k[b].values(i + 1), p.v[b].values(i + 1)
        for h in range(Hq):
            kept = np.ones(i + 1, bool) if keep is None else keep(b, h, i)
            want, want_l, A, S, _, n = R.attention(qh[b, h], K[:, h // G], V[:, h // G], kept, scale)
            rows = p.v[b].scales[np.arange(i + 1) // p.v[b].block, h // G]
            wmax, _ = R.weights(qh[b, h], K[:, h // G], rows, kept, scale)
            tol = R.tight_tolerance(want, A, S, wmax, code, n, q.dtype)
            off = np.abs(got[b, h] - want)
            assert (off <= tol).all(), (b, h, i, float((off / tol).max()))
            assert abs(got_l[b, h] - want_l) <= R.lse_tolerance(want_l, d, S, n), (b, h, got_l[b, h], want_l)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Hq,d,code", [(2, 64, "int8"), (8, 128, "e4m3"), (8, 64, "e4m3"), (4, 128, "int8")])
@pytest.mark.parametrize("big", [2.0 ** 20, 2.0 ** 40])
def test_a_large_v_that_another_head_keeps_costs_a_head_nothing(Hq, d, code, dtype, big):
    """Heads of one group under patterns: the columns of head 0 lie in a block whose V is `big` times the other heads'."""
    rng = np.random.default_rng(51)
    p = _filled(rng, [256], 1, d, code, 16, dtype)
    p.cache.v_scales[0] *= big
    p.v = R.unpack(p.cache, "v")
    L = 64
    P = np.zeros((Hq, L, L), np.float32)
    for h in range(Hq):
        for c in (3, 9) if h == 0 else range(17 + h, 40):
            P[h, c:, c] = 1
    shape = B.make_shape([0, 256], Hq, 1, d, dtype, DEV)
    blob, _ = B.dam_build_masks_from_scores(torch.from_numpy(P.reshape(-1)).to(DEV), shape, B.make_rule(L, 0.3, 0.8))
    masks = [orc.head_mask_from_probs(x, 256, 0.3, 0.8, 0.5, 1e-8) for x in P]

    def keep(b, h, i):
        return orc.extended_rows(masks[h].M, masks[h].D, masks[h].V, max(i + 1, L), [i])[0, :i + 1].astype(bool)
    q = torch.from_numpy(rng.standard_normal((1, Hq, d))).float().to(dtype).to(DEV)
    for i in (200, 60):
        O, lse, scratch = B.dam_cache_decode_attention(q, p.cache, _ints([i]), blob)
        assert B.dam_poll_status(scratch) == 0
        assert not keep(0, 1, i)[:16].any() and keep(0, 0, i).sum() == 2
        _check_tight(p, q, [i], O, lse, code, keep)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lengths,Hq,d,code,place", [
    ([300], 4, 64, "int8", 0), ([300], 8, 128, "e4m3", 5), ([20000], 8, 64, "e4m3", 0), ([20000, 500], 4, 128, "int8", 7),
    ([200] * 160, 6, 64, "int8", 3), ([600] * 200, 2, 128, "e4m3", 0)])
def test_a_large_v_of_an_improbable_key_costs_the_others_nothing(lengths, Hq, d, code, place, dtype):
    """Every key, in every form: the 16 tokens of one block have logits of about -40 and a V of 2^30 times the others'."""
    rng = np.random.default_rng(53)
    p = Pair(lengths, 1, d, code, 16, dtype)
    at = np.concatenate([np.arange(n) // 16 == place for n in lengths])[:, None, None]
    x, y = rng.standard_normal((sum(lengths), 1, d)) * 0.3, rng.standard_normal((sum(lengths), 1, d))
    x[:, :, 0] = np.where(at[:, :, 0], -41.0 * math.sqrt(d) / 8, x[:, :, 0])
    y = np.where(at, y * 2.0 ** 30, y)
    x, y = (torch.from_numpy(z).float().to(dtype).to(DEV) for z in (x, y))
    tokens = B.make_shape(_cu(lengths), 1, 1, d, dtype, DEV)
    assert B.dam_poll_status(B.dam_cache_write(x, y, tokens, p.cache)) == 0
    p.k, p.v = R.unpack(p.cache, "k"), R.unpack(p.cache, "v")
    q = rng.standard_normal((len(lengths), Hq, d))
    q[:, :, 0] = 8
    q = torch.from_numpy(q).float().to(dtype).to(DEV)
    positions = [n - 1 for n in lengths]
    O, lse, scratch = B.dam_cache_decode_attention(q, p.cache, _ints(positions))
    assert B.dam_poll_status(scratch) == 0
    _check_tight(p, q, positions, O, lse, code)


@pytest.mark.parametrize("lengths,Hq,d,code", [([300], 4, 64, "int8"), ([500], 8, 128, "e4m3"), ([20000], 8, 64, "e4m3"), ([20000, 500], 4, 128, "int8"),
                                               ([200] * 160, 6, 64, "int8"), ([600] * 200, 2, 128, "e4m3")])
def test_fp32_weights_far_below_those_of_keys_without_a_value(lengths, Hq, d, code):
    """Every 16th key has a probability 2^37 times the others' and a V of zero: the output is the others' alone."""
    rng = np.random.default_rng(55)
    T = sum(lengths)
    p = Pair(lengths, 1, d, code, 64, F32)
    sink = np.concatenate([np.arange(n) % 16 == 0 for n in lengths])[:, None, None]
    x, y = rng.standard_normal((T, 1, d)) * 0.1, np.where(sink, 0.0, 0.5 + rng.random((T, 1, d)))
    x[:, :, 0] = np.where(sink[:, :, 0], 37 * math.log(2) * math.sqrt(d) / 8, 0)
    x, y = (torch.from_numpy(z).float().to(DEV) for z in (x, y))
    tokens = B.make_shape(_cu(lengths), 1, 1, d, F32, DEV)
    assert B.dam_poll_status(B.dam_cache_write(x, y, tokens, p.cache)) == 0
    p.k, p.v = R.unpack(p.cache, "k"), R.unpack(p.cache, "v")
    q = rng.standard_normal((len(lengths), Hq, d)) * 0.1
    q[:, :, 0] = 8
    q = torch.from_numpy(q).float().to(DEV)
    positions = [n - 1 for n in lengths]
    O, lse, scratch = B.dam_cache_decode_attention(q, p.cache, _ints(positions))
    assert B.dam_poll_status(scratch) == 0
    _check_tight(p, q, positions, O, lse, code)
    # and under patterns: the last 48 keys
    L = 64
    P = np.tril(np.ones((L, L), np.float32)) - np.tril(np.ones((L, L), np.float32), -48)
    hm = orc.head_mask_from_probs(P, 200, 0.3, 0.8, 0.5, 1e-8)
    shape = B.make_shape([200 * k for k in range(len(lengths) + 1)], Hq, 1, d, F32, DEV)
    maps = torch.from_numpy(np.tile(P.reshape(-1), len(lengths) * Hq)).to(DEV)
    blob, _ = B.dam_build_masks_from_scores(maps, shape, B.make_rule(L, 0.3, 0.8))
    O, lse, scratch = B.dam_cache_decode_attention(q, p.cache, _ints(positions), blob)
    assert B.dam_poll_status(scratch) == 0
    _check_tight(p, q, positions, O, lse, code, lambda b, h, i: orc.extended_rows(hm.M, hm.D, hm.V, i + 1, [i])[0, :i + 1].astype(bool))


def test_borders_of_codes_under_the_smallest_scales():
    """int8 scales just above 2^-126: half of one with an odd last bit is no fp32 number."""
    unit = 2.0 ** -149
    for s in (2 ** 23 + 1, 2 ** 23 + 77, 2 ** 24 - 1, 2 ** 24 - 3):
        amax = float(np.float32(s * 127.0 * unit))
        assert R.scale_of(amax, "int8") == s * unit
        x = np.zeros((32, 1, 64))
        for k in range(100):                                  # the fp32 numbers on either side of the border above k, and of the one below -k
            border = (k + 0.5) * s * unit
            near = np.float32(border)
            around = [np.nextafter(near, np.float32(0)), near, np.nextafter(near, np.float32(1))]
            x.reshape(-1)[10 * k:10 * k + 6] = [float(a) for a in around] + [-float(a) for a in around]
        x[16:] = x[:16]
        x[0, 0, 63] = x[16, 0, 63] = amax
        rows = torch.from_numpy(x).to(torch.float32)
        assert np.array_equal(rows.double().numpy(), x)
        p = Pair([64], 1, 64, "int8", 16, F32)
        p.write(rows.to(DEV), rows.flip(2).contiguous().to(DEV), [32], [0])
        p.check()
        for i in range(16):                                   # and one by one: the first row has the scale, the others join it
            one = rows[i:i + 1].to(DEV)
            p.write(one, one, [1], [32 + i])
        p.check()


def test_tensors_in_host_memory_are_refused_whichever_they_are():
    """Before anything is launched."""
    rng = np.random.default_rng(57)
    p = _filled(rng, [256], 1, 64, "int8", 64, BF16)
    blob, _ = _blob(rng, [256], 2, 64)
    tokens, hosted = B.make_shape([0, 30], 1, 1, 64, BF16, DEV), B.make_shape([0, 30], 1, 1, 64, BF16)
    x = _rows(rng, 30, 1, 64, BF16)
    start, small = _ints([0]), torch.empty(256, dtype=torch.uint8, device=DEV)
    args = {"K": x, "V": x.clone(), "tokens": tokens, "starts": start, "scratch": small}
    for name in args:
        bad = dict(args)
        bad[name] = hosted if name == "tokens" else args[name].cpu()
        with pytest.raises(ValueError, match="on the device"):
            B.dam_cache_write(bad["K"], bad["V"], bad["tokens"], p.cache, bad["starts"], bad["scratch"])
        with pytest.raises(ValueError, match="on the device"):
            B.dam_cache_read(p.cache, bad["tokens"], bad["starts"], bad["K"], bad["V"], bad["scratch"])
    q = torch.ones(1, 2, 64, dtype=BF16, device=DEV)
    scratch = torch.empty(B.dam_cache_sizes(p.cache, 2)[1], dtype=torch.uint8, device=DEV)
    args = {"q": q, "positions": _ints([99]), "mask": blob, "O": torch.zeros_like(q), "lse": torch.zeros(1, 2, device=DEV), "scratch": scratch}
    for name in args:
        bad = dict(args)
        bad[name] = args[name].cpu()
        with pytest.raises(ValueError, match="on the device"):
            B.dam_cache_decode_attention(bad["q"], p.cache, bad["positions"], bad["mask"], 0.0, bad["O"], bad["lse"], bad["scratch"])
    p.check()
    assert not args["O"].any()
    B.dam_cache_decode_attention(**args, cache=p.cache)
    assert args["O"].any()


@pytest.mark.parametrize("Hkv,d,dtype,code,block", [(2, d, dtype, code, block) for d in (64, 128) for dtype in (BF16, F32) for code in ("int8", "e4m3")
                                                    for block in (16, 32, 64, 128) if (d, dtype, code, block) not in {f[1:] for f in FORMS}])
def test_write_and_read_bit_for_bit_in_every_other_form(Hkv, d, dtype, code, block):
    test_write_and_read_bit_for_bit(Hkv, d, dtype, code, block)


# fp32 queries of few heads (two numbers in one tile) and of many, in the list, in clusters and in a block each
FP32 = [([9000, 17000, 3], 8, 2, 64, "e4m3", 16), ([20000, 500], 8, 1, 64, "int8", 64), ([20000, 500], 8, 1, 128, "e4m3", 64), ([18000], 2, 1, 128, "int8", 128),
        ([1500, 40], 8, 1, 64, "int8", 64), ([1500, 40], 8, 1, 128, "e4m3", 32), ([33, 128, 190] * 100, 5, 1, 128, "int8", 64),
        ([40, 250, 129, 64, 1] * 40, 16, 4, 128, "e4m3", 32), ([300, 700] * 100, 6, 1, 64, "e4m3", 16), ([1000] * 160, 2, 1, 64, "int8", 64)]


@pytest.mark.parametrize("lengths,Hq,Hkv,d,code,block", FP32)
def test_attention_of_fp32_queries_however_the_keys_are_shared(lengths, Hq, Hkv, d, code, block):
    test_attention_however_the_keys_are_shared(lengths, Hq, Hkv, d, F32, code, block)


@pytest.mark.parametrize("lengths,Hq,Hkv,d,code,block,pcl", [
    ([700, 400], 8, 2, 128, "int8", 64, 128), ([700, 130, 1], 4, 4, 64, "e4m3", 16, 100), ([300, 500], 4, 1, 64, "int8", 128, 96),
    ([200] * 90, 9, 3, 128, "e4m3", 32, 64), ([200] * 120, 6, 2, 64, "int8", 16, 64), ([200] * 240, 5, 1, 128, "int8", 64, 64)])
def test_attention_of_fp32_queries_under_stored_patterns(lengths, Hq, Hkv, d, code, block, pcl):
    rng = np.random.default_rng(59)
    p = _filled(rng, lengths, Hkv, d, code, block, F32)
    blob, keep = _blob(rng, lengths, Hq, pcl, empty_head=1)
    q = torch.from_numpy(rng.standard_normal((len(lengths), Hq, d))).float().to(DEV)
    for at in (0, pcl - 1, pcl, 10 ** 6):
        positions = [min(n - 1, at) for n in lengths]
        O, lse, scratch = B.dam_cache_decode_attention(q, p.cache, _ints(positions), blob)
        assert B.dam_poll_status(scratch) == 0
        _check(p, q, positions, O, lse, keep, heads=sorted({0, 1, Hq // 2, Hq - 1}))


@pytest.mark.parametrize("num_seqs", [48, 49, 104, 105, 222, 223])
def test_attention_under_patterns_on_both_sides_of_every_split(num_seqs):
    """Clusters of 8, 4 and 2 blocks, and one block: the last number of sequences of each and the first of the next."""
    rng = np.random.default_rng(num_seqs)
    p = _filled(rng, [200] * num_seqs, 1, 64, "int8", 16, BF16)
    blob, keep = _blob(rng, [200] * num_seqs, 2, 96)
    q = torch.from_numpy(rng.standard_normal((num_seqs, 2, 64))).float().to(BF16).to(DEV)
    positions = [int(x) for x in rng.integers(0, 200, size=num_seqs)]
    O, lse, scratch = B.dam_cache_decode_attention(q, p.cache, _ints(positions), blob)
    assert B.dam_poll_status(scratch) == 0
    _check(p, q, positions, O, lse, keep)
