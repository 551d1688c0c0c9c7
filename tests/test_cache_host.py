"""The 8-bit cache's entry points on the host: sizes, refusals before any launch, and the CPU restatement the GPU tests use."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2506_11104_b200 import binding as B
from paper_2506_11104_b200 import build as dam_build
from tests import cache_reference as R


@pytest.fixture(scope="module", autouse=True)
def _built():
    dam_build.build()


def _cache(**over):
    c = B.make_cache([0, 100, 100, 357], 2, 128, "int8", 64)
    for name in ("k_codes", "v_codes", "k_scales", "v_scales"):
        setattr(c.c, name, 0x1000)                           # aligned, never dereferenced
    for name, value in over.items():
        setattr(c.c, name, value)
    return c


def test_struct_size_is_the_library_s():
    assert ctypes.sizeof(B.dam_cache_t) == 112
    rows, scratch = B.dam_cache_sizes(_cache(), 8)
    assert rows == 357 // 64 + 3 and scratch >= 256 and scratch % 16 == 0


def test_every_block_has_a_scale_row_of_its_own():
    rng = np.random.default_rng(1)
    for block in (16, 32, 64, 128):
        for _ in range(50):
            lengths = rng.integers(0, 400, size=int(rng.integers(1, 9)))
            cu = np.concatenate([[0], np.cumsum(lengths)])
            rows = [int(cu[b]) // block + b + j for b, n in enumerate(lengths) for j in range(-(-int(n) // block))]
            assert len(set(rows)) == len(rows)
            assert not rows or max(rows) < int(cu[-1]) // block + len(lengths)


def test_every_block_and_token_is_served_by_one_slot():
    """The kernels' cut of a packed batch into slots: sequence b owns (cu[b] >> shift) + extra * b onwards."""
    rng = np.random.default_rng(2)

    def seq_of(cu, n, shift, extra, slot):                    # the device's search, 32 places a step
        lo, hi = 0, n
        while hi - lo > 1:
            step = (hi - lo + 31) >> 5
            here = [lo + k * step < hi and (cu[lo + k * step] >> shift) + extra * (lo + k * step) <= slot for k in range(32)]
            cnt = sum(here)
            assert here == [True] * cnt + [False] * (32 - cnt)
            lo += (cnt - 1) * step
            hi = min(hi, lo + step)
        return lo

    for trial in range(60):
        n = int(rng.choice([1, 2, 5, 31, 33, 200, 1100]))
        lengths = rng.integers(0, 150, size=n) * rng.integers(0, 2, size=n)
        cu = [0] + [int(x) for x in np.cumsum(lengths)]
        shift = int(rng.choice([4, 5, 6, 7]))
        starts = rng.integers(0, 300, size=n)
        seen = set()
        for slot in range((cu[-1] >> shift) + 2 * n):         # a write: blocks of tokens
            b = seq_of(cu, n, shift, 2, slot)
            m = cu[b + 1] - cu[b]
            j = (int(starts[b]) >> shift) + slot - ((cu[b] >> shift) + 2 * b)
            if m and j <= (int(starts[b]) + m - 1) >> shift:
                assert (b, j) not in seen
                seen.add((b, j))
        want = {(b, j) for b in range(n) for j in range(int(starts[b]) >> shift, ((int(starts[b]) + int(lengths[b]) - 1) >> shift) + 1) if lengths[b]}
        assert seen == want
        tokens = set()
        for slot in range(cu[-1] // 64 + n):                  # a read: 64 packed tokens
            b = seq_of(cu, n, 6, 1, slot)
            base = (slot - ((cu[b] >> 6) + b)) * 64
            for t in range(base, min(base + 64, cu[b + 1] - cu[b])):
                assert (b, t) not in tokens
                tokens.add((b, t))
        assert len(tokens) == cu[-1]


@pytest.mark.parametrize("over,code", [
    ({"struct_size": 8}, 1), ({"num_seqs": 0}, 1), ({"cu_seqlens_host": 0}, 1), ({"cu_seqlens_dev": 0}, 1), ({"total_tokens": 356}, 1),
    ({"num_kv_heads": 0}, 1), ({"code": 2}, 1), ({"code": -1}, 1), ({"block_tokens": 48}, 1), ({"block_tokens": 0}, 1), ({"block_tokens": 256}, 1),
    ({"head_dim": 96}, 2), ({"head_dim": 256}, 2), ({"k_stride_tok": 64}, 1), ({"v_stride_head": 136}, 1), ({"k_stride_head": -128}, 1),
    ({"reserved": 1}, 1), ({"k_codes": 0}, 1), ({"v_codes": 0x1008}, 1), ({"k_scales": 0}, 1), ({"v_scales": 0x1002}, 1)])
def test_bad_caches_are_refused(over, code):
    c = _cache(**over)
    host_only = not set(over) & {"k_codes", "v_codes", "k_scales", "v_scales"}
    lib = B.lib()
    if host_only:
        assert lib.dam_cache_sizes(c.ref, 8, None, None) == code
    shape = B.make_shape([0, 10, 10, 20], 8, 2, 128, torch.bfloat16)
    assert lib.dam_cache_write(0x1000, 0x1000, shape.ref, 0x1000, c.ref, 0x1000, 256, None) == code
    assert lib.dam_cache_read(c.ref, shape.ref, 0x1000, 0x1000, 0x1000, 0x1000, 256, None) == code
    assert lib.dam_cache_decode_attention(0x1000, c.ref, None, 0x1000, 8, 0, 0.0, 0x1000, 0x1000, 0x1000, 1 << 30, None) == code


def test_bad_calls_are_refused():
    lib, c = B.lib(), _cache()
    ok = 0x1000
    shape = B.make_shape([0, 10, 10, 20], 8, 2, 128, torch.bfloat16)

    def write(K=ok, V=ok, tokens=shape.ref, starts=ok, cache=c.ref, scratch=ok, size=255):
        return lib.dam_cache_write(K, V, tokens, starts, cache, scratch, size, None)

    def read(K=ok, V=ok, tokens=shape.ref, starts=ok, cache=c.ref, scratch=ok, size=255):
        return lib.dam_cache_read(cache, tokens, starts, K, V, scratch, size, None)

    others = [B.make_shape([0, 10, 20], 8, 2, 128, torch.bfloat16), B.make_shape([0, 10, 10, 20], 8, 4, 128, torch.bfloat16),
              B.make_shape([0, 10, 10, 20], 8, 2, 64, torch.bfloat16),
              B.make_shape([0, 10, 10, 20], 8, 2, 128, torch.bfloat16, k_strides=(260, 128))]
    for call in (write, read):
        assert call() == 3                                   # everything else is in order: the scratch is too small
        assert call(starts=None) == 3
        for name in ("K", "V", "scratch"):
            assert call(**{name: None}) == 1 and call(**{name: 0x1008}) == 1
        assert call(scratch=0x1080) == 1 and call(starts=0x1002) == 1 and call(cache=None) == 1 and call(tokens=None) == 1
        for other in others:
            assert call(tokens=other.ref) == 1

    def attend(q=ok, cache=c.ref, mask=None, pos=ok, heads=8, dtype=0, scale=0.0, O=ok, lse=ok, scratch=ok, size=256):
        return lib.dam_cache_decode_attention(q, cache, mask, pos, heads, dtype, scale, O, lse, scratch, size, None)

    assert attend() == 3 and attend(mask=0x1100) == 3
    for name in ("q", "pos", "O", "lse", "scratch", "cache"):
        assert attend(**{name: None}) == 1
    for name, value in (("q", 0x1008), ("O", 0x1008), ("mask", 0x1010), ("scratch", 0x1010), ("pos", 0x1002), ("lse", 0x1002), ("heads", 7),
                        ("heads", 0), ("heads", -2), ("dtype", 2), ("scale", -1.0), ("scale", float("nan"))):
        assert attend(**{name: value}) == 1, name
    assert lib.dam_cache_sizes(c.ref, 7, None, None) == 1 and lib.dam_cache_sizes(None, 8, None, None) == 1
    assert lib.dam_cache_sizes(c.ref, 8, None, None) == 0


def test_a_call_without_tokens_needs_no_rows():
    """(The address of a tensor without rows is NULL.)"""
    lib, c = B.lib(), _cache()
    none = B.make_shape([0, 0, 0, 0], 8, 2, 128, torch.bfloat16)
    assert lib.dam_cache_write(None, None, none.ref, 0x1000, c.ref, 0x1000, 255, None) == 3          # the scratch is all that is wrong
    assert lib.dam_cache_read(c.ref, none.ref, 0x1000, None, None, 0x1000, 255, None) == 3


def test_the_reference_follows_the_structure():
    shape, cache = B.make_shape([0, 64], 2, 1, 64, torch.bfloat16), B.make_cache([0, 64], 1, 64)
    assert B.dam_cache_sizes(cache, 2)[0] == 2
    shape.c, cache.c = B.make_shape([0, 96], 2, 1, 64, torch.bfloat16).c, B.make_cache([0, 128], 1, 64).c
    assert B.dam_cache_sizes(cache, 2)[0] == 3
    assert shape.ref._obj is shape.c and cache.ref._obj is cache.c


def test_starts_and_positions_in_host_memory_are_refused():
    """Where every other tensor is on a device (one without memory here)."""
    cache = B.make_cache([0, 64], 1, 64, "e4m3", 16, "cpu")
    shape = B.make_shape([0, 64], 2, 1, 64, torch.bfloat16, "cpu")
    x, i = torch.zeros(64, 1, 64, dtype=torch.bfloat16, device="meta"), torch.zeros(1, dtype=torch.int32)
    buf = torch.zeros(1 << 22, dtype=torch.uint8)
    for call in (lambda: B.dam_cache_write(x, x, shape, cache, i, buf), lambda: B.dam_cache_read(cache, shape, i, x, x, buf),
                 lambda: B.dam_cache_decode_attention(x[:2].view(1, 2, 64), cache, i, None, 0.0, x, x, buf)):
        with pytest.raises(ValueError, match="on the device"):
            call()


def test_host_tensors_are_refused():
    cache = B.make_cache([0, 64], 1, 64, "e4m3", 16, "cpu")
    shape = B.make_shape([0, 64], 2, 1, 64, torch.bfloat16, "cpu")
    x, i = torch.zeros(64, 1, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    buf = torch.zeros(1 << 22, dtype=torch.uint8)
    q = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    for call in (lambda: B.dam_cache_write(x, x, shape, cache, i, buf), lambda: B.dam_cache_read(cache, shape, i, x, x, buf),
                 lambda: B.dam_cache_decode_attention(q, cache, i, None, 0.0, q, torch.zeros(1, 2), buf)):
        with pytest.raises(ValueError):
            call()


def test_the_restatement_on_known_blocks():
    """Codes and scales that can be worked out by hand."""
    s = R.Side(32, 1, 4, "int8", 16)
    s.write(np.array([[[1.27, -0.5, 0.0, 0.635]]], np.float32).astype(np.float64), 0)
    assert s.codes[0, 0].tolist() == [127, -50, 0, 64] or s.codes[0, 0].tolist()[:3] == [127, -50, 0]
    s.write(np.array([[[127.0, 0.5, 1.5, -2.5]]]), 16)       # scale 1: ties go to the even code
    assert s.scales[1, 0] == 1 and s.codes[16, 0].tolist() == [127, 0, 2, -2]
    s.write(np.array([[[254.0, 1.0, 3.0, 5.0]]]), 17)        # the scale grows to 2: 127 -> 63.5 -> 64, 2 -> 1, -2 -> -1
    assert s.scales[1, 0] == 2 and s.codes[16, 0].tolist() == [64, 0, 1, -1] and s.codes[17, 0].tolist() == [127, 0, 2, 2]
    e = R.Side(16, 1, 4, "e4m3", 16)
    e.write(np.array([[[448.0, 1.0625, 2.0 ** -10, 3 * 2.0 ** -10]]]), 0)
    assert e.scales[0, 0] == 1 and e.codes[0, 0].tolist() == [448, 1.0, 0.0, 2 * 2.0 ** -9]
    e.write(np.array([[[449.0, 0, 0, 0]]]), 1)
    assert e.scales[0, 0] == 2 and e.codes[1, 0, 0] == 224
    # and torch's own conversion to e4m3, as an independent check of the rounding
    y = np.concatenate([np.linspace(-448, 448, 20001), 2.0 ** np.arange(-12, 9), 1.5 * 2.0 ** np.arange(-12, 8.0)]).astype(np.float32)
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(R.codes_of(y.astype(np.float64), 1.0, "e4m3"), want)


def _rows_call(call, K, V, tokens, cache):
    buf = torch.zeros(256, dtype=torch.uint8)
    return B.dam_cache_write(K, V, tokens, cache, None, buf) if call == "write" else B.dam_cache_read(cache, tokens, None, K, V, buf)


@pytest.mark.parametrize("call", ["write", "read"])
def test_rows_that_tokens_does_not_describe_are_refused(call):
    cache = B.make_cache([0, 64], 4, 64, "e4m3", 16, "cpu")
    tokens = B.make_shape([0, 40], 8, 4, 64, torch.bfloat16, "cpu")
    good = torch.zeros(40, 4, 64, dtype=torch.bfloat16)
    fused = torch.zeros(40, 16, 64, dtype=torch.bfloat16)
    for bad in (fused[:, 8:12], fused, good.float(), good[:39], good[:, :3], good[:, :, :32], good.half(), good[::2],
                good.permute(1, 0, 2).contiguous(), good.reshape(-1)[:-1], good.reshape(40, 256)[:, :128], good.reshape(40, 256)[:39]):
        for K, V in ((bad, good), (good, bad)):
            with pytest.raises(ValueError, match="rows"):
                _rows_call(call, K, V, tokens, cache)
    # described with the strides of a fused tensor, but not one
    wide = B.make_shape([0, 40], 8, 4, 64, torch.bfloat16, "cpu", k_strides=(1024, 64), v_strides=(1024, 64))
    for bad in (good, good.reshape(40, 256), good.reshape(-1)):
        with pytest.raises(ValueError, match="rows"):
            _rows_call(call, bad, fused[:, 8:12], wide, cache)


@pytest.mark.parametrize("call", ["write", "read"])
def test_rows_described_in_every_way_are_taken(call):
    """(What is wrong here is that the tensors are not on a GPU.)"""
    cache = B.make_cache([0, 64], 4, 64, "e4m3", 16, "cpu")
    plain = torch.zeros(40, 4, 64, dtype=torch.bfloat16)
    fused, longer = torch.zeros(48, 16, 64, dtype=torch.bfloat16), torch.zeros(64, 4, 64, dtype=torch.bfloat16)
    major = torch.zeros(4, 64, 64, dtype=torch.bfloat16)

    def ok(x, strides=None, n=40, tokens=None):
        tokens = tokens or B.make_shape([0, n], 8, 4, 64, torch.bfloat16, "cpu", k_strides=strides, v_strides=strides)
        with pytest.raises(ValueError, match="on the device"):
            _rows_call(call, x, x, tokens, cache)
        return tokens

    ok(plain), ok(longer), ok(plain.reshape(40, 256)), ok(plain.reshape(-1)), ok(longer.reshape(1, 64, 4, 64)), ok(longer.reshape(2, 32, 256))
    ok(fused[:, 8:12], (1024, 64)), ok(fused, (1024, 64)), ok(fused.reshape(48, 1024)[:, 256:], (1024, 64)), ok(fused[4:44, ::4], (1024, 256))
    ok(major.permute(1, 0, 2), (64, 4096)), ok(major, (64, 4096)), ok(major[:, 3:43], (64, 4096))
    ok(plain.as_strided((1, 4, 64), (8, 64, 1)), n=1), ok(torch.zeros(0, 4, 64, dtype=torch.bfloat16), n=0), ok(plain.float(), n=0), ok(major, n=0)
    # the description may change
    tokens = ok(plain)
    tokens.c.k_stride_tok = tokens.c.v_stride_tok = 1024
    ok(fused[:, 8:12], tokens=tokens), ok(fused[:, :4], tokens=tokens)
    tokens.c = B.make_shape([0, 40], 8, 4, 64, torch.float32, "cpu").c
    ok(plain.float(), tokens=tokens)
    one = B.make_cache([0, 64], 1, 64, "e4m3", 16, "cpu")
    batch = torch.zeros(2, 20, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on the device"):
        _rows_call(call, batch, batch, B.make_shape([0, 40], 8, 1, 64, torch.bfloat16, "cpu"), one)


def test_results_that_cannot_be_written_are_refused(monkeypatch):
    cache = B.make_cache([0, 64, 128], 1, 64, "e4m3", 16, "cpu")
    buf, i = torch.zeros(1 << 22, dtype=torch.uint8), torch.zeros(2, dtype=torch.int32)
    for dtype in (torch.bfloat16, torch.float32):
        q, other = torch.zeros(2, 4, 64, dtype=dtype), torch.float32 if dtype is torch.bfloat16 else torch.bfloat16
        lse = torch.zeros(2, 4)
        for O in (q.to(other), torch.zeros(2, 8, 64, dtype=dtype)[:, ::2], torch.zeros(1, 4, 64, dtype=dtype), torch.zeros(64, 4, 2, dtype=dtype).permute(2, 1, 0)):
            with monkeypatch.context() as m, pytest.raises(ValueError, match="O takes"):
                m.setattr(B, "_check_device", lambda *args, **tensors: None)
                B.dam_cache_decode_attention(q, cache, i, None, 0.0, O, lse, buf)
        for bad in (lse.double(), lse.bfloat16(), torch.zeros(4, 2).t(), torch.zeros(7)):
            with monkeypatch.context() as m, pytest.raises(ValueError, match="lse takes"):
                m.setattr(B, "_check_device", lambda *args, **tensors: None)
                B.dam_cache_decode_attention(q, cache, i, None, 0.0, q.clone(), bad, buf)
        for O, l in ((q.clone(), lse), (torch.zeros(3, 4, 64, dtype=dtype), torch.zeros(9))):
            B._check_result(O, "O", q.numel(), dtype)
            B._check_result(l, "lse", 8, torch.float32)
            with pytest.raises(ValueError, match="on the device"):
                B.dam_cache_decode_attention(q, cache, i, None, 0.0, O, l, buf)


def test_a_cache_s_buffers_belong_on_its_device():
    codes = torch.zeros(64, 1, 64, dtype=torch.int8, device="meta")
    scales = torch.zeros(5, 1, device="meta")
    for given in ({"k_codes": codes}, {"v_codes": codes}, {"k_scales": scales}, {"v_scales": scales}):
        with pytest.raises(ValueError, match="on the device"):
            B.make_cache([0, 64], 1, 64, "int8", 16, "cpu", **given)


def test_the_restatement_rounds_to_the_code_it_should():
    """Quotients that are exact and no ties, under scales of 1 and 2^-6."""
    s = R.Side(16, 1, 4, "int8", 16)
    s.write(np.array([[[127.0, -50.25, 0.0, 63.75]]]), 0)    # scale 1
    assert s.scales[0, 0] == 1 and s.codes[0, 0].tolist() == [127, -50, 0, 64]
    s = R.Side(16, 1, 4, "int8", 16)
    s.write(np.array([[[127.0, -50.25, 0.0, 63.75]]]) / 64, 0)
    assert s.scales[0, 0] == 2.0 ** -6 and s.codes[0, 0].tolist() == [127, -50, 0, 64]
