"""A KV cache held in 8 bits, as cases that a timing harness can run one pass at a time.

The cache keeps K and V of every sequence as 8-bit codes with one fp32 scale for each block of tokens and KV head; a
value is code times scale.  Kinds:

  write   new tokens of every sequence are quantised into the cache, and what the cache then holds of them (and of the
          tokens that share their first block) is read back
  read    tokens of the cache are read back as K and V rows, as chunked prefill wants them
  attend  one new token per sequence attends to everything its sequence's cache holds
  masked  the same under the stored patterns of a mask blob: matched columns and diagonals only

Codes: "int8" with scale = amax / 127 (an IEEE division), code = the integer nearest to value / scale, ties to even;
"e4m3" with scale = the least power of two that brings amax to 448 or less, code = value / scale rounded to nearest
even.  No scale is below 2^-126.  A token that is added to a block whose scale is too small for it raises that scale,
and the tokens that are there already are read back and quantised again.
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
TINY = 2.0 ** -126


def _case(name, kind, lengths, heads=32, kv_heads=8, dim=128, dtype="bf16", code="int8", block=64, tokens=0, pcl=0):
    """`lengths`: tokens every sequence's cache has room for; `tokens`: how many of them a write brings (0: all);
    `pcl`: window of the masks' patterns."""
    return {"name": name, "kind": kind, "lengths": " ".join(str(n) for n in lengths), "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "code": code, "block": block, "tokens": tokens, "pcl": pcl}


def listed():
    return [
        # generation for a single user: the new token of one sequence enters the cache
        _case("write_1_token", "write", [8000], tokens=1),
        # generation for a full batch: one token of each of 64 sequences
        _case("write_64_tokens", "write", [2048] * 64, tokens=1, code="e4m3"),
        # prompts of mixed and odd lengths, just computed, enter the cache whole
        _case("write_prompts", "write", [4096, 16384, 777, 32768, 9001, 65536]),
        # the keys of a prompt that has reached 8k tokens, for its next chunk
        _case("read_8k", "read", [8192], code="e4m3"),
        # the same for a batch of mixed and odd lengths, fp32 rows of 64
        _case("read_mixed_fp32", "read", [4096, 16384, 777, 32768, 9001, 65536], heads=16, kv_heads=4, dim=64, dtype="fp32",
              block=32),
        # a short chat of an odd length: launches and latency
        _case("attend_1x1237", "attend", [1237], code="e4m3"),
        # a single user at an ordinary length
        _case("attend_1x8k", "attend", [8000]),
        # a single user at the longest context
        _case("attend_1x128k", "attend", [131072]),
        # requests of mixed and odd lengths, fp32 queries, rows of 64, four KV heads
        _case("attend_mixed_fp32", "attend", [4096, 16384, 777, 32768, 9001, 65536], heads=16, kv_heads=4, dim=64,
              dtype="fp32", code="e4m3", block=16),
        # a full batch
        _case("attend_64x32k", "attend", [32768] * 64),
        # a single user under the stored patterns
        _case("masked_1x8k", "masked", [8000], pcl=1024),
        # a full batch under the stored patterns
        _case("masked_64x32k", "masked", [32768] * 64, code="e4m3", pcl=1024),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("write", "write", "read", "attend", "attend", "masked"))
    heads, kv_heads = rng.choice(((32, 8), (32, 8), (16, 4), (8, 8), (24, 8), (8, 1), (32, 2)))
    form = {"heads": heads, "kv_heads": kv_heads, "dim": rng.choice((128, 128, 64)), "code": rng.choice(("int8", "e4m3")),
            "block": rng.choice((16, 32, 64, 64, 128)), "dtype": rng.choice(("bf16", "bf16", "bf16", "fp32"))}
    if kind in ("write", "read"):
        total = _log_uniform(rng, 64, 98304 if form["dtype"] == "bf16" else 49152)
        n = rng.choice((1, 2, 5, 16))
        cuts = sorted(rng.randrange(1, total) for _ in range(n - 1))
        lengths = [b - a for a, b in zip([0] + cuts, cuts + [total])]
        tokens = _log_uniform(rng, 1, 64) if kind == "write" and rng.random() < 0.4 else 0
        return _drawn(kind, lengths, tokens=tokens, **form)
    n = _log_uniform(rng, 1, 48)
    lengths = [_log_uniform(rng, 1, 32768) for _ in range(n)]
    return _drawn(kind, lengths, pcl=rng.choice((128, 512, 1024)) if kind == "masked" else 0, **form)


def _drawn(kind, lengths, **kwargs):
    case = _case("", kind, lengths, **kwargs)
    del case["name"]
    return case


def _lengths(case):
    return [int(n) for n in case["lengths"].split()]


def _cu(lengths):
    return [0] + list(np.cumsum(lengths).tolist())


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _added(case, lengths):
    """Tokens that a write brings, per sequence."""
    return [min(n, case["tokens"]) if case["tokens"] else n for n in lengths]


# ---- what the inputs are -----------------------------------------------------------------------------------------------


def _rows(gen, n, kv, d, dtype, gain):
    """K or V rows as a layer makes them: every channel has a size of its own, a few are large."""
    return (torch.randn(n, kv, d, generator=gen, device=DEVICE) * gain).to(dtype)


def _gain(gen, kv, d):
    return torch.exp(0.7 * torch.randn(kv, d, generator=gen, device=DEVICE))


def _filled(gen, case, lengths):
    """Codes and scales of a cache that is full: blocks of normal values, scaled to their largest."""
    T, kv, d, blk = sum(lengths), case["kv_heads"], case["dim"], case["block"]
    codes = torch.empty(T, kv, d, dtype=CODES[case["code"]], device=DEVICE)
    for at in range(0, T, 65536):
        x = torch.randn(min(65536, T - at), kv, d, generator=gen, device=DEVICE)
        if case["code"] == "int8":
            codes[at:at + 65536] = (x * 30).round().clamp(-127, 127).to(torch.int8)
        else:
            codes[at:at + 65536].view(torch.uint8).copy_((x * 75).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    rows = T // blk + len(lengths)
    unit = torch.exp(0.3 * torch.randn(rows, kv, generator=gen, device=DEVICE))
    if case["code"] == "int8":
        return codes, unit / 30
    return codes, torch.exp2(torch.round(torch.log2(unit)) - 6)


def _patterns(case, seed):
    """What the heads of every sequence keep, as truth values [sequence, head, window]: columns and diagonals of the true
    mask, and the columns and diagonals that match with mu = 0.8 (a pattern matches when its count of kept cells reaches
    mu times its size).  A cell is kept when its column or its diagonal is planted, so a column that is not planted has
    as many kept cells as there are planted diagonals short enough to cross it, and the other way round."""
    lengths, heads, pcl = _lengths(case), case["heads"], case["pcl"]
    L = [min(n, pcl) for n in lengths]
    longest = max(L)
    rng = np.random.RandomState((seed * 1009 + 17) % (2 ** 31))
    n = len(lengths)
    size = np.array(L)[:, None, None] - np.arange(longest)[None, None, :]          # cells of column or diagonal k
    exists = size > 0
    width = rng.choice([0, 0, 16, 48, 96, 192], size=(n, heads, 1))
    diag = (np.arange(longest)[None, None, :] < width) & exists
    col = (rng.rand(n, heads, longest) < rng.rand(n, heads, 1) ** 2 * 0.04) & exists
    col[:, :, 0] |= rng.rand(n, heads) < 0.85

    def match(planted, other):
        crossing = np.concatenate([np.zeros((n, heads, 1), np.int64), np.cumsum(other, axis=2)], axis=2)
        crossing = np.take_along_axis(crossing, np.broadcast_to(np.maximum(size, 0), planted.shape), axis=2)
        count = np.where(planted, size, crossing)
        return exists & (count.astype(np.float32) >= np.float32(0.8) * size.astype(np.float32))

    return L, col, diag, match(col, diag), match(diag, col)


def _positions(case, seed, lengths):
    rng = random.Random(seed)
    return [rng.randrange(n // 2, n) for n in lengths]


def prepare(case, seed):
    lengths, kind = _lengths(case), case["kind"]
    kv, d, dtype, n = case["kv_heads"], case["dim"], DTYPES[case["dtype"]], len(lengths)
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    s = {"kind": kind, "code": case["code"], "block": case["block"], "dtype": dtype, "G": case["heads"] // kv,
         "capacity": _ints(_cu(lengths))}
    s["k_codes"], s["k_scales"] = _filled(gen, case, lengths)
    s["v_codes"], s["v_scales"] = _filled(gen, case, lengths)
    if kind == "write":
        added = _added(case, lengths)
        rng = random.Random(case["lengths"])                     # (where a write begins sets the shape of what is read back)
        starts = [rng.randrange(c // 2, c - m + 1) if m < c // 2 else c - m for c, m in zip(lengths, added)]
        first = [p // case["block"] * case["block"] for p in starts]
        s["K"] = _rows(gen, sum(added), kv, d, dtype, _gain(gen, kv, d))
        s["V"] = _rows(gen, sum(added), kv, d, dtype, _gain(gen, kv, d))
        back = [p + m - f for p, m, f in zip(starts, added, first)]
        s["tokens_cu"], s["starts"] = _ints(_cu(added)), _ints(starts)
        s["back_cu"], s["back_starts"] = _ints(_cu(back)), _ints(first)
        counts = {"tokens": _cu(added), "back": _cu(back)}
        s["back_total"] = sum(back)
    elif kind == "read":
        s["back_cu"], s["back_starts"] = s["capacity"], _ints([0] * n)
        counts = {"back": _cu(lengths)}
        s["back_total"] = sum(lengths)
    else:
        positions = _positions(case, seed, lengths)
        s["q"] = torch.randn(n, case["heads"], d, generator=gen, device=DEVICE).to(dtype)
        s["positions"], s["longest"] = _ints(positions), max(positions) + 1
        if kind == "masked":
            L, col, diag, V, D = (x if isinstance(x, list) else torch.from_numpy(x).to(DEVICE) for x in _patterns(case, seed))
            inside = (s["positions"] < _ints(L))[:, None, None]
            s["columns"], s["diagonals"], s["window"] = torch.where(inside, col, V), torch.where(inside, diag, D), _ints(L)
    if not own:
        return s
    # what a program that uses the library keeps beside its data: descriptions of the cache and of the tokens, scratch,
    # outputs, the masks that were built when the prompt's window had been computed
    from paper_2506_11104_b200 import binding as dam
    s["cache"] = dam.make_cache(_cu(lengths), kv, d, case["code"], case["block"], DEVICE, s["k_codes"], s["v_codes"],
                                s["k_scales"], s["v_scales"])
    if kind in ("write", "read"):
        for name, cu in counts.items():
            s[name] = dam.make_shape(cu, case["heads"], kv, d, dtype, DEVICE)
        s["K_back"] = torch.empty(counts["back"][-1], kv, d, dtype=dtype, device=DEVICE)
        s["V_back"] = torch.empty_like(s["K_back"])
        s["scratch"] = torch.empty(256, dtype=torch.uint8, device=DEVICE)
        return s
    s["scratch"] = torch.empty(dam.dam_cache_sizes(s["cache"], case["heads"])[1], dtype=torch.uint8, device=DEVICE)
    s["O"], s["lse"] = torch.empty_like(s["q"]), torch.empty(n, case["heads"], device=DEVICE)
    s["mask"] = None
    if kind == "masked":
        maps = []
        for b, size in enumerate(L):
            i = torch.arange(size, device=DEVICE)
            r = i[:, None] - i[None, :]
            kept = col[b, :, None, :size] | diag[b][:, r.clamp(min=0)]
            maps.append((kept & (r >= 0)).float().reshape(-1))
        windows = dam.make_shape(_cu(L), case["heads"], kv, d, dtype, DEVICE)
        s["mask"], _ = dam.dam_build_masks_from_scores(torch.cat(maps), windows, dam.make_rule(case["pcl"], 0.3, 0.8))
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------


def run(s):
    kind = s["kind"]
    if own:
        from paper_2506_11104_b200 import binding as dam
        if kind in ("attend", "masked"):
            dam.dam_cache_decode_attention(s["q"], s["cache"], s["positions"], s["mask"], O=s["O"], lse=s["lse"],
                                           scratch=s["scratch"])
            return {"O": s["O"], "lse": s["lse"]}
        if kind == "write":
            dam.dam_cache_write(s["K"], s["V"], s["tokens"], s["cache"], s["starts"], scratch=s["scratch"])
        dam.dam_cache_read(s["cache"], s["back"], s["back_starts"], K=s["K_back"], V=s["V_back"], scratch=s["scratch"])
        out = {"K": s["K_back"], "V": s["V_back"]}
    elif kind in ("attend", "masked"):
        return _plain_attend(s)
    else:
        if kind == "write":
            _plain_write(s, s["K"], s["k_codes"], s["k_scales"])
            _plain_write(s, s["V"], s["v_codes"], s["v_scales"])
        out = {"K": _plain_read(s, s["k_codes"], s["k_scales"]), "V": _plain_read(s, s["v_codes"], s["v_scales"])}
    if kind == "write":
        out["k_scales"], out["v_scales"] = s["k_scales"], s["v_scales"]
    return out


# ---- the plain form ----------------------------------------------------------------------------------------------------


def _values(codes, at, scales, row):
    """The values that the codes of the tokens `at` stand for; `row`: their blocks."""
    c = codes.view(torch.uint8)[at].view(codes.dtype).float()
    return c * scales[row][..., None]


def _scale_of(amax, code):
    if code == "int8":
        return (amax / torch.full_like(amax, 127)).clamp(min=TINY)  # (a division by a number is a product with its inverse)
    mantissa, exponent = torch.frexp(amax)                       # amax = mantissa * 2^exponent, mantissa in [1/2, 1)
    exponent = torch.where(mantissa <= 0.875, exponent - 9, exponent - 8).clamp(min=-126)
    exponent = torch.where(amax > 0, exponent, torch.full_like(exponent, -126))
    return ((exponent + 127) << 23).view(torch.float32)


def _quantised(x, scale, code):
    if code == "int8":                                           # in 64 bits: values next to the border of two codes
        return torch.round(x.double() / scale.double()).clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return (x / scale).to(torch.float8_e4m3fn).view(torch.uint8)


def _places(cu, capacity, starts, total, block):
    """Of every packed token: its sequence, its place in the cache, and the row of its block's scales."""
    t = torch.arange(total, device=cu.device)
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    p = starts[seq] + t - cu[seq]
    return seq, capacity[seq] + p, capacity[seq] // block + seq + p // block


def _plain_write(s, x, codes, scales):
    code, blk, capacity, cu, starts = s["code"], s["block"], s["capacity"].long(), s["tokens_cu"].long(), s["starts"].long()
    seq, at, row = _places(cu, capacity, starts, x.shape[0], blk)
    x = x.float()
    amax = torch.zeros_like(scales).scatter_reduce_(0, row[:, None].expand(-1, scales.shape[1]), x.abs().amax(dim=2), "amax")
    fresh = _scale_of(amax, code)
    # a block that was begun before keeps its scale, or gets the larger one of its new tokens
    n = torch.arange(starts.numel(), device=x.device)
    old_row = capacity[:-1] // blk + n + starts // blk
    begun = (starts % blk > 0)[:, None]
    before, now = scales[old_row], fresh[old_row]
    now = torch.where(begun, torch.maximum(before, now), now)
    fresh[old_row] = now
    touched = torch.zeros(scales.shape[0], dtype=torch.bool, device=x.device)
    touched[row] = True
    # tokens that are there already are read back and quantised again where the scale grew
    j = torch.arange(blk, device=x.device)
    there = capacity[:-1, None] + (starts // blk * blk)[:, None] + j
    live = j < (starts % blk)[:, None]
    there = torch.where(live, there, at[0])                       # (no token yet: a place that is written below)
    bytes_ = codes.view(torch.uint8)
    held = _values(codes, there, scales, old_row[:, None].expand(-1, blk))
    again = _quantised(held, now[:, None, :, None], code)
    grew = live[:, :, None, None] & (now > before)[:, None, :, None]
    bytes_[there] = torch.where(grew, again, bytes_[there])
    scales.copy_(torch.where(touched[:, None], fresh, scales))
    bytes_[at] = _quantised(x, scales[row][..., None], code)


def _plain_read(s, codes, scales):
    cu, capacity, starts = s["back_cu"].long(), s["capacity"].long(), s["back_starts"].long()
    _, at, row = _places(cu, capacity, starts, s["back_total"], s["block"])
    return _values(codes, at, scales, row).to(s["dtype"])


def _plain_attend(s):
    capacity, pos, q = s["capacity"].long(), s["positions"].long(), s["q"]
    n, d, G, S, blk = pos.numel(), q.shape[2], s["G"], s["longest"], s["block"]
    j = torch.arange(S, device=q.device)
    keep = (j <= pos[:, None])[:, None, :]
    at = (capacity[:-1, None] + j).clamp(max=s["k_codes"].shape[0] - 1)
    row = (capacity[:-1, None] // blk + torch.arange(n, device=q.device)[:, None] + j // blk).clamp(max=s["k_scales"].shape[0] - 1)
    K = _values(s["k_codes"], at, s["k_scales"], row)
    x = torch.einsum("bkgd,bskd->bkgs", q.float().view(n, -1, G, d), K).reshape(n, -1, S) / math.sqrt(d)
    del K
    if s["kind"] == "masked":
        L, C, D = s["window"].long(), s["columns"], s["diagonals"]
        far = pos[:, None] - j                                    # how far behind the new token a key lies
        most = C.shape[2] - 1
        column = C[:, :, j.clamp(max=most)] & (j < L[:, None])[:, None, :]
        index = far.clamp(0, most)[:, None, :].expand(-1, C.shape[1], -1)
        diagonal = torch.gather(D, 2, index) & ((far >= 0) & (far < L[:, None]))[:, None, :]
        keep = keep & (column | diagonal)
    x = torch.where(keep, x, torch.full_like(x, -math.inf))
    m = x.amax(dim=2, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = torch.exp(x - m)
    l = p.sum(dim=2)
    V = _values(s["v_codes"], at, s["v_scales"], row)
    V = torch.where((j <= pos[:, None])[:, :, None, None], V, torch.zeros_like(V))
    O = torch.einsum("bkgs,bskd->bkgd", p.view(n, -1, G, S), V).reshape(n, -1, d) / torch.where(l > 0, l, torch.ones_like(l))[..., None]
    return {"O": O.to(q.dtype), "lse": m[..., 0] + torch.log(l)}


# ---- from the definition, in 64 bits -----------------------------------------------------------------------------------


def _exact_scale(amax, code):
    """The scale that the cache stores (an fp32 number) for a block whose largest magnitude is `amax`."""
    a = amax.cpu().numpy().astype(np.float64)
    if code == "int8":
        return torch.from_numpy(np.maximum(a.astype(np.float32) / np.float32(127), np.float32(TINY)).astype(np.float64)).to(DEVICE)
    k = np.where(a > 0, np.ceil(np.log2(np.where(a > 0, a, 1.0) / 448.0)), -126.0)
    k = np.where(a > 448.0 * np.exp2(k), k + 1, k)                # (log2 of a power of two may be off by its last bit)
    k = np.where(a <= 448.0 * np.exp2(k - 1), k - 1, k)
    return torch.from_numpy(np.exp2(np.maximum(k, -126.0))).to(DEVICE)


def _exact_codes(x, scale, code):
    y = x / scale
    if code == "int8":
        return torch.round(y).clamp(-127, 127)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)      # spacing of e4m3 around y
    return torch.round(y / step) * step


def _exact_cache(s, x, codes, scales):
    """Values [T, kv, d] and scales that the cache holds after the write of `x` (None: as it is)."""
    blk, code = s["block"], s["code"]
    cap = s["capacity"].tolist()
    scales = scales.double().clone()
    values = torch.empty(codes.shape, dtype=torch.float64, device=DEVICE)
    for b, (t0, t1) in enumerate(zip(cap[:-1], cap[1:])):
        row = t0 // blk + b + torch.arange(t1 - t0, device=DEVICE) // blk
        values[t0:t1] = codes[t0:t1].double() * scales[row][..., None]
    if x is None:
        return values, scales
    cu, starts = s["tokens_cu"].tolist(), s["starts"].tolist()
    for b, start in enumerate(starts):
        new = x[cu[b]:cu[b + 1]].double()
        t0, row0 = cap[b], cap[b] // blk + b
        end = start + new.shape[0]
        if end == start:
            continue
        first = start // blk * blk
        if start > first:                                        # the block that was begun before
            stop = min(first + blk, end)
            part, row = new[:stop - start], row0 + first // blk
            scale = torch.maximum(scales[row], _exact_scale(part.abs().amax(dim=(0, 2)), code))
            grew = (scale > scales[row])[None, :, None]
            held = values[t0 + first:t0 + start]
            held = held.float().double()                         # what is read back is an fp32 number
            values[t0 + first:t0 + start] = torch.where(grew, _exact_codes(held, scale[None, :, None], code) * scale[None, :, None], held)
            values[t0 + start:t0 + stop] = _exact_codes(part, scale[None, :, None], code) * scale[None, :, None]
            scales[row] = scale
            new, start = new[stop - start:], stop
        if end == start:
            continue
        count = -(-new.shape[0] // blk)
        padded = torch.zeros(count * blk, *new.shape[1:], dtype=torch.float64, device=DEVICE)
        padded[:new.shape[0]] = new
        padded = padded.view(count, blk, *new.shape[1:])
        scale = _exact_scale(padded.abs().amax(dim=(1, 3)), code)
        got = _exact_codes(padded, scale[:, None, :, None], code) * scale[:, None, :, None]
        values[t0 + start:t0 + end] = got.view(count * blk, *new.shape[1:])[:end - start]
        scales[row0 + start // blk:row0 + start // blk + count] = scale
    return values, scales


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    cap, blk = s["capacity"].tolist(), s["block"]
    if kind in ("write", "read"):
        out = {}
        for name, x in (("K", s.get("K")), ("V", s.get("V"))):
            low = name.lower()
            values, scales = _exact_cache(s, x, s[low + "_codes"], s[low + "_scales"])
            cu, starts = s["back_cu"].tolist(), s["back_starts"].tolist()
            out[name] = torch.cat([values[cap[b] + p:cap[b] + p + cu[b + 1] - cu[b]] for b, p in enumerate(starts)])
            if kind == "write":
                out[low + "_scales"] = scales
        return out
    n, heads, d = s["q"].shape
    O, lse = torch.zeros(n, heads, d, dtype=torch.float64, device=DEVICE), torch.full((n, heads), -math.inf, dtype=torch.float64, device=DEVICE)
    for b, i in enumerate(s["positions"].tolist()):
        row = cap[b] // blk + b + torch.arange(i + 1, device=DEVICE) // blk
        K, V = (s[c + "_codes"][cap[b]:cap[b] + i + 1].double() * s[c + "_scales"][row].double()[..., None] for c in "kv")
        kept = torch.ones(heads, i + 1, dtype=torch.bool, device=DEVICE)
        if kind == "masked":
            L = int(s["window"][b])
            kept[:] = False
            near = min(L, i + 1)
            kept[:, :near] |= s["columns"][b, :, :near]
            kept[:, i + 1 - near:] |= s["diagonals"][b, :, :near].flip(1)
        for h in range(heads):
            x = K[:, h // s["G"]] @ s["q"][b, h].double() / math.sqrt(d)
            x = x[kept[h]]
            if x.numel():
                O[b, h] = torch.softmax(x, 0) @ V[:, h // s["G"]][kept[h]]
                lse[b, h] = torch.logsumexp(x, 0)
    return {"O": O, "lse": lse}


# ---- what a pass cannot do without -------------------------------------------------------------------------------------


def work(case):
    lengths, heads, kv, d, blk = _lengths(case), case["heads"], case["kv_heads"], case["dim"], case["block"]
    item, kind = (2 if case["dtype"] == "bf16" else 4), case["kind"]
    if kind == "read":
        return {"bytes": sum(lengths) * 2 * kv * d * (1 + item) + sum(-(-n // blk) for n in lengths) * 2 * kv * 4,
                "flops": sum(lengths) * 2 * kv * d}
    if kind == "write":
        added = _added(case, lengths)
        begun = sum(m < c for c, m in zip(lengths, added)) * (blk - 1) / 2   # tokens that share the first block
        new, blocks = sum(added), sum(-(-m // blk) for m in added)
        return {"bytes": 2 * kv * (new * d * (2 * item + 1) + begun * d * (1 + item) + blocks * 4),
                "flops": 2 * kv * d * (4 * new + begun)}
    queries = len(lengths) * heads * (2 * d * item + 4)
    if kind == "attend":
        keys = sum(0.75 * n for n in lengths)                                # positions lie in the second half
        return {"bytes": keys * 2 * kv * (d + 4 / blk) + queries, "flops": keys * heads * 4 * d}
    L, col, diag, V, D = _patterns(case, 0)
    pos = np.array([3 * n // 4 for n in lengths])
    inside = (pos < np.array(L))[:, None, None]
    C, D = np.where(inside, col, V), np.where(inside, diag, D)
    k = np.arange(C.shape[2])[None, None, :]
    D = D & (k <= pos[:, None, None])
    C = C & (k <= pos[:, None, None])
    twice = (C & np.where(pos[:, None, None] - k < C.shape[2], np.take_along_axis(D, np.clip(pos[:, None, None] - k, 0, C.shape[2] - 1) + 0 * C, axis=2), False)).sum()
    per_head = C.sum() + D.sum() - twice
    group = (len(lengths), kv, heads // kv, C.shape[2])
    union = C.reshape(group).any(2).sum() + D.reshape(group).any(2).sum() - twice / (heads // kv)
    return {"bytes": float(union * 2 * (d + 4) + 2 * len(lengths) * heads * C.shape[2] / 8 + queries),
            "flops": float(per_head * 4 * d)}
