"""The attention operators on the GPU against plain implementations in 64 bits.

Tolerances of the attention tests (worst cases, per output element, derived from the arithmetic):
  scores      each of hd products and sums in fp32, the query possibly held as two 16-bit planes (2^-16 relative), the exponent's
              argument and the exponential to a few ulp:  ds = scale * sum_e |q_e k_e| * (2^-16 + hd 2^-23) + |score| 2^-21 + 2^-20
  weights     a relative error of a weight is at most 2 ds (its own and the denominator's), weights meet the values as two 16-bit
              planes (decode: 2^-16; one fp16, half a step of 2^-11, where the output is 16 bits and the cache is not bf16: with a
              single row the weight times the value's scale is rounded once and the output once more, 2^-11 + 2^-8 together) or
              rounded to the type (prompt: half a step, eps / 2, as the largest exact weight may lie anywhere in its binade), and n
              additions in fp32 lose n 2^-23 of the sum of absolute values
  output      half a step of its type
so |out - exact| <= (2 ds + w + n 2^-23) * sum_j p_j |v_j| + eps(out) / 2 * |exact| + the type's smallest step."""
import math

import pytest
import torch

from paper_2505_18164_b200 import mdi

pytestmark = pytest.mark.gpu

I8, E4M3, F16, BF16, F32 = torch.int8, torch.float8_e4m3fn, torch.float16, torch.bfloat16, torch.float32
DEV = "cuda"


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device=DEV)


def starts(counts):
    s = [0]
    for c in counts:
        s.append(s[-1] + c)
    return ints(s)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


# ---- the cache's types from their definition -------------------------------------------------------------------------
def quantise(x, store):
    """(stored elements, scales) of rows x[..., hd], in 64 bits; rows with a non-finite element: zeros and a NaN scale."""
    if store in (F16, BF16):
        return x.to(store), None
    d = x.double()
    big = d.abs().amax(-1)
    bad = ~torch.isfinite(big)
    d, big = torch.where(bad[..., None], torch.zeros_like(d), d), torch.where(bad, torch.zeros_like(big), big)
    if store == I8:
        scale = (big / 127).float().double().clamp_min(2.0 ** -126)   # in 64 bits: a float tensor over a number is a product with its reciprocal
        q = torch.round(d / scale[..., None]).to(I8)
    else:
        k = torch.full_like(big, -126)
        for e in range(-126, 121):                       # the smallest power of two that is large enough
            k = torch.where(big > 448 * 2.0 ** e, torch.full_like(k, e + 1), k)
        scale = torch.exp2(k)
        y = d / scale[..., None]
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
        q = (torch.round(y / step) * step).float().to(E4M3)  # exact
    return q, torch.where(bad, torch.full_like(scale, math.nan), scale).float()


class Cache:
    """A pool whose pages are handed out in random order; everything not written holds garbage (NaN where the type has one)."""

    def __init__(self, store, kv, hd, page, capacity, slots, seed=0, spare=2, pages_per_seq=None):
        g = torch.Generator().manual_seed(seed)
        per = pages_per_seq or max(1, -(-capacity // page))
        n = slots * per + spare
        self.store, self.kv, self.hd, self.page, self.slots, self.per = store, kv, hd, page, slots, per
        if store in (I8, E4M3):
            raw = torch.full((n, 2, kv, page, hd), 127, dtype=I8, device=DEV)   # e4m3: 0x7f is NaN
            self.pool = raw if store == I8 else raw.view(E4M3)
            self.scale = torch.full((n, 2, kv, page), math.nan, device=DEV)
        else:
            self.pool, self.scale = torch.full((n, 2, kv, page, hd), math.nan, dtype=store, device=DEV), None
        self.table = torch.randperm(n, generator=g)[: slots * per].view(slots, per).to(torch.int32).to(DEV)
        self.handle = mdi.KvCache(self.pool, self.table, scale=self.scale)

    def raw(self):
        return self.pool.view(torch.uint8) if self.store == E4M3 else self.pool

    def put(self, slot, first, k, v):
        """Plain form of the append (k, v: [rows, kv, hd])."""
        at = torch.arange(first, first + k.shape[0], device=DEV)
        page, off = self.table[slot, at // self.page].long(), at % self.page
        for which, x in ((0, k), (1, v)):
            q, s = quantise(x, self.store)
            self.raw()[page, which, :, off] = q.view(torch.uint8) if self.store == E4M3 else q
            if s is not None:
                self.scale[page, which, :, off] = s

    def get(self, which, slot, first, count):
        """Stored values of rows first .. first + count - 1, [count, kv, hd] fp64."""
        at = torch.arange(first, first + count, device=DEV)
        page, off = self.table[slot, at // self.page].long(), at % self.page
        x = self.raw()[page, which, :, off]
        x = (x.view(E4M3) if self.store == E4M3 else x).double()
        return x if self.scale is None else x * self.scale[page, which, :, off].double()[..., None]


def attend(q, k, v, scale, seen):
    """(out, sum p|v|, ds without the rounding terms' constants) in 64 bits: q [heads, rows, hd], k, v [keys, kv, hd], seen [rows]."""
    heads, rows, hd = q.shape
    group = heads // k.shape[1]
    k, v = (x.double().transpose(0, 1).repeat_interleave(group, 0) for x in (k, v))
    q = q.double()
    s = q @ k.transpose(1, 2) * scale
    hidden = torch.arange(k.shape[1], device=DEV)[None, :] >= seen[:, None]
    ds = (q.abs() @ k.abs().transpose(1, 2) * scale * (2.0 ** -16 + hd * 2.0 ** -23) + s.abs() * 2.0 ** -21).masked_fill(hidden, 0)
    ds = ds.amax(-1) + 2.0 ** -20 if k.shape[1] else torch.zeros(heads, rows, device=DEV, dtype=torch.float64)
    s = s.masked_fill(hidden, -math.inf)
    m = s.amax(-1, keepdim=True) if k.shape[1] else torch.zeros(heads, rows, 1, device=DEV, dtype=torch.float64)
    p = torch.exp(s - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    v0 = torch.where(hidden.all(0)[None, :, None], torch.zeros_like(v), v)
    return p @ v0, p @ v0.abs(), ds


def close(got, want, mag, ds, n, w, dtype):
    tol = (2 * ds[..., None] + w + n * 2.0 ** -23) * mag + torch.finfo(dtype).eps / 2 * want.abs() + torch.finfo(dtype).tiny
    err = (got.double() - want).abs()
    assert torch.isfinite(got).all()
    worst = (err / tol).max().item()
    assert worst <= 1.0, f"error {err.max().item():.3g}, {worst:.2f} times the tolerance"


# ---- append and read -------------------------------------------------------------------------------------------------
STORES = [I8, E4M3, F16, BF16]


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("kv,hd,page", [(1, 16, 16), (3, 32, 16), (25, 64, 32), (8, 128, 64), (2, 128, 16)])
def test_append_and_read(store, dtype, kv, hd, page):
    counts, pos, slots = [5, 0, 1, 37, 130, 1], [3, 7, 15, 16, 0, 90], [4, 0, 5, 1, 2, 3]
    g = gen(kv * hd)
    c, ref = (Cache(store, kv, hd, page, 160, 6, seed=1) for _ in range(2))
    total, behind = sum(counts), 9
    # q, k and v are parts of one projection's rows: strides of the whole row
    proj = torch.randn(total + behind, 4 * kv, hd, generator=g, device=DEV) * torch.exp(torch.randn(4 * kv, 1, generator=g, device=DEV))
    proj = proj.to(dtype)
    k, v = proj[:, kv:2 * kv], proj[:, 3 * kv:]
    status = ints([0])
    mdi.kv_append(c.handle, k, v, starts(counts), ints(pos), slots=ints(slots), status=status)
    at = 0
    for n, p, s in zip(counts, pos, slots):
        if n:
            ref.put(s, p, k[at:at + n], v[at:at + n])
        at += n
    assert torch.equal(c.raw().view(torch.uint8), ref.raw().view(torch.uint8))      # every byte, the untouched ones too
    if c.scale is not None:
        assert torch.equal(c.scale.view(torch.int32), ref.scale.view(torch.int32))
    # back, as every type, into rows with other strides; rows behind the last sequence stay
    for out_t in (F32, F16, BF16):
        buf = torch.full((total + behind, 3 * kv, hd), 7.0, dtype=out_t, device=DEV)
        ko, vo = buf[:, :kv], buf[:, 2 * kv:]
        mdi.kv_read(c.handle, ko, vo, starts(counts), ints(pos), slots=ints(slots), status=status)
        assert (buf[total:] == 7).all() and (buf[:, kv:2 * kv] == 7).all()
        at = 0
        for n, p, s in zip(counts, pos, slots):
            for which, x in ((0, ko), (1, vo)):
                if n:
                    assert torch.equal(x[at:at + n], c.get(which, s, p, n).float().to(out_t))
            at += n
    assert status.item() == 0


@pytest.mark.parametrize("store", [I8, E4M3])
def test_append_borders_and_special_rows(store):
    hd = 64
    rows = [torch.zeros(hd), torch.full((hd,), 3.0e38), torch.full((hd,), 1e-44), torch.linspace(-2e-38, 2e-38, hd), torch.full((hd,), -0.0)]
    t = torch.zeros(hd); t[0] = 127; t[1:] = torch.arange(1, hd) + 0.5 - 32; rows.append(t)                  # scale 1: every element a tie
    t = torch.zeros(hd); t[0] = 127 * 3; t[1:] = (torch.arange(1, hd) + 0.5) * 3; rows.append(t)             # ties at scale 3
    t = torch.zeros(hd); t[0] = 448; t[1:] = torch.arange(1, hd) * 8 + 4.0; rows += [t, t / 1.0001, t * 1.01]  # borders of e4m3
    t = torch.zeros(hd); t[0] = 448; t[1:] = (torch.arange(1, hd) + 0.5) * 2.0 ** -9; rows.append(t)         # its smallest numbers
    rows += [torch.full((hd,), 448.0), torch.full((hd,), 449.0), torch.full((hd,), 448 * 2.0 ** -126), torch.full((hd,), 1.7e-38)]
    for bad in (math.inf, -math.inf, math.nan):
        t = torch.randn(hd, generator=torch.Generator().manual_seed(1)); t[17] = bad; rows.append(t)
    x = torch.stack(rows).to(DEV)
    big = torch.randn(4000, hd, generator=gen(5), device=DEV) * torch.exp(8 * torch.randn(4000, 1, generator=gen(6), device=DEV))
    x = torch.cat([x, big])[:, None].contiguous()
    n = x.shape[0]
    c, ref = (Cache(store, 1, hd, 16, n, 1) for _ in range(2))
    mdi.kv_append(c.handle, x, -x, starts([n]), ints([0]))
    ref.put(0, 0, x, -x)
    assert torch.equal(c.raw().view(torch.uint8) & 0x7f if store == E4M3 else c.raw(), ref.raw().view(torch.uint8) & 0x7f if store == E4M3 else ref.raw())
    assert torch.equal(torch.nan_to_num(c.scale, nan=-1.0), torch.nan_to_num(ref.scale, nan=-1.0))
    out = torch.empty_like(x)
    mdi.kv_read(c.handle, out, torch.empty_like(x), starts([n]))
    bad = ~torch.isfinite(x).all(-1)
    assert torch.isnan(out[bad]).all() and torch.isfinite(out[~bad]).all()
    # every finite element is within half a step of its row
    step = x[~bad].abs().amax(-1, keepdim=True).double() / 127 if store == I8 else None
    err = (out[~bad].double() - x[~bad].double()).abs()
    if store == I8:
        assert (err <= 0.5 * step.clamp_min(2.0 ** -126) * (1 + 2.0 ** -20)).all()
    else:
        big = x[~bad].abs().amax(-1, keepdim=True).double()
        assert (err <= torch.maximum(x[~bad].double().abs() / 16, big / 448 * 2 * 2.0 ** -10).clamp_min(2.0 ** -136)).all()


@pytest.mark.parametrize("store", STORES)
def test_bad_pages_positions_and_slots(store):
    kv, hd, page = 2, 32, 16
    c = Cache(store, kv, hd, page, 64, 4, seed=3)
    k = torch.randn(120, kv, hd, generator=gen(0), device=DEV)
    status = ints([0])
    mdi.kv_append(c.handle, k, k, starts([30, 30, 30, 30]), ints([0, 0, 0, 0]), status=status)
    before = c.raw().clone()
    assert status.item() == 0
    n_pages = c.pool.shape[0]
    for bad in (-1, n_pages, 2 ** 31 - 1, -2 ** 31):
        table = c.table.clone()
        table[1, 1] = bad
        h = mdi.KvCache(c.pool, table, scale=c.scale)
        status.zero_()
        out = torch.full_like(k, 5.0)
        mdi.kv_read(h, out, torch.empty_like(k), starts([30, 30, 30, 30]), status=status)
        assert status.item() == mdi.STATUS_PAGE
        assert (out[46:60] == 0).all()
        assert torch.equal(out[:46], torch.cat([c.get(0, 0, 0, 30), c.get(0, 1, 0, 16)]).float())
        status.zero_()
        mdi.kv_append(h, k, k, starts([30, 30, 30, 30]), ints([0, 0, 0, 0]), status=status)   # the same rows again
        assert status.item() == mdi.STATUS_PAGE and torch.equal(before.view(torch.uint8), c.raw().view(torch.uint8))
        q = torch.randn(4, 2 * kv, hd, generator=gen(1), device=DEV)
        o = torch.full_like(q, 9.0)
        status.zero_()
        ws = torch.empty(max(1, mdi.attn_decode_workspace(h, 2 * kv)), dtype=torch.uint8, device=DEV)
        mdi.attn_decode(h, q, o, ints([30, 30, 30, 30]), workspace=ws, status=status)
        assert status.item() == mdi.STATUS_PAGE
        kk, vv = c.get(0, 1, 0, 16), c.get(1, 1, 0, 16)       # the rows of the bad page are left out
        want, mag, ds = attend(q[1][:, None], kk, vv, hd ** -0.5, ints([16]))
        close(o[1][:, None], want, mag, ds, 16, 2.0 ** -15, F32)
    for pos in (-1, 64 - 29, 2 ** 31 - 1):
        status.zero_()
        mdi.kv_append(c.handle, k[:30], k[:30], starts([0, 30, 0, 0]), ints([0, pos, 0, 0]), status=status)
        assert status.item() == mdi.STATUS_RANGE
    for slot in (-1, 4, 2 ** 30):
        status.zero_()
        mdi.kv_append(c.handle, k[:3], k[:3], starts([3]), ints([0]), slots=ints([slot]), status=status)
        assert status.item() == mdi.STATUS_RANGE
    status.zero_()
    mdi.kv_append(c.handle, k[:10], k[:10], ints([0, 9, 4, 100000]), ints([0, 0, 0]), status=status)  # offsets that do not ascend
    assert status.item() in (0, mdi.STATUS_RANGE)


# ---- one new token ---------------------------------------------------------------------------------------------------
def decode_case(store, dtype, heads, kv, hd, page, lens, seed=0, max_len=0, slots=None, strided=False, k_gain=1.0, v_gain=None):
    g = gen(seed)
    n = len(lens)
    cap = max(max(lens), 1)
    c = Cache(store, kv, hd, page, cap, n, seed=seed)
    slots = slots or list(range(n))
    for i, ln in enumerate(lens):
        if ln:
            k, v = (torch.randn(ln, kv, hd, generator=g, device=DEV) for _ in range(2))
            c.put(slots[i], 0, k * k_gain, v if v_gain is None else v * v_gain(torch.arange(ln, device=DEV))[:, None, None])
    wide = torch.randn(n, heads + 3, hd, generator=g, device=DEV).to(dtype)
    q = wide[:, 1:1 + heads] if strided else wide[:, :heads].contiguous()
    buf = torch.full((n, heads + 5, hd), 7.0, dtype=dtype, device=DEV)
    out = buf[:, 2:2 + heads]
    ws = torch.full((max(1, mdi.attn_decode_workspace(c.handle, heads, max_len, n_seq=n)),), 255, dtype=torch.uint8, device=DEV)
    status = ints([0])
    mdi.attn_decode(c.handle, q, out, ints(lens), max_len, workspace=ws, slots=ints(slots), status=status)
    assert status.item() == 0
    assert (buf[:, :2] == 7).all() and (buf[:, 2 + heads:] == 7).all()
    return c, q, out, ws, slots


def check_decode(c, q, out, lens, slots, dtype):
    for i, ln in enumerate(lens):
        if ln == 0:
            assert (out[i] == 0).all()
            continue
        want, mag, ds = attend(q[i][:, None], c.get(0, slots[i], 0, ln), c.get(1, slots[i], 0, ln), c.hd ** -0.5, ints([ln]))
        close(out[i][:, None], want, mag, ds, ln, 2.0 ** -15 + (2.0 ** -11 if dtype != F32 and c.store != BF16 else 0.0), dtype)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("heads,kv,hd,page", [(1, 1, 16, 16), (6, 3, 32, 16), (12, 12, 64, 16), (25, 25, 64, 32), (32, 8, 128, 64), (40, 8, 128, 128), (16, 1, 128, 16), (33, 3, 64, 16)])
def test_decode(store, dtype, heads, kv, hd, page):
    lens = [1, 0, 15, 16, 17, 127, 128, 300, 1025]
    slots = [3, 1, 8, 0, 2, 7, 6, 5, 4]
    c, q, out, _, _ = decode_case(store, dtype, heads, kv, hd, page, lens, seed=heads + hd, slots=slots, strided=True)
    check_decode(c, q, out, lens, slots, dtype)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("heads,kv,hd", [(8, 8, 64), (8, 2, 128), (4, 1, 32), (64, 1, 128)])
def test_decode_long(store, heads, kv, hd):
    """Split over many blocks; max_len below, at and above the lengths changes the split, not the answer."""
    lens = [20001, 5, 4096]
    for max_len in (0, 1, 4096, 20001):
        c, q, out, _, s = decode_case(store, BF16, heads, kv, hd, 64, lens, seed=7, max_len=max_len)
        check_decode(c, q, out, lens, s, BF16)


@pytest.mark.parametrize("store", STORES)
def test_decode_values_of_very_different_size(store):
    """Scales that differ from row to row by many orders: the rows that matter come first, last, or in the middle."""
    for gain in (lambda j: 10.0 ** (-j / 40), lambda j: 10.0 ** (j / 40 - 5), lambda j: torch.where(j == 100, 1e4, 1e-4), lambda j: torch.where(j % 7 == 3, 300.0, 1e-3)):
        lens = [200, 97]
        c, q, out, _, s = decode_case(store, F32, 4, 2, 64, 16, lens, seed=11, v_gain=gain)
        check_decode(c, q, out, lens, s, F32)
    for k_gain in (1e-3, 30.0):
        lens = [333]
        c, q, out, _, s = decode_case(store, F32, 4, 2, 64, 16, lens, seed=12, k_gain=k_gain)
        check_decode(c, q, out, lens, s, F32)


def test_decode_large_and_small_queries():
    for gain in (1e-30, 1e-6, 1e5, 1e30):
        c, q, out, ws, s = decode_case(I8, F32, 4, 2, 64, 16, [100], seed=13)
        q = q * gain
        o = torch.empty_like(q)
        mdi.attn_decode(c.handle, q, o, ints([100]), scale=0.125 / gain, workspace=ws)
        want, mag, ds = attend(q[0][:, None], c.get(0, 0, 0, 100), c.get(1, 0, 0, 100), 0.125 / gain, ints([100]))
        close(o[0][:, None], want, mag, ds, 100, 2.0 ** -15, F32)


@pytest.mark.parametrize("store", STORES)
def test_decode_non_finite_rows(store):
    """A non-finite row within the length gives NaN to its sequence and head alone; behind the length nothing matters
    (the whole pool starts as NaN there already)."""
    kv, hd = 2, 64
    c, q, out, ws, _ = decode_case(store, F32, 4, kv, hd, 16, [40, 40], seed=3)
    page, off = c.table[1, 20 // 16].item(), 20 % 16
    if c.scale is not None:
        c.scale[page, 1, 0, off] = math.nan
    else:
        c.pool[page, 1, 0, off, 5] = math.nan
    o2 = torch.empty_like(q)
    mdi.attn_decode(c.handle, q, o2, ints([40, 40]), workspace=ws)
    assert torch.equal(o2[0], out[0]) and torch.equal(o2[1, 2:], out[1, 2:])
    assert torch.isnan(o2[1, :2]).all() if c.scale is not None else torch.isnan(o2[1, :2, 5]).all()
    mdi.attn_decode(c.handle, q, o2, ints([40, 20]), workspace=ws)   # ... and is not seen by a shorter length
    assert torch.isfinite(o2).all()


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("group", [1, 3, 4, 9])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_decode_queries_that_are_not_finite(store, group, bad):
    """NaN for that head of that sequence, all others as before."""
    lens = [300, 20]
    c, q, out, ws, s = decode_case(store, F32, 2 * group, 2, 64, 16, lens, seed=26)
    check_decode(c, q, out, lens, s, F32)
    q2, o = q.clone(), torch.empty_like(q)
    q2[0, group, 7] = bad
    mdi.attn_decode(c.handle, q2, o, ints(lens), workspace=ws)
    assert torch.isnan(o[0, group]).all()
    o[0, group] = out[0, group]
    assert torch.equal(o, out.contiguous())


@pytest.mark.parametrize("store", [F16, BF16])
def test_decode_scores_of_minus_infinity(store):
    """Keys that give a score of -inf weigh nothing, whether they come first or last."""
    c, q, out, ws, _ = decode_case(store, F32, 1, 1, 64, 16, [50], seed=4)
    q[0, 0, 0] = 1.0
    hide = list(range(0, 20)) + [30, 49]
    for t in hide:
        c.pool[c.table[0, t // 16].item(), 0, 0, t % 16, 0] = -math.inf
    mdi.attn_decode(c.handle, q, out, ints([50]), workspace=ws)
    keep = [t for t in range(50) if t not in hide]
    want, mag, ds = attend(q[0][:, None], c.get(0, 0, 0, 50)[keep], c.get(1, 0, 0, 50)[keep], 0.125, ints([len(keep)]))
    close(out[0][:, None], want, mag, ds, 50, 2.0 ** -15, F32)


def test_decode_lengths_out_of_range():
    c, q, out, ws, _ = decode_case(I8, F32, 4, 2, 64, 16, [48, 48, 48], seed=5)
    status = ints([0])
    o = torch.full_like(q, 3.0)
    mdi.attn_decode(c.handle, q, o, ints([2 ** 31 - 1, -5, 48]), workspace=ws, status=status)
    assert status.item() == mdi.STATUS_RANGE
    check_decode(c, q, o, [48, 0, 48], [0, 1, 2], F32)         # (how the work is shared out, and with it the bits, may change)
    status.zero_()
    mdi.attn_decode(c.handle, q, o, ints([48, 48, 48]), workspace=ws, slots=ints([0, 77, -1]), status=status)
    assert status.item() == mdi.STATUS_RANGE
    check_decode(c, q, o, [48, 0, 0], [0, 1, 2], F32)


@pytest.mark.parametrize("store", [I8, BF16])
@pytest.mark.parametrize("slots", [None, "other", "same"])
def test_decode_of_more_sequences_than_a_launch_takes(store, slots):
    n, heads, kv, hd, page = 600, 4, 2, 32, 16
    c = Cache(store, kv, hd, page, 96, n, seed=21)
    lens = [(37 * i) % 90 if i % 5 else 0 for i in range(n)]
    lens[255], lens[256], lens[511], lens[512], lens[599] = 90, 1, 0, 77, 33
    at = {None: list(range(n)), "other": [(7 * i + 3) % n for i in range(n)], "same": [5] * n}[slots]
    for slot in sorted(set(at)):
        k, v = (torch.randn(90, kv, hd, generator=gen(slot + j), device=DEV) for j in (0, 1000))
        c.put(slot, 0, k, v)
    q = torch.randn(n, heads, hd, generator=gen(1), device=DEV).to(BF16)
    ws = torch.empty(max(1, mdi.attn_decode_workspace(c.handle, heads, 90, n_seq=n)), dtype=torch.uint8, device=DEV)
    out, status = torch.full_like(q, 9.0), ints([0])
    mdi.attn_decode(c.handle, q, out, ints(lens), 90, workspace=ws, slots=None if slots is None else ints(at), status=status)
    assert status.item() == 0
    check_decode(c, q, out, lens, at, BF16)


@pytest.mark.parametrize("store", STORES)
def test_decode_of_nothing(store):
    """Zeros where no row is left: all pages missing, or all scores -inf; other sequences as before."""
    lens = [40, 700, 33, 0]
    c, q, out, ws, _ = decode_case(store, F32, 4, 2, 64, 16, lens, seed=22)
    table, status = c.table.clone(), ints([0])
    table[:2] = -1
    h = mdi.KvCache(c.pool, table, scale=c.scale)
    o = torch.full_like(q, 3.0)
    mdi.attn_decode(h, q, o, ints(lens), workspace=ws, status=status)
    assert status.item() == mdi.STATUS_PAGE
    assert (o[0] == 0).all() and (o[1] == 0).all() and (o[3] == 0).all()
    assert torch.equal(o[2], out[2])
    if c.scale is None:
        q[:, :, 0] = 1.0
        for i in (0, 1):
            for t in range(lens[i]):
                c.pool[c.table[i, t // 16].item(), 0, 0, t % 16, 0] = -math.inf   # the first key head of both
        mdi.attn_decode(c.handle, q, o, ints(lens), workspace=ws)
        assert (o[:2, :2] == 0).all()
        for i in (0, 1):
            want, mag, ds = attend(q[i][2:, None], c.get(0, i, 0, lens[i])[:, 1:], c.get(1, i, 0, lens[i])[:, 1:], 0.125, ints([lens[i]]))
            close(o[i][2:, None], want, mag, ds, lens[i], 2.0 ** -15, F32)


@pytest.mark.parametrize("store,gain", [(I8, 1e-22), (I8, 1e30), (I8, 1e36), (E4M3, 1e-22), (E4M3, 1e30), (E4M3, 1e36), (BF16, 1e-22), (BF16, 1e30)])
def test_decode_very_large_and_small_values(store, gain):
    lens = [300, 20]
    c, q, out, _, s = decode_case(store, F32, 4, 2, 64, 16, lens, seed=23, v_gain=lambda j: torch.where(j % 3 == 0, gain, gain / 100))
    check_decode(c, q, out, lens, s, F32)


def test_views_of_a_wider_page_table_and_repeated_inputs():
    kv, hd, page = 2, 64, 16
    c = Cache(F16, kv, hd, page, 100, 3, seed=24)
    wide = torch.full((3, 50), -7, dtype=torch.int32, device=DEV)
    wide[:, 11:11 + c.per] = c.table
    h = mdi.KvCache(c.pool, wide[:, 11:11 + c.per])
    k = torch.randn(1, kv, hd, generator=gen(1), device=DEV).expand(100, kv, hd)   # one row, a hundred times
    v = torch.randn(100, 1, hd, generator=gen(2), device=DEV).expand(100, kv, hd)  # one head, twice
    status = ints([0])
    mdi.kv_append(h, k, v, starts([60, 0, 35]), ints([0, 0, 3]), status=status)    # the last five rows belong to no sequence
    assert status.item() == 0
    assert torch.equal(c.get(0, 0, 0, 60).float(), k[:60].half().float()) and torch.equal(c.get(1, 2, 3, 35).float(), v[60:95].half().float())
    q = torch.randn(1, 1, hd, generator=gen(3), device=DEV).expand(3, 4, hd)
    out = torch.empty(3, 4, hd, device=DEV)
    ws = torch.empty(max(1, mdi.attn_decode_workspace(h, 4)), dtype=torch.uint8, device=DEV)
    mdi.attn_decode(h, q, out, ints([60, 0, 0]), workspace=ws, status=status)
    assert status.item() == 0
    check_decode(c, q, out, [60, 0, 0], [0, 1, 2], F32)
    one = torch.empty(1, kv, hd, device=DEV).expand(100, kv, hd)                   # an output whose rows are one another
    for f in (lambda: mdi.kv_read(h, one, torch.empty(100, kv, hd, device=DEV), starts([60, 0, 35])),
              lambda: mdi.attn_decode(h, q, torch.empty(3, 1, hd, device=DEV).expand(3, 4, hd), ints([1, 1, 1]), workspace=ws)):
        with pytest.raises(mdi.MdiError) as e:
            f()
        assert e.value.code == mdi.ERR_SHAPE


def test_calls_without_work():
    c, q, out, ws, _ = decode_case(I8, F32, 4, 2, 64, 16, [48], seed=25)
    before = c.raw().clone()
    k, none, status = torch.zeros(5, 2, 64, device=DEV), ints([]), ints([0])
    mdi.kv_append(c.handle, k, k, ints([0]), none, status=status)                  # no sequence
    mdi.kv_append(c.handle, k[:0], k[:0], ints([0, 0]), ints([0]), status=status)  # no rows
    o = torch.full_like(k, 4.0)
    mdi.kv_read(c.handle, o, o.clone(), ints([0]), status=status)
    mdi.kv_read(c.handle, o[:0], o[:0], ints([0, 0]), status=status)
    assert (o == 4).all() and torch.equal(before, c.raw())
    mdi.attn_decode(c.handle, q[:0], out[:0], none, status=status)
    p = torch.full((5, 2, 64), 4.0, dtype=BF16, device=DEV)
    mdi.attn_prompt(p, p, p, p, ints([0]), ints([0]), status=status)
    mdi.attn_prompt(p[:0], p, p, p[:0], ints([0, 0]), ints([0, 5]), status=status)
    assert (p == 4).all()
    mdi.attn_prompt(p.clone(), p[:0], p[:0], p, ints([0, 5]), ints([0, 0]), status=status)   # queries without keys
    assert (p == 0).all() and status.item() == 0


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("heads,kv,hd,n,longest", [(12, 12, 64, 1, 40), (12, 12, 64, 1, 1000), (16, 2, 128, 1, 4096), (16, 2, 128, 1, 4097), (32, 8, 128, 8, 1000),
                                                   (5, 5, 16, 30, 512), (64, 1, 32, 3, 250), (30, 10, 128, 14, 512), (148, 148, 32, 1, 300), (148, 148, 32, 2, 300)])
def test_decode_of_few_short_sequences(store, heads, kv, hd, n, longest):
    """Pairs with one to eight blocks to themselves, around the sizes where that ends; a length above max_len too."""
    lens = [longest] + [(i * 97) % (longest + 1) for i in range(1, n)]
    for max_len in (longest, max(1, longest // 7)):
        c, q, out, ws, s = decode_case(store, F32 if hd == 128 else F16, heads, kv, hd, 16, lens, seed=n, max_len=max_len)
        check_decode(c, q, out, lens, s, q.dtype)
        again = torch.empty_like(q)
        mdi.attn_decode(c.handle, q, again, ints(lens), max_len, workspace=ws)
        assert torch.equal(again, out.contiguous())


def test_decode_is_reproducible_on_streams_and_in_graphs():
    lens = [3000, 700, 0, 64]
    c, q, out, ws, s = decode_case(E4M3, BF16, 32, 8, 128, 64, lens, seed=6)
    first = out.clone()
    for _ in range(5):
        mdi.attn_decode(c.handle, q, out, ints(lens), workspace=ws)
        assert torch.equal(out, first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ln = ints(lens)
    outs = [torch.zeros_like(q) for _ in range(2)]
    graphs = []
    for o in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            mdi.attn_decode(c.handle, q, o, ln, workspace=ws, stream=torch.cuda.current_stream().cuda_stream)
        graphs.append(g)
    for short in (lens, [2999, 1, 0, 63]):                       # the graphs read the lengths when they are replayed
        ln.copy_(ints(short))
        for g in graphs:                                          # one workspace, one stream: one after the other
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1])
        check_decode(c, q, outs[0], short, s, BF16)
    with torch.cuda.stream(side):
        mdi.attn_decode(c.handle, q, outs[0], ints(lens), workspace=ws, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(outs[0].contiguous(), first.contiguous())


def test_decode_needs_its_workspace():
    c, q, out, ws, _ = decode_case(I8, F32, 4, 2, 64, 16, [5000], seed=5)
    need = mdi.attn_decode_workspace(c.handle, 4, 0, n_seq=1)
    if need:
        for w in (None, torch.empty(need - 1, dtype=torch.uint8, device=DEV)):
            with pytest.raises(mdi.MdiError) as e:
                mdi.attn_decode(c.handle, q, out, ints([5000]), workspace=w)
            assert e.value.code == mdi.ERR_ARG
    with pytest.raises(mdi.MdiError) as e:
        mdi.attn_decode(c.handle, q.cpu(), out, ints([5000]), workspace=ws)
    assert e.value.code == mdi.ERR_ARG


def test_pool_offsets_past_32_bits():
    """Pages whose byte and element offsets pass 2^32."""
    kv, hd, page = 8, 128, 128
    n = (2 ** 32) // (2 * kv * page * hd) + 40
    pool = torch.empty(n, 2, kv, page, hd, dtype=I8, device=DEV)
    scale = torch.empty(n, 2, kv, page, device=DEV)
    table = ints([n - 1, 3, n - 2]).view(1, 3)
    h = mdi.KvCache(pool, table, scale=scale)
    k, v = (torch.randn(300, kv, hd, generator=gen(s), device=DEV) for s in (1, 2))
    mdi.kv_append(h, k, v, starts([300]), ints([0]))
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    mdi.kv_read(h, ko, vo, starts([300]))
    for x, o in ((k, ko), (v, vo)):
        q, s = quantise(x, I8)
        assert torch.equal(o, (q.double() * s.double()[..., None]).float())
    q = torch.randn(1, 16, hd, generator=gen(3), device=DEV)
    out = torch.empty_like(q)
    ws = torch.empty(max(1, mdi.attn_decode_workspace(h, 16)), dtype=torch.uint8, device=DEV)
    mdi.attn_decode(h, q, out, ints([300]), workspace=ws)
    want, mag, ds = attend(q[0][:, None], ko, vo, hd ** -0.5, ints([300]))
    close(out[0][:, None], want, mag, ds, 300, 2.0 ** -15, F32)


# ---- whole prompts ---------------------------------------------------------------------------------------------------
def prompt_case(dtype, heads, kv, hd, nq, nk, seed=0, behind=0):
    g = gen(seed)
    tq, tk = sum(nq), sum(nk)
    q = torch.randn(tq + behind, heads, hd, generator=g, device=DEV).to(dtype)
    kvrows = torch.randn(tk + behind, 2 * kv + 1, hd, generator=g, device=DEV).to(dtype)
    return q, kvrows[:, 1:1 + kv], kvrows[:, 1 + kv:]


def check_prompt(q, k, v, out, nq, nk, dtype, scale=None):
    hd = q.shape[2]
    a = b = 0
    for x, y in zip(nq, nk):
        if x:
            seen = (torch.arange(x, device=DEV) + 1 + y - x).clamp_min(0)
            want, mag, ds = attend(q[a:a + x].transpose(0, 1), k[b:b + y], v[b:b + y], scale or hd ** -0.5, seen)
            got = out[a:a + x].transpose(0, 1)
            close(got, want, mag, ds, y, torch.finfo(dtype).eps / 2 + 2.0 ** -15, dtype)
            assert (got[:, seen == 0] == 0).all()
        a += x
        b += y


PROMPTS = [([1], [1]), ([1, 5, 0, 17, 128], [1, 5, 0, 17, 128]), ([127, 129, 255, 257], [127, 129, 255, 257]), ([300], [811]),
           ([64, 1, 200, 0, 3], [100, 77, 456, 9, 3]), ([130, 20], [100, 0]), ([700, 33], [700, 33])]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads,kv,hd", [(1, 1, 16), (6, 3, 32), (5, 5, 64), (8, 2, 128), (7, 1, 64), (4, 4, 128)])
@pytest.mark.parametrize("nq,nk", PROMPTS)
def test_prompt(dtype, heads, kv, hd, nq, nk):
    q, k, v = prompt_case(dtype, heads, kv, hd, nq, nk, seed=heads)
    out = torch.full_like(q, 5.0)
    status = ints([0])
    mdi.attn_prompt(q, k, v, out, starts(nq), starts(nk), status=status)
    assert status.item() == 0
    check_prompt(q, k, v, out, nq, nk, dtype)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_long(dtype, hd):
    nq, nk = [2049], [4100]
    q, k, v = prompt_case(dtype, 4, 2, hd, nq, nk, seed=1)
    out = torch.empty_like(q)
    mdi.attn_prompt(q, k, v, out, starts(nq), starts(nk))
    check_prompt(q, k, v, out, nq, nk, dtype)
    again = torch.empty_like(q)
    mdi.attn_prompt(q, k, v, again, starts(nq), starts(nk))
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_prompt_scores_that_grow(dtype):
    """The running maximum rises from tile to tile (and once falls by a lot): rescaling of what has been summed so far."""
    for gain in (lambda j: j / 100, lambda j: 6 - j / 100, lambda j: torch.where(j == 37, 40.0, 1.0), lambda j: torch.where(j == 600, 40.0, 1.0)):
        nq, nk = [900], [900]
        q, k, v = prompt_case(dtype, 2, 1, 64, nq, nk, seed=2)
        q = q.abs()
        k = (k.float() * gain(torch.arange(900, device=DEV).float())[:, None, None]).to(dtype)
        out = torch.empty_like(q)
        mdi.attn_prompt(q, k, v, out, starts(nq), starts(nk))
        check_prompt(q, k, v, out, nq, nk, dtype)


@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_non_finite_where_masked(hd):
    """Rows of another sequence, rows behind the last one, and keys and values a row may not see yet: infinities and NaN in
    them do not reach a row; what a row does see reaches it."""
    nq = nk = [200, 100]
    q, k, v = prompt_case(BF16, 4, 2, hd, nq, nk, seed=3, behind=60)
    out = torch.full_like(q, 5.0)
    mdi.attn_prompt(q, k, v, out, starts(nq), starts(nk))
    clean = out.clone()
    assert (out[300:] == 5).all()
    for bad in (math.nan, math.inf):
        for t in (150, 199, 40):
            k2, v2 = k.clone(), v.clone()
            v2[t, 0, 3] = bad
            v2[t, 1, 7] = -bad
            k2[t:200] = bad
            k2[300:], v2[300:] = bad, bad
            o = torch.full_like(q, 5.0)
            mdi.attn_prompt(q, k2, v2, o, starts(nq), starts(nk))
            assert torch.equal(o[:t], clean[:t]) and torch.equal(o[200:], clean[200:])
            assert torch.isnan(o[t:200]).all()
            o = torch.full_like(q, 5.0)
            mdi.attn_prompt(q, k, v2, o, starts(nq), starts(nk))          # the values alone: only their columns
            assert torch.equal(o[:t], clean[:t]) and torch.equal(o[200:], clean[200:])
            for heads, e, sign in ((slice(0, 2), 3, 1), (slice(2, 4), 7, -1)):
                got = o[t:200, heads, e]
                assert (torch.isnan(got).all() if math.isnan(bad) else (got == sign * bad).all())
                rest = [x for x in range(hd) if x != e]
                assert torch.equal(o[t:200, heads][..., rest], clean[t:200, heads][..., rest])


def test_prompt_bad_offsets():
    nq = nk = [50, 30]
    q, k, v = prompt_case(BF16, 2, 1, 64, nq, nk, seed=4)
    good = torch.empty_like(q)
    mdi.attn_prompt(q, k, v, good, starts(nq), starts(nk))
    for qs, ks in (([0, 50, 80], [0, 50, 81]), ([0, 50, 80], [0, 50, 2 ** 30]), ([0, 50, 80], [0, 50, 40]), ([0, 50, 81], [0, 50, 80]), ([0, 50, 2 ** 30], [0, 50, 80])):
        status = ints([0])
        out = torch.full_like(q, 3.0)
        mdi.attn_prompt(q, k, v, out, ints(qs), ints(ks), status=status)
        assert status.item() == mdi.STATUS_RANGE
        assert torch.equal(out[:50], good[:50])
        assert (out[50:] == 3).all()


@pytest.mark.parametrize("n", [64, 65, 150])
def test_prompt_of_many_sequences(n):
    """Around the number up to which tiles are ordered over all sequences; some empty, one whose offsets do not fit."""
    nq = [(61 * i) % 300 if i % 4 else 0 for i in range(n)]
    nk = [x + (i * 13) % 200 for i, x in enumerate(nq)]
    nq[n - 1], nk[n - 1] = 290, 1000
    nk[1] = 20                                                # fewer keys than queries
    q, k, v = prompt_case(BF16, 2, 1, 64, nq, nk, seed=n)
    out, status = torch.full_like(q, 3.0), ints([0])
    mdi.attn_prompt(q, k, v, out, starts(nq), starts(nk), status=status)
    assert status.item() == 0
    check_prompt(q, k, v, out, nq, nk, BF16)
    ks, bad = starts(nk), torch.full_like(q, 3.0)
    ks[n] = sum(nk) + 1                                       # the last one's keys end behind the rows
    mdi.attn_prompt(q, k, v, bad, starts(nq), ks, status=status)
    assert status.item() == mdi.STATUS_RANGE
    assert torch.equal(bad[:-290], out[:-290]) and (bad[-290:] == 3).all()


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_prompt_scores_of_minus_infinity(dtype):
    """Keys that give -inf weigh nothing; a row that sees no others gives zeros."""
    n = 200
    q, k, v = prompt_case(dtype, 2, 1, 64, [n], [n], seed=6)
    k, v = k.contiguous(), v.contiguous()
    q[:, :, 0] = 1.0
    k[:40, :, 0] = -math.inf
    out = torch.empty_like(q)
    mdi.attn_prompt(q, k, v, out, starts([n]), starts([n]))
    assert (out[:40] == 0).all()
    seen = torch.arange(1, n - 40 + 1, device=DEV)
    want, mag, ds = attend(q[40:].transpose(0, 1), k[40:], v[40:], 0.125, seen)
    close(out[40:].transpose(0, 1), want, mag, ds, n, torch.finfo(dtype).eps / 2 + 2.0 ** -15, dtype)


def test_prompts_on_two_streams():
    nq = [700, 33, 260]
    q, k, v = prompt_case(BF16, 8, 2, 128, nq, nq, seed=8)
    good = torch.empty_like(q)
    mdi.attn_prompt(q, k, v, good, starts(nq), starts(nq))
    qs = starts(nq)
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(q) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, o in zip(streams, outs):
            mdi.attn_prompt(q, k, v, o, qs, qs, stream=st.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(o, good) for o in outs)


def test_prompt_rows_past_32_bits():
    hd, heads = 64, 4
    rows, stride = 1100, 2 ** 21                             # the last rows start beyond 2^31 elements
    buf = torch.empty(rows * stride, dtype=BF16, device=DEV)
    view = buf.as_strided((rows, 3 * heads, hd), (stride, hd, 1))
    q0, k0, v0 = (torch.randn(rows, heads, hd, generator=gen(s), device=DEV).to(BF16) for s in (1, 2, 3))
    q, k, v = view[:, :heads], view[:, heads:2 * heads], view[:, 2 * heads:]
    q.copy_(q0), k.copy_(k0), v.copy_(v0)
    a, b = torch.empty_like(q0), torch.empty_like(q0)
    mdi.attn_prompt(q, k, v, a, starts([rows]), starts([rows]))
    mdi.attn_prompt(q0, k0, v0, b, starts([rows]), starts([rows]))
    assert torch.equal(a, b)
    mdi.attn_prompt(q0, k0, v0, q, starts([rows]), starts([rows]))
    assert torch.equal(q, b)


def test_prompt_head_major_rows_and_broadcast():
    """[head][row][element] tensors; a stride of zero is refused."""
    n, heads, kv, hd = 333, 4, 2, 64
    q, k, v = (torch.randn(h, n, hd, generator=gen(h), device=DEV).to(BF16).transpose(0, 1) for h in (heads, kv, kv))
    buf = torch.zeros(heads, n, hd, dtype=BF16, device=DEV)
    mdi.attn_prompt(q, k, v, buf.transpose(0, 1), starts([n]), starts([n]))
    out = torch.empty(n, heads, hd, dtype=BF16, device=DEV)
    mdi.attn_prompt(q.contiguous(), k.contiguous(), v.contiguous(), out, starts([n]), starts([n]))
    assert torch.equal(buf.transpose(0, 1), out)
    check_prompt(q, k, v, out, [n], [n], BF16)
    for x in (k[:, :1].expand(n, kv, hd), k[:1].expand(n, kv, hd)):
        with pytest.raises(mdi.MdiError) as e:
            mdi.attn_prompt(q, x, v, out, starts([n]), starts([n]))
        assert e.value.code == mdi.ERR_SHAPE


def test_prompt_in_a_graph_with_other_lengths():
    nq, nk = [300, 212], [300, 212]
    q, k, v = prompt_case(BF16, 4, 2, 128, nq, nk, seed=5)
    out = torch.zeros_like(q)
    qs, ks = starts(nq), starts(nk)
    mdi.attn_prompt(q, k, v, out, qs, ks)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mdi.attn_prompt(q, k, v, out, qs, ks, stream=torch.cuda.current_stream().cuda_stream)
    for other in ([300, 212], [512, 0], [1, 511], [100, 100]):
        qs.copy_(starts(other)), ks.copy_(starts(other))
        out.fill_(2.0)
        g.replay()
        torch.cuda.synchronize()
        check_prompt(q, k, v, out, other, other, BF16)
        assert (out[sum(other):] == 2).all()


# ---- together, as a serving loop uses them ---------------------------------------------------------------------------
@pytest.mark.parametrize("store", STORES)
def test_a_prompt_in_chunks_then_tokens(store):
    """Two sequences: first visits in two chunks (append, read back, attention of the chunk over everything so far), then one
    token at a time; against attention in 64 bits over the stored rows."""
    heads, kv, hd, page = 8, 2, 64, 16
    g = gen(9)
    c = Cache(store, kv, hd, page, 400, 2, seed=2)
    done = [0, 0]
    ws = torch.empty(max(1, mdi.attn_decode_workspace(c.handle, heads)), dtype=torch.uint8, device=DEV)
    for chunk in ([130, 60], [70, 33]):
        n = sum(chunk)
        q, k, v = (torch.randn(n, h, hd, generator=g, device=DEV).to(F16) for h in (heads, kv, kv))
        mdi.kv_append(c.handle, k, v, starts(chunk), ints(done))
        done = [a + b for a, b in zip(done, chunk)]
        kd, vd = (torch.empty(sum(done), kv, hd, dtype=F16, device=DEV) for _ in range(2))
        mdi.kv_read(c.handle, kd, vd, starts(done))
        out = torch.empty_like(q)
        mdi.attn_prompt(q, kd, vd, out, starts(chunk), starts(done))
        check_prompt(q, kd, vd, out, chunk, done, F16)
        for i in range(2):
            assert torch.equal(kd[sum(done[:i]):sum(done[:i + 1])], c.get(0, i, 0, done[i]).float().to(F16))
    for step in range(20):
        q, k, v = (torch.randn(2, h, hd, generator=g, device=DEV) for h in (heads, kv, kv))
        mdi.kv_append(c.handle, k, v, ints([0, 1, 2]), ints(done))
        done = [d + 1 for d in done]
        out = torch.empty_like(q)
        mdi.attn_decode(c.handle, q, out, ints(done), workspace=ws)
        check_decode(c, q, out, done, [0, 1], F32)
