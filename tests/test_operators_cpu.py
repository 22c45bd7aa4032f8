"""Refusals of the attention operators that need no GPU: what the host can see to be wrong is an error code before anything is
enqueued, and host memory never reaches a kernel."""
import pytest
import torch

from paper_2505_18164_b200 import mdi

I8, E4M3, F16, BF16 = torch.int8, torch.float8_e4m3fn, torch.float16, torch.bfloat16


def make(store=I8, pages=6, kv=2, page=16, hd=64, slots=2, per=3):
    pool = torch.zeros(pages, 2, kv, page, hd, dtype=store)
    scale = torch.ones(pages, 2, kv, page) if store in (I8, E4M3) else None
    return mdi.KvCache(pool, torch.zeros(slots, per, dtype=torch.int32), scale=scale)


def ints(*v):
    return torch.tensor(v, dtype=torch.int32)


def code(f, *a, **k):
    with pytest.raises(mdi.MdiError) as e:
        f(*a, **k)
    assert str(e.value)
    return e.value.code


def rows(n, heads, hd, dtype=BF16):
    return torch.zeros(n, heads, hd, dtype=dtype)


def test_cache_descriptions():
    make()
    assert code(mdi.KvCache, torch.zeros(4, 2, 2, 16, 64), torch.zeros(1, 4, dtype=torch.int32)) == mdi.ERR_ARG      # fp32 pool
    assert code(mdi.KvCache, torch.zeros(4, 3, 2, 16, 64, dtype=F16), torch.zeros(1, 4, dtype=torch.int32)) == mdi.ERR_ARG
    assert code(mdi.KvCache, torch.zeros(4, 2, 2, 16, 64, dtype=I8), torch.zeros(1, 4, dtype=torch.int32)) == mdi.ERR_ARG  # no scales
    assert code(mdi.KvCache, torch.zeros(4, 2, 2, 16, 64, dtype=F16), torch.zeros(1, 4)) == mdi.ERR_ARG
    for kw in (dict(hd=48), dict(page=8), dict(page=24), dict(kv=1025, hd=16)):
        c = make(**kw)
        hd, kv = c.head_dim, c.n_kv_head
        assert code(mdi.kv_append, c, rows(2, kv, hd), rows(2, kv, hd), ints(0, 2), ints(0)) == mdi.ERR_SHAPE
        assert code(mdi.attn_decode, c, rows(1, kv, hd), rows(1, kv, hd), ints(1)) == mdi.ERR_SHAPE


@pytest.mark.parametrize("f", [mdi.kv_append, mdi.kv_read])
def test_rows_of_the_cache(f):
    c = make()
    ok = rows(4, 2, 64)
    assert code(f, c, ok, rows(4, 2, 64, torch.float64), ints(0, 4), ints(0)) == mdi.ERR_ARG
    assert code(f, c, ok, rows(4, 2, 64, F16), ints(0, 4), ints(0)) == mdi.ERR_ARG              # k and v differ
    assert code(f, c, ok, rows(3, 2, 64), ints(0, 4), ints(0)) == mdi.ERR_ARG                   # fewer rows
    assert code(f, c, rows(4, 3, 64), rows(4, 3, 64), ints(0, 4), ints(0)) == mdi.ERR_ARG
    assert code(f, c, ok, ok, torch.zeros(2, dtype=torch.int64), ints(0)) == mdi.ERR_ARG
    assert code(f, c, ok, ok, ints(0, 4, 4, 4), ints(0, 0, 0)) == mdi.ERR_ARG                   # three sequences, two slots
    odd = torch.zeros(4, 2, 65, dtype=BF16)[:, :, :64]                                          # strides of 65 elements
    assert code(f, c, odd, ok, ints(0, 4), ints(0)) == mdi.ERR_SHAPE
    shifted = torch.zeros(4 * 2 * 64 + 1, dtype=BF16)[1:].view(4, 2, 64)                        # 2 bytes off
    assert code(f, c, shifted, ok, ints(0, 4), ints(0)) == mdi.ERR_SHAPE
    last = torch.zeros(4, 2, 128, dtype=BF16)[:, :, ::2]
    assert code(f, c, last, ok, ints(0, 4), ints(0)) == mdi.ERR_ARG
    assert code(f, c, ok, ok, ints(0, 4), ints(0)) in (mdi.ERR_ARG, mdi.ERR_CUDA)               # host memory / no device


def test_decode():
    c = make()
    q = rows(2, 8, 64)
    assert code(mdi.attn_decode, c, rows(2, 7, 64), rows(2, 7, 64), ints(1, 1)) == mdi.ERR_SHAPE
    assert code(mdi.attn_decode, c, rows(2, 256, 64), rows(2, 256, 64), ints(1, 1)) == mdi.ERR_SHAPE   # 128 heads share a key head
    assert code(mdi.attn_decode, c, q, rows(2, 8, 64, F16), ints(1, 1)) == mdi.ERR_ARG
    assert code(mdi.attn_decode, c, q, q, ints(1)) == mdi.ERR_ARG
    assert code(mdi.attn_decode, c, rows(3, 8, 64), rows(3, 8, 64), ints(1, 1, 1)) == mdi.ERR_ARG
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert code(mdi.attn_decode, c, q, q, ints(1, 1), scale=s) == mdi.ERR_ARG
    assert code(mdi.attn_decode, c, q, q, ints(1, 1), max_len=-1) == mdi.ERR_ARG
    assert code(mdi.attn_decode, c, q, q, ints(1, 1), workspace=torch.zeros(1 << 22, dtype=torch.uint8)) in (mdi.ERR_ARG, mdi.ERR_CUDA)
    assert code(mdi.attn_decode_workspace, c, 7) == mdi.ERR_SHAPE
    assert mdi.attn_decode_workspace(c, 8) >= 0


def test_prompt():
    q, k = rows(5, 4, 64), rows(7, 2, 64)
    one = ints(0, 5), ints(0, 7)
    assert code(mdi.attn_prompt, rows(5, 4, 48), rows(7, 2, 48), rows(7, 2, 48), rows(5, 4, 48), *one) == mdi.ERR_SHAPE
    assert code(mdi.attn_prompt, rows(5, 3, 64), k, k, rows(5, 3, 64), *one) == mdi.ERR_SHAPE
    assert code(mdi.attn_prompt, q.float(), k.float(), k.float(), q.float(), *one) == mdi.ERR_ARG
    assert code(mdi.attn_prompt, q, k.half(), k, q, *one) == mdi.ERR_ARG
    assert code(mdi.attn_prompt, q, k, k, rows(4, 4, 64), *one) == mdi.ERR_ARG
    assert code(mdi.attn_prompt, q, k, k, q, ints(0, 5), ints(0)) == mdi.ERR_ARG
    for s in (0.0, -0.5, float("nan"), float("inf")):
        assert code(mdi.attn_prompt, q, k, k, q, *one, scale=s) == mdi.ERR_ARG
    assert code(mdi.attn_prompt, q, k[:, :1].expand(7, 2, 64), k, q, *one) in (mdi.ERR_SHAPE, mdi.ERR_ARG, mdi.ERR_CUDA)
    odd = torch.zeros(7, 2, 68, dtype=BF16)[:, :, :64]
    assert code(mdi.attn_prompt, q, odd, k, q, *one) == mdi.ERR_SHAPE
    assert code(mdi.attn_prompt, q, k, k, q, *one) in (mdi.ERR_ARG, mdi.ERR_CUDA)


def test_outputs_that_overlap_themselves():
    c, q = make(), rows(2, 8, 64)
    assert code(mdi.attn_decode, c, q, q[:1].expand(2, 8, 64), ints(1, 1)) == mdi.ERR_SHAPE
    assert code(mdi.kv_read, c, rows(4, 1, 64).expand(4, 2, 64), rows(4, 2, 64), ints(0, 4), ints(0)) == mdi.ERR_SHAPE
    k, one = rows(7, 2, 64), (ints(0, 5), ints(0, 7))
    assert code(mdi.attn_prompt, rows(5, 4, 64), k, k, rows(1, 4, 64).expand(5, 4, 64), *one) == mdi.ERR_SHAPE


def test_scales_whose_product_with_log2_e_overflows():
    c, q = make(), rows(2, 8, 64)
    assert code(mdi.attn_decode, c, q, q, ints(1, 1), scale=2.9e38) == mdi.ERR_ARG
    assert code(mdi.attn_prompt, rows(5, 4, 64), rows(7, 2, 64), rows(7, 2, 64), rows(5, 4, 64), ints(0, 5), ints(0, 7), scale=2.9e38) == mdi.ERR_ARG
