"""Contexts with an 8-bit key/value cache (kv_cache_dtype MDI_KV_I8 / MDI_KV_E4M3): first visits and steps run through the
attention operators.  Reference: the whole decoder in torch fp64 with every key and value row rounded to the cache's type (a row's
rounding depends on that row alone, so the forward over all positions with rounded rows is what the cached steps compute).

Tolerance: 3e-2 absolute on logits, the bf16 tolerance of the parity tests.  It has to cover: 16-bit query and weight planes (2^-11
relative at worst, in first visits), and single elements that round to the other neighbour because the library's k or v differs
from the fp64 one by ~1e-5: one such element moves a score by at most |q_e| absmax / 127 / sqrt(hd) (int8), of which there is about
one per thousand elements."""
import numpy as np
import pytest
import torch

from paper_2505_18164_b200 import inputs as I, mdi
from helpers import make_oracle, tiny_shape

pytestmark = pytest.mark.gpu
KINDS = {"i8": mdi.KV_I8, "e4m3": mdi.KV_E4M3}


def rounded(x, kind):
    """Rows x[..., hd] (fp64) as the values that stand for them in the cache."""
    big = x.abs().amax(-1, keepdim=True)
    if kind == "i8":
        s = (big / 127).float().double().clamp_min(2.0 ** -126)
        return torch.round(x / s) * s
    s = torch.where(big > 0, torch.exp2(torch.ceil(torch.log2(big / 448) - 1e-12)), torch.ones_like(big))
    y = x / s
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(y / step) * step * s


def forward(shape, w, tokens, kind):
    """Logits of every position, fp64, keys and values rounded."""
    W = {k: torch.from_numpy(I.as_f32(v)).double() for k, v in w.items()}
    T, H, KV, hd, d = len(tokens), shape.n_head, shape.n_kv_head, shape.head_dim, shape.d_model
    gpt = shape.arch == I.ARCH_GPT
    x = W["wte"][torch.tensor(tokens)]
    if gpt:
        x = x + W["wpe"][:T]

    def norm(v, pfx):
        if gpt:
            m = v.mean(-1, keepdim=True)
            return (v - m) / torch.sqrt(((v - m) ** 2).mean(-1, keepdim=True) + shape.norm_eps) * W[pfx + ".g"] + W[pfx + ".b"]
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + shape.norm_eps) * W[pfx + ".g"]

    half = hd // 2
    ang = torch.arange(T, dtype=torch.float64)[:, None] * shape.rope_theta ** (-torch.arange(half, dtype=torch.float64) * 2 / hd) if not gpt else None

    def rope(t):
        if gpt:
            return t
        c, s = ang.cos()[:, None], ang.sin()[:, None]
        a, b = t[..., :half], t[..., half:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    for l in range(shape.n_layer):
        p = f"h.{l}."
        y = norm(x, p + "ln1") @ W[p + "attn.wqkv"].T + (W[p + "attn.bqkv"] if gpt else 0)
        q, k, v = y[:, :H * hd].view(T, H, hd), y[:, H * hd:(H + KV) * hd].view(T, KV, hd), y[:, (H + KV) * hd:].view(T, KV, hd)
        q, k, v = rope(q), rounded(rope(k), kind), rounded(v, kind)
        k, v = k.repeat_interleave(H // KV, 1), v.repeat_interleave(H // KV, 1)
        s = torch.einsum("ihd,jhd->hij", q, k) * hd ** -0.5
        s = s.masked_fill(torch.ones(T, T, dtype=torch.bool).triu(1), -torch.inf)
        o = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v).reshape(T, H * hd)
        x = x + o @ W[p + "attn.wo"].T + (W[p + "attn.bo"] if gpt else 0)
        y = norm(x, p + "ln2")
        if gpt:
            h = torch.nn.functional.gelu(y @ W[p + "mlp.w1"].T + W[p + "mlp.b1"], approximate="tanh")
            x = x + h @ W[p + "mlp.w2"].T + W[p + "mlp.b2"]
        else:
            x = x + (torch.nn.functional.silu(y @ W[p + "mlp.wgate"].T) * (y @ W[p + "mlp.wup"].T)) @ W[p + "mlp.wdown"].T
    return norm(x, "lnf") @ W["wte" if shape.tied_lm_head else "lm_head"].T


CASES = [
    # arch, L, d, H, n_kv, V, C, bounds, S, P, N, options
    ("llama", 4, 128, 2, 2, 211, 96, [0, 2, 4], 6, 9, 16, {}),                                # groups of 3
    ("llama", 4, 128, 2, 1, 211, 400, [0, 1, 4], 3, 290, 40, dict(page_tokens=16)),           # three chunks of a prompt, grouped heads
    ("llama", 2, 256, 2, 1, 300, 160, [0, 2], 8, 130, 12, {}),                                # head_dim 128, one partition, groups of 8
    ("gpt", 3, 128, 4, None, 523, 96, [0, 1, 2, 3], 2, 6, 20, dict(page_tokens=32)),          # head_dim 32, fewer samples than partitions
    ("gpt", 2, 64, 4, None, 97, 64, [0, 1, 2], 3, 1, 30, {}),                                 # head_dim 16, prompt of one token
]


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("arch,L,d,H,n_kv,V,C,bounds,S,P,N,opts", CASES)
def test_logits_against_rounded_rows(kind, arch, L, d, H, n_kv, V, C, bounds, S, P, N, opts):
    shape = tiny_shape(arch, I.DT_BF16, L=L, d=d, H=H, V=V, C=C, F=2 * d, n_kv=n_kv)
    w = I.make_weights(shape, 3, 0.05)
    prompts = I.make_prompts(V, S, P, seed=5)
    ctx = mdi.Context(shape, bounds, S, kv_cache_dtype=KINDS[kind], **opts)
    ctx.load_all(w)
    teacher = I.make_prompts(V, S, N, seed=6)
    for rounds in range(2):                                   # slots are used again: pages from other samples
        for s in range(S):
            ctx.set_teacher_tokens(s, [int(t) for t in teacher[s]])
            ctx.prefill(s, prompts[s])
        ref = [forward(shape, w, [int(t) for t in prompts[s]] + [int(t) for t in teacher[s]], kind) for s in range(S)]
        for s in range(S):
            assert np.abs(ctx.get_logits(s) - ref[s][P - 1].numpy()).max() <= 3e-2
        for n in (1, N // 2, N):                              # the last of n tokens was produced at position P + n - 2
            done = 0 if n == 1 else (1 if n == N // 2 else N // 2)
            ctx.generate(S, n - done)
            for s in range(S):
                assert np.abs(ctx.get_logits(s) - ref[s][P + n - 2].numpy()).max() <= 3e-2
        for s in range(S):
            ctx.reset_sample(s)
    st = ctx.stats()
    assert st.kv_element_bytes == 1 and sum(st.kv_pages_in_use[:len(bounds) - 1]) == 0
    ctx.close()


@pytest.mark.parametrize("kind", list(KINDS))
def test_steps_by_hand_equal_the_pipeline(kind):
    """mdi_step through both partitions (the operators called for one sequence) against mdi_generate on another context."""
    shape = tiny_shape("llama", I.DT_BF16, L=2, d=128, H=2, V=211, C=96, F=256, n_kv=1)
    w = I.make_weights(shape, 3, 0.05)
    prompt = I.make_prompts(211, 1, 20, seed=5)[0]
    a, b = (mdi.Context(shape, [0, 1, 2], 1, kv_cache_dtype=KINDS[kind]) for _ in range(2))
    for c in (a, b):
        c.load_all(w)
        c.prefill(0, prompt)
    toks = a.generate(1, 10)[0]
    la = a.get_logits(0)
    x = torch.empty(shape.d_model, device="cuda")
    tok = torch.empty(1, dtype=torch.int32, device="cuda")
    got = [int(b.generate(1, 1)[0][0])]
    for i in range(9):
        tok.fill_(got[-1])
        b.step(0, 0, tok, x)
        b.sync()
        b.step(1, 0, x, tok)
        b.sync()
        got.append(int(tok.item()))
    assert got == [int(t) for t in toks]
    assert np.array_equal(la, b.get_logits(0))
    a.close(), b.close()


def test_refusals():
    shape = tiny_shape("llama", I.DT_BF16, L=2, d=128, H=2, V=211, C=96, F=256)
    for kw, code in ((dict(scheduler=2), mdi.ERR_SHAPE), (dict(scheduler=4), mdi.ERR_SHAPE), (dict(prefill_mode=1), mdi.ERR_SHAPE),
                     (dict(page_tokens=8), mdi.ERR_SHAPE), (dict(kv_cache_dtype=6), mdi.ERR_ARG), (dict(kv_cache_dtype=-1), mdi.ERR_ARG)):
        with pytest.raises(mdi.MdiError) as e:
            mdi.Context(shape, [0, 1, 2], 2, **{"kv_cache_dtype": mdi.KV_I8, **kw})
        assert e.value.code == code
    with pytest.raises(mdi.MdiError) as e:
        mdi.Context(tiny_shape("gpt", I.DT_F32), [0, 2], 2, kv_cache_dtype=mdi.KV_E4M3)
    assert e.value.code == mdi.ERR_SHAPE
