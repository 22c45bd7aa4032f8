"""Performance cases of the attention operators: the paged key/value cache in 16 or 8 bits (written and read back), attention
of one new token over it, and causal attention over whole packed prompts.

``own`` false: the operators in elementary torch operations, 32 bits wide.  ``own`` true: the library's entry points.
``exact`` gives the outputs from the definitions in 64 bits.

Stored rows.  A row is the ``head_dim`` elements of one head at one position.  "f16" / "bf16": rounded to that type.  "i8":
scale = max(absmax / 127, 2^-126) in fp32, elements = x / scale rounded to the nearest integer, ties to even.  "e4m3":
scale = 2^k with the smallest k >= -126 for which absmax <= 448 * 2^k, elements = x / scale rounded to e4m3.  A stored element
stands for element * scale.
"""
import math
import random

import torch

own = False

STORE = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn, "f16": torch.float16, "bf16": torch.bfloat16}
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"i8": 1, "e4m3": 1, "f16": 2, "bf16": 2, "f32": 4}


def listed():
    return [
        # a decode step of the Llama-7B shape: 64 samples append one row each, straight from the fp32 projection
        {"name": "write_step_i8", "op": "write", "n_seq": 64, "new": 1, "past": 640, "kv_heads": 32, "head_dim": 128, "page": 16, "store": "i8", "dtype": "f32", "ragged": False, "shape": 1},
        # first visits of a batch of prompts, grouped heads
        {"name": "write_prompts_e4m3", "op": "write", "n_seq": 16, "new": 2048, "past": 0, "kv_heads": 8, "head_dim": 128, "page": 64, "store": "e4m3", "dtype": "bf16", "ragged": True, "shape": 2},
        # a first visit's next chunk wants the rows cached so far: 16 samples of the GPT-2-XL shape
        {"name": "read_xl_i8", "op": "read", "n_seq": 16, "len": 1024, "kv_heads": 25, "head_dim": 64, "page": 16, "store": "i8", "dtype": "f16", "ragged": True, "shape": 3},
        # long documents read back whole
        {"name": "read_long_e4m3", "op": "read", "n_seq": 4, "len": 32768, "kv_heads": 8, "head_dim": 128, "page": 128, "store": "e4m3", "dtype": "bf16", "ragged": False, "shape": 4},
        # one user, one token, the GPT-2-small shape: latency
        {"name": "decode_one_f16", "op": "decode", "n_seq": 1, "len": 1000, "heads": 12, "kv_heads": 12, "head_dim": 64, "page": 16, "store": "f16", "dtype": "f16", "ragged": False, "shape": 5},
        # 64 samples of the Llama-7B shape at the end of their generation, fp32 activations
        {"name": "decode_llama_7b_i8", "op": "decode", "n_seq": 64, "len": 640, "heads": 32, "kv_heads": 32, "head_dim": 128, "page": 16, "store": "i8", "dtype": "f32", "ragged": False, "shape": 6},
        # a serving batch of very different lengths, grouped heads, an idle slot among them
        {"name": "decode_ragged_bf16", "op": "decode", "n_seq": 32, "len": 8192, "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64, "store": "bf16", "dtype": "bf16", "ragged": True, "shape": 7},
        # a few long documents, groups of five heads
        {"name": "decode_long_e4m3", "op": "decode", "n_seq": 4, "len": 100003, "heads": 40, "kv_heads": 8, "head_dim": 128, "page": 128, "store": "e4m3", "dtype": "bf16", "ragged": False, "shape": 8},
        # one short prompt of the GPT-2-XL shape: latency of a first visit
        {"name": "prompt_short", "op": "prompt", "n_seq": 1, "new": 200, "past": 0, "heads": 25, "kv_heads": 25, "head_dim": 64, "dtype": "bf16", "ragged": False, "shape": 9},
        # first visits of a batch, packed
        {"name": "prompt_packed", "op": "prompt", "n_seq": 16, "new": 2048, "past": 0, "heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "f16", "ragged": True, "shape": 10},
        # one long prompt
        {"name": "prompt_long", "op": "prompt", "n_seq": 1, "new": 8192, "past": 0, "heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "ragged": False, "shape": 11},
        # the next chunk of four prompts behind what is cached already
        {"name": "prompt_chunk", "op": "prompt", "n_seq": 4, "new": 512, "past": 4096, "heads": 32, "kv_heads": 32, "head_dim": 128, "dtype": "bf16", "ragged": True, "shape": 12},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "read", "decode", "prompt"])
    kv = rng.choice([1, 2, 4, 5, 8, 12, 25, 32])
    head_dim = rng.choice([32, 64, 128])
    c = {"op": op, "kv_heads": kv, "head_dim": head_dim, "ragged": rng.random() < 0.7, "shape": rng.randrange(1 << 20)}
    row = kv * head_dim
    if op == "prompt":
        group = rng.choice([g for g in (1, 2, 3, 4, 5, 8) if g * kv <= 40])
        c |= {"heads": group * kv, "dtype": rng.choice(["f16", "bf16"]), "new": _spread(rng, 1, 6000), "past": rng.choice([0, 0, _spread(rng, 1, 6000)])}
        pairs = c["new"] * (c["new"] + c["past"]) * c["heads"]
        c["n_seq"] = max(1, min(_spread(rng, 1, 40), int(1.5e9 / pairs)))
        return c
    store = rng.choice(["i8", "e4m3", "f16", "bf16"])
    c |= {"page": rng.choice([16, 32, 64, 128]), "store": store, "dtype": rng.choice(["f32", "f16", "bf16"])}
    if op == "decode":
        group = rng.choice([g for g in (1, 2, 3, 4, 5, 8, 16) if g * kv <= 64])
        c |= {"heads": group * kv, "len": _spread(rng, 1, 120000)}
        c["n_seq"] = max(1, min(_spread(rng, 1, 200), int(2e8 / (c["len"] * row))))
        c["len"] = max(1, min(c["len"], int(2e8 / (c["n_seq"] * row))))
    elif op == "read":
        c |= {"len": _spread(rng, 1, 30000)}
        c["n_seq"] = max(1, min(_spread(rng, 1, 200), int(6e7 / (c["len"] * row))))
        c["len"] = max(1, min(c["len"], int(6e7 / (c["n_seq"] * row))))
    else:
        c |= {"new": rng.choice([1, _spread(rng, 1, 8000)]), "past": rng.choice([0, _spread(rng, 1, 4000)])}
        c["n_seq"] = max(1, min(_spread(rng, 1, 200), int(3e7 / (c["new"] * row))))
        c["new"] = max(1, min(c["new"], int(3e7 / (c["n_seq"] * row))))
    return c


def _lengths(case):
    """(rows of the call, rows before them) of every sequence: the first is the longest; ragged batches of eight or more hold an empty one."""
    rng = random.Random(case["shape"])
    n, new, past = case["n_seq"], case.get("new", case.get("len")), case.get("past", 0)
    if not case["ragged"]:
        return [new] * n, [past] * n
    rows = [new] + [_spread(rng, 1, new) for _ in range(n - 1)]
    before = [past] + [rng.randrange(past + 1) for _ in range(n - 1)]
    if n >= 8:
        rows[n // 2] = 0
    return rows, before


def _pairs(rows, before):
    return sum(r * p + r * (r + 1) // 2 for r, p in zip(rows, before))


def work(case):
    rows, before = _lengths(case)
    r, kv, d = sum(rows), case["kv_heads"], case["head_dim"]
    b = SIZE[case["dtype"]]
    if case["op"] == "prompt":
        return {"bytes": 2 * r * case["heads"] * d * b + 2 * (r + sum(before)) * kv * d * b, "flops": 4 * d * case["heads"] * _pairs(rows, before)}
    stored = SIZE[case["store"]] * d + (4 if SIZE[case["store"]] == 1 else 0)  # a row of one head with its scale
    if case["op"] == "write":  # the new rows come in, are stored, and are read back
        return {"bytes": 2 * r * kv * (d * b + 2 * stored + d * b), "flops": 8 * r * kv * d}
    if case["op"] == "read":
        return {"bytes": 2 * r * kv * (stored + d * b), "flops": 2 * r * kv * d}
    return {"bytes": 2 * r * kv * stored + 2 * case["n_seq"] * case["heads"] * d * b, "flops": 4 * r * case["heads"] * d}


def _starts(counts):
    s = [0]
    for c in counts:
        s.append(s[-1] + c)
    return torch.tensor(s, dtype=torch.int32, device="cuda")


def _rows(gen, n, heads, head_dim):
    """Activations: normal, channels of different strength (keys have a few strong ones)."""
    strength = torch.exp(0.4 * torch.randn(1, heads, head_dim, generator=gen, device="cuda"))
    return torch.randn(n, heads, head_dim, generator=gen, device="cuda") * strength


def _stored(x, store):
    """Rows as they are stored (elements, scales or None): the plain form of the cache's types."""
    if store in ("f16", "bf16"):
        return x.to(STORE[store]), None
    big = x.float().abs().amax(-1)
    if store == "i8":
        scale = (big.double() / 127).float().clamp_min(2.0 ** -126)
        return torch.round(x.double() / scale.double()[..., None]).clamp(-127, 127).to(torch.int8), scale  # borders need 64 bits
    m, e = torch.frexp(big.double())  # big = m * 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    k = (e - 9 + (m > 0.875)).clamp_min(-126)
    scale = torch.ldexp(torch.ones_like(m), torch.where(big > 0, k, torch.full_like(k, -126))).float()
    return (x.float() / scale[..., None]).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, before = _lengths(case)
    kv, d, dtype = case["kv_heads"], case["head_dim"], TYPES[case["dtype"]]
    st = {"case": case, "start": _starts(rows), "n_rows": sum(rows), "max_new": max(rows), "dtype": dtype}
    st["new"] = torch.tensor(rows, dtype=torch.int32, device="cuda")
    if case["op"] == "prompt":
        total = [r + p for r, p in zip(rows, before)]
        st["k_start"], st["max_all"] = _starts(total), max(total)
        st["q"] = _rows(gen, sum(rows), case["heads"], d).to(dtype)
        st["k"] = _rows(gen, sum(total), kv, d).to(dtype)
        st["v"] = _rows(gen, sum(total), kv, d).to(dtype)
        st["out"] = torch.zeros_like(st["q"])
        return st
    # the pool: pages handed out in no particular order, what lies behind a sequence's last row is left over from others
    page, n_seq = case["page"], case["n_seq"]
    pages = [-(-(r + p) // page) for r, p in zip(rows, before)]
    n_pages, width = sum(pages) + 3, max(max(pages), 1)
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((n_seq, width), -1, dtype=torch.int32, device="cuda")
    filled = torch.arange(width, device="cuda")[None, :] < torch.tensor(pages, device="cuda")[:, None]
    table[filled] = order[: sum(pages)]
    pool = torch.randint(-100, 100, (n_pages, 2, kv, page, d * SIZE[case["store"]]), generator=gen, device="cuda", dtype=torch.int8).view(STORE[case["store"]])
    scale = torch.rand(n_pages, 2, kv, page, generator=gen, device="cuda") if SIZE[case["store"]] == 1 else None
    if case["op"] != "write":
        for which in (0, 1):
            for p0 in range(0, n_pages, max(1, (1 << 27) // (kv * page * d))):
                part = pool[p0:p0 + max(1, (1 << 27) // (kv * page * d)), which]
                x = _rows(gen, part.shape[0] * page, kv, d).view(part.shape[0], page, kv, d).transpose(1, 2)
                q, s = _stored(x, case["store"])
                part.copy_(q)
                if s is not None:
                    scale[p0:p0 + part.shape[0], which] = s
    st |= {"pool": pool, "scale": scale, "table": table, "pos": torch.tensor(before, dtype=torch.int32, device="cuda")}
    if case["op"] == "decode":
        st["q"] = _rows(gen, n_seq, case["heads"], d).to(dtype)
        st["out"] = torch.zeros_like(st["q"])
    else:
        st["k_out"] = torch.zeros(sum(rows), kv, d, dtype=dtype, device="cuda")
        st["v_out"] = torch.zeros_like(st["k_out"])
    if case["op"] == "write":
        st["k"] = _rows(gen, sum(rows), kv, d).to(dtype)
        st["v"] = _rows(gen, sum(rows), kv, d).to(dtype)
    if own:  # the handle that a user's program keeps for as long as the cache lives, and the attention's working memory
        from paper_2505_18164_b200 import mdi
        st["cache"] = mdi.KvCache(pool, table, scale=scale)
        if case["op"] == "decode":
            st["ws"] = torch.empty(max(1, mdi.attn_decode_workspace(st["cache"], case["heads"], st["max_new"])), dtype=torch.uint8, device="cuda")
    return st


def run(state):
    return {"write": _write, "read": _read, "decode": _decode, "prompt": _prompt}[state["case"]["op"]](state)


def _places(st):
    """Sequence, page and row in the page of every row of the call."""
    i = torch.arange(st["n_rows"], dtype=torch.int32, device="cuda")
    seq = torch.searchsorted(st["start"][1:].contiguous(), i, right=True)
    at = (i - st["start"][seq] + st["pos"][seq]).long()
    page = st["case"]["page"]
    return st["table"][seq, at // page].long(), at % page


def _values(st, which, page, at):
    """Stored rows as fp32: pool[page, which, :, at] * scale."""
    q = st["pool"]
    if q.dtype == torch.float8_e4m3fn:
        x = q.view(torch.uint8)[page, which, :, at].view(torch.float8_e4m3fn).float()
    else:
        x = q[page, which, :, at].float()
    return x if st["scale"] is None else x * st["scale"][page, which, :, at][..., None]


def _write(st):
    if own:
        from paper_2505_18164_b200 import mdi
        stream = torch.cuda.current_stream().cuda_stream
        mdi.kv_append(st["cache"], st["k"], st["v"], st["start"], st["pos"], stream=stream)
        mdi.kv_read(st["cache"], st["k_out"], st["v_out"], st["start"], st["pos"], stream=stream)
        return st["k_out"], st["v_out"]
    page, at = _places(st)
    new = torch.stack((st["k"], st["v"]), 1)
    q, s = _stored(new, st["case"]["store"])
    q, pool = (q.view(torch.uint8), st["pool"].view(torch.uint8)) if q.dtype == torch.float8_e4m3fn else (q, st["pool"])
    pool[page, 0, :, at], pool[page, 1, :, at] = q[:, 0], q[:, 1]
    if s is not None:
        st["scale"][page, 0, :, at], st["scale"][page, 1, :, at] = s[:, 0], s[:, 1]
    return _values(st, 0, page, at).to(st["dtype"]), _values(st, 1, page, at).to(st["dtype"])


def _read(st):
    if own:
        from paper_2505_18164_b200 import mdi
        mdi.kv_read(st["cache"], st["k_out"], st["v_out"], st["start"], st["pos"], stream=torch.cuda.current_stream().cuda_stream)
        return st["k_out"], st["v_out"]
    page, at = _places(st)
    return _values(st, 0, page, at).to(st["dtype"]), _values(st, 1, page, at).to(st["dtype"])


def _softmax(s):
    """Rows of scores, -inf where masked; a row with nothing left gives zeros."""
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, torch.ones_like(total), total)


def _decode(st):
    if own:
        from paper_2505_18164_b200 import mdi
        mdi.attn_decode(st["cache"], st["q"], st["out"], st["new"], st["max_new"], workspace=st["ws"], stream=torch.cuda.current_stream().cuda_stream)
        return st["out"]
    c = st["case"]
    at = torch.arange(st["max_new"], device="cuda").expand(c["n_seq"], -1)
    there = at < st["new"][:, None]
    page = torch.gather(st["table"], 1, at // c["page"]).long().clamp_min(0)
    off = at % c["page"]
    zero = torch.zeros((), device="cuda")
    k = torch.where(there[..., None, None], _values(st, 0, page, off), zero).transpose(1, 2)  # [n_seq, kv_heads, len, head_dim]
    v = torch.where(there[..., None, None], _values(st, 1, page, off), zero).transpose(1, 2)
    q = st["q"].float().view(c["n_seq"], c["kv_heads"], -1, c["head_dim"])
    s = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(c["head_dim"])
    p = _softmax(s.masked_fill(~there[:, None, None], -math.inf))
    return torch.matmul(p, v).view(c["n_seq"], c["heads"], c["head_dim"]).to(st["dtype"])


def _padded(x, start, count, most):
    """Packed rows as [n_seq, most, heads, head_dim], zero behind each sequence's last row."""
    at = torch.arange(most, device="cuda")
    there = at[None, :] < count[:, None]
    i = torch.where(there, start[:-1, None] + at[None, :], torch.zeros((), dtype=torch.int32, device="cuda"))
    return torch.where(there[..., None, None], x[i].float(), torch.zeros((), device="cuda")), there


def _prompt(st):
    if own:
        from paper_2505_18164_b200 import mdi
        mdi.attn_prompt(st["q"], st["k"], st["v"], st["out"], st["start"], st["k_start"], stream=torch.cuda.current_stream().cuda_stream)
        return st["out"]
    c = st["case"]
    group = c["heads"] // c["kv_heads"]
    count = st["k_start"][1:] - st["k_start"][:-1]
    q, q_there = _padded(st["q"], st["start"], st["new"], st["max_new"])
    k, _ = _padded(st["k"], st["k_start"], count, st["max_all"])
    v, _ = _padded(st["v"], st["k_start"], count, st["max_all"])
    n, lq, lk = c["n_seq"], st["max_new"], st["max_all"]
    q = q.view(n, lq, c["kv_heads"], group, -1).permute(0, 2, 3, 1, 4).reshape(n, c["kv_heads"], group * lq, -1)
    s = torch.matmul(q, k.permute(0, 2, 3, 1)).view(n, c["kv_heads"], group, lq, lk)
    i, j = torch.arange(lq, device="cuda")[:, None], torch.arange(lk, device="cuda")[None, :]
    seen = j <= i + (count - st["new"])[:, None, None]  # the last new row sees all of its sequence
    p = _softmax(s.mul_(1 / math.sqrt(c["head_dim"])).masked_fill_(~seen[:, None, None], -math.inf))
    o = torch.matmul(p.view(n, c["kv_heads"], group * lq, lk), v.transpose(1, 2)).view(n, c["kv_heads"], group, lq, -1)
    return o.permute(0, 3, 1, 2, 4).reshape(n, lq, c["heads"], -1)[q_there].to(st["dtype"])


def exact(case, seed):
    st = prepare(case, seed)
    rows, before = _lengths(case)
    kv, d, page = case["kv_heads"], case["head_dim"], case.get("page")
    starts = [sum(rows[:n]) for n in range(len(rows))]
    if case["op"] == "prompt":
        out = torch.zeros(sum(rows), case["heads"], d, dtype=torch.float64, device="cuda")
        k0 = 0
        for r, p, q0 in zip(rows, before, starts):
            for a in range(0, r, 2048):  # query rows a..b of the sequence, all heads of one key/value head at a time
                b = min(r, a + 2048)
                hidden = torch.ones(b - a, p + b, dtype=torch.bool, device="cuda").triu(p + a + 1)
                for h in range(kv):
                    heads = slice(h * (case["heads"] // kv), (h + 1) * (case["heads"] // kv))
                    k, v = st["k"][k0:k0 + p + b, h].double(), st["v"][k0:k0 + p + b, h].double()
                    s = torch.einsum("ihd,jd->hij", st["q"][q0 + a:q0 + b, heads].double(), k) * d ** -0.5
                    w = torch.softmax(s.masked_fill(hidden, -math.inf), -1)
                    out[q0 + a:q0 + b, heads] = torch.einsum("hij,jd->ihd", w, v)
            k0 += r + p
        return out

    def cached(which, seq, first, count):
        """Rows first .. first + count - 1 of a sequence, [count, kv_heads, head_dim]."""
        pages = st["table"][seq, : -(-(first + count) // page)].long()
        x = (st["pool"].view(torch.uint8) if case["store"] == "e4m3" else st["pool"])[pages, which]
        x = (x.view(torch.float8_e4m3fn) if case["store"] == "e4m3" else x).double()
        if st["scale"] is not None:
            x = x * st["scale"][pages, which].double().unsqueeze(-1)
        return x.transpose(1, 2).reshape(-1, kv, d)[first:first + count]

    if case["op"] == "write":
        def after(x):
            x = x.double()
            if case["store"] in ("f16", "bf16"):
                return x.to(STORE[case["store"]]).double()
            big = x.abs().max(-1, keepdim=True).values
            if case["store"] == "i8":
                s = torch.maximum(big / 127, torch.full_like(big, 2.0 ** -126)).float().double()
                y = x / s
                return torch.clamp(y.round(), -127, 127) * s
            s = torch.where(big > 0, torch.exp2(torch.ceil(torch.log2(big / 448) - 1e-13).clamp_min(-126)), torch.full_like(big, 2.0 ** -126))
            y = (x / s).abs()
            step = torch.exp2(torch.floor(torch.log2(y.clamp_min(2.0 ** -6))) - 3)  # distance of neighbouring e4m3 numbers at y
            return torch.sign(x) * torch.round(y / step) * step * s
        return after(st["k"]), after(st["v"])
    if case["op"] == "read":
        k, v = (torch.cat([cached(w, n, p, r) for n, (r, p) in enumerate(zip(rows, before)) if r]) for w in (0, 1))
        return k, v
    out = torch.zeros(case["n_seq"], case["heads"], d, dtype=torch.float64, device="cuda")
    for n, r in enumerate(rows):
        if r:
            q = st["q"][n].double().view(kv, -1, d)
            s = torch.einsum("hgd,lhd->hgl", q, cached(0, n, 0, r)) * d ** -0.5
            w = torch.exp(s - torch.logsumexp(s, -1, keepdim=True))
            out[n] = torch.einsum("hgl,lhd->hgd", w, cached(1, n, 0, r)).reshape(case["heads"], d)
    return out
