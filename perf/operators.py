"""Timing cases of the operators that work on few-bit values outside the gradient exchange: the 4-bit cache of keys and values
(written, read back, attended to) and the matrix product in 8-bit integers.

A case is a dict of plain values. `op` says what one pass is:

  store    new tokens are quantised into the cache and come back as the values that the cache holds for them (a layer that
           attends to its new tokens densely, and to the same values later)
  read     the last tokens of every sequence, or all of them, are read back as dense keys and values
  attend   queries over the cache: one per sequence (generation), or a run of them (chunks of a prompt, verification)
  step     one layer of a generation step: the new token's key and value are stored, then attended to with the rest
  linear   x W^T: the rows of x are quantised, then multiplied with weights held in 8 bits
  product  both operands held in 8 bits

The cache is paged: a sequence's tokens lie in the pages that its row of `table` names. A page holds, for each head, tiles of 16 tokens:
key codes [head_dim / 64][16][32 bytes], key (lo, step) pairs [16][head_dim / 64], then the same for the values. A value is
lo + step * code, 64 values to a pair, both numbers in the cache's 16-bit type.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
GROUP, TILE = 64, 16


def listed():
    cache = lambda name, op, seqs, shortest, longest, queries, heads, kv_heads, dim, dtype, page: dict(
        name=name, op=op, seqs=seqs, shortest=shortest, longest=longest, queries=queries, heads=heads, kv_heads=kv_heads, dim=dim,
        dtype=dtype, page=page)
    product = lambda name, op, m, n, k, dtype, bias, padded: dict(name=name, op=op, m=m, n=n, k=k, dtype=dtype, bias=bias, padded=padded)
    return [
        # one layer, one user: the new token is stored and attended to with a short conversation
        cache("step_one_user", "step", 1, 1000, 1000, 1, 32, 8, 128, "bf16", 16),
        # prompts of twelve users, of very different lengths, enter the cache
        cache("store_prompts", "store", 12, 5, 2600, 0, 32, 8, 128, "bf16", 64),
        # a small model's generation step: seven tokens to store
        cache("store_tokens_fp16", "store", 7, 1, 1, 0, 8, 2, 64, "fp16", 16),
        # a long document goes back to a dense layout
        cache("read_document", "read", 1, 65536, 65536, 0, 32, 8, 128, "bf16", 128),
        # short and odd histories of wide heads
        cache("read_ragged_fp16", "read", 9, 1, 900, 0, 16, 4, 256, "fp16", 32),
        # generation for a batch of users
        cache("attend_batch", "attend", 64, 100, 8000, 1, 32, 8, 128, "bf16", 64),
        # generation at the end of a long document, eight query heads to a key head
        cache("attend_document", "attend", 1, 131071, 131071, 1, 64, 8, 128, "bf16", 64),
        # every query head with keys of its own
        cache("attend_own_keys_fp16", "attend", 33, 17, 1500, 1, 16, 16, 64, "fp16", 16),
        # chunks of four prompts over what is in the cache already
        cache("attend_chunks", "attend", 4, 700, 4096, 256, 32, 8, 128, "bf16", 64),
        # a generation step's product for one token, and for a batch of 37 with odd sizes
        product("linear_one_token", "linear", 1, 16384, 4096, "bf16", False, True),
        product("linear_batch_fp16", "linear", 37, 5000, 2885, "fp16", True, True),
        # a prompt's product
        product("product_prompt", "product", 8192, 8192, 4096, "bf16", False, True),
    ]


def spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["store", "read", "attend", "attend", "step", "linear", "linear", "product"])
    dtype = rng.choice(["bf16", "fp16"])
    if op in ("linear", "product"):
        case = dict(op=op, dtype=rng.choice(["bf16", "fp16", "fp32"]), bias=rng.random() < 0.5, padded=op == "linear" or rng.random() < 0.7)
        case["m"] = spread(rng, 1, 64) if rng.random() < 0.5 else spread(rng, 64, 6000)
        case["n"], case["k"] = spread(rng, 100, 10000), spread(rng, 64, 8000)
        if rng.random() < 0.6:
            case["n"], case["k"] = -(-case["n"] // 64) * 64, -(-case["k"] // 128) * 128
        return case
    dim = rng.choice([64, 128, 128, 192, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    seqs = spread(rng, 1, 64)
    most = 65536 * 8 * 128 // (kv_heads * dim)                 # tokens in all
    if op in ("store", "step", "attend"):
        most //= 2
    longest = spread(rng, 1 if op != "attend" else 16, max(16, most // seqs))
    longest = min(longest, 60000)
    shortest = rng.choice([longest, max(1, longest // 10), 1])
    group = rng.choice([1, 2, 4, 4, 8, 7, 12])
    queries = {"attend": rng.choice([1, 1, 1, 2, 5, min(64, spread(rng, 2, 128))]), "step": 1}.get(op, 0)
    return dict(op=op, seqs=seqs, shortest=shortest, longest=longest, queries=queries, heads=kv_heads * group, kv_heads=kv_heads,
                dim=dim, dtype=dtype, page=rng.choice([16, 16, 32, 64, 128]))


# -------------------------------------- what a case stands for --------------------------------------
def lengths(case):
    """Tokens of each sequence, from the shortest to the longest in a mixed order."""
    b, lo, hi = case["seqs"], case["shortest"], case["longest"]
    step = next(s for s in (37, 41, 43, 47, 53) if math.gcd(s, b) == 1)
    return [lo + (hi - lo) * (i * step % b) // max(b - 1, 1) if b > 1 else hi for i in range(b)]


def runs(case):
    """Tokens of each sequence that a pass deals with: what is stored or read (all of them), or the queries."""
    if case["op"] == "step":
        return [1] * case["seqs"]
    if case["op"] == "attend":
        # runs of different lengths, none longer than its sequence
        return [min(n, case["queries"] - i % 3 * (case["queries"] // 4)) for i, n in enumerate(lengths(case))]
    return lengths(case)


def work(case):
    """Each input read once, each output written once."""
    if case["op"] in ("linear", "product"):
        m, n, k, size = case["m"], case["n"], case["k"], 4 if case["dtype"] == "fp32" else 2
        given = m * k * size if case["op"] == "linear" else m * k + 4 * m
        return {"bytes": given + n * k + 4 * n + (4 * n if case["bias"] else 0) + m * n * size, "flops": 2 * m * n * k}
    h, d = case["kv_heads"], case["dim"]
    dense, held = 2 * h * d * 2, h * d * 9 // 8
    tokens, new = sum(lengths(case)), sum(runs(case))
    if case["op"] == "store":
        return {"bytes": new * 2 * (dense + held), "flops": 0}
    if case["op"] == "read":
        return {"bytes": new * (dense + held), "flops": 0}
    pairs = sum(q * n - q * (q - 1) // 2 for q, n in zip(runs(case), lengths(case)))
    total = tokens * held + new * case["heads"] * (4 * d + 4)
    if case["op"] == "step":
        total += new * dense
    return {"bytes": total, "flops": 4 * pairs * case["heads"] * d}


# ------------------------------------ what a program has in hand ------------------------------------
def normal(shape, seed, dtype=torch.float32, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def tokens_of(case, total, seed):
    """Keys and values of `total` tokens: each channel with a mean and a width of its own, as projections leave them."""
    h, d, dtype = case["kv_heads"], case["dim"], TYPES[case["dtype"]]
    pair = []
    for i in range(2):
        width = normal((h, d), seed + 10 + i).abs() + 0.2
        mean = normal((h, d), seed + 20 + i) * (1.0 if i == 0 else 0.1)
        out = torch.empty(total, h, d, dtype=dtype, device="cuda")
        for t in range(0, total, 32768):
            n = min(32768, total - t)
            out[t: t + n] = normal((n, h, d), seed + 31 * t + 30 + i) * width + mean
        pair.append(out)
    return pair


def prepare(case, seed):
    seed = 100000 * (seed + 1)
    if case["op"] in ("linear", "product"):
        return prepare_product(case, seed)
    dtype, page = TYPES[case["dtype"]], case["page"]
    h, d = case["kv_heads"], case["dim"]
    held, new = lengths(case), runs(case)
    pages = [-(-n // page) for n in held]
    n_pages = sum(pages) + 3
    g = torch.Generator().manual_seed(seed)
    order = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.zeros(len(held), max(pages), dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at: at + n]
        at += n
    st = {"case": case, "table": table.cuda(), "lengths": torch.tensor(held, dtype=torch.int32).cuda(),
          "data": torch.zeros(n_pages, h, page // TILE * 18 * d, dtype=torch.uint8, device="cuda"), "held": held, "new": new,
          "starts": torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32).cuda()}
    if max(new) == 1 and case["op"] != "read":
        st["starts"] = None                                  # one token of every sequence
    if case["op"] != "store":                                # what is in the cache already
        k, v = tokens_of(case, sum(held), seed)
        plain_write(st["data"], st["table"], places(held, held), page, k, v)
    if case["op"] in ("store", "step"):
        st["k"], st["v"] = tokens_of(case, sum(new), seed + 7)
    if case["op"] in ("store", "read"):
        st["k_out"], st["v_out"] = (torch.zeros(sum(new), h, d, dtype=dtype, device="cuda") for _ in range(2))
    if case["op"] in ("attend", "step"):
        st["q"] = normal((sum(new), case["heads"], d), seed + 3, dtype)
        st["out"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros(sum(new), case["heads"], device="cuda")
        st["scale"] = 1 / math.sqrt(d)
    st["places"] = places(held, new)
    if own:
        import paper_1610_02132_b200 as Q
        st["cache"] = Q.Cache(n_pages, page, h, d, dtype, data=st["data"])
        st["status"] = Q.new_status()
        if "q" in st:
            size = Q.qsgd_cache_attend_workspace_bytes(st["cache"], case["heads"])
            st["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return st


def prepare_product(case, seed):
    m, n, k, dtype = case["m"], case["n"], case["k"], TYPES[case["dtype"]]
    row = -(-k // 16) * 16 if case["padded"] else k          # rows that begin on 16-byte boundaries, or rows end to end
    st = {"case": case, "out": torch.zeros(m, n, dtype=dtype, device="cuda"), "bias": normal((n,), seed + 4) if case["bias"] else None}
    codes, st["w_scale"] = plain_rows(normal((n, k), seed + 1, scale=k ** -0.5))
    st["w"] = torch.zeros(n, row, dtype=torch.int8, device="cuda")[:, :k]
    st["w"].copy_(codes)
    # activations: a few channels are much larger than the others
    x = normal((m, k), seed + 2) * (1 + 9 * (torch.rand(k, generator=torch.Generator().manual_seed(seed)) < 0.01).float()).cuda()
    if case["op"] == "linear":
        st["x"] = x.to(dtype)
    else:
        codes, st["a_scale"] = plain_rows(x)
        st["a"] = torch.zeros(m, row, dtype=torch.int8, device="cuda")[:, :k]
        st["a"].copy_(codes)
    if own and case["op"] == "linear":
        import paper_1610_02132_b200 as Q
        st["workspace"] = torch.empty(Q.qsgd_linear_i8_workspace_bytes(m, k), dtype=torch.uint8, device="cuda")
    return st


def places(held, new):
    """(sequence, position) of every token that a pass deals with: the last new[b] of sequence b."""
    seq = torch.cat([torch.full((q,), b) for b, q in enumerate(new)]).cuda()
    pos = torch.cat([torch.arange(n - q, n) for n, q in zip(held, new)]).cuda()
    return seq, pos


# ------------------------------------------ the plain form ------------------------------------------
def parts(data, dim):
    """Views of the cache: key codes, key (lo, step), value codes, value (lo, step), each [page, head, tile, ...]."""
    tiles = data.view(data.shape[0], data.shape[1], -1, 18 * dim)
    out = []
    for at in (0, 9 * dim):
        out.append(tiles[..., at: at + 8 * dim].unflatten(-1, (dim // GROUP, TILE, 32)))
        out.append(tiles[..., at + 8 * dim: at + 9 * dim].view(torch.int16).unflatten(-1, (TILE, dim // GROUP, 2)))
    return out


def plain_quantize(x):
    """Codes and (lo, step) of groups of 64: step is the smallest number of the type with 15 * step >= max - min, and a value gets
    the nearest code, the lower one of two as near. In 64 bits: values of 16 bits often lie exactly between two codes."""
    v = x.double().unflatten(-1, (-1, GROUP))
    lo, hi = v.amin(-1, keepdim=True) + 0.0, v.amax(-1, keepdim=True)
    span = hi - lo
    step = (span / 15).to(x.dtype)
    up = (step.view(torch.int16) + 1).view(x.dtype)          # the next number above
    step = torch.where(15 * step.double() < span, up, step)
    step = torch.where(span < 15 * 2.0 ** -126, torch.zeros_like(step), step)
    codes = torch.where(step > 0, torch.ceil((v - lo) / step.double() - 0.5), torch.zeros_like(v))
    poisoned = ~torch.isfinite(span.float())                 # a value that is not finite, or a span beyond 32 bits
    nan = torch.full_like(step, math.nan)
    codes = torch.where(poisoned, torch.zeros_like(codes), codes).to(torch.uint8)
    pair = torch.cat([torch.where(poisoned, nan, lo.to(x.dtype)), torch.where(poisoned, nan, step)], -1)
    return codes, pair


def plain_write(data, table, where, page, k, v):
    seq, pos = where
    at = (table[seq, pos // page].long(), slice(None), pos % page // TILE)
    for x, codes_at, pair_at in zip((k, v), *(parts(data, k.shape[-1])[i::2] for i in range(2))):
        for i in range(0, x.shape[0], 32768):
            some = slice(i, i + 32768)
            codes, pair = plain_quantize(x[some])
            codes = codes[..., 0::2] | codes[..., 1::2] << 4
            page_at, slot = at[0][some], pos[some] % TILE
            codes_at[page_at, :, at[2][some], :, slot] = codes
            pair_at[page_at, :, at[2][some], slot] = pair.view(torch.int16)


def plain_read(data, table, where, page, dim, dtype):
    """Keys and values, in 32 bits."""
    seq, pos = where
    at, tile, slot = table[seq, pos // page].long(), pos % page // TILE, pos % TILE
    out = []
    for codes_at, pair_at in zip(*(parts(data, dim)[i::2] for i in range(2))):
        codes = codes_at[at, :, tile, :, slot]
        pair = pair_at[at, :, tile, slot].contiguous().view(dtype).float()
        codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float()
        out.append((pair[..., :1] + pair[..., 1:] * codes).flatten(-2))
    return out


def plain_attend(st):
    case = st["case"]
    at, group, dim, dtype = 0, case["heads"] // case["kv_heads"], case["dim"], st["q"].dtype
    for b, (n, q) in enumerate(zip(st["held"], st["new"])):
        pos = torch.arange(n, device="cuda")
        k, v = plain_read(st["data"], st["table"], (torch.full_like(pos, b), pos), case["page"], dim, dtype)
        rows = st["q"][at: at + q].float().unflatten(1, (-1, group)).permute(1, 0, 2, 3).flatten(1, 2)       # [kv head, q * group, dim]
        s = rows @ k.permute(1, 2, 0) * st["scale"]
        if q > 1:
            last = torch.arange(n - q, n, device="cuda").repeat_interleave(group)
            s = s.masked_fill(pos > last[:, None], -math.inf)
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        o = p @ v.permute(1, 0, 2) / total
        st["out"][at: at + q] = o.unflatten(1, (q, group)).permute(1, 0, 2, 3).flatten(1, 2).to(dtype)
        st["lse"][at: at + q] = (top + torch.log(total)).unflatten(1, (q, group)).permute(1, 0, 2, 3).flatten(1)
        at += q


def plain_rows(x):
    """8-bit codes of each row, and what one level stands for. In 64 bits: half the maximum lies between two codes."""
    v = x.double()
    top = v.abs().amax(-1, keepdim=True)
    codes = torch.round(v * 127 / top).to(torch.int8)
    return codes, (top / 127).float().squeeze(-1)


def run(st):
    return own_run(st) if own else plain_run(st)


def plain_run(st):
    case, op = st["case"], st["case"]["op"]
    if op in ("linear", "product"):
        a, scale = plain_rows(st["x"]) if op == "linear" else (st["a"], st["a_scale"])
        y = a.float() @ st["w"].float().t() * scale[:, None] * st["w_scale"]
        st["out"].copy_(y if st["bias"] is None else y + st["bias"])
        return st["out"]
    if op in ("store", "step"):
        plain_write(st["data"], st["table"], st["places"], case["page"], st["k"], st["v"])
    if op in ("store", "read"):
        for out, x in zip((st["k_out"], st["v_out"]),
                          plain_read(st["data"], st["table"], st["places"], case["page"], case["dim"], st["k_out"].dtype)):
            out.copy_(x)
        return {"k": st["k_out"], "v": st["v_out"]}
    plain_attend(st)
    return {"out": st["out"], "lse": st["lse"]}


# ------------------------------------------ a user's calls ------------------------------------------
def own_run(st):
    import paper_1610_02132_b200 as Q
    op = st["case"]["op"]
    if op == "linear":
        Q.qsgd_linear_i8(st["x"], st["w"], st["w_scale"], st["out"], st["workspace"], bias=st["bias"])
        return st["out"]
    if op == "product":
        Q.qsgd_matmul_i8(st["a"], st["a_scale"], st["w"], st["w_scale"], st["out"], bias=st["bias"])
        return st["out"]
    where = (st["cache"], st["table"], st["lengths"])
    if op in ("store", "step"):
        Q.qsgd_cache_write(*where, st["k"], st["v"], st["status"], starts=st["starts"])
    if op in ("store", "read"):
        Q.qsgd_cache_read(*where, st["k_out"], st["v_out"], st["status"], starts=st["starts"])
        return {"k": st["k_out"], "v": st["v_out"]}
    Q.qsgd_cache_attend(*where, st["q"], st["out"], st["workspace"], st["status"], starts=st["starts"], scale=st["scale"], lse=st["lse"])
    return {"out": st["out"], "lse": st["lse"]}


# -------------------------------------- the definition in 64 bits -----------------------------------
def exact_groups(x):
    """What a 4-bit cache of x's type holds for x."""
    v = x.double().reshape(*x.shape[:-1], -1, GROUP)
    lo = v.min(-1, keepdim=True).values
    ideal = (v.max(-1, keepdim=True).values - lo) / 15
    near = ideal.to(x.dtype)
    bits = near.view(torch.int16)                                                # not negative: the next number has the next pattern
    step = (bits + (near.double() < ideal)).to(torch.int16).view(x.dtype).double()
    thresholds = torch.arange(15, device="cuda") + 0.5                           # a code is the number of borders below the value
    codes = sum((v - lo > step * t).double() for t in thresholds)
    return (lo + step * codes).reshape(x.shape)


def exact_held(st, b, n):
    """Keys and values [n, head, dim] that the cache holds for a sequence, page by page."""
    case = st["case"]
    dim, page, dtype = case["dim"], case["page"], TYPES[case["dtype"]]
    pages = st["data"][st["table"][b, : -(-n // page)].long()]                   # [pages, head, bytes]
    tile = pages.reshape(pages.shape[0], pages.shape[1], page // TILE, 18 * dim)
    got = []
    for half in tile.split(9 * dim, -1):
        byte, pair = half[..., : 8 * dim].contiguous(), half[..., 8 * dim:].contiguous().view(dtype).double()
        value = torch.empty(*byte.shape, 2, dtype=torch.float64, device="cuda")
        value[..., 0], value[..., 1] = byte % 16, byte // 16
        value = value.reshape(*byte.shape[:3], dim // GROUP, TILE, GROUP).transpose(3, 4)
        pair = pair.reshape(*byte.shape[:3], TILE, dim // GROUP, 2)
        value = pair[..., 0, None] + pair[..., 1, None] * value
        got.append(value.reshape(*byte.shape[:3], TILE, dim).permute(0, 2, 3, 1, 4).reshape(-1, byte.shape[1], dim)[:n])
    return got


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op in ("linear", "product"):
        w, scale = st["w"].double(), st["w_scale"].double()
        if op == "linear":
            x = st["x"].double()
            top = x.abs().max(-1, keepdim=True).values
            a, a_scale = torch.round(x * 127 / top), top / 127
        else:
            a, a_scale = st["a"].double(), st["a_scale"].double()[:, None]
        y = torch.matmul(a, w.T) * a_scale * scale
        return y if st["bias"] is None else y + st["bias"].double()
    if op == "store":
        return {"k": exact_groups(st["k"]), "v": exact_groups(st["v"])}
    held, at = st["held"], 0
    if op == "read":
        got = [exact_held(st, b, n) for b, n in enumerate(held)]
        return {"k": torch.cat([k for k, _ in got]), "v": torch.cat([v for _, v in got])}
    group = case["heads"] // case["kv_heads"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(st["lse"].shape, dtype=torch.float64, device="cuda")
    for b, (n, q) in enumerate(zip(held, st["new"])):
        k, v = exact_held(st, b, n)
        if op == "step":
            k[-1], v[-1] = exact_groups(st["k"][b]), exact_groups(st["v"][b])
        for h in range(case["heads"]):
            s = torch.matmul(st["q"][at: at + q, h].double(), k[:, h // group].T) * st["scale"]
            s += torch.full((q, n), -math.inf, dtype=torch.float64, device="cuda").triu(n - q + 1)
            lse[at: at + q, h] = torch.logsumexp(s, -1)
            out[at: at + q, h] = torch.softmax(s, -1) @ v[:, h // group]
        at += q
    return {"out": out, "lse": lse}
