"""The operators of the paged 8-bit cache, as cases that can be timed and compared: appending a step's tokens with the
position rotation on the way, attention of one new token a sequence, and attention of many.

The cache (one layer): pages of 128 tokens, page block_table[b][n] holds tokens 128 n .. 128 n + 127 of sequence b,

    k_codes 8 bit [P][H][128 tokens][D]   v_codes 8 bit [P][H][D][128 tokens]   (signed integers, or e4m3)
    k_scales, v_scales fp32 [P][H]        one scale for each block of tokens and KV head: a code stands for code * scale
    k_res, v_res half [B][H][128][D]      the length mod 128 newest tokens, as they came (K rotated)

seq_lens are the tokens before the step, which brings rows cu_tokens[b] .. cu_tokens[b + 1] of its inputs to sequence b.

  append     token i of sequence b is at position p = seq_lens[b] + i.  q and k: of the first rotary_dim channels, pairs
             (x, y) become (x cos - y sin, x sin + y cos), rounded to 32 bits and then to the half type.  A block that the step completes is
             quantized: scale = max|x| / (127 or 448) in 32 bits, code = x / scale in 32 bits, to the nearest (ties to even).
             Returned: rotated q, and the cache as it is then.  Codes come as they are held, beside their scales: every
             step of their arithmetic is one defined rounding, so they have to be equal.
  attention  query i of sequence b, at p, over the length n = seq_lens[b] + (the step's tokens):  s_j = softmax_scale q.k_j,
             cap tanh(s_j / cap) if there is a cap, minus slope |p - j|; visible are j < prefix[b] (the prefix is seen whole,
             by its own tokens too) and j <= p with p - j < window (0: all).  out = sum softmax(s)_j v_j.

Head counts are 32 over 8 (the LLaMA-3.1-8B shape, which the benchmark uses) unless a case says otherwise.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
PAGE = 128
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
CODES = {"int8": (torch.int8, 127.0), "e4m3": (torch.float8_e4m3fn, 448.0)}


def _case(name, op, batch, context, tokens, code="int8", dtype="fp16", q_heads=32, kv_heads=8, head_dim=128, ragged=True,
          rotary_dim=None, interleaved=False, softcap=0.0, slopes=False, window=0, prefix=0):
    """context, tokens: the longest sequence's tokens before the step, and of the step.  ragged: the others have fewer."""
    c = {"op": op, "batch": batch, "context": context, "tokens": tokens, "code": code, "dtype": dtype, "q_heads": q_heads,
         "kv_heads": kv_heads, "head_dim": head_dim, "ragged": ragged}
    if op == "append":
        c |= {"rotary_dim": head_dim if rotary_dim is None else rotary_dim, "interleaved": interleaved}
    else:
        c |= {"softcap": softcap, "slopes": slopes, "window": window, "prefix": prefix}
    return c if name is None else {"name": name} | c


def listed():
    return [
        # one user's chat, one token: all latency
        _case("append_1", "append", 1, 700, 1),
        # serving: a token of each of 64 users, some of whom complete a block
        _case("append_64", "append", 64, 5000, 1, code="e4m3", dtype="bf16"),
        # prompts of a batch as they come, of any length; a rotation of half of the channels, interleaved
        _case("append_prompts_9x1333", "append", 9, 0, 1333, rotary_dim=64, interleaved=True),
        # one long prompt
        _case("append_prompt_16k", "append", 1, 0, 16384, code="e4m3", dtype="bf16"),
        # one user's chat of a few hundred tokens: all latency
        _case("decode_700", "attn", 1, 700, 1),
        # one user at 32K and at 128K tokens, the benchmark's two headline lengths
        _case("decode_32k", "attn", 1, 32768 + 20, 1),
        _case("decode_128k", "attn", 1, 131072 + 64, 1, code="e4m3", dtype="bf16"),
        # serving: a ragged batch, 8 query heads per KV head, capped scores
        _case("decode_40x8k_cap", "attn", 40, 8000, 1, code="e4m3", dtype="bf16", q_heads=64, softcap=50.0),
        # five drafted tokens a sequence are looked over at once
        _case("verify_16x4k", "attn", 16, 4000, 5),
        # ragged prompts of a smaller model: heads of 64 without groups, a bias by distance, a prefix that sees itself whole
        _case("prompts_6x1333_bias", "attn", 6, 0, 1333, code="e4m3", dtype="fp16", q_heads=16, kv_heads=16, head_dim=64, slopes=True,
              prefix=200),
        # a piece of a long prompt behind what is cached of it; a window
        _case("chunk_1k_after_31k", "attn", 1, 31744, 1024, dtype="bf16", softcap=30.0, window=16384),
        # a prompt in one piece
        _case("prompt_8k", "attn", 1, 0, 8192, code="e4m3", dtype="bf16"),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    d = {"code": rng.choice(["int8", "e4m3"]), "dtype": rng.choice(["fp16", "bf16"]), "head_dim": rng.choice([64, 128, 128]),
         "ragged": rng.random() < 0.7}
    kv = rng.choice([1, 2, 4, 8, 8, 12])
    d |= {"kv_heads": kv, "q_heads": kv * rng.choice([1, 3, 4, 4, 5, 8] if kv < 8 else [1, 2, 4, 4, 8])}
    how = rng.choice(["append_step", "append_prompt", "decode", "decode", "verify", "prompt", "prompt"])
    if how == "append_step":
        return _case(None, "append", _spread(rng, 1, 128), _spread(rng, 1, 8000), 1, rotary_dim=rng.choice([32, 64, d["head_dim"]]),
                     interleaved=rng.random() < 0.4, **d)
    if how == "append_prompt":
        batch = _spread(rng, 1, 12)
        return _case(None, "append", batch, 128 * rng.randrange(0, 20), _spread(rng, 2, 16384 // batch),
                     rotary_dim=rng.choice([32, 64, d["head_dim"]]), interleaved=rng.random() < 0.4, **d)
    d |= {"softcap": rng.choice([0.0, 0.0, 30.0, 50.0]), "slopes": rng.random() < 0.25, "window": rng.choice([0, 0, 0, _spread(rng, 100, 8192)]),
          "prefix": rng.choice([0, 0, 0, _spread(rng, 4, 600)])}
    if how in ("decode", "verify"):
        batch = _spread(rng, 1, 64)
        most = 131072 * 8 // (batch * kv)
        return _case(None, "attn", batch, _spread(rng, 30, min(131072, most)), 1 if how == "decode" else rng.randrange(2, 9), **d)
    batch = _spread(rng, 1, 8)
    context = rng.choice([0, 0, 128 * rng.randrange(1, 100)])
    # (scores of all queries against all keys: no more than the largest listed case)
    most = (8192 * 8192 * 32 // (batch * d["q_heads"]))
    tokens = int((math.sqrt(context * context + 4 * most) - context) / 2)
    return _case(None, "attn", batch, context, _spread(rng, 9, max(10, min(8192, tokens))), **d)


def _lengths(case):
    """Every sequence's tokens before the step, and of the step."""
    rng = random.Random(case["batch"] * 1000003 + case["context"] * 31 + case["tokens"])
    ctx, new = [], []
    for b in range(case["batch"]):
        part = 1.0 if b == 0 or not case["ragged"] else rng.uniform(0.2, 1.0)
        ctx.append(int(case["context"] * part) if case["tokens"] < 9 else int(case["context"] * part) // PAGE * PAGE)
        new.append(max(1, int(case["tokens"] * part)) if case["tokens"] >= 9 else case["tokens"])
        if case["op"] == "append" and b % 16 == 5 and case["tokens"] == 1:   # the token that completes a block
            ctx[b] = ctx[b] // PAGE * PAGE + PAGE - 1
    return ctx, new


def _quantized(x, code, dims):
    """Codes and scales of x, one scale over `dims`."""
    kind, most = CODES[code]
    scale = x.abs().amax(dims, keepdim=True) / torch.tensor(most, device=x.device)
    y = x / scale.clamp_min(1e-30)
    return (y.round() if code == "int8" else y).clamp(-most, most).to(kind), scale.reshape(scale.shape[:2])


def prepare(case, seed):
    ctx, new = _lengths(case)
    B, H, Hq, D, dtype = case["batch"], case["kv_heads"], case["q_heads"], case["head_dim"], TYPES[case["dtype"]]
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, device=DEVICE, generator=gen)   # noqa: E731
    channels = lambda: 1 + 9 * (torch.rand((1, H, 1, D), device=DEVICE, generator=gen) < 0.01).float()   # noqa: E731  (large ones)
    total, columns = sum(new), (max(c + n for c, n in zip(ctx, new)) + PAGE - 1) // PAGE + 1
    pages = B * columns
    k_large, v_large = channels(), channels()
    table = torch.randperm(pages, generator=gen, device=DEVICE).to(torch.int32).reshape(B, columns)
    # (a pool at a time: neither side of the largest cache is held in 32 bits twice)
    k_codes, k_scales = _quantized(normal(pages, H, PAGE, D).mul_(k_large), case["code"], (2, 3))
    v_codes, v_scales = _quantized(normal(pages, H, PAGE, D).mul_(v_large).transpose(2, 3), case["code"], (2, 3))
    s = {"case": case, "k_codes": k_codes.contiguous(), "v_codes": v_codes.contiguous(), "k_scales": k_scales.contiguous(),
         "v_scales": v_scales.contiguous(), "k_res": (normal(B, H, PAGE, D) * k_large).to(dtype), "v_res": (normal(B, H, PAGE, D) * v_large).to(dtype),
         "table": table, "lens": torch.tensor(ctx, dtype=torch.int32, device=DEVICE),
         "cu": torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32, device=DEVICE), "most": max(new), "longest": max(c + n for c, n in zip(ctx, new))}
    if case["op"] == "append":
        # q, k and v as the projection leaves them: parts of one row a token
        qkv = normal(total, Hq + 2 * H, D).to(dtype)
        s |= {"q": qkv[:, :Hq], "k": qkv[:, Hq:Hq + H], "v": qkv[:, Hq + H:], "q_out": torch.empty(total, Hq, D, dtype=dtype, device=DEVICE)}
        half = case["rotary_dim"] // 2
        angle = torch.arange(s["longest"], device=DEVICE, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, device=DEVICE, dtype=torch.float64) / half)
        s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    else:
        s |= {"q": normal(total, Hq, D).to(dtype), "out": torch.empty(total, Hq, D, dtype=dtype, device=DEVICE)}
        s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, Hq + 1, device=DEVICE) / Hq) if case["slopes"] else None
        s["prefix"] = torch.tensor([case["prefix"] * (b + 1) // B for b in range(B)], dtype=torch.int32, device=DEVICE) if case["prefix"] else None
    if own:   # the handle that a program keeps, over the same buffers
        from paper_2503_18773_amd import binding
        s["cache"] = binding.PagedKV8Cache(B, Hq, H, case["code"], pages, table, head_dim=D, dtype=dtype, seq_lens=s["lens"],
                                           buffers=[s[x] for x in ("k_codes", "v_codes", "k_scales", "v_scales", "k_res", "v_res")], device=DEVICE)
        s["cu_own"] = None if s["most"] == 1 else s["cu"]   # (one token a sequence: no list of rows)
        if case["op"] == "append":
            s["rotation"] = binding.Rotation(s["cos_sin"], interleaved=case["interleaved"])
    return s


def run(s):
    case = s["case"]
    if case["op"] == "append":
        if own:
            s["cache"].append(s["k"], s["v"], q=s["q"], q_out=s["q_out"], cu_tokens=s["cu_own"], max_tokens=s["most"], rotation=s["rotation"])
        else:
            _append(s)
        return {"q": s["q_out"], "k_codes": s["k_codes"], "v_codes": s["v_codes"], "k_scales": s["k_scales"], "v_scales": s["v_scales"],
                "k_res": s["k_res"], "v_res": s["v_res"]}
    if own:
        return s["cache"].attn(s["q"], 1 / math.sqrt(case["head_dim"]), s["out"], cu_tokens=s["cu_own"], max_tokens=s["most"], max_len=s["longest"],
                               softcap=case["softcap"], slopes=s["slopes"], window=case["window"], prefix_lens=s["prefix"])
    return _attention(s)


# ---- the plain forms -----------------------------------------------------------------------------

def _rows(s):
    """Sequence, index in the step and position of every row of the step."""
    t = torch.arange(s["q"].shape[0], device=DEVICE)
    seq = torch.searchsorted(s["cu"][1:].contiguous(), t.int(), right=True)
    i = t - s["cu"].long()[seq]
    return seq, i, s["lens"].long()[seq] + i


def _rotated(x, cos, sin, interleaved):
    r = 2 * cos.shape[1]
    y, c, s = x.double(), cos.double()[:, None], sin.double()[:, None]
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if interleaved else (y[..., :r // 2], y[..., r // 2:r])
    a, b = a * c - b * s, a * s + b * c
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned.float().to(x.dtype), x[..., r:]], -1)


def _append(s):
    case, lens, cu = s["case"], s["lens"].long(), s["cu"].long()
    kind, most = CODES[case["code"]]
    half = case["rotary_dim"] // 2
    _, _, pos = _rows(s)
    cos, sin = s["cos_sin"][pos, :half], s["cos_sin"][pos, half:]
    s["q_out"].copy_(_rotated(s["q"], cos, sin, case["interleaved"]))
    new = cu[1:] - cu[:-1]
    first, blocks = lens // PAGE, (s["most"] + 2 * PAGE - 2) // PAGE + 1   # blocks of a sequence that the step can touch
    at = first[:, None] * PAGE + torch.arange(blocks * PAGE, device=DEVICE)        # [B][tokens] positions
    is_new = (at >= lens[:, None]) & (at < (lens + new)[:, None])
    row = (cu[:-1, None] + at - lens[:, None]).clamp(0, s["q"].shape[0] - 1)
    which = (first[:, None] + torch.arange(blocks, device=DEVICE)).clamp(max=s["table"].shape[1] - 1)
    page = s["table"].long().gather(1, which)
    full = (first[:, None] + torch.arange(1, blocks + 1, device=DEVICE)) * PAGE <= (lens + new)[:, None]
    # (a block that the step does not complete goes to a page behind the pool, which is dropped)
    page = torch.where(full, page, s["k_codes"].shape[0]).flatten()
    slot = torch.arange(PAGE, device=DEVICE)
    tail_row = (lens + new) // PAGE * PAGE
    for_tail = ((tail_row[:, None] + slot >= lens[:, None]) & (slot < ((lens + new) % PAGE)[:, None]))[:, None, :, None]
    tail_from = (cu[:-1, None] + tail_row[:, None] + slot - lens[:, None]).clamp(0, s["q"].shape[0] - 1)
    for x, name in ((_rotated(s["k"], cos, sin, case["interleaved"]), "k"), (s["v"], "v")):
        res, codes, scales = s[name + "_res"], s[name + "_codes"], s[name + "_scales"]
        old = torch.cat([res, torch.zeros_like(res[:, :, :1]).expand(-1, -1, (blocks - 1) * PAGE, -1)], 2).transpose(1, 2)
        whole = torch.where(is_new[:, :, None, None], x[row], old).reshape(-1, blocks, PAGE, *x.shape[1:]).permute(0, 1, 3, 2, 4).float()
        scale = whole.abs().amax((3, 4)) / torch.tensor(most, device=DEVICE)
        y = whole / torch.where(scale > 0, scale, 1.0)[..., None, None]
        y = torch.where(scale[..., None, None] > 0, y.round() if case["code"] == "int8" else y, 0.0).clamp(-most, most).to(kind)
        y = (y if name == "k" else y.transpose(3, 4)).flatten(0, 1).contiguous()
        codes.copy_(torch.cat([codes.view(torch.uint8), torch.zeros_like(codes[:1]).view(torch.uint8)]).index_put_((page,), y.view(torch.uint8))[:-1].view(kind))
        scales.copy_(torch.cat([scales, scales[:1]]).index_put_((page,), scale.flatten(0, 1))[:-1])
        res.copy_(torch.where(for_tail, x[tail_from].transpose(1, 2), res))


def _cached(s, name):
    """The cached tokens' values in 32 bits, [B][H][padded length][D]."""
    codes, scales, res = s[name + "_codes"], s[name + "_scales"], s[name + "_res"].float()
    lens = s["lens"].long() + s["cu"].long().diff()
    n = s["table"].shape[1]
    x = codes[s["table"].long()].float() if codes.dtype == torch.int8 else codes.view(torch.uint8)[s["table"].long()].view(codes.dtype).float()
    x = x * scales[s["table"].long()][..., None, None]
    x = (x if name == "k" else x.transpose(3, 4)).transpose(1, 2).flatten(2, 3)
    at = torch.arange(n * PAGE, device=DEVICE)
    tail = (lens // PAGE * PAGE)[:, None]
    x = torch.where((at >= tail)[:, None, :, None], res.repeat(1, 1, n, 1), x)
    return torch.where((at < lens[:, None])[:, None, :, None], x, 0.0)


def _attention(s):
    case = s["case"]
    B, H, g = case["batch"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    new, n = s["cu"].long().diff(), s["most"]
    total = s["lens"].long() + new
    k, v = _cached(s, "k"), _cached(s, "v")
    seq, i, _ = _rows(s)
    i_of = torch.arange(n, device=DEVICE)
    rows = (s["cu"].long()[:-1, None] + i_of).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][rows].float().unflatten(2, (H, g)).permute(0, 2, 3, 1, 4).flatten(2, 3)   # [B][H][g n][D]
    x = torch.matmul(q, k.transpose(2, 3)).mul_(1 / math.sqrt(case["head_dim"])).unflatten(2, (g, n))
    if case["softcap"]:
        x = torch.tanh(x / case["softcap"]) * case["softcap"]
    p, j = (s["lens"].long()[:, None] + i_of)[:, :, None], torch.arange(k.shape[2], device=DEVICE)
    if s["slopes"] is not None:
        x = x - s["slopes"].reshape(1, H, g, 1, 1) * (p - j).abs()[:, None, None].float()
    seen = (j <= p) & (p - j < (case["window"] or 1 << 30))
    if s["prefix"] is not None:
        seen = seen | (j < s["prefix"][:, None, None])
    seen = (seen & (j < total[:, None, None]))[:, None, None]
    x = x.masked_fill_(~seen, -math.inf)
    x = torch.exp(x.sub_(x.amax(-1, keepdim=True).clamp_min(-1e30)))
    norm = x.sum(-1, keepdim=True)
    y = torch.matmul(x.flatten(2, 3), v).unflatten(2, (g, n)) / norm.clamp_min(1e-30)
    return y.flatten(1, 2)[seq, :, i].to(s["q"].dtype)   # [T][heads][D]


def work(case):
    ctx, new = _lengths(case)
    H, Hq, D = case["kv_heads"], case["q_heads"], case["head_dim"]
    rows = sum(new)
    if case["op"] == "append":
        done = sum((c + n) // PAGE - c // PAGE for c, n in zip(ctx, new))   # blocks completed
        moved = sum(c % PAGE for c, n in zip(ctx, new) if (c + n) // PAGE > c // PAGE)   # older tokens of those
        left = sum((c + n) % PAGE if (c + n) // PAGE > c // PAGE else n for c, n in zip(ctx, new))
        return {"bytes": rows * (2 * Hq + 2 * H) * D * 2 + (moved + left) * H * D * 4 + done * H * (PAGE * D + 4) * 2 + rows * case["rotary_dim"] * 4,
                "flops": rows * (Hq + H) * case["rotary_dim"] * 3}
    keys = pairs = 0
    for b, (c, n) in enumerate(zip(ctx, new)):
        prefix = min(case["prefix"] * (b + 1) // case["batch"], c + n)
        window = case["window"] or c + n
        start = max(0, c + 1 - window)            # the first key that the first query's window has
        keys += (c + n) - start + min(prefix, start)
        for p in range(c, c + n):
            low = max(0, p + 1 - window)
            pairs += p + 1 - low + min(prefix, low) + max(0, prefix - p - 1)
    return {"bytes": keys * H * 2 * D + rows * Hq * D * 4, "flops": 4 * D * Hq * pairs}


# ---- the definition in 64 bits ---------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_append(s, case) if case["op"] == "append" else _exact_attention(s, case)


def _exact_append(s, case):
    ctx, new = _lengths(case)
    kind, most = CODES[case["code"]]
    half, dtype = case["rotary_dim"] // 2, TYPES[case["dtype"]]
    out, row = {x: s[x].clone() for x in ("k_codes", "v_codes", "k_scales", "v_scales", "k_res", "v_res")}, 0
    q_out = []
    for b, (c, n) in enumerate(zip(ctx, new)):
        turn = torch.complex(s["cos_sin"][c:c + n, :half].double(), s["cos_sin"][c:c + n, half:].double())[:, None]

        def rotated(x):
            z = x[..., :2 * half].double()
            z = torch.view_as_complex(z.unflatten(-1, (half, 2))) if case["interleaved"] else torch.complex(z[..., :half], z[..., half:])
            re = z.real * turn.real - z.imag * turn.imag
            im = z.real * turn.imag + z.imag * turn.real
            z = torch.stack([re, im], -1).flatten(-2) if case["interleaved"] else torch.cat([re, im], -1)
            return torch.cat([z.float().to(dtype), x[..., 2 * half:]], -1)

        q_out.append(rotated(s["q"][row:row + n]))
        tokens = {"k": rotated(s["k"][row:row + n]), "v": s["v"][row:row + n]}
        row += n
        for name, x in tokens.items():
            old = c % PAGE
            x = torch.cat([s[name + "_res"][b, :, :old], x.transpose(0, 1)], 1)   # [H][tokens][D] from the last block's start on
            for block in range(x.shape[1] // PAGE):
                page = int(s["table"][b, c // PAGE + block])
                y = x[:, block * PAGE:(block + 1) * PAGE].double()
                scale = (y.abs().amax((1, 2)) / most).float()
                z = (y / torch.where(scale > 0, scale, 1.0).double()[:, None, None]).float()
                z = (z.round() if case["code"] == "int8" else z).clamp(-most, most).to(kind)
                out[name + "_codes"].view(torch.uint8)[page] = (z if name == "k" else z.transpose(1, 2)).contiguous().view(torch.uint8)
                out[name + "_scales"][page] = scale
            left = x.shape[1] % PAGE
            begin = 0 if x.shape[1] >= PAGE else old
            out[name + "_res"][b, :, begin:left] = x[:, x.shape[1] // PAGE * PAGE + begin:]
    return {"q": torch.cat(q_out), **out}


def _exact_attention(s, case):
    ctx, new = _lengths(case)
    H, Hq, D = case["kv_heads"], case["q_heads"], case["head_dim"]
    g, row, outs = Hq // H, 0, []
    for b, (c, n) in enumerate(zip(ctx, new)):
        length, full = c + n, (c + n) // PAGE
        values = []
        for name in ("k", "v"):
            pages = s["table"][b, :full].long()
            x = s[name + "_codes"].view(torch.uint8)[pages].view(s[name + "_codes"].dtype).double() * s[name + "_scales"][pages].double()[:, :, None, None]
            x = x if name == "k" else x.transpose(2, 3)
            values.append(torch.cat([x.transpose(0, 1).reshape(H, full * PAGE, D), s[name + "_res"][b, :, :length % PAGE].double()], 1))
        p, j = torch.arange(c, length, device=DEVICE)[:, None], torch.arange(length, device=DEVICE)[None]
        seen = (j <= p) if not case["window"] else (j <= p) & (j > p - case["window"])
        if case["prefix"]:
            seen = seen | (j < case["prefix"] * (b + 1) // case["batch"])
        y = torch.empty(n, Hq, D, dtype=torch.float64, device=DEVICE)
        for h in range(Hq):
            x = (s["q"][row:row + n, h].double() @ values[0][h // g].T) * D ** -0.5
            if case["softcap"]:
                x = torch.tanh(x / case["softcap"]) * case["softcap"]
            if case["slopes"]:
                x = x - float(s["slopes"][h]) * (p - j).abs()
            y[:, h] = torch.softmax(x.masked_fill(~seen, -math.inf), 1) @ values[1][h // g]
        outs.append(y)
        row += n
    return torch.cat(outs)
