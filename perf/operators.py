"""The attention operators whose speed counts: a key/value cache in 8 bits, the attention that reads it, and the attention over blocks
that a score selects.

Three kinds of case:

  append   new tokens' keys and values are rounded into the cache, and the blocks they touched are read back as values
  attend   every new token attends to the earlier ones in the cache (and to itself)
  focused  the same over the blocks of 64 tokens that a score selects for it; the selected blocks are an output

A sequence's new tokens are its last ones.  `new` = 1 is serving one token after another; `new` = `length` is a prompt in one piece,
in between lies a prompt that is read in pieces.  With `ragged` the sequences' lengths lie between a quarter of `length` and all of
it; `idle` sequences of the batch are empty slots (length zero), whose rows have nothing to attend to.

Keys share a direction within a block, which differs from block to block, as the tokens of one passage or one image region do.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 64


def _case(name, kind, batch, new, length, kv_heads, group, dim, dtype="bf16", ragged=False, idle=0, first=0, last=0, top=0):
    return dict(name=name, kind=kind, batch=batch, new=new, length=length, kv_heads=kv_heads, group=group, dim=dim, dtype=dtype,
                ragged=ragged, idle=idle, first=first, last=last, top=top)


def listed():
    return [
        # one user's next token enters the cache: launches only
        _case("append_step_b1", "append", 1, 1, 1000, 8, 4, 128),
        # a full batch's next tokens
        _case("append_step_b256", "append", 256, 1, 4096, 8, 4, 128, ragged=True),
        # prompts enter the cache, blocks begun and left unfinished at both ends
        _case("append_prompt", "append", 6, 4001, 5000, 8, 4, 128, ragged=True),
        # one user's next token, a short dialogue: latency
        _case("attend_step_b1", "attend", 1, 1, 1000, 8, 4, 128),
        # a full batch's next tokens, ragged, some slots empty: the cache's bandwidth
        _case("attend_step_b64", "attend", 64, 1, 8192, 8, 4, 128, ragged=True, idle=3),
        # one user's next token over a very long cache: few rows, a long axis
        _case("attend_step_long", "attend", 1, 1, 131000, 8, 8, 128),
        # a prompt in one piece
        _case("attend_prompt", "attend", 1, 8192, 8192, 8, 4, 128),
        # pieces of prompts in 16-bit floats, head size off the tile sizes, as many key heads as query heads
        _case("attend_pieces_f16", "attend", 3, 517, 5003, 12, 1, 80, "f16", ragged=True),
        # one user's next token over 512 blocks
        _case("focused_step_b1", "focused", 1, 1, 32768, 8, 4, 128, first=1, last=2, top=13),
        # a batch's next tokens over long caches
        _case("focused_step_b16", "focused", 16, 1, 65000, 8, 4, 128, ragged=True, idle=1, first=1, last=2, top=29),
        # a piece of a long prompt: every token selects for itself; the largest
        _case("focused_prompt", "focused", 1, 4096, 32768, 8, 4, 128, first=1, last=2, top=13),
        # ragged pieces, an odd head size and an odd group
        _case("focused_pieces_f16", "focused", 2, 700, 9001, 2, 5, 96, "f16", ragged=True, first=2, last=1, top=6),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "focused", "focused"])
    kv_heads, group, dim = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 64, 80, 96, 128, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    ragged = rng.random() < 0.6
    if rng.random() < 0.5:          # single tokens
        batch, new, length = _log(rng, 1, 128), 1, _log(rng, 64, 131072)
    else:                           # prompts and pieces of them
        batch, length = _log(rng, 1, 8), _log(rng, 64, 16384)
        new = length if rng.random() < 0.5 else _log(rng, 2, length)
    while batch > 1 and batch * length > 1 << 20:
        batch //= 2
    while batch * new * length * kv_heads * group * dim > 1.3e11:
        new = max(1, new // 2)
    case = _case("", kind, batch, new, length, kv_heads, group, dim, dtype, ragged, 1 if batch > 2 and rng.random() < 0.3 else 0)
    if kind == "focused":
        case.update(first=rng.choice([0, 1, 1, 2]), last=rng.choice([1, 1, 2, 4]), top=_log(rng, 2, 32))
    del case["name"]
    return case


# ---- inputs -------------------------------------------------------------------

def _lengths(case):
    """(length, new tokens) of every sequence; a function of the case alone."""
    rng = random.Random(case["batch"] * 1000003 + case["length"])
    lengths, news = [], []
    for b in range(case["batch"]):
        length, new = case["length"], case["new"]
        if case["ragged"] and b:
            length = rng.randint((length + 3) // 4, length)
            new = new if new == 1 else min(length, rng.randint((new + 3) // 4, new))
        if b >= case["batch"] - case["idle"]:
            length = 0
            new = 1 if case["new"] == 1 else 0
        lengths.append(length)
        news.append(new)
    return lengths, news


def _inputs(case, seed):
    """Keys and values of every token, queries of the new ones, the sequences' blocks in the pool."""
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    dtype, hk, d = DTYPES[case["dtype"]], case["kv_heads"], case["dim"]
    lengths, news = _lengths(case)
    k = torch.empty((sum(lengths), hk, d), dtype=dtype, device=DEVICE)
    v = torch.empty_like(k)
    at = 0
    for length in lengths:
        blocks = -(-length // BLOCK)
        shared = torch.randn((blocks, hk, d), generator=gen, device=DEVICE).mul_(0.6).repeat_interleave(BLOCK, 0)[:length]
        k[at:at + length] = torch.randn((length, hk, d), generator=gen, device=DEVICE).mul_(0.8).add_(shared)
        v[at:at + length] = torch.randn((length, hk, d), generator=gen, device=DEVICE)
        at += length
    q = torch.randn((sum(news), hk * case["group"], d), generator=gen, device=DEVICE).mul_(1.5).to(dtype)
    needed = [-(-length // BLOCK) for length in lengths]
    pool = sum(needed) + 3
    order = torch.randperm(pool, generator=gen, device=DEVICE).to(torch.int32)
    table = torch.full((case["batch"], max(needed + [1])), -1, dtype=torch.int32, device=DEVICE)
    at = 0
    for b, n in enumerate(needed):
        table[b, :n] = order[at:at + n]
        at += n
    return dict(lengths=lengths, news=news, k=k, v=v, q=q, pool=pool, table=table)


def _sums(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _new_rows(x, lengths, news):
    """The rows of every sequence's new tokens."""
    starts = _sums(lengths)
    return torch.cat([x[starts[b + 1] - min(n, lengths[b]):starts[b + 1]] for b, n in enumerate(news)]).contiguous()


# ---- the plain form -------------------------------------------------------------

def _pow2(e):
    """2^e in 32 bits, e a tensor of whole numbers of [-126, 127]."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _scale_of(amax):
    """The least power of two s with amax <= 448 s."""
    m, e = torch.frexp(amax)
    return _pow2(torch.where(m <= 0.875, e - 9, e - 8).clamp(-64, 120))


def _unit_of(amax):
    """The exponent of the least power of two s with amax <= 127 s."""
    m, e = torch.frexp(amax)
    return torch.where(m <= 127 / 128, e - 7, e - 6).clamp(-126, 120)


def _fill_block_scales(x, old=0, old_scale=None):
    """x [blocks, 64, heads, dim] in 32 bits, zeros behind the last token -> (codes, scales [blocks, heads]); the first `old` tokens of
    the first block were there before, under `old_scale`, and keep the block from taking a smaller one."""
    s = _scale_of(x.abs().amax(dim=(1, 3)))
    if old:
        s[0] = torch.maximum(_scale_of(x[0, old:].abs().amax(dim=(0, 2))), old_scale)
    return (x / s[:, None, :, None]).to(torch.float8_e4m3fn), s


def _blocks_of(x, lead=0):
    """[tokens, heads, dim] -> [blocks, 64, heads, dim] in 32 bits, `lead` places left free before the first token."""
    n = lead + x.shape[0]
    out = torch.zeros((-(-n // BLOCK) * BLOCK,) + tuple(x.shape[1:]), dtype=torch.float32, device=x.device)
    out[lead:n] = x
    return out.view(-1, BLOCK, *x.shape[1:])


def _plain_pool(inputs, case, upto):
    """The cache in the plain form's layout, holding the first upto[b] tokens of every sequence."""
    hk, d = case["kv_heads"], case["dim"]
    pool = {n: torch.zeros((inputs["pool"], BLOCK, hk, d), dtype=torch.float8_e4m3fn, device=DEVICE) for n in "kv"}
    scales = {n: torch.ones((inputs["pool"], hk), device=DEVICE) for n in "kv"}
    starts = _sums(inputs["lengths"])
    for b, length in enumerate(upto):
        if length <= 0:
            continue
        at = inputs["table"][b, :-(-length // BLOCK)].long()
        for n in "kv":
            codes, s = _fill_block_scales(_blocks_of(inputs[n][starts[b]:starts[b] + length]))
            pool[n].view(torch.uint8)[at] = codes.view(torch.uint8)
            scales[n][at] = s
    return pool, scales


def _plain_append(state):
    out = {"k": [], "v": []}
    at = 0
    for b, (length, new) in enumerate(zip(state["lengths"], state["news"])):
        if min(length, new) == 0:
            continue
        had = length - new
        old = had % BLOCK
        first = int(had // BLOCK)
        for n in "kv":
            x = _blocks_of(state[n][at:at + new], old)
            old_scale = None
            if old:
                page = state["table"][b, first].long()
                old_scale = state["scales"][n][page]
                x[0, :old] = state["pool"][n][page, :old].float() * old_scale[None, :, None]
            codes, s = _fill_block_scales(x, old, old_scale)
            out[n].append((codes.float() * s[:, None, :, None]).view(-1, *x.shape[2:])[:old + new])
        at += new
    return [torch.cat(out["k"]), torch.cat(out["v"])]


def _gathered(state, b, n):
    """One sequence's keys or values in 32 bits, [kv heads, tokens, dim]."""
    length = state["lengths"][b]
    at = state["table"][b, :-(-length // BLOCK)].long()
    x = state["pool"][n].view(torch.uint8)[at].view(torch.float8_e4m3fn).float() * state["scales"][n][at][:, None, :, None]
    return x.view(-1, *x.shape[2:])[:length].transpose(0, 1).contiguous()


def _plain_select(state, b, q, positions):
    """The blocks of every query [rows, kv heads, dim of the list], ascending, -1 behind the last."""
    case = state["case"]
    first, last, top = case["first"], case["last"], case["top"]
    hk, group = case["kv_heads"], case["group"]
    rows = q.shape[0]
    width = first + last + top
    length = state["lengths"][b]
    full = length // BLOCK
    blocks = -(-length // BLOCK)
    at = state["table"][b, :full].long()
    # a block's sketch: the sum of its keys' codes, rounded to 8 bits under a power of two
    sums = state["pool"]["k"].view(torch.uint8)[at].view(torch.float8_e4m3fn).float().sum(dim=1)
    e = _unit_of(sums.abs().amax(dim=2))
    sketch = torch.round(sums * _pow2(-e)[:, :, None])
    weight = state["scales"]["k"][at] * _pow2(e) / BLOCK
    # the queries of a group, rounded alike
    q = q.float().view(rows, hk, group, -1)
    q8 = torch.round(q * _pow2(-_unit_of(q.abs().amax(dim=(2, 3))))[:, :, None, None]).sum(dim=2)
    score = torch.zeros((rows, hk, blocks), device=DEVICE)
    score[:, :, :full] = torch.matmul(q8.transpose(0, 1), sketch.permute(1, 2, 0).contiguous()).transpose(0, 1) * weight.t()[None]
    number = torch.arange(blocks, device=DEVICE)
    own_block = (positions // BLOCK)[:, None, None]
    always = (number < first) | (number > own_block - last)
    score = torch.where(always, float("inf"), score)
    score = torch.where(number > own_block, float("-inf"), score)
    order = torch.sort(score, dim=2, descending=True, stable=True).indices
    forced = (always & (number <= own_block)).sum(dim=2, keepdim=True)
    wanted = torch.minimum(forced + top, own_block + 1)
    place = torch.arange(width, device=DEVICE)
    if blocks < width:
        order = torch.cat([order, order.new_zeros((rows, order.shape[1], width - blocks))], dim=2)
    chosen = torch.where(place < wanted, order[:, :, :width].expand(rows, hk, width), blocks)
    chosen = torch.sort(chosen, dim=2).values
    return torch.where(chosen < blocks, chosen, -1).to(torch.int32)


def _plain_attend(state, focused):
    case = state["case"]
    hk, group, d = case["kv_heads"], case["group"], case["dim"]
    scale = 1.0 / math.sqrt(d)
    out = torch.zeros_like(state["q"])
    width = case["first"] + case["last"] + case["top"]
    lists = torch.full((out.shape[0], hk, width), -1, dtype=torch.int32, device=DEVICE) if focused else None
    row = 0
    for b, (length, new) in enumerate(zip(state["lengths"], state["news"])):
        if length == 0 or new == 0:
            row += new
            continue
        k, v = _gathered(state, b, "k").transpose(1, 2).contiguous(), _gathered(state, b, "v")
        token = torch.arange(length, device=DEVICE)
        step = max(1, (1 << 28) // (hk * group * length))
        for at in range(0, new, step):
            n = min(step, new - at)
            q = state["q"][row + at:row + at + n]
            position = length - new + at + torch.arange(n, device=DEVICE)
            seen = (token <= position[:, None])[None]
            if focused:
                chosen = _plain_select(state, b, q, position)
                lists[row + at:row + at + n] = chosen
                marks = torch.zeros((n, hk, -(-length // BLOCK) + 1), dtype=torch.bool, device=DEVICE)
                marks.scatter_(2, torch.where(chosen < 0, marks.shape[2] - 1, chosen).long(), True)
                seen = seen & marks[:, :, token // BLOCK].transpose(0, 1)
            z = torch.matmul(q.float().view(n, hk, group, d).permute(1, 0, 2, 3).reshape(hk, n * group, d), k)
            z = z.mul_(scale).view(hk, n, group, length)
            z = z.masked_fill_(~seen[:, :, None, :], float("-inf"))
            z = z.sub_(z.amax(dim=3, keepdim=True)).exp_()
            z = z.div_(z.sum(dim=3, keepdim=True)).view(hk, n * group, length)
            got = torch.matmul(z, v).view(hk, n, group, d).permute(1, 0, 2, 3)
            out[row + at:row + at + n] = got.reshape(n, hk * group, d).to(out.dtype)
        row += new
    return [out, lists] if focused else out


# ---- what is timed --------------------------------------------------------------

def prepare(case, seed):
    x = _inputs(case, seed)
    lengths, news = x["lengths"], x["news"]
    append = case["kind"] == "append"
    had = [max(0, length - new) for length, new in zip(lengths, news)]
    state = dict(case=case, kind=case["kind"], lengths=lengths, news=news, table=x["table"], q=x["q"])
    if append:
        state.update(k=_new_rows(x["k"], lengths, news), v=_new_rows(x["v"], lengths, news))
    if not own:
        state["pool"], state["scales"] = _plain_pool(x, case, had if append else lengths)
        return state
    from paper_2207_10741_amd import attention as A
    cache = A.KVCache(x["pool"], case["kv_heads"], case["dim"], device=DEVICE)
    before = had if append else lengths
    starts = _sums(lengths)
    rows = [torch.cat([t[starts[b]:starts[b] + n] for b, n in enumerate(before)]) for t in (x["k"], x["v"])]
    if rows[0].shape[0]:
        A.kv_append(cache, rows[0], rows[1], x["table"], _int32(before), starts=_int32(_sums(before)), max_new=max(before))
    length = _int32(lengths)
    most = max(max(lengths), 1)
    if append:
        news = [min(length, new) for length, new in zip(lengths, news)]
        touched = [n + h % BLOCK if n else 0 for n, h in zip(news, had)]
        state["calls"] = [A.PreparedAppend(cache, state["k"], state["v"], x["table"], length, starts=_int32(_sums(news)),
                                           max_new=max(news), max_len=most),
                          A.PreparedRead(cache, x["table"], length, starts=_int32(_sums(touched)), tokens=sum(touched),
                                         max_new=max(touched), max_len=most)]
    elif case["kind"] == "attend":
        state["calls"] = [A.PreparedAttention(cache, x["q"], x["table"], length, starts=_int32(_sums(news)), max_new=max(news),
                                              max_len=most, causal=True)]
    else:
        state["calls"] = [A.PreparedFocusedAttention(cache, x["q"], x["table"], length, starts=_int32(_sums(news)), max_new=max(news),
                                                     max_len=most, first=case["first"], last=case["last"], top=case["top"])]
    return state


def run(state):
    if own:
        for call in state["calls"]:
            out = call()
        return list(out) if isinstance(out, tuple) else out
    if state["kind"] == "append":
        return _plain_append(state)
    return _plain_attend(state, state["kind"] == "focused")


def _visible(case):
    """Over all sequences: (pairs of a new token and a token it may attend to, cached tokens, blocks of all new tokens)."""
    pairs = blocks = 0
    lengths, news = _lengths(case)
    for length, new in zip(lengths, news):
        new = min(length, new)
        pairs += new * length - new * (new - 1) // 2
        blocks += sum((length - new + i) // BLOCK + 1 for i in range(new))
    return pairs, sum(length for length, new in zip(lengths, news) if new), blocks


def work(case):
    hk, group, d = case["kv_heads"], case["group"], case["dim"]
    lengths, news = _lengths(case)
    rows = sum(news)
    pairs, cached, blocks = _visible(case)
    if case["kind"] == "append":
        new = sum(min(a, b) for a, b in zip(lengths, news))
        touched = sum(min(a, b) + max(0, a - b) % BLOCK for a, b in zip(lengths, news) if min(a, b))
        # keys and values: 16-bit ones in, codes out, then the touched blocks' codes in and 32-bit values out
        return {"bytes": 2 * hk * d * (2 * new + new + touched + 4 * touched), "flops": 0}
    moved = 2 * rows * hk * group * d * 2
    if case["kind"] == "attend":
        return {"bytes": moved + cached * hk * (2 * d + 8 / BLOCK), "flops": 4.0 * d * hk * group * pairs}
    width = case["first"] + case["last"] + case["top"]
    chosen = tokens = 0
    for length, new in zip(lengths, news):
        new = min(length, new)
        for i in range(new):
            position = length - new + i
            n = min(width, position // BLOCK + 1)
            chosen += n
            tokens += (n - 1) * BLOCK + position % BLOCK + 1 if case["last"] else n * BLOCK
    sketches = cached // BLOCK
    return {"bytes": moved + 4 * rows * hk * width + sketches * hk * (d + 4) + hk * min(cached, chosen * BLOCK) * 2 * d,
            "flops": 4.0 * d * hk * group * tokens + 2.0 * d * hk * blocks}


# ---- the definition in 64 bits ----------------------------------------------------

def _power(e):
    """2^e in 64 bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _pow2_at_least(a, limit, lo, hi):
    """The least 2^e with a <= limit 2^e, e held to [lo, hi], element by element."""
    e = torch.ceil(torch.log2(a.clamp_min(1e-300) / limit)).clamp(lo, hi)
    s = _power(e)
    down = (a <= limit * s / 2) & (e > lo)      # (the logarithm's own rounding)
    s = torch.where(down, s / 2, s)
    up = a > limit * s
    return torch.where(up, s * 2, s)


def _e4m3(x):
    """The nearest value of the 8-bit format (3 bits behind the point, least exponent -6), ties to even."""
    e = torch.floor(torch.log2(x.abs().clamp_min(1e-300))).clamp_min(-6)
    e = torch.where(_power(e) > x.abs(), e - 1, e).clamp_min(-6)
    step = _power(e - 3)
    return torch.round(x / step) * step


def _exact_cached(x, had, new):
    """One sequence's tokens [tokens, heads, dim] -> (codes, scale of every token) after `had` tokens and then `new` more."""
    x = x.double()
    codes, scale = torch.empty_like(x), torch.empty(x.shape[:2], dtype=torch.float64, device=x.device)
    for at in range(0, x.shape[0], BLOCK):
        part = x[at:at + BLOCK]
        before = min(max(had - at, 0), part.shape[0])
        s = None
        if before:
            s = _pow2_at_least(part[:before].abs().amax(dim=(0, 2)), 448, -64, 120)
            kept = _e4m3(part[:before] / s[:, None])
        if before < part.shape[0]:
            more = _pow2_at_least(part[before:].abs().amax(dim=(0, 2)), 448, -64, 120)
            grown = more if s is None else torch.maximum(s, more)
            if before:
                codes[at:at + before] = _e4m3(kept * (s / grown)[:, None])
            codes[at + before:at + BLOCK] = _e4m3(part[before:] / grown[:, None])
            s = grown
        else:
            codes[at:at + BLOCK] = kept
        scale[at:at + BLOCK] = s
    return codes, scale


def _exact_whole(x):
    """The same for all blocks at once, every token new."""
    n = x.shape[0]
    padded = torch.zeros((-(-n // BLOCK) * BLOCK,) + tuple(x.shape[1:]), dtype=torch.float64, device=x.device)
    padded[:n] = x.double()
    padded = padded.view(-1, BLOCK, *x.shape[1:])
    s = _pow2_at_least(padded.abs().amax(dim=(1, 3)), 448, -64, 120)
    codes = _e4m3(padded / s[:, None, :, None])
    return codes.view(-1, *x.shape[1:])[:n], s.repeat_interleave(BLOCK, 0)[:n]


def exact(case, seed):
    x = _inputs(case, seed)
    hk, group, d = case["kv_heads"], case["group"], case["dim"]
    lengths, news = x["lengths"], x["news"]
    starts = _sums(lengths)
    if case["kind"] == "append":
        if case["batch"] * case["length"] > 1 << 16 and case["new"] > 1:
            return None
        out = {"k": [], "v": []}
        for b, (length, new) in enumerate(zip(lengths, news)):
            new = min(length, new)
            if new == 0:
                continue
            had = length - new
            begin = had - had % BLOCK
            for n in "kv":
                codes, s = _exact_cached(x[n][starts[b] + begin:starts[b] + length], had - begin, new)
                out[n].append(codes * s[:, :, None])
        return [torch.cat(out["k"]), torch.cat(out["v"])]
    focused = case["kind"] == "focused"
    if 4 * sum(n * m for n, m in zip(lengths, news)) * hk * group * d > 3e12:
        return None
    out = torch.zeros(x["q"].shape, dtype=torch.float64, device=DEVICE)
    width = case["first"] + case["last"] + case["top"]
    lists = torch.full((out.shape[0], hk, width), -1, dtype=torch.int32, device=DEVICE)
    row = 0
    for b, (length, new) in enumerate(zip(lengths, news)):
        if length == 0 or new == 0:
            row += new
            continue
        position = torch.arange(length - new, length, device=DEVICE)
        token = torch.arange(length, device=DEVICE)
        for h in range(hk):
            kc, ks = _exact_whole(x["k"][starts[b]:starts[b] + length, h:h + 1])
            vc, vs = _exact_whole(x["v"][starts[b]:starts[b] + length, h:h + 1])
            k, v = (kc * ks[:, :, None])[:, 0], (vc * vs[:, :, None])[:, 0]
            q = x["q"][row:row + new, h * group:(h + 1) * group].double()
            if focused:
                full = length // BLOCK
                sums = kc[:full * BLOCK, 0].view(full, BLOCK, d).sum(dim=1)
                w = _pow2_at_least(sums.abs().amax(dim=1), 127, -100, 100)
                sketch = torch.round(sums / w[:, None])
                weight = w / BLOCK * ks[:full * BLOCK:BLOCK, 0]
                unit = _pow2_at_least(q.abs().amax(dim=(1, 2)), 127, -126, 126)
                total = torch.round(q / unit[:, None, None]).sum(dim=1)
                score = torch.zeros((new, -(-length // BLOCK)), dtype=torch.float64, device=DEVICE)
                score[:, :full] = torch.matmul(total, sketch.t().contiguous()) * weight
            step = max(1, (1 << 27) // (group * length))
            for at in range(0, new, step):
                rows = slice(at, min(new, at + step))
                seen = token[None] <= position[rows, None]
                if focused:
                    number = torch.arange(score.shape[1], device=DEVICE)[None]
                    mine = (position[rows] // BLOCK)[:, None]
                    take = ((number < case["first"]) | (number > mine - case["last"])) & (number <= mine)
                    rest = torch.where((number <= mine) & ~take, score[rows], float("-inf"))
                    rank = torch.argsort(torch.argsort(-rest, dim=1, stable=True), dim=1)
                    take = take | ((rank < case["top"]) & (rest > float("-inf")))
                    seen = seen & take[:, token // BLOCK]
                    index = torch.where(take, number, score.shape[1])
                    index = torch.sort(index, dim=1).values[:, :width]
                    lists[row + at:row + at + index.shape[0], h, :index.shape[1]] = torch.where(index < score.shape[1], index, -1).to(torch.int32)
                z = torch.matmul(q[rows].reshape(-1, d), k.t().contiguous()).view(-1, group, length) / math.sqrt(d)
                z = torch.where(seen[:, None], z, float("-inf"))
                p = torch.exp(z - z.amax(dim=2, keepdim=True))
                p = p / p.sum(dim=2, keepdim=True)
                o = torch.matmul(p.view(-1, length), v).view(-1, group, d)
                out[row + at:row + at + o.shape[0], h * group:(h + 1) * group] = o
        row += new
    return [out, lists] if focused else out
