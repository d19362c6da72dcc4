"""The operators around attention whose speed counts: matrix products with what follows them, group norms of feature maps, and the
pages of a key/value cache.

Five kinds of case:

  linear   rows times weights, with bias, activation and residual: the projections before and after attention and the layers between.
           One row is one user's next token, some dozens a batch's, thousands a prompt or a frame's kept positions; with `counted` only
           a share of the rows is there, how many is known on the device alone, and the rows behind them stay as they were
  norm     group norm of channels-last feature maps with an activation; with `kept` a mask keeps that share of the positions, the
           statistics are theirs and the others become zero; with `ragged` the rows of all images lie behind each other, each with its own number
  fork     slots of a batch become copies of other slots, as the beams of a search or the samples of one prompt do: full blocks
           are shared, unfinished ones copied; the unfinished blocks' tokens are read back
  resize   a batch's sequences end (or are cut) and others begin: blocks go back to the pool and are given out again
  compact  the blocks in use move to another, smaller cache, in order; all tokens are read back from there

Cached values are eighths up to 15/8, which the cache holds exactly.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BLOCK = 64
EPS = 1e-5


def _linear(name, rows, k, n, dtype="bf16", out="", bias=True, residual=False, activation="none", counted=0.0):
    return dict(name=name, kind="linear", rows=rows, k=k, n=n, dtype=dtype, out=out or dtype, bias=bias, residual=residual,
                activation=activation, counted=counted)


def _norm(name, images, positions, channels, groups, dtype="bf16", activation="none", kept=0.0, ragged=False):
    return dict(name=name, kind="norm", images=images, positions=positions, channels=channels, groups=groups, dtype=dtype,
                activation=activation, kept=kept, ragged=ragged)


def _pages(name, kind, batch, length, kv_heads, dim, copies=1, spare=8):
    return dict(name=name, kind=kind, batch=batch, length=length, kv_heads=kv_heads, dim=dim, copies=copies, spare=spare)


def listed():
    return [
        # one user's next token through the projection behind attention: the weights' bytes, and latency
        _linear("linear_step_b1", 1, 4096, 4096, residual=True),
        # a batch's next tokens through a wide layer: the weights' bytes
        _linear("linear_step_b64", 64, 4096, 16384, activation="gelu"),
        # a frame's kept positions, 2 of 5 at most there, sizes off every tile and alignment, a 32-bit output
        _linear("linear_rows_odd", 4811, 1001, 515, "f16", "f32", residual=True, activation="silu", counted=0.4),
        # a long prompt's projection: the matrix cores; the largest
        _linear("linear_prompt", 8192, 8192, 8192, residual=True),
        # a small feature map: latency
        _norm("norm_small", 1, 256, 512, 32, activation="silu"),
        # frames of which a mask keeps half
        _norm("norm_frames", 8, 16384, 256, 32, "f16", activation="relu", kept=0.48),
        # large feature maps: memory
        _norm("norm_large", 16, 65536, 128, 32, activation="silu"),
        # 32-bit rows of images of different sizes, an odd number of channels a group
        _norm("norm_ragged_f32", 5, 6000, 60, 4, "f32", activation="gelu", ragged=True),
        # a search with four beams
        _pages("fork_b4", "fork", 4, 1000, 8, 128, copies=4),
        # a batch of 64 prompts, four samples each
        _pages("fork_b256", "fork", 256, 4096, 8, 128, copies=4),
        # of every four sequences one ends and another begins, the others have one more token
        _pages("resize_b256", "resize", 256, 8192, 1, 64),
        # the cache after a busy hour
        _pages("compact", "compact", 24, 8192, 8, 128, spare=1000),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "norm", "norm", "fork", "resize", "compact"])
    if kind == "linear":
        rows = rng.choice([1, _log(rng, 1, 64), _log(rng, 65, 16384), _log(rng, 65, 16384)])
        k, n = _log(rng, 64, 16384), _log(rng, 64, 16384)
        if rng.random() < 0.6:
            k, n = -(-k // 64) * 64, -(-n // 64) * 64
        while rows * k * n > 1 << 39:
            rows = (rows + 1) // 2
        dtype = rng.choice(["bf16", "bf16", "f16"])
        case = _linear("", rows, k, n, dtype, "f32" if rng.random() < 0.2 else dtype, rng.random() < 0.7, rng.random() < 0.5,
                       rng.choice(["none", "none", "relu", "silu", "gelu"]), round(rng.uniform(0.1, 0.9), 2) if rows > 64 and rng.random() < 0.3 else 0.0)
    elif kind == "norm":
        images, positions = _log(rng, 1, 32), _log(rng, 16, 262144)
        channels, groups = rng.choice([(32, 8), (60, 4), (64, 32), (96, 1), (128, 32), (256, 32), (320, 32), (512, 32), (515, 5), (960, 32), (1280, 32)])
        while images * positions * channels > 1 << 27:
            images, positions = max(1, images // 2), positions if images > 1 else positions // 2
        kept, ragged = (round(rng.uniform(0.1, 0.9), 2), False) if rng.random() < 0.4 else (0.0, rng.random() < 0.4)
        case = _norm("", images, positions, channels, groups, rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice(["none", "relu", "silu", "gelu"]),
                     kept, ragged)
    else:
        kv_heads, dim, length = rng.choice([1, 2, 4, 8, 12]), rng.choice([64, 80, 96, 128, 128]), _log(rng, 64, 16384)
        batch, copies = _log(rng, 2, 256), rng.choice([2, 3, 4, 8])
        while batch > 2 and batch * length * kv_heads * dim > 1 << (28 if kind == "compact" else 31):
            batch //= 2
        case = _pages("", kind, batch, length, kv_heads, dim, copies, _log(rng, 4, 1000))
    del case["name"]
    return case


# ---- inputs ---------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _sums(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def _rows_there(case):
    return int(case["rows"] * case["counted"]) if case["counted"] else case["rows"]


def _linear_inputs(case, seed):
    gen, rows, k, n = _generator(seed), case["rows"], case["k"], case["n"]
    dtype = DTYPES[case["dtype"]]
    normal = lambda *shape: torch.randn(shape, generator=gen, device=DEVICE)
    x = normal(rows, k).to(dtype)
    w = normal(n, k).mul_(k ** -0.5).to(dtype)
    bias = normal(n).mul_(0.3) if case["bias"] else None
    residual = normal(rows, n).to(DTYPES[case["out"]]) if case["residual"] else None
    count = _int32([_rows_there(case)]) if case["counted"] else None
    return dict(x=x, w=w, bias=bias, residual=residual, count=count)


def _image_rows(case):
    """The rows of every image; a function of the case alone."""
    if not case["ragged"]:
        return [case["positions"]] * case["images"]
    rng = random.Random(case["images"] * 1000003 + case["positions"])
    return [case["positions"]] + [rng.randint((case["positions"] + 3) // 4, case["positions"]) for _ in range(case["images"] - 1)]


def _norm_inputs(case, seed):
    gen, c = _generator(seed), case["channels"]
    rows = _image_rows(case)
    # a channel's mean and spread are its own, as behind a convolution
    mean = torch.randn((c,), generator=gen, device=DEVICE)
    spread = torch.rand((c,), generator=gen, device=DEVICE).add_(0.3)
    x = torch.empty((sum(rows), c), dtype=DTYPES[case["dtype"]], device=DEVICE)
    step = max(1, (1 << 27) // c)
    for at in range(0, x.shape[0], step):
        part = x[at:at + step]
        part.copy_(torch.randn(part.shape, generator=gen, device=DEVICE).mul_(spread).add_(mean))
    weight = torch.randn((c,), generator=gen, device=DEVICE).mul_(0.2).add_(1.0)
    bias = torch.randn((c,), generator=gen, device=DEVICE).mul_(0.3)
    mask = None
    if case["kept"]:        # runs of positions, as an object's lines in an image
        run = 16
        mask = torch.rand((case["images"], -(-case["positions"] // run)), generator=gen, device=DEVICE) < case["kept"]
        mask = mask.repeat_interleave(run, 1)[:, :case["positions"]].to(torch.uint8).contiguous()
    if not case["ragged"]:
        x = x.view(case["images"], case["positions"], c)
    return dict(x=x, weight=weight, bias=bias, mask=mask, starts=_int32(_sums(rows)) if case["ragged"] else None)


def _lengths(case):
    """Tokens of the sequences of a case about pages; a function of the case alone."""
    rng = random.Random(case["batch"] * 1000003 + case["length"])
    return [case["length"]] + [rng.randint((case["length"] + 3) // 4, case["length"]) for _ in range(case["batch"] - 1)]


def _blocks(lengths):
    return [-(-n // BLOCK) for n in lengths]


def _table(blocks, width, order):
    """Sequences' blocks, taken from `order` in turn; -1 behind them."""
    table = torch.full((len(blocks), width), -1, dtype=torch.int32, device=DEVICE)
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = order[at:at + n]
        at += n
    return table


def _pages_inputs(case, seed):
    """The pages before the call: the sequences' tokens (eighths), their lengths, blocks in the pool and what the call is given."""
    gen, kind, batch = _generator(seed), case["kind"], case["batch"]
    lengths = _lengths(case)
    x = dict(kind=kind)
    if kind == "fork":          # every copies-th slot has a sequence, the slots behind it are free and become its copies
        parents = [b - b % case["copies"] for b in range(batch)]
        lengths = [n if parents[b] == b else 0 for b, n in enumerate(lengths)]
        more = batch
        x["parents"] = _int32(parents)
        x["after"] = [lengths[p] for p in parents]
        x["read"] = [n % BLOCK for n in x["after"]]
    elif kind == "resize":      # the call: sequences end, then others begin
        before, after = list(lengths), list(lengths)
        for b in range(batch):
            if b % 4 == 0:
                before[b] = 0
            elif b % 4 == 1:
                after[b] = before[b] // 2
            else:
                after[b] = min(before[b] + 1, case["length"])
        x["steps"] = [_int32(before), _int32(after)]
        lengths, more = after, sum(max(p, q) - q for p, q in zip(_blocks(before), _blocks(after)))
    else:
        more = 0
        x["after"] = x["read"] = lengths
    blocks = _blocks(lengths)
    pool = sum(blocks) + more + case["spare"]
    order = torch.randperm(pool, generator=gen, device=DEVICE).to(torch.int32)
    x.update(pool=pool, to_pool=sum(blocks) + 1, lengths=lengths, table=_table(blocks, max(_blocks([case["length"]])) + 1, order))
    x["users"] = torch.zeros((pool,), dtype=torch.int32, device=DEVICE)
    x["users"][order[:sum(blocks)].long()] = 1
    if kind != "resize":
        shape = (sum(lengths), case["kv_heads"], case["dim"])
        x["k"], x["v"] = (torch.randint(-15, 16, shape, generator=gen, device=DEVICE, dtype=torch.int8).to(torch.bfloat16).mul_(0.125) for _ in "kv")
    return x


# ---- the plain form ---------------------------------------------------------------

def _activate(y, activation):
    if activation == "relu":
        return torch.where(y < 0, 0.0, y)
    if activation == "silu":
        return y / (1.0 + torch.exp(-y))
    if activation == "gelu":
        return 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    return y


def _plain_linear(state):
    case = state["case"]
    y = torch.matmul(state["x"].float(), state["w"].float().t())
    if state["bias"] is not None:
        y = y + state["bias"]
    y = _activate(y, case["activation"])
    if state["residual"] is not None:
        y = y + state["residual"].float()
    y = y.to(DTYPES[case["out"]])
    if state["count"] is not None:
        there = torch.arange(y.shape[0], device=DEVICE)[:, None] < state["count"]
        y = torch.where(there, y, state["out"])
    return y


def _plain_norm(state):
    """Sums over images of different sizes by the rows' image numbers; over images of one size directly."""
    case, x = state["case"], state["x"].float()
    c, groups = case["channels"], case["groups"]
    if case["ragged"]:
        image = torch.searchsorted(state["starts"][1:].contiguous(), torch.arange(x.shape[0], dtype=torch.int32, device=DEVICE), right=True)
        n = (state["starts"][1:] - state["starts"][:-1]).float()[:, None, None] * (c // groups)
        x = x.view(-1, groups, c // groups)
        zero = torch.zeros((case["images"], groups, 1), device=DEVICE)
        mean = zero.index_add(0, image, x.sum(dim=2, keepdim=True)) / n
        x = x - mean[image]
        var = zero.index_add(0, image, x.square().sum(dim=2, keepdim=True)) / n
        y = x * torch.rsqrt(var + EPS)[image]
    else:
        x = x.view(case["images"], -1, groups, c // groups)
        n = float(case["positions"] * (c // groups))
        if state["mask"] is not None:
            seen = (state["mask"] != 0)[:, :, None, None]
            n = seen.sum(dim=1, keepdim=True).float().clamp_min(1.0) * (c // groups)
            x = torch.where(seen, x, 0.0)
        x = x - x.sum(dim=(1, 3), keepdim=True) / n
        if state["mask"] is not None:
            x = torch.where(seen, x, 0.0)
        y = x * torch.rsqrt(x.square().sum(dim=(1, 3), keepdim=True) / n + EPS)
    y = y * state["weight"].view(groups, -1) + state["bias"].view(groups, -1)
    y = _activate(y, case["activation"])
    if state["mask"] is not None:
        y = torch.where(seen, y, 0.0)
    return y.reshape(state["x"].shape).to(state["x"].dtype)


def _uses(users, entries, by):
    """users, with `by` more for every entry that is a block."""
    there = entries >= 0
    return users.index_add(0, entries.clamp_min(0).flatten().long(), (there * by).flatten().to(torch.int32))


def _give(users, wanted):
    """(blocks for the wanted places in their order, the lowest free ones, -1 where none is left; users with them)"""
    order = torch.sort((users != 0).to(torch.uint8), stable=True).indices
    rank = torch.cumsum(wanted.flatten(), 0) - 1
    given = order[rank.clamp(0, users.shape[0] - 1)]
    left = (users == 0).sum()
    given = torch.where(wanted.flatten() & (rank < left), given, -1).view(wanted.shape).to(torch.int32)
    return given, _uses(users, given, 1)


def _plain_resize(state):
    missing = None
    for lengths in state["steps"]:
        table, users = state["table"], state["users"]
        need = (lengths + BLOCK - 1) // BLOCK
        inside = torch.arange(table.shape[1], device=DEVICE) < need[:, None]
        users = _uses(users, torch.where(inside, -1, table), -1)
        table = torch.where(inside, table, -1)
        wanted = inside & (table < 0)
        given, users = _give(users, wanted)
        table = torch.where(wanted, given, table)
        missing = (wanted & (given < 0)).sum().to(torch.int32).view(1)
        state["table"], state["users"] = table, users
    return [state["table"], state["users"], missing]


def _read(state, table):
    """The tokens that are read back, of all sequences one after another."""
    at = table[state["slot"], state["place"] // BLOCK].long()
    return [state["pool"][n].view(torch.uint8)[at, state["place"] % BLOCK].view(torch.float8_e4m3fn).float() for n in "kv"]


def _plain_fork(state):
    table, users, lengths, parents = state["table"], state["users"], state["lengths"], state["parents"].long()
    slot = torch.arange(parents.shape[0], device=DEVICE)
    stays = parents == slot
    length = lengths[parents]
    need = (length + BLOCK - 1) // BLOCK
    rows = torch.where(torch.arange(table.shape[1], device=DEVICE) < need[:, None], table[parents], -1)
    # an unfinished last block stays with the parent's slot or goes to the lowest of its copies; the others get one of their own
    first = torch.full_like(parents, parents.shape[0]).scatter_reduce(0, parents, torch.where(stays, -1, slot), "amin")
    last = (need - 1).clamp_min(0)[:, None].long()
    from_block = rows.gather(1, last)[:, 0]
    copied = (length % BLOCK != 0) & (first[parents] != torch.where(stays, -1, slot)) & (from_block >= 0)
    shared = rows.scatter(1, last, torch.where(copied, -1, from_block)[:, None])
    users = _uses(users, torch.where(stays[:, None], -1, table), -1)
    users = _uses(users, torch.where(stays[:, None], -1, shared), 1)
    given, users = _give(users, copied)
    rows = torch.where(stays[:, None], table, rows.scatter(1, last, torch.where(copied, given, from_block)[:, None]))
    source = from_block.clamp_min(0).long()
    target = torch.where(copied & (given >= 0), given.long(), source)
    for n in "kv":
        bytes_ = state["pool"][n].view(torch.uint8)
        bytes_[target] = bytes_[source]
    state["table"], state["users"], state["lengths"] = rows, users, length
    return [rows, users, length] + _read(state, rows)


def _plain_compact(state):
    used = state["users"] > 0
    number = torch.where(used, torch.cumsum(used, 0) - 1, -1).to(torch.int32)
    table = torch.where(state["table"] >= 0, number[state["table"].clamp_min(0).long()], -1)
    order = torch.sort((~used).to(torch.uint8), stable=True).indices[:state["to_pool"]]
    there = used[order]
    users = torch.where(there, state["users"][order], 0)
    moved = {n: state["pool"][n].view(torch.uint8)[order].view(torch.float8_e4m3fn) for n in "kv"}
    return [table, users] + _read({**state, "pool": moved}, table)


# ---- what is timed ----------------------------------------------------------------

def _read_places(x):
    """(slot, place) of every token that is read back: the last ones of every sequence."""
    slot = torch.repeat_interleave(torch.arange(len(x["read"]), device=DEVICE), torch.tensor(x["read"], device=DEVICE))
    first = torch.tensor([a - r for a, r in zip(x["after"], x["read"])], device=DEVICE) - torch.tensor(_sums(x["read"])[:-1], device=DEVICE)
    return slot, torch.arange(slot.shape[0], device=DEVICE) + first[slot]


def _prepare_pages(case, seed):
    x = _pages_inputs(case, seed)
    state = dict(case=case, kind=x["kind"], table=x["table"], users=x["users"], lengths=_int32(x["lengths"]))
    if not own:
        state.update({n: x[n] for n in ("parents", "steps", "to_pool") if n in x})
        if x["kind"] != "resize":
            state["slot"], state["place"] = _read_places(x)
            state["pool"] = {n: torch.zeros((x["pool"], BLOCK, case["kv_heads"], case["dim"]), dtype=torch.float8_e4m3fn, device=DEVICE) for n in "kv"}
            at = _sums(x["lengths"])
            for b, n in enumerate(x["lengths"]):
                place = torch.arange(n, device=DEVICE)
                block = x["table"][b, place // BLOCK].long()
                for name in "kv":
                    codes = x[name][at[b]:at[b + 1]].to(torch.float8_e4m3fn).view(torch.uint8)
                    state["pool"][name].view(torch.uint8)[block, place % BLOCK] = codes
        return state
    from paper_2207_10741_amd import attention as A, pages as P
    cache = A.KVCache(x["pool"], case["kv_heads"], case["dim"], device=DEVICE)
    if x["kind"] == "resize":
        state["calls"] = [P.PreparedResize(cache, state["users"], state["table"], lengths) for lengths in x["steps"]]
        state["outputs"] = lambda got: [state["table"], state["users"], got]
        return state
    A.kv_append(cache, x["k"], x["v"], state["table"], state["lengths"], starts=_int32(_sums(x["lengths"])), max_new=max(x["lengths"]))
    table = state["table"]
    if x["kind"] == "fork":
        state["calls"] = [P.PreparedFork(cache, state["users"], table, state["lengths"], x["parents"])]
        state["outputs"] = lambda got: [state["table"], state["users"], state["lengths"], got[0], got[1]]
    else:
        cache_to = A.KVCache(x["to_pool"], case["kv_heads"], case["dim"], device=DEVICE)
        users, table = torch.zeros((x["to_pool"],), dtype=torch.int32, device=DEVICE), torch.empty_like(table)
        state["calls"] = [P.PreparedCompact(cache, state["users"], state["table"], cache_to, users, table)]
        state["outputs"] = lambda got: [table, users, got[0], got[1]]
        cache = cache_to
    if sum(x["read"]):
        state["calls"].append(A.PreparedRead(cache, table, state["lengths"], starts=_int32(_sums(x["read"])), tokens=sum(x["read"]),
                                             max_new=max(x["read"]), max_len=max(x["after"])))
    else:
        nothing = torch.empty((0, case["kv_heads"], case["dim"]), device=DEVICE)
        state["calls"].append(lambda: (nothing, nothing))
    return state


def prepare(case, seed):
    if case["kind"] not in ("linear", "norm"):
        return _prepare_pages(case, seed)
    state = _linear_inputs(case, seed) if case["kind"] == "linear" else _norm_inputs(case, seed)
    state.update(case=case, kind=case["kind"])
    if case["kind"] == "linear":
        state["out"] = torch.zeros((case["rows"], case["n"]), dtype=DTYPES[case["out"]], device=DEVICE)
    if not own:
        return state
    from paper_2207_10741_amd import layers as L
    if case["kind"] == "linear":
        call = L.PreparedLinear(state["x"], state["w"], state["bias"], residual=state["residual"], activation=case["activation"],
                                count=state["count"], out=state["out"])
    else:
        call = L.PreparedGroupNorm(state["x"], case["groups"], state["weight"], state["bias"], mask=state["mask"], starts=state["starts"],
                                   max_rows=case["positions"], eps=EPS, activation=case["activation"])
    state.update(calls=[call], outputs=lambda got: got)
    return state


def run(state):
    if own:
        for call in state["calls"]:
            got = call()
        return state["outputs"](got)
    return {"linear": _plain_linear, "norm": _plain_norm, "fork": _plain_fork, "resize": _plain_resize, "compact": _plain_compact}[state["kind"]](state)


def work(case):
    if case["kind"] == "linear":
        rows, k, n, out = _rows_there(case), case["k"], case["n"], DTYPES[case["out"]].itemsize
        return {"bytes": 2 * (rows * k + n * k) + 4 * n * case["bias"] + rows * n * out * (1 + case["residual"]), "flops": 2.0 * rows * k * n}
    if case["kind"] == "norm":
        positions, size = sum(_image_rows(case)), case["channels"] * DTYPES[case["dtype"]].itemsize
        seen = case["kept"] or 1.0
        return {"bytes": positions * size * (1 + seen) + (positions if case["kept"] else 0) + 8 * case["channels"], "flops": 0}
    kept = _lengths(case)
    token, block = 2 * case["kv_heads"] * case["dim"], 2 * BLOCK * case["kv_heads"] * case["dim"]
    entries = 4 * case["batch"] * (-(-case["length"] // BLOCK) + 1)
    if case["kind"] == "resize":
        return {"bytes": 4 * entries, "flops": 0}
    if case["kind"] == "fork":
        after = [kept[b - b % case["copies"]] for b in range(case["batch"])]
        copies = sum(1 for b, n in enumerate(after) if b % case["copies"] and n % BLOCK)
        return {"bytes": 2 * entries + 2 * copies * block + 5 * token * sum(n % BLOCK for n in after), "flops": 0}
    return {"bytes": 2 * entries + 2 * sum(_blocks(kept)) * block + 5 * token * sum(kept), "flops": 0}


# ---- the definition in 64 bits ------------------------------------------------------

def _activated(y, activation):
    if activation == "relu":
        return y.clamp_min(0.0)
    if activation == "silu":
        return y * torch.sigmoid(y)
    if activation == "gelu":
        return y * (0.5 * torch.erfc(-y / math.sqrt(2.0)))
    return y


def exact(case, seed):
    if case["kind"] == "linear":
        x = _linear_inputs(case, seed)
        there = _rows_there(case)
        out = torch.zeros((case["rows"], case["n"]), dtype=torch.float64, device=DEVICE)
        w = x["w"].double().t().contiguous()
        for at in range(0, there, 4096):
            rows = slice(at, min(there, at + 4096))
            y = x["x"][rows].double() @ w
            if case["bias"]:
                y += x["bias"].double()
            y = _activated(y, case["activation"])
            out[rows] = y if x["residual"] is None else y + x["residual"][rows].double()
        return out
    if case["kind"] == "norm":
        x = _norm_inputs(case, seed)
        rows, c = x["x"].view(-1, case["channels"]), case["channels"]
        out = torch.zeros(rows.shape, dtype=torch.float64, device=DEVICE)
        at = 0
        for b, n in enumerate(_image_rows(case)):
            keep = torch.arange(n, device=DEVICE) if x["mask"] is None else torch.nonzero(x["mask"][b])[:, 0]
            if keep.numel():
                part = rows[at:at + n][keep].double().view(-1, case["groups"], c // case["groups"]).transpose(0, 1)
                spread, mean = torch.var_mean(part, dim=(1, 2), correction=0, keepdim=True)
                y = ((part - mean) / torch.sqrt(spread + EPS)).transpose(0, 1).reshape(-1, c) * x["weight"].double() + x["bias"].double()
                out[at + keep] = _activated(y, case["activation"])
            at += n
        return out.view(x["x"].shape)
    if case["kind"] == "resize":
        return None
    # what is read back is what was cached: the last tokens of every slot's sequence
    x = _pages_inputs(case, seed)
    parents = x["parents"].tolist() if case["kind"] == "fork" else range(case["batch"])
    ends = _sums(x["lengths"])[1:]
    values = [torch.cat([x[n][ends[p] - x["read"][b]:ends[p]] for b, p in enumerate(parents)]).double() for n in "kv"]
    return [None] * (3 if case["kind"] == "fork" else 2) + values
