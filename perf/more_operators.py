"""Performance cases of the operators for long-lived serving caches: 8-bit pages, a sliding window, forks.

Three operators, used together by a serving loop whose sequences are long or branch:

  append     queries and keys of a step's tokens are normalised per head (optional) and rotated; keys and values go to an
             8-bit paged cache: e4m3 codes with one power of two for every 16 positions of a head
  attention  every query row attends to its own sequence's positions (and the prefix before them), to all of them or to
             a window of the latest and a few first ones, over 16-bit or 8-bit pages
  fork       a new batch whose rows continue rows of the old one: full pages are shared and counted, the partly filled
             last page is copied in every layer's cache, pages without a reader are given back

The head layouts are those of this repository's model shapes (16 heads of 128, 55 heads of 96, 4 heads of 64), and
generic ones with shared key/value heads.  A case's lengths come from the case itself (`ragged` seeds them); the seed of
`prepare` decides every value.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
CODE, SCALE = torch.float8_e4m3fn, torch.float8_e8m0fnu
BLOCK = 16                                  # positions that share a scale
LEAST = -64                                 # the smallest exponent of a scale


def _append(name, seqs, new, context, prefix, heads, kv_heads, head_dim, rot, page, dtype, norm, ragged):
    return dict(name=name, op="append", seqs=seqs, new=new, context=context, prefix=prefix, heads=heads,
                kv_heads=kv_heads, head_dim=head_dim, rot=rot, page=page, dtype=dtype, norm=norm, ragged=ragged)


def _attention(name, seqs, new, context, prefix, window, sinks, heads, kv_heads, head_dim, page, dtype, eight, ragged):
    return dict(name=name, op="attention", seqs=seqs, new=new, context=context, prefix=prefix, window=window,
                sinks=sinks, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, dtype=dtype, eight=eight,
                ragged=ragged)


def _fork(name, seqs, children, context, window, sinks, layers, kv_heads, head_dim, page, dtype, eight, ragged):
    return dict(name=name, op="fork", seqs=seqs, children=children, context=context, window=window, sinks=sinks,
                layers=layers, kv_heads=kv_heads, head_dim=head_dim, page=page, dtype=dtype, eight=eight, ragged=ragged)


def listed():
    return [
        # one token of one sequence, the Ouro head shape: nothing but latency
        _append("append8_decode_1", 1, 1, 700, 0, 16, 16, 128, 128, 16, "f16", False, 1),
        # a decode step of a large batch behind a long prefix, shared key/value heads, norms of queries and keys
        _append("append8_decode_96", 96, 1, 2000, 20000, 32, 8, 128, 128, 32, "bf16", True, 2),
        # ragged prompts of a few sequences, the Raven head shape
        _append("append8_prompts_raven", 5, 900, 300, 1000, 55, 55, 96, 96, 16, "f16", False, 3),
        # one long prompt, half of each head rotated, seven query heads to a key/value head
        _append("append8_prompt_long", 1, 16001, 0, 0, 28, 4, 128, 64, 64, "bf16", True, 4),
        # three sequences and a short window, the tiny decoder's heads: latency
        _attention("window_few", 3, 1, 600, 0, 128, 4, 4, 4, 64, 16, "f16", False, 5),
        # a decode step of a batch over a window of long histories, four query heads to a key/value head
        _attention("window_decode_64", 64, 1, 12000, 0, 4096, 4, 32, 8, 128, 32, "bf16", False, 6),
        # one long prompt under a window, seven query heads to a key/value head: the matrix cores are the bound
        _attention("window_prompt", 1, 8001, 0, 0, 2048, 16, 28, 4, 128, 64, "bf16", False, 7),
        # an ordinary decode step over 8-bit pages, the Ouro head shape
        _attention("quantized_ouro_32", 32, 1, 8192, 0, 0, 0, 16, 16, 128, 16, "f16", True, 8),
        # several rows in flight per sequence (drafts to be verified) behind a prefix that all share, 8-bit pages
        _attention("quantized_prefix_128", 128, 3, 256, 8007, 0, 0, 32, 8, 128, 32, "bf16", True, 9),
        # ragged prompts of a few sequences over their histories, the Raven head shape, 8-bit pages
        _attention("quantized_prompts_raven", 5, 900, 1000, 0, 0, 0, 55, 55, 96, 16, "f16", True, 10),
        # two drafts of each of a few sequences, two layers: latency
        _fork("fork_drafts", 4, 8, 700, 0, 0, 2, 16, 128, 16, "f16", False, 11),
        # a beam search's step: a large batch resampled from its own rows, 8-bit pages of several layers
        _fork("fork_beams", 192, 192, 1000, 512, 16, 6, 8, 128, 64, "bf16", True, 12),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "fork"])
    largest = [work(c) for c in listed() if c["op"] == op]
    limit = {k: max(w[k] for w in largest) for k in ("bytes", "flops")}
    heads, kv_heads, head_dim = rng.choice(
        [(16, 16, 128), (55, 55, 96), (4, 4, 64), (32, 8, 128), (28, 4, 128), (32, 4, 64), (5, 1, 128), (8, 8, 32)])
    page, dtype, ragged = rng.choice([16, 32, 48, 64, 128]), rng.choice(["f16", "bf16"]), rng.randrange(1 << 30)
    window, sinks = rng.choice([0, _spread(rng, 60, 5000)]), rng.choice([0, 4, _spread(rng, 1, 100)])
    eight = rng.random() < 0.6
    prompt = rng.random() < 0.4
    if op == "append":
        case = _append("", _spread(rng, 1, 6 if prompt else 192), _spread(rng, 2, 5000) if prompt else 1,
                       _spread(rng, 1, 2000), rng.choice([0, _spread(rng, 16, 40000)]), heads, kv_heads, head_dim,
                       rng.choice([head_dim, head_dim // 2]), page, dtype, rng.random() < 0.5, ragged)
        shrink = ["new", "seqs"]
    elif op == "attention":
        case = _attention("", _spread(rng, 1, 6 if prompt else 128), _spread(rng, 10, 3000) if prompt
                          else rng.choice([1, 1, 3, 9]), _spread(rng, 1, 10000), rng.choice([0, 0, _spread(rng, 16, 8000)]),
                          window, sinks, heads, kv_heads, head_dim, page, dtype, eight, ragged)
        shrink = ["context", "prefix", "seqs", "new"]
    else:
        case = _fork("", _spread(rng, 1, 192), _spread(rng, 1, 192), _spread(rng, 1, 2000), window, sinks,
                     rng.randint(1, 6), kv_heads, head_dim, page, dtype, eight, ragged)
        shrink = ["context", "children", "seqs"]

    def too_much():
        if any(work(case)[k] > limit[k] for k in limit):
            return True
        # the plain form's own intermediates: keys per sequence and scores
        if op != "attention":
            return op == "fork" and 6 * case["layers"] * kv_heads * head_dim * case["seqs"] * (case["context"] + 128) > 6e9
        _, lens = _lengths(case)
        most = case["prefix"] + max(lens)
        return case["seqs"] * most * head_dim * kv_heads > 1.2e9 or case["seqs"] * case["new"] * heads * most > 2e9
    while too_much():
        for key in list(shrink):
            if case[key] > 8 or (len(shrink) == 1 and case[key] > 1):
                case[key] = case[key] * 3 // 4
            elif len(shrink) > 1:
                shrink.remove(key)
    del case["name"]
    return case


def _lengths(case):
    """(tokens of this step, positions with them) of every sequence."""
    r = random.Random(case["ragged"])
    new = [case["new"] if i == 0 else r.randint(max(1, case["new"] // 4), case["new"]) for i in range(case["seqs"])]
    return new, [n + (case["context"] if i == 0 else r.randint(0, case["context"])) for i, n in enumerate(new)]


def _branches(case):
    """Positions of every sequence and the parent of every child (-1: a row without a sequence; the first has one)."""
    r = random.Random(case["ragged"])
    lens = [max(1, case["context"] if i == 0 else r.randint(0, case["context"])) for i in range(case["seqs"])]
    return lens, [r.randrange(case["seqs"]) if i == 0 or r.random() < 0.95 else -1 for i in range(case["children"])]


def _seen(case, n, length):
    """Positions seen by the n tokens of a sequence (each summed over, and how many distinct ones)."""
    at = np.arange(case["prefix"] + length - n, case["prefix"] + length)
    if not case["window"]:
        return int((at + 1).sum()), int(at[-1]) + 1
    start = np.maximum(0, at - case["window"] + 1)
    first = np.minimum(case["sinks"], start)
    return int((at - start + 1 + first).sum()), int(at[-1] - start[0] + 1 + min(case["sinks"], start[0]))


def work(case):
    if case["op"] == "fork":
        lens, parent = _branches(case)
        heirs, tails = set(), 0
        for p in parent:
            if p in heirs:
                tails += lens[p] % case["page"]
            elif p >= 0:
                heirs.add(p)
        width = -(-max(lens) // case["page"])
        per = 2 * case["layers"] * case["kv_heads"] * case["head_dim"] * (1 if case["eight"] else 2)
        return {"bytes": 2 * tails * per + 4 * width * (case["seqs"] + case["children"])
                + 8 * (sum(-(-n // case["page"]) for n in lens) + case["children"]), "flops": 0}
    H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
    new, lens = _lengths(case)
    T = sum(new)
    if case["op"] == "append":
        return {"bytes": 4 * T * H * D + 6 * T * G * D, "flops": T * (H + G) * (3 * case["rot"] + (4 * D if case["norm"] else 0))}
    seen = [_seen(case, n, length) for n, length in zip(new, lens)]
    # positions of the prefix count once for all sequences
    distinct = sum(d for _, d in seen) if case["window"] else case["prefix"] + sum(lens)
    return {"bytes": 2 * distinct * G * D * (1 if case["eight"] else 2) + 4 * T * H * D + 4 * T * H,
            "flops": 4 * H * D * sum(s for s, _ in seen)}


# ---------------------------------------------------------------------------------------------------------------------
# what a program has in hand before the call
# ---------------------------------------------------------------------------------------------------------------------
def _pages(gen, case, n_pages, G, D):
    """Keys or values [n_pages, G, page, D] of a cache in use, and the scales of 8-bit ones."""
    x = torch.randn((n_pages, G, case["page"], D), generator=gen, device=DEV)
    if not case.get("eight", True):
        return x.to(TYPES[case["dtype"]]), None
    x *= torch.exp(0.5 * torch.randn((n_pages, G, 1, 1), generator=gen, device=DEV))
    x = x.view(n_pages, G, -1, BLOCK, D)
    e = _exponent(x.abs().amax((3, 4)))
    codes = (x * torch.exp2(-e.float())[..., None, None]).to(CODE).view(n_pages, G, case["page"], D)
    return codes, (e + 127).to(torch.uint8).view(SCALE)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    host = random.Random(seed)
    G, D, page = case["kv_heads"], case["head_dim"], case["page"]
    if case["op"] == "fork":
        return _prepare_fork(case, gen, host)
    H, dtype = case["heads"], TYPES[case["dtype"]]
    new, lens = _lengths(case)
    T = sum(new)
    n_prefix = -(-case["prefix"] // page) * (case["op"] == "attention")
    n_own = [-(-L // page) for L in lens]
    pages = list(range(n_prefix + sum(n_own) + 3))
    n_pages = len(pages)
    host.shuffle(pages)
    prefix_table = [pages.pop() for _ in range(n_prefix)]
    table = np.zeros((len(new), max(n_own)), np.int32)
    for b, n in enumerate(n_own):
        table[b, :n] = [pages.pop() for _ in range(n)]
    k_cache, k_scale = _pages(gen, case, n_pages, G, D)
    v_cache, v_scale = _pages(gen, case, n_pages, G, D)
    qkv = torch.randn((T, (H + 2 * G) * D), generator=gen, device=DEV).to(dtype)
    state = dict(case=case, k_cache=k_cache, v_cache=v_cache, k_scale=k_scale, v_scale=v_scale, new=new, lens=lens,
                 q=qkv[:, :H * D].view(T, H, D), k=qkv[:, H * D:(H + G) * D].view(T, G, D),
                 v=qkv[:, (H + G) * D:].view(T, G, D),
                 table=torch.from_numpy(table).to(DEV), seq_len=torch.tensor(lens, dtype=torch.int32, device=DEV),
                 q_start=torch.tensor(np.cumsum([0] + new), dtype=torch.int32, device=DEV),
                 prefix_table=torch.tensor(prefix_table, dtype=torch.int32, device=DEV),
                 freq=1e4 ** (-torch.arange(case.get("rot", 0) // 2, dtype=torch.float64, device=DEV)
                              * 2 / max(1, case.get("rot", 0))))
    if case["op"] == "attention":
        state["q"] = state["q"] * 1.5       # scores with a standard deviation of about 1.5
    elif case["norm"]:
        state["q_gain"], state["k_gain"] = (1 + 0.2 * torch.randn(D, generator=gen, device=DEV) for _ in range(2))
    if own:
        from paper_2609_17184_amd import serving
        state["cache"] = _cache(state["k_cache"], state["v_cache"], k_scale, v_scale)
        state["batch"] = serving.Batch(
            state["seq_len"], state["table"], q_start=state["q_start"] if case["new"] > 1 else None,
            prefix_len=case["prefix"], prefix_table=state["prefix_table"] if n_prefix else None)
    return state


def _cache(k, v, k_scale, v_scale):
    from paper_2609_17184_amd import serving
    return serving.PagedCache(k, v) if k_scale is None else serving.QuantizedCache(k, v, k_scale, v_scale)


def _prepare_fork(case, gen, host):
    lens, parent = _branches(case)
    page = case["page"]
    n_own = [-(-L // page) for L in lens]
    n_pages = sum(n_own) + case["children"] + 5
    pages = list(range(n_pages))
    host.shuffle(pages)
    table = np.full((len(lens), max(n_own)), -1, np.int32)
    for b, n in enumerate(n_own):
        table[b, :n] = [pages.pop() for _ in range(n)]
        # earlier forks: first full pages in common with the sequence before
        shared = min(host.choice([0, 0, 1, 2]), lens[b] // page, lens[b - 1] // page) if b else 0
        table[b, :shared] = table[b - 1, :shared]
    refs = np.bincount(table[table >= 0], minlength=n_pages).astype(np.int32)
    layers = [_pages(gen, case, n_pages, case["kv_heads"], case["head_dim"])
              + _pages(gen, case, n_pages, case["kv_heads"], case["head_dim"]) for _ in range(case["layers"])]
    layers = [(k, v, ks, vs) for k, ks, v, vs in layers]
    state = dict(case=case, layers=layers, lens=lens, table=torch.from_numpy(table).to(DEV),
                 refs=torch.from_numpy(refs).to(DEV), seq_len=torch.tensor(lens, dtype=torch.int32, device=DEV),
                 parent=torch.tensor(parent, dtype=torch.int32, device=DEV))
    if own:
        state["caches"] = [_cache(*x) for x in layers]
    return state


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(state):
    return {"append": _run_append, "attention": _run_attention, "fork": _run_fork}[state["case"]["op"]](state)


def _exponent(amax):
    """The smallest e from LEAST on with amax <= 448 * 2^e."""
    m, e = torch.frexp(amax)
    return torch.where(amax > 0, e - 9 + (m > 0.875), LEAST).clamp(min=LEAST).int()


def _power(e):
    return torch.ldexp(torch.ones((), device=DEV), e)


def _places(state):
    """Sequence and own position of every token."""
    start = state["q_start"].long()
    n = start[1:] - start[:-1]
    seq = torch.repeat_interleave(torch.arange(len(n), device=DEV), n, output_size=len(state["q"]))
    place = state["seq_len"].long()[seq] - n[seq] + torch.arange(len(seq), device=DEV) - start[seq]
    return seq, place


def _run_append(state):
    case = state["case"]
    if own:
        from paper_2609_17184_amd import serving
        q = serving.rope_append(state["q"], state["k"], state["v"], state["cache"], state["batch"], state["freq"],
                                q_norm=state.get("q_gain"), k_norm=state.get("k_gain"), eps=1e-6)
        return [q] + [state[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")]
    seq, place = _places(state)
    page_size, half = case["page"], case["rot"] // 2
    angle = (place + case["prefix"])[:, None].double() * state["freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def rotated(x, gain):
        x = x.float()
        if gain is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gain
        a, b = x[..., :half], x[..., half:2 * half]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]], -1)
    page = state["table"].long()[seq, place // page_size]
    # the blocks that hold positions from before this step: those of the sequences' first tokens
    first = state["q_start"].long()[:-1]
    kept, at = place[first] % BLOCK, page[first]
    line = (place[first] % page_size // BLOCK * BLOCK)[:, None] + torch.arange(BLOCK, device=DEV)
    old = torch.arange(BLOCK, device=DEV) < kept[:, None]
    _append8(state["k_cache"], state["k_scale"], rotated(state["k"], state.get("k_gain")), page, place % page_size, first, at, line, old)
    _append8(state["v_cache"], state["v_scale"], state["v"].float(), page, place % page_size, first, at, line, old)
    return [rotated(state["q"], state.get("q_gain")).to(state["q"].dtype)] + [
        state[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")]


def _append8(codes, scale, x, page, offset, first, at, line, old):
    """Rows x [T, G, D] to (page, offset); `old` marks the places of blocks (at, line) that keep their positions."""
    bits, exponents = codes.view(torch.uint8), scale.view(torch.uint8)
    n_pages, G, units = exponents.shape
    block = page * units + offset // BLOCK
    amax = torch.zeros((n_pages * units, G), device=DEV).scatter_reduce_(0, block[:, None].expand(-1, G), x.abs().amax(-1), "amax")
    e = _exponent(amax)[block]
    # a block that keeps positions keeps at least their scale
    before = exponents[at, :, offset[first] // BLOCK].int() - 127
    floor = torch.full((n_pages * units, G), LEAST, dtype=torch.int32, device=DEV)
    floor[block[first]] = torch.where(old[:, :1], before, LEAST)
    e = torch.maximum(e, floor[block])
    lines = bits[at[:, None], :, line].view(CODE).float()
    again = (lines * _power(before - e[first])[:, None, :, None]).to(CODE).view(torch.uint8)
    bits[at[:, None], :, line] = torch.where(old[..., None, None], again, bits[at[:, None], :, line])
    bits[page, :, offset] = (x * _power(-e)[..., None]).to(CODE).view(torch.uint8)
    exponents[page, :, offset // BLOCK] = (e + 127).to(torch.uint8)


def _history(state):
    """Pages [B, J] and offsets [B, J] of all positions of all sequences (any page behind a sequence's last), and which
    are theirs."""
    case = state["case"]
    j = torch.arange(case["prefix"] + max(state["lens"]), device=DEV)
    mine = (j - case["prefix"]).clamp(min=0)
    page = state["table"].long()[:, mine // case["page"]]
    offset = mine % case["page"]
    if case["prefix"]:
        shared = j < case["prefix"]
        in_prefix = j.clamp(max=case["prefix"] - 1)
        page = torch.where(shared, state["prefix_table"].long()[in_prefix // case["page"]], page)
        offset = torch.where(shared, in_prefix % case["page"], offset)
    return page, offset.expand_as(page), j < case["prefix"] + state["seq_len"].long()[:, None]


def _values(codes, scale, page, offset, kind):
    """Keys or values [B, G, J, D] of 16-bit or 8-bit pages."""
    if scale is None:
        return codes[page, :, offset].permute(0, 2, 1, 3).to(kind)
    x = codes.view(torch.uint8)[page, :, offset].view(CODE).to(kind)
    e = scale.view(torch.uint8)[page, :, offset // BLOCK].int() - 127
    return (x * _power(e).to(kind)[..., None]).permute(0, 2, 1, 3)


def _run_attention(state):
    case = state["case"]
    if own:
        from paper_2609_17184_amd import serving
        return list(serving.window_attention(state["q"], state["cache"], state["batch"], window=case["window"],
                                             sinks=case["sinks"], return_lse=True))
    q, G, D = state["q"], case["kv_heads"], case["head_dim"]
    T, per, B = len(q), case["heads"] // case["kv_heads"], case["seqs"]
    page, offset, theirs = _history(state)
    J = page.shape[1]
    keys = _values(state["k_cache"], state["k_scale"], page, offset, torch.float32)
    seq, place = _places(state)
    slot = torch.arange(T, device=DEV) - state["q_start"].long()[seq]
    padded = torch.zeros((B, G, case["new"], per, D), device=DEV)
    padded[seq, :, slot] = q.view(T, G, per, D).float()
    at = torch.zeros((B, case["new"]), dtype=torch.long, device=DEV)        # (rows of no token see the first position)
    at[seq, slot] = place + case["prefix"]
    s = torch.matmul(padded.view(B, G, -1, D), keys.transpose(2, 3).contiguous()) * D ** -0.5
    del keys
    j = torch.arange(J, device=DEV)
    hidden = j > at[..., None]
    if case["window"]:
        hidden = hidden | ((j <= at[..., None] - case["window"]) & (j >= case["sinks"]))
    s = s.view(B, G, case["new"], per, J).masked_fill_(hidden[:, None, :, None], -math.inf)
    peak = s.amax(-1, keepdim=True)
    s = s.sub_(peak).exp_()
    total = s.sum(-1)
    values = _values(state["v_cache"], state["v_scale"], page, offset, torch.float32)
    values = values * theirs[:, None, :, None]
    out = torch.matmul(s.view(B, G, -1, J), values).view(B, G, case["new"], per, D) / total[..., None]
    lse = peak[..., 0] + torch.log(total)
    return [out[seq, :, slot].reshape(T, -1, D).to(q.dtype), lse[seq, :, slot].reshape(T, -1)]


def _run_fork(state):
    case, page = state["case"], state["case"]["page"]
    if own:
        from paper_2609_17184_amd import serving
        made = serving.fork_pages(state["seq_len"], state["table"], state["parent"], state["refs"], state["caches"],
                                  window=case["window"], sinks=case["sinks"])
        return list(made) + [t for x in state["layers"] for t in x if t is not None]
    table, refs = state["table"].long(), state["refs"].long()
    n, width = table.shape
    parent = state["parent"].long()
    m = len(parent)
    live = parent >= 0
    src = parent.clamp(min=0)
    order = torch.arange(m, device=DEV)
    heir = torch.full((n + 1,), m, device=DEV).scatter_reduce_(0, torch.where(live, src, n), order, "amin")[:n]
    is_heir = live & (heir[src] == order)
    length = state["seq_len"].long()
    i = torch.arange(width, device=DEV)
    # pages that the next position does not see
    gone = torch.zeros((n, width), dtype=torch.bool, device=DEV)
    if case["window"]:
        gone = ((i + 1) * page <= length[:, None] + 1 - case["window"]) & (i * page >= case["sinks"])
    used = i < -(-length // page)[:, None]
    full = i < (length // page)[:, None]
    row = torch.where(gone, -1, table)
    kept = torch.where(is_heir[:, None] | full[src], row[src], -1)
    new_table = torch.where(live[:, None], kept, -1)
    copied = live & ~is_heir & (length[src] % page > 0)

    def count(t, by):
        return torch.zeros(len(refs) + 1, dtype=torch.long, device=DEV).index_add_(
            0, torch.where(t < 0, len(refs), t).flatten(), by.flatten())[:-1]
    new_refs = refs - count(table, torch.ones_like(table)) + count(new_table, torch.ones_like(new_table))
    free = torch.argsort((new_refs != 0).int(), stable=True)
    rank = torch.cumsum(copied, 0) - 1
    given = copied & (rank < (new_refs == 0).sum())
    fresh = free[rank.clamp(min=0, max=len(refs) - 1)]
    tail = (length // page)[src].clamp(max=width - 1)
    new_table[order, tail] = torch.where(copied, torch.where(given, fresh, -1), new_table[order, tail])
    new_refs = new_refs + count(torch.where(given, fresh, -1), torch.ones_like(fresh))
    # rows that copy nothing rewrite a page that is their parent's (or the first child's parent's)
    whose = torch.where(live, src, src[0])
    last = table[whose, (-(-length // page) - 1)[whose]]
    dst = torch.where(given, fresh, last)
    copies = torch.where(given, (length % page)[src], 0)
    for layer in state["layers"]:
        for x in layer:
            if x is not None:
                x = x if x.dtype in TYPES.values() else x.view(torch.uint8)
                per = page // x.shape[2]
                here = torch.arange(0, page, per, device=DEV) < copies[:, None]
                here = here[:, None] if x.dim() == 3 else here[:, None, :, None]
                x[dst] = torch.where(here, x[last], x[dst])
    short = (copied & ~given).sum()
    return [torch.where(live, length[src], -1).int(), new_table.int(), new_refs.int(), short.int().view(1)] + [
        t for x in state["layers"] for t in x if t is not None]


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    state = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention, "fork": _exact_fork}[case["op"]](case, state)


def _e4m3(x):
    """The nearest of 0, +-2^-9 .. +-448, ties to even."""
    step = 2.0 ** (torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_append(case, state):
    D, rot, page = case["head_dim"], case["rot"], case["page"]
    q_out = torch.empty(state["q"].shape, dtype=torch.float64, device=DEV)
    freq = torch.tensor([1e4 ** (-2 * j / rot) for j in range(rot // 2)], dtype=torch.float64, device=DEV)
    codes = [state[n].double() for n in ("k_cache", "v_cache")]
    scales = [torch.exp2(state[n].view(torch.uint8).double() - 127) for n in ("k_scale", "v_scale")]

    def turn(x, gain, positions):
        x = x.double()
        if gain is not None:
            x = gain.double() * x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / D + 1e-6)
        pair = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot].contiguous())
        pair = pair * torch.exp(1j * (positions.double()[:, None] * freq))[:, None]
        return torch.cat([pair.real, pair.imag, x[..., rot:]], -1)
    at = 0
    for b, (n, length) in enumerate(zip(state["new"], state["lens"])):
        place = torch.arange(length - n, length, device=DEV)
        rows = slice(at, at + n)
        q_out[rows] = turn(state["q"][rows], state.get("q_gain"), place + case["prefix"])
        new = [turn(state["k"][rows], state.get("k_gain"), place + case["prefix"]), state["v"][rows].double()]
        for x, code, scale in zip(new, codes, scales):
            done = 0
            while done < n:
                s = length - n + done
                p, u, keep = int(state["table"][b, s // page]), s % page // BLOCK, s % BLOCK
                rest = x[done:done + BLOCK - keep]
                size = torch.exp2(torch.ceil(torch.log2(rest.abs().amax((0, 2)) / 448)).clamp(min=LEAST))
                line = code[p, :, u * BLOCK:(u + 1) * BLOCK]
                if keep:
                    size = torch.maximum(size, scale[p, :, u])
                    line[:, :keep] = _e4m3(line[:, :keep] * (scale[p, :, u] / size)[:, None, None])
                line[:, keep:keep + len(rest)] = _e4m3(rest.transpose(0, 1) / size[:, None, None])
                scale[p, :, u] = size
                done += len(rest)
        at += n
    return [q_out] + codes + scales


def _exact_attention(case, state):
    G, D, P = case["kv_heads"], case["head_dim"], case["prefix"]
    per, T = case["heads"] // G, len(state["q"])
    if 8 * T * case["heads"] * (P + max(state["lens"])) > 4e11:
        return None
    out = torch.empty((T, G, per, D), dtype=torch.float64, device=DEV)
    lse = torch.empty((T, G, per), dtype=torch.float64, device=DEV)

    def positions(codes, scale, table, n):
        table = table[:-(-n // case["page"])].long()
        if scale is None:
            x = codes[table].double()
        else:
            x = codes.view(torch.uint8)[table].view(CODE).double()
            x = x * torch.exp2(scale.view(torch.uint8)[table].double() - 127).repeat_interleave(BLOCK, 2)[..., None]
        return x.transpose(0, 1).reshape(G, -1, D)[:, :n]
    pools = [(state["k_cache"], state["k_scale"]), (state["v_cache"], state["v_scale"])]
    prefix = [positions(*pool, state["prefix_table"], P) for pool in pools]
    at = 0
    for b, (n, length) in enumerate(zip(state["new"], state["lens"])):
        K, V = (torch.cat([p, positions(*pool, state["table"][b], length)], 1) for p, pool in zip(prefix, pools))
        for i in range(0, n, 512):          # tokens at a time
            rows = slice(at + i, at + min(n, i + 512))
            q = state["q"][rows].double()
            here = P + length - n + torch.arange(i, i + len(q), device=DEV)[:, None]
            j = torch.arange(P + length, device=DEV)
            sees = j <= here
            if case["window"]:
                sees &= (here - j < case["window"]) | (j < case["sinks"])
            s = q.view(len(q), G, per, D).transpose(0, 1).reshape(G, -1, D) @ K.mT / math.sqrt(D)
            s = s.view(G, len(q), per, -1).masked_fill(~sees[None, :, None], -math.inf)
            lse[rows] = torch.logsumexp(s, -1).transpose(0, 1)
            out[rows] = (torch.softmax(s, -1).view(G, -1, P + length) @ V).view(G, len(q), per, D).transpose(0, 1)
        at += n
    return [out.view(T, -1, D), lse.view(T, -1)]


def _exact_fork(case, state):
    page, window, sinks = case["page"], case["window"], case["sinks"]
    old, refs = state["table"].tolist(), state["refs"].tolist()
    lens, parent = _branches(case)
    width = len(old[0])
    table, heirs, wanted = [], {}, []
    for row in old:
        for x in row:
            if x >= 0:
                refs[x] -= 1
    for j, p in enumerate(parent):
        row = [-1] * width
        if p >= 0:
            for i in range(width):
                unseen = window and (i + 1) * page <= lens[p] + 1 - window and i * page >= sinks
                if not unseen and (p not in heirs or (i + 1) * page <= lens[p]):
                    row[i] = old[p][i]
            if p in heirs and lens[p] % page:
                wanted.append(j)
            heirs.setdefault(p, j)
        table.append(row)
        for x in row:
            if x >= 0:
                refs[x] += 1
    free = [x for x, r in enumerate(refs) if r == 0]
    caches = [[t if t is None else t.clone() if t.dtype in TYPES.values() else t.view(torch.uint8).clone() for t in x]
              for x in state["layers"]]
    for j, x in zip(wanted, free):
        p = parent[j]
        table[j][lens[p] // page], refs[x] = x, 1
        source, n = old[p][lens[p] // page], lens[p] % page
        for k, v, ks, vs in caches:
            for t in (k, v):
                t[x, :, :n] = t[source, :, :n]
            for t in (ks, vs):
                if t is not None:
                    t[x, :, :-(-n // BLOCK)] = t[source, :, :-(-n // BLOCK)]

    def whole(x):
        return torch.tensor(x, dtype=torch.int32, device=DEV)
    flat = [t if t.dtype in TYPES.values() else t.view(CODE if t.dim() == 4 else SCALE) for x in caches for t in x if t is not None]
    return [whole([lens[p] if p >= 0 else -1 for p in parent]), whole(table), whole(refs),
            whole([max(0, len(wanted) - len(free))])] + flat
