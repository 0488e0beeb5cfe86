"""Performance cases of the serving operators: a batch of sequences over a paged cache, step by step.

Three operators, in the order in which a serving loop calls them for one layer and one step:

  append     queries and keys of the step's tokens are normalised per head (optional) and rotated to their positions;
             keys and values go to the pages of their sequences
  attention  every query row attends to one long prefix that all sequences share, and to its own sequence's positions
  sample     one token per row from its logits: temperature, top-k, top-p and min-p, with given uniform numbers

The head layouts are those of this repository's model shapes (16 heads of 128, 55 heads of 96, 4 heads of 64), and
generic ones with shared key/value heads; the vocabularies are its models' (49152 and 65536) and a larger, odd one.
A case's lengths come from the case itself (`ragged` seeds them); the seed of `prepare` decides every value.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _append(name, seqs, new, context, prefix, heads, kv_heads, head_dim, rot, page, dtype, norm, ragged):
    return dict(name=name, op="append", seqs=seqs, new=new, context=context, prefix=prefix, heads=heads,
                kv_heads=kv_heads, head_dim=head_dim, rot=rot, page=page, dtype=dtype, norm=norm, ragged=ragged)


def _attention(name, seqs, new, context, prefix, heads, kv_heads, head_dim, page, dtype, ragged):
    return dict(name=name, op="attention", seqs=seqs, new=new, context=context, prefix=prefix, heads=heads,
                kv_heads=kv_heads, head_dim=head_dim, page=page, dtype=dtype, ragged=ragged)


def _sample(name, rows, vocab, dtype, temperature, top_k, top_p, min_p):
    return dict(name=name, op="sample", rows=rows, vocab=vocab, dtype=dtype, temperature=temperature, top_k=top_k,
                top_p=top_p, min_p=min_p)


def listed():
    return [
        # one token of one sequence, the Ouro head shape: nothing but latency
        _append("append_decode_1", 1, 1, 700, 0, 16, 16, 128, 128, 16, "f16", False, 1),
        # a decode step of a large batch behind a long prefix, shared key/value heads, norms of queries and keys
        _append("append_decode_96", 96, 1, 2000, 20000, 32, 8, 128, 128, 32, "bf16", True, 2),
        # ragged prompts of a few sequences, the Raven head shape
        _append("append_prompts_raven", 5, 900, 300, 1000, 55, 55, 96, 96, 16, "f16", False, 3),
        # one long prompt, half of each head rotated, seven query heads to a key/value head
        _append("append_prompt_long", 1, 16001, 0, 0, 28, 4, 128, 64, 64, "bf16", True, 4),
        # three sequences and a short prefix, the tiny decoder's heads: latency
        _attention("attention_few", 3, 1, 40, 500, 4, 4, 64, 16, "f16", 5),
        # an ordinary decode step of the Ouro head shape
        _attention("attention_ouro_32", 32, 1, 256, 8192, 16, 16, 128, 16, "f16", 6),
        # several rows in flight per sequence (drafts to be verified), the Raven head shape
        _attention("attention_rows_raven", 48, 5, 300, 4007, 55, 55, 96, 32, "bf16", 7),
        # a large batch over a long prefix, four query heads to a key/value head: the matrix cores are the bound
        _attention("attention_long_192", 192, 1, 256, 32768, 32, 8, 128, 64, "bf16", 8),
        # a single request
        _sample("sample_1", 1, 49152, "f32", 0.8, 0, 0.95, 0.0),
        # a batch of requests, each row with its own settings
        _sample("sample_mixed_48", 48, 65536, "bf16", -1.0, -1, -1.0, -1.0),
        # a large batch from the whole distribution
        _sample("sample_whole_256", 256, 130003, "f32", 1.0, 0, 1.0, 0.0),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attention", "sample"])
    largest = [work(c) for c in listed() if c["op"] == op]
    limit = {k: max(w[k] for w in largest) for k in ("bytes", "flops")}
    if op == "sample":
        case = _sample("", _spread(rng, 1, 256), _spread(rng, 1000, 140000), rng.choice(["f32", "bf16", "f16"]),
                       rng.choice([-1.0, 0.7, 1.0, 1.3]), rng.choice([-1, 0, 40, 1000]),
                       rng.choice([-1.0, 0.9, 1.0]), rng.choice([-1.0, 0.0, 0.05]))
        shrink = "rows"
    else:
        heads, kv_heads, head_dim = rng.choice(
            [(16, 16, 128), (55, 55, 96), (4, 4, 64), (32, 8, 128), (28, 4, 128), (32, 4, 64), (5, 1, 128), (8, 8, 32)])
        page, dtype, ragged = rng.choice([16, 32, 48, 64, 128]), rng.choice(["f16", "bf16"]), rng.randrange(1 << 30)
        if op == "append":
            prompt = rng.random() < 0.5
            case = _append("", _spread(rng, 1, 6 if prompt else 192), _spread(rng, 2, 5000) if prompt else 1,
                           _spread(rng, 1, 2000), rng.choice([0, _spread(rng, 16, 40000)]), heads, kv_heads, head_dim,
                           rng.choice([head_dim, head_dim // 2]), page, dtype, rng.random() < 0.5, ragged)
        else:
            case = _attention("", _spread(rng, 1, 192), rng.choice([1, 1, 1, 3, 9]), _spread(rng, 1, 600),
                              _spread(rng, 100, 33000), heads, kv_heads, head_dim, page, dtype, ragged)
        shrink = "seqs" if op == "attention" else "new"
    while any(work(case)[k] > limit[k] for k in limit):
        if case[shrink] == 1:
            shrink = "prefix" if op == "attention" else "seqs"
        case[shrink] = max(1, case[shrink] * 3 // 4)
    del case["name"]
    return case


def _lengths(case):
    """(tokens of this step, positions with them) of every sequence."""
    r = random.Random(case["ragged"])
    new = [case["new"] if i == 0 else r.randint(max(1, case["new"] // 4), case["new"]) for i in range(case["seqs"])]
    return new, [n + (case["context"] if i == 0 else r.randint(0, case["context"])) for i, n in enumerate(new)]


def work(case):
    size = {"f16": 2, "bf16": 2, "f32": 4}[case["dtype"]]
    if case["op"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * size + case["rows"] * 20, "flops": n * 8}
    H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
    new, lens = _lengths(case)
    T = sum(new)
    if case["op"] == "append":
        return {"bytes": 2 * T * (H + 2 * G) * D * size,
                "flops": T * (H + G) * (3 * case["rot"] + (4 * D if case["norm"] else 0))}
    seen = sum(n * case["prefix"] + n * (L - n) + n * (n + 1) // 2 for n, L in zip(new, lens))
    return {"bytes": 2 * (case["prefix"] + sum(lens)) * G * D * size + 2 * T * H * D * size + 4 * T * H,
            "flops": 4 * H * D * seen}


# ---------------------------------------------------------------------------------------------------------------------
# what a program has in hand before the call
# ---------------------------------------------------------------------------------------------------------------------
def _normal(gen, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * std).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    host = random.Random(seed)
    dtype = TYPES[case["dtype"]]
    if case["op"] == "sample":
        rows, V = case["rows"], case["vocab"]
        logits = torch.randn((rows, V), generator=gen, device=DEV) * 2.5
        # a readout's few likely tokens, one in each of 24 stretches of the vocabulary
        peaks = torch.randint(0, V // 24, (rows, 24), generator=gen, device=DEV)
        peaks += torch.arange(24, device=DEV) * (V // 24)
        logits.scatter_(1, peaks, 6.0 + 3.0 * torch.randn((rows, 24), generator=gen, device=DEV))

        def per_row(value, low, choices, kind):
            if value != low:
                return value
            return torch.tensor([host.choice(choices) for _ in range(rows)], dtype=kind, device=DEV)
        return dict(case=case, logits=logits.to(dtype),
                    u=torch.rand(rows, generator=gen, device=DEV, dtype=torch.float64),
                    temperature=per_row(case["temperature"], -1.0, [0.0, 0.6, 0.8, 1.0, 1.25], torch.float32),
                    top_k=per_row(case["top_k"], -1, [0, 1, 20, 50, 400], torch.int32),
                    top_p=per_row(case["top_p"], -1.0, [0.5, 0.9, 0.95, 1.0], torch.float32),
                    min_p=per_row(case["min_p"], -1.0, [0.0, 0.02, 0.1], torch.float32))

    H, G, D, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    new, lens = _lengths(case)
    T = sum(new)
    n_prefix = -(-case["prefix"] // page)
    n_own = [-(-L // page) for L in lens]
    pages = list(range(n_prefix * (case["op"] == "attention") + sum(n_own) + 3))
    n_pages = len(pages)
    host.shuffle(pages)
    prefix_table = [pages.pop() for _ in range(n_prefix)] if case["op"] == "attention" else []
    table = np.zeros((len(new), max(n_own)), np.int32)
    for b, n in enumerate(n_own):
        table[b, :n] = [pages.pop() for _ in range(n)]
    k_cache = _normal(gen, (n_pages, G, page, D), dtype)
    v_cache = _normal(gen, (n_pages, G, page, D), dtype)
    qkv = _normal(gen, (T, (H + 2 * G) * D), dtype)
    state = dict(case=case, k_cache=k_cache, v_cache=v_cache, new=new, lens=lens,
                 q=qkv[:, :H * D].view(T, H, D), k=qkv[:, H * D:(H + G) * D].view(T, G, D),
                 v=qkv[:, (H + G) * D:].view(T, G, D),
                 table=torch.from_numpy(table).to(DEV), seq_len=torch.tensor(lens, dtype=torch.int32, device=DEV),
                 q_start=torch.tensor(np.cumsum([0] + new), dtype=torch.int32, device=DEV),
                 prefix_table=torch.tensor(prefix_table, dtype=torch.int32, device=DEV),
                 freq=1e4 ** (-torch.arange(case.get("rot", 0) // 2, dtype=torch.float64, device=DEV)
                              * 2 / max(1, case.get("rot", 0))))
    if case["op"] == "attention":
        state["q"] = state["q"] * 2         # scores with a standard deviation of 2
    elif case["norm"]:
        state["q_gain"], state["k_gain"] = (1 + 0.2 * torch.randn(D, generator=gen, device=DEV) for _ in range(2))
    if own:
        from paper_2609_17184_amd import serving
        state["cache"] = serving.PagedCache(k_cache, v_cache)
        state["batch"] = serving.Batch(
            state["seq_len"], state["table"], q_start=state["q_start"] if case["new"] > 1 else None,
            prefix_len=case["prefix"], prefix_table=state["prefix_table"] if case["op"] == "attention" else None)
    return state


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(state):
    return {"append": _run_append, "attention": _run_attention, "sample": _run_sample}[state["case"]["op"]](state)


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
        return [q, state["k_cache"], state["v_cache"]]
    seq, place = _places(state)
    angle = (place + case["prefix"])[:, None].double() * state["freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    half, dtype = case["rot"] // 2, state["q"].dtype

    def rotated(x, gain):
        x = x.float()
        if gain is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gain
        a, b = x[..., :half], x[..., half:2 * half]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]], -1).to(dtype)
    page = state["table"].long()[seq, place // case["page"]]
    state["k_cache"][page, :, place % case["page"]] = rotated(state["k"], state.get("k_gain"))
    state["v_cache"][page, :, place % case["page"]] = state["v"]
    return [rotated(state["q"], state.get("q_gain")), state["k_cache"], state["v_cache"]]


def _run_attention(state):
    case = state["case"]
    if own:
        from paper_2609_17184_amd import serving
        return list(serving.prefix_attention(state["q"], state["cache"], state["batch"], return_lse=True))
    q, G, D, P = state["q"], case["kv_heads"], case["head_dim"], case["prefix"]
    T, per = len(q), case["heads"] // case["kv_heads"]
    scale = D ** -0.5
    # the prefix: [G, P, D] against all rows
    kp, vp = (c[state["prefix_table"].long()].transpose(0, 1).reshape(G, -1, D)[:, :P].float()
              for c in (state["k_cache"], state["v_cache"]))
    qp = q.view(T, G, per, D).permute(1, 0, 2, 3).reshape(G, T * per, D).float()
    sp = torch.matmul(qp, kp.transpose(1, 2).contiguous()) * scale
    # each sequence's own positions, padded to the longest
    B, width = state["table"].shape
    seq, place = _places(state)
    slot = torch.arange(T, device=DEV) - state["q_start"].long()[seq]
    ko, vo = (c[state["table"].long()].transpose(1, 2).reshape(B, G, -1, D).float()
              for c in (state["k_cache"], state["v_cache"]))
    vo = vo.masked_fill((torch.arange(vo.shape[2], device=DEV) >= state["seq_len"][:, None])[:, None, :, None], 0.0)
    qo = torch.zeros((B, G, case["new"], per, D), device=DEV)
    qo[seq, :, slot] = q.view(T, G, per, D).float()
    limit = torch.full((B, case["new"]), -1, dtype=torch.long, device=DEV)
    limit[seq, slot] = place
    so = torch.matmul(qo.view(B, G, -1, D), ko.transpose(2, 3).contiguous()) * scale
    so = so.view(B, G, case["new"], per, -1)
    so = so.masked_fill((torch.arange(so.shape[-1], device=DEV) > limit[..., None])[:, None, :, None], -math.inf)

    def rows_of(x):             # [B, G, new, per, ...] -> [G, T * per, ...]
        return x[seq, :, slot].transpose(0, 1).reshape(G, T * per, *x.shape[4:])
    peak = torch.maximum(sp.amax(-1), rows_of(so.amax(-1)))
    padded = torch.zeros((B, G, case["new"], per), device=DEV)
    padded[seq, :, slot] = peak.view(G, T, per).transpose(0, 1)
    ep, eo = torch.exp(sp - peak[..., None]), torch.exp(so - padded[..., None])
    total = ep.sum(-1) + rows_of(eo.sum(-1))
    out = torch.matmul(ep, vp) + rows_of(torch.matmul(eo.flatten(2, 3), vo).view(B, G, case["new"], per, D))
    out = (out / total[..., None]).view(G, T, per, D).transpose(0, 1).reshape(T, -1, D).to(q.dtype)
    return [out, (peak + torch.log(total)).view(G, T, per).transpose(0, 1).reshape(T, -1)]


def _run_sample(state):
    z, u = state["logits"], state["u"]
    if own:
        from paper_2609_17184_amd import serving
        return list(serving.sample(z, u, temperature=state["temperature"], top_k=state["top_k"], top_p=state["top_p"],
                                   min_p=state["min_p"]))
    V = z.shape[1]

    def column(x, kind):
        return torch.as_tensor(x, dtype=kind, device=DEV).expand(len(z))[:, None]
    temperature = column(torch.as_tensor(state["temperature"], dtype=torch.float32), torch.float64)
    top_p = column(torch.as_tensor(state["top_p"], dtype=torch.float32), torch.float64)
    min_p = column(torch.as_tensor(state["min_p"], dtype=torch.float32), torch.float64)
    top_k = column(state["top_k"], torch.long)
    top_k = torch.where(temperature == 0, 1, torch.where(top_k <= 0, V, top_k))
    zs, ids = torch.sort(z, dim=1, descending=True, stable=True)
    w = torch.exp((zs.double() - zs[:, :1].double()) / torch.where(temperature == 0, 1.0, temperature))
    rank = torch.arange(V, device=DEV)
    w_k = w * (rank < top_k)
    before = torch.cumsum(w_k, 1) - w_k
    keep = (rank < top_k) & ((before < top_p * w_k.sum(1, keepdim=True)) | (top_p >= 1)) & (w >= min_p)
    kept = torch.zeros_like(w).scatter_(1, ids, w * keep)
    mass = torch.cumsum(kept, 1)
    token = (mass <= u[:, None] * mass[:, -1:]).sum(1, keepdim=True)
    prob = kept.gather(1, token) / mass[:, -1:]
    return [token[:, 0].int(), prob[:, 0].float(), keep.sum(1).int()]


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    state = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention, "sample": _exact_sample}[case["op"]](case, state)


def _exact_append(case, state):
    D, rot = case["head_dim"], case["rot"]
    q_out = torch.empty(state["q"].shape, dtype=torch.float64, device=DEV)
    caches = [state["k_cache"].double(), state["v_cache"].double()]
    freq = torch.tensor([1e4 ** (-2 * j / rot) for j in range(rot // 2)], dtype=torch.float64, device=DEV)

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
        page = state["table"][b].long()[place // case["page"]]
        caches[0][page, :, place % case["page"]] = turn(state["k"][rows], state.get("k_gain"), place + case["prefix"])
        caches[1][page, :, place % case["page"]] = state["v"][rows].double()
        at += n
    return [q_out] + caches


def _exact_attention(case, state):
    G, D, P = case["kv_heads"], case["head_dim"], case["prefix"]
    per = case["heads"] // G
    T = len(state["q"])
    out = torch.empty((T, G, per, D), dtype=torch.float64, device=DEV)
    lse = torch.empty((T, G, per), dtype=torch.float64, device=DEV)

    def positions(cache, table, n):
        return cache[table[:-(-n // case["page"])].long()].double().transpose(0, 1).reshape(G, -1, D)[:, :n]
    prefix = [positions(c, state["prefix_table"], P) for c in (state["k_cache"], state["v_cache"])]
    at = 0
    for b, (n, length) in enumerate(zip(state["new"], state["lens"])):
        K, V = (torch.cat([p, positions(c, state["table"][b], length)], 1)
                for p, c in zip(prefix, (state["k_cache"], state["v_cache"])))
        q = state["q"][at:at + n].double().view(n, G, per, D).transpose(0, 1).reshape(G, n * per, D)
        s = (q @ K.mT / math.sqrt(D)).view(G, n, per, P + length)
        future = torch.arange(P + length, device=DEV) > (P + length - n + torch.arange(n, device=DEV))[:, None]
        s = s.masked_fill(future[None, :, None], -math.inf)
        lse[at:at + n] = torch.logsumexp(s, -1).transpose(0, 1)
        out[at:at + n] = (torch.softmax(s, -1).view(G, n * per, -1) @ V).view(G, n, per, D).transpose(0, 1)
        at += n
    return [out.view(T, -1, D), lse.view(T, -1)]


def _exact_sample(case, state):
    logits, u = state["logits"].float().cpu().numpy().astype(np.float64), state["u"].cpu().numpy()
    rows, V = logits.shape

    def settings(x):
        x = x.cpu().numpy() if torch.is_tensor(x) else np.float32(x)
        return np.broadcast_to(x, (rows,)).astype(np.float64)
    temperature, top_k, top_p, min_p = (settings(state[n]) for n in ("temperature", "top_k", "top_p", "min_p"))
    tokens, probs, counts = [], [], []
    for z, uniform, t, k, p, least in zip(logits, u, temperature, top_k, top_p, min_p):
        if t == 0:
            tokens, probs, counts = tokens + [int(z.argmax())], probs + [1.0], counts + [1]
            continue
        w = np.exp((z - z.max()) / t)
        order = np.argsort(-z, kind="stable")[:int(k) if k > 0 else V]
        if p < 1:
            order = order[:np.searchsorted(np.cumsum(w[order]), p * w[order].sum(), side="left") + 1]
        order = np.sort(order[w[order] >= least])
        mass = np.cumsum(w[order])
        i = int(np.searchsorted(mass, uniform * mass[-1], side="right"))
        tokens, probs, counts = tokens + [int(order[i])], probs + [w[order[i]] / mass[-1]], counts + [len(order)]
    return [torch.tensor(tokens, dtype=torch.int32, device=DEV), torch.tensor(probs, dtype=torch.float64, device=DEV),
            torch.tensor(counts, dtype=torch.int32, device=DEV)]
