"""Performance cases of the operators around verification: a prompt's way into the cache, and from logits to tokens.

  append  rotary positions applied to the queries and keys of new tokens, keys and values written to the paged cache, the
          representatives of the blocks that grew
  attend  attention of a ragged batch of new tokens (chunks of prompts, single tokens) over the paged cache
  sample  temperature, top-k, top-p and min-p on rows of logits: the distributions that acceptance takes, and tokens drawn
          from them with given random numbers

``own`` chooses between the operators' plain form (elementary torch operations in 32 bits, rounded once at the end) and the
calls of this package.

Keys of a case.  append and attend: seqs, lo, hi (tokens of a sequence cached before, uniform in lo..hi), new_lo, new_hi (new
tokens of a sequence), singles (how many of the sequences have one new token instead), heads (query), kv_heads, block (tokens
of a page); append also: rot (rotated dims of a head), interleaved (pairs are neighbours), fused (q, k and v are slices of one
projection's output).  sample: seqs, rows (of a sequence), vocab, pad (entries between rows), half (logits in bfloat16), dist
(the distributions are wanted too), temperature, top_k, top_p, min_p (what the sequences' own values lie around; 0: off).

Inputs are random with the shape of the real thing: attention logits with a standard deviation of about 3, pages in random
order, logits of a vocabulary with a standard deviation of 1 / 0.35.  A token is a whole number decided by sums in 32 bits, so
the random numbers and the top-p values are moved to the middle of what decides the same: the mass of one token.
"""
import math
import random

import torch

own = False

HEAD_DIM = 128
SIGMA = math.sqrt(3.0)       # of queries and keys: logits q.k / sqrt(128) then have a standard deviation of 3
THETA = 500000.0             # base of the rotary angles
SPARE_BLOCKS = 2             # entries of the block table behind the blocks in use


def _cache(op, seqs, lo, hi, new_lo, new_hi, heads, kv_heads, block, singles=0, **more):
    return dict(op=op, seqs=seqs, lo=lo, hi=hi, new_lo=new_lo, new_hi=new_hi, singles=singles, heads=heads, kv_heads=kv_heads,
                block=block, **more)


def _append(*shape, singles=0, rot=128, interleaved=False, fused=True):
    return _cache("append", *shape, singles=singles, rot=rot, interleaved=interleaved, fused=fused)


def _attend(*shape, singles=0):
    return _cache("attend", *shape, singles=singles)


def _sample(seqs, rows, vocab, pad=0, half=False, dist=False, temperature=0.8, top_k=0, top_p=0.0, min_p=0.0):
    return dict(op="sample", seqs=seqs, rows=rows, vocab=vocab, pad=pad, half=half, dist=dist, temperature=temperature,
                top_k=top_k, top_p=top_p, min_p=min_p)


def listed():
    return [
        # a decoding step of a batch: one token a sequence
        dict(_append(64, 500, 1500, 1, 1, 32, 8, 64), name="append_64_tokens"),
        # continuous batching: chunks of several prompts next to decoding sequences, odd lengths, half of a head rotated in neighbours
        dict(_append(12, 0, 2001, 100, 777, 28, 4, 128, singles=5, rot=64, interleaved=True, fused=False), name="append_ragged_batch"),
        # a whole prompt in one piece
        dict(_append(1, 0, 0, 32768, 32768, 32, 8, 64), name="append_prompt_32k"),
        # the smallest call: one token of one short sequence on a small model
        dict(_attend(1, 4095, 4095, 1, 1, 8, 2, 64), name="attend_token_4k_small_model"),
        # a decoding batch of 16 requests of different lengths
        dict(_attend(16, 4096, 16384, 1, 1, 32, 8, 64), name="attend_16_tokens_ragged"),
        # continuous batching: three chunks of prompts and nine decoding sequences in one call, seven query heads a KV head
        dict(_attend(12, 501, 5001, 300, 701, 28, 4, 128, singles=9), name="attend_ragged_batch"),
        # a prompt of 8K tokens in one piece
        dict(_attend(1, 0, 0, 8192, 8192, 32, 8, 64), name="attend_prompt_8k"),
        # a later chunk of a long document, eight query heads a KV head
        dict(_attend(1, 30001, 30001, 2048, 2048, 64, 8, 128), name="attend_chunk_2k_at_30k"),
        # the next token of one request
        dict(_sample(1, 1, 128256, top_k=50, top_p=0.9), name="sample_one_row"),
        # a decoding batch with bfloat16 logits out of a padded projection, nucleus sampling over the whole vocabulary
        dict(_sample(64, 1, 151936, pad=128, half=True, top_p=0.95), name="sample_64_rows_bf16"),
        # the target's distributions of 16 drafts of five tokens, for acceptance
        dict(_sample(16, 5, 128256, dist=True, temperature=1.0, top_p=0.9), name="sample_16_drafts_dist"),
        # many rows over a small vocabulary of odd size, min-p
        dict(_sample(256, 1, 32003, dist=True, top_k=40, min_p=0.05), name="sample_256_rows_odd"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("append", "attend", "sample")}
    while True:
        op = rng.choice(["append", "attend", "attend", "sample"])
        if op == "sample":
            case = _sample(_log(rng, 1, 256), rng.choice([1, 1, 1, 2, 5, 9]), rng.choice([32000, 32003, 50257, 128256, 151936]),
                           rng.choice([0, 0, 64, 61]), rng.random() < 0.4, rng.random() < 0.5, round(rng.uniform(0.5, 1.5), 2),
                           rng.choice([0, 0, _log(rng, 2, 1000)]), rng.choice([0.0, round(rng.uniform(0.3, 0.99), 2)]),
                           rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.3), 2)]))
        else:
            heads, kv_heads = rng.choice([(8, 2), (32, 8), (32, 8), (64, 8), (28, 4), (40, 8), (16, 16)])
            hi = rng.choice([0, _log(rng, 64, 32768), _log(rng, 64, 32768)])
            lo = hi if rng.random() < 0.4 else rng.randint(0, hi)
            new_hi = rng.choice([1, _log(rng, 2, 8192), _log(rng, 2, 8192)])
            new_lo = new_hi if rng.random() < 0.4 else rng.randint(1, new_hi)
            seqs = _log(rng, 1, 64)
            shape = (seqs, lo, hi, new_lo, new_hi, heads, kv_heads, rng.choice([64, 64, 128]))
            singles = rng.choice([0, rng.randint(0, seqs - 1)])
            if op == "append":
                case = _append(*shape, singles=singles, rot=rng.choice([128, 128, 64, 32]), interleaved=rng.random() < 0.4,
                               fused=rng.random() < 0.5)
            else:
                case = _attend(*shape, singles=singles)
        if _cost(case) <= most[op]:
            return case


def _cost(case):
    """What a case may not exceed the listed ones in: what its plain form holds on the device."""
    if case["op"] == "sample":
        return case["seqs"] * case["rows"] * case["vocab"]
    before, new = _lengths(case)
    if case["op"] == "append":
        return sum(new) * (case["heads"] + 2 * case["kv_heads"]) + sum(before) * case["kv_heads"] // 4
    return case["seqs"] * case["heads"] * max(new) * (max(b + n for b, n in zip(before, new)) + 64)


def _lengths(case):
    """Tokens cached before and new tokens of every sequence: the case's own, whatever the seed."""
    rng = random.Random(str(sorted((k, v) for k, v in case.items() if k != "name")))
    before = [rng.randint(case["lo"], case["hi"]) for _ in range(case["seqs"])]
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    for s in rng.sample(range(case["seqs"]), case["singles"]):
        new[s] = 1
    return before, new


# ------------------------------------------------------------------------------------------------ inputs


def _normal(gen, *shape, sigma=1.0):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, sigma, generator=gen)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _prepare_cache(case, gen, seed):
    S, B, Hq, Hkv = case["seqs"], case["block"], case["heads"], case["kv_heads"]
    before, new = _lengths(case)
    blocks = [-(-(b + n) // B) for b, n in zip(before, new)]
    width = max(blocks) + SPARE_BLOCKS
    pages = torch.randperm(sum(blocks) + 1, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((S, width), -1, dtype=torch.int32)
    at = 0
    for s in range(S):
        table[s, :blocks[s]] = torch.tensor(pages[at:at + blocks[s]], dtype=torch.int32)
        at += blocks[s]
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    N = starts[-1]
    st = dict(op=case["op"], heads=Hq, kv_heads=Hkv, block=B, longest=max(new), width=width,
              grown=max(-(-(b + n) // B) - b // B for b, n in zip(before, new)), table=table.cuda(), q_start=_ints(starts),
              before=_ints(before), after=_ints([b + n for b, n in zip(before, new)]))
    st["k_pool"] = _normal(gen, len(pages), Hkv, B, HEAD_DIM, sigma=SIGMA)
    st["v_pool"] = _normal(gen, len(pages), Hkv, B, HEAD_DIM)
    if case["op"] == "attend":
        st["q"] = _normal(gen, N, Hq, HEAD_DIM, sigma=SIGMA)
        st["out"] = torch.empty_like(st["q"])
        return st
    if case["fused"]:
        st["q"], st["k"], st["v"] = _normal(gen, N, Hq + 2 * Hkv, HEAD_DIM, sigma=SIGMA).split([Hq, Hkv, Hkv], dim=1)
    else:
        st["q"], st["k"], st["v"] = (_normal(gen, N, h, HEAD_DIM, sigma=SIGMA) for h in (Hq, Hkv, Hkv))
    half = case["rot"] // 2
    angle = torch.arange(max(b + n for b, n in zip(before, new)), device="cuda", dtype=torch.float64)[:, None] * \
        THETA ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    st["rope"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
    st["interleaved"] = case["interleaved"]
    st["q_out"] = torch.empty((N, Hq, HEAD_DIM), dtype=torch.bfloat16, device="cuda")
    st["new_lens"] = torch.empty_like(st["before"])
    # the representatives that the cache had before; those of blocks that are not there yet are zero
    st["reps"] = torch.zeros((S, Hkv, width, HEAD_DIM), device="cuda")
    for s in range(S):
        n = -(-before[s] // B)
        if n:
            k = st["k_pool"][st["table"][s, :n].long()].float().transpose(0, 1)
            held = (torch.arange(n * B, device="cuda") < before[s]).view(1, n, B, 1)
            st["reps"][s, :, :n] = (k * held).sum(2) / held.sum(2)
    return st


def _prepare_sample(case, gen):
    S, T, V = case["seqs"], case["rows"], case["vocab"]
    R = S * T
    dtype = torch.bfloat16 if case["half"] else torch.float32
    logits = (torch.randn((S, T, V + case["pad"]), generator=gen, device="cuda") / 0.35).to(dtype)[..., :V]
    rand = lambda: torch.rand((S,), generator=gen, device="cuda")   # noqa: E731
    st = dict(op="sample", logits=logits, temperature=None, top_k=None, top_p=None, min_p=None, dist=case["dist"])
    st["temperature"] = case["temperature"] * (0.75 + 0.5 * rand())
    if S >= 4:
        st["temperature"][S // 2] = 0.0                                # one request of a batch is decoded greedily
    if case["top_k"]:
        st["top_k"] = (case["top_k"] * (0.5 + rand())).int().clamp(min=1)
    if case["min_p"]:
        st["min_p"] = case["min_p"] * (0.5 + rand())
    top_p = (1.0 - (1.0 - case["top_p"]) * (0.5 + rand())).clamp(min=0.1) if case["top_p"] else None
    u = torch.rand((R,), generator=gen, device="cuda", dtype=torch.float64)
    # top-p and the random numbers go to the middle of the token's mass that they fall in, of the first row of a sequence and of
    # every row; a draw of a token too unlikely for sums in 32 bits to tell is moved to the likeliest one
    temp = st["temperature"].double().clamp(min=1e-3)
    if top_p is not None:
        p = torch.softmax(logits[:, 0].double() / temp[:, None], dim=-1).sort(dim=-1, descending=True).values
        if case["top_k"]:
            p = p * (torch.arange(V, device="cuda") < st["top_k"][:, None])
            p = p / p.sum(-1, keepdim=True)
        cum = p.cumsum(-1)
        at = (cum < top_p.double()[:, None]).sum(-1, keepdim=True).clamp(max=V - 1)
        st["top_p"] = (cum - p / 2).gather(1, at)[:, 0].clamp(max=1.0).float()
    row_u = []
    for s in range(S):                                                 # a sequence at a time: sorted copies in 64 bits are large
        kept, _ = _warp(logits[s].double(), *(st[k] if st[k] is None else st[k][s:s + 1].double() for k in _PARAMETERS))
        cum = kept.cumsum(-1)
        at = (cum < u[s * T:(s + 1) * T, None] * cum[:, -1:]).sum(-1, keepdim=True).clamp(max=V - 1)
        at = torch.where(kept.gather(1, at) < 1e-5 * cum[:, -1:], kept.argmax(-1, keepdim=True), at)
        row_u.append(((cum - kept / 2).gather(1, at)[:, 0] / cum[:, -1]).float())
    st["u"] = torch.cat(row_u)
    st["tokens"] = torch.empty((R,), dtype=torch.int32, device="cuda")
    st["probs"] = torch.empty((S, T, V), device="cuda") if case["dist"] else None
    return st


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return _prepare_sample(case, gen) if case["op"] == "sample" else _prepare_cache(case, gen, seed)


# ------------------------------------------------------------------------------------------------ one pass: the plain forms

_PARAMETERS = ("temperature", "top_k", "top_p", "min_p")


def _per_token(st, first, pad):
    """Sequence, place among its new tokens and position of every new token; or, padded, of every sequence's places."""
    n = (st["q_start"][1:] - st["q_start"][:-1]).long()
    if pad:
        place = torch.arange(st["longest"], device="cuda").expand(len(n), -1)
        return n, place, first.long()[:, None] + place
    seq = torch.repeat_interleave(torch.arange(len(n), device="cuda"), n, output_size=st["q"].shape[0])
    place = torch.arange(len(seq), device="cuda") - st["q_start"][:-1].long()[seq]
    return seq, place, first.long()[seq] + place


def _rotate(x, cos, sin, interleaved):
    half = cos.shape[-1]
    x = x.float()
    turned = x[..., :2 * half].reshape(*x.shape[:-1], half, 2).transpose(-1, -2) if interleaved else \
        x[..., :2 * half].reshape(*x.shape[:-1], 2, half)
    a, b = turned[..., 0, :], turned[..., 1, :]
    turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-2)
    turned = turned.transpose(-1, -2) if interleaved else turned
    return torch.cat([turned.reshape(*x.shape[:-1], 2 * half), x[..., 2 * half:]], dim=-1).to(torch.bfloat16)


def _plain_append(st):
    B = st["block"]
    seq, _, position = _per_token(st, st["before"], False)
    cos, sin = st["rope"][position].chunk(2, dim=-1)
    st["q_out"].copy_(_rotate(st["q"], cos[:, None], sin[:, None], st["interleaved"]))
    page = st["table"].long()[seq, position // B]
    st["k_pool"][page, :, position % B] = _rotate(st["k"], cos[:, None], sin[:, None], st["interleaved"])
    st["v_pool"][page, :, position % B] = st["v"]
    st["new_lens"].copy_(st["after"])
    # the means of the blocks that grew: block g of a sequence's grown ones
    block = (st["before"].long() // B)[:, None] + torch.arange(st["grown"], device="cuda")
    held = (st["after"].long()[:, None] - block * B).clamp(0, B)
    block = block.clamp(max=st["width"] - 1)
    s, g = (held > 0).nonzero(as_tuple=True)
    k = st["k_pool"][st["table"].long()[s, block[s, g]]].float()
    k = k * (torch.arange(B, device="cuda") < held[s, g, None])[:, None, :, None]
    st["reps"][s, :, block[s, g]] = k.sum(2) / held[s, g, None, None]
    return dict(q=st["q_out"], k_pool=st["k_pool"], v_pool=st["v_pool"], reps=st["reps"], lens=st["new_lens"])


def _plain_attend(st):
    Hkv, G = st["kv_heads"], st["heads"] // st["kv_heads"]
    n, place, position = _per_token(st, st["after"] - st["q_start"][1:] + st["q_start"][:-1], True)
    S, longest = position.shape
    token = (st["q_start"][:-1].long()[:, None] + place).clamp(max=st["q"].shape[0] - 1)
    q = st["q"].float()[token].view(S, longest, Hkv, G, HEAD_DIM).permute(0, 2, 3, 1, 4).reshape(S, Hkv, G * longest, HEAD_DIM)
    pages = st["table"].long()[:, :st["width"] - SPARE_BLOCKS].clamp(min=0)
    held = torch.arange(pages.shape[1] * st["block"], device="cuda") < st["after"].long()[:, None]           # [S][tokens]
    k, v = (pool[pages].transpose(1, 2).flatten(2, 3).float() * held[:, None, :, None] for pool in (st["k_pool"], st["v_pool"]))
    scores = torch.matmul(q, k.transpose(-1, -2)).div_(math.sqrt(HEAD_DIM)).view(S, Hkv, G, longest, -1)
    hidden = torch.arange(held.shape[1], device="cuda") > position[:, None, None, :, None]
    scores.masked_fill_(hidden, -math.inf)
    scores.sub_(scores.amax(-1, keepdim=True)).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.view(S, Hkv, G * longest, -1), v).view(S, Hkv, G, longest, HEAD_DIM) / total
    out = out.permute(0, 3, 1, 2, 4).reshape(S, longest, st["heads"], HEAD_DIM)
    st["out"].copy_(out[place < n[:, None]])
    return st["out"]


def _warp(logits, temperature, top_k, top_p, min_p):
    """The kept mass of every entry of rows of logits, in vocabulary order, not normalised.  Parameters: one a row, or one."""
    V = logits.shape[-1]
    greedy = (temperature == 0)[:, None]
    x, order = logits.sort(dim=-1, descending=True, stable=True)      # equal ones: the lowest index first
    e = torch.exp((x - x[:, :1]) / torch.where(greedy, torch.ones_like(temperature[:, None]), temperature[:, None]))
    rank = torch.arange(V, device=logits.device)
    keep = torch.ones_like(x, dtype=torch.bool)
    if top_k is not None:
        keep &= rank < top_k[:, None]
    if top_p is not None:
        mass = e * keep
        keep &= (mass.cumsum(-1) - mass) < top_p[:, None] * mass.sum(-1, keepdim=True)
    if min_p is not None:
        keep &= e >= min_p[:, None]
    keep = torch.where(greedy, (rank == 0).expand_as(keep), keep | (rank == 0))
    return torch.zeros_like(e).scatter_(-1, order, e * keep), order


def _plain_sample(st):
    S, T, V = st["logits"].shape
    row = [None if st[k] is None else st[k].repeat_interleave(T) for k in _PARAMETERS]
    kept, _ = _warp(st["logits"].reshape(S * T, V).float(), *row)
    p = kept / kept.sum(-1, keepdim=True)
    cum = p.cumsum(-1)
    reached = (cum >= st["u"][:, None] * cum[:, -1:]) & (p > 0)
    st["tokens"].copy_(reached.int().argmax(-1))
    if not st["dist"]:
        return st["tokens"]
    st["probs"].copy_(p.view(S, T, V))
    return dict(tokens=st["tokens"], probs=st["probs"])


# ------------------------------------------------------------------------------------------------ one pass: this package's calls


def _plan(st):
    """What a serving loop keeps between calls: the descriptors of its cache and the scratch of the attention."""
    import paper_2512_21911_b200 as sv
    if st["op"] != "sample":
        st["geom"] = sv.make_geom(len(st["before"]), st["heads"], st["kv_heads"], HEAD_DIM, st["block"], st["width"], 1)
        st["kv"] = sv.make_kv(st["k_pool"], st["v_pool"], st["table"], st["after"])
    if st["op"] == "attend":
        size = sv.sv_chunk_workspace_bytes(st["geom"], st["q"].shape[0])
        st["workspace"] = torch.empty(max(16, size), dtype=torch.uint8, device="cuda")
    st["sv"] = sv


def _own_run(st):
    if "sv" not in st:
        _plan(st)
    sv = st["sv"]
    if st["op"] == "append":
        sv.sv_rope_append(st["geom"], st["k_pool"], st["v_pool"], st["table"], st["before"], st["q"], st["k"], st["v"], st["q_start"],
                          st["q_out"], st["new_lens"], rope=st["rope"], interleaved=st["interleaved"], reps=st["reps"])
        return dict(q=st["q_out"], k_pool=st["k_pool"], v_pool=st["v_pool"], reps=st["reps"], lens=st["new_lens"])
    if st["op"] == "attend":
        sv.sv_chunk_attn(st["geom"], st["q"], st["kv"], st["q_start"], st["out"], workspace=st["workspace"])
        return st["out"]
    sv.sv_sample(st["logits"], st["u"], st["tokens"], probs=st["probs"], temperature=st["temperature"], top_k=st["top_k"],
                 top_p=st["top_p"], min_p=st["min_p"])
    return dict(tokens=st["tokens"], probs=st["probs"]) if st["dist"] else st["tokens"]


def run(state):
    if own:
        return _own_run(state)
    return dict(append=_plain_append, attend=_plain_attend, sample=_plain_sample)[state["op"]](state)


# ------------------------------------------------------------------------------------------------ what a pass needs, and its exact outputs


def work(case):
    """Bytes and operations of one pass: every input read once, every output written once."""
    Hq, Hkv = case.get("heads"), case.get("kv_heads")
    if case["op"] == "sample":
        entries = case["seqs"] * case["rows"] * case["vocab"]
        return dict(bytes=entries * ((2 if case["half"] else 4) + (4 if case["dist"] else 0)), flops=entries * 4)
    before, new = _lengths(case)
    N, row = sum(new), HEAD_DIM * 2
    if case["op"] == "append":
        B = case["block"]
        grown = sum(-(-(b + n) // B) - b // B for b, n in zip(before, new))
        old = sum(b % B for b in before)                                      # keys that the first of the grown blocks held
        table = case["rot"] * 4 * len({p for b, n in zip(before, new) for p in range(b, b + n)})
        return dict(bytes=2 * N * (Hq + 2 * Hkv) * row + Hkv * (old * row + grown * HEAD_DIM * 4) + table,
                    flops=N * (Hq + Hkv) * case["rot"] * 3)
    pairs = sum(n * b + n * (n + 1) // 2 for b, n in zip(before, new))
    return dict(bytes=2 * N * Hq * row + 2 * Hkv * row * sum(b + n for b, n in zip(before, new)), flops=4 * pairs * Hq * HEAD_DIM)


def _exact_append(case, st):
    B = case["block"]
    before, new = _lengths(case)
    start, half = st["q_start"].tolist(), case["rot"] // 2
    k_pool, v_pool, reps = st["k_pool"].double(), st["v_pool"].double(), st["reps"].double()
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else (slice(0, half), slice(half, 2 * half))

    def turned(x, c, s):
        y = x.clone()
        y[..., first] = x[..., first] * c - x[..., second] * s
        y[..., second] = x[..., second] * c + x[..., first] * s
        return y

    q_out = st["q"].double()
    for s, (b, n) in enumerate(zip(before, new)):
        at = slice(start[s], start[s] + n)
        t = torch.arange(b, b + n, device="cuda")
        c, sn = (st["rope"][b:b + n, i * half:(i + 1) * half].double()[:, None] for i in (0, 1))
        q_out[at] = turned(st["q"][at].double(), c, sn)
        page = st["table"][s].long()[t // B]
        k_pool[page, :, t % B] = turned(st["k"][at].double(), c, sn)
        v_pool[page, :, t % B] = st["v"][at].double()
        for j in range(b // B, -(-(b + n) // B)):
            m = min(B, b + n - j * B)
            # the representative is the mean of the keys that the cache holds, in the cache's type
            reps[s, :, j] = k_pool[int(st["table"][s, j]), :, :m].to(torch.bfloat16).double().mean(1)
    return dict(q=q_out, k_pool=k_pool, v_pool=v_pool, reps=reps, lens=st["after"].clone())


def _exact_attend(case, st):
    B, G = case["block"], case["heads"] // case["kv_heads"]
    before, new = _lengths(case)
    start = st["q_start"].tolist()
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    for s, (b, n) in enumerate(zip(before, new)):
        pages = st["table"][s, :-(-(b + n) // B)].long()
        for h in range(case["kv_heads"]):
            k, v = (pool[pages, h].reshape(-1, HEAD_DIM)[:b + n].double() for pool in (st["k_pool"], st["v_pool"]))
            for at in range(0, n, 512):
                m = min(512, n - at)
                q = st["q"][start[s] + at:start[s] + at + m, h * G:(h + 1) * G].double().reshape(m * G, HEAD_DIM)
                w = q @ k.T / math.sqrt(HEAD_DIM)
                last = b + at + torch.arange(m, device="cuda").repeat_interleave(G)
                w[torch.arange(b + n, device="cuda") > last[:, None]] = -math.inf
                out[start[s] + at:start[s] + at + m, h * G:(h + 1) * G] = (torch.softmax(w, dim=-1) @ v).view(m, G, HEAD_DIM)
    return out


def _exact_sample(case, st):
    S, T, V = st["logits"].shape
    value = lambda name, s: None if st[name] is None else float(st[name][s])   # noqa: E731
    tokens = torch.empty((S * T,), dtype=torch.int32)
    probs = torch.zeros((S, T, V), dtype=torch.float64, device="cuda") if case["dist"] else None
    for s in range(S):
        temperature, k, p, m = (value(name, s) for name in _PARAMETERS)
        for t in range(T):
            x = st["logits"][s, t].double()
            if temperature == 0:
                chosen, e = x.argmax().view(1), torch.ones_like(x)
            else:
                e = torch.exp((x - x.max()) / temperature)
                chosen = torch.argsort(x, descending=True, stable=True)
                if k:
                    chosen = chosen[:int(k)]
                if p is not None:
                    ahead = torch.cat([torch.zeros(1, device="cuda", dtype=torch.float64), e[chosen].cumsum(0)[:-1]])
                    chosen = chosen[:max(1, int((ahead < p * e[chosen].sum()).sum()))]
                if m is not None:
                    chosen = chosen[:max(1, int((e[chosen] >= m).sum()))]
            chosen = chosen.sort().values
            cum = e[chosen].cumsum(0)
            tokens[s * T + t] = int(chosen[int((cum < float(st["u"][s * T + t]) * cum[-1]).sum())])
            if probs is not None:
                probs[s, t, chosen] = e[chosen] / cum[-1]
    return dict(tokens=tokens, probs=probs) if case["dist"] else tokens


def exact(case, seed):
    st = prepare(case, seed)
    return dict(append=_exact_append, attend=_exact_attend, sample=_exact_sample)[case["op"]](case, st)
