"""Performance cases of the operators that keep a long cache small: held in 4 bits, and freed of the tokens that nobody attends to.

  append   new tokens into a 4-bit paged cache: rotary positions, codes and scales, representatives of the blocks that grew; the
           values that the cache then holds for them are read back
  verify   attention of draft tokens (chain or tree) over kept blocks of the 4-bit cache, or all of them, and their own keys
  chunk    causal attention of a ragged batch of new tokens over the 4-bit cache that holds them
  weigh    the attention weight that draft tokens give every cached token, added to what earlier steps gave it
  evict    the tokens of least accumulated weight leave the cache, the others close up in their order

``own`` chooses between the operators' plain form (elementary torch operations in 32 bits, rounded once at the end) and the
calls of this package.

Keys of a case.  All: seqs, lo, hi (tokens of a sequence cached before, uniform in lo..hi), heads (query), kv_heads, block (tokens
of a page).  append and chunk: new_lo, new_hi (new tokens of a sequence), singles (how many of the sequences have one instead);
append: rot (rotated dims of a head), interleaved (pairs are neighbours), fused (q, k and v are slices of one projection's output).
verify and weigh: draft (tokens of a draft), tree (else a chain), keep (kept blocks of a KV head, 0: all).  weigh: accepted (only the
accepted rows count).  evict: budget (the share of the longest sequence's tokens that a sequence may keep), sink, recent (tokens
kept at either end).

Inputs are random with the shape of the real thing: attention logits with a standard deviation of about 3, pages in random
order, accumulated weights over several decades.

A group of 64 values x of a cached row is held as 4-bit codes c, a scale D and an offset M in bfloat16: D = 16 (max - min) / 15,
M = min - D, c = the nearest code of (x - M) 16 / D - 16; it stands for bfloat16((1 + c / 16) D + M).
"""
import math
import random

import torch

own = False

HEAD_DIM = 128
GROUP = 64                   # values that share a scale
SLAB = 9216                  # bytes of 64 tokens of a KV head
SIGMA = math.sqrt(3.0)       # of queries and keys: logits q.k / sqrt(128) then have a standard deviation of 3
THETA = 500000.0             # base of the rotary angles
SPARE_BLOCKS = 2             # entries of the block table behind the blocks in use
ORDER = [0, 4, 1, 5, 2, 6, 3, 7]   # where the eight values of a 32-bit word lie among its nibbles


def _case(op, seqs, lo, hi, heads, kv_heads, block, **more):
    return dict(op=op, seqs=seqs, lo=lo, hi=hi, heads=heads, kv_heads=kv_heads, block=block, **more)


def _append(*shape, new_lo=1, new_hi=1, singles=0, rot=128, interleaved=False, fused=True):
    return _case("append", *shape, new_lo=new_lo, new_hi=new_hi, singles=singles, rot=rot, interleaved=interleaved, fused=fused)


def _verify(*shape, draft=1, tree=False, keep=0):
    return _case("verify", *shape, draft=draft, tree=tree, keep=keep)


def _chunk(*shape, new_lo=1, new_hi=1, singles=0):
    return _case("chunk", *shape, new_lo=new_lo, new_hi=new_hi, singles=singles)


def _weigh(*shape, draft=1, keep=0, accepted=False):
    return _case("weigh", *shape, draft=draft, keep=keep, accepted=accepted)


def _evict(*shape, budget=0.5, sink=4, recent=64):
    return _case("evict", *shape, budget=budget, sink=sink, recent=recent)


def listed():
    return [
        # a decoding step of a batch: one token a sequence
        dict(_append(64, 500, 1500, 32, 8, 64), name="append_64_tokens"),
        # a whole prompt in one piece
        dict(_append(1, 0, 0, 32, 8, 64, new_lo=16384, new_hi=16384), name="append_prompt_16k"),
        # the smallest call: one token of one short sequence on a small model
        dict(_verify(1, 4095, 4095, 8, 2, 64), name="verify_token_4k_small_model"),
        # one request of a 32K context: a chain of eight over the kept 64 blocks of every KV head
        dict(_verify(1, 32768, 32768, 32, 8, 64, draft=8, keep=64), name="verify_32k_kept_64"),
        # four trees of 60 tokens over kept blocks, seven query heads a KV head
        dict(_verify(4, 6001, 20001, 28, 4, 128, draft=60, tree=True, keep=40), name="verify_4_trees_60"),
        # long requests of different lengths, a chain of five each
        dict(_verify(8, 16384, 131072, 32, 8, 64, draft=5), name="verify_8_chains_long"),
        # continuous batching: three chunks of prompts and nine decoding sequences in one call
        dict(_chunk(12, 501, 5001, 28, 4, 128, new_lo=300, new_hi=701, singles=9), name="chunk_ragged_batch"),
        # a later chunk of a long document
        dict(_chunk(1, 30001, 30001, 32, 8, 64, new_lo=1024, new_hi=1024), name="chunk_1k_at_30k"),
        # a step's weights: a chain of eight over 32K tokens, the rows that were accepted
        dict(_weigh(1, 32768, 32768, 32, 8, 64, draft=8, accepted=True), name="weigh_32k_chain8"),
        # a batch over kept blocks
        dict(_weigh(16, 4096, 16384, 32, 8, 64, draft=5, keep=48), name="weigh_16_kept_48"),
        # a long request back to a quarter
        dict(_evict(1, 32768, 32768, 32, 8, 64, budget=0.25), name="evict_32k_to_8k"),
        # a batch of different lengths, the short ones of which stay as they are
        dict(_evict(16, 4001, 16001, 28, 4, 128, budget=0.5), name="evict_16_ragged"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("append", "verify", "chunk", "weigh", "evict")}
    while True:
        op = rng.choice(["append", "verify", "verify", "chunk", "weigh", "evict"])
        heads, kv_heads = rng.choice([(8, 2), (32, 8), (32, 8), (64, 8), (28, 4), (40, 8), (16, 16)])
        block = rng.choice([64, 64, 128])
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 64, 131072) if op in ("verify", "weigh", "evict") else rng.choice([0, _log(rng, 64, 16384), _log(rng, 64, 16384)])
        lo = hi if rng.random() < 0.4 else rng.randint(min(1, hi), hi)
        shape = (seqs, lo, hi, heads, kv_heads, block)
        if op in ("append", "chunk"):
            new_hi = rng.choice([1, _log(rng, 2, 4096), _log(rng, 2, 4096)])
            new_lo = new_hi if rng.random() < 0.4 else rng.randint(1, new_hi)
            more = dict(new_lo=new_lo, new_hi=new_hi, singles=rng.choice([0, rng.randint(0, seqs - 1)]))
            case = _chunk(*shape, **more) if op == "chunk" else _append(*shape, rot=rng.choice([128, 128, 64, 32]), interleaved=rng.random() < 0.4,
                                                                        fused=rng.random() < 0.5, **more)
        elif op == "evict":
            case = _evict(*shape, budget=round(rng.uniform(0.1, 0.9), 2), sink=rng.choice([0, 4, 17]), recent=rng.choice([1, 64, 300]))
        else:
            draft = rng.choice([1, 1, rng.randint(2, 16), rng.randint(17, 64)])
            keep = rng.choice([0, _log(rng, 2, 200)])
            case = _verify(*shape, draft=draft, tree=rng.random() < 0.4, keep=keep) if op == "verify" else \
                _weigh(*shape, draft=draft, keep=keep, accepted=rng.random() < 0.5)
        if _cost(case) <= most[op]:
            return case


def _cost(case):
    """What a case may not exceed the listed ones in: what its plain form holds on the device."""
    before, new = _lengths(case)
    if case["op"] == "append":
        return sum(new) * (case["heads"] + 2 * case["kv_heads"]) + sum(before) * case["kv_heads"] // 4
    if case["op"] == "chunk":
        return case["seqs"] * case["heads"] * max(new) * (max(b + n for b, n in zip(before, new)) + 64)
    if case["op"] == "evict":
        return case["seqs"] * case["kv_heads"] * max(before)
    return case["seqs"] * (case["heads"] * case["draft"] + 256 * case["kv_heads"]) * max(before)


def _lengths(case):
    """Tokens cached before and new tokens of every sequence: the case's own, whatever the seed."""
    rng = random.Random(str(sorted((k, v) for k, v in case.items() if k != "name")))
    before = [rng.randint(case["lo"], case["hi"]) for _ in range(case["seqs"])]
    new = [rng.randint(case.get("new_lo", 0), case.get("new_hi", 0)) for _ in range(case["seqs"])]
    for s in rng.sample(range(case["seqs"]), case.get("singles", 0)):
        new[s] = 1
    return before, new


# ------------------------------------------------------------------------------------------------ the cache's format


def _fit(x):
    """Codes of rows of values [...][128], and the scales and offsets of their groups [...][2], as they are held."""
    g = x.float().unflatten(-1, (-1, GROUP))
    low, high = g.amin(-1), g.amax(-1)
    scale = (16.0 * (high - low) / 15.0).to(torch.bfloat16)
    offset = (low - scale.float()).to(torch.bfloat16)
    d = scale.float().unsqueeze(-1)
    c = torch.where(d > 0, ((g - offset.float().unsqueeze(-1)) * 16.0 / d - 16.0).round(), torch.zeros_like(g))
    return c.clamp_(0, 15).flatten(-2).to(torch.uint8), scale, offset


def _value(codes, scale, offset):
    """What codes [...][groups][n] with scales and offsets [...][groups][1 or n] stand for."""
    return ((1.0 + codes.float() / 16.0) * scale.float() + offset.float()).to(torch.bfloat16)


def _words(codes):
    """Codes [...][32 n] as bytes [...][16 n]."""
    c = codes.unflatten(-1, (-1, 8))[..., [0, 2, 4, 6, 1, 3, 5, 7]].unflatten(-1, (4, 2))
    return (c[..., 0] | (c[..., 1] << 4)).flatten(-2)


def _codes(words):
    """... and back."""
    nibbles = torch.stack([words & 15, words >> 4], dim=-1).flatten(-2)
    return nibbles.unflatten(-1, (-1, 8))[..., ORDER].flatten(-2)


def _pack(k, v):
    """Slabs of 64 tokens: k, v [...][64][128] -> bytes [...][SLAB]."""
    kc, ks, ko = _fit(k)
    vc, vs, vo = _fit(v)
    k_part = _words(kc).unflatten(-1, (4, 16)).transpose(-2, -3).flatten(-3)                       # [chunk of 32 dims][token][16]
    v_part = _words(vc.transpose(-1, -2)).unflatten(-1, (2, 16)).transpose(-2, -3).flatten(-3)     # [chunk of 32 tokens][dim][16]
    k_scale = torch.stack([ks, ko], dim=-1).flatten(-3).contiguous().view(torch.uint8)             # [token][group][scale, offset]
    v_scale = torch.stack([vs, vo], dim=-1).movedim(-3, -1).flatten(-3).contiguous().view(torch.uint8)   # [group][scale, offset][token]
    return torch.cat([k_part, v_part, k_scale, v_scale], dim=-1)


def _unpack(slabs):
    """What slabs [...][SLAB] stand for: k, v [...][64][128] in bfloat16."""
    kc = _codes(slabs[..., :4096].unflatten(-1, (4, 64, 16))).transpose(-2, -3).flatten(-2)
    vc = _codes(slabs[..., 4096:8192].unflatten(-1, (2, 128, 16))).transpose(-2, -3).flatten(-2).transpose(-1, -2)
    ks = slabs[..., 8192:8704].contiguous().view(torch.bfloat16).unflatten(-1, (64, 2, 2))
    vs = slabs[..., 8704:9216].contiguous().view(torch.bfloat16).unflatten(-1, (2, 2, 64)).movedim(-1, -3)
    return tuple(_value(c.unflatten(-1, (2, GROUP)), s[..., :1], s[..., 1:]).flatten(-2) for c, s in ((kc, ks), (vc, vs)))


# ------------------------------------------------------------------------------------------------ inputs


def _normal(gen, *shape, sigma=1.0):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, sigma, generator=gen)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, S, B, Hq, Hkv = case["op"], case["seqs"], case["block"], case["heads"], case["kv_heads"]
    before, new = _lengths(case)
    blocks = [-(-(b + n) // B) for b, n in zip(before, new)]
    width = max(blocks) + SPARE_BLOCKS
    pages = torch.randperm(sum(blocks) + 1, generator=torch.Generator().manual_seed(seed)).int()
    row, col = torch.repeat_interleave(torch.arange(S), torch.tensor(blocks)), torch.cat([torch.arange(n) for n in blocks])
    table = torch.full((S, width), -1, dtype=torch.int32)
    table[row, col] = pages[:sum(blocks)]
    st = dict(op=op, heads=Hq, kv_heads=Hkv, block=B, width=width, table=table.cuda(), before=_ints(before), most=max(before),
              draft=case.get("draft", 1))
    k_pool = _normal(gen, len(pages), Hkv, B, HEAD_DIM, sigma=SIGMA)
    v_pool = _normal(gen, len(pages), Hkv, B, HEAD_DIM)
    if op in ("weigh", "evict"):
        st.update(k_pool=k_pool, v_pool=v_pool)
    else:
        st["pool"] = torch.empty((len(pages), Hkv, B // 64, SLAB), dtype=torch.uint8, device="cuda")
        for at in range(0, len(pages), 256):
            k, v = (x[at:at + 256].unflatten(2, (B // 64, 64)) for x in (k_pool, v_pool))
            st["pool"][at:at + 256] = _pack(k, v)
        del k_pool, v_pool
    if op in ("append", "chunk"):
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        N = starts[-1]
        st.update(q_start=_ints(starts), after=_ints([b + n for b, n in zip(before, new)]), longest=max(new))
        if op == "chunk":
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
        st["grown"] = max(-(-(b + n) // B) - b // B for b, n in zip(before, new))
        st["q_out"] = torch.empty((N, Hq, HEAD_DIM), dtype=torch.bfloat16, device="cuda")
        st["k_out"], st["v_out"] = (torch.empty((N, Hkv, HEAD_DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        st["new_lens"] = torch.empty_like(st["before"])
        st["reps"] = torch.zeros((S, Hkv, width, HEAD_DIM), device="cuda")
        return st
    if op == "evict":
        st["weights"] = torch.randn((S, Hkv, width * B), generator=gen, device="cuda").mul_(2.0).exp_()
        budget = max(1, int(case["budget"] * max(before)))
        st.update(budget=torch.full((S,), budget, dtype=torch.int32, device="cuda"), sink=case["sink"], recent=case["recent"], room=budget,
                  new_lens=torch.empty_like(st["before"]), new_weights=torch.zeros_like(st["weights"]),
                  reps=torch.zeros((S, Hkv, width, HEAD_DIM), device="cuda"))
        return st
    T = case["draft"]
    st["q"] = _normal(gen, S, T, Hq, HEAD_DIM, sigma=SIGMA)
    st["lists"] = None
    if case["keep"]:
        # the first and the last block and the likeliest of the others, an independent draw for every KV head
        n_blocks = _ints([-(-b // B) for b in before]).long()
        score = torch.rand((S, Hkv, width), generator=gen, device="cuda")
        place = torch.arange(width, device="cuda")
        score = torch.where((place == 0) | (place == n_blocks[:, None, None] - 1), 2.0, score)
        score = torch.where(place < n_blocks[:, None, None], score, -1.0)
        count = n_blocks.clamp(max=case["keep"])[:, None].expand(S, Hkv)
        kept = score.argsort(dim=-1, descending=True, stable=True)[..., :case["keep"]]
        kept = torch.where(torch.arange(kept.shape[-1], device="cuda") < count[..., None], kept, width).sort(dim=-1).values
        st["lists"] = (torch.where(kept < width, kept, 0).int().contiguous(), count.int().contiguous())
    if op == "verify":
        st["draft_k"], st["draft_v"] = _normal(gen, S, T, Hkv, HEAD_DIM, sigma=SIGMA), _normal(gen, S, T, Hkv, HEAD_DIM)
        st["parent"] = None
        if case["tree"]:
            rng = random.Random(seed)
            st["parent"] = _ints([[-1] + [rng.randint(max(0, i - 12), i - 1) for i in range(1, T)] for _ in range(S)])
        st["sees"] = _visible(st)
        st["out"], st["lse"] = torch.empty_like(st["q"]), torch.empty((S, T, Hq), device="cuda")
        return st
    # weigh: the denominators that the attention returned, over the tokens that it went over and its own
    n_path = [random.Random(seed + s).randint(1, T) for s in range(S)] if case["accepted"] else [T] * S
    path = torch.full((S, T), -1, dtype=torch.int32)
    for s, n in enumerate(n_path):
        path[s, :n] = torch.arange(n, dtype=torch.int32)
    st["path"], st["n_path"] = (path.cuda(), _ints(n_path)) if case["accepted"] else (None, None)
    scores, _ = _scores(st)
    own_keys = torch.randn(scores.shape[:-1], generator=gen, device="cuda")
    lse = torch.logaddexp(torch.logsumexp(scores, dim=-1), own_keys)                              # [S][Hkv][T][G]
    st["lse"] = lse.permute(0, 2, 1, 3).reshape(S, T, Hq).contiguous()
    st["weights"] = torch.rand((S, Hkv, width * B), generator=gen, device="cuda")
    st["new_weights"] = torch.zeros_like(st["weights"])
    return st


def _visible(st):
    """Which of the draft tokens j a draft token i sees: [S][T][T]."""
    S, T = st["q"].shape[:2]
    if st["parent"] is None:
        return torch.ones((T, T), dtype=torch.bool, device="cuda").tril().expand(S, T, T)
    sees = torch.eye(T, dtype=torch.bool, device="cuda").repeat(S, 1, 1)
    for i in range(1, T):
        sees[:, i] |= sees[torch.arange(S, device="cuda"), st["parent"][:, i].long()]
    return sees


# ------------------------------------------------------------------------------------------------ one pass: the plain forms


def _blocks_of(st):
    """The blocks that every KV head goes over: indices [S][Hkv][n], and which of their tokens are there [S][Hkv][n][B]."""
    S, B = len(st["before"]), st["block"]
    if st["lists"] is None:
        n = st["width"] - SPARE_BLOCKS
        index = torch.arange(n, device="cuda").expand(S, st["kv_heads"], n)
        real = torch.ones_like(index, dtype=torch.bool)
    else:
        index = st["lists"][0].long()
        real = torch.arange(index.shape[-1], device="cuda") < st["lists"][1][..., None]
    token = index[..., None] * B + torch.arange(B, device="cuda")
    return index, real[..., None] & (token < st["before"].long()[:, None, None, None])


def _scores(st):
    """Logits of every draft row and cached token that is gone over, -inf where there is none: [S][Hkv][T][G][tokens]; its blocks."""
    S, T = st["q"].shape[:2]
    Hkv, G = st["kv_heads"], st["heads"] // st["kv_heads"]
    index, there = _blocks_of(st)
    page = st["table"].long().clamp(min=0)[torch.arange(S, device="cuda")[:, None, None], index]
    head = torch.arange(Hkv, device="cuda")[None, :, None]
    if st["op"] == "weigh":
        k, v = st["k_pool"][page, head], None
    else:
        k, v = _unpack(st["pool"][page, head])
        k, v = k.flatten(3, 4), v.flatten(3, 4)
    q = st["q"].float().view(S, T, Hkv, G, HEAD_DIM).permute(0, 2, 1, 3, 4).reshape(S, Hkv, T * G, HEAD_DIM)
    scores = torch.matmul(q, k.flatten(2, 3).float().transpose(-1, -2)).div_(math.sqrt(HEAD_DIM))
    scores.masked_fill_(~there.flatten(2)[:, :, None], -math.inf)
    return scores.view(S, Hkv, T, G, -1), (index, there, v)


def _plain_verify(st):
    S, T = st["q"].shape[:2]
    Hkv, G = st["kv_heads"], st["heads"] // st["kv_heads"]
    scores, (_, there, v) = _scores(st)
    v = v.flatten(2, 3).float() * there.flatten(2)[..., None]
    q = st["q"].float().view(S, T, Hkv, G, HEAD_DIM)
    drafted = torch.einsum("sihgd,sjhd->shigj", q, st["draft_k"].float()) / math.sqrt(HEAD_DIM)
    drafted.masked_fill_(~st["sees"][:, None, :, None], -math.inf)
    top = torch.maximum(scores.amax(-1, keepdim=True), drafted.amax(-1, keepdim=True))
    scores, drafted = scores.sub_(top).exp_(), (drafted - top).exp()
    total = scores.sum(-1, keepdim=True) + drafted.sum(-1, keepdim=True)
    out = torch.matmul(scores.flatten(2, 3), v).view(S, Hkv, T, G, HEAD_DIM) + torch.einsum("shigj,sjhd->shigd", drafted, st["draft_v"].float())
    st["out"].copy_((out / total).permute(0, 2, 1, 3, 4).reshape(S, T, st["heads"], HEAD_DIM))
    st["lse"].copy_((top + total.log())[..., 0].permute(0, 2, 1, 3).reshape(S, T, st["heads"]))
    return dict(out=st["out"], lse=st["lse"])


def _plain_weigh(st):
    S, T = st["q"].shape[:2]
    Hkv, G, B = st["kv_heads"], st["heads"] // st["kv_heads"], st["block"]
    scores, (index, there, _) = _scores(st)
    scores.sub_(st["lse"].view(S, T, Hkv, G).permute(0, 2, 1, 3)[..., None]).exp_()
    if st["path"] is not None:
        counts = torch.zeros((S, T + 1), dtype=torch.bool, device="cuda")
        counts.scatter_(1, torch.where(torch.arange(T, device="cuda") < st["n_path"][:, None], st["path"], T).long(), True)
        scores.mul_(counts[:, None, :T, None, None])
    given = scores.sum(dim=(2, 3))                                                                # [S][Hkv][tokens]
    token = (index[..., None] * B + torch.arange(B, device="cuda")).flatten(2)
    there = there.flatten(2)
    spare = st["weights"].shape[-1] - 1                                                           # (a slot behind every sequence's end)
    added = torch.zeros_like(st["weights"]).scatter_(2, torch.where(there, token, spare), given * there)
    held = torch.arange(spare + 1, device="cuda") < st["before"][:, None, None]
    st["new_weights"].copy_(torch.where(held, st["weights"] + added, st["new_weights"]))
    return st["new_weights"]


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
    st["new_lens"].copy_(st["after"])
    # the blocks that grew, of every sequence: what they held (as it is) and the new tokens, each coded for itself
    block = (st["before"].long() // B)[:, None] + torch.arange(st["grown"], device="cuda")
    held = (st["after"].long()[:, None] - block * B).clamp(0, B)
    block = block.clamp(max=st["width"] - 1)
    s, g = (held > 0).nonzero(as_tuple=True)
    page = st["table"].long()[s, block[s, g]]
    position_in = block[s, g][:, None] * B + torch.arange(B, device="cuda")                      # [grown][B]
    fresh = (position_in >= st["before"].long()[s][:, None]) & (torch.arange(B, device="cuda") < held[s, g][:, None])
    row = (st["q_start"][:-1].long()[s][:, None] + position_in - st["before"].long()[s][:, None]).clamp(0, st["q"].shape[0] - 1)
    k = _rotate(st["k"], cos[:, None], sin[:, None], st["interleaved"])[row].transpose(1, 2)     # [grown][Hkv][B][128]
    v = st["v"][row].transpose(1, 2)
    coded = _pack(k.unflatten(2, (B // 64, 64)), v.unflatten(2, (B // 64, 64)))
    st["pool"][page] = _merge(st["pool"][page], coded, fresh.unflatten(1, (B // 64, 64))[:, None])
    k, v = (x.flatten(2, 3) for x in _unpack(st["pool"][page]))
    mean = (k.float() * (torch.arange(B, device="cuda") < held[s, g, None])[:, None, :, None]).sum(2) / held[s, g, None, None]
    st["reps"][s, :, block[s, g]] = mean
    st["k_out"][row[fresh]] = k.transpose(1, 2)[fresh]
    st["v_out"][row[fresh]] = v.transpose(1, 2)[fresh]
    return dict(q=st["q_out"], k=st["k_out"], v=st["v_out"], reps=st["reps"], lens=st["new_lens"])


def _merge(old, new, fresh):
    """Slabs with the tokens that are fresh [...][64] from `new` and the others from `old`."""
    # a token's bytes: of the keys whole ones, of the values one nibble of every word of its 32 tokens, of their scales two bytes a group
    f = fresh.to(torch.uint8) * 255
    k_mask = f[..., None, :, None].expand(*f.shape[:-1], 4, 64, 16).flatten(-3)
    v_mask = _words((f & 15).unflatten(-1, (2, 1, 32)).expand(*f.shape[:-1], 2, 128, 32)).flatten(-3)
    k_scale = f[..., None].expand(*f.shape, 8).flatten(-2)
    v_scale = f[..., None, :, None].expand(*f.shape[:-1], 4, 64, 2).flatten(-3)
    mask = torch.cat([k_mask, v_mask, k_scale, v_scale], dim=-1)
    return (old & ~mask) | (new & mask)


def _plain_chunk(st):
    Hkv, G = st["kv_heads"], st["heads"] // st["kv_heads"]
    n, place, position = _per_token(st, st["before"], True)
    S, longest = position.shape
    token = (st["q_start"][:-1].long()[:, None] + place).clamp(max=st["q"].shape[0] - 1)
    q = st["q"].float()[token].view(S, longest, Hkv, G, HEAD_DIM).permute(0, 2, 3, 1, 4).reshape(S, Hkv, G * longest, HEAD_DIM)
    pages = st["table"].long()[:, :st["width"] - SPARE_BLOCKS].clamp(min=0)
    held = torch.arange(pages.shape[1] * st["block"], device="cuda") < st["after"].long()[:, None]           # [S][tokens]
    k, v = (x.flatten(3, 4).transpose(1, 2).flatten(2, 3).float() * held[:, None, :, None] for x in _unpack(st["pool"][pages]))
    scores = torch.matmul(q, k.transpose(-1, -2)).div_(math.sqrt(HEAD_DIM)).view(S, Hkv, G, longest, -1)
    scores.masked_fill_(torch.arange(held.shape[1], device="cuda") > position[:, None, None, :, None], -math.inf)
    scores.sub_(scores.amax(-1, keepdim=True)).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.view(S, Hkv, G * longest, -1), v).view(S, Hkv, G, longest, HEAD_DIM) / total
    out = out.permute(0, 3, 1, 2, 4).reshape(S, longest, st["heads"], HEAD_DIM)
    st["out"].copy_(out[place < n[:, None]])
    return st["out"]


def _plain_evict(st):
    B, Hkv = st["block"], st["kv_heads"]
    S, most = len(st["before"]), st["most"]
    length = st["before"].long()[:, None, None]
    token = torch.arange(most, device="cuda")
    ends = (token < st["sink"]) | (token >= length - st["recent"])
    kept_len = torch.minimum(length, torch.maximum(st["budget"].long()[:, None, None], torch.clamp(length, max=st["sink"] + st["recent"])))
    weight = st["weights"][..., :most].masked_fill(ends, math.inf).masked_fill(token >= length, -math.inf)
    order = weight.argsort(dim=-1, descending=True, stable=True)                                 # equal ones: the earlier first
    source = torch.where(token < kept_len, order, most).sort(dim=-1).values                      # ascending, then nothing
    real = source < most
    source = source.clamp(max=most - 1)
    s, h = torch.arange(S, device="cuda")[:, None, None], torch.arange(Hkv, device="cuda")[:, None]
    page = st["table"].long()
    moved = [pool[page[s, source // B], h, source % B] for pool in (st["k_pool"], st["v_pool"])]
    to = (page[s, token // B].expand(S, Hkv, most)[real], h.expand(S, Hkv, most)[real], (token % B).expand(S, Hkv, most)[real])
    for pool, rows in zip((st["k_pool"], st["v_pool"]), moved):
        pool[to] = rows[real]
    st["new_lens"].copy_(kept_len[:, 0, 0])
    gathered = st["weights"].gather(2, source) * real
    st["new_weights"][..., :most] = torch.where(token < length, gathered, st["new_weights"][..., :most])
    blocks = -(-most // B)
    k = torch.nn.functional.pad(moved[0].float() * real[..., None], (0, 0, 0, blocks * B - most)).unflatten(2, (blocks, B))
    held = (kept_len[..., 0, None] - torch.arange(blocks, device="cuda")[:, None] * B).clamp(0, B)         # [S][blocks][1]
    held = held.view(S, 1, blocks, 1).expand(S, Hkv, blocks, HEAD_DIM) * (kept_len < length)[..., None]    # (only of those that lose tokens)
    st["reps"][:, :, :blocks] = torch.where(held > 0, k.sum(3) / held.clamp(min=1), st["reps"][:, :, :blocks])
    return dict(k_pool=st["k_pool"], v_pool=st["v_pool"], weights=st["new_weights"], reps=st["reps"], lens=st["new_lens"])


# ------------------------------------------------------------------------------------------------ one pass: this package's calls


def _plan(st):
    """What a serving loop keeps between calls: the descriptors of its cache and the scratch of the attention."""
    import paper_2512_21911_b200 as sv
    st["geom"] = sv.make_geom(len(st["before"]), st["heads"], st["kv_heads"], HEAD_DIM, st["block"], st["width"], st["draft"])
    if st["op"] in ("append", "chunk"):
        st["kv"] = sv.make_kv_q4(st["pool"], st["table"], st["after"])
    elif st["op"] == "verify":
        st["kv"] = sv.make_kv_q4(st["pool"], st["table"], st["before"])
    else:
        st["kv"] = sv.make_kv(st["k_pool"], st["v_pool"], st["table"], st["before"])
    if st["op"] in ("verify", "chunk"):
        size = sv.sv_workspace_bytes_q4(st["geom"])
        st["workspace"] = torch.empty(max(16, size), dtype=torch.uint8, device="cuda")
    st["sv"] = sv


def _own_run(st):
    if "sv" not in st:
        _plan(st)
    sv = st["sv"]
    if st["op"] == "append":
        sv.sv_rope_append_q4(st["geom"], st["pool"], st["table"], st["before"], st["q"], st["k"], st["v"], st["q_start"], st["q_out"],
                             st["new_lens"], rope=st["rope"], interleaved=st["interleaved"], reps=st["reps"])
        sv.sv_kv_read_q4(st["geom"], st["kv"], st["before"], st["q_start"], st["k_out"], st["v_out"])
        return dict(q=st["q_out"], k=st["k_out"], v=st["v_out"], reps=st["reps"], lens=st["new_lens"])
    if st["op"] == "chunk":
        sv.sv_chunk_attn_q4(st["geom"], st["q"], st["kv"], st["q_start"], st["out"], workspace=st["workspace"])
        return st["out"]
    if st["op"] == "evict":
        sv.sv_kv_evict(st["geom"], st["k_pool"], st["v_pool"], st["table"], st["before"], st["weights"], st["budget"], st["sink"], st["recent"],
                       st["new_lens"], st["new_weights"], reps=st["reps"])
        return dict(k_pool=st["k_pool"], v_pool=st["v_pool"], weights=st["new_weights"], reps=st["reps"], lens=st["new_lens"])
    idx, cnt = st["lists"] or (None, None)
    if st["op"] == "weigh":
        sv.sv_attn_weights(st["geom"], st["q"], st["kv"], st["lse"], st["weights"], st["new_weights"], sel_idx=idx, sel_cnt=cnt, path=st["path"],
                           n_path=st["n_path"])
        return st["new_weights"]
    sv.sv_verify_attn_q4(st["geom"], st["q"], st["kv"], st["draft_k"], st["draft_v"], st["parent"], idx, cnt, st["out"], lse=st["lse"],
                         workspace=st["workspace"])
    return dict(out=st["out"], lse=st["lse"])


def run(state):
    if own:
        return _own_run(state)
    return dict(append=_plain_append, verify=_plain_verify, chunk=_plain_chunk, weigh=_plain_weigh, evict=_plain_evict)[state["op"]](state)


# ------------------------------------------------------------------------------------------------ what a pass needs, and its exact outputs


def work(case):
    """Bytes and operations of one pass: every input read once, every output written once."""
    Hq, Hkv, S, B = case["heads"], case["kv_heads"], case["seqs"], case["block"]
    before, new = _lengths(case)
    row, small = HEAD_DIM * 2, SLAB // 64
    N = sum(new)
    if case["op"] == "append":
        grown = sum(-(-(b + n) // B) - b // B for b, n in zip(before, new))
        old = sum(b % B for b in before)                                      # tokens that the first of the grown blocks held
        table = case["rot"] * 4 * len({p for b, n in zip(before, new) for p in range(b, b + n)})
        return dict(bytes=2 * N * Hq * row + N * Hkv * (4 * row + 2 * small) + Hkv * (old * small // 2 + grown * HEAD_DIM * 4) + table,
                    flops=N * (Hq + Hkv) * case["rot"] * 3 + N * Hkv * HEAD_DIM * 12)
    if case["op"] == "chunk":
        pairs = sum(n * b + n * (n + 1) // 2 for b, n in zip(before, new))
        return dict(bytes=2 * N * Hq * row + Hkv * small * sum(b + n for b, n in zip(before, new)), flops=4 * pairs * Hq * HEAD_DIM)
    if case["op"] == "evict":
        budget = max(1, int(case["budget"] * max(before)))
        left = [min(b, max(budget, min(b, case["sink"] + case["recent"]))) for b in before]
        moved = sum(n for b, n in zip(before, left) if n < b)
        return dict(bytes=Hkv * (4 * moved * row + 4 * sum(before) * 2 + sum(-(-n // B) for b, n in zip(before, left) if n < b) * HEAD_DIM * 4), flops=Hkv * sum(before) * 8)
    T = case["draft"]
    gone_over = [min(b, case["keep"] * B) if case["keep"] else b for b in before]
    if case["op"] == "weigh":
        rows = S * T * Hq
        return dict(bytes=Hkv * row * sum(gone_over) + 8 * Hkv * sum(before) + rows * (row + 4), flops=2 * sum(gone_over) * T * Hq * HEAD_DIM)
    return dict(bytes=Hkv * small * sum(gone_over) + S * T * (2 * Hq * row + 2 * Hkv * row + 4 * Hq),
                flops=4 * (sum(gone_over) + S * T / 2) * T * Hq * HEAD_DIM)


def _coded(x):
    """Rows [n][128] in 64 bits as a 4-bit cache holds them: the values that the codes stand for."""
    g = x.double().reshape(-1, GROUP)
    low, high = g.min(1, keepdim=True).values, g.max(1, keepdim=True).values
    scale = (16 * (high - low) / 15).to(torch.bfloat16).double()
    offset = (low - scale).to(torch.bfloat16).double()
    code = torch.nan_to_num(((g - offset) * 16 / scale - 16).round(), nan=0.0).clamp(0, 15)
    return ((1 + code / 16) * scale + offset).to(torch.bfloat16).double().reshape(x.shape)


def _held(pool, page, h, block):
    """Keys and values of a KV head on pages of a 4-bit cache, in 64 bits, nibble by nibble: [n * block][128] each."""
    slab = pool[page, h].reshape(-1, SLAB).long()
    at = torch.arange(HEAD_DIM, device="cuda")
    t = torch.arange(64, device="cuda")

    def nibble(first, word, within):                                         # value `within` of 8 of a 32-bit word: byte and half of it
        n = torch.where(within % 2 == 0, within // 2, 4 + within // 2)
        return slab[:, first + 4 * word + n // 2] >> (4 * (n % 2)) & 15

    def number(first, place):
        raw = slab[:, first + 2 * place] | slab[:, first + 2 * place + 1] << 8
        return (raw << 16).to(torch.int32).view(torch.float32).double()

    tt, dd = torch.meshgrid(t, at, indexing="ij")
    k_code = nibble(0, ((dd // 32 * 64 + tt) * 4 + dd % 32 // 8), dd % 8)
    v_code = nibble(4096, ((tt // 32 * 128 + dd) * 4 + tt % 32 // 8), tt % 8)
    k = (1 + k_code.double() / 16) * number(8192, tt * 4 + dd // 64 * 2) + number(8192, tt * 4 + dd // 64 * 2 + 1)
    v = (1 + v_code.double() / 16) * number(8704, dd // 64 * 128 + tt) + number(8704, dd // 64 * 128 + 64 + tt)
    return tuple(x.to(torch.bfloat16).double().reshape(-1, HEAD_DIM) for x in (k, v))


def _exact_append(case, st):
    B = case["block"]
    before, new = _lengths(case)
    start, half = st["q_start"].tolist(), case["rot"] // 2
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else (slice(0, half), slice(half, 2 * half))

    def turned(x, c, s, steps=lambda y: y):
        y = x.clone()
        y[..., first] = steps(steps(x[..., first] * c) - steps(x[..., second] * s))
        y[..., second] = steps(steps(x[..., second] * c) + steps(x[..., first] * s))
        return y

    q_out, reps = st["q"].double(), st["reps"].double()
    k_out, v_out = torch.empty_like(st["k_out"], dtype=torch.float64), torch.empty_like(st["v_out"], dtype=torch.float64)
    for s, (b, n) in enumerate(zip(before, new)):
        at = slice(start[s], start[s] + n)
        c, sn = (st["rope"][b:b + n, i * half:(i + 1) * half].double()[:, None] for i in (0, 1))
        q_out[at] = turned(st["q"][at].double(), c, sn)
        # the keys that are coded are rounded ones, by the definition: products and sums to 32 bits, the result to the model's type
        k_out[at] = _coded(turned(st["k"][at].double(), c, sn, lambda y: y.float().double()).to(torch.bfloat16))
        v_out[at] = _coded(st["v"][at])
        for h in range(case["kv_heads"]):
            k_old = _held(st["pool"], st["table"][s, b // B:b // B + 1].long().clamp(min=0), h, B)[0][:b % B]
            k = torch.cat([k_old, k_out[at, h]])
            for j in range(-(-len(k) // B)):
                reps[s, h, b // B + j] = k[j * B:(j + 1) * B].mean(0)
    return dict(q=q_out, k=k_out, v=v_out, reps=reps, lens=st["after"].clone())


def _exact_chunk(case, st):
    B, G = case["block"], case["heads"] // case["kv_heads"]
    before, new = _lengths(case)
    start = st["q_start"].tolist()
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    for s, (b, n) in enumerate(zip(before, new)):
        pages = st["table"][s, :-(-(b + n) // B)].long()
        for h in range(case["kv_heads"]):
            k, v = (x[:b + n] for x in _held(st["pool"], pages, h, B))
            for at in range(0, n, 512):
                m = min(512, n - at)
                q = st["q"][start[s] + at:start[s] + at + m, h * G:(h + 1) * G].double().reshape(m * G, HEAD_DIM)
                w = q @ k.T / math.sqrt(HEAD_DIM)
                last = b + at + torch.arange(m, device="cuda").repeat_interleave(G)
                w[torch.arange(b + n, device="cuda") > last[:, None]] = -math.inf
                out[start[s] + at:start[s] + at + m, h * G:(h + 1) * G] = (torch.softmax(w, dim=-1) @ v).view(m, G, HEAD_DIM)
    return out


def _tokens(case, st, s, h):
    """The tokens of a sequence that a KV head goes over, in 64-bit indices."""
    B, b = case["block"], _lengths(case)[0][s]
    if st["lists"] is None:
        return torch.arange(b, device="cuda")
    kept = st["lists"][0][s, h, :int(st["lists"][1][s, h])].long()
    t = (kept[:, None] * B + torch.arange(B, device="cuda")).reshape(-1)
    return t[t < b]


def _exact_verify(case, st):
    B, G, T = case["block"], case["heads"] // case["kv_heads"], case["draft"]
    out, lse = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda"), torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
    for s, b in enumerate(_lengths(case)[0]):
        for h in range(case["kv_heads"]):
            t = _tokens(case, st, s, h)
            k, v = _held(st["pool"], st["table"][s, :-(-b // B)].long(), h, B)
            k, v = torch.cat([k[t], st["draft_k"][s, :, h].double()]), torch.cat([v[t], st["draft_v"][s, :, h].double()])
            for i in range(T):
                w = st["q"][s, i, h * G:(h + 1) * G].double() @ k.T / math.sqrt(HEAD_DIM)
                w[:, len(t):][:, ~st["sees"][s, i]] = -math.inf
                out[s, i, h * G:(h + 1) * G] = torch.softmax(w, dim=-1) @ v
                lse[s, i, h * G:(h + 1) * G] = torch.logsumexp(w, dim=-1)
    return dict(out=out, lse=lse)


def _exact_weigh(case, st):
    B, G, T = case["block"], case["heads"] // case["kv_heads"], case["draft"]
    weights = st["new_weights"].double()
    for s, b in enumerate(_lengths(case)[0]):
        rows = list(range(T)) if st["path"] is None else st["path"][s, :int(st["n_path"][s])].tolist()
        pages = st["table"][s, :-(-b // B)].long()
        for h in range(case["kv_heads"]):
            weights[s, h, :b] = st["weights"][s, h, :b]
            t = _tokens(case, st, s, h)
            k = st["k_pool"][pages, h].reshape(-1, HEAD_DIM)[t].double()
            for i in rows:
                w = st["q"][s, i, h * G:(h + 1) * G].double() @ k.T / math.sqrt(HEAD_DIM)
                weights[s, h, t] += torch.exp(w - st["lse"][s, i, h * G:(h + 1) * G].double()[:, None]).sum(0)
    return weights


def _exact_evict(case, st):
    B, budget = case["block"], st["room"]
    k_pool, v_pool = st["k_pool"].double(), st["v_pool"].double()
    reps, weights, lens = st["reps"].double(), st["new_weights"].double(), []
    for s, b in enumerate(_lengths(case)[0]):
        n = min(b, max(budget, min(b, case["sink"] + case["recent"])))
        lens.append(n)
        page = st["table"][s, torch.arange(b, device="cuda") // B].long()
        slot = torch.arange(b, device="cuda") % B
        for h in range(case["kv_heads"]):
            w = st["weights"][s, h, :b].double().clone()
            w[:case["sink"]] = math.inf
            w[max(0, b - case["recent"]):] = math.inf
            kept = torch.argsort(w, descending=True, stable=True)[:n].sort().values
            for pool in (k_pool, v_pool):
                pool[page[:n], h, slot[:n]] = pool[page[kept], h, slot[kept]]
            weights[s, h, :b] = 0.0
            weights[s, h, :n] = st["weights"][s, h, kept].double()
            k = k_pool[page[:n], h, slot[:n]]
            for j in range(-(-n // B) if n < b else 0):
                reps[s, h, j] = k[j * B:(j + 1) * B].mean(0)
    return dict(k_pool=k_pool, v_pool=v_pool, weights=weights, reps=reps, lens=_ints(lens))


def exact(case, seed):
    if case["op"] == "verify" and case["seqs"] * case["draft"] * case["kv_heads"] > 20000:
        return None
    st = prepare(case, seed)
    return dict(append=_exact_append, verify=_exact_verify, chunk=_exact_chunk, weigh=_exact_weigh, evict=_exact_evict)[case["op"]](case, st)
