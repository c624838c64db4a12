"""A serving loop around sparse verification, on a small decoder with random weights: the prompts go into the paged cache in
chunks, the first token is drawn from the last prompt token's logits, and then every step drafts a few tokens, verifies them in one
pass over the kept blocks, accepts a prefix and commits it to the cache.

    python examples/generate.py [--prompt 3000 700] [--new 32] [--layers 4] [--four-bits | --most-tokens 1000]

With --four-bits the cache is held in 4 bits; with --most-tokens a sequence that has more loses, between steps, those that the steps gave least
attention to, down to three quarters.

The draft model is the target's embedding and head without its layers.  Prompts, weights and random numbers are seeded."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2512_21911_b200 as sv  # noqa: E402

HEADS, KV_HEADS, DIM, WIDTH, VOCAB, BLOCK, DRAFT, THETA = 8, 2, 128, 512, 2048, 64, 5, 10000.0


class Decoder:
    def __init__(self, layers, longest, gen):
        matrix = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, shape[-1] ** -0.5, generator=gen)
        self.embedding = matrix(VOCAB, WIDTH)
        self.layers = [dict(qkv=matrix((HEADS + 2 * KV_HEADS) * DIM, WIDTH), out=matrix(WIDTH, HEADS * DIM), up=matrix(4 * WIDTH, WIDTH),
                            down=matrix(WIDTH, 4 * WIDTH)) for _ in range(layers)]
        angle = torch.arange(longest, device="cuda")[:, None] * THETA ** (-torch.arange(DIM // 2, device="cuda") / (DIM // 2))
        self.rope = torch.cat([angle.cos(), angle.sin()], 1)

    @staticmethod
    def norm(x):
        return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(torch.bfloat16)

    def project(self, layer, x):
        """q, k and v of tokens, as parts of one projection's output."""
        return (self.norm(x) @ layer["qkv"].T).view(-1, HEADS + 2 * KV_HEADS, DIM).split([HEADS, KV_HEADS, KV_HEADS], dim=1)

    def rest(self, layer, x, attended):
        x = x + attended.reshape(x.shape[0], -1) @ layer["out"].T
        return x + torch.nn.functional.silu(self.norm(x) @ layer["up"].T) @ layer["down"].T

    def logits(self, x):
        return 4.0 * (self.norm(x) @ self.embedding.T).float()

    def turn(self, x, positions):
        cos, sin = self.rope[positions][:, None].chunk(2, dim=-1)
        a, b = x.float().chunk(2, dim=-1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(torch.bfloat16)


def most_tokens(prompts, new):
    """Room that the longest sequence may need.  A step gives every sequence one token at least, so there are at most new - 1 of them; the
    sequence behind the longest prompt may keep all DRAFT rows of each, and the last step's rows are written behind those."""
    return max(map(len, prompts)) + max(0, new - 1) * DRAFT


def generate(prompts, new, layers=4, chunk=512, seed=0, temperature=0.8, top_p=0.95, four_bits=False, most=0):
    """Token lists of the prompts' continuations, at least `new` each, and the mean number of tokens a step keeps."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    S, longest = len(prompts), most_tokens(prompts, new)
    blocks = -(-longest // BLOCK)
    model = Decoder(layers, longest, gen)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    per_seq = lambda v, t=torch.float32: torch.full((S,), v, dtype=t, device="cuda")
    table = torch.randperm(S * blocks, generator=torch.Generator().manual_seed(seed)).int().view(S, blocks).cuda()
    keep = min(blocks, max(4, blocks // 4))
    verifier = sv.SparseVerifier(n_seq=S, n_q_heads=HEADS, n_kv_heads=KV_HEADS, head_dim=DIM, block_size=BLOCK, max_blocks=blocks, n_draft=DRAFT,
                                 n_layers=layers, block_table=table, seq_lens=ints([0] * S), budget_blocks=per_seq(keep, torch.int32), max_sel=keep,
                                 anchors=[l % 2 == 0 for l in range(layers)])
    if four_bits:
        for l in range(layers):
            verifier.set_layer_kv_q4(l, torch.zeros((S * blocks, KV_HEADS, BLOCK // 64, sv.SV_Q4_SLAB_BYTES), dtype=torch.uint8, device="cuda"))
    else:
        verifier.set_kv_stack(*(torch.zeros((layers, S * blocks, KV_HEADS, BLOCK, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    rand = lambda *shape: torch.rand(shape, generator=gen, device="cuda")
    warp = dict(temperature=per_seq(temperature), top_p=per_seq(top_p))

    # the prompts, a chunk of each at a time
    last = torch.zeros((S, WIDTH), dtype=torch.bfloat16, device="cuda")
    for begin in range(0, max(map(len, prompts)), chunk):
        parts = [p[begin:begin + chunk] for p in prompts]
        starts = [0]
        for p in parts:
            starts.append(starts[-1] + len(p))
        q_start, x = ints(starts), model.embedding[torch.cat([ints(p) for p in parts]).long()]
        for l, layer in enumerate(model.layers):
            q, k, v = model.project(layer, x)
            attended = torch.empty((x.shape[0], HEADS, DIM), dtype=torch.bfloat16, device="cuda")
            verifier.prefill_layer(l, q, k, v, q_start, attended, rope=model.rope)
            x = model.rest(layer, x, attended)
        verifier.end_prefill()
        for s, p in enumerate(prompts):
            if begin < len(p) <= begin + chunk:
                last[s] = x[starts[s + 1] - 1]
    _, root = verifier.draw(model.logits(last), rand(S), distributions=False, **warp)
    texts, steps, kept = [[t] for t in root.tolist()], 0, 0

    # verification steps
    while min(map(len, texts)) < new:
        # the draft: rows 1.. of a chain behind the token that is known, and the distributions they were drawn from
        tokens, p_draft = [root.view(S)], []
        for _ in range(DRAFT):
            p, t = verifier.draw(model.logits(model.embedding[tokens[-1].long()]), rand(S), **warp)
            p_draft.append(p)
            tokens.append(t)
        tokens, p_draft = torch.stack(tokens[:DRAFT], 1).contiguous(), torch.stack(p_draft, 1).contiguous()
        x = model.embedding[tokens.view(-1).long()]
        positions = (verifier.positions()[:, None] + torch.arange(DRAFT, device="cuda")).view(-1).long()
        draft_k, draft_v = (torch.empty((layers, S, DRAFT, KV_HEADS, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for l, layer in enumerate(model.layers):
            q, k, v = model.project(layer, x)
            draft_k[l].copy_(model.turn(k, positions).view(S, DRAFT, KV_HEADS, DIM))
            draft_v[l].copy_(v.view(S, DRAFT, KV_HEADS, DIM))
            attended = torch.empty((S, DRAFT, HEADS, DIM), dtype=torch.bfloat16, device="cuda")
            turned, lse = model.turn(q, positions).view(S, DRAFT, HEADS, DIM), torch.empty((S, DRAFT, HEADS), device="cuda")
            verifier.verify_layer(l, turned, draft_k[l], draft_v[l], attended, lse=lse)
            if most:
                verifier.weigh_layer(l, turned, lse)
            x = model.rest(layer, x, attended)
        p_target, _ = verifier.draw(model.logits(x).view(S, DRAFT, VOCAB), rand(S * DRAFT), **warp)
        path, n_path, root = verifier.accept(p_target, p_draft, tokens, rand(S, DRAFT), rand(S))
        verifier.commit(draft_k, draft_v, path, n_path)
        if most and int(verifier.seq_lens.max()) > most:
            verifier.evict(torch.where(verifier.seq_lens > most, most * 3 // 4, verifier.seq_lens).int())
        verifier.check_status()
        for s in range(S):
            texts[s] += tokens[s, 1:int(n_path[s])].tolist() + [int(root[s])]
        steps, kept = steps + 1, kept + float(n_path.float().mean())
    return texts, kept / max(1, steps), verifier


def main():
    args = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    args.add_argument("--prompt", type=int, nargs="+", default=[3000, 700], help="tokens of the prompts")
    args.add_argument("--new", type=int, default=32)
    args.add_argument("--layers", type=int, default=4)
    args.add_argument("--four-bits", action="store_true", help="hold the cache in 4 bits")
    args.add_argument("--most-tokens", type=int, default=0, help="evict from sequences with more tokens than these")
    a = args.parse_args()
    if a.four_bits and a.most_tokens:
        args.error("tokens are evicted from a bfloat16 cache only")
    rng = torch.Generator().manual_seed(1)
    texts, kept, _ = generate([torch.randint(0, VOCAB, (n,), generator=rng).tolist() for n in a.prompt], a.new, a.layers, four_bits=a.four_bits,
                              most=a.most_tokens)
    print(f"{kept:.2f} tokens kept a step")
    for n, t in zip(a.prompt, texts):
        print(f"behind {n} tokens:", " ".join(map(str, t[:a.new])))


if __name__ == "__main__":
    main()
