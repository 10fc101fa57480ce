"""A turn of a conversation over a memory of latent vectors: retrieval, rotated
cache writes and latent attention together.

Every chunk of the memory has an embedding in the bank and, in pages of an 8-bit
latent cache, one latent vector and one rotated key part per token; both go by
one directory.  Each request's turn then takes these steps, all on the GPU:

1. mem_append_chunks    a new chunk (bank row and pages) for the turn's own tokens
2. mem_retrieve_topk    the chunks that matter to the request
3. mem_latent_append    the turn's latent vectors and key parts into its chunk, with
                        the position rotation of key parts and queries on the way
4. mem_latent_attend    causal attention of the turn's tokens over the retrieved
                        chunks in time order and, last, over their own chunk: a turn
                        of many tokens in the expanded form, single tokens in the
                        absorbed one

Run: python examples/latent_memory.py
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_05708_amd as pm  # noqa: E402

PAGE_TOKENS, PPC = 64, 8     # a chunk holds up to 512 tokens
HEADS, HEAD_DIM, LATENT, ROPE = 16, 128, 512, 64
EMB = 1024


class Memory:
    """Bank, latent cache and lengths of up to `capacity` chunks."""

    def __init__(self, capacity: int, device="cuda"):
        fmt = pm.MEM_KV_FP8
        page_bytes = pm.mem_latent_page_bytes(PAGE_TOKENS, LATENT, ROPE, fmt)
        pool = torch.zeros((capacity * PPC, page_bytes), dtype=torch.uint8, device=device)
        table = torch.full((capacity, PPC), -1, dtype=torch.int32, device=device)
        emb = torch.zeros((capacity, EMB), dtype=torch.bfloat16, device=device)
        self.bank = pm.BankState(emb, 0, table, 0, capacity * PPC)
        self.cache = pm.LatentCache(pool, table, PAGE_TOKENS, LATENT, ROPE, fmt)
        self.tok_len = torch.zeros(capacity, dtype=torch.int32, device=device)
        pairs = torch.arange(ROPE // 2, dtype=torch.float64, device=device)
        self.freq = torch.pow(10000.0, -pairs / (ROPE // 2)).float()

    def open(self, emb: torch.Tensor) -> torch.Tensor:
        """New chunks for these embeddings; their ids."""
        first = self.bank.n
        pm.mem_append_chunks(self.bank, emb)
        return torch.arange(first, self.bank.n, dtype=torch.int32, device=emb.device)

    def store(self, chunks: torch.Tensor, x: torch.Tensor, start, t: torch.Tensor | None = None):
        """The same number of tokens for each of `chunks`, behind those that it holds: x [chunks * n, LATENT + ROPE]
        (latent vectors and key parts, as one projection leaves them), the first one at position start[i] of its
        conversation.  Returns the rotated part of the queries t [chunks * n, heads, ROPE]."""
        n = x.shape[0] // chunks.numel()
        step = torch.arange(n, dtype=torch.int32, device=x.device).repeat(chunks.numel())
        chunk = chunks.repeat_interleave(n)
        t = pm.mem_latent_append(self.cache, x[:, :LATENT], x[:, LATENT:], chunk, self.tok_len[chunk.long()] + step,
                                 start.repeat_interleave(n) + step, self.freq, q=t, pairs=True)
        self.tok_len[chunks.long()] += n
        return t


def turn(mem: Memory, embedding: torch.Tensor, q: torch.Tensor, x: torch.Tensor, w: torch.Tensor, start, top: int):
    """One turn of m requests with n tokens each: embedding [m, EMB], q [m * n, heads, HEAD_DIM + ROPE], x [m * n, LATENT
    + ROPE], start int32 [m].  Returns (out, ids): the attention's outputs and the chunks that each request saw, in
    context order."""
    found, _, _, _ = pm.mem_retrieve_topk(mem.bank.live, embedding, top, 1.0 / math.sqrt(EMB))
    own = mem.open(embedding)
    t = mem.store(own, x, start, q[..., HEAD_DIM:])
    ids = torch.cat([found.sort(dim=1).values, own.unsqueeze(1)], dim=1)  # chunk ids grow with time
    out = pm.mem_latent_attend(mem.cache, mem.tok_len, ids, q[..., :HEAD_DIM], t, w, 1.0 / math.sqrt(HEAD_DIM + ROPE),
                               causal=True)
    return out, ids


def main():
    g = torch.Generator("cuda").manual_seed(0)
    rand = lambda *s: torch.randn(s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    w = (rand(HEADS, 2 * HEAD_DIM, LATENT).float() / math.sqrt(LATENT)).to(torch.bfloat16)
    mem = Memory(4096)
    past = mem.open(rand(1024, EMB))
    mem.store(past, rand(1024 * 512, LATENT + ROPE), past * 512)          # 1,024 chunks of 512 tokens are known already
    for n in (512, 1, 1):                                                 # a turn of 512 tokens, then single ones
        m = 16
        start = torch.full((m,), mem.bank.n * 512, dtype=torch.int32, device="cuda")
        out, ids = turn(mem, rand(m, EMB), rand(m * n, HEADS, HEAD_DIM + ROPE), rand(m * n, LATENT + ROPE), w, start, top=5)
        torch.cuda.synchronize()
        print(f"{m} requests of {n} tokens over {ids.shape[1]} chunks each: out {tuple(out.shape)}, "
              f"rms {out.float().square().mean().sqrt().item():.3f}")


if __name__ == "__main__":
    main()
