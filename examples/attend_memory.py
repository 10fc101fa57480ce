"""A turn of a conversation over its memory: retrieval, cache and attention together.

Every chunk of the memory has an embedding in the bank and its keys and values
in pages of a 4-bit cache; both go by one directory.  Each request's turn then
takes these steps, all on the GPU:

1. mem_append_chunks    a new chunk (bank row and pages) for the turn's own tokens
2. mem_retrieve_topk    the chunks that matter to the request
3. mem_kv_write         the turn's keys and values, quantised into its chunk
4. mem_attend           causal attention of the turn's tokens over the retrieved
                        chunks in time order and, last, over their own chunk

Run: python examples/attend_memory.py
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_05708_amd as pm  # noqa: E402

PAGE_TOKENS, PPC = 64, 8     # a chunk holds up to 512 tokens
HEADS, HEADS_Q, HEAD_DIM = 8, 32, 128
EMB = 1024


class Memory:
    """Bank, cache and lengths of up to `capacity` chunks."""

    def __init__(self, capacity: int, device="cuda"):
        fmt = pm.MEM_KV_FP4
        page_bytes = pm.mem_kv_page_bytes(PAGE_TOKENS, HEADS, HEAD_DIM, fmt)
        pool = torch.zeros((capacity * PPC, page_bytes), dtype=torch.uint8, device=device)
        table = torch.full((capacity, PPC), -1, dtype=torch.int32, device=device)
        emb = torch.zeros((capacity, EMB), dtype=torch.bfloat16, device=device)
        self.bank = pm.BankState(emb, 0, table, 0, capacity * PPC)
        self.cache = pm.KvCache(pool, table, PAGE_TOKENS, HEADS, HEAD_DIM, fmt)
        self.tok_len = torch.zeros(capacity, dtype=torch.int32, device=device)

    def open(self, emb: torch.Tensor) -> torch.Tensor:
        """New chunks for these embeddings; their ids."""
        first = self.bank.n
        pm.mem_append_chunks(self.bank, emb)
        return torch.arange(first, self.bank.n, dtype=torch.int32, device=emb.device)

    def store(self, chunks: torch.Tensor, k: torch.Tensor, v: torch.Tensor) -> None:
        """The same number of tokens for each of `chunks`, behind those that it holds: k, v [chunks * n, heads, d]."""
        n = k.shape[0] // chunks.numel()
        chunk = chunks.repeat_interleave(n)
        pos = self.tok_len[chunk.long()] + torch.arange(n, dtype=torch.int32, device=k.device).repeat(chunks.numel())
        pm.mem_kv_write(self.cache, k, v, chunk, pos)
        self.tok_len[chunks.long()] += n


def turn(mem: Memory, embedding: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, top: int):
    """One turn of m requests with n tokens each: embedding [m, EMB], q [m * n, heads_q, d], k and v [m * n, heads, d].
    Returns (out, lse, ids): the attention's outputs and the chunks that each request saw, in context order."""
    found, _, _, _ = pm.mem_retrieve_topk(mem.bank.live, embedding, top, 1.0 / math.sqrt(EMB))
    own = mem.open(embedding)
    mem.store(own, k, v)
    ids = torch.cat([found.sort(dim=1).values, own.unsqueeze(1)], dim=1)  # chunk ids grow with time
    out, lse = pm.mem_attend(mem.cache, mem.tok_len, ids, q, 1.0 / math.sqrt(HEAD_DIM), causal=True)
    return out, lse, ids


def main():
    g = torch.Generator("cuda").manual_seed(0)
    rand = lambda *s: torch.randn(s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    mem = Memory(4096)
    past = mem.open(rand(1024, EMB))
    for part in past.split(128):                            # 1,024 chunks of 512 tokens are known already
        mem.store(part, rand(part.numel() * 512, HEADS, HEAD_DIM), rand(part.numel() * 512, HEADS, HEAD_DIM))
    for n in (512, 1, 1):                                   # a turn of 512 tokens, then single ones
        m = 16
        out, lse, ids = turn(mem, rand(m, EMB), rand(m * n, HEADS_Q, HEAD_DIM), rand(m * n, HEADS, HEAD_DIM),
                             rand(m * n, HEADS, HEAD_DIM), top=5)
        torch.cuda.synchronize()
        print(f"{m} requests of {n} tokens over {ids.shape[1]} chunks each: out {tuple(out.shape)}, "
              f"lse {lse.min().item():.2f} to {lse.max().item():.2f}")


if __name__ == "__main__":
    main()
