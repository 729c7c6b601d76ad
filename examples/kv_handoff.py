"""A request's key/value cache moves from the GPU that reads its prompt to the one
that answers (arXiv 2604.17172, section 5.3), held in 8 bits and coded on the way.

    python examples/kv_handoff.py

Prompt side: plan places for the prompts' tokens, store their keys and values in
8-bit pages, attend.  Hand-off: the pages of a request are gathered and coded as FP8
pairs, each plane of pages one stream; the other side decodes them into pages of its
own pool.  Answer side: plan, store and attend one token at a time, captured once in
a graph and replayed.  Both sides run here on one GPU, with random projections in
place of a model; the answers are compared with those over the cache that stayed.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2604_17172_amd as uz  # noqa: E402

HEADS, KV, DIM, PAGE = 32, 8, 128, 64
DEVICE = "cuda"


class Instance:
    """A pool of pages, its free list, and the requests' block tables."""

    def __init__(self, pages: int, requests: int, max_pages: int):
        self.cache = uz.KVCache.empty(pages, KV, DIM, PAGE, "e4m3fn", DEVICE)
        self.free = torch.randperm(pages, device=DEVICE).to(torch.int32)
        self.table = torch.full((requests, max_pages), -1, dtype=torch.int32, device=DEVICE)
        self.lens = torch.zeros(requests, dtype=torch.int32, device=DEVICE)

    def step(self, qkv: torch.Tensor, new: torch.Tensor, max_new: int, plan=None, out=None, lse=None, ws=None):
        """New tokens through plan, store and attend; qkv [rows, heads + 2 kv heads, dim]."""
        plan = uz.kv_plan(self.lens, new, self.free, self.table, PAGE, qkv.shape[0], out=plan)
        uz.kv_store(self.cache, qkv[:, HEADS:HEADS + KV], qkv[:, HEADS + KV:], plan.slots, plan.runs, plan.counts)
        out, lse = uz.kv_attend(qkv[:, :HEADS], self.cache, self.table, plan.lens, plan.q_start, max_new, out=out, lse=lse, ws=ws)
        return plan, out, lse

    def taken(self, plan) -> None:
        """The lengths and the free list after a step."""
        granted(plan)
        self.lens.copy_(plan.lens)
        self.free = self.free[int(plan.counts[0]):].contiguous()

    def give(self, pages: int) -> torch.Tensor:
        mine, self.free = self.free[:pages].clone(), self.free[pages:].contiguous()
        return mine


def granted(plan) -> None:
    """Every request of the step had its places."""
    if int(plan.status.item()) != uz.OK:
        raise uz.UzipError(int(plan.status.item()), "uzip_kv_plan")


def send(side: Instance, pages: torch.Tensor):
    """The pages' codes as streams of FP8 pairs (their exponents, a byte for each page and head, go as they are)."""
    at, streams = pages.long(), []
    for plane in (side.cache.k, side.cache.v):
        x = plane[at].view(torch.float8_e4m3fn)
        stream, size = uz.compress(x, 65536, check=True)
        streams.append((stream[: int(size.item())].clone(), x.numel() // 2))
    return streams, side.cache.k_exp[at], side.cache.v_exp[at]


def receive(side: Instance, sent, pages: torch.Tensor) -> None:
    streams, k_exp, v_exp = sent
    at = pages.long()
    for plane, (stream, pairs) in zip((side.cache.k, side.cache.v), streams):
        bits, status = uz.decompress(stream, "e4m3fn", pairs)
        if int(status.item()) != uz.OK:
            raise uz.UzipError(int(status.item()), "uzip_decompress")
        plane[at] = bits.view(torch.uint8).view(len(at), *plane.shape[1:])
    side.cache.k_exp[at], side.cache.v_exp[at] = k_exp, v_exp


def main(prompts=(1000, 37, 2050), answer: int = 70) -> float:
    torch.manual_seed(7)
    n = len(prompts)
    width = -(-(max(prompts) + answer) // PAGE) + 1
    reader, writer = Instance(160, n, width), Instance(200, n, width)

    def tokens(rows):
        return torch.randn(rows, HEADS + 2 * KV, DIM, device=DEVICE).to(torch.bfloat16)
    new = torch.tensor(prompts, dtype=torch.int32, device=DEVICE)
    plan, _, _ = reader.step(tokens(sum(prompts)), new, max(prompts))
    reader.taken(plan)

    coded = held = 0
    for i, length in enumerate(prompts):
        pages = reader.table[i, : -(-length // PAGE)]
        sent = send(reader, pages)
        mine = writer.give(len(pages))
        receive(writer, sent, mine)
        writer.table[i, : len(mine)] = mine
        coded += sum(s.numel() for s, _ in sent[0])
        held += 2 * sum(m for _, m in sent[0])
    writer.lens.copy_(reader.lens)
    print(f"handed over {n} requests: {held} bytes of 8-bit cache in {coded} bytes of streams ({coded / held:.3f})", flush=True)

    # one token of each request at a time, as a graph on the side that answers
    one = torch.ones(n, dtype=torch.int32, device=DEVICE)
    qkv = tokens(n)
    step_plan = uz.kv_plan_buffers(n, n, PAGE, DEVICE)
    out, lse = torch.empty(n, HEADS, DIM, dtype=torch.bfloat16, device=DEVICE), torch.empty(n, HEADS, device=DEVICE)
    ws = uz.kv_attend_workspace(qkv[:, :HEADS], writer.cache, n, 1)
    free = torch.zeros(n, dtype=torch.int32, device=DEVICE)          # pages on offer in a step: one for each request
    writer_free, writer.free = writer.free, free
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                                    # first use outside the capture; nothing is written
        uz.kv_plan(writer.lens, torch.zeros_like(one), free, writer.table, PAGE, n, out=step_plan)
        uz.kv_store(writer.cache, qkv[:, HEADS:HEADS + KV], qkv[:, HEADS + KV:], step_plan.slots, step_plan.runs, step_plan.counts)
        uz.kv_attend(qkv[:, :HEADS], writer.cache, writer.table, step_plan.lens, step_plan.q_start, 1, out=out, lse=lse, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        writer.step(qkv, one, 1, step_plan, out, lse, ws)
    worst = 0.0
    for _ in range(answer):
        qkv.copy_(tokens(n))
        free.copy_(writer_free[:n])
        graph.replay()
        granted(step_plan)
        writer.lens.copy_(step_plan.lens)
        writer_free = writer_free[int(step_plan.counts[0]):].contiguous()
        stayed, want, _ = reader.step(qkv, one, 1)                   # the same tokens over the cache that stayed
        reader.taken(stayed)
        worst = max(worst, (out.float() - want.float()).abs().max().item())
    print(f"{answer} tokens of each request: largest difference from the cache that stayed {worst}", flush=True)
    return worst


if __name__ == "__main__":
    sys.exit(0 if main() == 0 else 1)
