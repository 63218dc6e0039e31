"""Decoding with a 4-bit key/value cache: one attention layer as a serving loop runs it.

A batch of prompts is quantized into the cache and attended to (kv4_append,
kv4_attention); then single tokens follow, each appended, its pages chosen by the signs of
the keys (kv4_select), and attended to over those pages alone (kv4_attention with a list).
The steps run in one captured graph.  Random tensors stand for a model's, with queries
that look for one of the keys; the program prints how far each step is from attention
over the keys and values before they were quantized.

    python examples/kv4_decoding.py [--seqs 4] [--prompt 700] [--steps 40] [--keep 8]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2011_09398_amd as lce  # noqa: E402

PAGE = lce.KV4_PAGE


def exact(q, k, v, group):
    """Attention of one token of each sequence, float32: q [n, heads, d], lists of k, v."""
    out = []
    for i in range(q.shape[0]):
        kk = k[i].float().repeat_interleave(group, 1)
        vv = v[i].float().repeat_interleave(group, 1)
        s = (q[i].float()[None] * kk).sum(-1) * q.shape[-1] ** -0.5
        out.append((torch.softmax(s, 0)[..., None] * vv).sum(0))
    return torch.stack(out)


def run(seqs=4, prompt=700, steps=40, keep=8, q_heads=16, kv_heads=4, dim=128, seed=0):
    """Returns the relative errors of the prompt's last tokens, of steps over all pages, of
    steps over the kept pages, and the bytes of the cache over those of bfloat16."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    torch.manual_seed(seed)
    group, dtype = q_heads // kv_heads, torch.bfloat16
    lengths = [max(1, prompt * (b + 1) // seqs) for b in range(seqs)]
    width = -(-(max(lengths) + steps) // PAGE)
    cache = lce.KV4Cache(kv_heads, dim, pages=seqs * width + 1)
    # each sequence gets its pages from a shuffled pool
    table = torch.randperm(cache.pages, device="cuda", generator=g)[:seqs * width]
    table = table.to(torch.int32).view(seqs, width).contiguous()

    def normal(n, heads):
        return torch.randn(n, heads, dim, device="cuda", generator=g)

    def queries(k):
        """A query for each of k, which it is like."""
        return (normal(k.shape[0], q_heads) + k.float().repeat_interleave(group, 1)).to(dtype)

    def slots(seq, place):
        page = table.long()[seq, place // PAGE]
        return page * PAGE + place % PAGE

    # the prompts, all sequences in one call
    length = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    seq = torch.repeat_interleave(torch.arange(seqs, device="cuda"), length.long())
    place = torch.cat([torch.arange(n, device="cuda") for n in lengths])
    start = torch.zeros(seqs + 1, dtype=torch.int32, device="cuda")
    start[1:] = length.cumsum(0)
    k, v = normal(sum(lengths), kv_heads).to(dtype), normal(sum(lengths), kv_heads).to(dtype)
    q = queries(k)
    lce.kv4_append(cache, k, v, slots(seq, place))
    out = lce.kv4_attention(cache, q, table, start, length, max_q=max(lengths),
                            max_len=max(lengths))
    keys = [k[start[b]:start[b + 1]] for b in range(seqs)]
    values = [v[start[b]:start[b + 1]] for b in range(seqs)]
    last = start[1:].long() - 1

    def off(got, want):
        return float((got.float() - want).norm() / want.norm())

    error_prompt = off(out[last], exact(q[last], keys, values, group))

    # single tokens: static buffers, one graph of append, select and attention
    q1, k1, v1 = (torch.zeros(seqs, h, dim, dtype=dtype, device="cuda")
                  for h in (q_heads, kv_heads, kv_heads))
    at = torch.zeros(seqs, dtype=torch.int64, device="cuda")
    one = torch.arange(seqs + 1, dtype=torch.int32, device="cuda")
    pages = torch.empty(seqs, kv_heads, keep, dtype=torch.int32, device="cuda")
    dense, sparse = torch.empty_like(q1), torch.empty_like(q1)
    workspace = lce.kv4_workspace(cache, q1, table)

    def step():
        lce.kv4_append(cache, k1, v1, at)
        lce.kv4_select(cache, q1, table, one, length, keep, out=pages, workspace=workspace)
        lce.kv4_attention(cache, q1, table, one, length, pages=pages, out=sparse,
                          workspace=workspace)
        lce.kv4_attention(cache, q1, table, one, length, max_q=1, out=dense, workspace=workspace)

    at.fill_(-1)                                         # warm up without writing anything
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    error_dense, error_sparse = [], []
    for _ in range(steps):
        k, v = normal(seqs, kv_heads).to(dtype), normal(seqs, kv_heads).to(dtype)
        liked = torch.stack([a[int(torch.randint(len(a), (1,)))] for a in keys])
        q = queries(liked)
        q1.copy_(q), k1.copy_(k), v1.copy_(v)
        at.copy_(slots(torch.arange(seqs, device="cuda"), length.long()))
        length += 1
        graph.replay()
        keys = [torch.cat((a, k[b:b + 1])) for b, a in enumerate(keys)]
        values = [torch.cat((a, v[b:b + 1])) for b, a in enumerate(values)]
        want = exact(q, keys, values, group)
        error_dense.append(off(dense, want))
        error_sparse.append(off(sparse, want))
    size = cache.data.numel() / (cache.pages * PAGE * kv_heads * dim * 2 * 2)
    return {"prompt": error_prompt, "dense": max(error_dense), "sparse": max(error_sparse),
            "size": size}


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("seqs", 4), ("prompt", 700), ("steps", 40), ("keep", 8)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    r = run(a.seqs, a.prompt, a.steps, a.keep)
    print(f"prompt: {r['prompt']:.3f} off attention over bfloat16 keys and values")
    print(f"{a.steps} steps over all pages: at most {r['dense']:.3f} off")
    print(f"{a.steps} steps over {a.keep} pages each: at most {r['sparse']:.3f} off")
    print(f"the cache takes {r['size']:.3f} of a bfloat16 one")


if __name__ == "__main__":
    main()
