"""Serves a batch of sequences through one attention layer, or with --vocabulary
through a whole decoder layer with a feed-forward block and a classifier: prompts
first, then tokens one by one in a captured graph, and prints both rates.

    python examples/decode.py [--batch 16] [--prompt 2000] [--tokens 100]
                              [--vocabulary 32000]
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_1911_08076_amd as P


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=2000)
    ap.add_argument("--tokens", type=int, default=100)
    ap.add_argument("--vocabulary", type=int, default=0)
    a = ap.parse_args(argv)
    if a.vocabulary:
        return decode(a)
    hidden, heads, kv_heads, dim, page = 4096, 32, 8, 128, 64
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(1)

    def randn(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device=dev) * scale).to(torch.bfloat16)

    most = -(-(a.prompt + a.tokens) // page)
    layer = P.AttentionLayer(randn((heads + 2 * kv_heads) * dim, hidden, scale=hidden ** -0.5),
                             randn(hidden, heads * dim, scale=(heads * dim) ** -0.5), heads,
                             kv_heads, dim, num_pages=a.batch * most, max_pages=most,
                             page_tokens=page)
    pages = torch.randperm(a.batch * most, generator=g, device=dev).to(torch.int32).view(
        a.batch, most)

    # prompts of ragged lengths
    new = [a.prompt - i * (a.prompt // (2 * a.batch)) for i in range(a.batch)]
    offsets = torch.tensor([sum(new[:i]) for i in range(a.batch + 1)], dtype=torch.int32,
                           device=dev)
    lengths = torch.tensor(new, dtype=torch.int32, device=dev)
    x = randn(sum(new), hidden)
    for _ in range(2):                   # the second time with everything in place
        torch.cuda.synchronize()
        t = time.perf_counter()
        y = layer(x, offsets, lengths, pages, max_q=max(new), max_kv=max(new))
        torch.cuda.synchronize()
        t = time.perf_counter() - t
    print("prompts: %d tokens in %.3f ms, %.0f tokens/s" % (sum(new), 1e3 * t, sum(new) / t))

    # one token after another: the layer's output is its next input
    one = torch.arange(a.batch + 1, dtype=torch.int32, device=dev)
    token = y[offsets[1:].long() - 1].clone()
    out = torch.empty_like(token)

    def step():
        lengths.add_(1)
        layer(token, one, lengths, pages, max_q=1, max_kv=max(new) + a.tokens, out=out)
        torch.div(out, out.abs().amax(1, keepdim=True).clamp_min(1e-3), out=token)

    if a.tokens < 3:
        return                           # one to warm up, one to try the graph, the rest timed
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    graph.replay()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.tokens - 2):
        graph.replay()
    torch.cuda.synchronize()
    t = (time.perf_counter() - t) / (a.tokens - 2)
    assert out.isfinite().all()
    print("decoding: %d sequences, %.1f us a step, %.0f tokens/s" % (a.batch, 1e6 * t,
                                                                     a.batch / t))


def decode(a):
    """Tokens in, tokens out: embedding, attention, feed-forward, classifier. Each sequence's
    next token is the most probable one; its log probability is summed."""
    hidden, inner, heads, kv_heads, dim, page = 2048, 5632, 16, 4, 128, 64
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(1)

    def randn(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device=dev) * scale).to(torch.bfloat16)

    def normed(x):
        return (x.float() * torch.rsqrt(x.float().square().mean(1, keepdim=True) + 1e-6)).to(x.dtype)

    most = -(-(a.prompt + a.tokens) // page)
    embedding = randn(a.vocabulary, hidden)
    attention = P.AttentionLayer(randn((heads + 2 * kv_heads) * dim, hidden, scale=hidden ** -0.5),
                                 randn(hidden, heads * dim, scale=(heads * dim) ** -0.5), heads,
                                 kv_heads, dim, num_pages=a.batch * most, max_pages=most,
                                 page_tokens=page)
    feed = P.FeedForward(randn(inner, hidden, scale=hidden ** -0.5),
                         randn(inner, hidden, scale=hidden ** -0.5),
                         randn(hidden, inner, scale=inner ** -0.5))
    classifier = P.Classifier(randn(a.vocabulary, hidden, scale=3 * hidden ** -0.5))
    pages = torch.randperm(a.batch * most, generator=g, device=dev).to(torch.int32).view(
        a.batch, most)

    def layer(tokens, offsets, lengths, max_q, max_kv):
        x = embedding[tokens]
        x = x + attention(normed(x), offsets, lengths, pages, max_q=max_q, max_kv=max_kv)
        return x + feed(normed(x))

    new = [a.prompt - i * (a.prompt // (2 * a.batch)) for i in range(a.batch)]
    offsets = torch.tensor([sum(new[:i]) for i in range(a.batch + 1)], dtype=torch.int32,
                           device=dev)
    lengths = torch.tensor(new, dtype=torch.int32, device=dev)
    prompt = torch.randint(0, a.vocabulary, (sum(new),), generator=g, device=dev,
                           dtype=torch.int32)
    given = torch.cat([prompt[1:], prompt[:1]])
    given[offsets[1:].long() - 1] = -1              # nothing is given behind a prompt
    for _ in range(2):                              # the second time with everything in place
        torch.cuda.synchronize()
        t = time.perf_counter()
        x = normed(layer(prompt, offsets, lengths, max(new), max(new)))
        score = classifier(x, tokens=given).logprob
        torch.cuda.synchronize()
        t = time.perf_counter() - t
    assert score.isfinite().all() and (score <= 0).all()
    print("prompts: %d tokens scored in %.3f ms, %.0f tokens/s" % (sum(new), 1e3 * t, sum(new) / t))

    one = torch.arange(a.batch + 1, dtype=torch.int32, device=dev)
    token = classifier(x[offsets[1:].long() - 1].contiguous()).top_tokens[:, 0].clone()
    total = torch.zeros(a.batch, device=dev)

    def step():
        lengths.add_(1)
        x = normed(layer(token, one, lengths, 1, max(new) + a.tokens))
        answer = classifier(x, top=1)
        token.copy_(answer.top_tokens[:, 0])
        total.add_(answer.top_logprobs[:, 0])

    if a.tokens < 3:
        return                           # one to warm up, one to try the graph, the rest timed
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    graph.replay()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.tokens - 2):
        graph.replay()
    torch.cuda.synchronize()
    t = (time.perf_counter() - t) / (a.tokens - 2)
    assert total.isfinite().all()
    print("decoding: %d sequences, %.1f us a step, %.0f tokens/s" % (a.batch, 1e6 * t,
                                                                     a.batch / t))


if __name__ == "__main__":
    main()
