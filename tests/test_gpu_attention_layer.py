"""The attention layer on the GPU: its calls put together by hand give the same
bits; prompts and single tokens give the same outputs; and it is attention."""
import numpy as np
import pytest
import torch

import paper_1911_08076_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(hidden=272, heads=4, kv_heads=2, dim=64, dtype=torch.bfloat16, **kw):
    g = torch.Generator(device=DEV).manual_seed(3)
    w1 = torch.randn((heads + 2 * kv_heads) * dim, hidden, generator=g, device=DEV) * hidden ** -0.5
    w2 = torch.randn(hidden, heads * dim, generator=g, device=DEV) * (heads * dim) ** -0.5
    args = dict(num_pages=12, max_pages=4, page_tokens=32)
    args.update(kw)
    layer = P.AttentionLayer(w1.to(dtype), w2.to(dtype), heads, kv_heads, dim, **args)
    return layer, w1.to(dtype), w2.to(dtype), g


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def reference(x, w1, w2, heads, kv_heads, dim, base=10000.0):
    """Causal attention of one sequence in 64 bits on the CPU."""
    x, w1, w2 = (t.double().cpu() for t in (x, w1, w2))
    n = len(x)
    rows = (x @ w1.T).view(n, heads + 2 * kv_heads, dim)
    freq = base ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    turn = torch.polar(torch.ones(n, dim // 2, dtype=torch.float64),
                       torch.arange(n, dtype=torch.float64)[:, None] * freq)[:, None]
    qk = rows[:, :heads + kv_heads]
    z = torch.complex(qk[..., :dim // 2].contiguous(), qk[..., dim // 2:].contiguous()) * turn
    qk = torch.cat([z.real, z.imag], -1)
    out = torch.zeros(n, heads, dim, dtype=torch.float64)
    for h in range(heads):
        g = h // (heads // kv_heads)
        s = qk[:, h] @ qk[:, heads + g].T * dim ** -0.5
        s = s.masked_fill(torch.ones(n, n).triu(1).bool(), -np.inf)
        out[:, h] = torch.softmax(s, -1) @ rows[:, heads + kv_heads + g]
    return out.view(n, -1) @ w2.T


def test_layer_is_its_calls():
    layer, w1, w2, g = make()
    x = torch.randn(50, 272, generator=g, device=DEV).to(torch.bfloat16)
    offs, lens, pages = i32([0, 30, 50]), i32([30, 20]), i32([[3, 1, 0, 2], [7, 5, 4, 6]])
    got = layer(x, offs, lens, pages, max_q=30)
    cache = torch.zeros_like(layer.cache)

    def linear(x, lin):
        codes = torch.empty(len(x), lin.ld, dtype=torch.uint8, device=DEV)
        scales = torch.empty(-(-lin.k // 128), len(x), device=DEV)
        P.ifq_f8_quantize(P.f8_quant_desc(len(x), lin.k, P.IFQ_TYPE_BF16), x, codes, scales)
        y = torch.empty(len(x), lin.n, dtype=x.dtype, device=DEV)
        P.ifq_f8_matmul(P.f8_matmul_desc(len(x), lin.n, lin.ld, P.IFQ_TYPE_BF16), codes, scales,
                        lin.codes, lin.scales, y)
        return y

    rows = linear(x, layer.qkv).view(50, 8, 64)
    q, k, v = (t.contiguous() for t in (rows[:, :4], rows[:, 4:6], rows[:, 6:]))
    cos, sin = P.rotation_tables(128, 64)
    d = P.kv_desc(2, 50, 30, 128, 4, 2, 64, 32, 12, 4, P.IFQ_TYPE_BF16, scale=64 ** -0.5,
                  rot_dim=64, rot_len=128)
    turned, out = torch.empty_like(q), torch.empty_like(q)
    P.ifq_kv_append(d, q, k, v, cos, sin, offs, lens, pages, cache, turned)
    P.ifq_kv_attention(d, turned, offs, lens, pages, cache, out)
    assert torch.equal(cache, layer.cache)
    assert torch.equal(linear(out.view(50, -1), layer.out), got)


def test_layer_is_attention():
    """Within what the codes allow: 3.6 % rms for each 8-bit operand of a product
    and some 10 % for a 4-bit key or value (a step is 1/15 of a row's spread of
    about 5 standard deviations, its rms error 0.1 of one) add up to below 0.35
    of the output's norm; a wrong head, pair or position gives 1 and more."""
    layer, w1, w2, g = make()
    x = torch.randn(100, 272, generator=g, device=DEV).to(torch.bfloat16)
    got = layer(x, i32([0, 100]), i32([100]), i32([[3, 1, 0, 2]]), max_q=100).double().cpu()
    want = reference(x, w1, w2, 4, 2, 64)
    assert float((got - want).norm() / want.norm()) < 0.35


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_prompt_and_single_tokens_agree(window, sinks):
    """The products' sums are in another order for one row, so a rounding to 16
    bits or a code may come out beside the other: some hundredths at most."""
    for dtype in (torch.bfloat16, torch.float16):
        layer, w1, w2, g = make(dtype=dtype, window=window, sinks=sinks)
        x = torch.randn(70, 272, generator=g, device=DEV).to(dtype)
        pages = i32([[3, 1, 0, 2]])
        whole = layer(x, i32([0, 70]), i32([70]), pages, max_q=70)
        layer.cache.zero_()
        layer(x[:40].contiguous(), i32([0, 40]), i32([40]), pages, max_q=40)
        ones = [layer(x[i:i + 1].contiguous(), i32([0, 1]), i32([i + 1]), pages, max_q=1)
                for i in range(40, 70)]
        a, b = torch.cat(ones).double(), whole[40:].double()
        assert float((a - b).norm() / b.norm()) < 0.1


def test_layer_refuses_what_does_not_fit():
    w = torch.zeros(512, 272, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError, match="do not fit"):
        P.AttentionLayer(w, w, 4, 2, 64, 4, 4)
    with pytest.raises(ValueError, match="no cache"):
        make(page_tokens=48)
    layer, w1, w2, g = make()
    x = torch.zeros(5, 272, dtype=torch.bfloat16, device=DEV)
    args = [i32([0, 5]), i32([5]), i32([[3, 1, 0, 2]])]
    for bad in (x.float(), x[:, :256], x.t().contiguous().t()):
        with pytest.raises(ValueError, match="dense rows of 272"):
            layer(bad, *args, max_q=5)
    for i, name in enumerate(("offsets", "lengths", "pages")):
        bad = list(args)
        bad[i] = args[i].long()
        with pytest.raises(ValueError, match=name):
            layer(x, *bad, max_q=5)
    with pytest.raises(ValueError, match="pages"):
        layer(x, args[0], args[1], args[2][:, :3], max_q=5)
    with pytest.raises(P.IfqError):
        layer(x, *args, max_q=-1)


def test_nothing_new_and_a_captured_step():
    """No tokens give no rows; a captured step replayed over a growing sequence
    gives the eager steps' bits, and eager prompts in between leave it alone."""
    layer, w1, w2, g = make()
    none = layer(torch.empty(0, 272, dtype=torch.bfloat16, device=DEV), i32([0, 0]), i32([5]),
                 i32([[3, 1, 0, 2]]), max_q=0)
    assert none.shape == (0, 272)
    x = torch.randn(60, 272, generator=g, device=DEV).to(torch.bfloat16)
    pages, other = i32([[3, 1, 0, 2]]), i32([[7, 5, 4, 6]])
    eager = [layer(x[i:i + 1].contiguous(), i32([0, 1]), i32([i + 1]), pages, max_q=1)
             for i in range(20)]
    layer.cache.zero_()
    token, offs, lens = x[:1].clone(), i32([0, 1]), i32([1])
    out = torch.empty_like(token)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(token, offs, lens, pages, max_q=1, out=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(token, offs, lens, pages, max_q=1, out=out)
    for i in range(20):
        token.copy_(x[i:i + 1])
        lens.fill_(i + 1)
        graph.replay()
        assert torch.equal(out, eager[i])
        if i % 5 == 1:
            layer(x, i32([0, 60]), i32([60]), other, max_q=60)
            torch.cuda.synchronize()


def test_first_step_under_capture():
    """A workspace that a capture makes is zero at its replays only: an eager step
    between capture and replay, and the replays after it, are right."""
    layer, w1, w2, g = make(num_pages=64, max_pages=64)
    other = make(num_pages=64, max_pages=64)[0]
    x = torch.randn(1500, 272, generator=g, device=DEV).to(torch.bfloat16)
    pages = torch.arange(64, dtype=torch.int32, device=DEV).view(1, 64)
    args = i32([0, 1]), i32([1501]), pages
    token = torch.randn(1, 272, generator=g, device=DEV).to(torch.bfloat16)
    other(x, i32([0, 1500]), i32([1500]), pages, max_q=1500)
    want = other(token, *args, max_q=1)
    assert other.workspace._all            # the step is one that needs a workspace
    layer.cache.copy_(other.cache)
    out = torch.empty_like(token)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(token, *args, max_q=1, out=out)
    assert torch.equal(layer(token, *args, max_q=1), want)
    for _ in range(3):
        out.zero_()
        graph.replay()
        assert torch.equal(out, want)
        assert torch.equal(layer(token, *args, max_q=1), want)


def test_example_runs(capsys):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "decode.py")
    spec = importlib.util.spec_from_file_location("decode_example", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    mod.main(["--batch", "3", "--prompt", "150", "--tokens", "12"])
    said = capsys.readouterr().out
    assert "prompts:" in said and "decoding: 3 sequences" in said
