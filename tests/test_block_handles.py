"""LayerNorm, dropout and DocumentAttention together within programs that use autograd, several streams and graphs, on the GPU."""
import pytest
import torch

import block_reference as ref
import paper_2406_03285_amd as rb

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
OFFSETS, PREFIXES = [0, 33, 33, 150, 171, 290], [5, 0, 60, 0, 200]
TOKENS, HEADS, KV, DIM = 300, 4, 2, 16
WIDTH = HEADS * DIM


def tensors(seed=0, dtype=BF16):
    g = torch.Generator("cuda").manual_seed(seed)
    def new(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)
    return {"x": new(TOKENS, WIDTH), "qkv": new((HEADS + 2 * KV) * DIM, WIDTH, scale=WIDTH ** -0.5), "back": new(WIDTH, WIDTH, scale=WIDTH ** -0.5),
            "w1": 1 + new(WIDTH, scale=0.2), "b1": new(WIDTH, scale=0.2), "w2": 1 + new(WIDTH, scale=0.2), "grad": new(TOKENS, WIDTH)}


class Block:
    """norm -> queries, keys, values -> attention -> product -> dropout, residual, norm."""

    def __init__(self):
        self.norm = rb.LayerNorm(WIDTH, BF16)
        self.attention = rb.DocumentAttention(HEADS, DIM, KV, max_tokens=TOKENS)
        self.documents = rb.Documents(torch.tensor(OFFSETS, device="cuda"), None, torch.tensor(PREFIXES, device="cuda"))
        self.drop = rb.Drop(0.1, 11, 3)

    def __call__(self, t):
        y = self.norm(t["x"], t["w1"], t["b1"]).y
        q, k, v = (z.unflatten(1, (n, DIM)) for z, n in zip((y @ t["qkv"].t()).split([HEADS * DIM, KV * DIM, KV * DIM], 1), (HEADS, KV, KV)))
        a = self.attention(q, k, v, self.documents).flatten(1)
        o = self.norm(a @ t["back"].t(), t["w2"], None, residual=t["x"], drop=self.drop)
        return rb.dropout(o.y, self.drop._replace(step=4)) + o.total


def plain(t):
    """The same in 64 bits, without any of it."""
    y = ref.norm(t["x"], t["w1"], t["b1"], 1e-5)[0]
    q, k, v = (z.unflatten(1, (n, DIM)) for z, n in zip((y @ t["qkv"].t()).split([HEADS * DIM, KV * DIM, KV * DIM], 1), (HEADS, KV, KV)))
    mask = ref.seen(TOKENS, OFFSETS, None, PREFIXES)
    s = torch.einsum("ihd,jhd->hij", q, ref.spread(k, HEADS)) * DIM ** -0.5
    some = mask.any(1)
    p = torch.softmax(torch.where(mask | ~some[:, None], s, -float("inf")), 2) * some[:, None]
    a = torch.einsum("hij,jhd->ihd", p, ref.spread(v, HEADS)).flatten(1)
    x = a @ t["back"].t()
    total = x * ref.kept(TOKENS, WIDTH, rb.Drop(0.1, 11, 3)) + t["x"]
    return ref.norm(total, t["w2"], None, 1e-5)[0] * ref.kept(TOKENS, WIDTH, rb.Drop(0.1, 11, 4)) + total


def test_a_block_and_its_gradients():
    """Against the same in 64 bits.  Seven roundings to bfloat16 lie one behind another on the way to the result, and as many back: 16 half steps
    of the sizes on the way, of which results and gradients are sums (norms: sqrt(sum of squares) of errors at most that of sizes, with a factor of 2 for sizes that cancel)."""
    block, t = Block(), tensors()
    leaves = {n: x.clone().requires_grad_() for n, x in t.items()}
    out = block(leaves)
    out.backward(t["grad"])
    at = {n: ref.to64(x).requires_grad_() for n, x in t.items()}
    want = plain(at)
    want.backward(at["grad"].detach())
    assert (ref.to64(out) - want).norm() <= 32 * ref.BF16_HALF * want.norm()
    for n in t:
        if n != "grad":
            d = (ref.to64(leaves[n].grad) - at[n].grad).norm() / at[n].grad.norm()
            assert d <= 32 * ref.BF16_HALF, (n, float(d))


def test_a_captured_step_is_the_eager_one():
    """Forward and backward of a block in a graph, replayed with other inputs, the program's own work between the replays."""
    block = Block()
    norm, attention = block.norm, block.attention
    inputs = tensors(1)
    x, w, d = inputs["x"], inputs["w1"], block.drop
    q, k, v = (torch.randn((TOKENS, n, DIM), device="cuda").to(BF16) for n in (HEADS, KV, KV))
    g = torch.randn((TOKENS, HEADS, DIM), device="cuda").to(BF16)

    def step(into):
        o = norm.forward(x, w, None, residual=inputs["grad"], drop=d, out=into[0])
        n = norm.grad(inputs["grad"], o.total, w, o.mean, o.rstd, grad_total=x, drop=d, bias=False, out=into[1])
        a = attention.forward(q, k, v, block.documents, out=into[2])
        grads = attention.grad(q, k, v, block.documents, a.out, a.lse, g, out=into[3])
        return [*o, *[z for z in n if z is not None], *a, *grads, rb.dropout(x, d, out=into[4])]

    def new():
        return (norm.outputs(TOKENS, total=True), norm.gradients(TOKENS, bias=False, drop=True), attention.outputs(TOKENS), tuple(torch.empty_like(z) for z in (q, k, v)),
                torch.empty_like(x))
    kept, other = new(), new()
    step(kept)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(kept)
    for turn in range(4):
        for z in (x, w, inputs["grad"], q, k, v, g):
            z.copy_(torch.randn(z.shape, generator=torch.Generator("cuda").manual_seed(turn), device="cuda").to(BF16))
        graph.replay()
        torch.cuda.synchronize()
        got = [z.clone() for z in captured]
        for a, b in zip(got, step(other)):
            assert torch.equal(a, b), turn
        torch.cuda.synchronize()


def test_calls_on_streams_in_turn_and_handles_that_are_dropped_behind_them():
    norm, attention = rb.LayerNorm(5000, F32), rb.DocumentAttention(4, 64, 1, max_tokens=700)
    docs = rb.Documents(torch.tensor([0, 300, 700], device="cuda"))
    w = torch.ones(5000, device="cuda")
    x = [torch.randn((900, 5000), generator=torch.Generator("cuda").manual_seed(i), device="cuda") for i in range(3)]
    q = [[torch.randn((700, n, 64), generator=torch.Generator("cuda").manual_seed(10 * i + n), device="cuda").to(BF16) for n in (4, 1, 1, 4)] for i in range(3)]

    def both(i, into):
        o = norm.forward(x[i], w, out=into[0])
        n = norm.grad(x[i], x[i], w, o.mean, o.rstd, out=into[1])
        a = attention.forward(*q[i][:3], docs, out=into[2])
        return [o.y, n.total, n.weight, n.bias, a.out, *attention.grad(*q[i][:3], docs, a.out, a.lse, q[i][3], out=into[3])]

    def new():
        return norm.outputs(900), norm.gradients(900), attention.outputs(700), tuple(torch.empty((700, n, 64), dtype=BF16, device="cuda") for n in (4, 1, 1))
    want = [[z.clone() for z in both(i, new())] for i in range(3)]
    into = [new() for _ in range(3)]
    size = norm.workspace.numel(), attention.workspace.numel()
    streams = [torch.cuda.Stream() for _ in range(2)] + [torch.cuda.current_stream()]
    torch.cuda.synchronize()
    for turn in range(4):
        for i in range(3):
            with torch.cuda.stream(streams[(i + turn) % 3]):
                both(i, into[i])
    with torch.cuda.stream(streams[0]):
        got = [both(i, into[i]) for i in range(3)]
    del norm, attention
    for n in size:
        torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(y, z) for y, z in zip(a, b))


def test_backward_raises_for_what_a_call_has_overwritten():
    norm, attention = rb.LayerNorm(40, F32), rb.DocumentAttention(1, 8, max_tokens=6)
    x, w = torch.randn((6, 40), device="cuda"), torch.ones(40, device="cuda", requires_grad=True)
    o = norm(x, w)
    norm.forward(x.clone(), w.detach(), out=rb.Normed(x, None, o.mean.clone(), None))         # the row that was saved
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.y.sum().backward()
    q = torch.randn((6, 1, 8), device="cuda").to(BF16).requires_grad_()
    docs = rb.Documents(torch.tensor([0, 6], device="cuda"))
    y = (q * q).sum()
    attention.forward(q.detach().clone(), q.detach(), q.detach(), docs, out=rb.Attended(q.detach(), None))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    z = torch.randn((6, 40), device="cuda", requires_grad=True)
    y = (z * z).sum()
    with torch.no_grad():
        rb.dropout(z, rb.Drop(0.5, 1, 1), out=z)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_no_rows_and_no_positions():
    norm, attention = rb.LayerNorm(24, BF16), rb.DocumentAttention(2, 16, max_tokens=5)
    x, w = torch.empty((0, 24), dtype=BF16, device="cuda", requires_grad=True), torch.ones(24, dtype=BF16, device="cuda", requires_grad=True)
    o = norm(x, w, residual=x, drop=rb.Drop(0.5, 1, 1))
    assert o.y.shape == o.total.shape == (0, 24) and o.mean.shape == (0,)
    rb.dropout(o.y, rb.Drop(0.5, 1, 2)).sum().backward()
    assert x.grad.shape == (0, 24) and (w.grad == 0).all()
    q = torch.empty((0, 2, 16), dtype=BF16, device="cuda", requires_grad=True)
    out = attention(q, q, q, rb.Documents(torch.zeros(1, dtype=torch.int64, device="cuda")))
    out.sum().backward()
    assert out.shape == (0, 2, 16) and q.grad.shape == (0, 2, 16)


def test_gradients_that_are_broadcast_or_lie_anyhow():
    attention = rb.DocumentAttention(2, 16, max_tokens=50)
    docs = rb.Documents(torch.tensor([0, 20, 50], device="cuda"))
    q, k, v = (torch.randn((50, 2, 16), device="cuda").to(BF16).requires_grad_() for _ in range(3))
    out = attention(q, k, v, docs)
    out.sum().backward()                                  # strides of 0
    o = attention.forward(q.detach(), k.detach(), v.detach(), docs)
    want = attention.grad(q.detach(), k.detach(), v.detach(), docs, o.out, o.lse, torch.ones_like(o.out))
    assert all(torch.equal(x.grad, y) for x, y in zip((q, k, v), want))
    for x in (q, k, v):
        x.grad = None
    c = torch.randn((16, 2, 50), device="cuda").to(BF16)
    (attention(q, k, v, docs) * c.permute(2, 1, 0)).sum().backward()       # numbers of a head apart
    want = attention.grad(q.detach(), k.detach(), v.detach(), docs, o.out, o.lse, c.permute(2, 1, 0).contiguous())
    assert all(torch.equal(x.grad, y) for x, y in zip((q, k, v), want))


@pytest.mark.parametrize("causal,heads,kv,dim,cap", [(True, 8, 1, 64, 0.0), (True, 2, 2, 128, 20.0), (False, 4, 2, 40, 0.0)])
def test_keys_whose_queries_are_cut_into_parts(causal, heads, kv, dim, cap):
    """Long documents: parts that begin in the middle of a head, another number of parts for every length; against the sum head by head of the same call."""
    for tokens, offsets in ((1500, [0, 1500]), (2048, [0, 700, 2000]), (700, [0, 1, 699])):
        g = torch.Generator("cuda").manual_seed(tokens)
        q, d = (torch.randn((tokens, heads, dim), generator=g, device="cuda").to(BF16) for _ in range(2))
        k, v = (torch.randn((tokens, kv, dim), generator=g, device="cuda").to(BF16) for _ in range(2))
        a = rb.DocumentAttention(heads, dim, kv, max_tokens=tokens, causal=causal, cap=cap)
        docs = rb.Documents(torch.tensor(offsets, device="cuda"))
        o = a.forward(q, k, v, docs)
        whole = a.grad(q, k, v, docs, o.out, o.lse, d)
        one = rb.DocumentAttention(1, dim, 1, max_tokens=tokens, causal=causal, cap=cap)
        sums, sizes = [torch.zeros((tokens, kv, dim), dtype=torch.float64, device="cuda") for _ in range(2)], [torch.zeros((tokens, kv, dim), dtype=torch.float64, device="cuda") for _ in range(2)]
        for h in range(heads):
            of = h // (heads // kv)
            args = [x[:, i:i + 1] for x, i in ((q, h), (k, of), (v, of))]
            p = one.forward(*args, docs)
            assert torch.equal(p.out[:, 0], o.out[:, h]) and torch.equal(p.lse[0], o.lse[h])
            r = one.grad(*args, docs, p.out, p.lse, d[:, h:h + 1])
            assert torch.equal(r[0][:, 0], whole[0][:, h])
            for n in range(2):
                sums[n][:, of] += r[1 + n][:, 0].double()
                sizes[n][:, of] += r[1 + n][:, 0].double().abs()
        for n in range(2):
            # each head's was rounded once, and the sum once; sums in binary32 of up to 2048 terms in another order: their sizes are at most some 2^6 of the result's here
            assert ((whole[1 + n].double() - sums[n]).abs() <= 2.0 ** -8 * (sizes[n] + sums[n].abs()) + 2.0 ** -24 * 4096 * 64).all()


def test_many_documents():
    """More than a workgroup looks through."""
    tokens = 5000
    offsets = torch.arange(0, tokens + 1, 2, device="cuda")
    q, k, v = (torch.randn((tokens, 1, 16), device="cuda").to(BF16) for _ in range(3))
    a = rb.DocumentAttention(1, 16, max_tokens=tokens)
    got = a.forward(q, k, v, rb.Documents(offsets)).out.float()
    q64, k64, v64 = (x.double()[:, 0] for x in (q, k, v))
    assert torch.equal(got[::2, 0], v.float()[::2, 0])                # the first of each sees itself alone
    s0, s1 = (q64[1::2] * k64[0::2]).sum(1) / 4, (q64[1::2] * k64[1::2]).sum(1) / 4
    p = torch.sigmoid(s1 - s0)[:, None]
    want = (1 - p) * v64[0::2] + p * v64[1::2]
    assert ((got[1::2, 0] - want).abs() <= 2.0 ** -7 * ((1 - p) * v64[0::2].abs() + p * v64[1::2].abs()) * 1.1).all()
    assert torch.equal(a.forward(q[:4000], k[:4000], v[:4000], rb.Documents(offsets[:2001])).out, got[:4000].to(BF16))
