"""Accumulation into an embedding's gradient leaves rows without a token as they are, bit for bit; rows with one get the rounded sum."""
import pytest

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("to", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("N,V,D", [(1, 2, 1), (40, 5, 32), (3000, 5, 33), (20000, 8, 300), (20000, 16, 4), (1, 16, 1000), (70, 17, 9), (9000, 40, 130), (70000, 200, 5)])
def test_rows_without_a_token_keep_their_bits(N, V, D, dtype, to):
    import torch
    import paper_2103_07013_amd as bps
    g = torch.Generator().manual_seed(N + V + D)
    used = torch.rand(V, generator=g) < 0.5
    used[0], used[-1] = True, False
    some = used.nonzero()[:, 0]
    tokens = some[torch.randint(0, len(some), (N,), generator=g)]
    tokens[torch.rand(N, generator=g) < 0.1] = -1
    tokens[torch.rand(N, generator=g) < 0.1] = V
    used = torch.zeros(V, dtype=torch.bool)
    used[tokens[(tokens >= 0) & (tokens < V)]] = True
    grad = torch.randn((N, D), generator=g).to(getattr(torch, dtype))
    kind = getattr(torch, to)
    out = torch.randn((V, D), generator=g).to(kind)
    out[:, 0] = -0.0
    bits = torch.int32 if to == "float32" else torch.int16
    if D > 2:      # a NaN that arithmetic would make a quiet one, and an infinity
        out.view(bits)[~used, 1] = {"float32": 0x7F800123, "bfloat16": 0x7F83, "float16": 0x7C03}[to]
        out[~used, 2] = float("-inf")
    got = bps.embedding_backward(tokens.cuda(), grad.cuda(), V, scale=1.5, out=out.cuda(), accumulate=True).cpu()
    assert torch.equal(got.view(bits)[~used], out.view(bits)[~used])
    inside = (tokens >= 0) & (tokens < V)
    total, size = torch.zeros((V, D), dtype=torch.float64), torch.zeros((V, D), dtype=torch.float64)
    total.index_add_(0, tokens[inside], grad[inside].double())
    size.index_add_(0, tokens[inside], grad[inside].double().abs())
    ref = (out.double() + 1.5 * total)[used]
    # n terms of a sum in float32, their product, and its addition, then the type's half distance
    slack = ((N + 2) * E * 1.5 * size)[used] + E * ref.abs()
    half = {"float32": 0.0, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[to]
    assert ((got.double()[used] - ref).abs() <= slack + half * (ref.abs() + slack) + 2.0 ** -25 * (to == "float16")).all()


def test_a_table_that_others_write_to_meanwhile():
    """Two calls on two streams accumulate into different rows of one small table."""
    import torch
    import paper_2103_07013_amd as bps
    out = torch.zeros((8, 64), device="cuda")
    grad = torch.ones((4096, 64), device="cuda")
    tokens = [torch.full((4096,), k, dtype=torch.int32, device="cuda") for k in (2, 5)]
    streams = [torch.cuda.Stream() for _ in tokens]
    torch.cuda.synchronize()
    for _ in range(20):
        for t, s in zip(tokens, streams):
            bps.embedding_backward(t, grad, 8, out=out, accumulate=True, stream=s)
    torch.cuda.synchronize()
    assert (out[2] == 20 * 4096).all() and (out[5] == 20 * 4096).all() and int(torch.count_nonzero(out)) == 128


def test_replays_of_a_graph():
    """Which rows have a token is found in every replay."""
    import torch
    import paper_2103_07013_amd as bps
    out, grad = torch.full((8, 64), -0.0, device="cuda"), torch.ones((500, 64), device="cuda")
    tokens = torch.zeros(500, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bps.embedding_backward(tokens, grad, 8, out=out, accumulate=True)
    for k in (3, 1, 7, 3):
        tokens.fill_(k)
        out.fill_(-0.0)
        graph.replay()
        torch.cuda.synchronize()
        ref = torch.full((8, 64), -0.0)
        ref[k] = 500.0
        assert torch.equal(out.cpu().view(torch.int32), ref.view(torch.int32))
