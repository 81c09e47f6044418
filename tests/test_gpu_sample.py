"""GPU tests of the choice of tokens against the fp64 oracle: equal tokens, probabilities to fp32.

The library holds weights to 2^-42 of the row's largest or better, so a decision differs from
the oracle's only where a border lies within 2^-22 of it (2^20 weights) -- the random rows here, of at
most 2^18, come that close with a chance below 1e-6 a row; rows built on a border use exact weights."""
import numpy as np
import pytest

from gpu_common import log, torch_cuda
from oracle import serving as ref

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def compare(z, u, **settings):
    """z on the GPU, any dtype; settings as numpy arrays."""
    torch = torch_cuda()
    from paper_2607_09686_amd import sample
    n = z.shape[0]
    kinds = {"temperature": np.float32, "top_k": np.int32, "top_p": np.float32, "min_p": np.float32}
    given = {k: np.broadcast_to(np.asarray(v, kinds[k]), (n,)) for k, v in settings.items()}
    u = np.broadcast_to(np.asarray(u, np.float32), (n,))
    gpu = lambda a: torch.from_numpy(a.copy()).cuda()  # noqa: E731
    tokens, probs = sample(z, gpu(u), **{k: gpu(v) for k, v in given.items()})
    assert tokens.dtype == torch.int32 and probs.dtype == torch.float32
    tokens, probs, host = tokens.cpu().numpy(), probs.cpu().numpy(), z.double().cpu().numpy()
    for r in range(n):
        s = {k: (int(v[r]) if k == "top_k" else float(v[r])) for k, v in given.items()}
        token, prob = ref.choose(host[r], float(u[r]), **s)
        assert tokens[r] == token, (r, tokens[r], token, s, u[r])
        assert abs(probs[r] - prob) <= 2.0 ** -23 * prob + 2.0 ** -40, (r, probs[r], prob)
    return tokens, probs


def random_rows(torch, rows, vocab, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    z = 2 * torch.randn(rows, vocab, generator=g) - 2 * torch.log(torch.rand(rows, vocab, generator=g) + 1e-6)
    z[torch.rand(rows, vocab, generator=g) < 0.02] = -INF
    z[:, 0] = 1.0  # no row without a choice
    return z.to(dtype).cuda()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (5, 63), (4, 64), (4, 65), (9, 1000), (3, 4097), (2, 32003),
                                        (70, 5001), (3, 8192), (3, 8193), (3, 16384), (3, 16385), (2, 152001), (1, 262144)])
def test_random_rows_and_settings(dtype, rows, vocab):
    torch = torch_cuda()
    log(f"sample {rows} x {vocab} {dtype}")
    rng = np.random.default_rng(vocab)
    z = random_rows(torch, rows, vocab, getattr(torch, dtype), vocab)
    for trial in range(6):
        pick = lambda *v: rng.choice(v, rows)  # noqa: E731
        compare(z, rng.random(rows), temperature=pick(0.0, 0.3, 0.7, 1.0, 1.5, 3.0),
                top_k=pick(0, 1, 2, 50, 1000, vocab, vocab + 1, -3), top_p=pick(1.0, 0.1, 0.5, 0.9, 0.999, 2.0),
                min_p=pick(0.0, 0.01, 0.1, 0.5, 1.0, -1.0))


def test_the_longest_rows_and_the_most():
    torch = torch_cuda()
    rng = np.random.default_rng(12)
    z = random_rows(torch, 2, 1 << 20, torch.float32, 4)
    compare(z, rng.random(2), temperature=[1.0, 2.5], top_k=[0, 30000], top_p=[0.97, 0.8])
    z = random_rows(torch, 2500, 8500, torch.bfloat16, 5)
    compare(z, rng.random(2500), top_k=rng.integers(0, 300, 2500), top_p=rng.choice([1.0, 0.9], 2500))
    z = random_rows(torch, 65535, 5, torch.float32, 6)
    compare(z, rng.random(65535), min_p=rng.choice([0.0, 0.3], 65535))


def test_one_filter_at_a_time():
    torch = torch_cuda()
    rng = np.random.default_rng(1)
    z = random_rows(torch, 32, 20011, torch.float32, 3)
    u = rng.random(32)
    compare(z, u)
    compare(z, u, temperature=rng.uniform(0.1, 4, 32))
    compare(z, u, top_k=rng.integers(1, 20011, 32))
    compare(z, u, top_p=rng.random(32))
    compare(z, u, min_p=rng.random(32) ** 4)
    compare(z, u, temperature=1e6)  # nearly uniform: every token counts
    compare(z, u, temperature=1e-3)


@pytest.mark.parametrize("dtype,rows,vocab", [("float32", 12, 7001), ("bfloat16", 12, 20003), ("float32", 5, 152001)])
def test_min_p_alone(dtype, rows, vocab):
    torch = torch_cuda()
    rng = np.random.default_rng(vocab)
    z = random_rows(torch, rows, vocab, getattr(torch, dtype), vocab + 1)
    for least in (1.0, 0.3, 1e-3, 1e-9, 1e-30, 1e-45):
        compare(z, rng.random(rows), temperature=rng.choice([0.2, 1.0, 4.0, 1e-30, 1e30], rows), min_p=least)


def test_slices_of_more_than_one_step():
    torch = torch_cuda()
    rng = np.random.default_rng(8)
    z = random_rows(torch, 1040, 20001, torch.bfloat16, 9)  # a wave's part of a slice: 626 elements
    compare(z, rng.random(1040), temperature=rng.choice([1.0, 5.0], 1040), top_p=rng.choice([1.0, 0.999], 1040))


def test_ties():
    """Rows of few distinct logits: the filters cut inside runs of equal ones."""
    torch = torch_cuda()
    rng = np.random.default_rng(2)
    for vocab in (7, 3000, 8000, 70000):
        z = torch.from_numpy(rng.integers(-2, 3, (24, vocab)).astype(np.float32)).cuda()
        z[0] = 0.0
        z[1] = 0.0
        z[1, vocab // 2] = 1.0
        for t in (z, z.bfloat16()):
            compare(t, rng.random(24), top_k=rng.integers(0, vocab + 2, 24))
            # masses of integer logits at temperature 1 are no dyadic numbers: no p lies on a border
            compare(t, rng.random(24), top_p=rng.uniform(0.05, 0.95, 24), top_k=rng.integers(0, vocab + 2, 24))
            compare(t, rng.random(24), temperature=0.0)


def test_masses_that_the_bins_get_wrong():
    """A quarter million weights just below a half over a whole number of 2^-31, which is where the bins that
    choose what is ranked round to: all are rounded down, the cut lies a good part of a bin from
    where the bins put it.  The first token carries the draw; its share shows the cut (a bin's
    elements are 1e-4 of it, the comparison's 2^-23)."""
    torch = torch_cuda()
    rng = np.random.default_rng(14)
    for vocab in (8000, 1 << 18):
        whole = rng.integers(10, 1000, (24, vocab)) if vocab > 10000 else rng.integers(10, 40, (24, vocab)) * 1000
        z = np.log((whole + 0.49) / 2 ** 31)
        z[:, 0] = 0.0
        mass = np.exp(z.astype(np.float32).astype(np.float64)).sum(1)
        p = 1 / mass + (1 - 1 / mass) * np.linspace(0.05, 0.95, 24)  # cuts spread over the small weights
        tokens, _ = compare(torch.from_numpy(z).float().cuda(), 0.3, top_p=p)
        assert (tokens == 0).all()


def test_nearly_all_of_the_mass():
    """Cuts far out, where thousands of elements share a bin."""
    torch = torch_cuda()
    z = random_rows(torch, 12, 152001, torch.float32, 21)
    rng = np.random.default_rng(15)
    compare(z, rng.random(12), top_p=[0.99, 0.995, 0.999, 0.9995, 0.9999, 0.99999] * 2,
            temperature=[1.0] * 6 + [1.5] * 6)
    compare(z.bfloat16(), rng.random(12), top_p=[0.99, 0.995, 0.999, 0.9995, 0.9999, 0.99999] * 2,
            temperature=[1.0] * 6 + [2.0] * 6, top_k=[0, 100000] * 6)


def test_borders_on_exact_weights():
    """Four equal logits: masses 1/4 each, and p, u on the borders between them."""
    torch = torch_cuda()
    z = torch.full((1, 5000), -INF, device="cuda")
    at = [17, 1024, 1025, 4999]
    z[0, at] = 2.5
    for u, want in ((0.0, 17), (0.2499999, 17), (0.25, 1024), (0.5, 1025), (0.75, 4999), (0.9999999, 4999),
                    (1.0, 4999), (2.0, 4999), (-1.0, 17), (NAN, 17), (INF, 4999), (-INF, 17)):
        tokens, probs = compare(z, u)
        assert tokens[0] == want and probs[0] == 0.25
    for p, u, want in ((0.25, 0.99, 17), (0.250001, 0.99, 1024), (0.5, 0.99, 1024), (0.75, 0.99, 1025),
                       (0.76, 0.99, 4999), (0.0, 0.99, 17), (-1.0, 0.99, 17), (NAN, 0.99, 4999)):
        assert compare(z, u, top_p=p)[0][0] == want
    assert compare(z, 0.99, min_p=1.0)[0][0] == 4999
    assert compare(z, 0.99, min_p=NAN)[0][0] == 4999


def test_special_rows():
    torch = torch_cuda()
    V = 3001
    z = torch.zeros(12, V)
    z[0] = -INF
    z[1] = NAN
    z[2] = -INF
    z[2, 5] = NAN
    z[3, 10], z[3, 2000] = INF, INF
    z[4, 7] = NAN
    z[5] = -INF
    z[5, V - 1] = -1e30
    z[6] = 3e38
    z[6, 100:] = -3e38
    z[7, 0] = -0.0
    z[8] = -INF
    z[8, 40] = INF
    z[9] = torch.linspace(-1e-38, 1e-38, V)  # subnormals
    z[10, 3] = NAN
    z[10, 4] = INF
    z[11] = torch.arange(V) * 1e-3
    rng = np.random.default_rng(3)
    for dtype in (torch.float32, torch.bfloat16):
        zz = z.to(dtype).cuda()
        for s in ({}, {"top_k": 3}, {"top_p": 0.6}, {"min_p": 0.2}, {"temperature": 0.0}, {"temperature": 0.7, "top_k": 900},
                  {"top_k": 2000, "top_p": 0.5, "min_p": 0.9}, {"temperature": INF}, {"temperature": NAN},
                  {"temperature": -1.0}):
            compare(zz, rng.random(12), **s)


def test_strided_rows_and_no_rows():
    torch = torch_cuda()
    from paper_2607_09686_amd import sample
    wide = random_rows(torch, 6, 3000, torch.float32, 8)
    before = wide.clone()
    compare(wide[:, 5:2006], np.linspace(0, 0.99, 6), top_p=0.8)
    compare(wide[::2, 1:], np.linspace(0, 0.99, 3), top_k=40)
    assert torch.equal(wide, before)
    tokens, probs = sample(wide[:0], torch.empty(0, device="cuda"))
    assert tokens.shape == probs.shape == (0,)


def test_the_same_tokens_alone_in_a_batch_and_on_another_stream():
    torch = torch_cuda()
    from paper_2607_09686_amd import sample
    z = random_rows(torch, 130, 9001, torch.float32, 9)
    u = torch.rand(130, device="cuda")
    p = torch.full((130,), 0.9, device="cuda")
    tokens, probs = sample(z, u, top_p=p)
    for r in (0, 64, 129):
        t, q = sample(z[r:r + 1], u[r:r + 1], top_p=p[r:r + 1])
        assert t.item() == tokens[r].item() and q.item() == probs[r].item()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        t, q = sample(z, u, top_p=p)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(t, tokens) and torch.equal(q, probs)


def test_replayed_graphs():
    torch = torch_cuda()
    from paper_2607_09686_amd import sample
    graphs = []
    for rows, vocab in ((3, 40001), (40, 2003)):
        z, u = random_rows(torch, rows, vocab, torch.float32, rows), torch.rand(rows, device="cuda")
        k = torch.full((rows,), 100, dtype=torch.int32, device="cuda")
        p = torch.full((rows,), 0.9, device="cuda")
        sample(z, u, top_k=k, top_p=p)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = sample(z, u, top_k=k, top_p=p)
        graphs.append((g, out, z, u, k, p))
    for r in range(4):
        for g, out, z, u, k, p in graphs:
            z.copy_(z.roll(r + 1, 1))
            u.copy_(torch.rand_like(u))
            k.fill_((0, 5, 700, 1)[r])
            want = sample(z, u, top_k=k, top_p=p)
            out[0].fill_(-7)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_refusals():
    torch = torch_cuda()
    from paper_2607_09686_amd import MoeError, sample
    z, u = torch.zeros(2, 10, device="cuda"), torch.zeros(2, device="cuda")
    for bad in (z.cpu(), z[0], z.t()):
        with pytest.raises(ValueError):
            sample(bad, u)
    with pytest.raises(TypeError):
        sample(z.double(), u)
    with pytest.raises(ValueError):
        sample(z, u[:1])
    with pytest.raises(TypeError):
        sample(z, u, top_k=u)
    with pytest.raises(ValueError):
        sample(z, u, top_p=u.cpu())
    with pytest.raises(MoeError):
        sample(torch.zeros(1, (1 << 20) + 1, device="cuda"), u[:1])
    with pytest.raises(MoeError):  # rows that overlap
        sample(z.as_strided((2, 10), (4, 1)), u)
