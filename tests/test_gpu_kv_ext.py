"""GPU tests of norms at appending, of a cache of 8 bits (written, read back, attended to) and of
attention behind shared tokens, against the fp64 oracle."""
import numpy as np
import pytest

from gpu_common import log, torch_cuda
from kv_ext_common import LIMITS, ExtBatch
from oracle import serving as ref
from serving_common import half_step

pytestmark = pytest.mark.gpu

EDGES = [(1, n - 1) for n in (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 257, 1000)]


def types():
    torch = torch_cuda()
    return {"bf16": torch.bfloat16, "f16": torch.float16}


def pool_values(b, which, s, positions):
    """(numbers, exponents) or values of sequence s's tokens as the pools hold them, in 64 bits."""
    torch = b.torch
    at = np.asarray(positions)
    page = torch.from_numpy(b.table[s, at // b.page]).long().cuda()
    p = torch.from_numpy(at % b.page).cuda()
    pools = [x[0] for x in b.pools()]
    if which == "k":
        x = pools[0][page, :, p // 16, :, p % 16].flatten(2)
    else:
        x = pools[1][page, :, p // 16, p // 8 % 2, :, p % 8]
    if not b.held:
        return x.view(b.dtype).double().cpu().numpy()
    e = pools[2 if which == "k" else 3][page, :, p].long().cpu().numpy() - 127
    return x.contiguous().view(torch.float8_e4m3fn).double().cpu().numpy(), e


# ------------------------------------------------------------------------------ appending

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (256, 32)])
@pytest.mark.parametrize("seqs", [[(1, 0), (1, 6), (9, 7), (0, 30), (40, 129), (16, 16), (3, 500), (2, 63)],
                                  [(8, 8)], [(5, 3), (6, 8), (7, 1), (4, 4)]])
def test_numbers_and_scales(dtype, dim, page, seqs):
    """Without a turn what is written is the definition's, bit for bit; nothing else is touched."""
    torch = torch_cuda()
    b = ExtBatch(torch, seqs, 6, 2, dim, page, types()[dtype], seed=dim, pad_rows=2, filled=False)
    rng = np.random.default_rng(3)
    size = 2.0 ** rng.integers(-30, 30, (b.n, 2, 1)) if dtype == "bf16" else 2.0 ** rng.integers(-20, 16, (b.n, 2, 1))
    x = {n: torch.from_numpy((rng.standard_normal((b.n, 2, dim)) * size).astype(np.float32)) for n in "kv"}
    x["k"][0] = 0.0
    x["v"][-3] = 448.0  # exactly at a scale's end, and past it
    x["v"][-4] = torch.nextafter(torch.tensor(448.0), torch.tensor(500.0))
    before = [p.clone() for p in b.pools()]
    b.cache(rope_dim=0).append(x["k"].cuda(), x["v"].cuda(), *b.index())
    touched = 0
    for s in range(len(seqs)):
        pos = b.positions(s)
        if not len(pos):
            continue
        for name in "kv":
            got, e = pool_values(b, name, s, pos)
            want, exponent = ref.hold(x[name][b.rows(s)].double().numpy(), *LIMITS[str(b.dtype)])
            np.testing.assert_array_equal(e, exponent)
            np.testing.assert_array_equal(got, want)
        touched += len(pos)
    changed = [(p != q).sum().item() for p, q in zip(b.pools(), before)]
    assert changed[2] == changed[3] == 2 * touched
    assert changed[0] <= 2 * dim * touched and changed[1] <= 2 * dim * touched


@pytest.mark.parametrize("source", ["own", "f32"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_vectors_that_are_not_finite_or_out_of_range(dtype, source):
    torch = torch_cuda()
    t = types()[dtype]
    b = ExtBatch(torch, [(9, 5)], 2, 1, 64, 16, t, filled=False)
    inf, nan = float("inf"), float("nan")
    x = torch.randn(9, 1, 64, generator=torch.Generator().manual_seed(1))
    big = 3e38 if source == "f32" or dtype == "bf16" else 65504.0
    x[0, 0, 3], x[1, 0, 60], x[2, 0, 0], x[3], x[4] = nan, inf, -inf, nan, 0.0
    x[5] *= big / 8
    x[5, 0, 9], x[6, 0, 5], x[6, 0, 6], x[7] = big, inf, nan, x[7] * 1e-30
    x[8] = x[8] * 2.0 ** -13
    x = x.to(t) if source == "own" else x
    b.cache(rope_dim=0).append(x.cuda(), x.cuda(), *b.index())
    want, exponent = ref.hold(x.double().numpy(), *LIMITS[str(t)])
    for name in "kv":
        got, e = pool_values(b, name, 0, b.positions(0))
        np.testing.assert_array_equal(e, exponent)
        np.testing.assert_array_equal(got, want)
    k, v = b.cache().read(9, *b.index())
    stands = want * 2.0 ** exponent[..., None].astype(np.float64)
    for got in (k, v):  # the type holds what the numbers stand for, exactly
        np.testing.assert_array_equal(got.double().cpu().numpy(), stands)


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("dtype,source,weights", [("bf16", "bf16", "own"), ("bf16", "f32", "f32"), ("f16", "f16", "f32"),
                                                  ("f16", "f32", "own")])
@pytest.mark.parametrize("dim,rope_dim,adjacent,page", [(64, 64, False, 16), (128, 128, False, 64),
                                                        (128, 64, True, 32), (256, 256, True, 16),
                                                        (64, 16, False, 1024), (256, 0, False, 128)])
@pytest.mark.parametrize("which", ["both", "q", "k"])
def test_norms_and_turns(held, dtype, source, weights, dim, rope_dim, adjacent, page, which):
    """A norm's factor is off by (dim / 32 + 6) 2^-24 of itself at most (sums of 16 to a lane and five exchanges, a
    division, a root, a quotient, two products), a turn as in plain appending by 2^-20 of its pair; then an element's
    rounding to its type: half a step of 16 bits, or of e4m3: 2^-4 of it, or 2^-10 of the scale."""
    torch = torch_cuda()
    t, s = types()[dtype], torch.float32 if source == "f32" else types()[source]
    w = torch.float32 if weights == "f32" else t
    seqs = [(1, 0), (1, 6), (9, 7), (0, 30), (40, 129), (16, 16), (3, 5000)]
    b = ExtBatch(torch, seqs, 6, 2, dim, page, t, held=held, seed=dim, filled=False, pad_rows=2)
    rng = np.random.default_rng(5)
    x = {n: torch.from_numpy(3.0 * rng.standard_normal((b.n, h, dim))).to(s) for n, h in (("q", 6), ("k", 2), ("v", 2))}
    x["k"][0] = 0.0
    weight = {n: torch.from_numpy(1 + 0.3 * rng.standard_normal(dim)).to(w) for n in "qk"}
    give = {n + "_norm": weight[n].cuda() for n in "qk" if which in (n, "both")}
    eps = 1e-5
    cache = b.cache(rope_dim=rope_dim, rope_adjacent=adjacent, rope_theta=5e5)
    q_out = torch.full((b.n, 6, dim), 7.0, dtype=t, device="cuda")
    got_q = cache.append(x["k"].cuda(), x["v"].cuda(), *b.index(), q=x["q"].cuda(), q_out=q_out, norm_eps=eps, **give)
    assert got_q is q_out and (q_out[-2:] == 7).all()
    got_q = got_q.double().cpu().numpy()
    freqs = [5e5 ** (-2 * i / rope_dim) for i in range(rope_dim // 2)]
    h, tiny = half_step(t), float(torch.finfo(t).smallest_normal) * torch.finfo(t).eps
    for i, (n, before) in enumerate(seqs):
        r, pos = b.rows(i), b.positions(i)
        if not n:
            continue
        for name in ("q", "k"):
            a = x[name][r].double().numpy()
            if name + "_norm" in give:
                a = ref.head_norm(a, weight[name].double().numpy(), eps)
            want = ref.rotate(a, pos, freqs, adjacent)
            fp32 = (2.0 ** -20 + (dim / 32 + 6) * 2.0 ** -24) * np.abs(a).max() * 2
            if name == "q":
                assert (np.abs(got_q[r] - want) <= h * np.abs(want) + fp32 + tiny).all()
            elif not held:
                assert (np.abs(pool_values(b, "k", i, pos) - want) <= h * np.abs(want) + fp32 + tiny).all()
            else:
                c, e = pool_values(b, "k", i, pos)
                scale = 2.0 ** e[..., None].astype(np.float64)
                err = np.abs(c * scale - want)
                assert (err <= 2.0 ** -4 * np.abs(want) + 2.0 ** -10 * scale + fp32 * (1 + 2.0 ** -4)).all()
                most = np.abs(want).max(-1, keepdims=True)
                lo, hi = (2.0 ** p for p in LIMITS[str(t)])
                assert ((scale <= lo) | (most >= scale * 224 * (1 - 2.0 ** -15))).all()
                assert ((scale >= hi) | (most <= scale * 448 * (1 + 2.0 ** -15))).all()
        v = x["v"][r].double().numpy()
        if held:
            c, e = pool_values(b, "v", i, pos)
            want, exponent = ref.hold(v, *LIMITS[str(t)])
            np.testing.assert_array_equal(e, exponent)
            np.testing.assert_array_equal(c, want)
        else:
            np.testing.assert_array_equal(pool_values(b, "v", i, pos), x["v"][r].to(t).double().numpy())


def test_a_norm_of_q_in_its_own_place():
    torch = torch_cuda()
    for dim in (64, 128, 256):
        b = ExtBatch(torch, [(20, 3), (1, 9)], 4, 2, dim, 16, torch.bfloat16, held=False)
        k, w = torch.randn(b.n, 2, dim, device="cuda").to(b.dtype), torch.rand(dim, device="cuda")
        q = b.q_gpu()
        want = b.cache().append(k, k, *b.index(), q=q, q_norm=w, k_norm=w)
        assert b.cache().append(k, k, *b.index(), q=q, q_out=q, q_norm=w, k_norm=w) is q
        assert torch.equal(q, want)


def test_weights_of_one_without_a_norm():
    """A weight of ones on rows of mean square one, eps 0: the rows themselves, to their rounding."""
    torch = torch_cuda()
    b = ExtBatch(torch, [(33, 3)], 4, 2, 128, 16, torch.float16, held=False)
    q = torch.sign(torch.randn(b.n, 4, 128, device="cuda")).to(b.dtype)
    one = torch.ones(128, dtype=b.dtype, device="cuda")
    k = torch.zeros(b.n, 2, 128, dtype=b.dtype, device="cuda")
    got = b.cache(rope_dim=0).append(k, k, *b.index(), q=q, q_norm=one, norm_eps=0.0)
    assert torch.equal(got, q)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("size", [2.0 ** -60, 2.0 ** -20, 2.0 ** 20, 2.0 ** 55])
def test_the_range_of_a_norm(dim, size):
    """Elements of up to eight times `size`, eps 0: squares and their sum stay fp32's normal numbers, so that the
    tolerance is as ever (what lies far below the largest counts for nothing in the sum)."""
    torch = torch_cuda()
    b = ExtBatch(torch, [(33, 3), (1, 9)], 4, 2, dim, 16, torch.bfloat16, held=False)
    g = torch.Generator().manual_seed(dim)
    q, k = (torch.randn(b.n, h, dim, generator=g).clamp(-4, 4) * 2 * size for h in (4, 2))
    w = torch.rand(dim, generator=g) + 0.5
    got = b.cache(rope_dim=0).append(k.cuda(), k.cuda(), *b.index(), q=q.cuda(), q_norm=w.cuda(), norm_eps=0.0)
    want = ref.head_norm(q.double().numpy(), w.double().numpy(), 0.0)
    assert (np.abs(got.double().cpu().numpy() - want) <= (2.0 ** -8 + (dim / 32 + 6) * 2.0 ** -24) * np.abs(want)).all()


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim", [(7, 7, 64), (320, 64, 64), (1024, 1, 128), (130, 65, 256)])
def test_any_number_of_heads(held, heads, kv_heads, dim):
    """Each head of each token by itself: its norm, and what it is held as (no turn, no q for the second call)."""
    torch = torch_cuda()
    b = ExtBatch(torch, [(3, 30), (8, 8), (1, 77), (20, 3)], heads, kv_heads, dim, 16, torch.bfloat16, held=held, filled=False)
    g = torch.Generator().manual_seed(heads)
    q, k, v = (torch.randn(b.n, h, dim, generator=g) * 2 for h in (heads, kv_heads, kv_heads))
    w = torch.rand(dim, generator=g) + 0.5
    cache = b.cache(rope_dim=0)
    got = cache.append(k.cuda(), v.cuda(), *b.index(), q=q.cuda(), q_norm=w.cuda(), k_norm=w.cuda(), norm_eps=0.5)
    fp32 = (dim / 32 + 6) * 2.0 ** -24
    want = ref.head_norm(q.double().numpy(), w.double().numpy(), 0.5)
    assert (np.abs(got.double().cpu().numpy() - want) <= (2.0 ** -8 + fp32) * np.abs(want)).all()
    kk, vv = (x.double().cpu().numpy() for x in cache.read(b.n, *b.index()))
    want = ref.head_norm(k.double().numpy(), w.double().numpy(), 0.5)
    if held:
        most = np.abs(want).max(-1, keepdims=True)
        assert (np.abs(kk - want) <= (2.0 ** -4 + 2 * fp32) * np.abs(want) + 2.0 ** -17 * most).all()
        c, e = ref.hold(v.double().numpy(), -100, 119)
        np.testing.assert_array_equal(vv, c * 2.0 ** e[..., None].astype(np.float64))
    else:
        assert (np.abs(kk - want) <= (2.0 ** -8 + fp32) * np.abs(want)).all()
        np.testing.assert_array_equal(vv, v.bfloat16().double().numpy())
    pools = [p.clone() for p in b.pools()]
    assert cache.append(k.cuda(), v.cuda(), *b.index(), k_norm=w.cuda(), norm_eps=0.5) is None
    assert all(torch.equal(p, x) for p, x in zip(b.pools(), pools))


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 64), (4, 1, 64), (3, 3, 64), (1, 1, 128), (8, 1, 256)])
@pytest.mark.parametrize("seqs", [[(1, 0)], [(8, 8)], [(3, 30), (8, 8), (1, 77), (20, 3)], [(300, 5)]])
def test_few_heads_without_q(held, dtype, heads, kv_heads, dim, seqs):
    """Keys under a norm and values into pools that hold NaN, by a call that has no queries: both are there.
    Tolerances as test_norms_and_turns'; values are bit for bit."""
    torch = torch_cuda()
    t = types()[dtype]
    b = ExtBatch(torch, seqs, heads, kv_heads, dim, 16, t, held=held, filled=False)
    g = torch.Generator().manual_seed(dim)
    k, v = (2 * torch.randn(b.n, kv_heads, dim, generator=g) for _ in "kv")
    w = torch.rand(dim, generator=g) + 0.5
    assert b.cache(rope_dim=0).append(k.cuda(), v.cuda(), *b.index(), k_norm=w.cuda(), norm_eps=0.5) is None
    norm = (dim / 32 + 6) * 2.0 ** -24
    for s in range(len(seqs)):
        r, pos = b.rows(s), b.positions(s)
        want = ref.head_norm(k[r].double().numpy(), w.double().numpy(), 0.5)
        if held:
            c, e = pool_values(b, "k", s, pos)
            scale = 2.0 ** e[..., None].astype(np.float64)
            assert (np.abs(c * scale - want) <= (2.0 ** -4 + 2 * norm) * np.abs(want) + 2.0 ** -10 * scale).all()
            c, e = pool_values(b, "v", s, pos)
            number, exponent = ref.hold(v[r].double().numpy(), *LIMITS[str(t)])
            np.testing.assert_array_equal(c, number)
            np.testing.assert_array_equal(e, exponent)
        else:
            tiny = float(torch.finfo(t).smallest_normal) * half_step(t)
            assert (np.abs(pool_values(b, "k", s, pos) - want) <= (half_step(t) + 2 * norm) * np.abs(want) + tiny).all()
            np.testing.assert_array_equal(pool_values(b, "v", s, pos), v[r].to(t).double().numpy())


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("counts", [[1] * 64, [1] * 65, [n % 12 for n in range(300)], [1] * 1100, [0] * 90 + [9] + [0] * 90])
def test_many_sequences_written_and_read(held, counts):
    torch = torch_cuda()
    b = ExtBatch(torch, [(n, 7 * i % 50) for i, n in enumerate(counts)], 4, 2, 64, 16, torch.float16, held=held, filled=False,
                 pad_rows=2)
    x = torch.from_numpy(np.random.default_rng(1).standard_normal((2, b.n, 2, 64))).float()
    w = torch.ones(64, device="cuda")
    cache = b.cache(rope_dim=0)
    cache.append(x[0].cuda(), x[1].cuda(), *b.index(), k_norm=w)
    k = torch.full((b.n, 2, 64), 7.0, dtype=b.dtype, device="cuda")
    k, v = cache.read(b.n, *b.index(), k=k)
    new = b.n - 2
    assert (k[new:] == 7).all()
    if held:
        c, e = ref.hold(x[1, :new].double().numpy(), -15, 7)
        want = c * 2.0 ** e[..., None].astype(np.float64)
    else:
        want = x[1, :new].half().double().numpy()
    np.testing.assert_array_equal(v[:new].double().cpu().numpy(), want)
    want = ref.head_norm(x[0, :new].double().numpy(), np.ones(64), 1e-6)
    step = 2.0 ** -4 if held else 2.0 ** -11
    near = (step + 16 * 2.0 ** -24) * np.abs(want) + 2.0 ** -17 * np.abs(want).max(-1, keepdims=True)
    assert (np.abs(k[:new].double().cpu().numpy() - want) <= near).all()


@pytest.mark.parametrize("held", [False, True])
def test_strided_rows(held):
    """q, k and v as slices of one projection's output, with norms; rows read back into slices."""
    torch = torch_cuda()
    for seqs in ([(1, 77), (1, 5)], [(90, 20)]):
        b = ExtBatch(torch, seqs, 4, 2, 128, 64, torch.bfloat16, held=held, filled=False)
        flat = torch.randn(b.n, 8 * 128 + 64, device="cuda").to(b.dtype)
        q, k, v = flat[:, :512].view(b.n, 4, 128), flat[:, 512:768].view(b.n, 2, 128), flat[:, 768:1024].view(b.n, 2, 128)
        w = torch.rand(128, device="cuda") + 0.5
        wide = torch.full((b.n, 6, 128), 7.0, dtype=b.dtype, device="cuda")
        cache = b.cache()
        cache.append(k, v, *b.index(), q=q, q_out=wide[:, 1:5], q_norm=w, k_norm=w)
        pools = [p.clone() for p in b.pools()]
        got = cache.append(k.contiguous(), v.contiguous(), *b.index(), q=q.contiguous(), q_norm=w, k_norm=w)
        assert torch.equal(wide[:, 1:5], got) and (wide[:, 0] == 7).all() and (wide[:, 5] == 7).all()
        assert all(torch.equal(p, x) for p, x in zip(b.pools(), pools))
        o = torch.full((b.n, 6, 128), 7.0, dtype=b.dtype, device="cuda")
        cache.read(b.n, *b.index(), k=o[:, 1:3], v=o[:, 3:5])
        want = cache.read(b.n, *b.index())
        assert torch.equal(o[:, 1:3], want[0]) and torch.equal(o[:, 3:5], want[1])
        assert (o[:, 0] == 7).all() and (o[:, 5] == 7).all()


# ------------------------------------------------------------------------------ reading back

@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (256, 1024)])
def test_read(held, dtype, dim, page):
    torch = torch_cuda()
    seqs = [(1, 0), (0, 4), (40, 7), (8, 8), (3, 500), (16, 16), (9, 55), (70, 0)]
    b = ExtBatch(torch, seqs, 4, 2, dim, page, types()[dtype], held=held, seed=dim, pad_rows=3)
    k = torch.full((b.n, 2, dim), 7.0, dtype=b.dtype, device="cuda")
    wide = torch.full((b.n, 5, dim), 7.0, dtype=b.dtype, device="cuda")
    v = wide[:, 2:4]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = b.cache().read(b.n, *b.index(), k=k, v=v, status=status)
    assert got[0] is k and got[1] is v and status.item() == 0
    for s in range(len(seqs)):
        if b.new[s]:
            for got, want in ((k, b.k), (v, b.v)):
                np.testing.assert_array_equal(got[b.rows(s)].double().cpu().numpy(), want[s][-b.new[s]:])
    assert (k[-3:] == 7).all() and (wide[-3:] == 7).all() and (wide[:, :2] == 7).all() and (wide[:, 4] == 7).all()


@pytest.mark.parametrize("held", [False, True])
def test_read_what_cannot_be(held):
    torch = torch_cuda()
    b = ExtBatch(torch, [(20, 30), (20, 20), (5, 90)], 4, 2, 64, 16, torch.bfloat16, held=held)
    b.lengths[1] = 19
    b.pages[2, 5] = b.n_pages
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    k, v = b.cache().read(b.n, *b.index(), status=status)
    assert status.item() == 3
    for got, want in ((k, b.k), (v, b.v)):
        got = got.double().cpu().numpy()
        np.testing.assert_array_equal(got[b.rows(0)], want[0][-20:])
        assert np.isnan(got[b.rows(1)]).all()
        place = np.arange(90, 95) // 16 == 5
        assert place.any() and np.isnan(got[b.rows(2)][place]).all()
        np.testing.assert_array_equal(got[b.rows(2)][~place], want[2][-5:][~place])


def test_what_is_appended_is_read():
    """Whole sequences, appended by chunks and read at once."""
    torch = torch_cuda()
    from paper_2607_09686_amd import KvCache
    cache = KvCache(2, 4, 2, 128, 32, 40, rope_dim=0, storage=torch.float8_e4m3fn)
    pages = torch.randperm(40, generator=torch.Generator().manual_seed(2)).to(torch.int32).view(2, 20).cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    x = torch.randn(2, 2, 600, 2, 128, generator=torch.Generator().manual_seed(3)).cuda()  # k, v of two sequences
    at = 0
    for n in (1, 7, 8, 100, 3, 256, 1, 224):
        k, v = (y[:, at:at + n].flatten(0, 1).contiguous() for y in x)
        cache.append(k, v, pages, i32(0, n, 2 * n), i32(at + n, at + n), layer=1)
        at += n
    k, v = cache.read(1200, pages, i32(0, 600, 1200), i32(600, 600), layer=1)
    for got, want in ((k, x[0]), (v, x[1])):
        c, e = ref.hold(want.flatten(0, 1).double().cpu().numpy(), -100, 119)
        np.testing.assert_array_equal(got.double().cpu().numpy(), c * 2.0 ** e[..., None].astype(np.float64))


# ------------------------------------------------------------------------------ attention over 8 bits

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("group,page", [(1, 16), (3, 64), (8, 32), (40, 1024)])
def test_one_new_token(dtype, dim, group, page):
    torch = torch_cuda()
    log(f"8 bits, one new token {dtype} dim {dim} group {group} page {page}")
    b = ExtBatch(torch, EDGES, 2 * group, 2, dim, page, types()[dtype], seed=dim + group)
    log(f"  worst error / tolerance {b.check(b.cache().attend(b.q_gpu(), *b.index())):.3f}")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("group,page,window", [(1, 16, 0), (4, 64, 0), (5, 32, 50), (2, 128, 1), (8, 16, 200),
                                               (4, 256, 64)])
def test_chunks(dtype, dim, group, page, window):
    torch = torch_cuda()
    log(f"8 bits, chunks {dtype} dim {dim} group {group} page {page} window {window}")
    seqs = [(70, 0), (1, 300), (33, 31), (64, 64), (0, 100), (129, 190), (5, 640)]
    b = ExtBatch(torch, seqs, group, 1, dim, page, types()[dtype], seed=dim + window)
    b.check(b.cache(window=window).attend(b.q_gpu(), *b.index()), window)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("seqs,window", [([(1, 20000), (1, 100)], 0), ([(40, 6000)], 0), ([(6, 9000), (6, 30)], 7777),
                                         ([(1, 1500)] * 70, 1100), ([(90, 4000)], 64), ([(n % 3, 20 * n) for n in range(200)], 0)])
def test_split_and_many(seqs, window, dtype):
    torch = torch_cuda()
    b = ExtBatch(torch, seqs, 8, 2, 128, 64, types()[dtype], seed=len(seqs))
    out = b.cache(window=window).attend(b.q_gpu(), *b.index())
    b.check(out, window)
    assert torch.equal(out, b.cache(window=window).attend(b.q_gpu(), *b.index()))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new", [1, 5, 90])
@pytest.mark.parametrize("dim", [64, 256])
def test_scales_of_every_size(dtype, new, dim):
    """Tokens whose values differ by many powers of two, some of them all zero."""
    torch = torch_cuda()
    b = ExtBatch(torch, [(new, 500), (new, 40)], 8, 2, dim, 32, types()[dtype], seed=new, filled=False)
    rng = np.random.default_rng(2)
    lo, hi = LIMITS[str(b.dtype)]
    for s in range(2):
        n = b.total[s]
        most = rng.integers(lo + 9, hi + 8, (n, 2, 1)) if dtype == "f16" else rng.integers(-60, 60, (n, 2, 1))
        v = rng.standard_normal((n, 2, dim)) * 2.0 ** (most - 2)
        k = rng.standard_normal((n, 2, dim)) * 2.0 ** -rng.integers(0, 20, (n, 2, 1))
        v[rng.random(n) < 0.2], k[rng.random(n) < 0.2] = 0.0, 0.0
        for i, x in enumerate((k, v)):
            b.codes[i][s] = ref.hold(x, lo, hi)
            c, e = b.codes[i][s]
            (b.k, b.v)[i][s] = c * 2.0 ** e[..., None].astype(np.float64)
        b.fill(s)
    b.check(b.cache().attend(b.q_gpu(), *b.index()))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("gap", [14.0, 17.5])
@pytest.mark.parametrize("dim,new,shared", [(64, 1, 0), (128, 5, 0), (256, 1, 0), (128, 70, 0), (128, 1, 3000), (64, 70, 3000)])
def test_a_first_key_far_above_the_rest(dtype, gap, dim, new, shared):
    """The first key's score is `gap` above the others', its value zero in most elements.  fp16 adds to Batch.check's
    tolerance that of its smallest numbers: a probability is off by at most half of 2^-24 where the largest is at
    least 2^10, so the output by 2^-35 of the sum of |v|."""
    torch = torch_cuda()
    before, group = 4000, 8
    b = ExtBatch(torch, [(new, before)] * 2, 2 * group, 2, dim, 64, types()[dtype], shared=shared, seed=7, filled=False)
    limits, rng = LIMITS[str(b.dtype)], np.random.default_rng(8)
    for s in range(2):
        if s and shared:  # both sequences are the same
            b.k[1], b.v[1] = b.k[0].copy(), b.v[0].copy()
        else:
            b.k[s][:, :, 0], b.k[s][0] = 0.0, 0.0
            b.k[s][0, :, 0] = gap * dim ** 0.5 / 8
            b.v[s] = np.abs(b.v[s]) + 0.5
            b.v[s][0, :, 2:] = 0.0
        for i, x in enumerate((b.k, b.v)):
            c, e = b.codes[i][s] = ref.hold(x[s], *limits)
            x[s] = c * 2.0 ** e[..., None].astype(np.float64)
        b.fill(s)
    b.q = rng.standard_normal((2 * new, 2 * group, dim)) * 0.5
    b.q[:, :, 0] = 8.0
    b.q = b.rounded(b.q)
    out = b.cache().attend(b.q_gpu(), *b.index(), **b.front()).double().cpu().numpy()
    h, scale = half_step(b.dtype), dim ** -0.5
    tiny = float(torch.finfo(b.dtype).smallest_normal) * h
    for s in range(2):
        rows, pos = b.q[b.rows(s)], b.positions(s)
        want, weight = ref.attend(rows, b.k[s], b.v[s], pos, scale)
        big = np.linalg.norm(rows, axis=2).max() * np.linalg.norm(b.k[s], axis=2).max() * scale
        ds = (dim + 8) * 2.0 ** -24 * big
        tol = h * np.abs(want) + (h + 2 * ds + 2.0 ** -18) * (1 + h) * weight + 4 * tiny
        if dtype == "f16":
            tol += 2.0 ** -35 * np.repeat(np.cumsum(np.abs(b.v[s]), axis=0)[pos], group, axis=1)
        err = np.abs(out[b.rows(s)] - want)
        assert np.all(err <= tol), (s, float((err / tol).max()))


@pytest.mark.parametrize("dtype,gap", [("bf16", 17.0), ("bf16", 21.0), ("bf16", 30.0), ("f16", 5.0), ("f16", 17.0)])
@pytest.mark.parametrize("dim,new,shared", [(64, 1, 0), (128, 5, 0), (256, 1, 0), (128, 70, 0), (128, 1, 3000), (64, 70, 3000)])
def test_the_least_scale_under_a_first_key_far_above_the_rest(dtype, gap, dim, new, shared):
    """All values are held with the least power of two, 2^e, and the first key, whose value is zero in most elements,
    scores about `gap` above the others.  bf16 rounds p 2^e for the product: below 2^-126 to within 2^-134, so a row is off by
    2^-134 |c| a token more than Batch.check's tolerance (the largest p being at least 1).  A gap of 17 (16 or 17 in e4m3, 24.6
    of log2, and the others' scores within 0.5 of 0) keeps p 2^-100 above 2^-126.  fp16 as the test above."""
    torch = torch_cuda()
    before, group = 4000, 8
    b = ExtBatch(torch, [(new, before)] * 2, 2 * group, 2, dim, 64, types()[dtype], shared=shared, seed=7, filled=False)
    limits, rng = LIMITS[str(b.dtype)], np.random.default_rng(8)
    for s in range(2):
        if s and shared:  # both sequences are the same
            b.k[1], b.v[1] = b.k[0].copy(), b.v[0].copy()
        else:
            b.k[s][:, :, 0], b.k[s][0] = 0.0, 0.0
            b.k[s] *= 0.1
            b.k[s][0, :, 0] = gap * dim ** 0.5 / 8
            b.v[s] = (np.abs(b.v[s]) + 0.5) * 2.0 ** (limits[0] + 5)
            b.v[s][0, :, 2:] = 0.0
        for i, x in enumerate((b.k, b.v)):
            c, e = b.codes[i][s] = ref.hold(x[s], *limits)
            assert i == 0 or (e == limits[0]).all()
            x[s] = c * 2.0 ** e[..., None].astype(np.float64)
        b.fill(s)
    b.q = rng.standard_normal((2 * new, 2 * group, dim)) * 0.5
    b.q[:, :, 0] = 8.0
    b.q = b.rounded(b.q)
    out = b.cache().attend(b.q_gpu(), *b.index(), **b.front()).double().cpu().numpy()
    h, scale = half_step(b.dtype), dim ** -0.5
    tiny = float(torch.finfo(b.dtype).smallest_normal) * h
    for s in range(2):
        rows, pos = b.q[b.rows(s)], b.positions(s)
        want, weight = ref.attend(rows, b.k[s], b.v[s], pos, scale)
        big = np.linalg.norm(rows, axis=2).max() * np.linalg.norm(b.k[s], axis=2).max() * scale
        ds = (dim + 8) * 2.0 ** -24 * big
        tol = h * np.abs(want) + (h + 2 * ds + 2.0 ** -18) * (1 + h) * weight + 4 * tiny
        if dtype == "f16":
            tol += 2.0 ** -35 * np.repeat(np.cumsum(np.abs(b.v[s]), axis=0)[pos], group, axis=1)
        elif gap > 17:
            tol += 2.0 ** (-134 - limits[0]) * np.repeat(np.cumsum(np.abs(b.v[s]), axis=0)[pos], group, axis=1)
        err = np.abs(out[b.rows(s)] - want)
        log(f"least scale {dtype} gap {gap} dim {dim} new {new} shared {shared}: {float((err / tol).max()):.3f}")
        assert np.all(err <= tol), (s, float((err / tol).max()))


@pytest.mark.parametrize("new,before", [(1, 0), (1, 400), (5, 300), (90, 100)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_the_largest_scales(new, before, dim):
    """bf16 values up to the sums that the header allows: one of 2^127 alone, exactly, or hundreds of 2^107."""
    torch = torch_cuda()
    b = ExtBatch(torch, [(new, before)], 8, 2, dim, 16, torch.bfloat16, seed=new, filled=False)
    most = 127.0 if new + before == 1 else 107.0
    b.v[0] *= 2.0 ** most / np.abs(b.v[0]).max()
    for i, x in enumerate((b.k, b.v)):
        c, e = b.codes[i][0] = ref.hold(x[0], *LIMITS[str(b.dtype)])
        x[0] = c * 2.0 ** e[..., None].astype(np.float64)
    assert b.codes[1][0][1].max() == (119 if most == 127 else 99)
    b.fill(0)
    out = b.cache().attend(b.q_gpu(), *b.index())
    if most == 127:
        np.testing.assert_array_equal(out.double().cpu().numpy(), np.repeat(b.v[0], 4, axis=1))
    else:
        b.check(out)


@pytest.mark.parametrize("seqs,row", [([(5, 60)], 2), ([(120, 40)], 50), ([(120, 700)], 119)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_what_a_row_does_not_see_has_no_effect(seqs, row, dtype):
    """Token `row` of the new ones holds NaN numbers, or scales that are none: rows before it are as ever,
    the later ones get NaN in just those elements (of values), or in all (of keys)."""
    torch = torch_cuda()
    b = ExtBatch(torch, seqs, 4, 2, 64, 16, types()[dtype], seed=row)
    cache, q = b.cache(), b.q_gpu()
    clean = cache.attend(q, *b.index())
    t = seqs[0][1] + row
    page, place = int(b.table[0, t // 16]), t % 16
    keys, values, ks, vs = b.pools()
    for d in (3, 40):
        values[0, page, 1, 0, place // 8, d, place % 8] = 0xff
    out = cache.attend(q, *b.index())
    assert torch.equal(out[:row], clean[:row]) and torch.equal(out[:, :2], clean[:, :2])
    for d in range(64):
        got = out[row:, 2:, d]
        assert torch.isnan(got).all() if d in (3, 40) else torch.equal(got, clean[row:, 2:, d]), d
    b.fill(0)
    keys[0, page, 0, 0, 2, place, 1] = 0x7f
    out = cache.attend(q, *b.index())
    assert torch.equal(out[:row], clean[:row]) and torch.isnan(out[row:, :2]).all()
    assert torch.equal(out[:, 2:], clean[:, 2:])
    b.fill(0)
    ks[0, page, 0, place], vs[0, page, 0, place] = 255, 255
    out = cache.attend(q, *b.index())
    assert torch.equal(out[:row], clean[:row]) and torch.equal(out[:, 2:], clean[:, 2:])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim,new,page", [(64, 1, 16), (128, 3, 32), (256, 5, 16), (64, 40, 16), (128, 200, 64)])
def test_what_a_window_has_passed_has_no_effect(dtype, dim, new, page):
    """Old tokens with numbers and scales that are none, and page ids that are none before them."""
    torch = torch_cuda()
    window, before = 50, 420
    b = ExtBatch(torch, [(new, before), (new, 30)], 8, 2, dim, page, types()[dtype], seed=new, first_page=1)
    cache, q = b.cache(window=window), b.q_gpu()
    clean = cache.attend(q, *b.index())
    b.check(clean, window)
    gone = before - window + 1  # tokens that no new one sees
    keys, values, ks, vs = b.pools()
    for t in (gone - 1, gone - 2, gone - 40):
        pg, at = int(b.table[0, t // page]), t % page
        keys[0, pg, :, at // 16, :, at % 16], values[0, pg, :, at // 16, at // 8 % 2, :, at % 8] = 0x7f, 0xff
        ks[0, pg, :, at], vs[0, pg, :, at] = 255, 255
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert torch.equal(cache.attend(q, *b.index(), status=status), clean) and status.item() == 0
    b.pages[0, :gone // page] = -1
    assert torch.equal(cache.attend(q, *b.index(), status=status), clean) and status.item() == 0


@pytest.mark.parametrize("new", [1, 90])
def test_bad_lengths_and_pages(new):
    torch = torch_cuda()
    for length in (-1, new - 1, 10 ** 6, -2 ** 31, 2 ** 31 - 1):
        b = ExtBatch(torch, [(new, 30), (new, 20), (2, 50)], 4, 2, 64, 16, torch.bfloat16)
        b.lengths[1] = length
        cache, status = b.cache(), torch.zeros(1, dtype=torch.int32, device="cuda")
        out = cache.attend(b.q_gpu(), *b.index(), status=status)
        assert torch.isnan(out[b.rows(1)]).all() and status.item() == 2
        b.check(out, skip=(1,))
        own = torch.from_numpy(b.table[1, :-(-b.total[1] // 16)]).long().cuda()
        before = [p[0, own].clone() for p in b.pools()]
        k, w = torch.ones(b.n, 2, 64, dtype=b.dtype, device="cuda"), torch.ones(64, device="cuda")
        q = cache.append(k, k, *b.index(), q=b.q_gpu(), q_norm=w, k_norm=w)
        assert torch.isnan(q[b.rows(1)]).all() and not torch.isnan(q[b.rows(0)]).any()
        assert all(torch.equal(p[0, own], x) for p, x in zip(b.pools(), before))
    for page_id in (-1, 2 ** 31 - 1):
        b = ExtBatch(torch, [(new, 30), (new, 3000), (2, 50)], 4, 2, 64, 16, torch.bfloat16)
        b.pages[1, 3] = page_id
        cache, status = b.cache(), torch.zeros(1, dtype=torch.int32, device="cuda")
        out = cache.attend(b.q_gpu(), *b.index(), status=status)
        assert torch.isnan(out[b.rows(1)]).all() and status.item() == 1
        b.check(out, skip=(1,))
        b.pages[0, (30 + new - 1) // 16] = page_id  # the page of sequence 0's last new token
        last = int(b.table[0, (30 + new - 1) // 16])
        before = [p[0, last].clone() for p in b.pools()]
        k = torch.ones(b.n, 2, 64, dtype=b.dtype, device="cuda")
        status.zero_()
        q = cache.append(k, k, *b.index(), q=b.q_gpu(), status=status)
        assert status.item() == 1 and not torch.isnan(q).any()
        assert all(torch.equal(p[0, last], x) for p, x in zip(b.pools(), before))


@pytest.mark.parametrize("held,shared", [(True, 0), (False, 30), (True, 64)])
@pytest.mark.parametrize("seqs", [[(3, 70), (60, 79), (1, 500)], [(1, 80)] * 90 + [(60, 99)] * 3])
def test_starts_out_of_order_stay_in_bounds(held, shared, seqs):
    """Whatever starts, lengths and the shared count hold: the calls end, and rows outside the tensor's stay."""
    torch = torch_cuda()
    rng = np.random.default_rng(9)
    w = torch.ones(64, device="cuda")
    for trial in range(8):
        b = ExtBatch(torch, seqs, 4, 2, 64, 16, torch.bfloat16, held=held, shared=shared, seed=trial)
        n = len(seqs) + 1
        wrong = rng.integers(-2 ** 31, 2 ** 31 - 1, n) if trial % 2 else rng.integers(-5, b.n + 5, n)
        b.starts = torch.tensor(wrong, dtype=torch.int32, device="cuda")
        if shared and trial > 3:
            b.count.fill_(int(rng.integers(-2 ** 31, 2 ** 31 - 1)) if trial % 2 else int(rng.integers(-3, shared + 40)))
        whole = torch.full((b.n + 64, 4, 64), 7.0, dtype=b.dtype, device="cuda")
        rows = torch.full((2, b.n + 64, 2, 64), 7.0, dtype=b.dtype, device="cuda")
        out = whole[32:32 + b.n]
        cache = b.cache()
        cache.attend(b.q_gpu(), *b.index(), out=out, **b.front())
        k = torch.ones(b.n, 2, 64, dtype=b.dtype, device="cuda")
        cache.append(k, k, *b.index(), q=b.q_gpu(), q_out=out, q_norm=w, k_norm=w)
        cache.read(b.n, *b.index(), k=rows[0, 32:32 + b.n], v=rows[1, 32:32 + b.n])
        torch.cuda.synchronize()
        assert (whole[:32] == 7).all() and (whole[32 + b.n:] == 7).all()
        assert (rows[:, :32] == 7).all() and (rows[:, 32 + b.n:] == 7).all()


# ------------------------------------------------------------------------------ behind shared tokens

@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (256, 32)])
@pytest.mark.parametrize("shared,seqs", [
    (0, [(1, 5), (2, 90)]), (1, [(1, 5), (2, 90)]), (63, [(1, 0), (1, 9)]), (64, [(1, 0), (1, 70), (0, 3), (1, 300)]),
    (130, [(1, n) for n in (0, 1, 14, 15, 16, 62, 63, 64, 65)]), (640, [(5, 0), (5, 100), (1, 3), (0, 0), (8, 40)]),
    (1000, [(70, 0), (3, 700), (130, 90)]), (2048, [(1, n) for n in range(90)])])
def test_behind_shared_tokens(held, dtype, dim, page, shared, seqs):
    torch = torch_cuda()
    log(f"shared {shared}: held {held} {dtype} dim {dim} page {page} {seqs[:4]} x {len(seqs)}")
    seqs = [(n, shared + p) for n, p in seqs]
    b = ExtBatch(torch, seqs, 8, 2, dim, page, types()[dtype], held=held, shared=shared, seed=shared, pad_rows=1)
    if not shared:
        b.shared, b.prefix, b.count = 1, b.pages[0, :1].clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((b.n, 8, dim), 7.0, dtype=b.dtype, device="cuda")
    cache = b.cache()
    cache.attend(b.q_gpu(), *b.index(), out=out, **b.front())
    log(f"  worst error / tolerance {b.check(out):.3f}")
    assert (out[-1] == 7).all()
    again = cache.attend(b.q_gpu(), *b.index(), **b.front())
    assert torch.equal(out[:-1], again[:-1])


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("group,seqs", [(1, [(1, 3)] * 2), (8, [(1, 100)] * 8), (4, [(1, 9)] * 2), (40, [(1, 9), (2, 900)]),
                                        (2, [(1, n) for n in range(200)])])
def test_a_long_prefix(held, group, seqs):
    torch = torch_cuda()
    seqs = [(n, 9000 + p) for n, p in seqs]
    b = ExtBatch(torch, seqs, 2 * group, 2, 128, 64, torch.bfloat16, held=held, shared=9000, seed=group)
    b.check(b.cache().attend(b.q_gpu(), *b.index(), **b.front()))


def test_a_prefix_of_more_pages_than_one_list_of_ids():
    torch = torch_cuda()
    for new, n in ((1, 2), (1, 600), (9, 600)):
        b = ExtBatch(torch, [(new, 20000)], 2, 1, 64, 16, torch.bfloat16, shared=19990, seed=4)
        q = torch.from_numpy(np.random.default_rng(6).standard_normal((n * new, 2, 64))).to(b.dtype)
        pages, lengths = b.pages.expand(n, -1).contiguous(), b.lengths.expand(n).contiguous()
        starts = torch.arange(0, n * new + 1, new, dtype=torch.int32, device="cuda")
        out = b.cache().attend(q.cuda(), pages, starts, lengths, **b.front())
        for s in (0, 1, n // 2, n - 1):
            b.q = q[s * new:(s + 1) * new].double().numpy()
            b.check(out[s * new:(s + 1) * new])


def test_as_many_sequences_as_a_batch_may_have():
    """65536 of one token with 64 KV heads, 2^22 tiles, behind the same tokens: no more threads than a grid holds,
    and every row joined."""
    torch = torch_cuda()
    n = 65536
    b = ExtBatch(torch, [(1, 70)], 64, 64, 64, 16, torch.bfloat16, held=False, shared=64)
    q = torch.randn(n, 64, 64, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(b.dtype)
    starts = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    lengths = b.lengths - (torch.arange(n, dtype=torch.int32, device="cuda") % 6)
    out = torch.full_like(q, float("nan"))
    index = b.pages.expand(n, -1).contiguous(), starts, lengths
    b.cache().attend(q, *index, out=out, **b.front())
    near = b.cache().attend(q, *index)
    assert torch.isfinite(out).all()
    assert (out.float() - near.float()).norm() <= 2 * half_step(b.dtype) * near.float().norm()
    k, v = b.k[0], b.v[0]
    for s in (0, 1, n // 2, n - 5, n - 1):
        total = int(lengths[s])
        b.q, b.k[0], b.v[0], b.total[0] = q[s:s + 1].double().cpu().numpy(), k[:total], v[:total], total
        b.check(out[s:s + 1])


def test_the_prefix_may_lie_in_pages_of_its_own():
    torch = torch_cuda()
    b = ExtBatch(torch, [(1, 300), (2, 320), (40, 260)], 8, 2, 128, 16, torch.float16, held=False, shared=256, own_front=True)
    b.check(b.cache().attend(b.q_gpu(), *b.index(), **b.front()))


def test_less_is_shared_than_the_prefix_holds():
    """A table of prefix pages with room for more: the count decides, at replay too."""
    torch = torch_cuda()
    b = ExtBatch(torch, [(1, 700), (1, 650), (3, 690)], 8, 2, 64, 16, torch.bfloat16, shared=640)
    b.prefix = torch.cat([b.prefix, torch.full((500,), -1, dtype=torch.int32, device="cuda")])
    b.prefix[20:] = 2 ** 30  # not reached below
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache, q = b.cache(), b.q_gpu()
    g = torch.cuda.CUDAGraph()
    for count in (320, 319, 256, 64, 63, 0):
        b.count.fill_(count)
        out = cache.attend(q, *b.index(), status=status, **b.front())
        b.check(out)
        assert status.item() == 0
    with torch.cuda.graph(g):
        out = cache.attend(q, *b.index(), **b.front())
    for count in (100, 0, 320, 256):
        b.count.fill_(count)
        want = cache.attend(q, *b.index(), **b.front())
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("page,shared", [(16, 100), (16, 63), (32, 160), (64, 127), (128, 130)])
@pytest.mark.parametrize("new", [1, 40])
def test_which_of_the_prefix_pages_are_read(held, page, shared, new):
    """Those of its whole 64s of tokens: a bad id there makes every row NaN, one past them has no effect."""
    torch = torch_cuda()
    b = ExtBatch(torch, [(new, shared + 40), (new, shared), (2, 300)], 4, 2, 64, page, torch.bfloat16, held=held, shared=shared)
    cache, q, status = b.cache(), b.q_gpu(), torch.zeros(1, dtype=torch.int32, device="cuda")
    clean = cache.attend(q, *b.index(), status=status, **b.front())
    b.check(clean)
    read = -(-(shared // 64 * 64) // page)  # pages
    prefix = b.prefix.clone()
    for page_id in (-1, b.n_pages):
        b.prefix[:] = prefix
        b.prefix[read:] = page_id
        assert torch.equal(cache.attend(q, *b.index(), status=status, **b.front()), clean) and status.item() == 0
        if read:
            b.prefix[read - 1] = page_id
            assert torch.isnan(cache.attend(q, *b.index(), status=status, **b.front())).all() and status.item() == 1
            status.zero_()


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("many", [0, 80])
def test_what_is_no_prefix(new, many):
    """Sequences whose new tokens would lie in it, counts that are none, page ids that are none."""
    torch = torch_cuda()
    seqs = [(new, 140), (new, 100), (new, 200), (0, 3)] + [(new, 128)] * many
    b = ExtBatch(torch, seqs, 4, 2, 64, 16, torch.bfloat16, held=False, shared=100)
    cache, q, status = b.cache(), b.q_gpu(), torch.zeros(1, dtype=torch.int32, device="cuda")
    b.count.fill_(101)
    out = cache.attend(q, *b.index(), status=status, **b.front())
    assert torch.isnan(out[b.rows(1)]).all() and status.item() == 2
    assert not torch.isnan(out[b.rows(0)]).any() and not torch.isnan(out[b.rows(2)]).any()
    for count in (-1, 7 * 16 + 1, 2 ** 31 - 1, -2 ** 31):
        b.count.fill_(count)
        status.zero_()
        out = cache.attend(q, *b.index(), status=status, **b.front())
        assert torch.isnan(out).all() and status.item() == 2
    b.count.fill_(100)
    status.zero_()
    b.check(cache.attend(q, *b.index(), status=status, **b.front()))
    assert status.item() == 0
    for page_id in (-1, b.n_pages, 2 ** 31 - 1):
        b.prefix[2] = page_id
        status.zero_()
        out = cache.attend(q, *b.index(), status=status, **b.front())
        assert torch.isnan(out).all() and status.item() == 1


@pytest.mark.parametrize("new", [1, 70])
def test_a_bad_sequence_behind_a_prefix(new):
    torch = torch_cuda()
    b = ExtBatch(torch, [(new, 300), (new, 280), (2, 256)], 4, 2, 128, 16, torch.float16, shared=256)
    b.lengths[1] = 10 ** 6
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = b.cache().attend(b.q_gpu(), *b.index(), status=status, **b.front())
    assert torch.isnan(out[b.rows(1)]).all() and status.item() == 2
    b.check(out, skip=(1,))
    b.lengths[1] = b.total[1]
    b.pages[0, 16] = -1
    status.zero_()
    out = b.cache().attend(b.q_gpu(), *b.index(), status=status, **b.front())
    assert torch.isnan(out[b.rows(0)]).all() and status.item() == 1
    b.check(out, skip=(0,))


# ------------------------------------------------------------------------------ everything

@pytest.mark.parametrize("seed", range(60))
def test_random_batches(seed):
    torch = torch_cuda()
    rng = np.random.default_rng(2000 + seed)
    dim, page = int(rng.choice([64, 128, 256])), int(rng.choice([16, 32, 64, 256]))
    kv, group = int(rng.choice([1, 2, 3])), int(rng.choice([1, 2, 5, 8, 13]))
    most, far = int(rng.choice([1, 4, 8, 40, 150])), int(rng.choice([3, 90, 700, 2500]))
    n = int(rng.integers(1, 9 if most > 8 else 80 if far < 100 else 20))
    shared, held = int(rng.choice([0, 1, 64, 100, 777, 3000])), bool(rng.random() < 0.6)
    seqs = [(int(rng.integers(0 if rng.random() < 0.2 else min(1, most), most + 1)), shared + int(rng.integers(0, far + 1)))
            for _ in range(n)]
    window = 0 if shared else int(rng.choice([0, 0, 1, 17, 64, 333, 5000]))
    dtype = [torch.bfloat16, torch.float16][seed % 2]
    log(f"random {seed}: dim {dim} page {page} kv {kv} group {group} window {window} shared {shared} held {held} "
        f"{n} sequences {seqs[:3]} ...")
    b = ExtBatch(torch, seqs, kv * group, kv, dim, page, dtype, held=held, shared=shared, seed=seed,
                 pad_rows=int(rng.integers(0, 3)), width=-(-(shared + most + far) // page) + int(rng.integers(0, 40)))
    if b.n:
        b.check(b.cache(window=window).attend(b.q_gpu(), *b.index(), **b.front()), window)


@pytest.mark.parametrize("held", [False, True])
def test_streams_and_replayed_graphs(held):
    """Two captured graphs of all the operators, each replayed several times on new contents among eager
    calls."""
    torch = torch_cuda()
    side = torch.cuda.Stream()
    graphs = []
    for seed, seqs, shared in ((1, [(1, 300), (1, 7000), (1, 240)], 200), (2, [(3, 90), (80, 200)], 64), (3, [(1, 90)] * 70, 65)):
        b = ExtBatch(torch, seqs, 8, 2, 128, 32, torch.bfloat16, held=held, shared=shared, seed=seed, width=240, spare=20)
        cache = b.cache()
        q, w = b.q_gpu(), torch.rand(128, device="cuda") + 0.5
        k = torch.randn(b.n, 2, 128, device="cuda").to(b.dtype)

        def step(b=b, cache=cache, q=q, k=k, w=w):
            turned = cache.append(k, k, *b.index(), q=q, q_norm=w, k_norm=w)
            return (turned, cache.attend(turned, *b.index(), **b.front()), cache.attend(turned, *b.index()),
                    *cache.read(b.n, *b.index()))

        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((b, g, out, q, k, step))
    for r in range(4):
        for b, g, out, q, k, step in graphs:
            q.copy_(q.roll(1, 0))
            k.copy_(k.roll(1, 0))
            if r == 2:  # another length at replay: the sequence loses its last tokens
                b.lengths -= 1
            want = step()
            for x in out:
                x.fill_(0)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(out, want)), (r, b.seqs)
            near = (want[1].float() - want[2].float()).norm() / want[2].float().norm()
            assert near <= 2 * half_step(b.dtype)


@pytest.mark.parametrize("held", [False, True])
def test_two_streams_at_once(held):
    """All the operators on two batches, queued in turns on two streams without a wait between them, and a third
    batch that both read: as one after the other."""
    torch = torch_cuda()
    w = torch.rand(128, device="cuda") + 0.5
    sides = []
    for seed, seqs, shared in ((1, [(1, 2000 + 40 * n) for n in range(40)], 1900), (2, [(90, 700), (5, 4000), (300, 600)], 600),
                               (3, [(1, 500), (3, 3000)], 70)):
        b = ExtBatch(torch, seqs, 8, 2, 128, 32, torch.bfloat16, held=held, shared=shared, seed=seed)
        sides.append((b, b.cache(), b.q_gpu(), torch.randn(b.n, 2, 128, device="cuda").to(b.dtype)))
    common, common_cache, common_q, _ = sides.pop()

    def step(b, cache, q, k):
        turned = cache.append(k, k, *b.index(), q=q, q_norm=w, k_norm=w)
        return (turned, cache.attend(turned, *b.index(), **b.front()), cache.attend(turned, *b.index()),
                *cache.read(b.n, *b.index()), common_cache.attend(common_q, *common.index(), **common.front()))

    want = [step(*side) for side in sides]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sides]
    got = []
    for _ in range(20):
        for i, (side, stream) in enumerate(zip(sides, streams)):
            with torch.cuda.stream(stream):
                got.append((i, step(*side)))
    torch.cuda.synchronize()
    for i, out in got:
        assert all(torch.equal(x, y) for x, y in zip(out, want[i])), i


def test_pages_past_32_bit_offsets():
    torch = torch_cuda()
    page_elems = 8 * 1024 * 128
    first = 2 ** 32 // page_elems + 5  # element offsets past 2^32
    b = ExtBatch(torch, [(1, 1500), (80, 1000)], 8, 8, 128, 1024, torch.bfloat16, first_page=first, shared=900)
    cache = b.cache(rope_dim=0)
    b.check(cache.attend(b.q_gpu(), *b.index()))
    b.check(cache.attend(b.q_gpu(), *b.index(), **b.front()))
    k = torch.from_numpy(np.concatenate([x[-n:] for x, n in zip(b.k, b.new)])).to(b.dtype).cuda()
    for p in b.pools():
        p[:, first:] = 0
    cache.append(k, k, *b.index())
    got_k, got_v = cache.read(b.n, *b.index())
    assert torch.equal(got_k, k) and torch.equal(got_v, k)  # what 8 bits gave, they hold


def test_refusals():
    torch = torch_cuda()
    from paper_2607_09686_amd import MoeError
    b = ExtBatch(torch, [(4, 80)], 4, 2, 64, 16, torch.bfloat16, shared=64)
    cache, q = b.cache(), b.q_gpu()
    k, w = torch.zeros(4, 2, 64, dtype=b.dtype, device="cuda"), torch.ones(64, device="cuda")
    index, front = b.index(), b.front()
    for wrong in (dict(prefix=b.prefix), dict(shared=b.count), dict(prefix=b.prefix[:0], shared=b.count),
                  dict(prefix=b.prefix[None], shared=b.count), dict(prefix=b.prefix, shared=b.starts),
                  dict(prefix=b.prefix.cpu(), shared=b.count)):
        with pytest.raises((ValueError, MoeError)):
            cache.attend(q, *index, **wrong)
    with pytest.raises(TypeError):
        cache.attend(q, *index, prefix=b.prefix.long(), shared=b.count)
    with pytest.raises(TypeError):
        cache.attend(q, *index, prefix=[1], shared=b.count)
    with pytest.raises(MoeError):
        b.cache(window=5).attend(q, *index, **front)
    for wrong in (dict(k_norm=w[:32]), dict(k_norm=w.cpu()), dict(q_norm=w, q=None), dict(k_norm=torch.ones(128, device="cuda")[::2])):
        with pytest.raises(ValueError):
            cache.append(k, k, *index, **{"q": q, **wrong})
    for wrong in (dict(k_norm=w.half()), dict(k_norm=[1.0]), dict(q_norm=w, k_norm=w.to(b.dtype)), dict(k_norm=w.double())):
        with pytest.raises(TypeError):
            cache.append(k, k, *index, **{"q": q, **wrong})
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(MoeError):
            cache.append(k, k, *index, k_norm=w, norm_eps=eps)
    with pytest.raises(MoeError):  # not on 16 bytes
        cache.append(k, k, *index, k_norm=torch.ones(65, device="cuda")[1:])
    needs = w.clone().requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        cache.append(k, k, *index, k_norm=needs)
    with torch.no_grad():
        cache.append(k, k, *index, k_norm=needs)
    with pytest.raises(ValueError):
        cache.read(4, *index, k=k[:3])
    with pytest.raises(TypeError):
        cache.read(4, *index, v=k.float())
    with pytest.raises(ValueError):
        cache.read(4, b.pages, b.starts[:1], b.lengths)
    none = cache.read(0, b.pages[:0], b.starts[:1] * 0, b.lengths[:0])
    assert none[0].shape == none[1].shape == (0, 2, 64)
