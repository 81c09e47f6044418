"""CPU-side checks of the C entries for norms, caches of 8 bits and shared tokens: refusals come before
HIP is touched; the oracle's 8-bit numbers; the new kernels' registers."""
import ctypes
import os

import numpy as np
import pytest

from oracle import serving as ref
from test_kernel_registers import kernels
from test_serving_capi import BAD, batch


@pytest.fixture(scope="module")
def mc():
    from paper_2607_09686_amd import build, moecache
    if not os.path.exists(moecache.LIB_PATH):
        build.build()
    moecache.lib()
    return moecache


P = 1 << 12  # never dereferenced: every call here is refused, or has nothing to do


def scales(mc, **kw):
    return ctypes.byref(mc.KvScales(**dict(dict(keys=P, values=P), **kw)))


def norm(mc, **kw):
    return ctypes.byref(mc.KvNorm(**dict(dict(q_weight=P, k_weight=P, dtype=mc.MOE_F32, eps=1e-6), **kw)))


def prefix(mc, **kw):
    return ctypes.byref(mc.KvPrefix(**dict(dict(pages=P, tokens=P, n_pages=2, pad=0), **kw)))


@pytest.mark.parametrize("change", BAD, ids=str)
def test_a_bad_batch_is_refused(mc, change):
    L = mc.lib()
    b, size = batch(mc, **change), ctypes.c_uint64(7)
    for s in (None, scales(mc)):
        assert L.moe_kv_append_ext(b, s, None, None, b.dtype, P, 256, P, 256, None, 0, None, 0) == mc.MOE_EINVAL
        assert b"moe_kv_append_ext" in L.moe_last_error()
        assert L.moe_kv_attend_ext(b, s, None, 0, 0.1, P, 1024, P, 1024, P, 1 << 40) == mc.MOE_EINVAL
        assert L.moe_kv_read(b, s, P, 256, P, 256) == mc.MOE_EINVAL
        assert b"moe_kv_read" in L.moe_last_error()
        assert L.moe_kv_attend_ext_workspace(b, s, prefix(mc), size) == mc.MOE_EINVAL and size.value == 7


def test_bad_arguments_of_append(mc):
    L, nan, inf = mc.lib(), float("nan"), float("inf")
    b = batch(mc)
    ok = [ctypes.byref(b), scales(mc), None, norm(mc), mc.MOE_BF16, P, 256, P, 256, P, 1024, P, 1024]
    wrong = [(0, None), (1, scales(mc, keys=None)), (1, scales(mc, values=None)), (1, scales(mc, keys=P + 8)),
             (3, norm(mc, dtype=mc.MOE_F16)), (3, norm(mc, dtype=9)), (3, norm(mc, eps=-1.0)), (3, norm(mc, eps=nan)),
             (3, norm(mc, eps=inf)), (3, norm(mc, q_weight=P + 4)), (3, norm(mc, k_weight=P + 8)), (4, mc.MOE_F16),
             (5, None), (6, 255), (8, 64), (9, None), (10, 1020), (11, None), (12, 0)]
    for i, v in wrong:
        args = list(ok)
        args[i] = v
        assert L.moe_kv_append_ext(*args) == mc.MOE_EINVAL, (i, v)
        assert b"moe_kv_append_ext" in L.moe_last_error()


def test_bad_arguments_of_read(mc):
    L, b = mc.lib(), batch(mc)
    ok = [ctypes.byref(b), scales(mc), P, 256, P, 256]
    for i, v in ((0, None), (1, scales(mc, keys=None)), (2, None), (2, P + 8), (3, 128), (3, 260), (3, (1 << 32) + 8), (4, None),
                 (5, -256)):
        args = list(ok)
        args[i] = v
        assert L.moe_kv_read(*args) == mc.MOE_EINVAL, (i, v)


def test_bad_arguments_of_attend(mc):
    L, b = mc.lib(), batch(mc)
    plain, held, shared, size = (ctypes.c_uint64() for _ in range(4))
    assert L.moe_kv_attend_workspace(b, plain) == mc.MOE_OK
    assert L.moe_kv_attend_ext_workspace(b, None, None, size) == mc.MOE_OK and size.value == plain.value
    assert L.moe_kv_attend_ext_workspace(b, scales(mc), None, held) == mc.MOE_OK and held.value == plain.value
    assert L.moe_kv_attend_ext_workspace(b, scales(mc), prefix(mc), shared) == mc.MOE_OK and shared.value > 0
    assert L.moe_kv_attend_ext_workspace(b, None, None, None) == mc.MOE_EINVAL
    for p in (prefix(mc, pages=None), prefix(mc, tokens=None), prefix(mc, n_pages=0), prefix(mc, n_pages=-1),
              prefix(mc, n_pages=(1 << 26) + 1)):
        assert L.moe_kv_attend_ext_workspace(b, None, p, size) == mc.MOE_EINVAL
        assert L.moe_kv_attend_ext(b, None, p, 0, 0.1, P, 1024, P, 1024, P, 1 << 40) == mc.MOE_EINVAL
    ok = [ctypes.byref(b), scales(mc), prefix(mc), 0, 0.1, P, 1024, P, 1024, P, shared.value]
    for i, v in ((0, None), (1, scales(mc, values=P + 1)), (3, 5), (3, -1), (4, 0.0), (4, float("nan")), (5, None), (6, 1016),
                 (7, P + 8), (8, 0), (9, None), (9, P + 8), (10, shared.value - 1)):
        args = list(ok)
        args[i] = v
        assert L.moe_kv_attend_ext(*args) == mc.MOE_EINVAL, (i, v)


def test_workspaces_of_the_largest_batches(mc):
    """The sizes stay in 64 bits, and the launches' counts in 32, wherever a batch is allowed."""
    L, size = mc.lib(), ctypes.c_uint64()
    for kw in (dict(n_tokens=1 << 24, n_heads=8, n_kv_heads=8, n_seqs=65536), dict(n_tokens=1 << 17, n_heads=1024, n_kv_heads=1),
               dict(n_tokens=1 << 17, n_heads=1024, n_kv_heads=64, n_seqs=65536), dict(n_tokens=1, max_pages=1 << 26)):
        for p in (None, prefix(mc), prefix(mc, n_pages=1 << 26)):
            for dim in (64, 256):
                b = batch(mc, **dict(dict(head_dim=dim), **kw))
                assert L.moe_kv_attend_ext_workspace(b, scales(mc), p, size) == mc.MOE_OK
                rows = b.n_tokens * b.n_heads
                assert 0 < size.value <= 4 * (rows + 128 * (b.n_seqs + 1024) * b.n_heads) * (dim + 2) * 4


def test_nothing_to_do_is_no_error(mc):
    L = mc.lib()
    for change in (dict(n_tokens=0), dict(n_seqs=0), dict(n_tokens=0, n_seqs=0, pages=None, starts=None, lengths=None)):
        b = batch(mc, **change)
        for s in (None, scales(mc)):
            assert L.moe_kv_append_ext(b, s, None, norm(mc), b.dtype, None, 0, None, 0, None, 0, None, 0) == mc.MOE_OK
            assert L.moe_kv_attend_ext(b, s, prefix(mc), 0, 0.1, None, 0, None, 0, None, 0) == mc.MOE_OK
            assert L.moe_kv_read(b, s, None, 0, None, 0) == mc.MOE_OK


def test_a_cache_of_8_bits(mc):
    import torch
    from paper_2607_09686_amd import KvCache, plan_bytes
    kw = dict(n_layers=2, n_heads=8, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=3, device="cpu",
              storage=torch.float8_e4m3fn)
    c = KvCache(**kw)
    assert c.keys.shape == (2, 3, 2, 1, 4, 16, 16) and c.values.shape == (2, 3, 2, 1, 2, 64, 8)
    assert c.key_scales.shape == c.value_scales.shape == (2, 3, 2, 16)
    assert c.dtype == torch.bfloat16 and c.storage == c.keys.dtype == torch.float8_e4m3fn
    bytes_ = sum(x.numel() * x.element_size() for x in (c.keys, c.values, c.key_scales, c.value_scales))
    assert bytes_ == 3 * 16 * c.token_bytes
    plan = plan_bytes(dict(n_layers=2, n_experts=8, top_k=2, payload_bytes=100, kv_bytes_per_token=c.token_bytes), 10000, 48)
    assert plan["kv_bytes"] == bytes_
    assert KvCache(**dict(kw, storage=None)).storage == torch.bfloat16
    assert KvCache(**dict(kw, storage=None)).key_scales is None
    assert KvCache(**dict(kw, storage=torch.float16, dtype=torch.float16)).keys.shape == (2, 3, 2, 1, 8, 16, 8)
    for change in (dict(keys=c.keys.view(torch.uint8)), dict(values=c.values[:1]), dict(key_scales=c.key_scales[..., :8]),
                   dict(value_scales=c.value_scales.view(torch.uint8)), dict(storage=None, key_scales=c.key_scales)):
        with pytest.raises(ValueError):
            KvCache(**dict(kw, **change))
    for storage in (torch.float8_e5m2, torch.float16, torch.int8):
        with pytest.raises(TypeError):
            KvCache(**dict(kw, storage=storage))
    x = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):  # not on the GPU
        c.read(1, i[None], torch.zeros(2, dtype=torch.int32), i)
    with pytest.raises(ValueError):
        c.append(x, x, i[None], torch.zeros(2, dtype=torch.int32), i)


def test_numbers_of_8_bits():
    import torch
    c = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(c, ref.E4M3)
    rng = np.random.default_rng(1)
    x = rng.standard_normal((500, 64)) * 2.0 ** rng.integers(-130, 125, (500, 1))
    x[0], x[1, 3], x[2, 5] = 0, np.inf, np.nan
    v, e = ref.hold(x, -100, 119)
    assert e[0] == -100 and np.isnan(v[1, 3]) and np.isnan(v[2, 5])
    finite = np.where(np.isfinite(x), x, 0)
    want = torch.from_numpy(np.clip(finite * 2.0 ** -e[:, None].astype(float), -448, 448)).float().to(torch.float8_e4m3fn)
    np.testing.assert_array_equal(np.where(np.isfinite(x), v, 0), np.where(np.isfinite(x), want.double().numpy(), 0))
    most = np.abs(finite).max(1)
    inside = (e > -100) & (e < 119)
    assert inside.sum() > 300 and (most[inside] <= 448 * 2.0 ** e[inside]).all() and (most[inside] > 224 * 2.0 ** e[inside]).all()


def test_the_kernels_use_no_scratch(mc):
    found = {n: k for n, k in kernels(mc.LIB_PATH).items()
             if any(s in n for s in ("held_", "behind_", "append_ext_kernel", "read_kernel"))}
    # 8 bits: three tiles; behind shared tokens: six pairs of tiles, two storages; planned and joined: three tiles;
    # appended: two sources and storages, read: two storages; two types, three head sizes (plans: of all sizes and types)
    assert len(found) == 3 * 2 * (3 + 12 + 3) + 3 + 2 * 4 + 2 * 2
    for name, k in found.items():
        assert (k[".vgpr_spill_count"], k[".private_segment_fixed_size"]) == (0, 0), name
