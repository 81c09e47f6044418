"""CPU-side checks of the serving operators' C entries: refusals come before HIP is touched."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def mc():
    from paper_2607_09686_amd import build, moecache
    if not os.path.exists(moecache.LIB_PATH):
        build.build()
    moecache.lib()
    return moecache


def batch(mc, **kw):
    p = 1 << 12  # never dereferenced: every call here is refused, or has nothing to do
    base = dict(dtype=mc.MOE_BF16, n_heads=8, n_kv_heads=2, head_dim=128, page_tokens=16, n_pages=4, max_pages=2,
                n_seqs=1, n_tokens=1, pad=0, keys=p, values=p, pages=p, starts=p, lengths=p, status=None,
                hip_stream=None)
    return mc.KvBatch(**dict(base, **kw))


BAD = [dict(dtype=0), dict(dtype=2), dict(head_dim=96), dict(head_dim=0), dict(n_kv_heads=0), dict(n_kv_heads=3),
       dict(n_heads=0), dict(n_heads=-8, n_kv_heads=-2), dict(n_heads=2048), dict(page_tokens=0),
       dict(page_tokens=24), dict(page_tokens=8), dict(page_tokens=2048), dict(n_pages=0), dict(max_pages=0),
       dict(max_pages=1 << 27), dict(n_seqs=-1), dict(n_seqs=65537), dict(n_tokens=-1), dict(n_tokens=(1 << 24) + 1),
       dict(n_tokens=1 << 24, n_heads=16), dict(n_seqs=65536, n_heads=128, n_kv_heads=128), dict(keys=None),
       dict(values=None), dict(keys=4104), dict(pages=None), dict(starts=None), dict(lengths=None)]


@pytest.mark.parametrize("change", BAD, ids=str)
def test_a_bad_batch_is_refused(mc, change):
    L, p = mc.lib(), 1 << 12
    b = batch(mc, **change)
    size = ctypes.c_uint64(7)
    assert L.moe_kv_append(ctypes.byref(b), None, b.dtype, p, 256, p, 256, None, 0, None, 0) == mc.MOE_EINVAL
    assert L.moe_kv_attend(ctypes.byref(b), 0, 0.1, p, 1024, p, 1024, p, 1 << 40) == mc.MOE_EINVAL
    assert b"moe_kv_attend" in L.moe_last_error()
    assert L.moe_kv_attend_workspace(ctypes.byref(b), ctypes.byref(size)) == mc.MOE_EINVAL and size.value == 7


def test_bad_arguments_of_append(mc):
    L, p = mc.lib(), 1 << 12
    b = batch(mc)
    rope = lambda **kw: ctypes.byref(mc.KvRope(**dict(dict(dim=64, adjacent=0, freq=p), **kw)))  # noqa: E731
    ok = [ctypes.byref(b), rope(), mc.MOE_BF16, p, 256, p, 256, p, 1024, p, 1024]
    for i, v in ((0, None), (1, rope(dim=24)), (1, rope(dim=144)), (1, rope(dim=-16)), (1, rope(freq=None)),
                 (2, mc.MOE_F16), (2, 5), (3, None), (3, p + 8), (4, 255), (4, 128), (4, 260), (4, (1 << 32) + 8),
                 (5, None), (6, 0), (8, 512), (9, None), (9, p + 2), (10, 1020), (10, -1024)):
        args = list(ok)
        args[i] = v
        assert L.moe_kv_append(*args) == mc.MOE_EINVAL, (i, v)
        assert L.moe_last_error()


def test_bad_arguments_of_attend(mc):
    L, p = mc.lib(), 1 << 12
    b = batch(mc)
    size = ctypes.c_uint64()
    assert L.moe_kv_attend_workspace(ctypes.byref(b), ctypes.byref(size)) == mc.MOE_OK and size.value > 0
    assert L.moe_kv_attend_workspace(ctypes.byref(b), None) == mc.MOE_EINVAL
    ok = [ctypes.byref(b), 0, 0.1, p, 1024, p, 1024, p, size.value]
    nan, inf = float("nan"), float("inf")
    for i, v in ((0, None), (1, -1), (2, 0.0), (2, -1.0), (2, nan), (2, inf), (3, None), (3, p + 8), (4, 1016),
                 (4, 1028), (5, None), (6, 0), (7, None), (7, p + 8), (8, size.value - 1), (8, 0)):
        args = list(ok)
        args[i] = v
        assert L.moe_kv_attend(*args) == mc.MOE_EINVAL, (i, v)


def test_nothing_to_do_is_no_error(mc):
    L, p = mc.lib(), 1 << 12
    for change in (dict(n_tokens=0), dict(n_seqs=0), dict(n_tokens=0, n_seqs=0, pages=None, starts=None, lengths=None)):
        b = batch(mc, **change)
        assert L.moe_kv_append(ctypes.byref(b), None, b.dtype, None, 0, None, 0, None, 0, None, 0) == mc.MOE_OK
        assert L.moe_kv_attend(ctypes.byref(b), 0, 0.1, None, 0, None, 0, None, 0) == mc.MOE_OK


def test_bad_arguments_of_sample(mc):
    L, p = mc.lib(), 1 << 12
    base = dict(dtype=mc.MOE_F32, n_rows=2, vocab=100000, pad=0, logits=p, row_stride=100000, temperature=None, top_k=None,
                top_p=None, min_p=None, u=p, hip_stream=None)
    for change in (dict(dtype=7), dict(vocab=0), dict(vocab=(1 << 20) + 1), dict(n_rows=-1), dict(n_rows=65536),
                   dict(logits=None), dict(u=None), dict(row_stride=99999), dict(row_stride=-100),
                   dict(row_stride=(1 << 32) + 1), dict(logits=p + 2)):
        s = mc.SampleBatch(**dict(base, **change))
        assert L.moe_sample(ctypes.byref(s), p, p, p, 1 << 40) == mc.MOE_EINVAL, change
    size, s = ctypes.c_uint64(), mc.SampleBatch(**base)
    assert L.moe_sample_workspace(ctypes.byref(s), ctypes.byref(size)) == mc.MOE_OK and size.value > 0
    assert L.moe_sample_workspace(None, ctypes.byref(size)) == mc.MOE_EINVAL
    assert L.moe_sample_workspace(ctypes.byref(s), None) == mc.MOE_EINVAL
    for args in ((None, p, p, p, size), (s, None, p, p, size), (s, p, p, None, size), (s, p, p, p + 8, size),
                 (s, p, p, p, ctypes.c_uint64(size.value - 1))):
        b = None if args[0] is None else ctypes.byref(args[0])
        assert L.moe_sample(b, *args[1:]) == mc.MOE_EINVAL
    assert L.moe_sample(ctypes.byref(mc.SampleBatch(**dict(base, n_rows=0))), None, None, None, 0) == mc.MOE_OK
    short = mc.SampleBatch(**dict(base, vocab=100))
    assert L.moe_sample_workspace(ctypes.byref(short), ctypes.byref(size)) == mc.MOE_OK and size.value == 0
    for change in (dict(vocab=0), dict(vocab=(1 << 20) + 1), dict(n_rows=65536)):
        s = mc.SampleBatch(**dict(base, **change))
        assert L.moe_sample_workspace(ctypes.byref(s), ctypes.byref(size)) == mc.MOE_EINVAL


def test_the_cache_refuses_what_it_cannot_hold(mc):
    import torch
    from paper_2607_09686_amd import KvCache, plan_bytes, sample
    kw = dict(n_layers=2, n_heads=8, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=3, device="cpu")
    for change in (dict(n_layers=0), dict(n_heads=7), dict(n_kv_heads=0), dict(head_dim=80), dict(page_tokens=17),
                   dict(page_tokens=8), dict(n_pages=0), dict(rope_dim=72), dict(rope_dim=65), dict(rope_dim=-16),
                   dict(rope_freqs=[1.0]), dict(keys=torch.zeros(2, 3)),
                   dict(values=torch.zeros(2, 3, 2, 1, 2, 64, 8))):
        with pytest.raises(ValueError):
            KvCache(**dict(kw, **change))
    with pytest.raises(TypeError):
        KvCache(**dict(kw, dtype=torch.float32))
    c = KvCache(**kw)
    assert c.keys.shape == (2, 3, 2, 1, 8, 16, 8) and c.values.shape == (2, 3, 2, 1, 2, 64, 8)
    # every byte of a page belongs to one of its tokens: the plan's K(n)
    assert c.token_bytes * 16 * 3 == 2 * (c.keys.numel() + c.values.numel())
    plan = plan_bytes(dict(n_layers=2, n_experts=8, top_k=2, payload_bytes=1000, kv_bytes_per_token=c.token_bytes),
                      10000, 48)
    assert plan["kv_bytes"] == 2 * (c.keys.numel() + c.values.numel())
    i = lambda *v: torch.zeros(*v, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):  # a cache in host memory serves no call
        c.attend(torch.zeros(1, 8, 64, dtype=torch.bfloat16), i(1, 1), i(2), i(1))
    with pytest.raises(ValueError):
        sample(torch.zeros(1, 4), torch.zeros(1))


def test_the_cache_refuses_to_drop_a_gradient(mc):
    import torch
    from paper_2607_09686_amd import KvCache
    c = KvCache(n_layers=1, n_heads=4, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=3, device="cpu")
    i = lambda *v: torch.zeros(*v, dtype=torch.int32)  # noqa: E731
    index = i(1, 1), i(2), i(1)
    t = lambda heads, grad: torch.zeros(1, heads, 64, dtype=torch.bfloat16, requires_grad=grad)  # noqa: E731
    calls = [lambda g: c.attend(t(4, g), *index), lambda g: c.append(t(2, g), t(2, False), *index),
             lambda g: c.append(t(2, False), t(2, g), *index),
             lambda g: c.append(t(2, False), t(2, False), *index, q=t(4, g)),
             lambda g: c.append(t(2, False), t(2, False), *index, q=t(4, False), q_out=t(4, g)),
             lambda g: c.attend(t(4, False), *index, out=t(4, g))]
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call(True)
        with pytest.raises(ValueError, match="GPU"):  # no gradient to drop: refused for the host memory alone
            call(False)
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
            call(True)
        with torch.inference_mode(), pytest.raises(ValueError, match="GPU"):
            call(True)


def test_a_scale_beyond_what_scores_can_hold_is_refused(mc):
    """The kernels take scores in log2: a scale whose product with log2(e) is no finite fp32 is one as bad
    as an infinite one."""
    L, p = mc.lib(), 1 << 12
    b = batch(mc)
    size = ctypes.c_uint64()
    assert L.moe_kv_attend_workspace(ctypes.byref(b), ctypes.byref(size)) == mc.MOE_OK
    for scale in (2.4e38, 3.4e38):
        assert L.moe_kv_attend(ctypes.byref(b), 0, scale, p, 1024, p, 1024, p, size.value) == mc.MOE_EINVAL, scale
    none = batch(mc, n_tokens=0)  # as before: nothing to do, nothing launched
    assert L.moe_kv_attend(ctypes.byref(none), 0, 2.3e38, None, 0, None, 0, None, 0) == mc.MOE_OK
