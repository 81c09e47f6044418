"""The operators together, as a decoder serves several answers to one prompt: the prompt is appended once
(queries and keys normalised by head and turned, the cache in 8 bits), every answer's sequence begins with
its pages, tokens are attended to behind it, the MoE layer call follows, tokens are chosen; and a sequence is
taken out of the pages and put into others.  Every call is checked against the oracle on the GPU's own inputs."""
import numpy as np
import pytest

import synth
from gpu_common import check_routes, check_y, log, make_cache, oracle_layer_y, residual_slack, small_call_exact, store_buffer, torch_cuda
from kv_ext_common import LIMITS
from oracle import serving as ref
from serving_common import half_step
from test_gpu_serving import norm

pytestmark = pytest.mark.gpu

HEADS, KV_HEADS, DIM, PAGE, VOCAB, EPS = 8, 2, 64, 16, 1003, 1e-6


def held(cache, layer, pages, length):
    """One sequence's keys and values as the pools hold them: [tokens, kv heads, dim] each."""
    import torch
    t = np.arange(length)
    page, at = torch.as_tensor(pages[t // PAGE]).long().cuda(), torch.from_numpy(t % PAGE).cuda()
    k = cache.keys[layer].view(torch.uint8)[page, :, at // 16, :, at % 16].flatten(2)
    v = cache.values[layer].view(torch.uint8)[page, :, at // 16, at // 8 % 2, :, at % 8]
    number = lambda x: x.contiguous().view(torch.float8_e4m3fn).double()  # noqa: E731
    scale = lambda s: torch.exp2(s[layer].view(torch.uint8)[page, :, at].double() - 127)[..., None]  # noqa: E731
    return [(number(x) * scale(s)).cpu().numpy() for x, s in ((k, cache.key_scales), (v, cache.value_scales))]


def test_several_answers_to_one_prompt():
    torch = torch_cuda()
    from paper_2607_09686_amd import KvCache, plan_bytes, sample
    wl = synth.WORKLOADS["tiny"].with_(n_layers=2, n_experts=16, name="answers")
    keep, ptr, store = store_buffer(wl)
    routers_h = synth.router(wl)
    routers = torch.from_numpy(routers_h).cuda()
    moe = make_cache(wl, ptr, 8, residual=True, prenorm=True)
    kw = dict(n_layers=wl.n_layers, n_heads=HEADS, n_kv_heads=KV_HEADS, head_dim=DIM, page_tokens=PAGE,
              rope_theta=1e4, storage=torch.float8_e4m3fn)
    # the pages that a plan for 256 tokens leaves room for: nearly twice those of 16 bits
    probe = KvCache(n_pages=1, **kw)
    wide = KvCache(n_pages=1, **dict(kw, storage=None))
    assert probe.token_bytes * 2 * DIM == wide.token_bytes * (DIM + 1)
    plan = plan_bytes(dict(n_layers=wl.n_layers, n_experts=wl.n_experts, top_k=wl.top_k, payload_bytes=wl.payload_bytes,
                           kv_bytes_per_token=probe.token_bytes), 8 * 2 * wl.payload_bytes, 256)
    n_pages = plan["kv_bytes"] // (probe.token_bytes * PAGE)
    assert n_pages == 16
    cache = KvCache(n_pages=n_pages, **kw)
    for x in (cache.keys, cache.values, cache.key_scales, cache.value_scales):
        x.view(torch.uint8).fill_(255)
    g = torch.Generator().manual_seed(21)
    w = lambda *s: (torch.randn(*s, generator=g) * s[-2] ** -0.5).cuda()  # noqa: E731
    H, L = wl.hidden, wl.n_layers
    wqkv, wo = w(L, H, (HEADS + 2 * KV_HEADS) * DIM), w(L, HEADS * DIM, H)
    embed, head = w(VOCAB, H) * VOCAB ** 0.5, w(H, VOCAB) * 4
    q_norm, k_norm = ((1 + 0.2 * torch.randn(L, DIM, generator=g)).cuda() for _ in range(2))
    freqs = [1e4 ** (-2 * i / DIM) for i in range(DIM // 2)]
    rng = np.random.default_rng(4)
    u32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    h_bf = half_step(torch.bfloat16)
    fp32 = (2.0 ** -20 + (DIM / 32 + 6) * 2.0 ** -24) * 2  # a norm and a turn, of the largest element's

    def step(tokens, counts, lengths, table, what, shared=0):
        """Logits of the new tokens' rows, every call checked."""
        n, starts = len(tokens), np.cumsum([0] + counts)
        index = torch.from_numpy(table).cuda(), u32(starts.tolist()), u32(lengths)
        front = dict(prefix=index[0][0, :-(-shared // PAGE)].clone(), shared=u32([shared])) if shared else {}
        h, worst = embed[torch.from_numpy(np.asarray(tokens)).cuda()], 0.0
        for layer in range(L):
            x = norm(h) @ wqkv[layer]
            q, k, v = (y.view(n, -1, DIM) for y in x.split([HEADS * DIM, KV_HEADS * DIM, KV_HEADS * DIM], 1))
            turned = cache.append(k, v, *index, layer=layer, q=q, q_norm=q_norm[layer], k_norm=k_norm[layer], norm_eps=EPS)
            o = cache.attend(turned, *index, layer=layer, **front)
            host = {a: b.double().cpu().numpy() for a, b in (("q", q), ("k", k), ("v", v), ("turned", turned), ("o", o))}
            for s, (count, length) in enumerate(zip(counts, lengths)):
                r, pos = slice(starts[s], starts[s + 1]), np.arange(length - count, length)
                keys, values = held(cache, layer, table[s], length)
                for got, x_, weight in ((host["turned"][r], host["q"][r], q_norm), (None, host["k"][r], k_norm)):
                    a = ref.head_norm(x_, weight[layer].double().cpu().numpy(), EPS)
                    want, slack = ref.rotate(a, pos, freqs), fp32 * np.abs(a).max()
                    if got is not None:
                        assert (np.abs(got - want) <= h_bf * np.abs(want) + slack).all()
                    else:  # e4m3: 2^-4 of an element, or 2^-10 of the scale, which is at most 2^-7 of the largest
                        most = np.abs(want).max(-1, keepdims=True)
                        assert (np.abs(keys[-count:] - want) <= 2.0 ** -4 * np.abs(want) + 2.0 ** -17 * most + 1.1 * slack).all()
                c, e = ref.hold(host["v"][r], *LIMITS["torch.bfloat16"])
                np.testing.assert_array_equal(values[-count:], c * 2.0 ** e[..., None].astype(np.float64))
                qs = host["turned"][r]
                want, weight = ref.attend(qs, keys, values, pos, DIM ** -0.5)
                big = np.linalg.norm(qs, axis=2).max() * np.linalg.norm(keys, axis=2).max() * DIM ** -0.5
                tol = h_bf * np.abs(want) + (h_bf + 2 * (DIM + 8) * 2.0 ** -24 * big + 2.0 ** -18) * (1 + h_bf) * weight
                assert (np.abs(host["o"][r] - want) <= tol).all(), (what, layer, s)
            h = h + o.flatten(1).float() @ wo[layer]
            y = torch.empty_like(h)
            _, idx, ws = moe.layer_forward(h, routers[layer], layer, y, n_tokens=n, routes=True)
            x_, y_ = h.cpu().numpy(), y.cpu().numpy()
            io, w_o, z, fl = check_routes(x_, routers_h[layer], wl.top_k, idx, ws, prenorm=True)
            exact = small_call_exact(n, wl.hidden, wl.inter, np.unique(idx).size, 8)
            yo = oracle_layer_y(x_, routers_h[layer], store, wl, layer, io, w_o, z, idx, fl, bf16=not exact, prenorm=True)
            worst = max(worst, check_y(y_.astype(np.float64) - x_, yo, what, slack=residual_slack(y_)))
            h = y
        log(f"{what}: {n} rows, MoE worst error / rms {worst:.2e}")
        return norm(h) @ head

    def choose(logits):
        u = rng.random(len(logits)).astype(np.float32)
        temperature = torch.full((len(logits),), 0.9, device="cuda")
        got, probs = sample(logits, torch.from_numpy(u).cuda(), temperature=temperature)
        host = logits.double().cpu().numpy()
        for r, token in enumerate(got.tolist()):
            want, prob = ref.choose(host[r], float(u[r]), float(np.float32(0.9)))
            assert token == want and abs(probs[r].item() - prob) <= 2.0 ** -22 * prob
        return got.cpu().numpy().astype(np.int64)

    # the prompt, once: 83 tokens, five whole pages and a part
    prompt, pages = 83, [9, 2, 14, 5, 0, 7]
    table = np.full((1, 8), 2 ** 30, np.int32)
    table[0, :6] = pages
    logits = step(rng.integers(0, VOCAB, prompt), [prompt], [prompt], table, "prompt")
    # three answers: the whole pages are shared, the part is copied: taken out and appended again (no
    # turn: what 8 bits gave, they hold)
    own = [[7, 3], [1, 11], [15, 6]]
    answers = np.full((3, 8), 2 ** 30, np.int32)
    for s in range(3):
        answers[s, :5], answers[s, 5:7] = pages[:5], own[s]
    part = prompt - 5 * PAGE
    copy = KvCache(n_pages=n_pages, **dict(kw, rope_dim=0), keys=cache.keys, values=cache.values,
                   key_scales=cache.key_scales, value_scales=cache.value_scales)
    tail = torch.from_numpy(table).cuda(), u32([0, part]), u32([prompt])
    for layer in range(L):
        k, v = cache.read(part, *tail, layer=layer)
        for s in (1, 2):
            copy.append(k, v, torch.from_numpy(answers[s:s + 1]).cuda(), u32([0, part]), u32([prompt]), layer=layer)
        first = held(cache, layer, answers[0], prompt)
        for s in (1, 2):
            for a, b in zip(first, held(cache, layer, answers[s], prompt)):
                np.testing.assert_array_equal(a, b)
    tokens = choose(logits[-1:].expand(3, -1).contiguous())
    lengths = [prompt] * 3
    for i in range(4):
        lengths = [n + 1 for n in lengths]
        # what is shared may end inside a page: the copies hold the same
        logits = step(tokens, [1, 1, 1], lengths, answers, f"token {i}", shared=prompt if i % 2 else 5 * PAGE)
        tokens = choose(logits)
    # windows of drafts, of 1 to 4 tokens
    counts = [4, 1, 3]
    lengths = [n + c for n, c in zip(lengths, counts)]
    step(rng.integers(0, VOCAB, sum(counts)), counts, lengths, answers, "windows", shared=5 * PAGE)
    moe.close()
    keep.free()
