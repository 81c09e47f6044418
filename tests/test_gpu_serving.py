"""The operators as a decoder runs them: per layer the rotated keys and values go to the paged cache
(sized by the budget plan), the new tokens attend over it, and the MoE layer call follows; after the
last layer a token is chosen.  A ragged batch of prompts, then single tokens, then verification
windows with rejected drafts.  Every call is checked against the oracle on the GPU's own inputs."""
import numpy as np
import pytest

import synth
from gpu_common import (check_routes, check_y, log, make_cache, oracle_layer_y, residual_slack, small_call_exact,
                        store_buffer, torch_cuda)
from oracle import serving as ref
from serving_common import half_step

pytestmark = pytest.mark.gpu

HEADS, KV_HEADS, DIM, PAGE, VOCAB = 8, 2, 64, 16, 1003


def norm(h):
    return h * (h.pow(2).mean(-1, keepdim=True) + 1e-6).rsqrt()


class Decoder:
    def __init__(self, torch, wl, moe, routers, cache, pages):
        self.torch, self.wl, self.moe, self.routers, self.cache = torch, wl, moe, routers, cache
        g = torch.Generator().manual_seed(11)
        w = lambda *s: (torch.randn(*s, generator=g) * s[-2] ** -0.5).cuda()  # noqa: E731
        H, L = wl.hidden, wl.n_layers
        self.wqkv, self.wo = w(L, H, (HEADS + 2 * KV_HEADS) * DIM), w(L, HEADS * DIM, H)
        self.embed, self.head = w(VOCAB, H) * VOCAB ** 0.5, w(H, VOCAB) * 4
        self.pages = pages

    def forward(self, tokens, starts, lengths, seen):
        """Logits of the new tokens (rows of all sequences); every call's inputs and results in `seen`."""
        torch, n = self.torch, tokens.shape[0]
        q_size, kv_size = HEADS * DIM, KV_HEADS * DIM
        h = self.embed[tokens]
        for layer in range(self.wl.n_layers):
            x = norm(h) @ self.wqkv[layer]
            q = x[:, :q_size].view(n, HEADS, DIM)  # slices of one product: rows with a stride
            k = x[:, q_size:q_size + kv_size].view(n, KV_HEADS, DIM)
            v = x[:, q_size + kv_size:].view(n, KV_HEADS, DIM)
            turned = self.cache.append(k, v, self.pages, starts, lengths, layer=layer, q=q)
            o = self.cache.attend(turned, self.pages, starts, lengths, layer=layer)
            h = h + o.flatten(1).float() @ self.wo[layer]
            y = torch.empty_like(h)
            _, idx, w = self.moe.layer_forward(h, self.routers[layer], layer, y, n_tokens=n, routes=True)
            seen.append(dict(layer=layer, q=q, k=k, v=v, turned=turned, o=o, h=h, y=y, idx=idx, w=w))
            h = y
        return norm(h) @ self.head


def read_cache(cache, layer, pages, length):
    """One sequence's keys and values as [tokens, heads, dim]."""
    t = np.arange(length)
    page = pages[t // PAGE]
    k, v = cache.keys[layer].double().cpu().numpy(), cache.values[layer].double().cpu().numpy()
    d, h = np.arange(DIM)[None, None, :], np.arange(KV_HEADS)[None, :, None]
    at = (page[:, None, None], h)
    place = (t % PAGE)[:, None, None]
    return k[at + ref.key_place(place, d)], v[at + ref.value_place(place, d)]


def test_a_decoder_serves_prompts_tokens_and_windows():
    torch = torch_cuda()
    from paper_2607_09686_amd import KvCache, plan_bytes, sample
    wl = synth.WORKLOADS["tiny"].with_(n_layers=2, n_experts=16, name="serving")
    keep, ptr, store = store_buffer(wl)
    routers = synth.router(wl)
    moe = make_cache(wl, ptr, 8, residual=True, prenorm=True)
    # the pages that a plan for 192 tokens leaves room for
    probe = KvCache(wl.n_layers, HEADS, KV_HEADS, DIM, PAGE, 1)
    plan = plan_bytes(dict(n_layers=wl.n_layers, n_experts=wl.n_experts, top_k=wl.top_k,
                           payload_bytes=wl.payload_bytes, kv_bytes_per_token=probe.token_bytes), 8 * 2 * wl.payload_bytes,
                      192)
    assert plan["slots_per_layer"] == 8
    n_pages = plan["kv_bytes"] // (probe.token_bytes * PAGE)
    assert n_pages == 12
    cache = KvCache(wl.n_layers, HEADS, KV_HEADS, DIM, PAGE, n_pages, rope_theta=1e4)
    cache.keys.fill_(float("nan"))
    cache.values.fill_(float("nan"))
    table = np.array([[7, 2, 11, 0, 5], [1, 9, 3, 4, 10]], np.int32)
    pages = torch.from_numpy(table).cuda()
    net = Decoder(torch, wl, moe, torch.from_numpy(routers).cuda(), cache, pages)
    rng = np.random.default_rng(2)
    freqs = [1e4 ** (-2 * i / DIM) for i in range(DIM // 2)]
    u32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    settings = dict(temperature=torch.tensor([0.8, 1.2], device="cuda"), top_k=u32([50, 0]),
                    top_p=torch.tensor([0.95, 0.9], device="cuda"), min_p=torch.tensor([0.0, 0.02], device="cuda"))

    def step(tokens, counts, lengths, what):
        """One pass over `counts` new tokens per sequence, checked; logits of its rows."""
        starts = np.cumsum([0] + counts)
        seen = []
        logits = net.forward(torch.from_numpy(tokens).cuda(), u32(starts.tolist()), u32(lengths), seen)
        torch.cuda.synchronize()
        h_bf, worst = half_step(torch.bfloat16), 0.0
        for call in seen:
            host = {k: call[k].double().cpu().numpy() for k in ("q", "k", "v", "turned", "o")}
            for s, (n, length) in enumerate(zip(counts, lengths)):
                r, pos = slice(starts[s], starts[s + 1]), np.arange(length - n, length)
                k, v = read_cache(cache, call["layer"], table[s], length)
                for got, x in ((host["turned"][r], host["q"][r]), (k[-n:], host["k"][r])):
                    want = ref.rotate(x, pos, freqs)
                    assert (np.abs(got - want) <= h_bf * np.abs(want) + 2.0 ** -20 * 2 * np.abs(x).max()).all()
                np.testing.assert_array_equal(v[-n:], torch.from_numpy(host["v"][r]).bfloat16().double().numpy())
                q = host["turned"][r]
                want, weight = ref.attend(q, k, v, pos, DIM ** -0.5)
                big = np.linalg.norm(q, axis=2).max() * np.linalg.norm(k, axis=2).max() * DIM ** -0.5
                tol = h_bf * np.abs(want) + (h_bf + 2 * (DIM + 8) * 2.0 ** -24 * big + 2.0 ** -18) * (1 + h_bf) * weight
                assert (np.abs(host["o"][r] - want) <= tol).all(), (what, call["layer"], s)
            x, y = call["h"].cpu().numpy(), call["y"].cpu().numpy()
            io, wo, z, fl = check_routes(x, routers[call["layer"]], wl.top_k, call["idx"], call["w"], prenorm=True)
            exact = small_call_exact(len(x), wl.hidden, wl.inter, np.unique(call["idx"]).size, 8)
            yo = oracle_layer_y(x, routers[call["layer"]], store, wl, call["layer"], io, wo, z, call["idx"], fl,
                                bf16=not exact, prenorm=True)
            worst = max(worst, check_y(y.astype(np.float64) - x, yo, what, slack=residual_slack(y)))
        log(f"{what}: {len(tokens)} rows, MoE worst error / rms {worst:.2e}")
        return logits

    def choose(logits, u, rows_of):
        """A token for each row, row i with sequence rows_of[i]'s settings, checked."""
        own = {k: v[rows_of].contiguous() for k, v in settings.items()}
        got, probs = sample(logits, torch.from_numpy(u).cuda(), **own)
        got, probs, host = got.cpu().numpy(), probs.cpu().numpy(), logits.double().cpu().numpy()
        for r in range(len(got)):
            token, prob = ref.choose(host[r], float(u[r]), **{k: v[r].item() for k, v in own.items()})
            assert got[r] == token and abs(probs[r] - prob) <= 2.0 ** -22 * prob
        return got

    u = lambda n: rng.random(n).astype(np.float32)  # noqa: E731
    counts = [37, 20]
    lengths = list(counts)
    logits = step(rng.integers(0, VOCAB, sum(counts)), counts, lengths, "prompts")
    last = np.cumsum(counts) - 1
    tokens = choose(logits[last.tolist()], u(2), [0, 1])
    for i in range(4):
        lengths = [n + 1 for n in lengths]
        tokens = choose(step(tokens.astype(np.int64), [1, 1], lengths, f"token {i}"), u(2), [0, 1])
    # windows: the last token and three drafts per sequence; 1 and 3 drafts pass, the others' places
    # are written again by the next pass
    drafts = rng.integers(0, VOCAB, (2, 3))
    window = np.concatenate([np.concatenate([tokens[s:s + 1], drafts[s]]) for s in range(2)]).astype(np.int64)
    lengths = [n + 4 for n in lengths]
    got = choose(step(window, [4, 4], lengths, "windows"), u(8), [0] * 4 + [1] * 4)
    lengths = [lengths[0] - 2 + 1, lengths[1] + 1]
    tokens = np.array([got[1], got[7]], np.int64)
    choose(step(tokens, [1, 1], lengths, "after the windows"), u(2), [0, 1])
    moe.close()
    keep.free()
