"""A whole decoder layer on the GPU: Q8Layer with KvCacheQ4, steps of prompts and single tokens, eagerly and replayed."""
import numpy as np
import pytest
import torch

import attention_reference as ref
from helpers import decode64
from test_gpu_attention import host16
from test_gpu_backbone_layer import KIND, _Layer

pytestmark = pytest.mark.gpu


def _cache(t, n_reqs, dtype, **k):
    import paper_2310_18547_amd as sg
    from paper_2310_18547_amd.layer import KvCacheQ4
    a = dict(head_dim=64, n_heads=4, n_kv_heads=4, num_layers=2, page_size=16, n_pages=24, n_reqs=n_reqs, n_tokens=t.n, max_len=80)
    a.update(k)
    return KvCacheQ4(sg.F16 if dtype == "f16" else sg.BF16, **a)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("window", [0, 11])
def test_layer_with_attention(dtype, window):
    t = _Layer([5, 1, 3], dtype, h=256, ffn=520)
    L = t.layer
    cache = _cache(t, 3, dtype, window=window, rope_dim=32, adjacent=True)
    lens = np.zeros(3, int)
    held = [[[], []] for _ in range(2 * 3)]  # of a layer and a request: rotated k, v
    table = cache.rope_table.cpu().numpy()
    for new in ([5, 1, 3], [1, 7, 1], [3, -1, 2], [4, 5, 0]):
        new_lens = torch.tensor(new, dtype=torch.int32, device="cuda")
        cache.step(new_lens)
        for r, n in enumerate(new):
            if n < 0:
                for layer_idx in (0, 1):
                    held[layer_idx * 3 + r] = [[], []]
                lens[r] = 0
        rows = np.maximum(new, 0)
        starts = np.concatenate(([0], np.cumsum(rows)))
        at = np.concatenate([lens[r] + np.arange(rows[r]) for r in range(3)]).astype(int)
        lens += rows
        assert cache.lens.tolist() == lens.tolist() and cache.q_starts.tolist() == starts.tolist()
        residual, x = t.rows(), t.rows()
        for layer_idx in (0, 1):
            before = residual.clone()
            q, k, v = (host16(y).reshape(t.n, 4, 64) for y in L.qkv(x, residual, layer_idx))
            attention = cache.run(layer_idx, L.y["q"], L.y["k"], L.y["v"]).clone()
            n = int(starts[-1])
            tq, tk = (ref.rotate(z[:n], dtype, table, at, 32, True) for z in (q, k))
            for r in range(3):
                mine = held[layer_idx * 3 + r]
                mine[0] += list(tk[starts[r]:starts[r + 1]])
                mine[1] += list(v[starts[r]:starts[r + 1]])

            def of(r, positions):
                both = []
                for z in held[layer_idx * 3 + r]:
                    codes, s, m = ref.quantize(np.array(z), dtype)
                    both.append(codes * decode64(s, dtype)[..., None] + decode64(m, dtype)[..., None])
                return both
            want, _, off, spread = ref.attention(decode64(tq, dtype), of, starts, lens, 4, 4, 0.125, True, window)
            got = decode64(host16(attention), dtype).reshape(t.n, 4, 64)[:n]
            assert (np.abs(got - want) <= ref.tolerance(want, off, spread, dtype)).all()
            down = L.finish(attention, residual, layer_idx).clone()
            after = residual.clone()
            # the same in one call: the rows go to the same slots again
            residual.copy_(before)
            assert torch.equal(L.run(x, residual, layer_idx, cache), down) and torch.equal(residual, after)
            x = down
    assert cache.check() == 0 and L.check() == 0


def test_decode_steps_captured_and_replayed():
    """A captured step of two layers with its page assignment goes on from token to token as eager steps do."""
    t = _Layer([1] * 4, "f16", h=256, ffn=520, seed=3)
    L = t.layer
    new = torch.ones(4, dtype=torch.int32, device="cuda")
    x, residual = t.rows(), t.rows()
    static_x, static_residual = x.clone(), residual.clone()

    def step(cache, x, residual, stream):
        cache.step(new, stream)
        for layer_idx in (0, 1):
            x = L.run(x, residual, layer_idx, cache, stream=stream)
        return x

    eager, replayed = (_cache(t, 4, "f16", max_q_len=1) for _ in range(2))
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(replayed, static_x, static_residual, torch.cuda.current_stream())
    torch.cuda.synchronize()
    for i in range(20):
        x, residual = t.rows(), t.rows()
        static_x.copy_(x), static_residual.copy_(residual)
        want = step(eager, x, residual, None).clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(L.y["down"], want) and torch.equal(static_residual, residual), i
        assert replayed.lens.tolist() == [i + 1] * 4 and torch.equal(replayed.tables, eager.tables)
    assert replayed.check() == 0


def test_a_step_that_the_pages_do_not_suffice_for():
    """Refused as a whole: nothing is appended, the rows of the attention stay, and the status says why."""
    import paper_2310_18547_amd as sg
    t = _Layer([1] * 3, "f16", h=256, ffn=520)
    cache = _cache(t, 3, "f16", n_pages=2, n_tokens=3)
    kv = [torch.ones(3, 256, dtype=KIND["f16"], device="cuda") for _ in range(3)]
    cache.pages.zero_()
    cache.out.fill_(5.0)
    cache.step(torch.ones(3, dtype=torch.int32, device="cuda"))
    cache.run(0, *kv)
    assert cache.check() == sg.KV_NO_PAGES and int(cache.pages.max()) == 0 and bool((cache.out == 5.0).all()) and cache.lens.tolist() == [0, 0, 0]
    cache.step(torch.tensor([1, 1, 0], dtype=torch.int32, device="cuda"))
    cache.run(0, *kv)
    assert int(cache.status[0]) == 0 and cache.check() == sg.KV_NO_PAGES and bool((cache.out[:2] != 5.0).all()) and bool((cache.out[2] == 5.0).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("window", [0, 1500])
def test_prompts_and_single_tokens_over_long_contexts_of_shared_heads(dtype, window):
    """A cache of more rows than requests, eight heads over two: prompts in parts, then decode steps whose contexts are divided into slices."""
    import paper_2310_18547_amd as sg
    from paper_2310_18547_amd.layer import KvCacheQ4
    rng = np.random.default_rng(17)
    d, heads, kv_heads, rows, most = 128, 8, 2, 900, 2600
    cache = KvCacheQ4(sg.F16 if dtype == "f16" else sg.BF16, d, heads, kv_heads, 1, 64, 64, 2, rows, most, window=window, max_q_len=rows)
    table, held, lens = cache.rope_table.cpu().numpy(), [[[], []], [[], []]], np.zeros(2, int)
    steps = [[900, 0], [800, 100], [750, 150], [1, 1], [1, 0], [1, 1]]
    for new in steps:
        cache.hint(max(new), int((lens + new).max()))
        plan = sg.sgmv_plan_attention_q4(cache.cache, cache.batch, heads, window, cache.scratch, cache.scratch_bytes)
        if max(new) == 1:
            assert plan.kernel == sg.KERNEL_ATTENTION_FEW and plan.slices > 1
        cache.step(torch.tensor(new, dtype=torch.int32, device="cuda"))
        q, k, v = (torch.from_numpy(rng.standard_normal((rows, h * d)).astype(np.float32)).cuda().to(KIND[dtype]) for h in (heads, kv_heads, kv_heads))
        cache.out.fill_(-3.0)
        out = cache.run(0, q, k, v)
        n, starts = sum(new), np.concatenate(([0], np.cumsum(new)))
        at = np.concatenate([lens[r] + np.arange(new[r]) for r in range(2)]).astype(int)
        lens += new
        hq, hk, hv = (host16(x).reshape(rows, -1, d)[:n] for x in (q, k, v))
        tq, tk = (ref.rotate(x, dtype, table, at, d, 0) for x in (hq, hk))
        for r in range(2):
            held[r][0].append(tk[starts[r]:starts[r + 1]])
            held[r][1].append(hv[starts[r]:starts[r + 1]])
        assert cache.lens.tolist() == lens.tolist() and bool((out[n:] == -3.0).all())
        if max(new) > 1:
            continue

        def of(r, positions):
            both = []
            for x in held[r]:
                codes, s, m = ref.quantize(np.concatenate(x), dtype)
                both.append(codes * decode64(s, dtype)[..., None] + decode64(m, dtype)[..., None])
            return both
        want, _, off, spread = ref.attention(decode64(tq, dtype), of, starts, lens, heads, kv_heads, d ** -0.5, True, window)
        got = decode64(host16(out), dtype).reshape(rows, heads, d)[:n]
        assert (np.abs(got - want) <= ref.tolerance(want, off, spread, dtype)).all(), new
    assert cache.check() == 0
