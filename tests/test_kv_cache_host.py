"""What KvCacheQ4 and Q8Layer.run take and refuse, without a GPU: their calls are recorded in place of being made."""
import pytest
import torch

import paper_2310_18547_amd as sg
from paper_2310_18547_amd import layer as layer_module
from paper_2310_18547_amd.layer import KvCacheQ4
from test_layer_host import FFN, H, KIND, LAYERS, N, _layer, _rows, calls  # noqa: F401


@pytest.fixture
def kv_calls(monkeypatch, calls):  # noqa: F811
    for name in ("sgmv_kv_assign", "sgmv_kv_append_q4", "sgmv_attention_q4"):
        monkeypatch.setattr(layer_module.B, name, lambda *a, name=name, **k: calls.append(name) or 0)
    return calls


def _cache(**k):
    a = dict(dtype=sg.F16, head_dim=64, n_heads=1, n_kv_heads=1, num_layers=LAYERS, page_size=16, n_pages=6, n_reqs=3, n_tokens=N, max_len=50,
             device="cpu")
    a.update(k)
    return KvCacheQ4(**a)


def test_cache_and_its_first_state():
    t = _cache()
    assert t.width == 4 and t.tables.shape == (3, 4) and int(t.free_count) == 6 and t.free_pages.tolist() == list(range(6))
    assert t.pages.shape == (6, LAYERS * (16 * 64 + 128)) and t.scale == 64 ** -0.5
    assert t.rope_table.shape == (64, 64) and t.rope.rows == 64 and t.rope_table[0].tolist() == [1.0] * 32 + [0.0] * 32
    assert abs(float(t.rope_table[49, 32]) - torch.tensor(49.0, dtype=torch.float64).sin().item()) < 1e-7
    t.hint(1, 77)
    assert (t.batch.max_q_len, t.batch.max_kv_len) == (1, 77)
    assert _cache(rope_dim=0).rope is None and _cache(rope_dim=32).rope_table.shape == (64, 32)


@pytest.mark.parametrize("wrong", [dict(head_dim=96), dict(page_size=20), dict(n_pages=0), dict(n_heads=3, n_kv_heads=2), dict(n_reqs=0),
                                   dict(n_tokens=0), dict(max_len=0), dict(n_heads=0), dict(rope_dim=24), dict(rope_dim=80), dict(rope_dim=-16), dict(window=-1)])
def test_caches_that_are_refused(wrong):
    with pytest.raises(ValueError):
        _cache(**wrong)


def test_the_calls_of_a_step(kv_calls):
    t = _cache()
    t.step(torch.zeros(3, dtype=torch.int32))
    q = t.append(0, _rows(), _rows(), _rows())
    assert q is t.q and t.attend(0, q) is t.out
    plain = _cache(rope_dim=0)
    mine = _rows()
    assert plain.append(1, mine, _rows(), _rows()) is mine
    assert kv_calls == ["sgmv_kv_assign", "sgmv_kv_append_q4", "sgmv_attention_q4", "sgmv_kv_append_q4"]


def test_rows_and_lengths_that_are_not_the_caches(kv_calls):
    t, good = _cache(), _rows()
    bad = [_rows(N - 1), _rows(kind=torch.bfloat16), _rows(width=2 * H)[:, :H], _rows(width=H // 2), torch.empty(N, H, dtype=KIND, device="meta"), None]
    for b in bad:
        for call in (lambda: t.append(0, b, good, good), lambda: t.append(0, good, b, good), lambda: t.append(0, good, good, b), lambda: t.attend(0, b)):
            with pytest.raises(ValueError):
                call()
    for b in (torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int64), torch.zeros(6, dtype=torch.int32)[::2], [0, 0, 0]):
        with pytest.raises(ValueError):
            t.step(b)
    assert kv_calls == []


def test_a_whole_layer(kv_calls):
    layer, residual = _layer(), _rows()
    layer.run(_rows(), residual, 0, _cache())
    assert kv_calls[:2] == ["sgmv_rms_norm_q8", "sgmv_dense_q8"] and kv_calls.index("sgmv_kv_append_q4") < kv_calls.index("sgmv_attention_q4")
    assert kv_calls.index("sgmv_attention_q4") < kv_calls.index("sgmv_quantize_q8") and "sgmv_kv_assign" not in kv_calls
    before = len(kv_calls)
    for wrong in (dict(n_tokens=N + 1), dict(dtype=sg.BF16), dict(head_dim=128), dict(n_heads=2)):
        with pytest.raises(ValueError):
            layer.run(_rows(), residual, 0, _cache(**wrong))
    cache = _cache()
    for residual, layer_idx in ((cache.out, 0), (cache.q, 0), (_rows(), LAYERS), (_rows(), -1)):
        with pytest.raises(ValueError):
            layer.run(_rows(), residual, layer_idx, cache)
    assert len(kv_calls) == before and FFN > H


@pytest.mark.parametrize("n_reqs,n_tokens,max_len,hints", [(1, 1, 131072, (0, 0)), (1, 1, 131072, (1, 500)), (1, 512, 131072, (1, 131072)),
                                                           (1, 2048, 131072, (2048, 131072)), (64, 64, 4000, (1, 300)), (3, 700, 9000, (700, 9000))])
@pytest.mark.parametrize("window", [0, 5000])
def test_single_tokens_have_room_for_their_slices(n_reqs, n_tokens, max_len, hints, window):
    """Whatever the hints were when the cache was made: a decode step's plan is that of a workspace without end."""
    t = _cache(head_dim=128, n_heads=32, n_kv_heads=8, num_layers=1, n_reqs=n_reqs, n_tokens=n_tokens, max_len=max_len, max_q_len=hints[0],
               max_kv_len=hints[1], window=window, rope_dim=0)
    for longest in (0, max_len, max_len // 2, 400):
        t.hint(1, longest)
        own, free = (sg.sgmv_plan_attention_q4(t.cache, t.batch, 32, window, 1 << 8, n) for n in (t.scratch_bytes, 1 << 40))
        assert (own.kernel, own.slices, own.workgroups) == (free.kernel, free.slices, free.workgroups), longest
        assert t.scratch.numel() >= t.scratch_bytes
    t.hint(1, max_len)
    if window == 0 and n_reqs == 1:
        assert sg.sgmv_plan_attention_q4(t.cache, t.batch, 32, 0, 1 << 8, t.scratch_bytes).slices >= 8
