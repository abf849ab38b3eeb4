"""What Q8Layer takes and refuses, without a GPU: its calls are recorded in place of being made."""
import pytest
import torch

import paper_2310_18547_amd as sg
from paper_2310_18547_amd import layer as layer_module
from paper_2310_18547_amd.layer import PROJECTIONS, Q8Layer, projection_shapes

H, FFN, LAYERS, N = 64, 96, 2, 5
KIND = torch.float16


@pytest.fixture
def calls(monkeypatch):
    made = []
    for name in ("sgmv_dense_q8", "sgmv_rms_norm_q8", "sgmv_silu_mul_q8", "sgmv_quantize_q8", "sgmv_add_lora", "sgmv_add_lora_multi"):
        monkeypatch.setattr(layer_module.B, name, lambda *a, name=name, **k: made.append(name) or 0)
    monkeypatch.setattr(layer_module.B, "sgmv_workspace_init", lambda *a, **k: 0)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a, **k: None)
    return made


def _weights():
    return {name: [(torch.ones(o, i, dtype=torch.int8), torch.ones(o)) for _ in range(LAYERS)]
            for name, (i, o) in projection_shapes(H, FFN).items()}


def _norms():
    return [(torch.ones(H, dtype=KIND), torch.ones(H, dtype=KIND)) for _ in range(LAYERS)]


def _layer(weights=None, norms=None, n=N):
    pointers = {name: torch.zeros(1, dtype=torch.int64) for name in PROJECTIONS}
    return Q8Layer(H, FFN, 8, LAYERS, n, sg.F16, pointers, pointers, torch.tensor([0, n], dtype=torch.int32), 1, n,
                   weights or _weights(), norms or _norms(), device="cpu")


def _rows(n=N, width=H, kind=KIND):
    return torch.ones(n, width, dtype=kind)


WRONG_ROWS = {
    "too few": lambda: _rows(N - 1),
    "another type": lambda: _rows(kind=torch.bfloat16),
    "32 bits": lambda: _rows(kind=torch.float32),
    "a slice of wider rows": lambda: _rows(width=3 * H)[:, H:2 * H],
    "transposed": lambda: _rows(H, N).t(),
    "wider": lambda: _rows(width=2 * H),
    "narrower": lambda: _rows(2 * N, H // 2 - 8),
    "every other row": lambda: _rows(2 * N)[::2],
    "another device": lambda: torch.empty(N, H, dtype=KIND, device="meta"),
    "no tensor": lambda: _rows().numpy(),
}


@pytest.mark.parametrize("wrong", WRONG_ROWS)
def test_rows_that_are_not_the_layers(calls, wrong):
    t, good, bad = _layer(), _rows(), WRONG_ROWS[wrong]()
    for call in (lambda: t.qkv(bad, good, 0), lambda: t.qkv(good, bad, 0), lambda: t.qkv(None, bad, 0), lambda: t.finish(bad, good, 0),
                 lambda: t.finish(good, bad, 0), lambda: t.norm(1, bad, good, 0), lambda: t.norm(1, good, bad, 0),
                 lambda: t.project(("o",), t.q, bad, 0), lambda: t.project(("o",), bad, good, 0), lambda: t.dense(("o",), bad, 0)):
        with pytest.raises(ValueError, match="contiguous rows"):
            call()
        assert not calls, "something was enqueued"


def test_own_buffers_of_another_width_are_refused(calls):
    t = _layer()
    for call in (lambda: t.finish(t.act, _rows(), 0), lambda: t.finish(t.y["gate"], _rows(), 0), lambda: t.dense(("down",), t.q, 0),
                 lambda: t.project(("down",), t.q_ffn, t.x, 0)):
        with pytest.raises(ValueError, match="contiguous rows"):
            call()
    assert not calls


def test_rows_in_every_form_that_a_call_can_use(calls):
    """More rows than the batch has, heads as a dimension of their own, an address."""
    t = _layer()
    for rows in (_rows(), _rows(N + 3), _rows().view(N, 4, H // 4), _rows().view(1, N, H), _rows(N + 2)[1:], _rows().data_ptr()):
        t.qkv(rows, _rows(), 1)
        t.qkv(None, rows, 1)
        t.finish(rows, _rows(), 1)
        t.finish(_rows(), rows, 1)
    t.qkv(t.y["down"], _rows(), 0)
    t.finish(t.y["v"], _rows(), 0)
    one = ["sgmv_rms_norm_q8", "sgmv_dense_q8", "sgmv_add_lora_multi"]
    assert calls[:3] == one
    t.add_ons = False
    del calls[:]
    t.project(("o",), t.q, None, 0)               # nothing reads the 16-bit rows
    assert calls == ["sgmv_dense_q8"]


def test_weights_and_norms_that_are_not_the_layers(calls):
    def changed(name, layer_idx, pair):
        w = _weights()
        w[name][layer_idx] = pair
        return w

    good_w, good_s = _weights()["down"][0]
    for pair in ((good_w.float(), good_s), (good_w.t().contiguous(), good_s), (good_w.t().contiguous().t(), good_s), (good_w, good_s.half()),
                 (good_w, good_s[:-8]), (good_w, torch.ones(2 * H)[::2]), (good_w[:-8], good_s), (good_w.to("meta"), good_s)):
        with pytest.raises(ValueError, match="of down"):
            _layer(changed("down", 1, pair))
    few = _weights()
    few["v"].pop()
    with pytest.raises(ValueError, match="v: weights of 1 layers"):
        _layer(few)
    with pytest.raises(ValueError, match="norm weights of 1 layers"):
        _layer(norms=_norms()[:1])
    for bad in (torch.ones(H), torch.ones(H, dtype=torch.bfloat16), torch.ones(H - 8, dtype=KIND), torch.ones(2 * H, dtype=KIND),
                torch.ones(2 * H, dtype=KIND)[::2], torch.ones(H, dtype=KIND, device="meta")):
        with pytest.raises(ValueError, match="norm weight"):
            _layer(norms=[_norms()[0], (_norms()[1][0], bad)])
    _layer(norms=[tuple(w[None] for w in pair) for pair in _norms()])


def test_rows_in_buffers_that_the_call_overwrites_first(calls):
    """Attention in o's output is gone when o's add-on reads it, a residual in any buffer of a later stage when it is returned."""
    t = _layer()
    for call in (lambda: t.finish(t.y["o"], _rows(), 0), lambda: t.finish(t.y["o"].view(N, 4, H // 4), _rows(), 0),
                 lambda: t.project(("o",), t.q, t.y["o"], 0), lambda: t.project(("q", "k", "v"), t.q, t.y["v"], 0),
                 lambda: t.finish(_rows(), t.y["down"], 0), lambda: t.finish(_rows(), t.y["o"], 0), lambda: t.finish(_rows(), t.x, 0),
                 lambda: t.qkv(None, t.x, 0), lambda: t.qkv(_rows(), t.y["q"], 0)):
        with pytest.raises(ValueError, match="this call writes"):
            call()
        assert not calls
    t.qkv(t.y["down"], _rows(), 0)                # read before anything of it is written
    t.qkv(t.x, _rows(), 0)
    t.qkv(None, t.y["down"], 0)
    t.finish(t.x, _rows(), 0)
    t.finish(t.y["q"], t.y["k"], 0)
    t.add_ons = False
    t.finish(t.y["o"], _rows(), 0)                # in 8 bits before o is written, and read by nothing else


def test_a_batch_without_rows(calls):
    t = _layer(n=0)
    t.qkv(_rows(0), _rows(0), 0)
    t.finish(t.y["v"], _rows(0), 0)
