"""What the operators of a speculative step refuse before anything reaches a GPU."""
import ctypes as C

import pytest
import torch

from paper_2604_07609_b200 import binding as B
from synth import model_cfg

P = 0x10000        # an aligned address that nothing may touch


def _pool(m, blocks=8, base=P, block_size=16):
    return B.blink_kv_pool(C.sizeof(B.blink_kv_pool), block_size, base, blocks * B.kv_bytes_per_block(m))


def _tables(**kw):
    a = dict(ctx=P, new=P, held=P, n=4, free=P, cap=10, count=P, table=P, stride=8, rows=16, held_out=P, count_out=P, row_start=P, kv=P, pos=P,
             slot=P, status=P, stream=None)
    a.update(kw)
    return B.lib().blink_build_tables(*a.values())


@pytest.mark.parametrize("kw,rc", [(dict(n=0), B.BLINK_EINVAL), (dict(n=4097), B.BLINK_ETOOBIG), (dict(rows=0), B.BLINK_EINVAL),
                                   (dict(rows=1 << 30), B.BLINK_ETOOBIG), (dict(stride=0), B.BLINK_EINVAL), (dict(cap=-1), B.BLINK_EINVAL),
                                   (dict(pos=P + 2), B.BLINK_EINVAL)] + [(dict([(k, None)]), B.BLINK_EINVAL) for k in (
                                       "ctx", "new", "held", "free", "count", "table", "held_out", "count_out", "row_start", "kv", "pos", "slot", "status")])
def test_build_tables(kw, rc):
    assert _tables(**kw) == rc


def _norm_rope(m=model_cfg(2), cfg=None, kv=None, **kw):
    dim, q = m.qkv_dim, m.q_dim
    cfg, kv = cfg or B.make_model_cfg(m), kv or _pool(m)
    a = dict(layer=0, qkv=P, dt=B.DTYPE_BF16, stride=dim, qg=P, kg=P, pos=P, slot=P, rows=3, out=P, out_stride=q, stream=None)
    a.update(kw)
    return B.lib().blink_qk_norm_rope(C.byref(cfg), C.byref(kv), *a.values())


@pytest.mark.parametrize("kw", [dict(layer=-1), dict(layer=16), dict(qkv=None), dict(qkv=P + 8), dict(out=P + 2), dict(dt=2), dict(stride=3064),
                                dict(stride=3073), dict(out_stride=2040), dict(rows=-1), dict(pos=None), dict(slot=P + 1), dict(qg=P + 2),
                                dict(kv=_pool(model_cfg(2), base=P + 16)), dict(kv=_pool(model_cfg(2), base=None)),
                                dict(kv=_pool(model_cfg(2), block_size=32)), dict(m=model_cfg(1, dtype="fp32")),
                                dict(cfg=B.make_model_cfg(model_cfg(2, head_dim=96))), dict(cfg=B.make_model_cfg(model_cfg(2, n_kv_heads=5))),
                                dict(cfg=B.make_model_cfg(model_cfg(2, rope_theta=0.0)))])
def test_qk_norm_rope(kw):
    assert _norm_rope(**kw) == B.BLINK_EINVAL


def test_a_pool_without_a_block_and_one_beyond_31_bits():
    m = model_cfg(2)
    assert _norm_rope(kv=_pool(m, blocks=0)) == B.BLINK_ENOMEM
    assert _norm_rope(kv=_pool(m, blocks=1 << 25)) == B.BLINK_ETOOBIG
    assert _norm_rope(rows=0) == B.BLINK_OK         # nothing to do


def _attention(m=model_cfg(3), cfg=None, **kw):
    cfg, kv = cfg or B.make_model_cfg(m), _pool(m)
    ws = B.lib().blink_window_attention_workspace(C.byref(cfg), 1)
    a = dict(layer=0, q=P, q_stride=4096, rows=4, row_start=P, kv_len=P, n=4, table=P, stride=9, window=0, sinks=0, max_new=1, out=P, out_stride=4096,
             ws=P, ws_bytes=ws, stream=None)
    a.update(kw)
    return B.lib().blink_window_attention(C.byref(cfg), C.byref(kv), *a.values())


@pytest.mark.parametrize("kw", [dict(layer=32), dict(q=None), dict(q=P + 4), dict(out=P + 8), dict(row_start=None), dict(kv_len=P + 1), dict(table=None),
                                dict(rows=0), dict(n=0), dict(stride=0), dict(window=-1), dict(sinks=-1), dict(max_new=0), dict(q_stride=4088),
                                dict(q_stride=4097), dict(out_stride=4090), dict(ws=None), dict(ws=P + 16), dict(ws_bytes=100), dict(max_new=100, ws_bytes=1 << 22)])
def test_window_attention(kw):
    assert _attention(**kw) == B.BLINK_EINVAL


def test_window_attention_sizes_beyond_its_limits():
    for kw in (dict(n=4097), dict(rows=1 << 26), dict(stride=1 << 27), dict(window=1 << 30), dict(sinks=1 << 30)):
        assert _attention(**kw) == B.BLINK_ETOOBIG
    m = model_cfg(3)
    assert B.blink_window_attention_workspace(m, 1) > 0 and B.blink_window_attention_workspace(m, 0) == 0
    assert B.blink_window_attention_workspace(model_cfg(3, head_dim=80), 1) == 0


def _verify(**kw):
    a = dict(logits=P, stride=1000, rows=8, vocab=1000, row_start=P, n=3, draft=P, probs=P, probs_stride=1000, temperature=P, ua=P, up=P, tokens=P,
             accepted=P, ws=P, ws_bytes=B.blink_verify_workspace(8, 3, 1000), stream=None)
    a.update(kw)
    return B.lib().blink_verify_drafts(*a.values())


@pytest.mark.parametrize("kw", [dict(rows=0), dict(vocab=1), dict(n=0), dict(stride=999), dict(probs_stride=999), dict(probs=P + 1), dict(ws=None),
                                dict(ws=P + 8), dict(ws_bytes=10)] + [dict([(k, None)]) for k in ("logits", "row_start", "draft", "temperature", "ua",
                                                                                                "up", "tokens", "accepted")])
def test_verify_drafts(kw):
    assert _verify(**kw) == B.BLINK_EINVAL


def test_the_binding_refuses_host_tensors_and_wrong_shapes():
    i, f = torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    with pytest.raises(ValueError, match="CUDA"):
        B.blink_build_tables(i, i, i, i, i[:1], torch.zeros(2, 3, dtype=torch.int32), max_rows=4)
    with pytest.raises(ValueError, match="CUDA"):
        B.blink_verify_drafts(torch.zeros(3, 9), torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), None, f, torch.zeros(3), f)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rep", [1, 2, 4, 8])
def test_a_workspace_for_long_requests_serves_shorter_ones(rep, hd, dtype):
    """The size never falls as max_new grows."""
    m = model_cfg(1, n_q_heads=rep * 2, n_kv_heads=2, head_dim=hd, dtype=dtype)
    sizes = [B.blink_window_attention_workspace(m, k) for k in list(range(1, 80)) + [100, 1000, 4096, 1 << 24, (1 << 31) - 1]]
    assert sizes[0] > 0 and sizes == sorted(sizes)


@pytest.mark.parametrize("kw,what", [(dict(dtype="fp16"), "dtype"), (dict(dtype="float32"), "dtype"), (dict(dtype=torch.float32), "dtype"),
                                     (dict(n_layers=(1 << 32) + 2), "n_layers"), (dict(vocab=-(1 << 40)), "vocab"), (dict(head_dim=1 << 31), "head_dim")])
def test_the_binding_refuses_models_that_it_would_have_to_guess(kw, what):
    m = model_cfg(1, dtype="fp32")
    q, i = torch.zeros(2, m.q_dim), torch.zeros(2, dtype=torch.int32)
    bad = m.with_(**kw)
    with pytest.raises(ValueError, match=what):
        B._marshal().qk_norm_rope(bad, q, 0, q, None, None, i, i, q)
    with pytest.raises(ValueError, match=what):
        B._marshal().window_attention(bad, q, 0, q, i, i[:1], torch.zeros(1, 2, dtype=torch.int32), 0, 0, 1, q, None)
    with pytest.raises(ValueError, match="CUDA"):      # the model itself is taken
        B._marshal().qk_norm_rope(m, q, 0, q, None, None, i, i, q)
