"""Host-only checks of the paged cache's C ABI and of what its binding refuses."""
import ctypes
import os
import re

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2601_16238_amd as attn
from paper_2601_16238_amd import binding, paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000  # a non-NULL, aligned address; never dereferenced on the host


def test_every_declared_symbol_is_exported_and_bound():
    src = open(os.path.join(ROOT, "include", "attn_paged.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = sorted(set(re.findall(r"\b(attn_\w+)\s*\(", src)))
    assert sorted(paged.EXPORTS) == names
    for n in names:
        assert getattr(attn.lib(), n) is not None


def params(**kw):
    p = attn.make_paged_params(6, 3, 8, 2, 64, 20, 16, 5, 0.125, True)
    p.rot, p.table_rows = 64, 80
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def fwd(p, entry="attn_fwd_paged", scales=None, ws=None, ws_bytes=0, **at):
    paged._lib()
    a = dict(Q=FAKE, K=FAKE, V=FAKE, ks=scales, vs=scales, table=FAKE, q_start=FAKE, kv_lens=FAKE, O=FAKE, LSE=FAKE)
    a.update(at)
    return getattr(attn.lib(), entry)(*a.values(), ws, ws_bytes, None if p is None else ctypes.byref(p), None)


def append(p, entry="attn_paged_append", scales=None, **at):
    paged._lib()
    a = dict(K=FAKE, V=FAKE, Q=FAKE, Q_rot=FAKE, cos=FAKE, sin=FAKE, kc=FAKE, vc=FAKE, ks=scales, vs=scales,
             table=FAKE, q_start=FAKE, kv_lens=FAKE)
    a.update(at)
    return getattr(attn.lib(), entry)(*a.values(), None if p is None else ctypes.byref(p), None)


BAD = [
    (dict(T=-1), binding.ATTN_ERR_SHAPE), (dict(B=-1), binding.ATTN_ERR_SHAPE), (dict(Hq=0), binding.ATTN_ERR_SHAPE),
    (dict(Hkv=0), binding.ATTN_ERR_SHAPE), (dict(Hq=7), binding.ATTN_ERR_SHAPE), (dict(D=0), binding.ATTN_ERR_SHAPE),
    (dict(D=60), binding.ATTN_ERR_SHAPE), (dict(D=264), binding.ATTN_ERR_SHAPE), (dict(pages=0), binding.ATTN_ERR_SHAPE),
    (dict(page_size=8), binding.ATTN_ERR_SHAPE), (dict(page_size=48), binding.ATTN_ERR_SHAPE),
    (dict(page_size=8192), binding.ATTN_ERR_SHAPE), (dict(table_width=0), binding.ATTN_ERR_SHAPE),
    (dict(table_width=1 << 28, table_stride=1 << 28), binding.ATTN_ERR_SHAPE),
    (dict(table_width=(1 << 26) + 1, table_stride=1 << 27), binding.ATTN_ERR_SHAPE),
    (dict(table_stride=4), binding.ATTN_ERR_STRIDE),
    (dict(T=1 << 30), binding.ATTN_ERR_SHAPE), (dict(Hq=65536 * 2), binding.ATTN_ERR_SHAPE),
    (dict(q_stride_t=516), binding.ATTN_ERR_STRIDE), (dict(q_stride_h=4), binding.ATTN_ERR_STRIDE),
    (dict(q_stride_h=-64), binding.ATTN_ERR_STRIDE), (dict(out_stride_h=32), binding.ATTN_ERR_STRIDE),
    (dict(out_stride_t=56), binding.ATTN_ERR_STRIDE), (dict(out_stride_t=516), binding.ATTN_ERR_STRIDE),
    (dict(cache_stride_s=56), binding.ATTN_ERR_STRIDE), (dict(cache_stride_s=68), binding.ATTN_ERR_STRIDE),
    (dict(cache_stride_h=0), binding.ATTN_ERR_STRIDE), (dict(cache_stride_p=2052), binding.ATTN_ERR_STRIDE),
    (dict(cache_stride_s=1 << 27), binding.ATTN_ERR_STRIDE),
]


@pytest.mark.parametrize("kw,code", BAD)
@pytest.mark.parametrize("f16", [False, True])
def test_bad_parameters(kw, code, f16):
    assert fwd(params(**kw), "attn_fwd_paged" + "_f16" * f16) == code
    assert append(params(**kw), "attn_paged_append" + "_f16" * f16) == code


def test_bad_parameters_of_one_call():
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert fwd(params(scale=s)) == binding.ATTN_ERR_SCALE
    assert fwd(params(max_q=0)) == binding.ATTN_ERR_SHAPE
    long = dict(T=1 << 20, max_q=1 << 20, table_width=1 << 20, table_stride=1 << 20)   # rows times keys
    assert fwd(params(**long)) == binding.ATTN_ERR_SHAPE
    assert attn.lib().attn_fwd_paged_workspace_bytes(ctypes.byref(params(**long))) > 0
    assert fwd(params(D=72), scales=FAKE) == binding.ATTN_ERR_SHAPE            # e4m3: a multiple of 16
    assert fwd(params(cache_stride_s=72), scales=FAKE) == binding.ATTN_ERR_STRIDE
    for kw in (dict(rot=-8), dict(rot=4), dict(rot=72), dict(table_rows=79)):
        assert append(params(**kw)) == binding.ATTN_ERR_SHAPE
    assert append(params(kv_stride_t=132)) == binding.ATTN_ERR_STRIDE
    assert append(params(kv_stride_h=-64)) == binding.ATTN_ERR_STRIDE


def test_heads_times_keys():
    """What the spans of all heads count with is an int32: the longest table with 64 K/V heads is not."""
    p = params(T=1, B=1, Hq=64, Hkv=64, max_q=1, page_size=4096, table_width=1 << 18, table_stride=1 << 18,
               q_stride_t=64 * 64, out_stride_t=64 * 64, cache_stride_h=4096 * 64, cache_stride_p=64 * 4096 * 64)
    for q in (1, 64):
        p.T = p.max_q = q
        assert fwd(p) == fwd(p, "attn_fwd_paged_f16") == binding.ATTN_ERR_SHAPE


def test_pointers():
    for n in ("Q", "K", "V", "table", "q_start", "kv_lens", "O", "LSE"):
        assert fwd(params(), **{n: None}) == binding.ATTN_ERR_NULL
        assert fwd(params(), **{n: FAKE + 2}) == binding.ATTN_ERR_ALIGN
    for n in ("K", "V", "Q", "Q_rot", "cos", "sin", "kc", "vc", "table", "q_start", "kv_lens"):
        assert append(params(), **{n: None}) == binding.ATTN_ERR_NULL
        assert append(params(), **{n: FAKE + 2}) == binding.ATTN_ERR_ALIGN
    for call in (fwd, append):
        assert call(None) == binding.ATTN_ERR_NULL
        assert call(params(), ks=FAKE) == binding.ATTN_ERR_NULL
        assert call(params(), vs=FAKE) == binding.ATTN_ERR_NULL


def test_workspaces():
    p = params(T=4, B=4, max_q=1, table_width=4096, table_stride=4096)
    need = attn.lib().attn_fwd_paged_workspace_bytes(ctypes.byref(p))
    assert need > 0 and need % 256 == 0
    assert fwd(p, ws=FAKE, ws_bytes=need - 1) == binding.ATTN_ERR_WORKSPACE
    assert fwd(p, ws=FAKE + 16, ws_bytes=need) == binding.ATTN_ERR_WORKSPACE
    assert attn.lib().attn_fwd_paged_workspace_bytes(None) == 0
    assert attn.lib().attn_fwd_paged_workspace_bytes(ctypes.byref(params(D=60))) == 0


def test_an_empty_batch_is_nothing_to_do():
    for kw in (dict(T=0), dict(B=0)):
        assert fwd(params(**kw), Q=None, O=None, LSE=None, table=None) == binding.ATTN_OK
        assert append(params(**kw), K=None, V=None, Q=None, Q_rot=None) == binding.ATTN_OK


def on_gpu(*shape, dtype=torch.bfloat16, device="cuda"):
    """A tensor that says it is on a GPU and has no memory."""
    with FakeTensorMode():
        return torch.empty(shape, dtype=dtype, device=device)


def index(*shape, **k):
    return on_gpu(*shape, dtype=torch.int32, **k)


def f32(*shape, **k):
    return on_gpu(*shape, dtype=torch.float32, **k)


CACHE, CACHE8 = on_gpu(20, 2, 16, 64), on_gpu(20, 2, 16, 64, dtype=torch.float8_e4m3fn)
COMMON = dict(K_cache=CACHE, V_cache=CACHE, page_table=index(3, 5), q_start=index(4), kv_lens=index(3))
BAD_TENSORS = [
    dict(K_cache=on_gpu(20, 2, 16, 32), V_cache=on_gpu(20, 2, 16, 32)),
    dict(K_cache=on_gpu(20, 2, 16, 64, dtype=torch.float16), V_cache=on_gpu(20, 2, 16, 64, dtype=torch.float16)),
    dict(K_cache=on_gpu(20, 2, 16, 64, dtype=torch.float8_e5m2), V_cache=on_gpu(20, 2, 16, 64, dtype=torch.float8_e5m2)),
    dict(V_cache=on_gpu(20, 2, 32, 64)), dict(V_cache=CACHE8), dict(K_cache=CACHE8, V_cache=CACHE8),
    dict(K_cache=CACHE8, V_cache=CACHE8, k_scale=f32(20, 2)),
    dict(K_cache=CACHE8, V_cache=CACHE8, k_scale=f32(20, 2), v_scale=f32(2, 20)),
    dict(K_cache=CACHE8, V_cache=CACHE8, k_scale=f32(20, 2), v_scale=on_gpu(20, 2)),
    dict(k_scale=f32(20, 2), v_scale=f32(20, 2)), dict(K_cache=on_gpu(20, 2, 16, 64, device="cpu")),
    dict(page_table=index(4, 5)), dict(page_table=index(3)), dict(page_table=on_gpu(3, 5, dtype=torch.int64)),
    dict(page_table=index(3, 5, device="cpu")), dict(q_start=index(3)), dict(q_start=on_gpu(4, dtype=torch.int64)),
    dict(kv_lens=index(3, device="cpu")), dict(kv_lens=index(2, 3)), dict(K_cache=CACHE.transpose(2, 3)),
]


@pytest.mark.parametrize("kw", BAD_TENSORS)
def test_tensors_that_do_not_belong_together(kw):
    a = {**COMMON, **kw}
    for dtype in (torch.bfloat16,):
        with pytest.raises(ValueError):
            attn.attn_fwd_paged(on_gpu(6, 8, 64, dtype=dtype), scale=0.1, causal=True, O=on_gpu(6, 8, 64),
                                LSE=f32(6, 8), split=False, **a)
        with pytest.raises(ValueError):
            attn.attn_paged_append(on_gpu(6, 2, 64, dtype=dtype), on_gpu(6, 2, 64, dtype=dtype), **a)


@pytest.mark.parametrize("kw", [
    dict(Q=on_gpu(6, 8, 64, device="cpu")), dict(Q=f32(6, 8, 64)), dict(Q=on_gpu(6, 64)), dict(O=on_gpu(6, 4, 64)),
    dict(O=on_gpu(6, 8, 64, dtype=torch.float16)), dict(LSE=f32(8, 6)), dict(LSE=on_gpu(6, 8)),
    dict(workspace=on_gpu(8, dtype=torch.uint8, device="cpu")), dict(Q=on_gpu(6, 8, 128)[:, :, ::2])])
def test_attention_refuses(kw):
    a = dict(Q=on_gpu(6, 8, 64), O=on_gpu(6, 8, 64), LSE=f32(6, 8), split=False)
    with pytest.raises(ValueError):
        attn.attn_fwd_paged(**{**a, **kw}, scale=0.1, causal=True, **COMMON)


@pytest.mark.parametrize("kw", [
    dict(K=on_gpu(6, 4, 64), V=on_gpu(6, 4, 64)), dict(V=on_gpu(5, 2, 64)), dict(Q=on_gpu(5, 8, 64)),
    dict(Q=on_gpu(6, 8, 64, dtype=torch.float16)), dict(cos=f32(80, 32)), dict(sin=f32(80, 32)),
    dict(cos=f32(79, 32), sin=f32(79, 32)), dict(cos=f32(80, 36), sin=f32(80, 36)), dict(cos=f32(80, 6), sin=f32(80, 6)),
    dict(cos=f32(80, 32), sin=f32(80, 16)), dict(cos=on_gpu(80, 32), sin=on_gpu(80, 32)),
    dict(Q_rot=on_gpu(6, 8, 64)), dict(Q=on_gpu(6, 8, 64), Q_rot=on_gpu(6, 4, 64))])
def test_append_refuses(kw):
    a = dict(K=on_gpu(6, 2, 64), V=on_gpu(6, 2, 64))
    with pytest.raises(ValueError):
        attn.attn_paged_append(**{**a, **kw}, **COMMON)
