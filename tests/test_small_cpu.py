"""What the entry points of 8-bit caches, attention weights and eviction refuse, and what their plans say.  No GPU: refusals come before any device work."""
import ctypes as C

import pytest
import torch

import paper_2505_00570_amd as fk
from paper_2505_00570_amd import binding

FAKE = 1 << 20                        # an aligned address that is never read


def _layout(dtype, layers=2, batch=3, heads=2, cap=100, d=128):
    L = binding.Layout()
    L.dtype, L.n_layers, L.batch, L.token_capacity = dtype, layers, batch, cap
    L.stride_token, L.stride_head, L.stride_batch, L.stride_layer = d, cap * d, heads * cap * d, batch * heads * cap * d
    L.workspace, L.workspace_bytes = FAKE, 1 << 30
    return L


def _scales(block=32):
    S = binding.Scales()
    S.k = S.v = FAKE
    S.block_tokens, S.stride_layer, S.stride_batch, S.stride_head = block, 24, 8, 4
    return S


def _set(o, **kw):
    for k, v in kw.items():
        setattr(o, k, v)
    return o


def _quantize(L=None, L8=None, S=None, k=FAKE, v=FAKE, k8=FAKE, v8=FAKE, row=0, at=0, n=8, heads=2, d=128, rows=None):
    return fk.quantize(k, v, L or _layout(fk.BF16), row, k8, v8, L8 or _layout(fk.INT8), S or _scales(), at, n, heads, d, rows, check=False)


def _dequantize(L=None, L8=None, S=None, k=FAKE, v=FAKE, k8=FAKE, v8=FAKE, row=0, at=0, n=8, heads=2, d=128):
    return fk.dequantize(k8, v8, L8 or _layout(fk.E4M3), S or _scales(), at, k, v, L or _layout(fk.F32), row, n, heads, d, check=False)


@pytest.mark.parametrize("call", [_quantize, _dequantize])
def test_store_refuses(call):
    inv, uns = binding.E_INVALID, binding.E_UNSUPPORTED
    assert call(n=0) == fk.binding.NOOP
    for kw in (dict(k=None), dict(v=None), dict(k8=None), dict(v8=None), dict(k=FAKE + 8), dict(v8=FAKE + 8), dict(n=-1), dict(row=-1), dict(at=-1),
               dict(row=93), dict(at=93), dict(row=2 ** 31 - 1), dict(heads=0), dict(d=8), dict(L=_layout(fk.INT8)), dict(L8=_layout(fk.BF16)),
               dict(L=_layout(fk.BF16, layers=1)), dict(L=_layout(fk.BF16, batch=2)), dict(L=_set(_layout(fk.BF16), stride_token=64)),
               dict(L8=_set(_layout(fk.INT8), stride_token=136)), dict(L8=_set(_layout(fk.INT8), stride_head=8)), dict(L8=_set(_layout(fk.E4M3), stride_head=-16)),
               dict(L8=_set(_layout(fk.INT8), pointer_table=2)), dict(L8=_set(_layout(fk.INT8), flags=0x100)), dict(L=_set(_layout(fk.BF16), n_layers=0)),
               dict(S=_scales(8)), dict(S=_scales(48)), dict(S=_scales(256)), dict(S=_set(_scales(), k=None)), dict(S=_set(_scales(), v=FAKE + 2)),
               dict(S=_set(_scales(), stride_head=-1))):
        assert call(**kw) == inv, kw
    assert call(d=24, L=_layout(fk.BF16, d=32), L8=_layout(fk.INT8, d=32)) == uns
    assert call(d=272, L=_layout(fk.BF16, d=272), L8=_layout(fk.INT8, d=272)) == uns
    if call is _quantize:
        assert call(rows=FAKE + 2) == inv and call(rows=FAKE, n=101, L=_layout(fk.BF16, cap=200)) == inv


def _attend(L8=None, S=None, q=FAKE, k8=FAKE, v8=FAKE, out=FAKE, lse=None, dt=None, nq=8, nkv=2, d=128, cur=64, n=1, lens=None, base=1e4):
    return fk.attend_q8(q, k8, v8, out, lse, L8 or _layout(fk.INT8), S or _scales(), fk.BF16 if dt is None else dt, nq, nkv, d, cur, n, lens, base, check=False)


def test_attend_refuses():
    inv, uns = binding.E_INVALID, binding.E_UNSUPPORTED
    for kw in (dict(q=None), dict(out=None), dict(k8=None), dict(v8=None), dict(q=FAKE + 8), dict(out=FAKE + 4), dict(lse=FAKE + 8), dict(k8=FAKE + 4),
               dict(dt=fk.INT8), dict(dt=7), dict(nq=7), dict(nkv=0), dict(cur=0), dict(cur=101), dict(n=0), dict(n=65), dict(lens=FAKE + 1), dict(base=-1.0),
               dict(base=float("nan")), dict(base=float("inf")), dict(S=_scales(24)), dict(L8=_layout(fk.BF16)), dict(L8=_layout(fk.F32)),
               dict(L8=_set(_layout(fk.INT8), stride_token=120)), dict(L8=_set(_layout(fk.INT8), stride_layer=8))):
        assert _attend(**kw) == inv, kw
    assert _attend(d=96) == uns
    assert _attend(L8=_set(_layout(fk.INT8), stride_token=1 << 22)) == uns
    for kw in (dict(workspace=None), dict(workspace=FAKE + 128), dict(workspace_bytes=1000)):
        assert _attend(L8=_set(_layout(fk.INT8), **kw)) == binding.E_WORKSPACE
    with pytest.raises(fk.FreqKVError):
        fk.attend_q8_plan(_layout(fk.BF16), fk.BF16, 8, 2, 128, 64)


def _weights(L=None, q=FAKE, k=FAKE, lse=FAKE, w=FAKE, nq=8, nkv=2, d=128, cur=64, n=1, lens=None, acc=0, base=1e4):
    lib = fk.load()
    return lib.freqkv_attend_weights(q, k, lse, w, C.byref(L or _layout(fk.BF16)), nq, nkv, d, cur, n, lens, acc, base, None)


def test_weights_refuses():
    inv, uns = binding.E_INVALID, binding.E_UNSUPPORTED
    for kw in (dict(q=None), dict(k=None), dict(lse=None), dict(w=None), dict(q=FAKE + 8), dict(k=FAKE + 8), dict(lse=FAKE + 2), dict(w=FAKE + 1), dict(nq=7), dict(cur=0),
               dict(cur=101), dict(n=0), dict(n=65), dict(lens=FAKE + 1), dict(acc=2), dict(acc=-1), dict(base=-1.0), dict(base=float("nan")),
               dict(L=_layout(fk.INT8)), dict(L=_layout(fk.E4M3))):
        assert _weights(**kw) == inv, kw
    assert _weights(d=96) == uns
    for kw in (dict(workspace=None), dict(workspace=FAKE + 128), dict(workspace_bytes=1000)):
        assert _weights(L=_set(_layout(fk.BF16), **kw)) == binding.E_WORKSPACE


def _evict(L=None, k=FAKE, v=FAKE, w=FAKE, wo=None, kept=FAKE, heads=2, d=128, cur=64, sink=4, recent=8, keep=10, lens=None, new=None):
    return fk.evict(k, v, w, wo, kept, L or _layout(fk.BF16), heads, d, cur, sink, recent, keep, lens, new, check=False)


def test_evict_refuses():
    inv = binding.E_INVALID
    for kw in (dict(k=None), dict(v=None), dict(w=None), dict(kept=None), dict(k=FAKE + 8), dict(w=FAKE + 2), dict(wo=FAKE + 2), dict(kept=FAKE + 1), dict(lens=FAKE + 2),
               dict(new=FAKE + 2), dict(lens=FAKE, new=FAKE), dict(heads=0), dict(d=0), dict(cur=0), dict(cur=101), dict(sink=-1), dict(recent=-1), dict(keep=0), dict(keep=-3),
               dict(L=_layout(fk.INT8)), dict(L=_set(_layout(fk.BF16), stride_token=64)), dict(L=_set(_layout(fk.F32), stride_batch=-8))):
        assert _evict(**kw) == inv, kw
    assert _evict(d=20, L=_layout(fk.BF16, d=24)) == binding.E_UNSUPPORTED


def test_other_entry_points_refuse_codes():
    for dt in (fk.INT8, fk.E4M3):
        L = _layout(dt)
        assert fk.attend_plan(L, 8, 2, 128, 64, check=False)[0] == binding.E_INVALID
        assert fk.attend_prefill_plan(L, 8, 2, 128, 64, 5, check=False)[0] == binding.E_INVALID
        assert fk.plan(L, 2, 128, 64, 64, 4, 0.5, check=False)[0] == binding.E_INVALID
        assert fk.compress(FAKE, FAKE, L, 2, 128, 64, 64, 4, 0.5, check=False) == binding.E_INVALID


def test_plans():
    for d in (64, 128, 256):
        for cur in (1, 63, 64, 65, 4097):
            for n in {1, cur // 2 + 1, cur}:
                L8, L = _layout(fk.INT8, cap=5000, d=d), _layout(fk.F32, cap=5000, d=d)
                for dt in (fk.BF16, fk.F32):
                    _, p = fk.attend_q8_plan(L8, dt, 6, 2, d, cur, n)
                    assert p.n_split * p.chunk_rows >= cur > (p.n_split - 1) * p.chunk_rows
                    seen = sum(cur - n + i + 1 for i in range(n))
                    assert p.flops == 4.0 * d * seen * 6 * 6
                    assert p.bytes_algorithmic == 12 * (2 * cur * d + 2 * 3 * n * d * (2 if dt == fk.BF16 else 4))
                _, p = fk.attend_weights_plan(L, 6, 2, d, cur, n)
                assert p.flops == 2.0 * d * seen * 6 * 6 and p.workspace_bytes >= 35840


def test_caches_ask_for_what_their_calls_need():
    """Workspaces and buffers of the two caches that are kept small, and what their makers refuse."""
    from paper_2505_00570_amd.cache import CompressedKVCache, QuantizedKVCache
    c = CompressedKVCache(2, 1, 2, 64, 100, n_q_heads=8, by_weight=True, n_recent=10, device="cpu")
    assert c.weights.shape == (2, 1, 2, 100) and not bool(c.weights.any()) and c.kept.shape == (2, 1, 2, 38)
    assert c.compress() == binding.NOOP and c.cur_len == 0
    for n_recent in (-1, 48):
        with pytest.raises(ValueError):
            CompressedKVCache(2, 1, 2, 64, 100, by_weight=True, n_recent=n_recent, device="cpu")
    for code in (torch.int8, torch.float8_e4m3fn):
        c = QuantizedKVCache(5, 1, 2, 64, 100, n_q_heads=8, device="cpu", code_dtype=code, stage_layers=2)
        assert c.compress() == binding.NOOP and c.k_scale.shape == (5, 1, 2, 2) and c.stage_k.shape[0] == 2
        for n, q_len in ((1, 1), (50, 1), (100, 1), (100, 37), (100, 100)):
            # (a smaller one than planned is used all the same: down to that of one chunk)
            assert c.layout.workspace_bytes >= 35840
            assert fk.attend_q8_plan(c.layout, fk.BF16, 8, 2, 64, n, q_len)[1].workspace_bytes <= c.layout.workspace_bytes


def test_what_is_written_twice_is_refused():
    """K and V, or two layers, at one address: rows moved or rounded in place by two workgroups at once."""
    inv, far = binding.E_INVALID, FAKE + (1 << 20)
    apart = _set(_scales(), v=far)
    assert _quantize(v8=far) == inv and _quantize(S=apart) == inv                   # scales; codes
    assert _quantize(S=_set(_set(_scales(), v=far), stride_layer=0), v8=far) == inv
    assert _quantize(L8=_set(_layout(fk.INT8), stride_layer=0), S=apart, v8=far) == inv
    assert _dequantize() == inv and _dequantize(v=far, L=_set(_layout(fk.F32), stride_layer=0)) == inv
    assert _evict() == inv and _evict(v=far, L=_set(_layout(fk.BF16), stride_layer=0)) == inv
    table = (C.c_void_p * 2)(FAKE, far)
    assert _evict(k=table, v=table, L=_set(_layout(fk.BF16), pointer_table=1)) == inv
