"""Calls on caches kept small that lie at an edge: behind tables of pointers, past 4 GB, in other orders of memory, two at once, all registers taken."""
import ctypes
import math

import pytest
import torch

import _small as ref
import paper_2505_00570_amd as fk
from paper_2505_00570_amd import binding
from test_gpu_evict import _check_weights, _verify
from test_gpu_q8_attend import BASE, _attend, _check, _run

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _table(x):
    return (ctypes.c_void_p * x.shape[0])(*[x[i].data_ptr() for i in range(x.shape[0])])


def _q(shape, dtype, seed):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * 0.5).to(dtype).to(DEV)


@pytest.mark.parametrize("n", [1, 40])
def test_many_layers_behind_tables(n):
    """More layers than one launch takes; each layer's rows and codes at an address of their own, scales in one array."""
    L, H, G, T, d, block = 98, 1, 4, 70, 128, 32
    k, v = (ref.cache((L, 1, H, T, d), torch.bfloat16, i, DEV) for i in range(2))
    k8, v8 = (torch.empty((L, 1, H, T, d), dtype=torch.int8, device=DEV) for _ in range(2))
    ks, vs = (torch.empty((L, 1, H, 3), device=DEV) for _ in range(2))
    lay, (L8, S) = binding.layout_for(k), ref.layouts8(k8, ks, vs, block)
    lay.pointer_table = L8.pointer_table = 1
    assert fk.quantize(_table(k), _table(v), lay, 0, _table(k8), _table(v8), L8, S, 0, T, H, d) == 0
    torch.cuda.synchronize()
    for x, c, s in ((k, k8, ks), (v, v8, vs)):
        codes, scales = ref.eight_bits(x, "int8", block)
        assert torch.equal(c, codes) and torch.equal(s, scales)
    q = _q((L, 1, H * G, n, d), torch.bfloat16, 3)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:4], device=DEV)
    ws = ref.with_workspace(L8, fk.attend_q8_plan(L8, fk.BF16, H * G, H, d, T, n)[1].workspace_bytes)
    assert fk.attend_q8(q, _table(k8), _table(v8), out, lse, L8, S, fk.BF16, H * G, H, d, T, n, None, BASE) == 0
    torch.cuda.synchronize()
    lens = torch.full((1,), T, dtype=torch.int32, device=DEV)
    rows = [ref.values(c, s, block) for c, s in ((k8, ks), (v8, vs))]
    _check(q, None, None, None, block, lens, BASE, out, lse, rows, 2.0 ** -11)
    back = [torch.empty_like(k) for _ in range(2)]
    assert fk.dequantize(_table(k8), _table(v8), L8, S, 0, _table(back[0]), _table(back[1]), lay, 0, T, H, d) == 0
    torch.cuda.synchronize()
    assert all(torch.equal(b, r.bfloat16()) for b, r in zip(back, rows))
    _, l = ref.Scores(q, k, lens, BASE).softmax()
    lse = l.reshape(q.shape[:4]).float().contiguous()
    w = torch.zeros((L, 1, H, T), device=DEV)
    ws2 = ref.with_workspace(lay, fk.attend_weights_plan(lay, H * G, H, d, T, n)[1].workspace_bytes)
    assert fk.attend_weights(q, _table(k), lse, w, lay, H * G, H, d, T, n, rope_base=BASE) == 0
    torch.cuda.synchronize()
    _check_weights(q, k, lse, lens, BASE, w, torch.zeros_like(w), False)
    del ws, ws2


@pytest.mark.parametrize("order", [(1, 0, 2, 3), (2, 1, 0, 3), (3, 0, 1, 2), (3, 2, 1, 0)])
def test_orders_of_memory(order):
    """Layers, sequences, heads and tokens outside one another in any order: each operator gives what it gives for the usual one."""
    shape, d, G, T, block = (2, 3, 2, 90), 64, 2, 90, 16
    L, B, H, _ = shape

    def ordered(x):
        p = list(order) + [4]
        back = [p.index(i) for i in range(5)]
        return x.permute(p).contiguous().permute(back)

    k, v = (ref.cache((*shape, d), torch.float32, i, DEV) for i in range(2))
    got = []
    for put in (lambda x: x, ordered):
        kk, vv = put(k.clone()), put(v.clone())
        k8, v8 = (put(torch.zeros((*shape, d), dtype=torch.float8_e4m3fn, device=DEV).view(torch.uint8)).view(torch.float8_e4m3fn) for _ in range(2))
        ks, vs = (torch.zeros((L, B, H, 6), device=DEV) for _ in range(2))
        lay, (L8, S) = binding.layout_for(kk), ref.layouts8(k8, ks, vs, block)
        for lo, hi in ((0, 50), (50, 51), (51, T)):
            assert fk.quantize(kk, vv, lay, lo, k8, v8, L8, S, lo, hi - lo, H, d) == 0
        row = [k8, v8, ks, vs]
        for dtype, n in ((torch.bfloat16, 1), (torch.float32, 7)):
            q = _q((L, B, H * G, n, d), dtype, n)
            row += list(_attend(q, k8, v8, (ks, vs), block, T))
        lens = torch.full((B,), T, dtype=torch.int32, device=DEV)
        w = torch.zeros((L, B, H, T), device=DEV)
        for n in (1, 20):
            q = _q((L, B, H * G, n, d), torch.float32, n)
            _, l = ref.Scores(q, k, lens, BASE).softmax()
            lse = l.reshape(q.shape[:4]).float().contiguous()
            ws = ref.with_workspace(lay, fk.attend_weights_plan(lay, H * G, H, d, T, n)[1].workspace_bytes)
            assert fk.attend_weights(q, kk, lse, w, lay, H * G, H, d, T, n, accumulate=True, rope_base=BASE) == 0
            torch.cuda.synchronize()
            del ws
        kept = torch.empty((L, B, H, 30), dtype=torch.int32, device=DEV)
        w1 = w.clone()
        assert fk.evict(kk, vv, w, w, kept, lay, H, d, T, 3, 9, 30) == 0
        torch.cuda.synchronize()
        _verify(k, v, w1, kk, vv, w, kept, None, T, None, 3, 9, 30)
        row += [w1, w, kept, kk[:, :, :, :42], vv[:, :, :, :42]]
        got.append(row)
    for a, b in zip(*got):
        if a.dtype == torch.float8_e4m3fn:
            a, b = a.float(), b.float()
        assert torch.equal(a, b)


def test_codes_past_four_gigabytes():
    """The last sequences of a cache whose codes (and rows) take more bytes than 32 bits count."""
    B, H, T, d, block, G, n = 130, 32, 8192, 128, 64, 2, 1
    k8, v8 = (torch.zeros((1, B, H, T, d), dtype=torch.int8, device=DEV) for _ in range(2))
    k, v = (torch.zeros((1, B, H, T, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    assert k8[0, 129].data_ptr() - k8.data_ptr() >= 1 << 32
    ks, vs = (torch.zeros((1, B, H, T // block), device=DEV) for _ in range(2))
    # (rows strided so far apart that the last heads lie past 4 GB)
    big = torch.zeros(13 << 29, dtype=torch.int8, device=DEV)
    far = big.as_strided((1, 2, 2, 200, d), (0, 4 << 30, 2 << 30, 5 * d, 1))
    assert far[0, 1, 1, 199].data_ptr() - far.data_ptr() < big.numel()
    lay = binding.layout_for(k)
    for x, seed in ((k, 1), (v, 2)):
        x[:, 129, 30:] = ref.cache((1, 1, 2, T, d), torch.bfloat16, seed, DEV)[0]
    L8, S = ref.layouts8(k8, ks, vs, block)
    assert fk.quantize(k, v, lay, 0, k8, v8, L8, S, 0, T, H, d) == 0
    torch.cuda.synchronize()
    for x, c, s in ((k, k8, ks), (v, v8, vs)):
        want = ref.values(c[:, 129:, 30:], s[:, 129:, 30:], block)
        step = s[:, 129:, 30:].double()[..., torch.arange(T, device=DEV) // block, None]
        assert bool(((want - x[:, 129:, 30:].double()).abs() <= 0.5 * step).all()) and not bool(c[:, :129].any())
    q = _q((1, B, H * G, n, d), torch.bfloat16, 5)
    out, lse = _attend(q, k8, v8, (ks, vs), block, T)
    rows = [ref.values(c[:, 129:, 30:], s[:, 129:, 30:], block) for c, s in ((k8, ks), (v8, vs))]
    lens = torch.full((1,), T, dtype=torch.int32, device=DEV)
    _check(q[:, 129:, 60:], None, None, None, block, lens, BASE, out[:, 129:, 60:], lse[:, 129:, 60:], rows)
    # the same heads, 2 GB from one to the next
    two = k8[:, 128:, 30:, :200].clone()
    far.copy_(two)
    sc = [x[:, 128:, 30:, :4].contiguous() for x in (ks, vs)]
    qf = q[:, 128:, 60:].contiguous()
    near, nl = _attend(qf, two, two, sc, block, 200)
    there, tl = _attend(qf, far, far, sc, block, 200)
    assert torch.equal(near, there) and torch.equal(nl, tl)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("T", [33, 128, 129, 255, 640, 2000, 5000])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 3), (20, 1), (2, 19)])
def test_wide_heads_of_full_precision(fmt, T, G, n):
    """256 channels with fp32 queries: the kernel with most to hold."""
    _run(1, 2, 2, G, T, n, 256, torch.float32, fmt, 64, seed=T + n)


def test_two_streams_at_once():
    """Two calls that run beside each other, each with its workspace, give what they give alone."""
    cases = []
    for seed, (T, n, H) in enumerate(((3000, 1, 4), (900, 60, 40))):
        k, v = (ref.cache((1, 2, H, T, 128), torch.bfloat16, seed + i, DEV) for i in range(2))
        k8, v8 = (torch.zeros((1, 2, H, T, 128), dtype=torch.int8, device=DEV) for _ in range(2))
        ks, vs = (torch.zeros((1, 2, H, -(-T // 64)), device=DEV) for _ in range(2))
        lay, (L8, S) = binding.layout_for(k), ref.layouts8(k8, ks, vs, 64)
        q = _q((1, 2, 4 * H, n, 128), torch.bfloat16, seed)
        ws = (ref.with_workspace(lay, fk.attend_weights_plan(lay, 4 * H, H, 128, T, n)[1].workspace_bytes),
              ref.with_workspace(L8, fk.attend_q8_plan(L8, fk.BF16, 4 * H, H, 128, T, n)[1].workspace_bytes))
        out, lse, w = torch.empty_like(q), torch.empty(q.shape[:4], device=DEV), torch.zeros((1, 2, H, T), device=DEV)
        cases.append((k, v, k8, v8, ks, vs, lay, L8, S, q, out, lse, w, T, n, H, ws))

    def run(c, st):
        k, v, k8, v8, ks, vs, lay, L8, S, q, out, lse, w, T, n, H, _ = c
        assert fk.quantize(k, v, lay, 0, k8, v8, L8, S, 0, T, H, 128, stream=st) == 0
        assert fk.attend_q8(q, k8, v8, out, lse, L8, S, fk.BF16, 4 * H, H, 128, T, n, None, BASE, st) == 0
        assert fk.attend_weights(q, k, lse, w, lay, 4 * H, H, 128, T, n, rope_base=BASE, stream=st) == 0

    want = []
    for c in cases:
        run(c, torch.cuda.current_stream())
        torch.cuda.synchronize()
        want.append([x.clone() for x in (c[2], c[3], c[4], c[5], c[10], c[11], c[12])])
        for x in (c[2], c[3], c[4], c[5], c[10], c[11], c[12]):
            x.zero_()
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for i in range(3):
        for c, st in zip(cases, streams):
            run(c, st)
    torch.cuda.synchronize()
    for c, was in zip(cases, want):
        assert all(torch.equal(a, b) for a, b in zip((c[2], c[3], c[4], c[5], c[10], c[11], c[12]), was))
        assert not math.isnan(float(c[12].sum()))
