"""freqkv_attend_q8 against attention in 64 bits over what the codes stand for."""
import math

import pytest
import torch

import _small as ref
import paper_2505_00570_amd as fk
from paper_2505_00570_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda"
BASE = 10000.0


def _off(dtype, base, rows):
    """How far turned keys and queries are off, of their magnitude: the rounding of each operand (fp16 2^-11, a sum of two of them 2^-21 with the product of the two rests
    left out), and of cos/sin, up to 64 rotations of 2^-22 each from seeds good to 2^-22."""
    turned = 0.0 if base == 0 else (1 + min(64, rows / 64)) * 2.0 ** -22
    return 2.0 * ((2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -21) + turned)


def _check(q, k8, v8, scales, block, lens, base, out, lse, vals=None, of_values=0.0):
    k, v = (ref.values(c, s, block) for c, s in zip((k8, v8), scales)) if vals is None else vals
    sc = ref.Scores(q, k, lens, base)
    p, lse_ref = sc.softmax()
    L, B, hq, n, d = q.shape
    flat = lambda x: x.reshape(L, B, k.shape[2], -1, x.shape[-1])  # noqa: E731
    want = torch.matmul(flat(p), v).view(q.shape)
    # scores off by delta make weights off by 2 delta of themselves; sums of fp32 products over T rows; weights in fp16 (fp32: two fp16); results rounded
    T = k.shape[3]
    delta = (sc.size * sc.seen).amax(-1) * _off(q.dtype, base, T) + T * 2.0 ** -24 + 2.0 ** -22 * sc.s.masked_fill(~sc.seen, 0.0).abs().amax(-1)
    of_weight = torch.expm1(2 * delta) + (2.0 ** -11 if q.dtype == torch.bfloat16 else 2.0 ** -21) + T * 2.0 ** -24
    spread = torch.matmul(flat(p), v.abs()).view(q.shape)
    # (of_values: of values, where they are rounded to fp16 as well)
    bound = (of_weight.view(q.shape[:4])[..., None] + of_values) * spread + ref.HALF_STEP[q.dtype] * want.abs() + 1e-30
    # weights that fp16 rounds to its least step, 2^-25 off in all, times the largest value of the head
    bound = bound + 2.0 ** -24 * 4 * v.abs().amax((-1, -2)).repeat_interleave(hq // k.shape[2], 2)[..., None, None] * (T if q.dtype == torch.bfloat16 else 1) ** 0.5
    err = (out.double() - want).abs()
    assert bool(torch.isfinite(out).all())
    assert bool((err <= bound).all()), float((err / bound).max())
    if lse is not None:
        lr, l = lse_ref.reshape(q.shape[:4]), lse.double()
        none = lr == -math.inf
        assert torch.equal(l == -math.inf, none)
        d_l = (l - lr)[~none].abs()
        assert bool((d_l <= (delta.view(q.shape[:4]) + 2.0 ** -22 * (1 + lr.abs()))[~none]).all())
    return float((err / bound).max())


def _attend(q, k8, v8, scales, block, cur_len, lens=None, base=BASE, lse=True, workspace=None, stream=None):
    L, B, hq, n, d = q.shape
    H = k8.shape[2]
    L8, S = ref.layouts8(k8, scales[0], scales[1], block)
    dt = fk.BF16 if q.dtype == torch.bfloat16 else fk.F32
    _, p = fk.attend_q8_plan(L8, dt, hq, H, d, cur_len, n)
    ws = ref.with_workspace(L8, p.workspace_bytes if workspace is None else workspace)
    out = torch.full_like(q, math.nan)
    ls = torch.full(q.shape[:4], math.nan, device=DEV) if lse else None
    assert fk.attend_q8(q, k8, v8, out, ls, L8, S, dt, hq, H, d, cur_len, n, lens, base, stream) == 0
    torch.cuda.synchronize()
    del ws
    return out, ls


def _case(L, B, H, G, T, n, d, dtype, fmt, block, seed, token_major=False, spare=3):
    """Caches of T rows, behind which lie codes and scales that must not matter: NaN of e4m3, NaN."""
    g = torch.Generator().manual_seed(seed)
    kv = [ref.cache((L, B, H, T, d), torch.float32, seed + i, "cpu") for i in range(2)]
    got = [ref.eight_bits(x, fmt, block, "cpu") for x in kv]
    codes, scales = [], []
    blocks = (T + spare + block - 1) // block + 1
    for c, s in got:
        full = torch.full((L, B, H, T + spare, d), 127, dtype=torch.int8).view(ref.CODES[fmt])
        full[:, :, :, :T] = c
        sc = torch.full((L, B, H, blocks), math.nan)
        sc[..., :s.shape[-1]] = s
        codes.append(ref.strided(full.to(DEV), token_major))
        scales.append(sc.to(DEV))
    q = (torch.randn(L, B, H * G, n, d, generator=g) * 0.5).to(dtype).to(DEV)
    return q, codes[0], codes[1], scales


def _run(L, B, H, G, T, n, d, dtype, fmt, block, seed=1, base=BASE, token_major=False):
    print(L, B, H, G, T, n, d, dtype, fmt, block, base, flush=True)
    q, k8, v8, scales = _case(L, B, H, G, T, n, d, dtype, fmt, block, seed, token_major)
    out, lse = _attend(q, k8, v8, scales, block, T, base=base)
    lens = torch.full((B,), T, dtype=torch.int32, device=DEV)
    k, v = (ref.values(c[:, :, :, :T], s, block) for c, s in zip((k8, v8), scales))
    way = fk.attend_q8_kernel(binding.layout_for(k8), fk.BF16 if dtype == torch.bfloat16 else fk.F32, H * G, H, d, T, n)
    worst = _check(q, None, None, None, block, lens, base, out, lse, (k, v), 2.0 ** -11 if "operands" in way else 0.0)
    print("   worst share of the bound %.3f" % worst, flush=True)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("T", [1, 2, 17, 129, 700])
def test_one_token(fmt, dtype, d, T):
    _run(1, 2, 2, 4, T, 1, d, dtype, fmt, 16 if T < 100 else 64)


@pytest.mark.parametrize("G", [1, 2, 3, 5, 8, 16, 17])
def test_head_groups(G):
    _run(2, 1, 3, G, 333, 1, 128, torch.bfloat16, "int8", 32, seed=G)


@pytest.mark.parametrize("T,n,d,G,dtype", [
    (1, 1, 128, 1, torch.bfloat16), (40, 40, 128, 1, torch.bfloat16), (300, 5, 128, 3, torch.bfloat16), (257, 33, 64, 4, torch.bfloat16),
    (400, 64, 128, 4, torch.bfloat16), (513, 129, 128, 2, torch.float32), (200, 200, 256, 1, torch.float32), (130, 7, 64, 5, torch.float32),
    (1100, 301, 128, 4, torch.bfloat16), (96, 96, 128, 4, torch.bfloat16), (95, 33, 128, 8, torch.bfloat16)])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_chunks(T, n, d, G, dtype, fmt):
    _run(1, 2, 2, G, T, n, d, dtype, fmt, 32, seed=T + n)


@pytest.mark.parametrize("L,B,H,G,T,n", [(1, 1, 64, 4, 200, 50), (2, 16, 4, 2, 71, 71), (1, 256, 1, 1, 300, 97), (3, 2, 40, 3, 40, 40), (98, 1, 4, 4, 65, 33)])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("token_major", [False, True])
def test_chunks_of_many_heads(L, B, H, G, T, n, fmt, token_major):
    """Where operands are written first."""
    L8 = binding.layout_for(torch.empty((L, B, H, T, 128), dtype=ref.CODES[fmt], device=DEV))
    assert fk.attend_q8_kernel(L8, fk.BF16, H * G, H, 128, T, n) == "k_attend_prefill (operands of codes)"
    _run(L, B, H, G, T, n, 128, torch.bfloat16, fmt, 32, seed=T + n, token_major=token_major)


def test_nan_blocks_of_many_heads():
    """The same as for few: a NaN scale makes NaN what sees its rows, and nothing else."""
    T, n, block, H = 160, 60, 16, 100
    q, k8, v8, scales = _case(1, 1, H, 2, T, n, 128, torch.bfloat16, "int8", block, 11)
    assert fk.attend_q8_kernel(binding.layout_for(k8), fk.BF16, 2 * H, H, 128, T, n) == "k_attend_prefill (operands of codes)"
    sees = 128 - (T - n)
    good, _ = _attend(q, k8, v8, scales, block, T)
    for which in range(2):
        s = [x.clone() for x in scales]
        s[which][0, 0, 1, 8] = math.nan
        out, _ = _attend(q, k8, v8, s, block, T)
        hit = torch.zeros(out.shape, dtype=torch.bool, device=DEV)
        hit[:, :, 2:4, sees:] = True
        assert torch.equal(out[~hit], good[~hit]) and bool(out[hit].isnan().all())


@pytest.mark.parametrize("base", [0.0, 500000.0])
@pytest.mark.parametrize("T", [777, 9000])
def test_rotary_bases_and_long_caches(base, T):
    _run(1, 1, 1, 4, T, 1, 128, torch.float32, "int8", 128, base=base)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_token_major(d):
    _run(2, 2, 3, 4, 150, 1, d, torch.bfloat16, "e4m3", 16, token_major=True)
    _run(2, 2, 3, 2, 150, 20, d, torch.bfloat16, "int8", 16, token_major=True)
    _run(2, 2, 3, 2, 150, 70, d, torch.bfloat16, "int8", 16, token_major=True)


@pytest.mark.parametrize("n", [1, 7, 50])
def test_sequences_of_different_lengths(n):
    """Among them none at all, fewer rows than queries (whose first queries see nothing), and one beyond the bound (clamped)."""
    T, block = 180, 32
    q, k8, v8, scales = _case(2, 6, 2, 4, T, n, 128, torch.bfloat16, "int8", block, 3)
    given = torch.tensor([180, 1, 0, 100, 33, 500], dtype=torch.int32, device=DEV)
    out, lse = _attend(q, k8, v8, scales, block, T, given)
    lens = given.clamp(0, T)
    k, v = (ref.values(c[:, :, :, :T], s, block) for c, s in zip((k8, v8), scales))
    _check(q, None, None, None, block, lens, BASE, out, lse, (k, v))
    assert not bool(out[:, 2].any()) and bool((lse[:, 2] == -math.inf).all())


def test_less_workspace_is_fewer_chunks():
    q, k8, v8, scales = _case(1, 1, 1, 4, 2000, 1, 128, torch.float32, "int8", 64, 5)
    lens = torch.full((1,), 2000, dtype=torch.int32, device=DEV)
    k, v = (ref.values(c[:, :, :, :2000], s, 64) for c, s in zip((k8, v8), scales))
    for ws in (35840, 35840 + 5 * (4 * 128 * 4 + 32) + 256):
        out, lse = _attend(q, k8, v8, scales, 64, 2000, workspace=ws)
        _check(q, None, None, None, 64, lens, BASE, out, lse, (k, v))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,n", [(torch.bfloat16, 1), (torch.float32, 1), (torch.float32, 30)])
def test_magnitudes(fmt, dtype, n):
    """Scales and queries far from 1: keys by 2^60 and queries by 2^-60, values of blocks by 2^-40 .. 2^40."""
    T, block, d = 200, 16, 128
    q, k8, v8, scales = _case(1, 1, 2, 4, T, n, d, dtype, fmt, block, 9)
    scales[0].mul_(2.0 ** 60)
    q.mul_(2.0 ** -60)
    lens = torch.full((1,), T, dtype=torch.int32, device=DEV)
    for powers in (torch.linspace(-40, 40, scales[1].shape[-1]).round(), torch.linspace(40, -40, scales[1].shape[-1]).round()):
        vs = scales[1] * torch.exp2(powers).to(DEV)
        out, lse = _attend(q, k8, v8, [scales[0], vs], block, T)
        k, v = ref.values(k8[:, :, :, :T], scales[0], block), ref.values(v8[:, :, :, :T], vs, block)
        _check(q, None, None, None, block, lens, BASE, out, lse, (k, v))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_magnitudes_of_operands(fmt):
    """The same where operands are written first: keys by 2^60, queries by 2^-60 and the other way round, values by 2^90 and 2^-90, blocks of a head 2^-10 .. 1 of each other."""
    T, block, n = 200, 32, 50
    q, k8, v8, scales = _case(1, 1, 64, 4, T, n, 128, torch.bfloat16, fmt, block, 9)
    assert fk.attend_q8_kernel(binding.layout_for(k8), fk.BF16, 256, 64, 128, T, n) == "k_attend_prefill (operands of codes)"
    lens = torch.full((1,), T, dtype=torch.int32, device=DEV)
    for e in (60, -60):
        ks = scales[0] * 2.0 ** e
        vs = scales[1] * 2.0 ** (1.5 * e) * torch.exp2(-torch.arange(scales[1].shape[-1], device=DEV).float().clamp(max=10))
        qq = q * 2.0 ** -e
        out, lse = _attend(qq, k8, v8, [ks, vs], block, T)
        k, v = ref.values(k8[:, :, :, :T], ks, block), ref.values(v8[:, :, :, :T], vs, block)
        _check(qq, None, None, None, block, lens, BASE, out, lse, (k, v), of_values=2.0 ** -11)


@pytest.mark.parametrize("dtype,n", [(torch.bfloat16, 60), (torch.float32, 60), (torch.bfloat16, 32)])
def test_nan_blocks(dtype, n):
    """A NaN scale makes NaN what sees its rows, and nothing else."""
    T, block = 160, 16
    q, k8, v8, scales = _case(1, 1, 2, 2, T, n, 128, dtype, "int8", block, 11)
    sees = 128 - (T - n)                              # the first query that sees row 128
    good, _ = _attend(q, k8, v8, scales, block, T)
    for which in range(2):
        s = [x.clone() for x in scales]
        s[which][0, 0, 1, 8] = math.nan               # rows 128 .. 143 of the second head
        out, _ = _attend(q, k8, v8, s, block, T)
        assert torch.equal(out[:, :, :2], good[:, :, :2]) and torch.equal(out[:, :, 2:, :max(sees, 0)], good[:, :, 2:, :max(sees, 0)])
        assert bool(out[:, :, 2:, max(sees, 0):].isnan().all())


def test_zero_queries_and_zero_blocks():
    T, block = 100, 16
    q, k8, v8, scales = _case(1, 1, 2, 4, T, 1, 128, torch.bfloat16, "int8", block, 13)
    q[:, :, 1] = 0.0
    scales[0][..., 2] = 0.0
    scales[1][..., 0] = 0.0
    lens = torch.full((1,), T, dtype=torch.int32, device=DEV)
    out, lse = _attend(q, k8, v8, scales, block, T)
    k, v = (ref.values(c[:, :, :, :T], s, block) for c, s in zip((k8, v8), scales))
    _check(q, None, None, None, block, lens, BASE, out, lse, (k, v))
    _, l = ref.Scores(q, k, lens, BASE).softmax()
    assert abs(float(lse[0, 0, 1, 0]) - math.log(T)) < 1e-5


def test_replayed_graph_of_a_chunk():
    """Operands written first: captured by a call that finds none of its tables, replayed on other codes and queries, with eager calls between."""
    T, block, n = 300, 32, 40
    q, k8, v8, scales = _case(1, 32, 2, 4, T, n, 128, torch.bfloat16, "e4m3", block, 17)
    assert fk.attend_q8_kernel(binding.layout_for(k8), fk.BF16, 8, 2, 128, T, n) == "k_attend_prefill (operands of codes)"
    L8, S = ref.layouts8(k8, scales[0], scales[1], block)
    _, p = fk.attend_q8_plan(L8, fk.BF16, 8, 2, 128, T, n)
    ws = ref.with_workspace(L8, p.workspace_bytes)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:4], device=DEV)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        assert fk.attend_q8(q, k8, v8, out, lse, L8, S, fk.BF16, 8, 2, 128, T, n, None, 27183.0, st) == 0
    for i in range(3):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(i)).to(q.dtype).to(DEV) * 0.5)
        scales[1].mul_(3.0)
        g.replay()
        torch.cuda.synchronize()
        eager, el = _attend(q, k8, v8, scales, block, T, base=27183.0)
        assert torch.equal(out, eager) and torch.equal(lse, el)
    del ws


def test_stream_and_replayed_graph():
    """On a stream of its own; captured, then replayed with other rows, queries and lengths."""
    T, block, n = 600, 32, 1
    q, k8, v8, scales = _case(1, 3, 2, 4, T, n, 128, torch.bfloat16, "int8", block, 15)
    lens = torch.tensor([600, 77, 300], dtype=torch.int32, device=DEV)
    L8, S = ref.layouts8(k8, scales[0], scales[1], block)
    _, p = fk.attend_q8_plan(L8, fk.BF16, 8, 2, 128, T, n)
    ws = ref.with_workspace(L8, p.workspace_bytes)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:4], device=DEV)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    base = 31337.0                                    # a rotary table that no call has made before
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        assert fk.attend_q8(q, k8, v8, out, lse, L8, S, fk.BF16, 8, 2, 128, T, n, lens, base, st) == 0
    for i in range(4):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(i)).to(q.dtype).to(DEV) * 0.5)
        lens.copy_(torch.tensor([[600, 77, 300], [1, 600, 0], [64, 65, 128], [599, 2, 31]][i], dtype=torch.int32).to(DEV))
        out.fill_(math.nan)
        g.replay()
        torch.cuda.synchronize()
        k, v = (ref.values(c[:, :, :, :T], s, block) for c, s in zip((k8, v8), scales))
        _check(q, None, None, None, block, lens, base, out, lse, (k, v))
        eager, _ = _attend(q, k8, v8, scales, block, T, lens, base)
        assert torch.equal(out, eager)
    del ws
