"""Caches kept small, as they are used: chunk-wise prefill and decoding with triggers between, the 8-bit cache that a compression goes through and the cache
that evicts by the attention its rows got.  Every result is compared with 64 bits over what the cache holds at that moment."""
import math

import pytest
import torch

import _small as ref
import paper_2505_00570_amd as fk
from paper_2505_00570_amd import binding
from paper_2505_00570_amd.cache import CompressedKVCache, QuantizedKVCache
from test_gpu_evict import _check_weights, _expect
from test_gpu_q8_attend import _check

pytestmark = pytest.mark.gpu
DEV = "cuda"
BASE = 10000.0


def _tokens(L, B, H, G, T, d, dtype, seed):
    k, v = (ref.cache((L, B, H, T, d), dtype, seed + i, DEV, token_major=i == 1) for i in range(2))
    v = v.contiguous()
    q = (torch.randn((L, B, H * G, T, d), generator=torch.Generator().manual_seed(seed)) * 0.5).to(dtype).to(DEV)
    return k.contiguous(), v, q


@pytest.mark.parametrize("code,block", [(torch.int8, 64), (torch.float8_e4m3fn, 16)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantized_cache(code, block, dtype):
    L, B, H, G, d, W, S = 3, 2, 2, 4, 128, 132, 4
    cache = QuantizedKVCache(L, B, H, d, W, S, dtype=dtype, n_q_heads=H * G, rope_base=BASE, code_dtype=code, block_tokens=block, stage_layers=2)
    fmt = "int8" if code == torch.int8 else "e4m3"
    k, v, q = _tokens(L, B, H, G, 350, d, dtype, 3)
    plain = cache.compress
    sinks = (k[:, :, :, :S].clone(), v[:, :, :, :S].clone())

    def compress():
        """The same from what the codes stand for: rounded to the rows' type, compressed, rounded to codes."""
        n = cache.cur_len
        rows = [ref.values(c[:, :, :, :n], s, block).to(dtype).contiguous() for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]
        for x, s in zip(rows, sinks):
            x[:, :, :, :S] = s
        for l0, l1 in ((0, 2), (2, 3)):
            part = [x[l0:l1].contiguous() for x in rows]
            lay = binding.layout_for(part[0])
            _, p = fk.plan(lay, H, d, n, W, S, 0.5)
            ws = ref.with_workspace(lay, p.workspace_bytes)
            assert fk.compress(part[0], part[1], lay, H, d, n, W, S, 0.5) == 0
            for x, y in zip(rows, part):
                x[l0:l1] = y
            torch.cuda.synchronize()
            del ws
        assert plain() == 0
        torch.cuda.synchronize()
        m = cache.cur_len
        assert m == S + 64
        for x, c, s in zip(rows, (cache.k, cache.v), (cache.k_scale, cache.v_scale)):
            codes, scales = ref.eight_bits(x[:, :, :, :m], fmt, block)
            assert torch.equal(s[..., :scales.shape[-1]], scales)
            assert torch.equal(c[:, :, :, :m].float(), codes.float())
        return 0

    cache.compress = compress

    def check(out, qs):
        n = cache.cur_len
        lens = torch.full((B,), n, dtype=torch.int32, device=DEV)
        vals = [ref.values(c[:, :, :, :n], s, block) for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]
        _check(qs, None, None, None, block, lens, BASE, out, None, vals)

    done = 0
    for take in (1, 100, 60, 40, 130):                # prompts
        piece = [x[:, :, :, done:done + take].contiguous() for x in (k, v, q)]
        left = cache.room()
        out = cache.prefill(*piece)
        torch.cuda.synchronize()
        last = take if take <= left else (take - left - 1) % (W - S - 64) + 1
        check(out[:, :, :, take - last:].contiguous(), piece[2][:, :, :, take - last:].contiguous())
        done += take
    while done < 350:                                 # tokens
        cache.append(k[:, :, :, done:done + 1], v[:, :, :, done:done + 1])
        qs = q[:, :, :, done].contiguous()
        out = cache.attend_decode(qs)
        torch.cuda.synchronize()
        check(out[:, :, :, None], qs[:, :, :, None])
        done += 1
    assert cache.triggers == 4 and cache.cur_len == 350 - 4 * (W - S - 64)


@pytest.mark.parametrize("n_recent", [0, 16])
def test_cache_that_evicts(n_recent):
    L, B, H, G, d, W, S = 2, 2, 2, 4, 128, 100, 4
    cache = CompressedKVCache(L, B, H, d, W, S, n_q_heads=H * G, rope_base=BASE, by_weight=True, n_recent=n_recent)
    keep = cache.kept.shape[3]
    assert keep == 48 - n_recent
    k, v, q = _tokens(L, B, H, G, 260, d, torch.bfloat16, 5)
    # rows [L, B, H][row]: which token they are
    held = [[[[] for _ in range(H)] for _ in range(B)] for _ in range(L)]
    evict = cache.compress

    def compress():
        w = cache.weights.clone()
        assert evict() == 0
        torch.cuda.synchronize()
        for l in range(L):
            for b in range(B):
                for h in range(H):
                    rows, order = _expect(None, w[l, b, h].tolist(), W, S, n_recent, keep)
                    assert cache.kept[l, b, h].tolist() == order
                    held[l][b][h] = [held[l][b][h][r] for r in rows]
                    at = torch.tensor(rows, device=DEV)
                    assert torch.equal(cache.weights[l, b, h, :len(rows)], w[l, b, h, at]) and not bool(cache.weights[l, b, h, len(rows):].any())
        return 0

    cache.compress = compress
    write = cache._write

    def written(kn, vn, t0, take):
        write(kn, vn, t0, take)
        for l in range(L):
            for b in range(B):
                for h in range(H):
                    held[l][b][h] += range(done + t0, done + t0 + take)

    cache._write = written
    add = cache._add_weights

    def added(qs, lse, q_len):
        start, n = cache.weights.clone(), cache.cur_len
        add(qs, lse, q_len)
        torch.cuda.synchronize()
        # the cache holds the tokens that were to stay
        for l in range(L):
            for b in range(B):
                for h in range(H):
                    at = torch.tensor(held[l][b][h], device=DEV)
                    assert len(at) == n and torch.equal(cache.k[l, b, h, :n], k[l, b, h, at]) and torch.equal(cache.v[l, b, h, :n], v[l, b, h, at])
        lens = torch.full((B,), n, dtype=torch.int32, device=DEV)
        five = qs if qs.dim() == 5 else qs[:, :, :, None]
        _check_weights(five, cache.k[:, :, :, :n], lse.view(five.shape[:4]), lens, BASE, cache.weights[..., :n], start[..., :n], True)
        assert torch.equal(cache.weights[..., n:], start[..., n:])

    cache._add_weights = added
    done = 0
    for take in (70, 1, 80, 60):
        cache.prefill(*[x[:, :, :, done:done + take].contiguous() for x in (k, v, q)])
        done += take
    while done < 260:
        cache.append(k[:, :, :, done:done + 1], v[:, :, :, done:done + 1])
        cache.attend_decode(q[:, :, :, done].contiguous())
        done += 1
    torch.cuda.synchronize()
    assert cache.triggers == 4 and cache.cur_len == 260 - 4 * (W - S - 48)


def test_evicted_rows_into_codes():
    """Prefill with its lse, the weights of its last queries, an eviction by them, and what stays as codes of an 8-bit cache that decoding reads."""
    B, H, G, d, T, keep, block = 3, 2, 4, 128, 300, 100, 32
    k, v, q = _tokens(1, B, H, G, T, d, torch.bfloat16, 7)
    lay = binding.layout_for(k)
    need = max(fk.attend_prefill_plan(lay, H * G, H, d, T, 32)[1].workspace_bytes, fk.attend_weights_plan(lay, H * G, H, d, T, 32)[1].workspace_bytes)
    ws = ref.with_workspace(lay, need)
    tail = q[:, :, :, T - 32:].contiguous()
    out, lse = torch.empty_like(tail), torch.empty(tail.shape[:4], device=DEV)
    w = torch.empty((1, B, H, T), device=DEV)
    kept = torch.empty((1, B, H, keep), dtype=torch.int32, device=DEV)
    assert fk.attend_prefill(tail, k, v, out, lse, lay, H * G, H, d, T, 32, BASE) == 0
    assert fk.attend_weights(tail, k, lse, w, lay, H * G, H, d, T, 32, rope_base=BASE) == 0
    torch.cuda.synchronize()
    lens = torch.full((B,), T, dtype=torch.int32, device=DEV)
    # lse as attention gives it, from turned keys and queries of 8 bits or more: a query's weights sum to 1 within what its scores may be off
    sc = ref.Scores(tail, k, lens, BASE)
    delta = float((sc.size * sc.seen).max()) * 2 * 2.0 ** -9 + T * 2.0 ** -24
    assert abs(float(w.double().sum()) / (B * H * G * 32) - 1) <= math.expm1(delta)
    n = 4 + keep + 16
    assert fk.evict(k, v, w, w, kept, lay, H, d, T, 4, 16, keep) == 0
    k8 = torch.zeros((1, B, H, n + 1, d), dtype=torch.int8, device=DEV)
    v8 = torch.zeros_like(k8)
    ks, vs = (torch.zeros((1, B, H, -(-(n + 1) // block)), device=DEV) for _ in range(2))
    L8, S = ref.layouts8(k8, ks, vs, block)
    assert fk.quantize(k, v, lay, 0, k8, v8, L8, S, 0, n, H, d) == 0
    new = _tokens(1, B, H, G, 1, d, torch.bfloat16, 9)
    at = torch.tensor([n, n, -1], dtype=torch.int32, device=DEV)                     # the last sequence gets no token
    assert fk.quantize(new[0], new[1], binding.layout_for(new[0]), 0, k8, v8, L8, S, 0, 1, H, d, code_rows=at) == 0
    lens = torch.tensor([n + 1, n + 1, n], dtype=torch.int32, device=DEV)
    ws8 = ref.with_workspace(L8, fk.attend_q8_plan(L8, fk.BF16, H * G, H, d, n + 1, 1)[1].workspace_bytes)
    out, lse = torch.empty_like(new[2]), torch.empty(new[2].shape[:4], device=DEV)
    assert fk.attend_q8(new[2], k8, v8, out, lse, L8, S, fk.BF16, H * G, H, d, n + 1, 1, lens, BASE) == 0
    torch.cuda.synchronize()
    rows = [ref.values(c, s, block) for c, s in ((k8, ks), (v8, vs))]
    _check(new[2], None, None, None, block, lens, BASE, out, lse, rows)
    # the codes are those of the rows that stayed (a token behind them may have doubled the last block's scale)
    for x, c, s in ((k, k8, ks), (v, v8, vs)):
        full = n // block * block
        codes, scales = ref.eight_bits(x[:, :, :, :full], "int8", block)
        assert torch.equal(c[:, :, :, :full], codes) and torch.equal(s[..., :n // block], scales)
        step = s.double()[..., torch.arange(n, device=DEV) // block, None]
        assert bool(((ref.values(c[:, :, :, :n], s, block) - x[:, :, :, :n].double()).abs() <= step).all())
    del ws, ws8


def test_weights_with_less_workspace():
    """Fewer parts of the queries: sums in another order, within the same bound; too little for one part is refused."""
    T, n, H, G, d = 700, 300, 1, 2, 128
    k = ref.cache((1, 1, H, T, d), torch.bfloat16, 1, DEV)
    q = (torch.randn((1, 1, H * G, n, d), generator=torch.Generator().manual_seed(1)) * 0.5).bfloat16().to(DEV)
    lens = torch.full((1,), T, dtype=torch.int32, device=DEV)
    _, l = ref.Scores(q, k, lens, BASE).softmax()
    lse = l.reshape(q.shape[:4]).float().contiguous()
    lay = binding.layout_for(k)
    p = fk.attend_weights_plan(lay, H * G, H, d, T, n)[1]
    assert p.n_split > 4
    one = p.workspace_bytes - p.n_split * T * 4
    start = torch.zeros((1, 1, H, T), device=DEV)
    for parts in (4, 2, 0):
        ws = ref.with_workspace(lay, one + parts * T * 4)
        w = torch.full((1, 1, H, T), math.nan, device=DEV)
        assert fk.attend_weights(q, k, lse, w, lay, H * G, H, d, T, n, rope_base=BASE) == 0
        torch.cuda.synchronize()
        _check_weights(q, k, lse, lens, BASE, w, start, False)
        del ws
    lay.workspace_bytes = one - 1
    with pytest.raises(fk.FreqKVError):
        fk.attend_weights(q, k, lse, w, lay, H * G, H, d, T, n, rope_base=BASE)
