"""Trigger schedule around freqkv_compress (Sec. 3.4): a bounded KV cache that compresses itself, and the
attention calls over it (chunk-wise for prefill, one token for decode; rotary embedding at read time).

Thin host logic only: it owns the K/V tensors, the workspace and `cur_len`, asks freqkv_plan for
the lengths, and calls freqkv_compress when the cache is full and more tokens arrive (the lazy
trigger that yields the paper's compression counts: none at 4K, 3 at 8K, ... 127 at 256K for a
4096-token window).  All arithmetic on cache contents happens inside libfreqkv.

CompressedKVCache(by_weight=True) evicts rows by the attention they got in the place of a compression;
QuantizedKVCache holds its rows in 8 bits.
"""
from __future__ import annotations

import torch

from . import binding as fk


class CompressedKVCache:
    def __init__(self, n_layers, batch, n_heads, head_dim, window, n_sink=4, retain_ratio=0.5,
                 dtype=torch.bfloat16, device="cuda", capacity=None, flags=0, stream=None,
                 n_q_heads=None, rope_base=10000.0, by_weight=False, n_recent=0):
        """by_weight: a trigger keeps, of the rows between the sinks and the n_recent latest, those that got the most attention since they came, as
        many as leave the cache as long as a compression would (every attention call then adds to self.weights [L, B, H, capacity])."""
        self.window, self.n_sink, self.retain_ratio = window, n_sink, retain_ratio
        self.n_heads, self.head_dim = n_heads, head_dim
        self.capacity = window if capacity is None else capacity
        shape = (n_layers, batch, n_heads, self.capacity, head_dim)
        self.k = torch.empty(shape, dtype=dtype, device=device)
        self.v = torch.empty(shape, dtype=dtype, device=device)
        self.cur_len = 0
        self.triggers = 0
        self.stream = stream
        self.layout = fk.layout_for(self.k, flags=flags)
        _, p = fk.plan(self.layout, n_heads, head_dim, window, window, n_sink, retain_ratio)
        self.plan = p
        self.n_q_heads = n_heads if n_q_heads is None else n_q_heads
        self.rope_base = rope_base
        # the near/far form (7) wants the least that the library accepts, the matrix forms run faster with more
        need = max(p.workspace_min_bytes if p.runs == 7 else p.workspace_bytes, 256)
        # a shorter cache may want more row chunks than a full one
        for n in range(self.capacity, 0, -max(64, self.capacity // 256)):
            rc, ap = fk.attend_plan(self.layout, self.n_q_heads, n_heads, head_dim, n, check=False)
            if rc == fk.OK:
                need = max(need, ap.workspace_bytes)
        rc, pp = fk.attend_prefill_plan(self.layout, self.n_q_heads, n_heads, head_dim, self.capacity, self.capacity,
                                        check=False)
        self.can_prefill = rc == fk.OK
        if self.can_prefill:
            need = max(need, pp.workspace_bytes)
            # chunks shorter than the cache are cut along the keys as well, which takes room of its own
            q_len = 1
            while q_len < self.capacity:
                _, pp = fk.attend_prefill_plan(self.layout, self.n_q_heads, n_heads, head_dim, self.capacity, q_len)
                need = max(need, pp.workspace_bytes)
                q_len *= 2
        self.by_weight, self.n_recent = by_weight, n_recent
        if by_weight:
            if not 0 <= n_recent < p.retained_len:
                raise ValueError("n_recent: of the %d rows that a trigger leaves behind the sinks at least one is chosen" % p.retained_len)
            self.weights = torch.zeros(shape[:4], dtype=torch.float32, device=device)
            self.kept = torch.full((*shape[:3], p.retained_len - n_recent), -1, dtype=torch.int32, device=device)
            for q_len in (1, self.capacity):
                need = max(need, fk.attend_weights_plan(self.layout, self.n_q_heads, n_heads, head_dim, self.capacity, q_len)[1].workspace_bytes)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device)
        self.layout.workspace = self.workspace.data_ptr()
        self.layout.workspace_bytes = self.workspace.numel()

    @property
    def free_after_trigger(self) -> int:
        return self.window - self.n_sink - self.plan.retained_len

    def compress(self) -> int:
        """One trigger (if the cache is full); returns the library status."""
        if self.by_weight:
            return self._evict()
        rc = fk.compress(self.k, self.v, self.layout, self.n_heads, self.head_dim, self.cur_len,
                         self.window, self.n_sink, self.retain_ratio, self.stream)
        if rc == fk.OK and self.cur_len >= self.window:
            _, p = fk.plan(self.layout, self.n_heads, self.head_dim, self.cur_len, self.window,
                           self.n_sink, self.retain_ratio)
            self.cur_len = p.new_len
            self.triggers += 1
        return rc

    def _evict(self) -> int:
        if self.cur_len < self.window:
            return fk.NOOP
        rc = fk.evict(self.k, self.v, self.weights, self.weights, self.kept, self.layout, self.n_heads, self.head_dim, self.cur_len,
                      self.n_sink, self.n_recent, self.kept.shape[3], stream=self.stream)
        self.cur_len = self.n_sink + self.plan.retained_len
        self.triggers += 1
        return rc

    def room(self) -> int:
        return self.window - self.cur_len

    def append(self, k_new: torch.Tensor, v_new: torch.Tensor) -> None:
        """Append [L, B, H, T, d] tokens, compressing whenever the cache is full and tokens remain."""
        T, t0 = k_new.shape[3], 0
        while t0 < T:
            if self.cur_len >= self.window:
                self.compress()
            take = min(T - t0, self.window - self.cur_len)
            self._write(k_new, v_new, t0, take)
            t0 += take

    def _write(self, k_new, v_new, t0: int, take: int) -> None:
        """Tokens t0 .. t0 + take - 1 behind the last row."""
        self.k[:, :, :, self.cur_len:self.cur_len + take] = k_new[:, :, :, t0:t0 + take]
        self.v[:, :, :, self.cur_len:self.cur_len + take] = v_new[:, :, :, t0:t0 + take]
        self.cur_len += take

    # ---- attention over [sinks | compressed rows | tokens since], positions = rows of the cache ----------

    def attend_decode(self, q: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
        """q [L, B, Hq, d]: the query of the token appended last (it sits in row cur_len - 1)."""
        out = torch.empty_like(q) if out is None else out
        lse = self._lse(q)
        fk.attend_decode(q, self.k, self.v, out, lse, self.layout, self.n_q_heads, self.n_heads, self.head_dim,
                         self.cur_len, -1, self.rope_base, self.stream)
        self._add_weights(q, lse, 1)
        return out

    def attend_prefill(self, q: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
        """q [L, B, Hq, T, d]: the queries of the T tokens appended last (rows cur_len - T .. cur_len - 1)."""
        out = torch.empty_like(q) if out is None else out
        lse = self._lse(q)
        fk.attend_prefill(q, self.k, self.v, out, lse, self.layout, self.n_q_heads, self.n_heads, self.head_dim,
                          self.cur_len, q.shape[3], self.rope_base, self.stream)
        self._add_weights(q, lse, q.shape[3])
        return out

    def _lse(self, q):
        return torch.empty(q.shape[:-1], dtype=torch.float32, device=q.device) if self.by_weight else None

    def _add_weights(self, q, lse, q_len: int) -> None:
        if self.by_weight:
            fk.attend_weights(q, self.k, lse, self.weights, self.layout, self.n_q_heads, self.n_heads, self.head_dim, self.cur_len, q_len,
                              accumulate=True, rope_base=self.rope_base, stream=self.stream)

    def prefill(self, k_new: torch.Tensor, v_new: torch.Tensor, q_new: torch.Tensor) -> torch.Tensor:
        """Chunk-wise prefill of Sec. 3.4: K/V/q of T new tokens ([L, B, H|Hq, T, d]); the tokens go into the
        cache in pieces that fit (a trigger whenever it is full and tokens remain) and every piece attends to
        the cache as it stands then.  Returns the attention outputs [L, B, Hq, T, d]."""
        T, t0 = k_new.shape[3], 0
        out = torch.empty_like(q_new)
        while t0 < T:
            if self.cur_len >= self.window:
                self.compress()
            take = min(T - t0, self.window - self.cur_len)
            self._write(k_new, v_new, t0, take)
            out[:, :, :, t0:t0 + take] = self.attend_prefill(q_new[:, :, :, t0:t0 + take].contiguous())
            t0 += take
        return out


class QuantizedKVCache(CompressedKVCache):
    """The same with rows of 8 bits: appended tokens are rounded to codes with a scale for every block_tokens of them, attention reads the codes, and a trigger
    compresses the rows that they stand for, in a buffer of the type `dtype` for stage_layers layers at a time.  The sinks, whose values no trigger may change,
    are kept as they came for that (n_sink rows), and rounded from these each time.  Queries, results and appended rows have the type `dtype`.
    The library works on `stream`, copies on the current one: they are the same, or the caller orders them."""

    def __init__(self, n_layers, batch, n_heads, head_dim, window, n_sink=4, retain_ratio=0.5, dtype=torch.bfloat16, device="cuda",
                 capacity=None, flags=0, stream=None, n_q_heads=None, rope_base=10000.0, code_dtype=torch.int8, block_tokens=64, stage_layers=4):
        self.window, self.n_sink, self.retain_ratio = window, n_sink, retain_ratio
        self.n_heads, self.head_dim = n_heads, head_dim
        self.capacity = window if capacity is None else capacity
        self.cur_len = self.triggers = 0
        self.stream = stream
        self.n_q_heads = n_heads if n_q_heads is None else n_q_heads
        self.rope_base = rope_base
        self.by_weight, self.can_prefill = False, True
        self.block_tokens, self.stage_layers = block_tokens, max(1, min(stage_layers, n_layers))
        self.q_dtype = {torch.bfloat16: fk.BF16, torch.float32: fk.F32}[dtype]
        shape = (n_layers, batch, n_heads, self.capacity, head_dim)
        self.k = torch.empty(shape, dtype=code_dtype, device=device)
        self.v = torch.empty(shape, dtype=code_dtype, device=device)
        blocks = (*shape[:3], -(-self.capacity // block_tokens))
        self.k_scale = torch.empty(blocks, dtype=torch.float32, device=device)
        self.v_scale = torch.empty(blocks, dtype=torch.float32, device=device)
        stage = (self.stage_layers, batch, n_heads, window, head_dim)
        self.stage_k = torch.empty(stage, dtype=dtype, device=device)
        self.stage_v = torch.empty(stage, dtype=dtype, device=device)
        sinks = (*shape[:3], n_sink, head_dim)
        self.sink_k = torch.empty(sinks, dtype=dtype, device=device)
        self.sink_v = torch.empty(sinks, dtype=dtype, device=device)
        self.layout = fk.layout_for(self.k)
        self.scales = fk.scales_for(self.k_scale, self.v_scale, block_tokens)
        self.stage_layout = fk.layout_for(self.stage_k, flags=flags)
        need = 256
        for n in {n_layers % self.stage_layers or self.stage_layers, self.stage_layers}:      # (the last layers may be fewer)
            self.stage_layout.n_layers = n
            _, p = fk.plan(self.stage_layout, n_heads, head_dim, window, window, n_sink, retain_ratio)
            need = max(need, p.workspace_min_bytes if p.runs == 7 else p.workspace_bytes)
        self.plan = p
        q_len = 1
        while q_len < 2 * self.capacity:
            for n in {min(q_len, self.capacity), self.capacity}:
                _, ap = fk.attend_q8_plan(self.layout, self.q_dtype, self.n_q_heads, n_heads, head_dim, n, min(q_len, self.capacity))
                need = max(need, ap.workspace_bytes)
            q_len *= 2
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device)
        for L in (self.layout, self.stage_layout):
            L.workspace, L.workspace_bytes = self.workspace.data_ptr(), self.workspace.numel()

    def compress(self) -> int:
        """One trigger (if the cache is full); returns the library status."""
        if self.cur_len < self.window:
            return fk.NOOP
        new_len, rc = self.n_sink + self.plan.retained_len, fk.OK
        for l0 in range(0, self.k.shape[0], self.stage_layers):
            at = slice(l0, min(l0 + self.stage_layers, self.k.shape[0]))
            k, v = self.k[at], self.v[at]
            n = k.shape[0]
            codes, scales = fk.layout_for(k), fk.scales_for(self.k_scale[at], self.v_scale[at], self.block_tokens)
            stage = self.stage_layout
            stage.n_layers = n
            fk.dequantize(k, v, codes, scales, 0, self.stage_k, self.stage_v, stage, 0, self.cur_len, self.n_heads, self.head_dim, self.stream)
            self.stage_k[:n, :, :, :self.n_sink] = self.sink_k[at]
            self.stage_v[:n, :, :, :self.n_sink] = self.sink_v[at]
            rc = fk.compress(self.stage_k, self.stage_v, stage, self.n_heads, self.head_dim, self.cur_len, self.window, self.n_sink,
                             self.retain_ratio, self.stream)
            fk.quantize(self.stage_k, self.stage_v, stage, 0, k, v, codes, scales, 0, new_len, self.n_heads, self.head_dim, stream=self.stream)
        self.cur_len = new_len
        self.triggers += 1
        return rc

    def _write(self, k_new, v_new, t0: int, take: int) -> None:
        fk.quantize(k_new, v_new, fk.layout_for(k_new), t0, self.k, self.v, self.layout, self.scales, self.cur_len, take, self.n_heads,
                    self.head_dim, stream=self.stream)
        sinks = min(self.n_sink - self.cur_len, take)
        if sinks > 0:
            self.sink_k[:, :, :, self.cur_len:self.cur_len + sinks] = k_new[:, :, :, t0:t0 + sinks]
            self.sink_v[:, :, :, self.cur_len:self.cur_len + sinks] = v_new[:, :, :, t0:t0 + sinks]
        self.cur_len += take

    def attend_decode(self, q: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
        out = torch.empty_like(q) if out is None else out
        return self._attend(q, out, 1)

    def attend_prefill(self, q: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
        out = torch.empty_like(q) if out is None else out
        return self._attend(q, out, q.shape[3])

    def _attend(self, q, out, q_len: int):
        fk.attend_q8(q, self.k, self.v, out, None, self.layout, self.scales, self.q_dtype, self.n_q_heads, self.n_heads, self.head_dim,
                     self.cur_len, q_len, rope_base=self.rope_base, stream=self.stream)
        return out
