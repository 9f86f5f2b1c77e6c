"""A decoder's key / value cache in 8 bits that never grows beyond a bound: what a program decoding long images or video keeps in the
place of the bf16 cache of `vvs_verify`.

Per layer and step: `append` turns the block's queries and keys to their positions (time, row, column, ..) and puts keys and values behind the
cache, `attend` reads it and adds the weights that every key got.  `commit` moves the fill levels behind the accepted rows (a tree's rows on the
accepted path are put again, side by side, layer by layer, and keep the weights that `attend` gave them).  `make_room` brings every layer back to
the budget when a block could pass the capacity: the tokens of the least accumulated weight leave, the first and the last ones never.  Positions
are the caller's: a token keeps the ones it was turned to, whatever slot it lies in.  Sequences begin in slot 0: there is no padding on the left.

The library's kernels do the work on the current stream, a few small torch operations a step the bookkeeping; nothing here waits for the device.
`python -m paper_2511_13587_b200.bounded_cache` decodes a synthetic clip through it."""
from __future__ import annotations

import torch

from . import binding as vb


class BoundedCache:
    def __init__(self, ctx: int, n_layers: int, n_seqs: int, n_heads: int, n_kv_heads: int, head_dim: int, budget: int, max_rows: int,
                 inv_freq: torch.Tensor, axis: torch.Tensor, slack: int = 256, block: int = 64, n_sink: int = 4, n_recent: int = 64,
                 halves: bool = False, mass_decay: float = 1.0, dtype: torch.dtype = torch.bfloat16, device: str = "cuda"):
        """`budget` tokens stay after `make_room`; `slack` more may come before it has to run again; a block has at most `max_rows` rows.
        inv_freq float32 and axis int32 [pairs] as for `make_rope_axes`."""
        if min(n_layers, n_seqs, n_kv_heads, budget, max_rows) < 1 or slack < 0 or n_heads < 1 or n_heads % n_kv_heads:
            raise ValueError("layers, sequences, heads, budget and max_rows have to be positive, slack not negative, n_heads a multiple of n_kv_heads")
        if block not in (16, 32, 64, 128) or head_dim not in (64, 128):
            raise ValueError("a block has 16, 32, 64 or 128 slots, a head 64 or 128 elements")
        if n_sink < 0 or n_recent < 0 or n_sink + n_recent > budget:
            raise ValueError("n_sink + n_recent tokens do not fit the budget")
        if not 0.0 <= mass_decay < float("inf"):
            raise ValueError("mass_decay has to be finite and not negative")
        if -(-(budget + slack + max_rows) // block) * block > vb.VVS_QCACHE_EVICT_CAP:
            raise ValueError(f"budget + slack + max_rows pass the {vb.VVS_QCACHE_EVICT_CAP} slots that an eviction takes")
        self.ctx, self.n_layers, self.n_seqs, self.n_heads = ctx, n_layers, n_seqs, n_heads
        self.budget, self.max_rows, self.n_sink, self.n_recent, self.mass_decay = budget, max_rows, n_sink, n_recent, mass_decay
        self.inv_freq, self.axis, self.halves = inv_freq, axis, halves
        self.cap = -(-(budget + slack + max_rows) // block) * block
        z = lambda shape, dt: torch.zeros(shape, dtype=dt, device=device)
        shape = (n_layers, n_seqs, n_kv_heads, self.cap)
        self.k, self.v = z(shape + (head_dim,), torch.float8_e4m3fn), z(shape + (head_dim,), torch.float8_e4m3fn)
        self.k_scale, self.v_scale = (z((n_layers, n_seqs, n_kv_heads, self.cap // block), torch.float32) for _ in range(2))
        # weights and ages have two buffers: an eviction reads one and writes the other
        self.mass, self.age = z((2,) + shape, torch.float32), z((2,) + shape, torch.int32)
        self.kept = z((n_seqs, n_kv_heads, budget), torch.int32)
        self.fill, self.fill_next, self.next_age = (z((n_seqs,), torch.int32) for _ in range(3))
        self.rotated = z((n_seqs, max_rows, n_heads, head_dim), dtype)
        self.turn = 0                                          # which of the two buffers holds the weights and ages
        self.fill_most = 0                                     # no sequence's fill is above it
        self.evictions = 0
        self._rows = torch.arange(max_rows, device=device)
        self._picked = None                                    # of a tree that was put again: the block's rows, and their new places,
        self._picked_by = -1                                   # .. and the layer that was the first
        self._caches = [[self._cache(layer, turn) for layer in range(n_layers)] for turn in range(2)]
        self._unweighted = [self._cache(layer, None) for layer in range(n_layers)]

    def _cache(self, layer: int, turn: int | None):
        """Without a turn, keys and values alone: an append leaves weights and ages as they are."""
        more = () if turn is None else (self.mass[turn][layer], self.age[turn][layer])
        return vb.make_qcache(self.k[layer], self.v[layer], self.k_scale[layer], self.v_scale[layer], *more)

    def rope(self, pos: torch.Tensor):
        """pos int32 [axes, n_seqs, rows] of a block, for the layers' `append` calls."""
        return vb.make_rope_axes(self.inv_freq, self.axis, pos, self.halves)

    def append(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, rope, row_count: torch.Tensor | None = None) -> torch.Tensor:
        """A block's rows [n_seqs, rows, heads, head_dim], as the projection left them; returns the turned queries (a buffer of this object)."""
        if layer == self._picked_by:                           # (a block in the place of one that was put again and not committed)
            self._picked, self._picked_by = None, -1
        turned = self.rotated[:, :q.shape[1]]
        vb.vvs_quant_cache_append(self.ctx, self._caches[self.turn][layer], k, v, self.fill, rope=rope, q=q, q_out=turned, row_count=row_count,
                                  next_age=self.next_age)
        return turned

    def attend(self, layer: int, q: torch.Tensor, out: torch.Tensor, mass_rows: int = 1, row_count: torch.Tensor | None = None,
               visible: torch.Tensor | None = None) -> torch.Tensor:
        """The appended block over the cache; the first `mass_rows` rows (those known to stay: the forced ones) count for eviction."""
        vb.vvs_quant_cache_attend(self.ctx, self._caches[self.turn][layer], q, out, self.fill, row_count=row_count, visible=visible,
                                  mass_rows=mass_rows, mass_decay=self.mass_decay, max_len=min(self.cap, self.fill_most + q.shape[1]))
        return out

    def put_again(self, layer: int, k: torch.Tensor, v: torch.Tensor, rope, path: torch.Tensor, n_commit: torch.Tensor) -> None:
        """After a tree call and before `commit`: the rows path[b, :n_commit[b]] of the block lie side by side behind the cache.  Path and
        number are the same for all layers; `commit` moves the rows' weights along."""
        if self._picked is None:
            rows = self._rows[:path.shape[1]].expand(path.shape)
            self._picked_by = layer
            self._picked = torch.stack((torch.where(rows < n_commit.view(-1, 1), path, rows), rows))
        # (the places have their ages from the block's own append: that of the place, not of the row)
        vb.vvs_quant_cache_append(self.ctx, self._unweighted[layer], k, v, self.fill, rope=rope, row_count=n_commit, row_index=path,
                                  next_age=self.next_age)

    def commit(self, n_commit: torch.Tensor, most: int) -> None:
        """n_commit int32 [n_seqs]: rows of the block that stay, at most `most` of any sequence."""
        if self._picked is not None:
            # (places behind the last committed row keep what they have; the bounds are for rows out of range and blocks that did not fit,
            # which the append has left out and told of)
            mass = self.mass[self.turn]
            rows, places = (self._picked + self.fill.view(-1, 1)).clamp_(0, self.cap - 1)[:, None, :, None].expand((2,) + mass.shape[:3] + (-1,))
            mass.scatter_(3, places, mass.gather(3, rows))
            self._picked, self._picked_by = None, -1
        self.fill += n_commit
        self.next_age += n_commit
        self.fill_most += most

    def make_room(self) -> bool:
        """Call between steps: evicts if the next block might not fit.  Every layer keeps `budget` tokens of its own choice."""
        if self.fill_most + self.max_rows <= self.cap:
            return False
        other = 1 - self.turn
        for layer in range(self.n_layers):
            vb.vvs_quant_cache_evict(self.ctx, self._caches[self.turn][layer], self.fill, self.budget, self.n_sink, self.n_recent, self.next_age,
                                     self.mass[other][layer], self.age[other][layer], self.fill_next, self.kept)
        self.fill, self.fill_next, self.turn = self.fill_next, self.fill, other
        self.fill_most = self.budget
        self.evictions += 1
        return True


def clip_positions(first: torch.Tensor, rows: int, height: int, width: int) -> torch.Tensor:
    """(time, row, column) of `rows` tokens of a clip from token first[b] on: int32 [3, n_seqs, rows]."""
    t = first.view(-1, 1) + torch.arange(rows, device=first.device, dtype=torch.int32)
    return torch.stack((t // (height * width), t % (height * width) // width, t % width)).to(torch.int32).contiguous()


def demo(steps: int = 200, n_layers: int = 4, n_seqs: int = 2, n_heads: int = 16, n_kv_heads: int = 4, head_dim: int = 64, budget: int = 448,
         rows: int = 9, height: int = 16, width: int = 16, seed: int = 7, verbose: bool = True) -> dict:
    """Decodes a clip of random projections: blocks of `rows` rows of which a random prefix is accepted.  Returns what it counted."""
    from vvs_synth.configs import ModelShape
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ctx = vb.vvs_create(vb.make_desc(ModelShape("clip", 0, 64, 0, 0, 0, 128), 1, 1))
    pairs = head_dim // 2
    axis = (torch.arange(pairs, device="cuda") * 3 // pairs).to(torch.int32)
    inv_freq = torch.pow(10000.0, -(torch.arange(pairs, device="cuda") % (pairs // 3 + 1)).float() / (pairs // 3 + 1))
    cache = BoundedCache(ctx, n_layers, n_seqs, n_heads, n_kv_heads, head_dim, budget, rows, inv_freq, axis)
    out = torch.zeros((n_seqs, rows, n_heads, head_dim), dtype=torch.bfloat16, device="cuda")
    for _ in range(steps):
        cache.make_room()
        rope = cache.rope(clip_positions(cache.next_age, rows, height, width))
        for layer in range(n_layers):
            qkv = torch.randn((n_seqs, rows, n_heads + 2 * n_kv_heads, head_dim), generator=g, device="cuda").to(torch.bfloat16)
            q, k, v = qkv.split((n_heads, n_kv_heads, n_kv_heads), dim=2)
            cache.attend(layer, cache.append(layer, q, k, v, rope), out)
        cache.commit(torch.randint(1, rows + 1, (n_seqs,), generator=g, device="cuda", dtype=torch.int32), rows)
    got = dict(tokens=cache.next_age.tolist(), fill=cache.fill.tolist(), evictions=cache.evictions, status=vb.vvs_device_status(ctx),
               bytes=cache.k.numel() + cache.v.numel() + 4 * (cache.k_scale.numel() + cache.v_scale.numel()), finite=bool(out.isfinite().all()))
    vb.vvs_destroy(ctx)
    if verbose:
        print(got)
    return got


if __name__ == "__main__":
    demo()
