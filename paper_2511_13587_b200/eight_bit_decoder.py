"""Decoder layers whose weights and activations are 8 bits wide, over a `BoundedCache`: what a program decoding long images or video runs in
the place of `vvs_verify`'s bf16 layers where their weights' bytes, or the products of its prompts, are what it waits for: for 18 rows a layer of 4096
columns takes 81 us in the place of 97, but one of 1280 columns, whose ten launches cost more than its bytes, 41 in the place of 18.

`EightBitDecoder` rounds a model's weights once, block by block (`vvs_weight_quant`).  A step takes a block's rows through all layers: norm with
the residual's addition into 8 bits, q, k and v, append and attention of the cache, 8 bits, output projection, norm, gate and up, SwiGLU
into 8 bits, down projection; behind the last layer the final norm, not rounded to 8 bits, is what an LM head takes.  The residual stream and
what lies between a product and the next rounding have the context's type.  The bookkeeping of the cache (`commit`, `make_room`, trees) is the
caller's, as for the cache alone.

Everything runs on the current stream into buffers of the decoder; nothing here waits for the device, and a step may be captured into a graph.
`python -m paper_2511_13587_b200.eight_bit_decoder` decodes a synthetic clip."""
from __future__ import annotations

import torch

from . import binding as vb
from .bounded_cache import BoundedCache, clip_positions


def quantise_weight(ctx: int, w: torch.Tensor):
    """[outputs, inputs] of the context's type -> what `vvs_block_matmul` takes."""
    outs, ins = w.shape
    codes = torch.empty((outs, ins), dtype=torch.float8_e4m3fn, device=w.device)
    scale = torch.empty((-(-outs // 128), -(-ins // 128)), dtype=torch.float32, device=w.device)
    vb.vvs_weight_quant(ctx, w, codes, scale)
    return vb.make_qweight(codes, scale)


class EightBitDecoder:
    def __init__(self, ctx: int, weights: dict, cache: BoundedCache, d_ff: int, rms_eps: float = 1e-5):
        """weights: 'norm_f' and 'layers', each with w_qkv [(n_heads + 2 n_kv_heads) * head_dim, d_model], w_o [d_model, n_heads * head_dim],
        w_gate, w_up [d_ff, d_model], w_down [d_model, d_ff], norm1, norm2 [d_model], of the context's type."""
        if len(weights["layers"]) != cache.n_layers:
            raise ValueError(f"{len(weights['layers'])} layers of weights for a cache of {cache.n_layers}")
        self.ctx, self.cache, self.d_ff, self.eps = ctx, cache, d_ff, rms_eps
        self.n_seqs, self.n_heads, self.head_dim = cache.n_seqs, cache.n_heads, cache.k.shape[-1]
        self.n_kv_heads, self.d_model = cache.k.shape[2], weights["norm_f"].numel()
        self.norm_f, self.layers = weights["norm_f"], []
        inner, width = self.n_heads * self.head_dim, (self.n_heads + 2 * self.n_kv_heads) * self.head_dim
        for w in weights["layers"]:
            for name, shape in (("w_qkv", (width, self.d_model)), ("w_o", (self.d_model, inner)), ("w_gate", (d_ff, self.d_model)),
                                ("w_up", (d_ff, self.d_model)), ("w_down", (self.d_model, d_ff)), ("norm1", (self.d_model,)), ("norm2", (self.d_model,))):
                if tuple(w[name].shape) != shape:
                    raise ValueError(f"{name}: expected {shape}, got {tuple(w[name].shape)}")
            # gate and up are one product: their rows side by side
            both = quantise_weight(ctx, torch.cat((w["w_gate"], w["w_up"])))
            self.layers.append(dict(qkv=quantise_weight(ctx, w["w_qkv"]), o=quantise_weight(ctx, w["w_o"]), both=both,
                                    down=quantise_weight(ctx, w["w_down"]), norm1=w["norm1"], norm2=w["norm2"]))
        most, dt, dev = cache.n_seqs * cache.max_rows, weights["norm_f"].dtype, weights["norm_f"].device
        self._room = {}
        for name, cols in (("stream", self.d_model), ("delta", self.d_model), ("features", self.d_model), ("qkv", width), ("attended", inner),
                           ("both", 2 * d_ff)):
            self._room[name] = torch.zeros((most, cols), dtype=dt, device=dev)
        for name, cols in (("x", self.d_model), ("a", inner), ("h", d_ff)):
            self._room[name] = (torch.zeros((most, cols), dtype=torch.float8_e4m3fn, device=dev),
                                torch.zeros((most * -(-cols // 128),), dtype=torch.float32, device=dev))

    def _coded(self, name: str, n: int):
        codes, scale = self._room[name]
        blocks = -(-codes.shape[1] // 128)
        return codes[:n], scale[:n * blocks].view(n, blocks)

    def step(self, x: torch.Tensor, pos: torch.Tensor, mass_rows: int = 1, row_count: torch.Tensor | None = None,
             visible: torch.Tensor | None = None) -> torch.Tensor:
        """x [n_seqs, rows, d_model] of a block (embeddings), pos int32 [axes, n_seqs, rows]: its features [n_seqs, rows, d_model] (a buffer of
        this object).  The rows lie behind the cache's fill until `cache.commit`.  Rows of x from row_count on go through norms and products with
        the others: their features mean nothing, and numbers there that are not finite are told of like any."""
        b, rows, d = x.shape
        if b != self.n_seqs or d != self.d_model or rows > self.cache.max_rows:
            raise ValueError(f"expected [{self.n_seqs}, up to {self.cache.max_rows}, {self.d_model}]")
        n, ctx, rope = b * rows, self.ctx, self.cache.rope(pos)
        stream, delta, qkv, attended, both = (self._room[name][:n] for name in ("stream", "delta", "qkv", "attended", "both"))
        cx, ca, ch = (self._coded(name, n) for name in ("x", "a", "h"))
        heads = (self.n_heads, self.n_kv_heads, self.n_kv_heads)
        stream.copy_(x.reshape(n, d))
        for i, w in enumerate(self.layers):
            if i == 0:
                vb.vvs_norm_quant(ctx, stream, w["norm1"], self.eps, *cx)
            else:
                vb.vvs_norm_quant(ctx, delta, w["norm1"], self.eps, *cx, residual=stream, sum_out=stream)
            vb.vvs_block_matmul(ctx, *cx, w["qkv"], qkv)
            q, k, v = qkv.view(b, rows, sum(heads), self.head_dim).split(heads, dim=2)
            out = attended.view(b, rows, self.n_heads, self.head_dim)
            self.cache.attend(i, self.cache.append(i, q, k, v, rope, row_count), out, mass_rows, row_count, visible)
            vb.vvs_rows_quant(ctx, attended, *ca)
            vb.vvs_block_matmul(ctx, *ca, w["o"], delta)
            vb.vvs_norm_quant(ctx, delta, w["norm2"], self.eps, *cx, residual=stream, sum_out=stream)
            vb.vvs_block_matmul(ctx, *cx, w["both"], both)
            vb.vvs_rows_quant(ctx, both[:, self.d_ff:], *ch, gate=both[:, :self.d_ff])
            vb.vvs_block_matmul(ctx, *ch, w["down"], delta)
        features = self._room["features"][:n]
        vb.vvs_norm_quant(ctx, delta, self.norm_f, self.eps, *cx, residual=stream, norm_out=features)
        return features.view(b, rows, d)

    def weight_bytes(self) -> int:
        return sum(t.numel() * t.element_size() for w in self.layers for name in ("qkv", "o", "both", "down") for t in w[name]._keep)


def random_weights(g: torch.Generator, n_layers: int, d_model: int, n_heads: int, n_kv_heads: int, head_dim: int, d_ff: int,
                   dtype: torch.dtype = torch.bfloat16) -> dict:
    def r(*shape):
        return (0.02 * torch.randn(shape, generator=g, device="cuda")).to(dtype)

    def one():
        return (1.0 + 0.1 * torch.randn((d_model,), generator=g, device="cuda")).to(dtype)
    layers = [dict(w_qkv=r((n_heads + 2 * n_kv_heads) * head_dim, d_model), w_o=r(d_model, n_heads * head_dim), w_gate=r(d_ff, d_model),
                   w_up=r(d_ff, d_model), w_down=r(d_model, d_ff), norm1=one(), norm2=one()) for _ in range(n_layers)]
    return dict(layers=layers, norm_f=one())


def demo(steps: int = 60, n_layers: int = 4, n_seqs: int = 2, d_model: int = 1280, n_heads: int = 20, n_kv_heads: int = 20, head_dim: int = 64,
         d_ff: int = 3456, budget: int = 448, rows: int = 9, height: int = 16, width: int = 16, seed: int = 7, verbose: bool = True) -> dict:
    """Decodes a clip of random embeddings: blocks of `rows` rows of which a random prefix is accepted.  Returns what it counted."""
    from vvs_synth.configs import ModelShape
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ctx = vb.vvs_create(vb.make_desc(ModelShape("clip", 0, 64, 0, 0, 0, 128), 1, 1))
    pairs = head_dim // 2
    axis = (torch.arange(pairs, device="cuda") * 3 // pairs).to(torch.int32)
    inv_freq = torch.pow(10000.0, -(torch.arange(pairs, device="cuda") % (pairs // 3 + 1)).float() / (pairs // 3 + 1))
    cache = BoundedCache(ctx, n_layers, n_seqs, n_heads, n_kv_heads, head_dim, budget, rows, inv_freq, axis)
    decoder = EightBitDecoder(ctx, random_weights(g, n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ff), cache, d_ff)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    finite = torch.ones((), dtype=torch.bool, device="cuda")
    for i in range(steps):
        if i == min(10, steps - 1):
            begin.record()
        cache.make_room()
        x = torch.randn((n_seqs, rows, d_model), generator=g, device="cuda").to(torch.bfloat16)
        features = decoder.step(x, clip_positions(cache.next_age, rows, height, width))
        finite &= features.isfinite().all()
        cache.commit(torch.randint(1, rows + 1, (n_seqs,), generator=g, device="cuda", dtype=torch.int32), rows)
    end.record()
    torch.cuda.synchronize()
    got = dict(tokens=cache.next_age.tolist(), fill=cache.fill.tolist(), evictions=cache.evictions, status=vb.vvs_device_status(ctx),
               finite=bool(finite), weight_bytes=decoder.weight_bytes(), ms_per_step=begin.elapsed_time(end) / max(1, steps - min(10, steps - 1)))
    vb.vvs_destroy(ctx)
    if verbose:
        print(got)
    return got


if __name__ == "__main__":
    demo()
