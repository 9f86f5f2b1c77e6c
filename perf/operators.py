"""The measured work of the 8-bit key / value cache and of what goes with it, through the public entry points of
`paper_2511_13587_b200.binding`, and the same operators in plain torch.

A case is a dict of plain values; `op` names the operator:

  rotate  `vvs_rotate_axes`: rotary positions with several axes on query and key heads
  append  `vvs_quant_cache_append`: a block's keys and values, rotated and rounded to e4m3 with one scale for each block of
          slots and head, go behind what a cache holds; the queries are rotated on the way
  attend  `vvs_quant_cache_attend`: attention of a block's rows over such a cache, and the weight that every key got
  evict   `vvs_quant_cache_evict`: the keys of the least accumulated weight leave, later ones move into their slots

Definitions.  The angle of pair i of row t is the 32-bit product pos[axis[i], t] * inv_freq[i].  A scale is the smallest
power of two (2^-60 at least) by which the block's largest magnitude is at most 448; behind rows that the block holds already
it only grows, and those rows are rounded again.  A row t of a block of n rows sees the slots first_slot .. cache_len - 1 and,
of the block, the rows its mask names (a chain: 0 .. t); rows from row_count on are zero.
"""
from __future__ import annotations

import math

import torch

own = False

HEADS = {"xl": (20, 20, 64), "7b": (32, 32, 128), "gqa": (32, 8, 128), "gqa8": (16, 2, 64), "tiny": (4, 4, 64)}
INF = float("inf")


# ---------------------------------------------------------------------------------------------
# the cases


def listed():
    def c(name, op, model, n_seqs, rows, **more):
        return dict(name=name, op=op, model=model, n_seqs=n_seqs, rows=rows, **more)
    return [
        # one image with guidance: the nine rows of a verified block, grid positions (row, column); latency is what counts
        c("rotate step xl", "rotate", "xl", 2, 9, f32=False, axes=2, halves=False, part=1.0),
        # prompts of four clips: time, height and width; a shared-head model that pairs its halves
        c("rotate clip prompt", "rotate", "gqa", 4, 1365, f32=False, axes=3, halves=True, part=1.0),
        # a float32 context, an odd number of rows, a quarter of the head unrotated
        c("rotate odd float32", "rotate", "tiny", 3, 77, f32=True, axes=2, halves=False, part=0.75),
        # the same verified block, into the cache of one image with guidance
        c("append step xl", "append", "xl", 2, 9, f32=False, axes=2, halves=False, block=64, cap=640, fill_lo=311, fill_hi=311),
        # a batch of sixteen images with guidance, fills all different
        c("append step 7b batch", "append", "7b", 32, 9, f32=False, axes=1, halves=False, block=64, cap=2432, fill_lo=70, fill_hi=2380),
        # prompts of eight clips into an empty cache, an odd number of rows
        c("append clip prompt", "append", "gqa", 8, 1301, f32=False, axes=3, halves=True, block=128, cap=1408, fill_lo=0, fill_hi=0),
        # one token of a float32 context: the smallest call
        c("attend token float32", "attend", "tiny", 3, 1, f32=True, block=16, cap=160, fill_lo=0, fill_hi=127, tree=False, mass_rows=0),
        # one image with guidance, its verified block, weights counted for eviction
        c("attend step xl", "attend", "xl", 2, 9, f32=False, block=64, cap=640, fill_lo=311, fill_hi=311, tree=False, mass_rows=9),
        # sixteen images with guidance late in a long image, the forced row's weights counted
        c("attend step 7b batch", "attend", "7b", 32, 9, f32=False, block=64, cap=2432, fill_lo=900, fill_hi=2380, tree=False, mass_rows=1),
        # candidate trees behind long clips, shared heads: 27 x 4 rows of queries over each cached head
        c("attend tree clip", "attend", "gqa", 2, 27, f32=False, block=128, cap=33024, fill_lo=30001, fill_hi=32768, tree=True, mass_rows=0),
        # a cache of one image with guidance brought back to its bound
        c("evict xl", "evict", "xl", 2, 0, block=64, cap=640, fill_lo=576, fill_hi=576, keep=448, sink=1, recent=64),
        # long clips
        c("evict clip", "evict", "gqa", 4, 0, block=128, cap=33024, fill_lo=32001, fill_hi=32768, keep=24576, sink=64, recent=2048),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(("rotate", "append", "attend", "attend", "evict"))
    model = rng.choice(tuple(HEADS))
    block = rng.choice((16, 32, 64, 128))
    heads, kv_heads, hd = HEADS[model]
    c = dict(op=op, model=model)
    if op == "rotate":
        c.update(n_seqs=_log_int(rng, 1, 32), rows=_log_int(rng, 1, 1400), f32=rng.random() < 0.3, axes=rng.randint(1, 4),
                 halves=rng.random() < 0.5, part=rng.choice((0.25, 0.5, 1.0, 1.0)))
        c["n_seqs"] = max(1, min(c["n_seqs"], 5000 // c["rows"]))
    elif op == "append":
        rows = _log_int(rng, 1, 1400)
        c.update(n_seqs=max(1, min(_log_int(rng, 1, 32), 10000 // rows)), rows=rows, f32=rng.random() < 0.25, axes=rng.randint(1, 3),
                 halves=rng.random() < 0.5, block=block)
        c["fill_lo"], c["fill_hi"] = sorted((rng.randint(0, 1000), rng.randint(0, 1000)))
        c["cap"] = -(-(c["fill_hi"] + rows + rng.randint(0, 200)) // block) * block
    elif op == "attend":
        tree = rng.random() < 0.4
        rows = _log_int(rng, 2, 32) if tree else _log_int(rng, 1, 64)
        fill = _log_int(rng, 1, 32768)
        n_seqs = max(1, min(_log_int(rng, 1, 32), int(1.5e8 / ((fill + rows) * kv_heads * hd)), int(2e8 / ((fill + rows) * heads * rows))))
        c.update(n_seqs=n_seqs, rows=rows, f32=rng.random() < 0.2, block=block, fill_lo=rng.randint(0, fill), fill_hi=fill, tree=tree,
                 mass_rows=rng.choice((0, 0, 1, rows)))
        c["cap"] = -(-(fill + rows + rng.randint(0, 200)) // block) * block
    else:
        fill = _log_int(rng, 40, 32768)
        n_seqs = max(1, min(_log_int(rng, 1, 32), int(1.2e8 / (fill * kv_heads * hd))))
        keep = rng.randint(max(1, fill // 3), fill)
        c.update(n_seqs=n_seqs, rows=0, block=block, fill_lo=rng.randint(fill // 2, fill), fill_hi=fill, keep=keep,
                 sink=rng.randint(0, keep // 8), recent=rng.randint(0, keep // 2))
        c["cap"] = -(-(fill + rng.randint(0, 200)) // block) * block
    return c


# ---------------------------------------------------------------------------------------------
# the inputs


class State:
    pass


def _scale_of(amax):
    """The smallest power of two, 2^-60 at least, by which `amax` is at most 448 = 0.875 * 2^9."""
    frac, exp = torch.frexp(amax)
    exp = torch.where(amax > 0, exp - 9 + (frac > 0.875).to(exp.dtype), -60)
    return torch.ldexp(torch.ones_like(amax), exp.clamp(min=-60))


def _frequencies(hd, axes, part):
    """Every axis has a share of the pairs, with a geometric ladder of its own."""
    n = max(axes, int(hd // 2 * part))
    axis = torch.arange(n) * axes // n
    first = torch.searchsorted(axis, torch.arange(axes))
    count = torch.bincount(axis, minlength=axes)
    place = (torch.arange(n) - first[axis]).float() / count[axis].float()
    return torch.pow(10000.0, -place).float().cuda(), axis.to(torch.int32).cuda()


def _positions(g, axes, n_seqs, rows, start):
    """Token t of a sequence that began at `start`: the text axis alone, or (time,) row and column of 24 x 24 grids."""
    t = start.view(-1, 1) + torch.arange(rows, device="cuda")
    if axes == 1:
        return t.to(torch.int32).view(1, n_seqs, rows).contiguous()
    parts = [t // 576, t % 576 // 24, t % 24, t]
    return torch.stack(parts[1:3] if axes == 2 else parts[:axes]).to(torch.int32).contiguous()


def prepare(case, seed):
    s = State()
    s.case = case
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    heads, kv_heads, hd = HEADS[case["model"]]
    b, t = case["n_seqs"], case["rows"]
    s.dtype = torch.float32 if case.get("f32") else torch.bfloat16

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def ints(lo, hi, shape):
        return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)

    channel = torch.exp(0.5 * normal(hd))                  # keys have channels larger than others
    if case["op"] in ("rotate", "append"):
        # what the QKV projection leaves: q, k and v heads of a row side by side
        qkv = normal(b, t, heads + 2 * kv_heads, hd)
        qkv[:, :, heads:heads + kv_heads] *= channel
        qkv = qkv.to(s.dtype)
        s.q, s.k, s.v = qkv.split((heads, kv_heads, kv_heads), dim=2)
        s.q_out = torch.zeros((b, t, heads, hd), dtype=s.dtype, device="cuda")
        s.inv_freq, s.axis = _frequencies(hd, case["axes"], case.get("part", 1.0))
    if case["op"] == "rotate":
        s.pos = _positions(g, case["axes"], b, t, ints(0, 4000, (b,)))
        s.k_out = torch.zeros((b, t, kv_heads, hd), dtype=s.dtype, device="cuda")
        return s
    cap, blk = case["cap"], case["block"]
    s.cache_len = ints(case["fill_lo"], case["fill_hi"], (b,))
    s.k_scale, s.v_scale, s.k_codes, s.v_codes = [], [], [], []
    for scales, codes, wide in ((s.k_scale, s.k_codes, channel), (s.v_scale, s.v_codes, 1.0)):
        x = normal(b, kv_heads, cap // blk, blk, hd) * wide
        x[:, :, :, 0] *= torch.exp(normal(b, kv_heads, cap // blk, 1))      # blocks have scales of their own
        sc = _scale_of(x.abs().amax(dim=(3, 4)))
        scales.append(sc)
        codes.append((x / sc[..., None, None]).to(torch.float8_e4m3fn).view(b, kv_heads, cap, hd))
        del x
    s.k_scale, s.v_scale, s.k_codes, s.v_codes = s.k_scale[0], s.v_scale[0], s.k_codes[0], s.v_codes[0]
    # accumulated weights have a few heavy keys; ages are those of a cache that has lost keys before
    s.mass = torch.exp(1.5 * normal(b, kv_heads, cap)) / 16.0
    s.next_age = s.cache_len + ints(0, 3000, (b,))
    lost = torch.sort(torch.rand((b, kv_heads, cap), generator=g, device="cuda"), dim=2).values * (s.next_age - s.cache_len).view(b, 1, 1)
    s.age = torch.arange(cap, device="cuda", dtype=torch.int32) + lost.to(torch.int32)
    s.cache = None
    if case["op"] == "append":
        s.pos = _positions(g, case["axes"], b, t, s.next_age)
        s.row_count = None
    elif case["op"] == "attend":
        s.q = (1.5 * normal(b, t, heads, hd)).to(s.dtype)
        s.out = torch.zeros((b, t, heads, hd), dtype=s.dtype, device="cuda")
        s.lse = torch.zeros((b, t, heads), device="cuda")
        s.visible = s.row_count = None
        if case["tree"]:
            # every node hangs below one of the six rows before it; a row sees itself and the rows on its way up
            seen = torch.zeros((b, t, t), dtype=torch.bool, device="cuda")
            seen[:, 0, 0] = True
            up = torch.randint(0, 6, (b, t), generator=g, device="cuda")
            at = torch.arange(b, device="cuda")
            for i in range(1, t):
                seen[:, i] = seen[at, (i - 1 - up[:, i]).clamp(min=0)]
                seen[:, i, i] = True
            s.visible = (seen.to(torch.int64) << torch.arange(t, device="cuda")).sum(-1).to(torch.uint32).view(torch.int32)
        else:
            s.row_count = ints(max(1, t // 2), t, (b,))
        s.first_slot = torch.minimum(ints(0, 40, (b,)), s.cache_len)     # sequences padded on the left
    else:
        s.mass_out, s.age_out = torch.zeros_like(s.mass), torch.full_like(s.age, -1)
        s.new_len = torch.zeros_like(s.cache_len)
        s.kept = torch.full((b, kv_heads, case["keep"]), -1, dtype=torch.int32, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------
# plain forms, in 32 bits; the cache and its bookkeeping are the program's own buffers, which hold the new state after a call


def _rotate(x, s):
    """x [B, T, H, hd] -> 32 bits, rotated."""
    x, n = x.float(), s.inv_freq.numel()
    angle = s.pos.float()[s.axis.long()].permute(1, 2, 0) * s.inv_freq              # [B, T, n]
    c, sn = torch.cos(angle).unsqueeze(2), torch.sin(angle).unsqueeze(2)
    turned, rest = x[..., :2 * n], x[..., 2 * n:]
    if s.case["halves"]:
        x0, x1 = turned[..., :n], turned[..., n:]
        return torch.cat((x0 * c - x1 * sn, x1 * c + x0 * sn, rest), dim=-1)
    x0, x1 = turned[..., 0::2], turned[..., 1::2]
    return torch.cat((torch.stack((x0 * c - x1 * sn, x1 * c + x0 * sn), dim=-1).flatten(-2), rest), dim=-1)


def _put(codes, scale, x, s):
    """x [B, T, H, hd] in 32 bits goes behind the cached rows, into the blocks that it reaches."""
    b, h, cap, hd = codes.shape
    blk, t = s.case["block"], x.shape[1]
    base = s.cache_len.long().view(b, 1)
    block = (base // blk + torch.arange((t + blk - 2) // blk + 1, device="cuda")).clamp(max=cap // blk - 1)     # [B, n]
    slot = block.unsqueeze(-1) * blk + torch.arange(blk, device="cuda")                                       # [B, n, blk]
    live, mine = slot < base.unsqueeze(-1), (slot >= base.unsqueeze(-1)) & (slot < base.unsqueeze(-1) + t)
    row = (slot - base.unsqueeze(-1)).clamp(0, t - 1)
    at = torch.arange(b, device="cuda").view(b, 1)
    new = torch.where(mine[..., None, None], x[at.unsqueeze(-1), row], 0.0).permute(0, 3, 1, 2, 4)            # [B, H, n, blk, hd]
    old_scale = torch.gather(scale, 2, block.unsqueeze(1).expand(b, h, -1))
    old = codes.view(b, h, cap // blk, blk, hd).view(torch.uint8)[at, :, block].view(codes.dtype).float().transpose(1, 2)
    fresh = _scale_of(new.abs().amax(dim=(3, 4)))
    grown = torch.where(live.any(-1).unsqueeze(1), torch.maximum(old_scale, fresh), fresh)
    grown = torch.where(mine.any(-1).unsqueeze(1), grown, old_scale)
    kept = torch.where(live.unsqueeze(1).unsqueeze(-1), old * (old_scale / grown)[..., None, None], old)
    out = torch.where(mine.unsqueeze(1).unsqueeze(-1), new / grown[..., None, None], kept).to(codes.dtype)
    codes.view(b, h, cap // blk, blk, hd).view(torch.uint8)[at, :, block] = out.transpose(1, 2).view(torch.uint8)
    scale.scatter_(2, block.unsqueeze(1).expand(b, h, -1), grown)


def _plain_append(s):
    b, t = s.q.shape[:2]
    _put(s.k_codes, s.k_scale, _rotate(s.k, s), s)
    _put(s.v_codes, s.v_scale, s.v.float(), s)
    slot = (s.cache_len.long().view(b, 1) + torch.arange(t, device="cuda")).unsqueeze(1).expand(b, s.k.shape[2], t)
    age = (s.next_age.view(b, 1) + torch.arange(t, device="cuda", dtype=torch.int32)).unsqueeze(1).expand(b, s.k.shape[2], t)
    return dict(q=_rotate(s.q, s).to(s.dtype), k_codes=s.k_codes, v_codes=s.v_codes, k_scale=s.k_scale, v_scale=s.v_scale,
                mass=s.mass.scatter_(2, slot, 0.0), age=s.age.scatter_(2, slot, age))


def _seen(s, t, n_keys):
    """[B, T, n_keys]: what a row sees."""
    case, b = s.case, s.cache_len.numel()
    slot = torch.arange(n_keys, device="cuda").view(1, 1, -1)
    length, row = s.cache_len.view(b, 1, 1), torch.arange(t, device="cuda").view(1, t, 1)
    at = slot - length
    if case["tree"]:
        inside = (at >= 0) & (at < t) & ((s.visible.view(b, t, 1).long() >> at.clamp(0, 31)) & 1).bool()
        return ((slot < length) & (slot >= s.first_slot.view(b, 1, 1))) | inside
    inside = (at >= 0) & (at <= row)
    return (((slot < length) & (slot >= s.first_slot.view(b, 1, 1))) | inside) & (row < s.row_count.view(b, 1, 1))


def _plain_attend(s):
    case = s.case
    b, t, heads, hd = s.q.shape
    kv_heads, blk = s.k_codes.shape[1], case["block"]
    n = -(-(case["fill_hi"] + t) // blk) * blk
    group = heads // kv_heads
    k = s.k_codes[:, :, :n].float() * s.k_scale[:, :, :n // blk].repeat_interleave(blk, dim=2).unsqueeze(-1)
    v = s.v_codes[:, :, :n].float() * s.v_scale[:, :, :n // blk].repeat_interleave(blk, dim=2).unsqueeze(-1)
    q = s.q.float().view(b, t, kv_heads, group, hd).permute(0, 2, 3, 1, 4).reshape(b, kv_heads, group * t, hd)
    score = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(hd))
    seen = _seen(s, t, n).view(b, 1, 1, t, n)
    score = score.view(b, kv_heads, group, t, n).masked_fill(~seen, -INF)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -INF, 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    out = torch.matmul(p.view(b, kv_heads, group * t, n), v).view(b, kv_heads, group, t, hd)
    out = out.permute(0, 3, 1, 2, 4).reshape(b, t, heads, hd).to(s.dtype)
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 3, 1, 2).reshape(b, t, heads)
    if not case["mass_rows"]:
        return dict(out=out, lse=lse)
    s.mass[:, :, :n] += p[:, :, :, :case["mass_rows"]].sum(dim=(2, 3))
    return dict(out=out, lse=lse, mass=s.mass)


def _survivors(s):
    """kept [B, H, keep]: the slot that each kept slot's row comes from, -1 behind the last; and the new fill."""
    keep, cap = s.case["keep"], s.mass.shape[2]
    b = s.cache_len.numel()
    slot = torch.arange(cap, device="cuda").view(1, 1, cap)
    length, end = s.cache_len.view(b, 1, 1), s.next_age.view(b, 1, 1)
    valid = slot < length
    guarded = (s.age < s.case["sink"]) | (s.age >= end - s.case["recent"])
    worth = torch.where(valid, torch.where(guarded, INF, s.mass), -INF)
    order = torch.sort(worth, dim=2, descending=True, stable=True).indices[:, :, :keep]
    stays = torch.zeros_like(valid.expand_as(s.mass)).scatter(2, order, True) & valid
    hole = ~stays[:, :, :keep]
    mover = stays & (slot >= keep)
    movers = torch.sort((~mover).to(torch.int32), dim=2, stable=True).indices
    rank = (torch.cumsum(hole.to(torch.int64), dim=2) - 1).clamp(min=0)
    source = torch.where(hole, torch.gather(movers, 2, rank), slot[:, :, :keep])
    new_len = torch.clamp(s.cache_len, max=keep)
    kept = torch.where((slot[:, :, :keep] < new_len.view(b, 1, 1)) & valid[:, :, :keep], source, -1)
    return kept.to(torch.int32), new_len


def _moved(codes, scale, kept, s):
    """The moves: a block's scale grows to the largest that its new rows come with."""
    b, h, cap, hd = codes.shape
    blk, keep = s.case["block"], s.case["keep"]
    slot = torch.arange(keep, device="cuda")
    moves = (kept >= 0) & (kept != slot)
    source = kept.clamp(min=0).long()
    came = torch.gather(scale, 2, source // blk)
    new = scale.scatter_reduce(2, (slot // blk).expand(b, h, keep), torch.where(moves, came, 0.0), "amax")
    ratio = (scale / new).repeat_interleave(blk, dim=2).unsqueeze(-1)
    out = codes.float() * ratio
    ratio_in = (came / torch.gather(new, 2, (slot // blk).expand(b, h, keep))).unsqueeze(-1)
    arrived = torch.gather(codes.view(torch.uint8), 2, source.unsqueeze(-1).expand(b, h, keep, hd)).view(codes.dtype).float() * ratio_in
    out[:, :, :keep] = torch.where(moves.unsqueeze(-1), arrived, out[:, :, :keep])
    codes.copy_(out)
    scale.copy_(new)


def _plain_evict(s):
    kept, new_len = _survivors(s)
    b, h, cap = s.mass.shape
    _moved(s.k_codes, s.k_scale, kept, s)
    _moved(s.v_codes, s.v_scale, kept, s)
    live = kept >= 0
    mass, age = torch.zeros_like(s.mass), torch.full_like(s.age, -1)
    source = kept.clamp(min=0).long()
    mass[:, :, :kept.shape[2]] = torch.where(live, torch.gather(s.mass, 2, source), 0.0)
    age[:, :, :kept.shape[2]] = torch.where(live, torch.gather(s.age, 2, source), -1)
    return dict(kept=kept, new_len=new_len, k_codes=s.k_codes, v_codes=s.v_codes, k_scale=s.k_scale, v_scale=s.v_scale, mass=mass, age=age)


def _plain(s):
    if s.case["op"] == "rotate":
        return dict(q=_rotate(s.q, s).to(s.dtype), k=_rotate(s.k, s).to(s.dtype))
    return {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[s.case["op"]](s)


# ---------------------------------------------------------------------------------------------
# the framework's calls

_contexts = {}


def _context(dtype):
    """A decoding program has one context; these operators need its storage type and its status word."""
    from paper_2511_13587_b200 import binding as vb
    from vvs_synth.configs import DTYPE_BF16, DTYPE_FP32, ModelShape
    if dtype not in _contexts:
        shape = ModelShape("cache", 0, 64, 0, 0, 0, 128, dtype=DTYPE_FP32 if dtype == torch.float32 else DTYPE_BF16)
        _contexts[dtype] = vb, vb.vvs_create(vb.make_desc(shape, 1, 1))
    return _contexts[dtype]


def _own(s):
    vb, ctx = _context(s.dtype)
    case = s.case
    if case["op"] in ("rotate", "append"):
        rope = vb.make_rope_axes(s.inv_freq, s.axis, s.pos, halves=case["halves"])
    if case["op"] == "rotate":
        vb.vvs_rotate_axes(ctx, rope, s.q, s.q_out, s.k, s.k_out)
        return dict(q=s.q_out, k=s.k_out)
    if s.cache is None:
        s.cache = vb.make_qcache(s.k_codes, s.v_codes, s.k_scale, s.v_scale, s.mass, s.age)
    if case["op"] == "append":
        vb.vvs_quant_cache_append(ctx, s.cache, s.k, s.v, s.cache_len, rope=rope, q=s.q, q_out=s.q_out, next_age=s.next_age)
        return dict(q=s.q_out, k_codes=s.k_codes, v_codes=s.v_codes, k_scale=s.k_scale, v_scale=s.v_scale, mass=s.mass, age=s.age)
    if case["op"] == "attend":
        vb.vvs_quant_cache_attend(ctx, s.cache, s.q, s.out, s.cache_len, row_count=s.row_count, first_slot=s.first_slot,
                                  visible=s.visible, lse=s.lse, mass_rows=case["mass_rows"], max_len=case["fill_hi"] + case["rows"])
        return dict(out=s.out, lse=s.lse, mass=s.mass) if case["mass_rows"] else dict(out=s.out, lse=s.lse)
    vb.vvs_quant_cache_evict(ctx, s.cache, s.cache_len, case["keep"], case["sink"], case["recent"], s.next_age, s.mass_out, s.age_out,
                             s.new_len, s.kept)
    return dict(kept=s.kept, new_len=s.new_len, k_codes=s.k_codes, v_codes=s.v_codes, k_scale=s.k_scale, v_scale=s.v_scale,
                mass=s.mass_out, age=s.age_out)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    heads, kv_heads, hd = HEADS[case["model"]]
    b, t = case["n_seqs"], case["rows"]
    es = 4 if case.get("f32") else 2
    if case["op"] == "rotate":
        n = b * t * (heads + kv_heads) * hd
        return {"bytes": 2 * n * es + b * t * case["axes"] * 4, "flops": 3 * n}
    if case["op"] == "append":
        n_q, n_kv = b * t * heads * hd, b * t * kv_heads * hd
        return {"bytes": 2 * n_q * es + 2 * n_kv * (es + 1) + b * t * kv_heads * 8 + b * t * case["axes"] * 4, "flops": 3 * (n_q + n_kv) + 4 * n_kv}
    fill = (case["fill_lo"] + case["fill_hi"]) / 2
    if case["op"] == "attend":
        keys = b * kv_heads * (fill + t)
        n_bytes = keys * (2 * hd + 8 / case["block"] + (8 if case["mass_rows"] else 0)) + 2 * b * t * heads * hd * es + b * t * heads * 4
        return {"bytes": n_bytes, "flops": 4.0 * b * heads * t * (fill + t / 2) * hd}
    # masses and ages read and written; of the rows that stay, those behind `keep` move (weights say nothing of a slot's place)
    goes = max(0.0, fill - case["keep"])
    moves = goes * min(case["keep"], fill) / max(1.0, fill)
    n = b * kv_heads
    return {"bytes": n * (fill * 8 + min(case["keep"], fill) * 12 + moves * 4 * hd), "flops": n * fill}


# ---------------------------------------------------------------------------------------------
# from the definitions, in 64 bits


def _exact_rotate(x, s):
    """Complex numbers of modulus one in the place of the pairs' matrices."""
    x, n = x.double(), s.inv_freq.numel()
    angle = (s.pos[s.axis.long()].permute(1, 2, 0).float() * s.inv_freq).double()     # the operator's angle is a 32-bit number
    turn = torch.polar(torch.ones_like(angle), angle).unsqueeze(2)
    out = x.clone()
    first, second = (slice(0, n), slice(n, 2 * n)) if s.case["halves"] else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _e4m3(x):
    """64-bit values to the nearest e4m3 value, ties to the even code: steps of 2^-3 of the leading power, 2^-9 at least."""
    step = torch.ldexp(torch.ones_like(x), torch.frexp(x).exponent.clamp(min=-5) - 4)
    return torch.round(x / step) * step


def _power(amax):
    e = torch.ceil(torch.log2(amax / 448.0)).clamp(min=-60)
    return torch.ldexp(torch.ones_like(amax), e.to(torch.int32))


def _exact_put(codes, scale, x, s):
    codes, scale, blk = codes.double(), scale.double(), s.case["block"]
    for i, base in enumerate(s.cache_len.tolist()):
        end = base + x.shape[1]
        for n in range(base // blk, -(-end // blk)):
            lo, hi = max(base, n * blk), min(end, (n + 1) * blk)
            rows = x[i, lo - base:hi - base].transpose(0, 1)                          # [H, rows, hd]
            sc = _power(rows.abs().amax(dim=(1, 2)))
            if n * blk < base:
                sc = torch.maximum(sc, scale[i, :, n])
                codes[i, :, n * blk:base] = _e4m3(codes[i, :, n * blk:base] * (scale[i, :, n] / sc).view(-1, 1, 1))
            codes[i, :, lo:hi] = _e4m3(rows / sc.view(-1, 1, 1))
            scale[i, :, n] = sc
    return codes, scale


def _exact_attend(s):
    case = s.case
    b, t, heads, hd = s.q.shape
    kv_heads, blk = s.k_codes.shape[1], case["block"]
    group = heads // kv_heads
    out = torch.zeros((b, t, heads, hd), dtype=torch.float64, device="cuda")
    lse = torch.full((b, t, heads), -INF, dtype=torch.float64, device="cuda")
    mass = s.mass.double()
    counts = [t] * b if s.row_count is None else s.row_count.tolist()
    for i, (length, n, first) in enumerate(zip(s.cache_len.tolist(), counts, s.first_slot.tolist())):
        keys = length + n
        at = torch.arange(keys, device="cuda")
        for h in range(kv_heads):
            k = s.k_codes[i, h, :keys].double() * s.k_scale[i, h, at // blk].double().view(-1, 1)
            v = s.v_codes[i, h, :keys].double() * s.v_scale[i, h, at // blk].double().view(-1, 1)
            mine = slice(h * group, (h + 1) * group)
            q = s.q[i, :n, mine].double()                                            # [n, group, hd]
            score = torch.einsum("tgd,kd->tgk", q, k) / math.sqrt(hd)
            sees = (at >= first) & (at < length)
            sees = sees.expand(n, keys).clone()
            for r in range(n):
                if s.visible is None:
                    sees[r, length:length + r + 1] = True
                else:
                    bits = int(s.visible_host[i][r])
                    sees[r, length:] = torch.tensor([bool(bits >> j & 1) for j in range(n)], device="cuda")
            score = score.masked_fill(~sees.view(n, 1, keys), -INF)
            p = torch.nan_to_num(torch.softmax(score, dim=-1))
            out[i, :n, mine] = torch.einsum("tgk,kd->tgd", p, v)
            lse[i, :n, mine] = torch.logsumexp(score, dim=-1)
            mass[i, h, :keys] += p[:case["mass_rows"]].sum(dim=(0, 1))
    return dict(out=out, lse=lse, mass=mass) if case["mass_rows"] else dict(out=out, lse=lse)


def _exact_evict(s):
    """One head of one sequence at a time, on the host."""
    case = s.case
    keep, blk = case["keep"], case["block"]
    b, h, cap = s.mass.shape
    mass, age = s.mass.double().cpu(), s.age.cpu()
    mass_out = torch.zeros_like(mass)
    k_codes, v_codes, k_scale, v_scale = (x.double() for x in (s.k_codes, s.v_codes, s.k_scale, s.v_scale))
    for i, (length, end) in enumerate(zip(s.cache_len.tolist(), s.next_age.tolist())):
        for j in range(h):
            m, a = mass[i, j, :length].tolist(), age[i, j, :length].tolist()
            if length <= keep:
                mass_out[i, j, :length] = mass[i, j, :length]
                continue
            rank = sorted(range(length), key=lambda x: (not (a[x] < case["sink"] or a[x] >= end - case["recent"]), -m[x]
                                                        if not (a[x] < case["sink"] or a[x] >= end - case["recent"]) else 0.0, x))
            stays = set(rank[:keep])
            source = list(range(keep))
            movers = iter(sorted(x for x in stays if x >= keep))
            moved = []
            for x in range(keep):
                if x not in stays:
                    source[x] = next(movers)
                    moved.append(x)
            mass_out[i, j, :keep] = mass[i, j, source]
            if not moved:
                continue
            to, origin = torch.tensor(moved, device="cuda"), torch.tensor([source[x] for x in moved], device="cuda")
            for codes, scale in ((k_codes[i, j], k_scale[i, j]), (v_codes[i, j], v_scale[i, j])):
                came, rows, before = scale[origin // blk], codes[origin], scale.clone()
                scale.scatter_reduce_(0, to // blk, came, "amax")
                codes.copy_(_e4m3(codes * (before / scale).repeat_interleave(blk).view(-1, 1)))
                codes[to] = _e4m3(rows * (came / scale[to // blk]).view(-1, 1))
    return dict(kept=None, new_len=None, k_codes=k_codes, v_codes=v_codes, k_scale=k_scale, v_scale=v_scale, mass=mass_out, age=None)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotate":
        return dict(q=_exact_rotate(s.q, s), k=_exact_rotate(s.k, s))
    if case["op"] == "append":
        k_codes, k_scale = _exact_put(s.k_codes, s.k_scale, _exact_rotate(s.k, s), s)
        v_codes, v_scale = _exact_put(s.v_codes, s.v_scale, s.v.double(), s)
        mass = s.mass.double()
        for i, base in enumerate(s.cache_len.tolist()):
            mass[i, :, base:base + case["rows"]] = 0.0
        return dict(q=_exact_rotate(s.q, s), k_codes=k_codes, v_codes=v_codes, k_scale=k_scale, v_scale=v_scale, mass=mass, age=None)
    if case["op"] == "attend":
        if case["n_seqs"] * HEADS[case["model"]][1] > 1200:
            return None
        s.visible_host = None if s.visible is None else (s.visible.long() & 0xFFFFFFFF).tolist()
        return _exact_attend(s)
    return _exact_evict(s)
