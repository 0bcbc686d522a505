"""Cases of the paged 8-bit serving operators: what a server that decodes image
tokens for many requests calls between its projections, one step after the other.

  slots    block tables, slot maps, row positions and row offsets from request lengths
  axes     rotary positions with several axes (time, height, width) on queries and keys
  append   new keys and values into the 8-bit cache, one scale for each block of
           tokens and head
  attend   causal attention of each request's newest rows over that cache
  sample   a token of every row's logits: temperature, top-k, top-p, min-p, given uniforms

The cache: keys [n_blocks][n_kv_heads][block][head_dim] and values
[n_blocks][n_kv_heads][head_dim][block] as e4m3 codes, and one exponent byte s for
each block and head (its codes stand for code * 2^(s - 127)).  A request's token p
lies at offset p % block of the cache block that its table names for p // block.

Sizes are those of the decoders in synth/ (1B, 7B and 8B class in bf16, the tiny
one in fp32) with prompts and image grids of their workloads, and longer contexts
and larger batches of the same kind.
"""
import math
import random

import numpy as np
import torch

own = False

# heads, kv heads, head dim, image codes, dtype
WIDTHS = {"tiny": (4, 4, 64, 1024, "f32"), "1b": (16, 16, 128, 16384, "bf16"), "7b": (32, 32, 128, 8192, "bf16"),
          "8b": (32, 8, 128, 32768, "bf16")}
THETA = 1e4
CODE_MAX = 448.0  # largest e4m3 value
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases
def _slots(name, B, held, fresh, block):
    return {"name": name, "op": "slots", "B": B, "held": held, "fresh": fresh, "block": block}


def _axes(name, width, T, dtype):
    return {"name": name, "op": "axes", "width": width, "T": T, "dtype": dtype}


def _append(name, width, B, held, fresh, block, dtype):
    return {"name": name, "op": "append", "width": width, "B": B, "held": held, "fresh": fresh, "block": block,
            "dtype": dtype}


def _attend(name, width, B, held, fresh, block, dtype):
    return {"name": name, "op": "attend", "width": width, "B": B, "held": held, "fresh": fresh, "block": block,
            "dtype": dtype}


def _sample(name, R, V, top_k, top_p, min_p, temperature):
    return {"name": name, "op": "sample", "R": R, "V": V, "top_k": top_k, "top_p": top_p, "min_p": min_p,
            "temperature": temperature}


def listed():
    return [
        # a decode step of 64 requests, one token each
        _slots("slots-step", 64, 4352, 1, 64),
        # a prefill step of many requests with prompts of ragged lengths
        _slots("slots-prompts", 2048, 4096, 64, 32),
        # a row of the tiny fp32 decoder's image, all latency
        _axes("axes-row-f32", "tiny", 24, "f32"),
        # the prompts and images of a prefill step at the 8B widths, all bandwidth
        _axes("axes-prompts-8b", "8b", 16384, "bf16"),
        # a decode step: one token of 64 requests into partly filled blocks
        _append("append-step-8b", "8b", 64, 4352, 1, 64, "bf16"),
        # a prefill step of ragged prompts and images
        _append("append-prompts-8b", "8b", 16, 1, 2048, 64, "bf16"),
        # one request, one token, in the middle of a 24x24 image of the 1B decoder
        _attend("attend-token-1b", "1b", 1, 411, 1, 32, "bf16"),
        # single tokens of 64 requests of ragged lengths: the cache is read once, all bandwidth
        _attend("attend-tokens-8b", "8b", 64, 16384, 1, 64, "bf16"),
        # verify rounds: a drafted 64-token row of each of eight 64x64 images, grouped KV heads
        _attend("attend-rows-8b", "8b", 8, 4288, 64, 64, "bf16"),
        # the fp32 decoder's verify rounds: odd lengths, small heads
        _attend("attend-rows-f32", "tiny", 4, 1063, 33, 16, "f32"),
        # the next code of four images of the 1B decoder
        _sample("sample-1b", 4, 16384, 2000, 0.95, 0.0, 1.0),
        # rows of eight 8B images, a request's own settings in every row, no top-k in half of them
        _sample("sample-rows-8b", 512, 32768, -1, -1.0, -1.0, -1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("slots", "axes", "append", "append", "attend", "attend", "attend", "attend", "sample", "sample"))
    if op == "slots":
        c = _slots("", _log_int(rng, 1, 2048), _log_int(rng, 1, 16384), _log_int(rng, 1, 64), rng.choice((16, 32, 64, 128)))
    elif op == "axes":
        c = _axes("", rng.choice(("tiny", "1b", "7b", "8b")), _log_int(rng, 1, 8192), rng.choice(("f32", "bf16", "bf16")))
    elif op == "append":
        fresh = rng.choice((1, _log_int(rng, 2, 128), _log_int(rng, 2, 2048)))
        B = _log_int(rng, 1, max(1, min(128, 16384 // fresh)))
        c = _append("", rng.choice(("tiny", "1b", "8b")), B, _log_int(rng, 1, 4096), fresh, rng.choice((16, 32, 64, 128)),
                    rng.choice(("f32", "bf16", "bf16")))
    elif op == "attend":
        width = rng.choice(("tiny", "1b", "7b", "8b", "8b"))
        heads, kv, D = WIDTHS[width][:3]
        fresh = rng.choice((1, 1, _log_int(rng, 2, 16), _log_int(rng, 17, 160)))
        B = _log_int(rng, 1, 64)
        # neither the cache nor the products go past half of the largest listed cases'
        most = min(32 * 16384 * 8 * 128 // (B * kv * D), 4 * 4352 * 64 * 32 * 128 // (B * fresh * heads * D), 16384)
        held = _log_int(rng, 1, max(2, most))
        c = _attend("", width, B, held, fresh, rng.choice((16, 32, 64, 64, 128)), rng.choice(("f32", "bf16", "bf16")))
    else:
        V = rng.choice((1024, 8192, 16384, 32768, _log_int(rng, 33, 65536)))
        if rng.random() < 0.4:
            c = _sample("", _log_int(rng, 1, 256), V, -1, -1.0, -1.0, -1.0)
        else:
            c = _sample("", _log_int(rng, 1, 256), V, rng.choice((0, 1, _log_int(rng, 2, max(3, V // 2)))),
                        rng.choice((1.0, 0.9, 0.95, 0.5)), rng.choice((0.0, 0.02, 0.1)), rng.choice((0.0, 0.7, 1.0, 1.3)))
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs
class State:
    pass


def _generator(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1009 + stream)
    return g


def _normal(shape, seed, stream, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=_generator(seed, stream))


def _lengths(case):
    """Tokens held and new tokens of every request: ragged, the case's own (not the seed's), so that its work is known."""
    rng = random.Random(case["B"] * 7919 + case["held"] * 31 + case["fresh"])
    B, most, fresh = case["B"], case["held"], case["fresh"]
    held = [most] + [rng.randint(most // 4, most) for _ in range(B - 1)]
    new = [fresh] + [fresh if fresh == 1 or rng.random() < 0.5 else rng.randint(0, fresh) for _ in range(B - 1)]
    return held, new


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _layout(case, seed):
    """Request lengths and a table of blocks in shuffled order, as a server's step has them."""
    s = State()
    held, new = _lengths(case)
    T = case["block"]
    lens = [h + n for h, n in zip(held, new)]
    s.block, s.B = T, case["B"]
    s.width = max(1, max(-(-x // T) for x in lens))
    s.n_rows = sum(new)
    s.max_q, s.max_len = max(new), max(lens)
    blocks = [-(-x // T) for x in lens]
    s.n_blocks = sum(blocks) + 3
    s.held, s.new, s.lens = _int(held), _int(new), _int(lens)
    s.cu = _int(np.concatenate([[0], np.cumsum(new)]).tolist())
    order = torch.randperm(s.n_blocks, generator=_generator(seed, 1), device="cuda").to(torch.int32)
    first = _int(np.concatenate([[0], np.cumsum(blocks)[:-1]]).tolist())
    col = torch.arange(s.width, device="cuda", dtype=torch.int32)
    used = col[None] < _int(blocks)[:, None]
    at = (first[:, None] + col[None]).clamp(max=s.n_blocks - 1).long()
    s.table = torch.where(used, order[at], torch.full_like(at, -1, dtype=torch.int32)).contiguous()
    s.seq, s.pos = _rows(s.cu, s.held, s.n_rows)
    s.slots = (s.table[s.seq, s.pos // T] * T + s.pos % T).to(torch.int32)
    return s


def _rows(cu, held, n_rows):
    """Request and position of every new row."""
    r = torch.arange(n_rows, device="cuda")
    seq = torch.searchsorted(cu[1:].contiguous().long(), r, right=True)
    return seq, r - cu[seq] + held[seq]


def _exponent(amax):
    """Smallest s >= 1 with amax <= 448 * 2^(s - 127), as int32 (frexp: 448 = 0.875 * 2^9)."""
    m, x = torch.frexp(amax)
    return torch.where(amax > 0, (x - 9 + (m > 0.875) + 127).clamp(min=1), torch.ones_like(x)).to(torch.int32)


def _scale(s):
    return torch.ldexp(torch.ones((), device=s.device), s.to(torch.int32) - 127)


def _codes(x):
    """e4m3 codes of values within +-448: round to nearest, ties to even."""
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def _values(codes):
    return codes.view(torch.float8_e4m3fn).float()


def _cache(s, kv, D, seed):
    """A cache in use: keys with gains of their own in every channel, values of about one."""
    shape = (s.n_blocks, kv, s.block, D)
    gain = torch.exp(_normal((1, kv, 1, D), seed, 3, 0.5))
    k = _normal(shape, seed, 4) * gain
    ks = _exponent(k.abs().amax((2, 3)))
    s.k = _codes(k / _scale(ks)[:, :, None, None])
    del k
    v = _normal((s.n_blocks, kv, D, s.block), seed, 5)
    vs = _exponent(v.abs().amax((2, 3)))
    s.v = _codes(v / _scale(vs)[:, :, None, None])
    s.ks, s.vs = ks.to(torch.uint8), vs.to(torch.uint8)


def _grid_positions(T, seed):
    """Axes (time, height, width) of T tokens: prompts counted on all three, then the rows and columns of an image."""
    rng = random.Random(seed)
    pos = np.zeros((3, T), np.int32)
    t = 0
    while t < T:
        P, H, f0 = rng.randint(8, 256), rng.choice((8, 24, 32, 64)), rng.randint(0, 4096)
        n = min(P, T - t)
        pos[:, t:t + n] = f0 + np.arange(n)
        t += n
        n = min(H * H, T - t)
        i = np.arange(n)
        pos[0, t:t + n], pos[1, t:t + n], pos[2, t:t + n] = f0 + P, f0 + P + i // H, f0 + P + i % H
        t += n
    return torch.from_numpy(pos).cuda()


def _sections(D):
    return (D // 8, 3 * D // 16, 3 * D // 16)  # of the D / 2 pairs


def _settings(case, seed):
    """(temperature, top_k, top_p, min_p) of every row, each a tensor, or a number for all rows."""
    if case["top_k"] >= 0:
        return case["temperature"], case["top_k"], case["top_p"], case["min_p"]
    R, V = case["R"], case["V"]
    g = _generator(seed, 9)
    def pick(options, dtype):
        return torch.tensor(options, dtype=dtype, device="cuda")[
            torch.randint(0, len(options), (R,), generator=g, device="cuda")]
    return (pick((0.0, 0.7, 0.8, 1.0, 1.0, 1.2), torch.float32), pick((0, 0, 0, 50, min(2000, V), V // 2), torch.int32),
            pick((1.0, 0.9, 0.95, 0.5), torch.float32), pick((0.0, 0.0, 0.05, 0.2), torch.float32))


def prepare(case, seed):
    op = case["op"]
    if op == "slots":
        s = _layout(case, seed)
        s.n_rows += 5  # a padded batch
        # the tables as the last step left them, and the free blocks
        T, full = case["block"], s.table
        have = (s.held + T - 1) // T
        col = torch.arange(s.width, device="cuda", dtype=torch.int32)
        s.table = torch.where(col[None] < have[:, None], full, torch.full_like(full, -1)).contiguous()
        taken = torch.zeros(s.n_blocks + 1, dtype=torch.bool, device="cuda")
        taken[s.table.long().flatten()] = True  # (-1: the last entry)
        order = torch.randperm(s.n_blocks, generator=_generator(seed, 2), device="cuda")
        s.pool = order[~taken[order]].to(torch.int32).contiguous()
        s.lens, s.cu = torch.zeros_like(s.lens), torch.zeros_like(s.cu)
        s.slots = torch.zeros(s.n_rows, dtype=torch.int32, device="cuda")
        s.pos = torch.zeros_like(s.slots)
        s.used = torch.zeros(1, dtype=torch.int32, device="cuda")
    elif op == "axes":
        heads, kv, D = WIDTHS[case["width"]][:3]
        s, T, dt = State(), case["T"], DTYPE[case["dtype"]]
        s.heads, s.kv, s.D, s.T = heads, kv, D, T
        s.qkv = _normal((T, (heads + 2 * kv) * D), seed, 4).to(dt)  # rows of the QKV projection
        s.pos = _grid_positions(T, seed)
        s.q_out = torch.zeros((T, heads, D), dtype=dt, device="cuda")
        s.k_out = torch.zeros((T, kv, D), dtype=dt, device="cuda")
    elif op == "append":
        heads, kv, D = WIDTHS[case["width"]][:3]
        s, dt = _layout(case, seed), DTYPE[case["dtype"]]
        s.heads, s.kv, s.D = heads, kv, D
        _cache(s, kv, D, seed)
        gain = torch.exp(_normal((1, kv, D), seed, 3, 0.5))
        s.k_new = (_normal((s.n_rows, kv, D), seed, 6, 1.5) * gain).to(dt)
        s.v_new = _normal((s.n_rows, kv, D), seed, 7, 1.5).to(dt)
    elif op == "attend":
        heads, kv, D = WIDTHS[case["width"]][:3]
        s, dt = _layout(case, seed), DTYPE[case["dtype"]]
        s.heads, s.kv, s.D = heads, kv, D
        _cache(s, kv, D, seed)
        s.q = _normal((s.n_rows, heads, D), seed, 8, 1.5).to(dt)
        s.out = torch.zeros_like(s.q)
    else:
        s, R, V = State(), case["R"], case["V"]
        # a trained output layer's: a few codes far above a long tail, more or less so from row to row
        s.logits = _normal((R, V), seed, 4) * (1.0 + 1.5 * torch.rand((R, 1), generator=_generator(seed, 5), device="cuda"))
        top = torch.randint(0, V, (R, 8), generator=_generator(seed, 6), device="cuda")
        s.logits.scatter_add_(1, top, _normal((R, 8), seed, 7, 2.0) + 6.0)
        s.u = torch.rand((R,), generator=_generator(seed, 8), device="cuda")
        s.settings = _settings(case, seed)
        s.tokens = torch.zeros(R, dtype=torch.int32, device="cuda")
        s.probs = torch.zeros(R, dtype=torch.float32, device="cuda")
    s.case, s.handle = case, None
    return s


# ---------------------------------------------------------------- the framework's calls
def _bind(s):
    """The descriptors and the workspace that a program makes once and keeps."""
    import paper_2606_20543_amd as ssd
    case = s.case
    op = case["op"]
    dtype = ssd.SSD_BF16 if case.get("dtype") == "bf16" else ssd.SSD_F32
    if op == "slots":
        p = ssd.ssd_kvq_slot_params()
        p.n_seqs, p.block, p.table_width, p.n_pool, p.n_rows = s.B, s.block, s.width, s.pool.numel(), s.n_rows
    elif op == "axes":
        p = ssd.ssd_rope_params()
        p.n_heads, p.n_kv_heads, p.head_dim, p.dtype, p.theta = s.heads, s.kv, s.D, dtype, THETA
        p.n_axes = 3
        p.section[0], p.section[1], p.section[2] = _sections(s.D)
        p.ld_q = p.ld_k = s.qkv.shape[1]
        p.ld_q_out, p.ld_k_out = s.heads * s.D, s.kv * s.D
    elif op == "sample":
        p = ssd.ssd_sample_params()
        p.vocab = p.ld = case["V"]
        T, k, tp, mp = s.settings
        if case["top_k"] >= 0:
            p.temperature, p.top_k, p.top_p, p.min_p = T, k, tp, mp
        else:
            p.temperatures, p.top_ks, p.top_ps, p.min_ps = (x.data_ptr() for x in s.settings)
    else:
        c = s.cache = ssd.ssd_kvq_cache()
        c.k, c.v, c.k_exp, c.v_exp = s.k.data_ptr(), s.v.data_ptr(), s.ks.data_ptr(), s.vs.data_ptr()
        c.n_blocks, c.block, c.n_kv_heads, c.head_dim = s.n_blocks, s.block, s.kv, s.D
        p = ssd.ssd_kvq_append_params() if op == "append" else ssd.ssd_kvq_attn_params()
        p.dtype = dtype
        if op == "append":
            p.n_rows, p.ld_k, p.ld_v = s.n_rows, s.kv * s.D, s.kv * s.D
        else:
            p.n_seqs, p.n_rows, p.n_heads, p.table_width = s.B, s.n_rows, s.heads, s.width
            p.max_q, p.max_len = s.max_q, s.max_len
            p.ld_q = p.ld_out = s.heads * s.D
            p.scale = 1.0 / math.sqrt(s.D)
            p.workspace_bytes = ssd.ssd_kvq_workspace(c, p)
            s.workspace = torch.empty(max(p.workspace_bytes, 16), dtype=torch.uint8, device="cuda")
    s.params, s.handle = p, ssd
    return ssd


def _run_own(s):
    ssd = s.handle or _bind(s)
    op = s.case["op"]
    stream = torch.cuda.current_stream().cuda_stream
    if op == "slots":
        ssd.ssd_kvq_slots(s.params, s.held, s.new, s.pool, s.table, s.lens, s.cu, s.slots, s.pos, s.used, stream)
    elif op == "axes":
        q = s.qkv.data_ptr()
        ssd.ssd_rope_axes(s.params, s.T, q, q + s.heads * s.D * s.qkv.element_size(), s.pos, s.q_out, s.k_out, stream)
    elif op == "append":
        ssd.ssd_kvq_append(s.cache, s.params, s.slots, s.k_new, s.v_new, stream)
    elif op == "attend":
        ssd.ssd_kvq_attention(s.cache, s.params, s.q, s.cu, s.lens, s.table, s.out, s.workspace, stream)
    else:
        ssd.ssd_sample_logits(s.params, s.case["R"], s.logits, s.u, s.tokens, s.probs, stream)


# ---------------------------------------------------------------- the plain forms
def _plain_slots(s):
    T, n = s.block, s.n_rows
    have, want = (s.held + T - 1) // T, (s.held + s.new + T - 1) // T
    take = want - have
    start = torch.cumsum(take, 0) - take
    col = torch.arange(s.width, device="cuda")
    j = start[:, None] + col[None] - have[:, None]
    grown = (col[None] >= have[:, None]) & (col[None] < want[:, None])
    s.table.copy_(torch.where(grown, s.pool[j.clamp(0, s.pool.numel() - 1)], s.table))
    s.cu[1:] = torch.cumsum(s.new, 0)
    s.lens.copy_(s.held + s.new)
    s.used.copy_(take.sum(0, keepdim=True))
    r = torch.arange(n, device="cuda")
    seq = torch.searchsorted(s.cu[1:].contiguous().long(), r, right=True)
    live = seq < s.B
    seq = seq.clamp(max=s.B - 1)
    pos = r - s.cu[seq] + s.held[seq]
    at = s.table[seq, (pos // T).clamp(max=s.width - 1)]
    s.slots.copy_(torch.where(live, at * T + pos % T, -1))
    s.pos.copy_(torch.where(live, pos, -1))


def _plain_axes(s):
    half = sum(_sections(s.D))
    axis = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor(_sections(s.D), device="cuda"),
                                   output_size=half)
    freq = THETA ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    angle = s.pos[axis].t() * freq  # far positions: 64 bits
    c, sn = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    q, k = s.qkv[:, :s.heads * s.D], s.qkv[:, s.heads * s.D:(s.heads + s.kv) * s.D]
    x = torch.cat([q, k], 1).view(s.T, s.heads + s.kv, s.D).float()
    a, b = x[..., :half], x[..., half:2 * half]
    y = torch.cat([a * c - b * sn, b * c + a * sn, x[..., 2 * half:]], -1)
    s.q_out.copy_(y[:, :s.heads])
    s.k_out.copy_(y[:, s.heads:])


def _plain_append(s):
    T = s.block
    slot = s.slots.long()
    page, off = slot // T, slot % T
    # the block that each request's first new row falls into holds older tokens before it
    # (a request without new rows repeats another's)
    head = s.cu[s.seq[s.cu[:-1].long().clamp(max=s.n_rows - 1)]].long()
    hpage, hoff = page[head], off[head]
    token = torch.arange(T, device="cuda")
    for codes, exps, x, dim in ((s.k, s.ks, s.k_new, 2), (s.v, s.vs, s.v_new, 3)):  # keys [T][D], values [D][T]
        x = x.float()
        need = torch.zeros_like(exps, dtype=torch.int32)
        need.scatter_reduce_(0, page[:, None].expand(-1, x.shape[1]), _exponent(x.abs().amax(-1)), "amax")
        old = exps[hpage].int()  # keys before the first new row keep at least their scale
        both = torch.where((hoff > 0)[:, None], torch.maximum(old, need[hpage]), need[hpage])
        kept = codes[hpage]
        again = _codes(_values(kept) * _scale(old - both + 127)[:, :, None, None])
        before = token < hoff[:, None]
        before = before[:, None, :, None] if dim == 2 else before[:, None, None, :]
        codes[hpage] = torch.where(before, again, kept)
        exps[page] = need[page].to(torch.uint8)
        exps[hpage] = both.to(torch.uint8)
        y = _codes(x / _scale(exps[page])[:, :, None])
        if dim == 2:
            codes[page, :, off] = y
        else:
            codes[page, :, :, off] = y


def _plain_attend(s):
    B, T, W, g = s.B, s.block, s.width, s.heads // s.kv
    S, n = W * T, s.max_q
    at = s.table.clamp(min=0).long()
    k = _values(s.k[at]) * _scale(s.ks[at])[..., None, None]  # [B][W][kv][T][D]
    k = k.permute(0, 2, 4, 1, 3).reshape(B, s.kv, s.D, S)
    v = _values(s.v[at]) * _scale(s.vs[at])[..., None, None]  # [B][W][kv][D][T]
    v = v.permute(0, 2, 1, 4, 3).reshape(B, s.kv, S, s.D)
    i = s.seq, torch.arange(s.n_rows, device="cuda") - s.cu[s.seq]
    q = torch.zeros((B, n, s.heads, s.D), device="cuda")
    q[i] = s.q.float()
    q = q.view(B, n, s.kv, g, s.D).permute(0, 2, 3, 1, 4).reshape(B, s.kv, g * n, s.D)
    score = (q @ k).mul_(1.0 / math.sqrt(s.D)).view(B, s.kv, g, n, S)
    last = (s.lens - s.new)[:, None] + torch.arange(n, device="cuda")[None]  # the last position each row sees
    hidden = torch.arange(S, device="cuda")[None, None] > last[:, :, None]
    score.masked_fill_(hidden[:, None, None], -math.inf)
    score -= score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = score.exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(B, s.kv, g * n, S) @ v).view(B, s.kv, g, n, s.D) / total.clamp(min=1e-38)
    s.out.copy_(o.permute(0, 3, 1, 2, 4).reshape(B, n, s.heads, s.D)[i])


def _row(x, R):
    return x.double()[:, None] if isinstance(x, torch.Tensor) else torch.full((R, 1), float(x), dtype=torch.float64, device="cuda")


def _plain_sample(s):
    R, V = s.logits.shape
    T, top_k, top_p, min_p = (_row(x, R) for x in s.settings)
    # 64 bits: sums of many small weights, and uniforms next to a border
    x, idx = torch.sort(s.logits.double(), dim=1, descending=True, stable=True)  # equal logits: lower ids first
    rank = torch.arange(V, device="cuda")[None]
    w = torch.where(T > 0, torch.exp((x - x[:, :1]) / T.clamp(min=1e-30)), (rank == 0).double())
    w = w * ((rank < top_k) | (top_k < 1))
    before = torch.cumsum(w, 1) - w
    keep = (before < top_p * w.sum(1, keepdim=True)) | (top_p >= 1) | (rank == 0)
    w = w * keep * (w >= min_p)
    w = torch.zeros_like(w).scatter_(1, idx, w)
    c = torch.cumsum(w, 1)
    t = (c <= s.u.double()[:, None] * c[:, -1:]).sum(1, keepdim=True).clamp(max=V - 1)
    s.tokens.copy_(t[:, 0])
    s.probs.copy_((w.gather(1, t) / c[:, -1:])[:, 0])


def run(s):
    op = s.case["op"]
    if own:
        _run_own(s)
    elif op == "slots":
        _plain_slots(s)
    elif op == "axes":
        _plain_axes(s)
    elif op == "append":
        _plain_append(s)
    elif op == "attend":
        _plain_attend(s)
    else:
        _plain_sample(s)
    if op == "slots":
        return {"table": s.table, "lens": s.lens, "cu": s.cu, "slots": s.slots, "positions": s.pos, "used": s.used}
    if op == "axes":
        return {"q": s.q_out, "k": s.k_out}
    if op == "append":
        return {"k": s.k.view(torch.float8_e4m3fn), "v": s.v.view(torch.float8_e4m3fn), "k_exp": s.ks, "v_exp": s.vs}
    if op == "attend":
        return {"out": s.out}
    return {"tokens": s.tokens, "probs": s.probs}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    op = case["op"]
    if op == "sample":
        R, V = case["R"], case["V"]
        return {"bytes": R * (4.0 * V + 12), "flops": 10.0 * R * V}
    es = 2 if case.get("dtype") == "bf16" else 4
    if op == "axes":
        heads, kv, D = WIDTHS[case["width"]][:3]
        return {"bytes": case["T"] * ((heads + kv) * D * 2.0 * es + 12), "flops": case["T"] * (heads + kv) * D * 3.0}
    held, new = _lengths(case)
    T, B, n = case["block"], case["B"], sum(new)
    if op == "slots":
        grown = sum(-(-(h + m) // T) - -(-h // T) for h, m in zip(held, new))
        return {"bytes": 4.0 * (4 * B + 2 * grown + 3 * n + 12), "flops": 4.0 * (B + n)}
    heads, kv, D = WIDTHS[case["width"]][:3]
    if op == "append":
        blocks = sum(-(-(h + m) // T) - h // T for h, m in zip(held, new) if m)
        return {"bytes": 2.0 * n * kv * D * (es + 1) + 4 * n + 2 * blocks * kv, "flops": 4.0 * n * kv * D}
    lens = [h + m for h, m in zip(held, new)]
    blocks = sum(-(-x // T) for x, m in zip(lens, new) if m)
    b = 2.0 * kv * sum(x * D for x, m in zip(lens, new) if m) + blocks * (2 * kv + 4) + 2 * n * heads * D * es + 8 * B
    seen = sum(m * h + m * (m + 1) / 2 for h, m in zip(held, new))
    return {"bytes": b, "flops": 4.0 * heads * D * seen}


# ---------------------------------------------------------------- the same in 64 bits, from the definitions
def _round_e4m3(x):
    """Nearest e4m3 value (three fraction bits, exponents from -6; ties to even) of 64-bit values within +-448."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -20))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def _exact_append(s):
    T, out = s.block, {}
    slots = s.slots.cpu().tolist()
    runs, r = [], 0
    while r < len(slots):  # rows of one block
        e = r + 1
        while e < len(slots) and slots[e] == slots[e - 1] + 1 and slots[e] % T:
            e += 1
        runs.append((r, e))
        r = e
    for name, codes, exps, x in (("k", s.k, s.ks, s.k_new), ("v", s.v.transpose(2, 3), s.vs, s.v_new)):
        val = codes.contiguous().view(torch.float8_e4m3fn).double()  # [blocks][kv][T][D]
        exp = exps.double()
        x = x.double()
        for a, e in runs:
            pg, o = slots[a] // T, slots[a] % T
            rows = x[a:e].transpose(0, 1)  # [kv][n][D]
            big = rows.abs().amax((1, 2))
            need = torch.ceil(torch.log2(big.clamp(min=2.0 ** -149) / CODE_MAX)) + 127
            need = torch.where(big > 0, need, torch.zeros_like(need)).clamp(min=1)
            if o:
                new = torch.maximum(need, exp[pg])
                val[pg, :, :o] = _round_e4m3(val[pg, :, :o] * torch.exp2(exp[pg] - new)[:, None, None])
                need = new
            exp[pg] = need
            val[pg, :, o:o + e - a] = _round_e4m3(rows * torch.exp2(127 - need)[:, None, None])
        out[name] = val if name == "k" else val.transpose(2, 3).contiguous()
        out[name + "_exp"] = exp.to(torch.uint8)
    return out


def _exact_attend(s):
    out = torch.zeros((s.n_rows, s.heads, s.D), dtype=torch.float64, device="cuda")
    cu, held, lens = s.cu.tolist(), s.held.tolist(), s.lens.tolist()
    g = s.heads // s.kv
    for b in range(s.B):
        a, e, L = cu[b], cu[b + 1], lens[b]
        if a == e:
            continue
        at = s.table[b, :-(-L // s.block)].long()
        key = s.k[at].view(torch.float8_e4m3fn).double() * torch.exp2(s.ks[at].double() - 127)[..., None, None]
        val = s.v[at].view(torch.float8_e4m3fn).double() * torch.exp2(s.vs[at].double() - 127)[..., None, None]
        pos = torch.arange(L, device="cuda")
        seen = pos[None] <= held[b] + torch.arange(e - a, device="cuda")[:, None]
        for h in range(s.kv):
            kh = key[:, h].reshape(-1, s.D)[:L]
            vh = val[:, h].transpose(1, 2).reshape(-1, s.D)[:L]
            for j in range(h * g, (h + 1) * g):
                x = (s.q[a:e, j].double() @ kh.t().contiguous()) / math.sqrt(s.D)
                out[a:e, j] = torch.softmax(x.masked_fill(~seen, -math.inf), -1) @ vh
    return {"out": out}


def _exact_sample(s):
    R, V = s.logits.shape
    T, top_k, top_p, min_p = (x.cpu().numpy().astype(np.float64) if isinstance(x, torch.Tensor) else np.full(R, float(x))
                              for x in s.settings)
    L, u = s.logits.cpu().numpy().astype(np.float64), s.u.cpu().numpy().astype(np.float64)
    tokens, probs = np.zeros(R, np.int32), np.zeros(R)
    for r in range(R):
        order = np.lexsort((np.arange(V), -L[r]))
        if not T[r] > 0:
            tokens[r], probs[r] = order[0], 1.0
            continue
        w = np.exp((L[r][order] - L[r].max()) / T[r])
        n = V if top_k[r] < 1 else min(V, int(top_k[r]))
        w = w[:n]
        if top_p[r] < 1:
            n = max(1, int(np.searchsorted(np.cumsum(w), top_p[r] * w.sum(), side="left")) + 1)
        ids = order[:n][w[:n] >= min_p[r]]
        ids.sort()
        p = np.exp((L[r][ids] - L[r].max()) / T[r])
        p /= p.sum()
        j = min(int(np.searchsorted(np.cumsum(p), u[r], side="right")), len(ids) - 1)
        tokens[r], probs[r] = ids[j], p[j]
    return {"tokens": tokens, "probs": probs}


def exact(case, seed):
    op = case["op"]
    if op == "slots":
        return None
    s = prepare(case, seed)
    if op == "append":
        return _exact_append(s)
    if op == "attend":
        return _exact_attend(s)
    if op == "sample":
        return _exact_sample(s)
    half = sum(_sections(s.D))
    x = s.qkv.double()[:, :(s.heads + s.kv) * s.D].reshape(s.T, s.heads + s.kv, s.D)
    y, j0 = x.clone(), 0
    for axis, n in enumerate(_sections(s.D)):
        j = torch.arange(j0, j0 + n, dtype=torch.float64, device="cuda")
        z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                        s.pos[axis].double()[:, None] * torch.exp(-j / half * math.log(THETA)))[:, None]
        i = j.long()
        turned = torch.complex(x[..., i], x[..., i + half]) * z
        y[..., i], y[..., i + half] = turned.real, turned.imag
        j0 += n
    return {"q": y[:, :s.heads].contiguous(), "k": y[:, s.heads:].contiguous()}
