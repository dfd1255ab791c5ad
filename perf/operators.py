"""The operators on the dense cache that is held in 8 bits, as cases that can be timed.

A layer that is not compressed keeps K and V of its KV heads in blocks of ``block`` tokens.  A complete block of one
head is a page of 8-bit values with one scale for K and one for V; the block that is still being filled is the tail,
kept in the cache's own type.  A serving program writes a prompt into such a cache, pushes tokens, attends to it with
one query per row or with a chunk of them, and reads it back (to hand it to the compression, for instance).

  int8   scale = amax / 127, value = round(x * 127 / amax), half to even
  e4m3   scale = amax / 448, value = the nearest e4m3 number to x * 448 / amax, half to even

A case:
  op        "attend": attention of the last n_q tokens of every row (causal);  "step": ``steps`` times a push of one token
            and the attention of its query;  "store": a prompt written (``chunk`` > 0: in chunks) and read back;
            "read": tokens from ``start`` on read back
  dtype     of K, V, q and results: "bf16" or "f32";  fmt: "int8" or "e4m3"
  batch, q_heads, kv_heads, head_dim, block
  tokens    of the longest row;  ragged: rows of different length, the second one empty
"""
import math

import torch

own = False


def _case(op, batch, q_heads, kv_heads, head_dim, tokens, block=64, fmt="int8", dtype="bf16", ragged=False, n_q=1, steps=0, chunk=0, start=0, name=None):
    c = dict(op=op, batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, tokens=tokens, block=block, fmt=fmt, dtype=dtype, ragged=ragged,
             n_q=n_q, steps=steps, chunk=chunk, start=start)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user of a short chat: the latency of a call
        _case("attend", 1, 32, 8, 128, 1003, name="attend_1k_chat"),
        # one user at 32K tokens
        _case("attend", 1, 32, 8, 128, 32001, name="attend_32k"),
        # long context, batch 4: the most bytes of a single-token call
        _case("attend", 4, 32, 8, 128, 131000, block=128, fmt="e4m3", name="attend_128k_b4"),
        # a ragged batch of users, one of whom has no token yet; three query heads to a KV head, small pages
        _case("attend", 6, 24, 8, 128, 12345, block=16, fmt="e4m3", ragged=True, name="attend_ragged_b6"),
        # a toy fp32 model
        _case("attend", 1, 4, 1, 128, 1024, dtype="f32", name="attend_toy_f32"),
        # five tokens a row are verified at once (drafted by a smaller model), heads of 64
        _case("attend", 4, 16, 4, 64, 6001, block=32, n_q=5, ragged=True, name="attend_verify5_b4"),
        # a chunk of a prompt attends to what the cache holds of it, itself included: the most arithmetic
        _case("attend", 1, 32, 8, 128, 16384, n_q=2048, name="attend_chunk2048_16k"),
        # the token steps of an MHA batch, over the end of a block
        _case("step", 8, 32, 32, 128, 4090, steps=8, name="step_4k_mha_b8"),
        # one user's token steps at 8K tokens
        _case("step", 1, 32, 8, 128, 8150, block=128, fmt="e4m3", steps=8, name="step_8k"),
        # a short prompt arrives in chunks and is read back
        _case("store", 1, 32, 8, 128, 300, chunk=100, name="store_300_chunks"),
        # a prompt of 32K tokens is written and read back: what stands in front of compressing it
        _case("store", 1, 32, 8, 128, 32768, fmt="e4m3", name="store_32k"),
        # the later part of a ragged MHA batch is read back
        _case("read", 8, 32, 32, 128, 4001, block=32, ragged=True, start=77, name="read_4k_mha_b8"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attend", "attend", "attend", "attend", "step", "store", "read"))
    q_heads, kv_heads, d = rng.choice(((32, 8, 128), (32, 8, 128), (24, 8, 128), (32, 32, 128), (16, 4, 64), (8, 8, 64), (16, 1, 128), (8, 2, 256)))
    block, fmt = rng.choice((16, 32, 64, 64, 128)), rng.choice(("int8", "e4m3"))
    dtype = "f32" if rng.random() < 0.15 else "bf16"
    batch = _log_int(rng, 1, 16)
    ragged = batch > 1 and rng.random() < 0.6
    most = {"attend": 131000, "step": 131000, "store": 32768, "read": 32768}[op]
    # K and V of the longest listed call of the kind, in values
    room = {"attend": 1 << 30, "step": 1 << 28, "store": 1 << 26, "read": 1 << 28}[op] // (2 * batch * kv_heads * d)
    if dtype == "f32":
        room //= 2
    tokens = _log_int(rng, 1, max(2, min(most, room)))
    n_q = steps = chunk = start = 0
    if op == "attend":
        # half of the calls have one query a row; the products of the others stay below the longest listed chunk's
        n_q = 1 if rng.random() < 0.5 else _log_int(rng, 2, max(2, min(2048, tokens, int(3e7 / (tokens * batch) * 32 / q_heads * 128 / d))))
    elif op == "step":
        steps = rng.randint(1, 4) if tokens * batch * kv_heads * d > 1 << 25 else rng.randint(1, 12)
    elif op == "store":
        chunk = 0 if tokens < 8 or rng.random() < 0.5 else -(-tokens // rng.randint(2, 5))
    else:
        start = rng.randint(0, tokens // 2)
    return _case(op, batch, q_heads, kv_heads, d, tokens, block, fmt, dtype, ragged, max(1, n_q), steps, chunk, start)


def _lengths(c):
    """Tokens of every row in front of the call (attend: behind its queries' own push)."""
    if not c["ragged"]:
        return [c["tokens"]] * c["batch"]
    n = [c["tokens"]] + [(c["tokens"] * (3 + 5 * b % 7)) // (11 + b % 3) for b in range(1, c["batch"])]
    n[1] = 0
    return n


def _dims(c):
    most = c["tokens"] + c["steps"]
    return (c["batch"], c["kv_heads"], c["head_dim"], c["block"], -(-most // c["block"]),
            torch.float32 if c["dtype"] == "f32" else torch.bfloat16)


def _round8(y, fmt):
    """The 8-bit number next to y (in 64 bits), as a number."""
    if fmt == "int8":
        return torch.round(y)
    e = (torch.frexp(y)[1] - 1).clamp_min(-6) - 3              # the step of e4m3 at y is 2^e
    return torch.ldexp(torch.round(torch.ldexp(y, -e)), e)


def _quantise(x, fmt):
    """Blocks [..., block, d] -> their 8-bit numbers (int8 or e4m3) and their scales [...] in 32 bits."""
    top = 127.0 if fmt == "int8" else 448.0
    x = x.double()
    amax = x.abs().amax((-1, -2))
    y = x * top / torch.where(amax > 0, amax, torch.ones_like(amax))[..., None, None]
    return _round8(y, fmt).float().to(torch.int8 if fmt == "int8" else torch.float8_e4m3fn), (amax / top).float()


def _keys_values(g, shape, heads_at, d, dtype):
    """Keys with a few strong channels, as rotated keys have, and plain values."""
    k = torch.randn(shape, generator=g, device="cuda")
    view = [1] * len(shape)
    view[heads_at], view[-1] = shape[heads_at], d
    k *= torch.exp(0.5 * torch.randn(view, generator=g, device="cuda"))
    v = torch.randn(shape, generator=g, device="cuda")
    return k.to(dtype), v.to(dtype)


def prepare(c, seed):
    B, H, d, blk, nb, dt = _dims(c)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")
    pages = B * nb + 3
    S = dict(case=c, fmt=c["fmt"], block=blk, dtype=dt, scale=d ** -0.5, n0=n)
    # the block table gives every block of a row a page of its own, in no order
    S["table"] = torch.randperm(pages, generator=g, device="cuda")[:B * nb].reshape(B, nb).to(torch.int32)
    if c["op"] == "store":
        byte = torch.int8 if c["fmt"] == "int8" else torch.float8_e4m3fn
        S["k_pages"], S["v_pages"] = (torch.zeros((pages, H, blk, d), dtype=torch.uint8, device="cuda").view(byte) for _ in range(2))
        S["k_scale"], S["v_scale"] = (torch.zeros((pages, H), device="cuda") for _ in range(2))
    else:
        # heads in front: the channels' strengths belong to the heads
        k, v = _keys_values(g, (pages, H, blk, d), 1, d, dt)
        S["k_pages"], S["k_scale"] = _quantise(k, c["fmt"])
        S["v_pages"], S["v_scale"] = _quantise(v, c["fmt"])
        del k, v
    # tails, their largest magnitudes and the rows' state in one buffer, so that a pass that pushes tokens can start over with one copy
    eb = dt.itemsize
    tail, amax = B * H * blk * d * eb, -(-B * H * 2 * 4 // 16) * 16
    S["live"] = torch.zeros(2 * tail + amax + B * 16, dtype=torch.uint8, device="cuda")
    S["k_tail"], S["v_tail"] = (S["live"][i * tail:(i + 1) * tail].view(dt).view(B, H, blk, d) for i in range(2))
    S["tail_amax"] = S["live"][2 * tail:2 * tail + B * H * 8].view(torch.float32).view(B, H, 2)
    S["state"] = S["live"][2 * tail + amax:].view(torch.int32).view(B, 4)
    if c["op"] != "store":
        k, v = _keys_values(g, (B, H, blk, d), 1, d, dt)
        filled = (torch.arange(blk, device="cuda") < (n % blk)[:, None])[:, None, :, None]
        S["k_tail"].copy_(torch.where(filled, k, 0))
        S["v_tail"].copy_(torch.where(filled, v, 0))
        S["tail_amax"].copy_(torch.stack((S["k_tail"].float().abs().amax((2, 3)), S["v_tail"].float().abs().amax((2, 3))), -1))
        S["state"][:, 0] = n
    S["live0"] = S["live"].clone()
    if c["op"] == "attend":
        S["q"] = torch.randn((B, c["n_q"], c["q_heads"], d), generator=g, device="cuda").to(dt)
        S["out"] = torch.empty_like(S["q"])
    elif c["op"] == "step":
        S["q"] = torch.randn((c["steps"], B, c["q_heads"], d), generator=g, device="cuda").to(dt)
        S["k_new"], S["v_new"] = _keys_values(g, (c["steps"], B, H, d), 2, d, dt)
        S["out"] = torch.empty_like(S["q"])
        S["each"] = list(zip(S["q"], S["k_new"], S["v_new"], S["out"]))
        # what the steps may have changed: the last block in front of them and the one behind
        S["start"] = max(0, c["tokens"] - blk)
        S["k_out"], S["v_out"] = (torch.zeros((B, c["tokens"] + c["steps"] - S["start"], H, d), dtype=dt, device="cuda") for _ in range(2))
    elif c["op"] == "store":
        S["k"], S["v"] = _keys_values(g, (B, c["tokens"], H, d), 2, d, dt)
    if c["op"] in ("store", "read"):
        S["start"] = c["start"]
        S["k_out"], S["v_out"] = (torch.zeros((B, c["tokens"] - c["start"], H, d), dtype=dt, device="cuda") for _ in range(2))
    if c["op"] == "store" and c["chunk"]:
        # the chunks of the prompt, and how many tokens of each belong to each row
        at = list(range(0, c["tokens"], c["chunk"]))
        S["chunks"] = [(S["k"][:, a:a + c["chunk"]], S["v"][:, a:a + c["chunk"]], (n - a).clamp(0, min(c["chunk"], c["tokens"] - a)).to(torch.int32)) for a in at]
    if own:
        from paper_2506_11886_b200 import fa
        S["fa"] = fa
        S["layout"] = fa.Q8Layout(batch=B, n_q_heads=c["q_heads"], n_kv_heads=H, head_dim=d, block=blk, max_blocks=nb, n_pages=pages,
                                  format=fa.FA_Q8_INT8 if c["fmt"] == "int8" else fa.FA_Q8_E4M3,
                                  kv_dtype=fa.FA_F32 if c["dtype"] == "f32" else fa.FA_BF16, softmax_scale=S["scale"])
        S["cache"] = fa.Q8Cache(S["layout"], buffers=dict(k_pages=S["k_pages"], v_pages=S["v_pages"], k_scale=S["k_scale"], v_scale=S["v_scale"],
                                                          k_tail=S["k_tail"], v_tail=S["v_tail"], tail_amax=S["tail_amax"],
                                                          block_table=S["table"], state=S["state"]))
        S["ws"] = fa.new_q8_workspace(S["layout"], c["n_q"])
    return S


# ---- the plain form -----------------------------------------------------------------------------------------------
def _pages_of(pages, scale, table):
    """Values [B, H, blocks * block, d] of the pages of every row, in 32 bits."""
    byte = pages.dtype
    x = pages.view(torch.uint8)[table.long()].view(byte).float() * scale[table.long()][..., None, None]
    B, nb, H, blk, d = x.shape
    return x.transpose(1, 2).reshape(B, H, nb * blk, d)


def _dense(S, n):
    """K, V [B, H, tokens, d] in 32 bits of the rows' n tokens: pages, then the tails put in their places."""
    blk, nb = S["block"], S["table"].shape[1]
    pos = torch.arange(nb * blk, device="cuda")
    first = n // blk * blk                                      # of the tail
    in_tail = (pos >= first[:, None]) & (pos < n[:, None])
    seen = pos < first[:, None]
    slot = (pos - first[:, None]).clamp(0, blk - 1)
    both = []
    for side in ("k", "v"):
        x = _pages_of(S[side + "_pages"], S[side + "_scale"], S["table"])
        x = torch.where(seen[:, None, :, None], x, 0)
        t = S[side + "_tail"].float()
        t = torch.take_along_dim(t, slot[:, None, :, None].expand(-1, t.shape[1], -1, t.shape[3]), 2)
        both.append(torch.where(in_tail[:, None, :, None], t, x))
    return both


def _attend(S, q):
    """q [B, n_q, Hq, d]: the queries of every row's last n_q tokens."""
    n = S["state"][:, 0].long()
    k, v = _dense(S, n)
    B, n_q, Hq, d = q.shape
    H = k.shape[1]
    G = Hq // H
    x = q.float().reshape(B, n_q, H, G, d).permute(0, 2, 1, 3, 4).reshape(B, H, n_q * G, d)
    s = x @ k.transpose(2, 3) * S["scale"]
    last = n[:, None] - n_q + torch.arange(n_q, device="cuda")  # the last token that a query sees
    seen = (torch.arange(k.shape[2], device="cuda") <= last[..., None]).repeat_interleave(G, 1)[:, None]
    s = torch.where(seen, s, -torch.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isfinite(top), top, 0))
    o = p @ v / p.sum(-1, keepdim=True).clamp_min(1e-30)
    return o.reshape(B, H, n_q, G, d).permute(0, 2, 1, 3, 4).reshape(B, n_q, Hq, d).to(S["dtype"])


def _push(S, k_new, v_new):
    """One token [B, H, d] to every row: into the tail, which becomes a page when it is full."""
    n, blk = S["state"][:, 0].long(), S["block"]
    rows = torch.arange(n.shape[0], device="cuda")
    full = (n + 1) % blk == 0
    page = torch.take_along_dim(S["table"].long(), (n // blk)[:, None], 1)[:, 0]
    for i, (side, new) in enumerate((("k", k_new), ("v", v_new))):
        tail, pages = S[side + "_tail"], S[side + "_pages"].view(torch.uint8)
        tail[rows, :, n % blk] = new
        q, scale = _quantise(tail, S["fmt"])
        pages[page] = torch.where(full[:, None, None, None], q.view(torch.uint8), pages[page])
        S[side + "_scale"][page] = torch.where(full[:, None], scale, S[side + "_scale"][page])
    S["state"][:, 0] += 1


def _read(S, start):
    n = S["state"][:, 0].long()
    k, v = _dense(S, n)
    stop = start + S["k_out"].shape[1]
    there = (torch.arange(start, stop, device="cuda") < n[:, None])[:, :, None, None]
    return [torch.where(there, x[:, :, start:stop].transpose(1, 2).to(S["dtype"]), old) for x, old in ((k, S["k_out"]), (v, S["v_out"]))]


def _store(S):
    """The whole prompt: blocks that are complete become pages, what is left of a row its tail."""
    n, blk = S["n0"].long(), S["block"]
    B, nb = S["table"].shape
    rows, slots = torch.arange(B, device="cuda"), torch.arange(blk, device="cuda")
    whole = torch.arange(nb, device="cuda") < (n // blk)[:, None]
    last = (n // blk).clamp_max(nb - 1)
    filled = (slots < (n - last * blk)[:, None]) & (n % blk > 0)[:, None]
    for side in ("k", "v"):
        x = S[side]
        H, d = x.shape[2:]
        x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, nb * blk - x.shape[1])).reshape(B, nb, blk, H, d).transpose(2, 3)
        q, scale = _quantise(x, S["fmt"])
        pages, at = S[side + "_pages"].view(torch.uint8), S["table"].long()
        pages[at] = torch.where(whole[..., None, None, None], q.view(torch.uint8), pages[at])
        S[side + "_scale"][at] = torch.where(whole[..., None], scale, S[side + "_scale"][at])
        tail = S[side + "_tail"]
        tail.copy_(torch.where(filled[:, None, :, None], x[rows, last], tail))
    S["state"][:, 0] = S["n0"]


def run(S):
    op = S["case"]["op"]
    if own:
        fa, layout, cache, ws = S["fa"], S["layout"], S["cache"], S["ws"]
        if op == "attend":
            fa.fa_q8_attention(layout, cache, S["q"], S["out"], ws)
            return S["out"]
        if op == "read":
            fa.fa_q8_read(layout, cache, S["k_out"], S["v_out"], S["start"])
            return S["k_out"], S["v_out"]
        if op == "store":
            if S["case"]["chunk"]:
                fa.fa_q8_reset(layout, cache)
                for k, v, n in S["chunks"]:
                    fa.fa_q8_append(layout, cache, k, v, n)
            else:
                fa.fa_q8_write(layout, cache, S["k"], S["v"], S["n0"])
            fa.fa_q8_read(layout, cache, S["k_out"], S["v_out"], 0)
            return S["k_out"], S["v_out"], S["state"][:, 0]
        S["live"].copy_(S["live0"])
        for q, k, v, o in S["each"]:
            fa.fa_q8_step(layout, cache, q, k, v, o, ws)
        fa.fa_q8_read(layout, cache, S["k_out"], S["v_out"], S["start"])
        return S["out"], S["k_out"], S["v_out"], S["state"][:, 0]
    if op == "attend":
        return _attend(S, S["q"])
    if op == "read":
        return tuple(_read(S, S["start"]))
    if op == "store":
        _store(S)
        return (*_read(S, 0), S["state"][:, 0])
    S["live"].copy_(S["live0"])
    out = []
    for q, k, v, _ in S["each"]:
        _push(S, k, v)
        out.append(_attend(S, q[:, None])[:, 0])
    return (torch.stack(out), *_read(S, S["start"]), S["state"][:, 0])


def work(c):
    B, H, d, blk, _, dt = _dims(c)
    eb, Hq, n = dt.itemsize, c["q_heads"], _lengths(c)

    def cached(t):
        """Bytes of the first t tokens of a row: pages with their scales, then the tail."""
        return (t // blk * (blk * d + 4) + t % blk * d * eb) * 2 * H

    if c["op"] == "attend":
        pairs = sum(max(0, t - c["n_q"] + 1 + i) for t in n for i in range(c["n_q"]))
        return {"bytes": sum(cached(t) for t in n) + 2 * B * c["n_q"] * Hq * d * eb, "flops": 4 * Hq * d * pairs}
    if c["op"] == "step":
        per = [sum(cached(t + i + 1) for t in n) + B * (2 * Hq + 2 * H) * d * eb for i in range(c["steps"])]
        return {"bytes": sum(per), "flops": 4 * Hq * d * sum(t + i + 1 for t in n for i in range(c["steps"]))}
    if c["op"] == "store":
        # K and V read; pages, scales and tails written and read again; K and V written
        return {"bytes": sum(2 * cached(t) + 4 * t * H * d * eb for t in n), "flops": 0}
    return {"bytes": sum(max(0, cached(t) - cached(min(t, c["start"]))) + 2 * max(0, t - c["start"]) * H * d * eb for t in n), "flops": 0}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------
def _numbers(fmt):
    """All 8-bit numbers of a format in order."""
    if fmt == "int8":
        return torch.arange(-127, 128, dtype=torch.float64, device="cuda")
    m = torch.arange(8, dtype=torch.float64)
    pos = torch.cat([m * 2.0 ** -9] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16)])[:127]
    return torch.cat((-pos.flip(0), pos[1:])).cuda()


def _held(x, fmt):
    """What a complete block [block, d] of one head stands for, by search among the format's numbers."""
    z = _numbers(fmt)
    x = x.double()
    amax = x.abs().max()
    if amax == 0:
        return torch.zeros_like(x)
    top = z[-1]
    # 2 x top against (z_i + z_(i+1)) amax: both sides whole, so that ties are seen as ties
    twice = (x * (2 * top)).reshape(-1).contiguous()
    border = (z[1:] + z[:-1]) * amax
    lo, hi = torch.searchsorted(border, twice), torch.searchsorted(border, twice, right=True)
    odd = torch.arange(z.numel(), device="cuda") - z.numel() // 2
    pick = torch.where((lo != hi) & (odd[lo] % 2 != 0), hi, lo)
    return (z[pick] * (amax / top)).reshape(x.shape)


def _row(S, b, h, side):
    """The cached tokens of a row's head in 64 bits, from the state in front of the pass."""
    blk, n = S["block"], int(S["n0"][b])
    at = S["table"][b, :n // blk].long()
    x = S[side + "_pages"][:, h].view(torch.uint8)[at].view(S[side + "_pages"].dtype).to(torch.float64) * S[side + "_scale"][at, h].double()[:, None, None]
    return torch.cat((x.reshape(n // blk * blk, x.shape[-1]), S[side + "_tail"][b, h, :n % blk].double()))


def _softmax_rows(q, k, v, first, scale):
    """Rows of q see k[: first + row + 1]."""
    if k.shape[0] == 0:
        return torch.zeros_like(q)
    s = (q @ k.T) * scale
    hide = torch.arange(k.shape[0], device="cuda")[None] > first + torch.arange(q.shape[0], device="cuda")[:, None]
    s.masked_fill_(hide, -math.inf)
    return torch.nan_to_num(torch.softmax(s, -1), nan=0.0) @ v


def exact(c, seed):
    S = prepare(c, seed)
    B, H, d, blk, _, _ = _dims(c)
    n = _lengths(c)
    if c["op"] == "attend":
        out = torch.zeros((B, c["n_q"], c["q_heads"], d), dtype=torch.float64, device="cuda")
        G = c["q_heads"] // H
        for b in range(B):
            for h in range(H):
                k, v = _row(S, b, h, "k"), _row(S, b, h, "v")
                for j in range(G):
                    out[b, :, h * G + j] = _softmax_rows(S["q"][b, :, h * G + j].double(), k, v, n[b] - c["n_q"], S["scale"])
        return out
    back = [torch.zeros(S["k_out"].shape, dtype=torch.float64, device="cuda") for _ in range(2)]
    start = S["start"]
    if c["op"] == "store":
        for b in range(B):
            for h in range(H):
                for x, o in ((S["k"], back[0]), (S["v"], back[1])):
                    r = x[b, :n[b], h].double()
                    for t in range(0, n[b] // blk * blk, blk):
                        r[t:t + blk] = _held(r[t:t + blk], c["fmt"])
                    o[b, :n[b], h] = r
        return (*back, None)
    if c["op"] == "read":
        for b in range(B):
            for h in range(H):
                for side, o in (("k", back[0]), ("v", back[1])):
                    r = _row(S, b, h, side)[start:]
                    o[b, :r.shape[0], h] = r
        return tuple(back)
    out = torch.zeros(S["q"].shape, dtype=torch.float64, device="cuda")
    G = c["q_heads"] // H
    for b in range(B):
        for h in range(H):
            rows = [_row(S, b, h, side) for side in "kv"]
            for i in range(c["steps"]):
                for j, new in enumerate((S["k_new"], S["v_new"])):
                    rows[j] = torch.cat((rows[j], new[i, b, h].double()[None]))
                    t = rows[j].shape[0]
                    if t % blk == 0:                            # the tail is complete: its tokens are held in 8 bits from here on
                        rows[j][t - blk:] = _held(rows[j][t - blk:], c["fmt"])
                out[i, b, h * G:(h + 1) * G] = _softmax_rows(S["q"][i, b, h * G:(h + 1) * G].double(), rows[0], rows[1], rows[0].shape[0], S["scale"])
            for r, o in zip(rows, back):
                o[b, :max(0, r.shape[0] - start), h] = r[start:]
    return (out, *back, None)
