"""Operators over caches that requests have in common, as cases that can be timed and compared with a plain form:

  prefix   xq_prefix_attention: queries of a batch against a prompt that its sequences share (one cache for all of them,
           or one for every few), then against each sequence's own cache;
  cross    xq_cross_attention: query tokens against a whole cache of encoder states, every sequence's of its own length;
  gather   xq_gather_sequences: a cache whose sequences are chosen from another one's, or reordered in place (a prompt
           forked for several answers, beams that go on, finished sequences left out).

Keys, values and queries follow the recipe of workloads.py: N(0, 1), three outlier key channels of each head ten times
as large, the second layer of a pair close to the first and without codes of its own.  Where `own` is false nothing of
the library is used: the caches are quantized here, by the formulas of the paper (min-max groups, keys by channel and
values by token, calibrated scale and zero-point in fp16), and run() computes in 32 bits with elementary operations.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

ETA = {1: 1.0 / 6.0, 2: 0.045}  # calibration parameters of the paper's main results, by bits
LAYERS = 2                      # prefix and cross: a pair of layers that share their codes


def _attention(name, op, *, batch, q_heads, kv_heads, length, tokens=1, prefixes=1, mine=0, head_dim=128, group=32,
               residual=128, kbits=2, vbits=2, f16=False, ragged=False):
    return dict(name=name, op=op, batch=batch, prefixes=prefixes, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                length=length, mine=mine, tokens=tokens, group=group, residual=residual, kbits=kbits, vbits=vbits,
                f16=f16, ragged=ragged)


def _gather(name, *, layers, batch, take, kv_heads, length, place, head_dim=128, group=32, residual=128, kbits=2,
            vbits=2, f16=False):
    return dict(name=name, op="gather", layers=layers, batch=batch, take=take, kv_heads=kv_heads, length=length,
                place=place, head_dim=head_dim, group=group, residual=residual, kbits=kbits, vbits=vbits, f16=f16)


def listed():
    return [
        # a small model's few users behind a short instruction: a call's own time
        _attention("prefix_small", "prefix", batch=4, q_heads=4, kv_heads=4, head_dim=64, length=512, mine=33,
                   residual=32),
        # sixteen chats behind one system prompt, one new token each
        _attention("prefix_16_at_8k", "prefix", batch=16, q_heads=32, kv_heads=8, length=8192, mine=300, vbits=1),
        # many users of one long document
        _attention("prefix_64_at_32k", "prefix", batch=64, q_heads=32, kv_heads=8, length=32768, mine=500, vbits=1),
        # eight samples of each of four prompts, groups of five heads, quantization groups and window of 64, half precision
        _attention("prefix_samples_4x8", "prefix", batch=32, prefixes=4, q_heads=40, kv_heads=8, length=5000, mine=77,
                   group=64, residual=64, f16=True),
        # the users' own prompts, ragged, behind a shared one
        _attention("prefix_prompts_100", "prefix", batch=4, q_heads=32, kv_heads=8, length=16384, mine=250, tokens=100,
                   vbits=1),
        # a decoder's token against the encoder's states of each of sixteen inputs, every head with its own kv head
        _attention("cross_token_1500", "cross", batch=16, q_heads=32, kv_heads=32, length=1500, ragged=True),
        # a decoder's whole prompt of 200 tokens against four images or documents of ragged length
        _attention("cross_200_at_6404", "cross", batch=4, q_heads=32, kv_heads=8, length=6404, tokens=200, ragged=True),
        # a few tokens against one long recording, 1-bit keys
        _attention("cross_16_at_40k", "cross", batch=1, q_heads=32, kv_heads=8, length=40000, tokens=16, kbits=1,
                   f16=True),
        # a step of beam search: four prompts of four beams each; some beams end and others go on in their place
        _gather("gather_beams", layers=32, batch=16, take=16, kv_heads=8, length=1000, place="beams", vbits=1),
        # a prompt forked for 32 answers
        _gather("gather_fork_32", layers=8, batch=1, take=32, kv_heads=8, length=8192, place="fork", vbits=1),
        # finished sequences left out of a batch
        _gather("gather_compact", layers=4, batch=24, take=17, kv_heads=32, length=4100, place="compact", f16=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["prefix", "prefix", "prefix", "cross", "cross", "gather", "gather"])
    head_dim = 64 if rng.random() < 0.2 else 128
    kv_heads = rng.choice([1, 2, 4, 8, 8, 8, 16, 32])
    group = rng.choice([32, 32, 64])
    residual = rng.choice([64, 128, 128, 256])
    bits = dict(kbits=rng.choice([1, 2, 2]), vbits=rng.choice([1, 2]), f16=rng.random() < 0.3)
    if op == "gather":
        place = rng.choice(["beams", "fork", "compact"])
        layers = 2 * _log_int(rng, 1, 16)
        batch, take = {"beams": lambda: (4 * _log_int(rng, 1, 12),) * 2,
                       "fork": lambda: (_log_int(rng, 1, 4), _log_int(rng, 1, 48)),
                       "compact": lambda: (_log_int(rng, 2, 48), 0)}[place]()
        if place == "compact":
            take = rng.randint(1, batch)
        most = 20_000_000 // (layers * max(batch, take) * kv_heads)
        length = max(1, min(_log_int(rng, 1, 32768), most))
        case = _gather("", layers=layers, batch=batch, take=take, kv_heads=kv_heads, length=length, place=place,
                       head_dim=head_dim, group=group, residual=residual, **bits)
    else:
        q_heads = kv_heads * rng.choice([1, 2, 3, 4, 4, 5, 7, 8])
        tokens = rng.choice([1, 1, 1, 1, _log_int(rng, 2, 512)])
        batch = _log_int(rng, 1, 64) if tokens == 1 else _log_int(rng, 1, 8)
        prefixes = 1
        if op == "prefix" and rng.random() < 0.3:
            prefixes = _log_int(rng, 1, 8)
            batch = prefixes * max(1, batch // prefixes)
        # every query reads every token: bounded by heads x tokens x length, and the caches by streams x length
        most = min(60_000_000 // (batch * q_heads * tokens),
                   3_000_000 // (kv_heads * (prefixes if op == "prefix" else batch)))
        length = max(1, min(_log_int(rng, 16, 65536), most))
        mine = 0
        if op == "prefix":
            mine = tokens + _log_int(rng, 1, 1000) - 1
            mine = min(mine, max(tokens, 1_500_000 // (batch * kv_heads)))
            if rng.random() < 0.05:
                mine = 0
        case = _attention("", op, batch=batch, prefixes=prefixes, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                          length=length, mine=mine, tokens=tokens, group=group, residual=residual,
                          ragged=op == "cross" and rng.random() < 0.7, **bits)
    del case["name"]
    return case


# ---- inputs: made from the seed alone, the same for either form ----

def _generator(seed, part):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 64 + part)
    return gen


def _dtype(c):
    return torch.float16 if c["f16"] else torch.bfloat16


def _keys_values(c, gen, batch, tokens):
    """K and V of a layer pair: [2][batch, kv_heads, tokens, head_dim] each."""
    shape = (batch, c["kv_heads"], tokens, c["head_dim"])
    mult = torch.ones(c["kv_heads"], c["head_dim"], device="cuda")
    for h in range(c["kv_heads"]):
        mult[h, torch.randperm(c["head_dim"], generator=gen, device="cuda")[:3]] = 10.0
    k0 = torch.randn(shape, generator=gen, device="cuda").mul_(mult[None, :, None, :]).to(_dtype(c))
    v0 = torch.randn(shape, generator=gen, device="cuda").to(_dtype(c))
    near = [(x + 0.1 * torch.randn(shape, generator=gen, device="cuda")).to(_dtype(c)) for x in (k0, v0)]
    return [k0, near[0]], [v0, near[1]]


def _queries(c, seed):
    return torch.randn(LAYERS, c["tokens"], c["batch"], c["q_heads"], c["head_dim"], generator=_generator(seed, 1),
                       device="cuda").to(_dtype(c))


def _lengths(c, seed):
    """Tokens of each sequence that exist (int32, on the GPU), or None: all.  Few sequences are empty."""
    if not c["ragged"]:
        return None
    rng = np.random.default_rng(seed)
    n = [0 if rng.random() < 0.04 else max(1, round(c["length"] * (0.3 + 0.7 * rng.random()))) for _ in range(c["batch"])]
    n[int(rng.integers(c["batch"]))] = c["length"]
    return torch.tensor(n, dtype=torch.int32, device="cuda")


def _index(c, seed):
    """The source of each sequence of the result."""
    rng = np.random.default_rng(seed)
    B, n = c["batch"], c["take"]
    if c["place"] == "fork":  # every prompt as often as the others
        pick = [i * B // n if n >= B else i for i in range(n)]
    elif c["place"] == "compact":
        pick = sorted(rng.permutation(B)[:n].tolist())
    else:  # beams of four: one or two of them end, survivors go on in their own places and in those
        pick = list(range(B))
        for first in range(0, B, 4):
            slots = rng.permutation(4)
            ends = int(rng.integers(1, 3))
            for dead in slots[:ends]:
                pick[first + int(dead)] = first + int(slots[ends + int(rng.integers(4 - ends))])
    return torch.tensor(pick, dtype=torch.int32, device="cuda")


# ---- the quantizer (Eq. 1, 2, 12): fp32, one rounding for each operation ----

def _params(mn, mx, bits):
    top = (1 << bits) - 1
    s = (mx - mn) / torch.full_like(mn, float(top))
    eta = np.float32(ETA[bits])
    zero = mn + (s * float(eta)) * float(top)
    scale = s * float(np.float32(1.0) - np.float32(2.0) * eta)
    return s, scale.half(), zero.half()


def _codes(x, mn, s, bits):
    code = torch.where(s > 0, (x - mn) / torch.where(s > 0, s, torch.ones_like(s)), torch.zeros_like(x))
    return code.round_().clamp_(0, (1 << bits) - 1).to(torch.uint8)


def _quantize(c, K, V, lent=None):
    """A layer's cache: codes (those of `lent` where it shares that layer's), scales and zero-points, window."""
    B, H, S, D = K.shape
    g, R = c["group"], c["residual"]
    r = (S - 1) % R + 1 if S else 0
    n = S - r
    x = K[:, :, :n].float().view(B, H, n // g, g, D)
    mn, mx = x.amin(3, keepdim=True), x.amax(3, keepdim=True)
    s, ks, kz = _params(mn, mx, c["kbits"])
    out = dict(ks=ks[:, :, :, 0], kz=kz[:, :, :, 0])
    out["kc"] = lent["kc"] if lent else _codes(x, mn, s, c["kbits"]).view(B, H, n, D)
    x = V[:, :, :n].float().view(B, H, n, D // g, g)
    mn, mx = x.amin(4, keepdim=True), x.amax(4, keepdim=True)
    s, vs, vz = _params(mn, mx, c["vbits"])
    out.update(vs=vs[..., 0], vz=vz[..., 0])
    out["vc"] = lent["vc"] if lent else _codes(x, mn, s, c["vbits"]).view(B, H, n, D)
    out.update(wk=K[:, :, n:].contiguous(), wv=V[:, :, n:].contiguous())
    return out


def _pair(c, K, V):
    first = _quantize(c, K[0], V[0])
    return [first, _quantize(c, K[1], V[1], lent=first)]


# ---- the cache in the library's layout (csrc/xq_layout.cuh): bytes of each stream, [batch * kv_heads, bytes] ----

def _packed(c, layer, owner):
    """The regions of a layer in the library's order; an owner's begin with its codes."""
    B, H, n, D = layer["kc"].shape
    S, g = B * H, c["group"]
    flat = lambda x: x.contiguous().view(torch.uint8).reshape(S, x.numel() * x.element_size() // S)  # noqa: E731
    out = []
    if owner:
        bits = c["kbits"]
        per, width = 32 // bits, min(16, D * bits // 8)  # codes of a word (channel d of a row in byte d % 4); bytes of a chunk
        x = layer["kc"].reshape(S, n, D // per, per // 4, 4)
        row = sum(x[:, :, :, j] << (bits * j) for j in range(per // 4))
        out.append(flat(row.reshape(S, n // 32, 32, D * bits // 8 // width, width).transpose(2, 3)))
        bits = c["vbits"]
        per, nb = 32 // bits, (n + 127) // 128
        x = torch.nn.functional.pad(layer["vc"].reshape(S, n, D), (0, 0, 0, nb * 128 - n))
        x = x.reshape(S, nb, 128 // per, per // 4, 4, D)
        row = sum(x[:, :, :, j] << (bits * j) for j in range(per // 4))  # [stream, batch, word, byte, channel]
        row = row.permute(0, 1, 4, 2, 3).reshape(S, nb, D, bits, 16)
        out.append(flat(row.transpose(2, 3)))
    order = lambda x: x.reshape(S, n // g, D // 32, 32).transpose(2, 3).reshape(S, n // g, D)  # noqa: E731
    out.append(flat(torch.stack([order(layer["ks"]), order(layer["kz"])], 2)))
    out.append(flat(torch.stack([layer["vs"], layer["vz"]], 3)))
    return out + [flat(layer["wk"]), flat(layer["wv"])]


# ---- what a program has in hand ----

def _config(c, layers, batch, q_heads, max_seq):
    import paper_2510_11236_b200 as xq
    return xq.make_config(n_layers=layers, batch=batch, n_q_heads=q_heads, n_kv_heads=c["kv_heads"],
                          head_dim=c["head_dim"], max_seq=max_seq, group_size=c["group"], residual_len=c["residual"],
                          kq=layers if c["kbits"] == 2 else 0, vq=layers if c["vbits"] == 2 else 0, eta1=ETA[1],
                          eta2=ETA[2], io_dtype=xq.XQ_F16 if c["f16"] else xq.XQ_BF16)


def _cache(c, layers, batch, q_heads, max_seq, K=None, V=None):
    import paper_2510_11236_b200 as xq
    cache = xq.Cache(_config(c, layers, batch, q_heads, max_seq))
    cache.workspace.zero_()  # what no token has reached reads as zero
    if K is not None and K[0].shape[2]:
        for layer in range(layers):
            cache.append_kv(layer, K[layer % 2], V[layer % 2])
    return cache


def _views(c, cache, layers):
    """The used bytes of every region, [layers / 2, streams, bytes]: the even layers' six kinds, then the odd layers' four
    that are their own."""
    import paper_2510_11236_b200 as xq
    S, D, g, R = c["length"], c["head_dim"], c["group"], c["residual"]
    r = (S - 1) % R + 1
    n = S - r
    used = [n * D * c["kbits"] // 8, (n + 127) // 128 * 16 * D * c["vbits"], n // g * 4 * D, n * 4 * (D // g), 2 * r * D,
            2 * r * D]
    views = []
    for first, which in [(0, w) for w in range(6)] + [(1, w) for w in range(2, 6)]:
        place = [xq.xq_region(cache.handle, layer, which) for layer in range(first, layers, 2)]
        step = place[1][1] - place[0][1] if len(place) > 1 else 0
        assert all(p[0] == 0 and p[1] == place[0][1] + i * step for i, p in enumerate(place))
        streams = cache.cfg.batch * cache.cfg.n_kv_heads
        views.append(torch.as_strided(cache.workspace, (len(place), streams, used[which]), (step, place[0][2], 1), place[0][1]))
    return views


def prepare(case, seed):
    c = case
    state = dict(case=c)
    if c["op"] == "gather":
        K, V = _keys_values(c, _generator(seed, 0), c["batch"], c["length"])
        state["index"] = _index(c, seed)
        L, heads = c["layers"], c["kv_heads"]
        if own:
            state["source"] = source = _cache(c, L, c["batch"], heads, c["length"] + 64, K, V)
            state["cache"] = source if c["place"] == "beams" else _cache(c, L, c["take"], heads, c["length"] + 64)
            state["views"] = _views(c, state["cache"], L)
        else:
            pair = _pair(c, K, V)
            packed = _packed(c, pair[0], True) + _packed(c, pair[1], False)
            state["source"] = [x[None].repeat(L // 2, 1, 1) for x in packed]
        torch.cuda.synchronize()
        return state
    batch = c["prefixes"] if c["op"] == "prefix" else c["batch"]
    K, V = _keys_values(c, _generator(seed, 0), batch, c["length"])
    state["q"] = _queries(c, seed)
    state["lengths"] = _lengths(c, seed) if c["op"] == "cross" else None
    mine = _keys_values(c, _generator(seed, 2), c["batch"], c["mine"]) if c["op"] == "prefix" else None
    if own:
        import paper_2510_11236_b200 as xq
        state["shared"] = shared = _cache(c, LAYERS, batch, c["q_heads"], c["length"], K, V)
        if c["op"] == "prefix":
            state["cache"] = _cache(c, LAYERS, c["batch"], c["q_heads"], c["mine"] + 64, *mine)
            need = xq.xq_prefix_workspace_bytes(state["cache"].handle, shared.handle, c["tokens"])
        else:
            need = xq.xq_cross_workspace_bytes(shared.handle, c["tokens"])
        state["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        state["out"] = torch.empty_like(state["q"])
    else:
        state["shared"] = _pair(c, K, V)
        state["cache"] = _pair(c, *mine) if c["op"] == "prefix" else None
    torch.cuda.synchronize()
    return state


# ---- one pass ----

def _restored(c, layer):
    """Keys and values of a layer in 32 bits: code * scale + zero-point, then the window."""
    g = c["group"]
    k = layer["kc"].float() * layer["ks"].float().repeat_interleave(g, 2) + layer["kz"].float().repeat_interleave(g, 2)
    v = layer["vc"].float() * layer["vs"].float().repeat_interleave(g, 3) + layer["vz"].float().repeat_interleave(g, 3)
    return torch.cat([k, layer["wk"].float()], 2), torch.cat([v, layer["wv"].float()], 2)


def _softmax(x):
    """exp(x - max) and its sum over the last axis; rows without a finite entry: zeros."""
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    return e, e.sum(-1, keepdim=True)


def _plain_prefix(c, shared, mine, q):
    T, B, Hq, D = q.shape
    P, H = c["prefixes"], c["kv_heads"]
    n, G = B // P, Hq // H
    x = q.float().view(T, P, n, H, G, D) / math.sqrt(D)
    kp, vp = _restored(c, shared)
    lp = x.permute(1, 3, 2, 0, 4, 5).reshape(P, H, n * T * G, D) @ kp.transpose(2, 3)  # [P, H, (n, T, G), length]
    lp = lp.view(P, H, n, T, G, -1)
    ko, vo = _restored(c, mine)
    S = ko.shape[2]
    lo = x.permute(1, 2, 3, 0, 4, 5).reshape(B, H, T * G, D) @ ko.transpose(2, 3)
    lo = lo.view(P, n, H, T, G, S).transpose(1, 2)
    seen = torch.arange(S, device=q.device)[None, :] <= S - T + torch.arange(T, device=q.device)[:, None]
    lo = lo.masked_fill(~seen[:, None, :], -math.inf)
    e, total = _softmax(torch.cat([lp, lo], -1))
    ep, eo = e[..., :lp.shape[-1]], e[..., lp.shape[-1]:]
    out = (ep.reshape(P, H, n * T * G, -1) @ vp).view(P, H, n, T, G, D)
    out = out + (eo.transpose(1, 2).reshape(B, H, T * G, S) @ vo).view(P, n, H, T, G, D).transpose(1, 2)
    return (out / total).permute(3, 0, 2, 1, 4, 5).reshape(T, B, Hq, D).to(q.dtype)


def _plain_cross(c, shared, q, lengths):
    T, B, Hq, D = q.shape
    H = c["kv_heads"]
    G = Hq // H
    k, v = _restored(c, shared)
    x = (q.float() / math.sqrt(D)).view(T, B, H, G, D).permute(1, 2, 0, 3, 4).reshape(B, H, T * G, D)
    logits = x @ k.transpose(2, 3)
    if lengths is not None:
        there = torch.arange(k.shape[2], device=q.device)[None, :] < lengths[:, None]
        logits.masked_fill_(~there[:, None, None, :], -math.inf)
    e, total = _softmax(logits)
    out = (e @ v) / torch.where(total > 0, total, torch.ones_like(total))
    return out.view(B, H, T, G, D).permute(2, 0, 1, 3, 4).reshape(T, B, Hq, D).to(q.dtype)


def _plain_gather(c, source, index):
    index = index.long()
    taken = []
    for x in source:
        L, streams, size = x.shape
        y = x.view(L, c["batch"], streams // c["batch"], size)[:, index].reshape(L, c["take"] * c["kv_heads"], size)
        if c["place"] == "beams":  # in place
            x.copy_(y)
            y = x
        taken.append(y)
    return taken


def run(state):
    c = state["case"]
    if c["op"] == "gather":
        if own:
            state["cache"].gather_sequences(state["source"], state["index"])
            return state["views"]
        return _plain_gather(c, state["source"], state["index"])
    outs = []
    for layer in range(LAYERS):
        q = state["q"][layer]
        if c["op"] == "prefix":
            if own:
                outs.append(state["cache"].prefix_attention(state["shared"], layer, q, out=state["out"][layer],
                                                            workspace=state["workspace"]))
            else:
                outs.append(_plain_prefix(c, state["shared"][layer], state["cache"][layer], q))
        elif own:
            outs.append(state["shared"].cross_attention(layer, q, lengths=state["lengths"], out=state["out"][layer],
                                                        workspace=state["workspace"]))
        else:
            outs.append(_plain_cross(c, state["shared"][layer], q, state["lengths"]))
    return outs


# ---- the definition in 64 bits: query by query head, over the tokens that the row sees ----

def _restored64(c, layer, b, h):
    g = c["group"]
    n, D = layer["kc"].shape[2:]
    at = torch.arange(n, device="cuda")
    ch = torch.arange(D, device="cuda")
    k = layer["kc"][b, h].double() * layer["ks"][b, h].double()[at // g] + layer["kz"][b, h].double()[at // g]
    v = layer["vc"][b, h].double() * layer["vs"][b, h].double()[:, ch // g] + layer["vz"][b, h].double()[:, ch // g]
    return torch.cat([k, layer["wk"][b, h].double()]), torch.cat([v, layer["wv"][b, h].double()])


def exact(case, seed):
    c = case
    if c["op"] == "gather":
        return None  # bytes: nothing is computed
    batch = c["prefixes"] if c["op"] == "prefix" else c["batch"]
    shared = _pair(c, *_keys_values(c, _generator(seed, 0), batch, c["length"]))
    mine = _pair(c, *_keys_values(c, _generator(seed, 2), c["batch"], c["mine"])) if c["op"] == "prefix" else None
    queries, lengths = _queries(c, seed), _lengths(c, seed) if c["op"] == "cross" else None
    lengths = lengths.tolist() if lengths is not None else None
    T, B, H = c["tokens"], c["batch"], c["kv_heads"]
    G, each = c["q_heads"] // H, B // batch
    outs = []
    for layer in range(LAYERS):
        out = torch.zeros(T, B, c["q_heads"], c["head_dim"], dtype=torch.float64, device="cuda")
        for h in range(H):
            for u in range(batch):
                kp, vp = _restored64(c, shared[layer], u, h)
                for b in range(u * each, (u + 1) * each):
                    if lengths is not None:
                        if lengths[b] == 0:
                            continue
                        kp, vp = kp[:lengths[b]], vp[:lengths[b]]
                    q = queries[layer, :, b, h * G:(h + 1) * G].double()  # [T, G, D]
                    k, v = kp, vp
                    if mine is not None:
                        ko, vo = _restored64(c, mine[layer], b, h)
                        k, v = torch.cat([kp, ko]), torch.cat([vp, vo])
                    logits = torch.einsum("tgd,sd->tgs", q, k) * c["head_dim"] ** -0.5
                    if mine is not None and c["mine"]:
                        for t in range(T - 1):
                            logits[t, :, k.shape[0] - (T - 1 - t):] = -math.inf
                    weight = torch.exp(logits - torch.logsumexp(logits, -1, keepdim=True))
                    out[:, b, h * G:(h + 1) * G] = torch.einsum("tgs,sd->tgd", weight, v)
        outs.append(out)
    return outs


# ---- what a pass cannot do without ----

def _cache_bytes(c, layers, batch, tokens):
    """A cache's bytes: codes once for each pair of layers, the rest for every layer."""
    D, g, R = c["head_dim"], c["group"], c["residual"]
    r = (tokens - 1) % R + 1 if tokens else 0
    n = tokens - r
    return batch * c["kv_heads"] * (layers // 2 * n * D * (c["kbits"] + c["vbits"]) // 8
                                    + layers * (n // g * 4 * D + n * 4 * (D // g) + 4 * r * D))


def work(case):
    c = case
    if c["op"] == "gather":
        if c["place"] == "beams":  # about three in eight are written; each is read from one that stays
            return {"bytes": int(2 * 0.375 * _cache_bytes(c, c["layers"], c["batch"], c["length"])), "flops": 0}
        read = min(c["batch"], c["take"])
        return {"bytes": _cache_bytes(c, c["layers"], read + c["take"], c["length"]), "flops": 0}
    T, B = c["tokens"], c["batch"]
    io = 4 * LAYERS * T * B * c["q_heads"] * c["head_dim"]
    part = 0.65 if c["ragged"] else 1.0
    seen = part * T * c["length"] + (sum(range(c["mine"] - T + 1, c["mine"] + 1)) if c["mine"] else 0)
    batch = c["prefixes"] if c["op"] == "prefix" else B
    size = part * _cache_bytes(c, LAYERS, batch, c["length"]) + _cache_bytes(c, LAYERS, B, c["mine"])
    return {"bytes": int(io + size), "flops": int(4 * LAYERS * B * c["q_heads"] * c["head_dim"] * seen)}
