"""Operators over caches that sequences have in common (prefix attention, cross attention, gathered sequences): refusals on the
host, and on the GPU the results against plain 64-bit attention over what the oracle's packing restores."""
import math

import numpy as np
import pytest
import torch

import paper_2510_11236_b200 as xq
from tests import util

DEV = "cuda:0"
KERNELS = [xq.XQ_KERNEL_GENERIC, xq.XQ_KERNEL_AUTO]
ETAS = dict(eta1=1 / 6, eta2=0.045)


def _config(**kw):
    base = dict(n_layers=2, batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, max_seq=1024, group_size=32,
                residual_len=64, km=0, vm=0, **ETAS)
    base.update(kw)
    return xq.make_config(**base)


# ---- host: refusals, workspace sizes ----

def _handle(**kw):
    rc, h = xq.xq_create(_config(**kw), 256, 1 << 50)
    assert rc == xq.XQ_OK
    return h


def test_prefix_refusals():
    c, p = _handle(batch=8), _handle(batch=2)
    A = 1 << 12
    call = lambda c=c, p=p, layer=0, q=A, out=A, n=1, w=A, size=1 << 40: xq.xq_prefix_attention(c, p, layer, q, out, n, w, size)  # noqa: E731
    assert call() == xq.XQ_ERR_ARG  # both empty
    for bad in (dict(layer=2), dict(layer=-1), dict(n=0), dict(n=-3), dict(q=0), dict(out=0), dict(q=A + 2), dict(out=A + 8)):
        assert call(**bad) == xq.XQ_ERR_ARG, bad
    assert call(c=None) == xq.XQ_ERR_ARG and call(p=None) == xq.XQ_ERR_ARG
    assert call(p=c) == xq.XQ_ERR_CONFIG
    for other in (dict(batch=3), dict(batch=2, n_layers=4), dict(batch=2, head_dim=64), dict(batch=2, n_q_heads=4),
                  dict(batch=2, n_kv_heads=4), dict(batch=2, io_dtype=xq.XQ_F16), dict(batch=2, sm_scale=0.1), dict(batch=16)):
        h = _handle(**other)
        assert call(p=h) == xq.XQ_ERR_CONFIG, other
        assert xq.xq_prefix_workspace_bytes(c, h, 1) == 0
        xq.xq_destroy(h)
    # what may differ
    h = _handle(batch=2, group_size=64, residual_len=128, kq=0, vq=0, km=2, vm=2, max_seq=77)
    assert call(p=h) == xq.XQ_ERR_ARG and xq.xq_prefix_workspace_bytes(c, h, 1) > 0
    for x in (c, p, h):
        xq.xq_destroy(x)


def test_cross_refusals():
    c = _handle()
    A = 1 << 12
    call = lambda layer=0, q=A, out=A, n=1, lengths=0, w=A, size=1 << 40: xq.xq_cross_attention(c, layer, q, out, n, lengths, w, size)  # noqa: E731
    assert call() == xq.XQ_ERR_ARG  # empty layer
    for bad in (dict(layer=2), dict(n=0), dict(q=0), dict(out=A + 4), dict(lengths=A + 2), dict(n=1 << 30)):
        assert call(**bad) == xq.XQ_ERR_ARG, bad
    assert xq.xq_cross_attention(None, 0, A, A, 1, 0, A, 1 << 40) == xq.XQ_ERR_ARG
    xq.xq_destroy(c)


def test_gather_refusals():
    src = _handle()
    A = 1 << 12
    for kw in (dict(n_layers=4), dict(n_kv_heads=4), dict(head_dim=64), dict(group_size=64), dict(residual_len=128), dict(kq=0),
               dict(vq=0), dict(km=2), dict(vm=2), dict(io_dtype=xq.XQ_F16), dict(share_dominant=1), dict(gamma1=0.4)):
        h = _handle(**kw)
        assert xq.xq_gather_sequences(h, src, A) == xq.XQ_ERR_CONFIG, kw
        xq.xq_destroy(h)
    assert xq.xq_gather_sequences(src, src, 0) == xq.XQ_ERR_ARG
    assert xq.xq_gather_sequences(src, src, A + 2) == xq.XQ_ERR_ARG
    assert xq.xq_gather_sequences(None, src, A) == xq.XQ_ERR_ARG and xq.xq_gather_sequences(src, None, A) == xq.XQ_ERR_ARG
    many = _handle(batch=1506, n_kv_heads=1, n_q_heads=1, max_seq=128)
    assert xq.xq_gather_sequences(many, many, A) == xq.XQ_ERR_CAPACITY
    for x in (src, many):
        xq.xq_destroy(x)


def test_workspace_bytes_bound_every_length():
    c, p = _handle(batch=8, max_seq=100000), _handle(batch=2, max_seq=100000)
    rows = 8 * 8
    one = xq.xq_prefix_workspace_bytes(c, p, 1)
    assert one >= rows * (2 * 128 * 4 + 8 + 4)
    assert xq.xq_prefix_workspace_bytes(c, p, 700) >= 700 * rows * (2 * 128 * 4 + 8 + 4)
    assert xq.xq_prefix_workspace_bytes(c, p, 0) == 0 and xq.xq_prefix_workspace_bytes(c, None, 1) == 0
    assert xq.xq_cross_workspace_bytes(c, 1) >= rows * (128 * 4 + 8)
    assert xq.xq_cross_workspace_bytes(c, 0) == 0 and xq.xq_cross_workspace_bytes(None, 1) == 0
    for x in (c, p):
        xq.xq_destroy(x)


# ---- inputs and the 64-bit reference ----

def _tokens(cfg, seed, S, batch=None, outliers=True):
    """K, V of a layer pair: bf16 or fp16 [2][batch, heads, S, D], three outlier key channels, second layer close to the first."""
    g = torch.Generator().manual_seed(seed)
    dtype = torch.float16 if cfg.io_dtype == xq.XQ_F16 else torch.bfloat16
    shape = (batch or cfg.batch, cfg.n_kv_heads, S, cfg.head_dim)
    k, v = torch.randn(shape, generator=g), torch.randn(shape, generator=g)
    if outliers:
        k[..., torch.randperm(cfg.head_dim, generator=g)[:3]] *= 10.0
    k1, v1 = (x + 0.1 * torch.randn(shape, generator=g) for x in (k, v))
    return [k.to(dtype), k1.to(dtype)], [v.to(dtype), v1.to(dtype)]


def _queries(cfg, seed, T, batch=None):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(T, batch or cfg.batch, cfg.n_q_heads, cfg.head_dim, generator=g)
    return q.to(torch.float16 if cfg.io_dtype == xq.XQ_F16 else torch.bfloat16)


def _filled(cfg, K, V):
    cache = xq.Cache(cfg, DEV)
    for layer in range(cfg.n_layers):
        if K[0].shape[2]:
            cache.append_kv(layer, K[layer % 2].to(DEV), V[layer % 2].to(DEV))
    return cache


def _restored(cfg, K, V, layer, b, h):
    """Keys and values of one stream in 64 bits, as the cache stands for them: code * scale + zero-point, then the window; and,
    of the same shapes, the size of the terms that the products add up: |scale (code - 1)| + |scale| + |zero|."""
    S, D, g = K[0].shape[2], cfg.head_dim, cfg.group_size
    if S == 0:
        return [np.zeros((0, D))] * 4
    oc = util.oracle_for_stream(cfg, [0, 1], b, h, {l: (K[l], V[l]) for l in (0, 1)})
    st = oc.layers[layer]
    n = oc.n_quantized(layer)
    k, v, ka, va = (np.zeros((S, D)) for _ in range(4))
    if n:
        kc, ks, kz, vc, vs, vz = (np.asarray(x[0, 0], dtype=np.float64) for x in oc.codes_and_meta(layer))
        ks, kz = np.repeat(ks, g, 0), np.repeat(kz, g, 0)
        vs, vz = np.repeat(vs, g, 1), np.repeat(vz, g, 1)
        k[:n], v[:n] = kc * ks + kz, vc * vs + vz
        ka[:n], va[:n] = (np.abs(kc - 1) + 1) * ks + np.abs(kz), (np.abs(vc - 1) + 1) * vs + np.abs(vz)
    k[n:], v[n:] = st["win_k"][0, 0], st["win_v"][0, 0]
    ka[n:], va[n:] = np.abs(k[n:]), np.abs(v[n:])
    return k, v, ka, va


def _reference(q, part, own, scale, seen_own, pairs):
    """Softmax attention of one query vector over `part` (all tokens) and the first seen_own of `own`; and how far the kernels may
    be off, channel by channel.

    Over `part`: numerators rounded to half precision, off by at most 2^-11 each, under their own sum: |sum w e (v - out)| <=
    2^-11 sum w |v - out|; pairs: to two halves, off by 2^-21 at most as far as the second one's subnormals reach, taken as 2^-18.  A logit: q as half precision relative to the row's largest element, below 2^-24 of it nothing is
    kept (sum 2^-25 max|q| |k|), and sums of fp32 that drop what lies below their last digit, one for each 16 products and
    the two of the bias: (D / 16 + 4) 2^-23 of the terms' sizes; an error d of the logits moves the result by at most
    2 d sum w |v - out|.  The value sums: one for each 16 tokens, twice at the join, 2^-23 of the terms' sizes each.
    Over `own`: the bound that the decode and chunk kernels are tested with, 2e-3, by that part's weight, and 1e-4 of its
    denominator, which moves the result by at most that times the two parts' distance."""
    k, v, ka, va = (np.concatenate([a, b[:seen_own]]) for a, b in zip(part, own))
    n, D = len(part[0]), len(q)
    if len(k) == 0:
        return np.zeros(D), np.zeros(D)
    x = scale * (k @ q)
    w = np.exp(x - x.max())
    w /= w.sum()
    out = w @ v
    spread = w @ np.abs(v - out)
    off = np.zeros(D)
    if n:
        d = scale * ((D // 16 + 4) * 2.0 ** -23 * (ka[:n] @ np.abs(q)).max() + 2.0 ** -25 * np.abs(q).max() * ka[:n].sum(1).max())
        steps = n / 16 + 8
        off += (2.0 ** (-18 if pairs else -11) + 2 * d) * spread + steps * 2.0 ** -23 * (w[:n] @ va[:n])
    if seen_own:
        share = w[n:].sum()
        off += 2e-3 * share
        if n:
            off += 1e-4 * share * np.abs(w[n:] @ v[n:] / max(share, 1e-300) - out)
    return out, off + 1e-6 * np.abs(out)


def _check(cfg, out32, out16, q, restore_part, restore_own, T, own_len, heads=None, batch=None, rows=0):
    """Every row of the sequences and heads (all, or those named) against the reference.  restore_*(b, h): the stream's tokens.
    rows: of a kv head, more than the decode kernels take: half precision then goes with pairs."""
    pairs = cfg.io_dtype == xq.XQ_F16 and rows > 16 * 8
    B, G = q.shape[1], cfg.n_q_heads // cfg.n_kv_heads
    scale = cfg.sm_scale if cfg.sm_scale > 0 else 1 / math.sqrt(cfg.head_dim)
    o32, o16, qd = out32.double().cpu().numpy(), out16.double().cpu().numpy(), q.double().cpu().numpy()
    half = torch.finfo(q.dtype).eps / 2
    worst = 0.0
    for b in range(B) if batch is None else batch:
        for h in range(cfg.n_kv_heads) if heads is None else heads:
            part, own = restore_part(b, h), restore_own(b, h)
            for j in range(T):
                for a in range(h * G, (h + 1) * G):
                    ref, off = _reference(qd[j, b, a], part, own, scale, max(0, own_len - T + j + 1), pairs)
                    err = np.abs(o32[j, b, a] - ref)
                    assert (err <= off).all(), (b, h, j, a, err.max(), off[err.argmax()])
                    assert (np.abs(o16[j, b, a] - ref) <= off + half * (np.abs(ref) + off) + 2.0 ** -25).all(), (b, h, j, a)
                    worst = max(worst, (err / np.maximum(off, 1e-30)).max())
    return worst


SHAPES = [
    # D, Hq, Hkv, g, R, kq, vq, f16
    (128, 8, 2, 32, 64, 2, 0, False),
    (128, 6, 2, 64, 64, 0, 2, True),
    (128, 2, 2, 32, 128, 2, 2, False),
    (64, 6, 2, 32, 32, 2, 2, False),
    (64, 4, 1, 64, 64, 0, 0, True),
    (128, 12, 1, 32, 32, 0, 0, False),   # more than eight heads on a kv head
    (64, 8, 2, 32, 64, 0, 2, True),
    (128, 5, 1, 64, 128, 2, 0, False),
]


def _shape(shape, **kw):
    D, Hq, Hkv, g, R, kq, vq, f16 = shape
    return _config(head_dim=D, n_q_heads=Hq, n_kv_heads=Hkv, group_size=g, residual_len=R, kq=kq, vq=vq,
                   io_dtype=xq.XQ_F16 if f16 else xq.XQ_BF16, **kw)


# ---- prefix attention ----

def _prefix_case(shape, kernel, P, each, Sp, S, T, seed=0, **more):
    cp = _shape(shape, batch=P, max_seq=max(Sp, 1), kernel=kernel, **more)
    cc = _shape(shape, batch=P * each, max_seq=max(S, 1) + 64, kernel=kernel, **more)
    kp, vp = _tokens(cp, seed + 1, Sp)
    ko, vo = _tokens(cc, seed + 2, S)
    prefix, cache = _filled(cp, kp, vp), _filled(cc, ko, vo)
    for layer in (0, 1):
        q = _queries(cc, seed + 3 + layer, T)
        o32 = cache.prefix_attention(prefix, layer, q.to(DEV), f32=True)
        o16 = cache.prefix_attention(prefix, layer, q.to(DEV))
        worst = _check(cc, o32, o16, q, lambda b, h: _restored(cp, kp, vp, layer, b // each, h),
                       lambda b, h: _restored(cc, ko, vo, layer, b, h), T, S, rows=T * each * cc.n_q_heads // cc.n_kv_heads)
        print(f"worst error / bound: {worst:.2f}")
    cache.check_device()


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("shape", SHAPES)
def test_prefix_one_token(shape, kernel):
    _prefix_case(shape, kernel, 1, 5, 333, 70, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("Sp,S", [(1, 1), (1, 0), (31, 3), (32, 33), (64, 1), (65, 65), (128, 0), (129, 17), (192, 200), (193, 1),
                                  (513, 129), (1500, 40)])
def test_prefix_lengths(kernel, Sp, S):
    _prefix_case(SHAPES[0], kernel, 1, 3, Sp, S, 1, seed=Sp)


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("shape", [SHAPES[1], SHAPES[3], SHAPES[5]])
def test_prefix_several_prompts(shape, kernel):
    _prefix_case(shape, kernel, 3, 2, 150, 40, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("shape,T", [(SHAPES[0], 2), (SHAPES[0], 33), (SHAPES[3], 40), (SHAPES[5], 3), (SHAPES[6], 20)])
def test_prefix_several_tokens(shape, kernel, T):
    _prefix_case(shape, kernel, 1, 2, 200, T + 30, T)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[3], SHAPES[7]])
@pytest.mark.parametrize("S,T", [(40, 1), (0, 1), (7, 3)])
def test_prefix_of_its_own(shape, S, T):
    # a prompt for every sequence: as many caches as sequences
    _prefix_case(shape, xq.XQ_KERNEL_AUTO, 3, 1, 333, S, T)


@pytest.mark.gpu
@pytest.mark.parametrize("Sp,S,T", [(700, 33, 1), (50, 9, 3), (129, 0, 1)])
@pytest.mark.parametrize("shape,P,each", [(SHAPES[2], 1, 8), (SHAPES[2], 2, 3), (SHAPES[0], 2, 2), (SHAPES[3], 3, 2), (SHAPES[4], 1, 2),
                                          ((64, 2, 2, 32, 32, 0, 2, False), 2, 4)])
def test_prefix_few_rows(shape, P, each, Sp, S, T):
    # at most eight rows of a kv head: the decode kernels, several sequences' heads on one cache
    _prefix_case(shape, xq.XQ_KERNEL_AUTO, P, each, Sp, S, T)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[6]])
def test_prefix_behind_long_tails(shape):
    # the sequences' own tokens in several splits: one token (decode kernels) and twenty (chunk kernel)
    _prefix_case(shape, xq.XQ_KERNEL_AUTO, 1, 2, 100, 1500, 1)
    _prefix_case(shape, xq.XQ_KERNEL_AUTO, 1, 2, 100, 1500, 20)


@pytest.mark.gpu
def test_prefix_more_rows_than_a_tile():
    # 3 sequences x 20 tokens x 4 heads = 240 rows; 23 x 12 = 276
    _prefix_case(SHAPES[0], xq.XQ_KERNEL_AUTO, 1, 3, 300, 20, 20)
    _prefix_case(SHAPES[5], xq.XQ_KERNEL_AUTO, 1, 23, 100, 2, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [SHAPES[1], SHAPES[4], SHAPES[6]])
def test_half_precision_in_pairs(shape):
    # more than 128 rows of a kv head, which no decode kernel takes; the prompt alone: its own tokens have a wider bound
    _prefix_case(shape, xq.XQ_KERNEL_AUTO, 1, 3, 700, 0, 60)
    _cross_case(shape, xq.XQ_KERNEL_AUTO, 2, 333, 70, lengths=[333, 140])


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("each", [1, 2, 40])  # decode kernels, rows kernel
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[6]])
def test_query_that_is_not_a_number(shape, each, kernel):
    # its rows are not numbers, the others are as if it were one
    cp, cc = _shape(shape, batch=1, max_seq=300, kernel=kernel), _shape(shape, batch=each, max_seq=40, kernel=kernel)
    prefix, cache = _filled(cp, *_tokens(cp, 1, 300)), _filled(cc, *_tokens(cc, 2, 40))
    alone = xq.Cache(cc, DEV)
    q = _queries(cc, 3, 1).to(DEV)
    bad = q.clone()
    bad[0, each - 1, 5] = float("nan")
    mine = torch.zeros(q.shape[:3], dtype=torch.bool, device=DEV)
    mine[0, each - 1, 5] = True
    for call in (lambda q: cache.prefix_attention(prefix, 0, q, f32=True), lambda q: alone.prefix_attention(prefix, 0, q, f32=True)):
        want, got = call(q), call(bad)
        assert got[mine].isnan().all()
        assert torch.equal(got[~mine], want[~mine])


@pytest.mark.gpu
@pytest.mark.parametrize("shape,each", [(SHAPES[0], 2), (SHAPES[3], 2), (SHAPES[7], 1), (SHAPES[4], 1),
                                        (SHAPES[0], 12), (SHAPES[7], 8), (SHAPES[4], 9), (SHAPES[5], 2)])  # (rows kernel)
@pytest.mark.parametrize("T", [1, 2])
def test_prefix_calls_one_after_the_other(shape, each, T):
    # launches of a call and of the next one overlap: each call's result is that of the call by itself, eager and from a graph
    cp, cc = _shape(shape, batch=3, max_seq=900), _shape(shape, batch=3 * each, max_seq=300)
    prefix, cache = _filled(cp, *_tokens(cp, 1, 900)), _filled(cc, *_tokens(cc, 2, 270))
    qs = [_queries(cc, 10 + i, T).to(DEV) for i in range(12)]
    work = torch.empty(xq.xq_prefix_workspace_bytes(cache.handle, prefix.handle, T), dtype=torch.uint8, device=DEV)
    want = []
    for i, q in enumerate(qs):
        want.append(cache.prefix_attention(prefix, i % 2, q, f32=True, workspace=work))
        torch.cuda.synchronize()
    outs = [torch.empty_like(w) for w in want]

    def run():
        for i, q in enumerate(qs):
            cache.prefix_attention(prefix, i % 2, q, out=outs[i], f32=True, workspace=work)
    for _ in range(20):
        for o in outs:
            o.zero_()
        run()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(20):
        for o in outs:
            o.zero_()
        graph.replay()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    cache.check_device()


@pytest.mark.gpu
def test_prefix_empty_is_chunk_attention():
    cfg = _config(batch=2)
    K, V = _tokens(cfg, 1, 100)
    cache, prefix = _filled(cfg, K, V), xq.Cache(_config(batch=1), DEV)
    q = _queries(cfg, 2, 30).to(DEV)
    assert torch.equal(cache.prefix_attention(prefix, 1, q), cache.attention_chunk(1, q))


# ---- cross attention ----

def _cross_case(shape, kernel, B, S, T, lengths=None, seed=0, fill=None):
    cfg = _shape(shape, batch=B, max_seq=S, kernel=kernel)
    K, V = _tokens(cfg, seed + 1, S)
    cache = _filled(cfg, K, V)
    if fill:
        fill(cache)
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    n = [S] * B if lengths is None else [min(max(x, 0), S) for x in lengths]
    for layer in (0, 1):
        q = _queries(cfg, seed + 3 + layer, T)
        o32 = cache.cross_attention(layer, q.to(DEV), lengths=ln, f32=True)
        o16 = cache.cross_attention(layer, q.to(DEV), lengths=ln)
        part = lambda b, h: [x[:n[b]] for x in _restored(cfg, K, V, layer, b, h)]  # noqa: E731
        none = [np.zeros((0, cfg.head_dim))] * 4
        worst = _check(cfg, o32, o16, q, part, lambda b, h: none, T, 0, rows=T * cfg.n_q_heads // cfg.n_kv_heads)
        print(f"worst error / bound: {worst:.2f}")
    cache.check_device()


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("T", [3, 17])  # few tokens go to the decode kernels, one by one
@pytest.mark.parametrize("shape", SHAPES)
def test_cross_shapes(shape, T, kernel):
    _cross_case(shape, kernel, 3, 275, T, lengths=[275, 100, 17])


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("T", [1, 18])
@pytest.mark.parametrize("S", [1, 2, 63, 64, 65, 128, 129, 191, 193, 257, 700])
def test_cross_all_tokens(kernel, S, T):
    _cross_case(SHAPES[0], kernel, 2, S, T, seed=S)


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("lengths", [[0, 0, 0, 0], [0, 1, 400, 399], [31, 32, 33, 63], [64, 65, 127, 128], [-5, 401, 2 ** 31 - 1, -2 ** 31],
                                     [384, 385, 383, 200]])
@pytest.mark.parametrize("shape,T", [(SHAPES[0], 2), (SHAPES[0], 17), (SHAPES[6], 1), (SHAPES[1], 1)])
def test_cross_lengths(kernel, lengths, shape, T):
    _cross_case(shape, kernel, 4, 400, T, lengths=lengths)


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("T", [2, 17])
def test_cross_masked_tokens_that_are_not_finite(kernel, bad, T):
    # what lies behind a sequence's length reaches nothing: window rows and the packed tokens' parameters
    shape, S = SHAPES[0], 300

    def fill(cache):
        h = {float("nan"): 0x7e00}.get(bad, 0x7c00 if bad > 0 else 0xfc00) if bad == bad else 0x7e00
        for layer in (0, 1):
            for which, row in ((4, 2 * 128), (5, 2 * 128)):
                w = cache.region(layer, which).view(torch.bfloat16).view(3, 2, -1, 128)
                w[1:, :, :] = bad            # sequences 1 and 2 end before the window
            v = cache.region(layer, 3).view(torch.int16).view(3, 2, -1, 8)
            v[2, :, 70:] = h - 65536 if h >= 32768 else h
            k = cache.region(layer, 2).view(torch.int16).view(3, 2, -1, 256)
            k[2, :, 3:] = h - 65536 if h >= 32768 else h  # token groups from 96 on
    _cross_case(shape, kernel, 3, S, T, lengths=[300, 256, 70], fill=fill)


@pytest.mark.gpu
def test_cross_many_rows():
    _cross_case(SHAPES[2], xq.XQ_KERNEL_AUTO, 1, 260, 300)
    _cross_case(SHAPES[0], xq.XQ_KERNEL_AUTO, 2, 130, 65, lengths=[130, 41])


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,f16,ragged", [(16, 40, False, True), (6, 40, False, False), (13, 33, True, True), (40, 33, False, False)])
def test_cross_more_tiles_than_half_the_device(B, T, f16, ragged):
    # several waves of CTAs.  Some streams against the reference, all against the scalar kernel: off by at most 2^-11 of the
    # values' spread, and by little more.
    kw = dict(batch=B, n_q_heads=32, n_kv_heads=8, max_seq=700, vq=0, io_dtype=int(f16))
    cfg, other = _config(**kw), _config(kernel=xq.XQ_KERNEL_GENERIC, **kw)
    K, V = _tokens(cfg, B, 700)
    cache, slow = _filled(cfg, K, V), _filled(other, K, V)
    n = np.random.default_rng(B).integers(0, 701, B) if ragged else np.full(B, 700)
    n[0], n[1] = (0, 700) if ragged else (700, 700)
    lengths = torch.tensor(n, dtype=torch.int32, device=DEV) if ragged else None
    q = _queries(cfg, 3, T)
    o32, o16 = cache.cross_attention(1, q.to(DEV), lengths=lengths, f32=True), cache.cross_attention(1, q.to(DEV), lengths=lengths)
    want = slow.cross_attention(1, q.to(DEV), lengths=lengths, f32=True)
    assert (o32 - want).abs().max() <= 2.0 ** -11 * 2 * V[1].abs().max().item() * 1.1
    none = [np.zeros((0, 128))] * 4
    for b, h in ((1, 0), (B - 1, 7), (B // 2, 3)):
        _check(cfg, o32, o16, q, lambda b, h: [x[:n[b]] for x in _restored(cfg, K, V, 1, b, h)], lambda b, h: none, T, 0, heads=[h], batch=[b], rows=4 * T)
    cache.check_device()


@pytest.mark.gpu
@pytest.mark.parametrize("B", [1, 3, 31, 32, 33])
@pytest.mark.parametrize("kind", ["equal", "none", "two", "rising", "out of range"])
def test_cross_order_of_lengths(B, kind):
    # more CTAs than the device takes at once: they go by length, up to 32 sequences.  Against the scalar kernel, as above.
    T, S = 8000 // B, 300
    kw = dict(batch=B, n_q_heads=4, n_kv_heads=2, max_seq=S)
    cfg, other = _config(**kw), _config(kernel=xq.XQ_KERNEL_GENERIC, **kw)
    K, V = _tokens(cfg, B, S)
    cache, slow = _filled(cfg, K, V), _filled(other, K, V)
    n = {"equal": [S] * B, "none": [0] * B, "two": [S if b % 3 else 65 for b in range(B)], "rising": [1 + b * 9 for b in range(B)],
         "out of range": [[-7, 2 ** 31 - 1, -2 ** 31, 128][b % 4] for b in range(B)]}[kind]
    lengths = torch.tensor(n, dtype=torch.int32, device=DEV)
    q = _queries(cfg, 3, T).to(DEV)
    got, want = (c.cross_attention(0, q, lengths=lengths, f32=True) for c in (cache, slow))
    assert (got - want).abs().max() <= 2.0 ** -11 * 2 * V[0].abs().max().item() * 1.1
    for b in range(B):
        if n[b] <= 0:
            assert not got[:, b].any()
    cache.check_device()


@pytest.mark.gpu
@pytest.mark.parametrize("shape,P", [(SHAPES[0], 1), (SHAPES[3], 5)])
def test_prefix_more_tiles_than_half_the_device(shape, P):
    # 8 sequences of 40 tokens behind each prompt, eight kv heads
    D, Hq, Hkv, g, R, kq, vq, f16 = shape
    shape = (D, 32, 8, g, R, kq, vq, f16)
    cp, cc = _shape(shape, batch=P, max_seq=900), _shape(shape, batch=8 * P, max_seq=80)
    kp, vp = _tokens(cp, 1, 900)
    ko, vo = _tokens(cc, 2, 55)
    prefix, cache = _filled(cp, kp, vp), _filled(cc, ko, vo)
    q = _queries(cc, 3, 40)
    o32, o16 = cache.prefix_attention(prefix, 0, q.to(DEV), f32=True), cache.prefix_attention(prefix, 0, q.to(DEV))
    for b, h in ((0, 0), (8 * P - 1, 7), (3, 5)):
        _check(cc, o32, o16, q, lambda b, h: _restored(cp, kp, vp, 0, b // 8, h), lambda b, h: _restored(cc, ko, vo, 0, b, h), 40, 55,
               heads=[h], batch=[b])
    # without own tokens
    alone = xq.Cache(cc, DEV)
    o32, o16 = alone.prefix_attention(prefix, 1, q.to(DEV), f32=True), alone.prefix_attention(prefix, 1, q.to(DEV))
    none = [np.zeros((0, D))] * 4
    for b, h in ((0, 0), (8 * P - 1, 7), (3, 5)):
        _check(cc, o32, o16, q, lambda b, h: _restored(cp, kp, vp, 1, b // 8, h), lambda b, h: none, 40, 0, heads=[h], batch=[b])
    cache.check_device()


# ---- gathered sequences ----

def _sequence_bytes(cache, cfg, S):
    """{(layer, region): [batch, kv heads, used bytes]} of what the tokens occupy (a copy); of the value codes whole words."""
    D, g, R = cfg.head_dim, cfg.group_size, cfg.residual_len
    r = (S - 1) % R + 1 if S else 0
    n = S - r
    out = {}
    for layer in range(cfg.n_layers):
        bk, bv = 2 if layer < cfg.kq else 1, 2 if layer < cfg.vq else 1
        used = [n * D * bk // 8, -(-n // 128) * 16 * D * bv, n // g * 4 * D, n * 4 * (D // g), 2 * r * D, 2 * r * D]
        for which in range(6):
            x = cache.region(layer, which)[:, :used[which]].reshape(cfg.batch, cfg.n_kv_heads, -1).clone()
            out[layer, which] = x
    return out


def _cleared(cfg, K, V):
    cache = xq.Cache(cfg, DEV)
    cache.workspace.zero_()
    for layer in range(cfg.n_layers):
        if K[0].shape[2]:
            K1, V1 = (x[layer % 2].to(DEV) + (layer // 2) * 0.25 for x in (K, V))  # other values in every pair
            cache.append_kv(layer, K1, V1)
    return cache


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("S", [1, 128, 301])
def test_gather_to_another_cache(shape, S):
    src_cfg, dst_cfg = _shape(shape, batch=3, n_layers=2, max_seq=S), _shape(shape, batch=5, n_layers=2, max_seq=S + 200)
    src = _cleared(src_cfg, *_tokens(src_cfg, 1, S))
    dst = xq.Cache(dst_cfg, DEV)
    dst.workspace.fill_(0xa5)
    index = torch.tensor([2, 2, 0, 1, 2], dtype=torch.int32, device=DEV)
    before = dst.workspace.clone()
    dst.gather_sequences(src, index)
    dst.check_device()
    assert all(dst.seq_len(l) == S for l in (0, 1))
    want, got = _sequence_bytes(src, src_cfg, S), _sequence_bytes(dst, dst_cfg, S)
    for key in want:
        assert torch.equal(got[key], want[key][index.long()]), key
    # what was not written is as it was: everything behind the used bytes of every stream
    mask = torch.zeros_like(dst.workspace, dtype=torch.bool)
    for layer in (0, 1):
        for which in range(6):
            rc, off, stride = xq.xq_region(dst.handle, layer, which)
            n = got[layer, which].shape[2]
            torch.as_strided(mask, (5 * dst_cfg.n_kv_heads, n), (stride, 1), off).fill_(True)
    changed = dst.workspace != before
    rc, first, stride = xq.xq_region(dst.handle, 0, 4)
    regions = max(xq.xq_region(dst.handle, l, w)[1] + xq.xq_region(dst.handle, l, w)[2] * 5 * dst_cfg.n_kv_heads
                  for l in (0, 1) for w in range(6))
    assert not (changed & ~mask)[:regions].any()
    src.close(), dst.close()


@pytest.mark.gpu
@pytest.mark.parametrize("B", [1, 4, 130, 450])
@pytest.mark.parametrize("kind", ["permutation", "cycle", "one", "beams", "same"])
def test_gather_in_place(B, kind):
    S = 200
    cfg = _config(batch=B, n_layers=4, n_q_heads=2, n_kv_heads=2, head_dim=64, max_seq=256, vq=0, kq=4)
    cache = _cleared(cfg, *_tokens(cfg, 1, S))
    rng = np.random.default_rng(B)
    index = dict(permutation=rng.permutation(B), cycle=np.roll(np.arange(B), 1), one=np.full(B, B - 1),
                 beams=rng.integers(0, B, B), same=np.arange(B))[kind]
    index = torch.tensor(index, dtype=torch.int32, device=DEV)
    want = _sequence_bytes(cache, cfg, S)
    cache.gather_sequences(cache, index)
    cache.check_device()
    got = _sequence_bytes(cache, cfg, S)
    for key in want:
        assert torch.equal(got[key], want[key][index.long()]), key


@pytest.mark.gpu
def test_gather_more_layers_than_a_launch():
    cfg = _config(batch=2, n_layers=70, n_q_heads=1, n_kv_heads=1, head_dim=64, max_seq=200, residual_len=32, kq=70, vq=70)
    src, dst = _cleared(cfg, *_tokens(cfg, 1, 150)), xq.Cache(cfg, DEV)
    dst.workspace.zero_()
    index = torch.tensor([1, 0], dtype=torch.int32, device=DEV)
    dst.gather_sequences(src, index)
    want, got = _sequence_bytes(src, cfg, 150), _sequence_bytes(dst, cfg, 150)
    for key in want:
        assert torch.equal(got[key], want[key][index.long()]), key


@pytest.mark.gpu
@pytest.mark.parametrize("place", [False, True])
def test_gather_index_out_of_range(place):
    cfg = _config(batch=4, max_seq=300)
    src = _cleared(cfg, *_tokens(cfg, 1, 200))
    dst = src if place else _cleared(cfg, *_tokens(cfg, 2, 200))
    was, want = _sequence_bytes(dst, cfg, 200), _sequence_bytes(src, cfg, 200)
    dst.gather_sequences(src, torch.tensor([3, -1, 4, 0], dtype=torch.int32, device=DEV))
    with pytest.raises(xq.XQError) as e:
        dst.check_device()
    assert e.value.code == xq.XQ_ERR_DEVICE
    got = _sequence_bytes(dst, cfg, 200)
    for key in want:
        assert torch.equal(got[key][0], want[key][3]) and torch.equal(got[key][3], want[key][0]), key
        assert torch.equal(got[key][1:3], was[key][1:3]), key


@pytest.mark.gpu
def test_gather_layers_of_different_length_and_empty():
    # a pair's second layer one block behind, another pair empty
    cfg = _config(batch=2, n_layers=4, max_seq=400)
    K, V = _tokens(cfg, 1, 200)
    src, dst = xq.Cache(cfg, DEV), xq.Cache(_config(batch=3, n_layers=4, max_seq=500), DEV)
    src.append_kv(0, K[0].to(DEV), V[0].to(DEV))
    src.append_kv(1, K[1][:, :, :130].contiguous().to(DEV), V[1][:, :, :130].contiguous().to(DEV))
    dst.gather_sequences(src, torch.tensor([1, 0, 1], dtype=torch.int32, device=DEV))
    assert [dst.seq_len(l) for l in range(4)] == [200, 130, 0, 0]
    q = _queries(cfg, 5, 1)[0]
    for layer in (0, 1):
        a = src.decode_attention(layer, q.to(DEV))
        b = dst.decode_attention(layer, q[[1, 0, 1]].to(DEV))
        assert torch.equal(b, a[[1, 0, 1]])
    short = xq.Cache(_config(batch=2, n_layers=4, max_seq=199), DEV)
    with pytest.raises(xq.XQError) as e:
        short.gather_sequences(src, torch.tensor([1, 0], dtype=torch.int32, device=DEV))
    assert e.value.code == xq.XQ_ERR_CAPACITY and short.seq_len(0) == 0


# ---- a run of them together ----

@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
def test_prompt_shared_and_forked(kernel):
    """Three answers to one prompt, six tokens each, with a beam replaced midway: once over the shared prompt, once with the prompt
    forked into every sequence; both give attention over the same tokens."""
    Sp, steps = 200, 6
    one, three = _config(batch=1, max_seq=300, kernel=kernel), _config(batch=3, max_seq=300, kernel=kernel)
    kp, vp = _tokens(one, 1, Sp)
    prefix = _filled(one, kp, vp)
    mine, forked = xq.Cache(three, DEV), xq.Cache(three, DEV)
    forked.gather_sequences(prefix, torch.zeros(3, dtype=torch.int32, device=DEV))
    ks, vs = _tokens(three, 2, steps)
    index = torch.tensor([0, 2, 2], dtype=torch.int32, device=DEV)
    kept = [[x[:, :, :0] for x in ks], [x[:, :, :0] for x in vs]]
    for t in range(steps):
        if t == 3:
            mine.gather_sequences(mine, index)
            forked.gather_sequences(forked, index)
            kept = [[x[index.cpu().long()] for x in y] for y in kept]
        kept = [[torch.cat([x, n[:, :, t:t + 1]], 2) for x, n in zip(y, new)] for y, new in zip(kept, (ks, vs))]
        for layer in (0, 1):
            new = [x[layer][:, :, t:t + 1].contiguous().to(DEV) for x in (ks, vs)]
            mine.append_kv(layer, *new)
            forked.append_kv(layer, *new)
            q = _queries(three, 10 + t, 1)
            shared = mine.prefix_attention(prefix, layer, q.to(DEV), f32=True)
            shared16 = mine.prefix_attention(prefix, layer, q.to(DEV))
            _check(three, shared, shared16, q, lambda b, h: _restored(one, kp, vp, layer, 0, h),
                   lambda b, h: _restored(three, *kept, layer, b, h), 1, t + 1)
            # the forked sequences hold all tokens themselves: the prompt's last block is still 16-bit in both
            alone = forked.decode_attention(layer, q[0].to(DEV), f32=True)
            assert (alone - shared[0]).abs().max() < 4e-3  # 2e-3 for either kernel
    mine.check_device(), forked.check_device()


@pytest.mark.gpu
def test_calls_on_other_streams_and_in_a_graph():
    one, four = _config(batch=1, max_seq=500), _config(batch=4, max_seq=300)
    prefix, cache = _filled(one, *_tokens(one, 1, 400)), _filled(four, *_tokens(four, 2, 90))
    q = _queries(four, 3, 1).to(DEV)
    lengths = torch.tensor([90, 0, 5, 77], dtype=torch.int32, device=DEV)
    want = [cache.prefix_attention(prefix, 1, q), cache.cross_attention(1, q, lengths=lengths)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [cache.prefix_attention(prefix, 1, q), cache.cross_attention(1, q, lengths=lengths)]
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    space = torch.empty(max(xq.xq_prefix_workspace_bytes(cache.handle, prefix.handle, 1), xq.xq_cross_workspace_bytes(cache.handle, 1)),
                        dtype=torch.uint8, device=DEV)
    outs = [torch.empty_like(x) for x in want]
    spare = xq.Cache(four, DEV)
    index = torch.tensor([1, 1, 3, 0], dtype=torch.int32, device=DEV)
    spare.gather_sequences(cache, index)
    spare.check_device()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.prefix_attention(prefix, 1, q, out=outs[0], workspace=space)
        cache.cross_attention(1, q, lengths=lengths, out=outs[1], workspace=space)
        spare.gather_sequences(cache, index)
    for k in range(3):  # replayed with other inputs in the same places
        q.copy_(_queries(four, 20 + k, 1))
        lengths.copy_(torch.tensor([k, 90 - k, 64, 33], dtype=torch.int32))
        index.copy_(torch.tensor([k, 0, 3 - k, 2], dtype=torch.int32))
        spare.workspace[:1 << 16].random_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], cache.prefix_attention(prefix, 1, q))
        assert torch.equal(outs[1], cache.cross_attention(1, q, lengths=lengths))
        x = _queries(four, 30, 1)[0].to(DEV)
        assert torch.equal(spare.decode_attention(0, x[index.long()].contiguous()), cache.decode_attention(0, x)[index.long()])
    cache.check_device()


@pytest.mark.gpu
def test_first_call_of_a_handle_in_a_graph_that_never_runs():
    # the handle's counters are cleared by a first call; one that is only captured does not count
    cfg = _config(batch=2, max_seq=2000)
    K, V = _tokens(cfg, 1, 1500)
    q = _queries(cfg, 2, 1).to(DEV)
    want = _filled(cfg, K, V).cross_attention(0, q)
    cache = _filled(cfg, K, V)
    cache.workspace[xq.xq_region(cache.handle, 1, 3)[1] + xq.xq_region(cache.handle, 1, 3)[2] * 4:].fill_(0xff)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.cross_attention(0, q)
    assert torch.equal(cache.cross_attention(0, q), want)
    cache.check_device()


@pytest.mark.gpu
def test_refused_calls_change_nothing():
    one, four = _config(batch=1, max_seq=500), _config(batch=4, max_seq=300)
    prefix, cache = _filled(one, *_tokens(one, 1, 400)), _filled(four, *_tokens(four, 2, 90))
    q, out = _queries(four, 3, 1).to(DEV), torch.full((1, 4, 8, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    n = xq.xq_launch_count(cache.handle)
    small = torch.empty(256, dtype=torch.uint8, device=DEV)
    for call in (lambda: cache.prefix_attention(prefix, 0, q, out=out, workspace=small),
                 lambda: cache.cross_attention(0, q, out=out, workspace=small)):
        with pytest.raises(xq.XQError) as e:
            call()
        assert e.value.code == xq.XQ_ERR_CAPACITY
    with pytest.raises(xq.XQError) as e:
        cache.prefix_attention(prefix, 0, _queries(four, 3, 91).to(DEV))
    assert e.value.code == xq.XQ_ERR_ARG
    for bad in (lambda: cache.cross_attention(0, q[0]), lambda: cache.cross_attention(0, q.half()),
                lambda: cache.cross_attention(0, q, lengths=torch.zeros(4, device=DEV)),
                lambda: cache.cross_attention(0, q, lengths=torch.zeros(5, dtype=torch.int32, device=DEV)),
                lambda: cache.prefix_attention(prefix, 0, q[:, :3].contiguous()),
                lambda: cache.prefix_attention(prefix, 0, q.transpose(2, 3).contiguous().transpose(2, 3)),
                lambda: cache.gather_sequences(cache, torch.zeros(4, dtype=torch.int64, device=DEV)),
                lambda: cache.gather_sequences(cache, torch.zeros(3, dtype=torch.int32, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    # a layer that is ahead of the one whose codes it reads
    K, V = _tokens(one, 1, 400)
    ahead = xq.Cache(_config(batch=1, max_seq=500), DEV)
    ahead.append_kv(1, K[1].to(DEV), V[1].to(DEV))
    with pytest.raises(xq.XQError) as e:
        cache.prefix_attention(ahead, 1, q)
    assert e.value.code == xq.XQ_ERR_ORDER
    assert xq.xq_launch_count(cache.handle) == n and (out == 7).all()
