"""Prefix and cross attention over caches of unusual magnitude, window, length and sharing pattern, against plain 64-bit attention
over what the oracle's packing restores."""
import math

import numpy as np
import pytest
import torch

import paper_2510_11236_b200 as xq
from tests import util
from tests.test_shared_cache import DEV, KERNELS, SHAPES, _check, _filled, _queries, _restored, _shape, _tokens

BLOCK = 128  # tokens whose window rows share an exponent


def _exponent(mx):
    """Power of two that the kernels scale a block of bfloat16 window rows by: its largest magnitude into half precision's range."""
    return 0 if 0.0625 <= mx < 32768.0 or mx == 0.0 else 14 - math.floor(math.log2(mx))


def _window_steps(x, n, rise):
    """What half precision leaves of window rows x[n:], taken relative to the largest of their 128: at most half a step of its
    subnormal numbers, 2^-25, in the block's scale, token by token.  rise: a block is scaled by at most 2^60 more than any before
    it, packed tokens counted with 2^0 (values)."""
    off, most = np.zeros(len(x)), 60 if n else 126
    for a in range(n, len(x), BLOCK):
        e = min(_exponent(np.abs(x[a:a + BLOCK]).max()), most if rise else 126)
        most = min(most, e + 60)
        off[a:a + BLOCK] = 2.0 ** (-25 - e)
    return off


def _expect(q, k, v, ka, va, n, scale, pairs, f16, products=1):
    """Attention of the rows q [rows, D] over k, v (n of them packed) and how far the kernels may be off.

    Numerators: half precision, 2^-11 of each, under their own sum (pairs: 2^-18); below 2^-14 of the largest number that half
    precision has for them a fixed 2^-25: they are scaled by 2^7 against a reference that the largest logit is at most one (log2)
    below, so 2^-31 of the largest weight.  Logits: q as half precision relative to the row's largest (2^-25), window keys as above,
    and (D / 16 + 4) sums of fp32 that drop their last digit, each of `products` times.  Value sums: one for each 16 tokens,
    `products` times, twice at the join."""
    S, D = k.shape
    kw, vw = (np.zeros(S), np.zeros(S)) if f16 else (_window_steps(k, n, False), _window_steps(v, n, True))
    out, off = np.zeros(q.shape), np.zeros(q.shape)
    for r, row in enumerate(q):
        x = scale * (k @ row)
        w = np.exp(x - x.max())
        w /= w.sum()
        o = w @ v
        away = np.abs(v - o)
        top = np.abs(row).max()
        d = scale * (products * (D // 16 + 4) * 2.0 ** -23 * (ka @ np.abs(row)).max() + 2.0 ** -25 * top * ka.sum(1).max()
                     + kw.max() * np.abs(row).sum())
        steps = products * S / 16 + 8
        out[r] = o
        off[r] = ((2.0 ** (-18 if pairs else -11) + 2 * d) * (w @ away) + 2.0 ** -31 * w.max() * away.sum(0)
                  + steps * 2.0 ** -23 * (w @ va) + w @ vw + 1e-6 * np.abs(o) + 2.0 ** -60 * np.abs(v).max())
    return out, off


def _compare(cfg, o32, o16, q, restored, n, heads, batch, pairs, products=1, tokens=None):
    """Rows of the named sequences, kv heads and query tokens against _expect; restored(b, h): a stream's (k, v, ka, va)."""
    G, f16 = cfg.n_q_heads // cfg.n_kv_heads, cfg.io_dtype == xq.XQ_F16
    scale = cfg.sm_scale if cfg.sm_scale > 0 else 1 / math.sqrt(cfg.head_dim)
    o32, o16, qd = o32.double().cpu().numpy(), o16.double().cpu().numpy(), q.double().cpu().numpy()
    half, worst = torch.finfo(q.dtype).eps / 2, 0.0
    at = list(range(len(qd))) if tokens is None else tokens
    for b in batch:
        for h in heads:
            k, v, ka, va = restored(b, h)
            rows = [x[at, b, h * G:(h + 1) * G].reshape(-1, cfg.head_dim) for x in (qd, o32, o16)]
            ref, off = _expect(rows[0], k, v, ka, va, n, scale, pairs, f16, products)
            err = np.abs(rows[1] - ref)
            assert (err <= off).all(), (b, h, err.max(), off.reshape(-1)[np.nan_to_num(err / off, nan=np.inf).argmax()])
            assert (np.abs(rows[2] - ref) <= off + half * (np.abs(ref) + off) + 2.0 ** -25).all(), (b, h)
            worst = max(worst, (err / off).max())
    print(f"worst error / bound: {worst:.2f}")


# ---- windows ----

# window capacity, tokens, size of each block of 128 window rows
WINDOWS = [
    (128, 300, [1e-30]), (128, 300, [1e-35]), (128, 300, [1e-39]), (128, 300, [0.0]), (128, 300, [1e5]), (128, 300, [1e30]),
    (512, 1000, [1.0, 1e-30, 1e4, 1e-4]), (512, 1000, [1e20, 1e-30, 1.0, 1e-38]), (512, 480, [1e-38, 1e-30, 1e-36, 1.0]),
    (512, 400, [1e30, 1e-38, 1e-38, 1e-38]), (512, 500, [1e-36] * 4),
    (1024, 2000, [1.0, 1e-3, 1e3, 1e-5, 1e5, 1.0, 1e-2, 1e2]),
    (4096, 8100, [10.0 ** (3 * (i * 7 % 5) - 6) for i in range(32)]),
]


def _sized(x, r, sizes):
    """The last r tokens of every [batch, heads, S, D] tensor in x, block by block times `sizes`."""
    S = x[0].shape[2]
    f = torch.ones(S)
    for i, s in enumerate(sizes):
        f[S - r + i * BLOCK:S - r + (i + 1) * BLOCK] = s
    return [(t.float() * f[:, None]).to(t.dtype) for t in x]


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("T", [1, 17, 1300])  # decode kernels, rows kernel, and so many rows that a CTA takes all the tokens
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[3]])
@pytest.mark.parametrize("R,S,sizes", WINDOWS)
def test_window_values_of_every_size(R, S, sizes, shape, T, kernel):
    D, Hq, Hkv, g, _, kq, vq, f16 = shape
    cfg = _shape((D, Hq, Hkv, g, R, kq, vq, f16), batch=2, max_seq=S, kernel=kernel)
    K, V = _tokens(cfg, 1, S)
    r = (S - 1) % R + 1
    V = _sized(V, r, sizes)
    cache = _filled(cfg, K, V)
    q = _queries(cfg, 3, T)
    o32, o16 = cache.cross_attention(1, q.to(DEV), f32=True), cache.cross_attention(1, q.to(DEV))
    _compare(cfg, o32, o16, q, lambda b, h: _restored(cfg, K, V, 1, b, h), S - r, [0, 1], [0, 1], False, tokens=[0, T - 1])
    cache.check_device()


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("T", [1, 17, 1300])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[3]])
@pytest.mark.parametrize("R,S,sizes", [w for w in WINDOWS if max(w[2]) <= 1e5] + [(128, 300, [3e8])])
def test_window_keys_of_every_size(R, S, sizes, shape, T, kernel):
    # queries so small that the largest keys' logits are of ordinary size
    D, Hq, Hkv, g, _, kq, vq, f16 = shape
    cfg = _shape((D, Hq, Hkv, g, R, kq, vq, f16), batch=2, max_seq=S, kernel=kernel)
    K, V = _tokens(cfg, 1, S, outliers=False)
    r = (S - 1) % R + 1
    K = _sized(K, r, sizes)
    cache = _filled(cfg, K, V)
    q = (_queries(cfg, 3, T).float() / max(1.0, *sizes)).to(torch.bfloat16)
    o32, o16 = cache.cross_attention(1, q.to(DEV), f32=True), cache.cross_attention(1, q.to(DEV))
    _compare(cfg, o32, o16, q, lambda b, h: _restored(cfg, K, V, 1, b, h), S - r, [0, 1], [0, 1], False, tokens=[0, T - 1])
    cache.check_device()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [SHAPES[1], SHAPES[6]])
def test_long_windows_in_half_precision(shape):
    D, Hq, Hkv, g, _, kq, vq, f16 = shape
    cfg = _shape((D, Hq, Hkv, g, 1024, kq, vq, f16), batch=2, max_seq=2000)
    K, V = _tokens(cfg, 1, 2000)
    V = _sized(V, 976, [1.0, 1e-3, 1e3, 1e-4, 1e4, 1.0, 1e-2, 1e2])
    cache = _filled(cfg, K, V)
    q = _queries(cfg, 3, 60)
    o32, o16 = cache.cross_attention(1, q.to(DEV), f32=True), cache.cross_attention(1, q.to(DEV))
    _compare(cfg, o32, o16, q, lambda b, h: _restored(cfg, K, V, 1, b, h), 1024, [0, 1], [0, 1], True, tokens=[0, 31, 59])
    cache.check_device()


# ---- scales that are too large to be doubled in half precision ----

def _wide(x, bits, f16, of_tokens, seed, g=32):
    """Every third group of x's tensors (g tokens of a channel, or a token's g channels) spread over all that a scale can span: to
    both ends of half precision for inputs of that type, else 3 (1-bit: 1) times a scale of 62000."""
    rng = np.random.default_rng(seed)
    lo, hi = (-65504.0, 65504.0) if f16 and bits == 2 else (-60000.0, 126000.0) if bits == 2 else (-30000.0, 32000.0)
    B, H, S, D = x[0].shape
    groups = (B, H, -(-S // g), D) if of_tokens else (B, H, S, D // g)
    pick = torch.from_numpy(rng.random(groups) < 1 / 3)
    pick = pick.repeat_interleave(g, 2)[:, :, :S] if of_tokens else pick.repeat_interleave(g, 3)
    ends = torch.from_numpy(np.where(rng.random(x[0].shape) < 0.5, lo, hi).astype(np.float32))
    inner = torch.from_numpy(rng.uniform(lo, hi, x[0].shape).astype(np.float32))
    wide = torch.where(torch.from_numpy(rng.random(x[0].shape) < 0.5), ends, inner).to(x[0].dtype)
    return [torch.where(pick, wide, t) for t in x]


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("T", [1, 17, 1300])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[2], SHAPES[3], SHAPES[6], (64, 4, 1, 64, 64, 2, 2, False),
                                   (128, 4, 1, 64, 64, 2, 2, True)])
@pytest.mark.parametrize("which", ["keys", "values"])
def test_packed_elements_beyond_half_precision(shape, which, T, kernel):
    D, Hq, Hkv, g, R, kq, vq, f16 = shape
    S = 700
    cfg = _shape(shape, batch=2, max_seq=S, kernel=kernel)
    K, V = _tokens(cfg, 1, S, outliers=False)
    q = _queries(cfg, 3, T)
    if which == "keys":
        K = _wide(K, 2 if kq else 1, f16, True, 4, g)
        q = (q.float() * 2.0 ** -13).to(q.dtype)  # logits of ordinary size
    else:
        V = _wide(V, 2 if vq else 1, f16, False, 5, g)
    cache = _filled(cfg, K, V)
    n = [S, 333]
    lengths = torch.tensor(n, dtype=torch.int32, device=DEV)
    pairs = f16 and T * cfg.n_q_heads // cfg.n_kv_heads > 128
    for layer in (0, 1):
        o32, o16 = (cache.cross_attention(layer, q.to(DEV), lengths=lengths, f32=f32) for f32 in (True, False))
        for b in (0, 1):
            _compare(cfg, o32, o16, q, lambda b, h: [x[:n[b]] for x in _restored(cfg, K, V, layer, b, h)],
                     min(n[b], S - (S - 1) % R - 1), range(Hkv), [b], pairs, products=4, tokens=[0, T - 1])
    cache.check_device()


# ---- the tensor-core kernel by name ----

@pytest.mark.gpu
@pytest.mark.parametrize("shape", [SHAPES[5], SHAPES[3], SHAPES[4]])  # twelve heads on a kv head; head_dim 64
def test_tensor_core_kernel_by_name(shape):
    # the decode kernel of that name takes neither shape, the rows kernel any: over a whole cache there is nothing to refuse
    named = dict(kernel=xq.XQ_KERNEL_MMA)
    cp, cc = _shape(shape, batch=1, max_seq=300, **named), _shape(shape, batch=3, max_seq=200, **named)
    kp, vp = _tokens(cp, 1, 300)
    ko, vo = _tokens(cc, 2, 200)
    prefix, cache, alone = _filled(cp, kp, vp), _filled(cc, ko, vo), xq.Cache(cc, DEV)
    heads = range(cc.n_kv_heads)
    for T in (1, 7):
        q = _queries(cc, 3, T)
        n = [S - (S - 1) % cc.residual_len - 1 for S in (300, 200)]
        o32, o16 = (alone.prefix_attention(prefix, 1, q.to(DEV), f32=f32) for f32 in (True, False))
        _compare(cc, o32, o16, q, lambda b, h: _restored(cp, kp, vp, 1, 0, h), n[0], heads, range(3), False)
        o32, o16 = (cache.cross_attention(1, q.to(DEV), f32=f32) for f32 in (True, False))
        _compare(cc, o32, o16, q, lambda b, h: _restored(cc, ko, vo, 1, b, h), n[1], heads, range(3), False)
        with pytest.raises(xq.XQError) as e:  # the sequences' own tokens are the decode kernel's
            cache.prefix_attention(prefix, 1, q.to(DEV))
        assert e.value.code == xq.XQ_ERR_CONFIG
    cache.check_device(), alone.check_device()


# ---- long caches: more splits than one trip of the join, than a warp of the decode kernels' merge ----

def _splits_used(space, rows, D):
    """Splits of a rows call, by how far it wrote its workspace (filled with 0xa5 before): partial sums, then two words a partial."""
    end = int((space != 0xa5).nonzero().max()) + 1
    for ns in range(1, 1000):
        sums = -(-rows * ns * D * 4 // 256) * 256
        if end <= sums + rows * ns * 8:
            return ns if end > sums else 0
    return 0


LONG = [  # shape, tokens
    ((128, 4, 1, 32, 128, 2, 0, False), 20011), ((128, 4, 1, 64, 256, 0, 2, True), 46000), ((64, 2, 1, 32, 64, 2, 2, False), 30000),
    ((64, 8, 1, 64, 64, 0, 0, True), 23456),
]


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("shape,S", LONG)
def test_more_splits_than_one_trip_of_the_join(shape, S, kernel):
    cfg = _shape(shape, batch=1, max_seq=S, kernel=kernel)
    K, V = _tokens(cfg, 1, S)
    cache = _filled(cfg, K, V)
    T, n = 17, S - (S - 1) % cfg.residual_len - 1
    q = _queries(cfg, 3, T)
    space = torch.full((xq.xq_cross_workspace_bytes(cache.handle, T),), 0xa5, dtype=torch.uint8, device=DEV)
    o32 = cache.cross_attention(1, q.to(DEV), f32=True, workspace=space)
    assert _splits_used(space, T * cfg.n_q_heads, cfg.head_dim) > 16
    o16 = cache.cross_attention(1, q.to(DEV))
    _compare(cfg, o32, o16, q, lambda b, h: _restored(cfg, K, V, 1, b, h), n, [0], [0], False, tokens=[0, 16])
    cache.check_device()


@pytest.mark.gpu
@pytest.mark.parametrize("shape,S", LONG)
def test_prefix_of_many_splits_behind_own_tokens(shape, S):
    D, Hq, Hkv, g, R, kq, vq, f16 = shape
    cp, cc = _shape(shape, batch=1, max_seq=S), _shape(shape, batch=17, max_seq=200)
    kp, vp = _tokens(cp, 1, S)
    ko, vo = _tokens(cc, 2, 70)
    prefix, cache = _filled(cp, kp, vp), _filled(cc, ko, vo)
    q = _queries(cc, 3, 1)
    o32, o16 = (cache.prefix_attention(prefix, 1, q.to(DEV), f32=f32) for f32 in (True, False))
    whole = _restored(cp, kp, vp, 1, 0, 0)
    _check(cc, o32, o16, q, lambda b, h: whole, lambda b, h: _restored(cc, ko, vo, 1, b, h), 1, 70, batch=[0, 16], rows=17 * Hq)
    cache.check_device()


@pytest.mark.gpu
@pytest.mark.parametrize("shape,S", LONG)
def test_more_splits_than_a_warp_of_the_merge(shape, S):
    # up to eight rows of a kv head: the decode kernels, whose last CTA of a stream merges
    cfg = _shape(shape, batch=1, max_seq=S)
    K, V = _tokens(cfg, 1, S)
    cache = _filled(cfg, K, V)
    rc, splits, _ = xq.xq_split_plan(cache.handle, 1)
    assert rc == 0 and splits > 32
    n = S - (S - 1) % cfg.residual_len - 1
    whole = _restored(cfg, K, V, 1, 0, 0)
    for lengths in (None, [S - 5000], [1000]):
        q = _queries(cfg, 3, 1)
        ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
        o32, o16 = (cache.cross_attention(1, q.to(DEV), lengths=ln, f32=f32) for f32 in (True, False))
        seen = S if lengths is None else lengths[0]
        _compare(cfg, o32, o16, q, lambda b, h: [x[:seen] for x in whole], min(n, seen), [0], [0], False)
    cache.check_device()


# ---- logits that rise or fall through the tokens ----

@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("T", [1, 17, 1300])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[3], SHAPES[6]])
@pytest.mark.parametrize("course", ["rising", "falling", "waves", "equal"])
def test_course_of_the_logits(course, shape, T, kernel):
    # the reference of the softmax is raised in every tile, in none behind the first, in every other one
    S = 1200
    cfg = _shape(shape, batch=2, max_seq=S, kernel=kernel)
    K, V = _tokens(cfg, 1, S, outliers=False)
    t = torch.arange(S)
    level = {"rising": t / S, "falling": 1 - t / S, "waves": ((t // 64) % 2) * (t / S), "equal": 0.0 * t}[course] * 200.0
    rng = np.random.default_rng(7)
    u = torch.from_numpy(rng.choice([-1.0, 1.0], cfg.head_dim)).float()
    scale = 1 / math.sqrt(cfg.head_dim)
    along = level[:, None] * u / (scale * cfg.head_dim)
    K = [((0.0 if course == "equal" else 0.02) * x.float() + along).to(x.dtype) for x in K]
    cache = _filled(cfg, K, V)
    q = (_queries(cfg, 3, T).float() * 0.1 + u).to(K[0].dtype)
    q[..., 1::2, :] *= -1  # every other head: the other way round
    o32, o16 = (cache.cross_attention(1, q.to(DEV), f32=f32) for f32 in (True, False))
    n = S - (S - 1) % cfg.residual_len - 1
    _compare(cfg, o32, o16, q, lambda b, h: _restored(cfg, K, V, 1, b, h), n, [0, 1][:cfg.n_kv_heads], [0, 1],
             cfg.io_dtype == xq.XQ_F16 and T * cfg.n_q_heads // cfg.n_kv_heads > 128, tokens=[0, T - 1])
    cache.check_device()


# ---- sharing patterns ----

PATTERNS = [dict(n_layers=3, share_group=3, share_dominant=1), dict(n_layers=3, share_group=3, share_dominant=2),
            dict(n_layers=4, share_group=4, share_dominant=0), dict(n_layers=4, share_group=4, share_dominant=3),
            dict(n_layers=2, gamma1=0.4), dict(n_layers=2, share_dominant=1)]


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [2, 1])
@pytest.mark.parametrize("pattern", PATTERNS)
@pytest.mark.parametrize("D", [128, 64])
def test_sharing_patterns(D, pattern, bits):
    """Prefix, cross attention and gathered sequences over layers that share codes in other ways than pairs."""
    L, S = pattern["n_layers"], 333
    order = sorted(range(L), key=lambda l: l != pattern.get("share_dominant", 0))  # the layer that owns the codes first
    kw = dict(head_dim=D, n_q_heads=6, n_kv_heads=2, group_size=32, residual_len=64, kq=L * (bits - 1), vq=L * (bits - 1), km=0, vm=0,
              eta1=1 / 6, eta2=0.045, **pattern)
    one, three = xq.make_config(batch=2, max_seq=S, **kw), xq.make_config(batch=6, max_seq=S, **kw)

    def filled(cfg, K, V):
        cache = xq.Cache(cfg, DEV)
        for layer in order:
            cache.append_kv(layer, K[layer].to(DEV), V[layer].to(DEV))
        return cache

    def tokens(cfg, seed, n):
        K, V = _tokens(cfg, seed, n)
        g = torch.Generator().manual_seed(seed + 50)
        return [[(x[0].float() + 0.1 * torch.randn(x[0].shape, generator=g)).to(x[0].dtype) for _ in range(L)] for x in (K, V)]

    def restored(cfg, K, V, layer, b, h):
        oc = util.oracle_for_stream(cfg, order, b, h, {l: (K[l], V[l]) for l in order})
        n, st, g = oc.n_quantized(layer), oc.layers[layer], cfg.group_size
        kc, ks, kz, vc, vs, vz = (np.asarray(x[0, 0], dtype=np.float64) for x in oc.codes_and_meta(layer))
        ks, kz, vs, vz = np.repeat(ks, g, 0), np.repeat(kz, g, 0), np.repeat(vs, g, 1), np.repeat(vz, g, 1)
        k, v = (np.concatenate([x, st[w][0, 0]]) for x, w in ((kc * ks + kz, "win_k"), (vc * vs + vz, "win_v")))
        ka, va = np.abs(k), np.abs(v)
        ka[:n], va[:n] = (np.abs(kc - 1) + 1) * ks + np.abs(kz), (np.abs(vc - 1) + 1) * vs + np.abs(vz)
        return k, v, ka, va

    kp, vp = tokens(one, 1, S)
    ko, vo = tokens(three, 2, 150)
    prefix, cache, spare = filled(one, kp, vp), filled(three, ko, vo), xq.Cache(three, DEV)
    index = torch.tensor([5, 0, 0, 3, 2, 1], dtype=torch.int32, device=DEV)
    spare.gather_sequences(cache, index)
    for layer in range(L):
        for T in (1, 12):
            q = _queries(three, 3 + layer, T)
            o32, o16 = (cache.prefix_attention(prefix, layer, q.to(DEV), f32=f32) for f32 in (True, False))
            _check(three, o32, o16, q, lambda b, h: restored(one, kp, vp, layer, b // 3, h), lambda b, h: restored(three, ko, vo, layer, b, h),
                   T, 150, heads=[1], batch=[0, 5], rows=T * 9)
            o32, o16 = (cache.cross_attention(layer, q.to(DEV), f32=f32) for f32 in (True, False))
            _compare(three, o32, o16, q, lambda b, h: restored(three, ko, vo, layer, b, h), 128, [0], [0, 5], False)
            assert torch.equal(spare.cross_attention(layer, q[:, index.long().cpu()].contiguous().to(DEV), f32=True), o32[:, index.long()])
    cache.check_device(), spare.check_device()
