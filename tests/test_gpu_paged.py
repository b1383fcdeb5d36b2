"""The rotary and paged-cache calls on the GPU against float64 references (paged_ref.py).

Tolerances, from the arithmetic alone.  A rotated element is rounded once to float32 (2^-24
relative) and, in bf16, once more (2^-8); the float64 rotation before it errs by a few 2^-53
of its pair.  A stored value is exact for its code and words up to one rounding.  An
attention output: a score sums d products whose absolute values sum to `spread`, in float32
and over at most a few dozen partial sums, and errs by less than 16 * 2^-24 * spread, which is
the relative error of its weight; the weights' own roundings, their sum and the value sums add
a few dozen 2^-24 more, in the numerator and the denominator.  So an output is within
2^-18 * (1 + spread) of the weighted sum of |v|, and the log-sum-exp within
2^-19 * (1 + spread) + 2^-23 |lse|."""
import math

import numpy as np
import pytest

import paged_ref as ref
from gpu_harness import torch_cuda
from paper_2607_27692_amd import retopk as R

pytestmark = pytest.mark.gpu

EPS = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8 + 2.0 ** -24}


def tdt(dtype):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]


def dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t if dtype is None else t.to(tdt(dtype))).cuda()


def ints(x):
    return dev(np.asarray(x, np.int32))


def f64(t):
    return t.double().cpu().numpy()


def rope_of(rot, interleaved, scaling="none", theta=1e4):
    kw = dict(factor=4.0, original_len=8192, low=1.0, high=32.0) if scaling != "none" else {}
    return R.make_rope(rot, theta, interleaved, scaling, **kw)


def rotated(rope, x, pos, inverse=False):
    return ref.rotate(x, pos, list(rope.freq), rope.factor, rope.rot_dim, rope.interleaved,
                      inverse)


def assert_rotated(got, want, x, dtype, what):
    # 2^-45: float64 roundings of a pair whose sum cancels, of angles up to 2^31
    pair = np.abs(x).max(-1, keepdims=True)
    tol = EPS[dtype] * np.abs(want) + 2.0 ** -45 * pair
    worst = np.max(np.abs(got - want) - tol)
    assert worst <= 0, f"{what}: {worst:.3g} past the tolerance"


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,rot,interleaved,T,H,start,scaling", [
    (128, 128, False, 1, 40, 131072, "none"), (128, 128, True, 17, 3, 0, "ramp"),
    (64, 64, False, 33, 2, 100, "ntk"), (64, 64, True, 1, 1, 2 ** 31 - 1, "none"),
    (128, 64, False, 15, 5, 2 ** 31 - 20, "bands"), (128, 96, True, 16, 4, 7, "linear"),
    # halves that are no whole lanes, down to one pair
    (128, 36, False, 31, 7, 999, "none"), (64, 10, False, 65, 3, 5, "linear"),
    (64, 2, False, 3, 9, 12345, "none"), (128, 2, True, 3, 9, 12345, "none"),
    (128, 126, False, 50, 1, -40, "none"), (64, 62, True, 20, 2, -2 ** 31, "none"),
    (128, 128, False, 2500, 33, 0, "none"),
])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotary(dtype, d, rot, interleaved, T, H, start, scaling, inverse):
    torch = torch_cuda()
    print(f"rotary {dtype} d={d} rot={rot} T={T} H={H} start={start}", flush=True)
    rng = np.random.default_rng(T * 131 + rot)
    x = dev(rng.standard_normal((T, H, d)), dtype)
    pos = np.arange(start, start + T).astype(np.int64).clip(-2 ** 31, 2 ** 31 - 1)
    rope = rope_of(rot, interleaved, scaling)
    out = torch.full_like(x, float("nan"))
    R.rotary_embed(rope, x, ints(pos), out, inverse=inverse)
    want = rotated(rope, f64(x), pos, inverse)
    assert_rotated(f64(out), want, f64(x), dtype, "out")
    assert torch.equal(out[..., rot:], x[..., rot:])
    # the same in place, and in place on a slice of a wider tensor
    wide = torch.full((T, H + 3, d), 7.0, dtype=x.dtype, device="cuda")
    part = wide[:, 2:2 + H]
    part.copy_(x)
    R.rotary_embed(rope, part, ints(pos), part, inverse=inverse)
    assert torch.equal(part, out)
    assert bool((wide[:, :2] == 7).all()) and bool((wide[:, 2 + H:] == 7).all())


def test_rotary_strides_and_orders():
    """Heads outermost in memory, one position for all tokens' heads, broadcast inputs."""
    torch = torch_cuda()
    rng = np.random.default_rng(5)
    rope, pos = rope_of(128, False), ints([3, 70000, 5, 5, 0])
    a = dev(rng.standard_normal((6, 5, 128)), "bf16")
    want = rotated(rope, f64(a).transpose(1, 0, 2), pos.cpu().numpy())
    out = torch.empty((6, 5, 128), dtype=a.dtype, device="cuda")
    R.rotary_embed(rope, a.transpose(0, 1), pos, out.transpose(0, 1))
    assert_rotated(f64(out).transpose(1, 0, 2), want, f64(a).transpose(1, 0, 2), "bf16", "heads first")
    one = dev(rng.standard_normal((1, 1, 128)), "bf16").expand(5, 6, 128)
    out = torch.empty((5, 6, 128), dtype=a.dtype, device="cuda")
    R.rotary_embed(rope, one, pos, out)
    assert_rotated(f64(out), rotated(rope, f64(one), pos.cpu().numpy()), f64(one), "bf16", "broadcast")


def test_rotary_gradient_against_differences():
    """The inverse rotation is the gradient of sum(g * rotated(x)): against differences of that
    sum along single elements (linear in x, so a difference over 2 is exact up to float32
    roundings of the two rotations, 2^-23 of the pair's size)."""
    torch = torch_cuda()
    rng = np.random.default_rng(6)
    for interleaved, rot, scaling in ((False, 64, "ramp"), (True, 40, "none"), (False, 28, "linear")):
        rope, pos = rope_of(rot, interleaved, scaling), ints([0, 9, 40000])
        x = dev(rng.standard_normal((3, 2, 64)), "f32")
        g = dev(rng.standard_normal((3, 2, 64)), "f32")
        dx = torch.empty_like(x)
        R.rotary_embed(rope, g, pos, dx, inverse=True)
        for t, h, e in ((0, 0, 0), (1, 1, 5), (2, 0, rot // 2), (2, 1, rot - 1), (1, 0, 63)):
            sides = []
            for step in (1.0, -1.0):
                y = x.clone()
                y[t, h, e] = step
                out = torch.empty_like(x)
                R.rotary_embed(rope, y, pos, out)
                sides.append(float((out.double() * g.double()).sum()))
            want = (sides[0] - sides[1]) / 2
            bound = 64 * 2.0 ** -23 * 4 * float(g.abs().max())
            assert abs(float(dx[t, h, e]) - want) <= bound, (interleaved, t, h, e)


def test_rotary_copies_what_is_not_rotated():
    """Infinities and NaN past rot_dim stay what they are and touch nothing else."""
    torch = torch_cuda()
    x = torch.ones((4, 2, 64), device="cuda")
    x[..., 32:] = float("inf")
    x[1, 0, 40] = float("nan")
    out = torch.empty_like(x)
    R.rotary_embed(rope_of(32, False), x, ints([0, 1, 2, 3]), out)
    assert bool(torch.isfinite(out[..., :32]).all())
    assert torch.equal(out[..., 32:].nan_to_num(5.0), x[..., 32:].nan_to_num(5.0))


# ---------------------------------------------------------------------------
# Caches
# ---------------------------------------------------------------------------

def make_cache(fmt, hkv, d, page, lens, rng, spare=2, width=None):
    """A cache with room for sequences of these lengths on shuffled pages, every byte of it
    junk (NaN among it)."""
    torch = torch_cuda()
    need = [-(-n // page) for n in lens]
    n_pages, width = sum(need) + spare, width or max(1, max(need))
    c = R.PagedCache.allocate(fmt, n_pages, hkv, page, d, len(lens), width)
    order = rng.permutation(n_pages)
    table = np.full((len(lens), width), -1, np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    c.table.copy_(torch.from_numpy(table))
    for x in c.tensors[:2] + c.tensors[3:]:
        if x is not None:
            b = x.view(torch.uint8)
            b.copy_(torch.randint(0, 256, b.shape, dtype=torch.uint8, device="cuda"))
            if x.is_floating_point():
                x[..., ::5] = float("nan")
            elif x.dtype == torch.int32:
                x.fill_(0x7FC07FC0)          # scale and middle NaN
    return c


def bytes_of(c):
    torch = torch_cuda()
    return [x.view(torch.uint8).clone() for x in c.tensors[:2] + c.tensors[3:] if x is not None]


def rows_in(c, fmt, name, s, positions):
    """(codes, words) or float64 rows [n, Hkv, .] of positions of sequence s."""
    k, v, table, kp, vp = c.tensors
    page = k.shape[2]
    ids = table[s].cpu().numpy()[np.asarray(positions) // page]
    slot = np.asarray(positions) % page
    x, p = (k, kp) if name == "k" else (v, vp)
    if fmt == "q4":
        return x.cpu().numpy()[ids, :, slot], p.cpu().numpy()[ids, :, slot]
    return f64(x)[ids, :, slot]


def assert_stored4(codes, words, x, loose, what):
    """4-bit rows against float32 rows x; loose: x itself may be a rounding off, so that an
    element next to a border may take either code."""
    mid, scale = ref.group_params(x)
    got_mid, got_scale = ref.params_of_words(words)
    if loose:
        np.testing.assert_allclose(got_mid, mid, rtol=2.0 ** -7, atol=1e-30)
        np.testing.assert_allclose(got_scale, scale, rtol=2.0 ** -7, atol=1e-30)
        mid, scale = got_mid, got_scale
    else:
        assert np.array_equal(got_mid, mid) and np.array_equal(got_scale, scale), what
    m, sc = np.repeat(mid, ref.GROUP, -1), np.repeat(scale, ref.GROUP, -1)
    c = ref.unpack(codes)
    live = sc > 0
    t = np.where(live, (np.asarray(x, np.float64) - m) / np.where(live, sc, 1), 0)
    want = np.clip(np.floor(t), -8, 7) + 0.5
    off = live & (c != want)
    if loose:
        off &= np.abs(t - np.rint(t)) > 1e-4
    assert not off.any(), f"{what}: {int(off.sum())} codes differ"


CASES = [
    # fmt, dtype, d, hq, hkv, page, lengths before, tokens each
    ("bf16", "bf16", 128, 32, 8, 64, [0, 100, 63], [70, 1, 2]),
    ("f32", "f32", 64, 6, 2, 17, [5, 0, 16, 40], [30, 1, 1, 18]),
    ("q4", "bf16", 128, 28, 4, 16, [0, 15, 16], [33, 1, 47]),
    ("q4", "f32", 64, 8, 8, 48, [1000, 3], [1, 90]),
    ("q4", "f32", 128, 3, 3, 32, [0], [1]),
    ("q4", "bf16", 64, 8, 1, 64, [0, 1], [700, 300]),
    ("bf16", "bf16", 64, 5, 5, 1, [0, 9], [3, 4]),
    ("f32", "f32", 128, 16, 2, 300, [299, 0], [2, 600]),
]


@pytest.mark.parametrize("fmt,dtype,d,hq,hkv,page,before,counts", CASES)
@pytest.mark.parametrize("rotate", [True, False])
def test_append_and_gather(fmt, dtype, d, hq, hkv, page, before, counts, rotate):
    torch = torch_cuda()
    print(f"append {fmt} {dtype} d={d} {hq}/{hkv} page={page}", flush=True)
    rng = np.random.default_rng(page * 7 + d)
    torch.manual_seed(page)
    lens = [b + n for b, n in zip(before, counts)]
    c = make_cache(fmt, hkv, d, page, lens, rng)
    seq = [s for s, n in enumerate(counts) for _ in range(n)]
    pos = [b + i for b, n in zip(before, counts) for i in range(n)]
    # padding, a sequence that is none, positions without a page: none of them writes a row
    n_seqs, beyond = len(lens), c.table.shape[1] * page
    extra = [(-1, 0), (n_seqs, 3), (-5, beyond), (0, -1), (0, beyond), (0, 2 ** 31 - 1)]
    order = rng.permutation(len(seq) + len(extra))
    live = np.array([True] * len(seq) + [False] * len(extra))[order]
    in_seq = np.array([True] * len(seq) + [False] * 3 + [True] * 3)[order]
    seq = np.array(seq + [s for s, _ in extra])[order]
    pos = np.array(pos + [p for _, p in extra])[order]
    T = len(seq)
    qkv = dev(rng.standard_normal((T, hq + 2 * hkv, d)), dtype)
    q, k, v = qkv.split((hq, hkv, hkv), 1)
    rope = rope_of(d - 10 if fmt != "q4" else d, fmt == "f32", "ramp") if rotate else None
    kept, old = qkv.clone(), bytes_of(c)
    q_out = torch.full((T, hq, d), 9.0, dtype=q.dtype, device="cuda")
    if rotate:
        R.paged_append(c, ints(seq), ints(pos), k, v, rope=rope, q=q, q_out=q_out)
    else:
        R.paged_append(c, ints(seq), ints(pos), k, v)
    assert torch.equal(qkv, kept)
    x = rotated(rope, f64(k), pos) if rotate else f64(k)
    if rotate:
        assert_rotated(f64(q_out)[in_seq], rotated(rope, f64(q), pos)[in_seq], f64(q)[in_seq], dtype, "q")
        assert bool((q_out[torch.from_numpy(~in_seq).cuda()] == 9).all())
    else:
        assert bool((q_out == 9).all())
    for s in range(n_seqs):
        mine = np.flatnonzero(live & (seq == s))
        got_k, got_v = (rows_in(c, fmt, n, s, pos[mine]) for n in "kv")
        if fmt == "q4":
            assert_stored4(*got_k, x[mine].astype(np.float32), rotate, f"keys of {s}")
            assert_stored4(*got_v, f64(v)[mine].astype(np.float32), False, f"values of {s}")
        else:
            assert_rotated(got_k, x[mine], f64(k)[mine], dtype, f"keys of {s}")
            assert np.array_equal(got_v, f64(v)[mine])
    # every other row holds the bytes it held
    new, written = bytes_of(c), np.zeros((c.k.shape[0], page), bool)
    table = c.table.cpu().numpy()
    for s, p in zip(seq[live], pos[live]):
        written[table[s, p // page], p % page] = True
    for a, b in zip(old, new):
        same = (a.view(*a.shape[:3], -1) == b.view(*b.shape[:3], -1)).all(-1).cpu().numpy()
        assert same.transpose(0, 2, 1)[~written].all()
    # and back: the values, into tensors whose other rows stay
    outs = [torch.full((T, hkv, d), 5.0, dtype=q.dtype, device="cuda") for _ in range(2)]
    R.paged_gather(c, ints(seq), ints(pos), *outs)
    only = torch.full_like(outs[0], 5.0)
    R.paged_gather(c, ints(seq), ints(pos), v=only)
    assert torch.equal(only, outs[1])
    for name, out in zip("kv", outs):
        assert bool((out[torch.from_numpy(~live).cuda()] == 5).all())
        for s in range(n_seqs):
            mine = np.flatnonzero(live & (seq == s))
            rows = rows_in(c, fmt, name, s, pos[mine])
            if fmt == "q4":
                want = torch.from_numpy(ref.values4(*rows).astype(np.float32)).to(q.dtype).double().numpy()
            else:
                want = rows
            assert np.array_equal(f64(out)[mine], want), f"{name} of {s}"
    # queries in place give the same
    if rotate:
        R.paged_append(c, ints(seq), ints(pos), k, v, rope=rope, q=q, q_out=q)
        mask = torch.from_numpy(in_seq).cuda()
        assert torch.equal(q[mask], q_out[mask]) and torch.equal(q[~mask], kept[:, :hq][~mask])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("recipe", ["equal", "zero", "negative zero", "huge", "tiny", "offset", "ties",
                                    "one far"])
def test_append_4bit_extremes(dtype, recipe):
    """Groups whose range or size is extreme are stored by the same rule, and what comes back is
    within half a scale of what went in (more only where bf16's steps of mid or scale do it)."""
    torch = torch_cuda()
    rng = np.random.default_rng(3)
    x = rng.standard_normal((8, 2, 128)).astype(np.float32)
    x = {"equal": np.full_like(x, -1.7182817), "zero": 0 * x, "negative zero": -0.0 * np.abs(x),
         "huge": x * 5e37, "tiny": x * 1e-39, "offset": x + 1000,
         "ties": np.round(x * 2) / 2, "one far": np.where(rng.random(x.shape) < 0.01, 300 * x, x)}[recipe]
    c = make_cache("q4", 2, 128, 16, [8], rng)
    v = dev(x, dtype)
    R.paged_append(c, ints([0] * 8), ints(range(8)), v, v)
    x = f64(v)
    codes, words = rows_in(c, "q4", "v", 0, range(8))
    assert_stored4(codes, words, x.astype(np.float32), False, recipe)
    back = torch.empty((8, 2, 128), device="cuda")
    R.paged_gather(c, ints([0] * 8), ints(range(8)), k=back)
    mid, scale = (np.repeat(a, ref.GROUP, -1) for a in ref.params_of_words(words))
    # half a scale; 7.5 times a scale rounded down by 2^-8 leaves 0.03 of one at the ends.  A
    # subnormal scale has steps of 2^-133, is off by up to 2^-134, and 7.5 of those are left there.
    tol = 0.535 * scale + 2.0 ** -24 * np.abs(x) + 1e-38 * (scale == 0) + 7.5 * 2.0 ** -134
    worst = float((np.abs(f64(back) - x) - tol).max())
    assert worst <= 0


def test_gather_into_the_contiguous_layout_and_its_attention():
    """Prompts stored in 4 bits, read back into [B, Hkv, max_len, d] by strides, give the exact
    path the rows that paged_attention reads: the same outputs from both."""
    torch = torch_cuda()
    rng = np.random.default_rng(12)
    B, hq, hkv, d, L, maxl = 2, 8, 2, 128, 700, 768
    c = make_cache("q4", hkv, d, 64, [L, L], rng)
    k, v = (dev(rng.standard_normal((B * L, hkv, d)), "bf16") for _ in range(2))
    seq, pos = ints(np.repeat(range(B), L)), ints(np.tile(range(L), B))
    R.paged_append(c, seq, pos, k, v, rope=rope_of(128, False))
    K, V = (torch.zeros((B, hkv, maxl, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for b in range(B):
        R.paged_gather(c, ints([b] * L), ints(range(L)), K[b, :, :L].transpose(0, 1), V[b, :, :L].transpose(0, 1))
    q = dev(rng.standard_normal((B, hq, d)), "bf16")
    h = R.Handle(batch=B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, max_len=maxl, k=L, cache_cap=4, r=1,
                 window=8, tau=0.8, refresh=0, dtype="bf16")
    exact, full, out = (torch.empty((B, hq, d), device="cuda") for _ in range(3))
    h.exact(q, K, V, L, exact)
    h.full(q, K, V, L, full)
    R.paged_attention(c, ints(range(B)), ints([L - 1] * B), q, out, L)
    torch.cuda.synchronize()
    h.close()
    # bf16 rounds the stored values once more (2^-8 of every value and key element)
    size = float(full.abs().max())
    assert float((out - full).abs().max()) <= 2.0 ** -6 * size
    assert float((exact - full).abs().max()) <= 2.0 ** -8 * size


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------

def fill(c, fmt, dtype, lens, rng, scale=1.0):
    """Rows of every sequence written by paged_append; the float64 rows as the cache holds them."""
    hkv, d = c.n_kv_heads, c.head_dim
    rows = []
    for s, n in enumerate(lens):
        if n == 0:
            rows.append((np.zeros((0, hkv, d)),) * 2)
            continue
        k, v = (dev(scale * rng.standard_normal((n, hkv, d)), dtype) for _ in range(2))
        R.paged_append(c, ints([s] * n), ints(range(n)), k, v)
        got = []
        for name in "kv":
            x = rows_in(c, fmt, name, s, range(n))
            got.append(ref.values4(*x) if fmt == "q4" else x)
        rows.append(tuple(got))
    return rows


def check_attention(out, lse, q, seq, pos, rows, hq, hkv, window=0, limit=None, gone=None):
    """gone: {sequence: bool array of positions that have no page}."""
    out, lse, q = f64(out), f64(lse), f64(q)
    G, worst = hq // hkv, 0.0
    for t, (s, p) in enumerate(zip(seq, pos)):
        for h in range(hq):
            n = 0 if s < 0 or s >= len(rows) else min(p + 1, limit or p + 1)
            k, v = (x[:, h // G] for x in rows[s]) if n > 0 else (np.zeros((0, q.shape[-1])),) * 2
            at = np.arange(k.shape[0])
            keep = (at < n) & (at > p - window if window else True)
            if gone is not None and s in gone and n > 0:
                keep &= ~gone[s][:k.shape[0]]
            o, want, spread, size = ref.attend(q[t, h], k, v, keep)
            if want == -math.inf:
                assert lse[t, h] == -math.inf and (out[t, h] == 0).all(), (t, h)
                continue
            tol = 2.0 ** -18 * (1 + spread) * size.max()
            err = np.abs(out[t, h] - o).max()
            assert err <= tol, f"row {t} head {h}: {err:.3g} > {tol:.3g}"
            assert abs(lse[t, h] - want) <= 2.0 ** -19 * (1 + spread) + 2.0 ** -23 * abs(want), (t, h)
            worst = max(worst, err / max(np.abs(o).max(), 1e-30))
    print(f"worst error against the largest element: {worst:.3g}", flush=True)


def attend(c, seq, pos, q, max_len, window=0):
    torch = torch_cuda()
    out = torch.full((q.shape[0], q.shape[1], c.head_dim), float("nan"), device="cuda")
    lse = torch.full((q.shape[0], q.shape[1]), float("nan"), device="cuda")
    R.paged_attention(c, ints(seq), ints(pos), q, out, max_len, window=window, lse=lse)
    torch.cuda.synchronize()
    return out, lse


ATTEND = [
    # fmt, dtype, d, hq, hkv, page, lengths, window
    ("f32", "f32", 64, 1, 1, 17, [2048], 0),
    ("f32", "f32", 128, 10, 2, 1, [1, 2, 300], 0),
    ("f32", "f32", 128, 8, 1, 1000, [31, 0, 999, 1700], 0),
    ("f32", "f32", 64, 12, 4, 16, [600, 33], 100),
    ("bf16", "bf16", 128, 32, 8, 64, [1, 63, 64, 65, 2500], 0),
    ("bf16", "bf16", 128, 28, 4, 48, [0, 15, 16, 17, 1000], 0),
    ("bf16", "bf16", 64, 8, 8, 3, [32, 33, 700], 40),
    ("bf16", "bf16", 64, 16, 2, 5000, [4500, 1], 0),
    ("bf16", "bf16", 128, 3, 3, 7, [129, 255, 257], 31),
    ("bf16", "bf16", 128, 6, 1, 31, [3000], 1),
    ("q4", "bf16", 128, 32, 8, 64, [1, 15, 16, 17, 31, 32, 33, 2500], 0),
    ("q4", "bf16", 128, 28, 4, 16, [0, 1000, 63], 0),
    ("q4", "bf16", 64, 8, 8, 48, [640, 5, 47], 0),
    ("q4", "bf16", 64, 8, 1, 4096, [4100, 4096], 0),
    ("q4", "f32", 128, 5, 1, 32, [3000, 257], 0),
    ("q4", "f32", 64, 12, 2, 16, [255, 256, 513], 100),
    ("q4", "f32", 128, 4, 4, 80, [100, 2000], 33),
    ("q4", "bf16", 128, 2, 1, 16, [4000], 15),
    ("q4", "f32", 64, 1, 1, 16, [1], 0),
]


@pytest.mark.parametrize("fmt,dtype,d,hq,hkv,page,lens,window", ATTEND)
def test_attention(fmt, dtype, d, hq, hkv, page, lens, window):
    """Ragged batches on junk-filled, shuffled pages, with padded rows and a query that is a
    slice of a wider tensor."""
    torch = torch_cuda()
    print(f"attention {fmt} {dtype} d={d} {hq}/{hkv} page={page} {lens} window={window}", flush=True)
    rng = np.random.default_rng(page + 3 * d + hq)
    torch.manual_seed(page)
    c = make_cache(fmt, hkv, d, page, lens, rng)
    rows = fill(c, fmt, dtype, lens, rng)
    seq = list(range(len(lens))) + [-1, len(lens), 0]
    pos = [n - 1 for n in lens] + [5, 5, -1]
    wide = dev(rng.standard_normal((len(seq), hq + 2, d)) * 2, dtype)
    q = wide[:, 1:1 + hq]
    out, lse = attend(c, seq, pos, q, max(lens), window)
    check_attention(out, lse, q, seq, pos, rows, hq, hkv, window)
    again, _ = attend(c, seq, pos, q, max(lens), window)
    assert torch.equal(out, again)
    # several tokens of one sequence, and a bound that cuts the longest sequence
    last, cut = max(range(len(lens)), key=lambda s: lens[s]), max(1, max(lens) - 37)
    seq, pos = [last] * 4, [lens[last] - 1, 0, lens[last] // 2, lens[last] - 1]
    q = q[:1].expand(4, hq, d) if len(lens) == 1 else q[:4]
    out, lse = attend(c, seq, pos, q, cut, window)
    check_attention(out, lse, q, seq, pos, rows, hq, hkv, window, limit=cut)


@pytest.mark.parametrize("fmt,dtype,d,hq,hkv,page,tokens,longest,window", [
    # more tokens than are shared out tile by tile: fixed chunks, sixteen tiles of one wave
    ("q4", "bf16", 128, 7, 1, 32, 1100, 2300, 0), ("q4", "f32", 64, 2, 1, 48, 1030, 2200, 0),
    ("bf16", "bf16", 128, 5, 1, 37, 1100, 2300, 0), ("f32", "f32", 64, 8, 1, 64, 1030, 2150, 0),
    ("q4", "bf16", 64, 4, 2, 16, 1050, 3100, 2500),
    # as many groups as fill the chip: a block each, with up to 64 tiles
    ("q4", "bf16", 128, 4, 1, 64, 600, 2000, 0), ("bf16", "bf16", 64, 2, 2, 5, 300, 1900, 0),
    ("f32", "f32", 128, 1, 1, 100, 520, 2048, 1000),
    # hundreds of tokens shared out tile by tile, most of them short
    ("q4", "f32", 128, 8, 1, 16, 700, 2600, 0), ("bf16", "bf16", 128, 8, 1, 64, 513, 2500, 0),
    # as many as a wave counts by itself, and one more
    ("q4", "bf16", 64, 4, 1, 16, 64, 1500, 0), ("f32", "f32", 64, 3, 1, 7, 64, 1500, 700),
    ("bf16", "bf16", 64, 2, 1, 32, 65, 1500, 0), ("q4", "f32", 128, 8, 2, 32, 65, 2000, 0),
])
def test_attention_of_many_tokens(fmt, dtype, d, hq, hkv, page, tokens, longest, window):
    """Queries of many tokens over a few sequences, at every kind of split; some of them checked."""
    torch = torch_cuda()
    print(f"attention of {tokens} tokens {fmt} {dtype} d={d} {hq}/{hkv} page={page}", flush=True)
    rng = np.random.default_rng(tokens)
    torch.manual_seed(2)
    lens = [longest, 700, 1]
    c = make_cache(fmt, hkv, d, page, lens, rng)
    rows = fill(c, fmt, dtype, lens, rng)
    seq = rng.integers(-1, len(lens) + 1, tokens)
    pos = np.array([rng.integers(-1, lens[s]) if 0 <= s < len(lens) else 5 for s in seq])
    seq[:3], pos[:3] = [0, 1, 2], [n - 1 for n in lens]
    seq[-2:], pos[-2:] = [0, 0], [longest - 1, 0]
    q = dev(rng.standard_normal((tokens, hq, d)), dtype)
    out, lse = attend(c, seq, pos, q, longest, window)
    assert not bool(torch.isnan(out).any()) and not bool(torch.isnan(lse).any())
    some = np.unique(np.r_[0:3, tokens - 2:tokens, rng.integers(0, tokens, 30)])
    check_attention(out[some], lse[some], q[some], seq[some], pos[some], rows, hq, hkv, window)


@pytest.mark.parametrize("fmt,dtype,d,hq", [("q4", "bf16", 64, 3), ("q4", "bf16", 128, 4), ("bf16", "bf16", 64, 2)])
def test_attention_of_one_long_sequence(fmt, dtype, d, hq):
    """Many tiles a wave in every block of the chip, one KV head: 300 000 positions."""
    torch = torch_cuda()
    rng = np.random.default_rng(d)
    n, page = 300_000, 512
    c = make_cache(fmt, 1, d, page, [n], rng)
    k, v = (dev(rng.standard_normal((n, 1, d)).astype(np.float32), dtype) for _ in range(2))
    R.paged_append(c, ints([0] * n), ints(range(n)), k, v)
    back = [torch.empty((n, 1, d), device="cuda") for _ in range(2)] if fmt == "q4" else [k, v]
    if fmt == "q4":          # the stored values, in float32
        R.paged_gather(c, ints([0] * n), ints(range(n)), *back)
    q = dev(rng.standard_normal((1, hq, d)) * 2, dtype)
    out, lse = attend(c, [0], [n - 1], q, n)
    K, V, Q = (x.double() for x in (back[0][:, 0], back[1][:, 0], q[0]))
    s = (Q @ K.T) / math.sqrt(d)
    p = torch.softmax(s, -1)
    want, size = p @ V, float((p @ V.abs()).max())
    spread = float((Q.abs() @ K.abs().T).max()) / math.sqrt(d)
    # the bound of the other tests; and, since the weights' errors of up to 2^-20 (1 + spread) know
    # nothing of the values, an error of the sum of weighted values of that part of its own size
    assert float((out[0].double() - want).abs().max()) <= 2.0 ** -18 * (1 + spread) * size
    assert float((out[0].double() - want).norm() / want.norm()) <= 2.0 ** -20 * (1 + spread)
    assert float((lse[0].double() - torch.logsumexp(s, -1)).abs().max()) <= 2.0 ** -19 * (1 + spread)


@pytest.mark.parametrize("fmt,dtype,d,hq", [
    ("q4", "bf16", 64, 2), ("q4", "bf16", 128, 4), ("q4", "f32", 128, 7), ("bf16", "bf16", 64, 3),
    ("bf16", "bf16", 128, 8), ("f32", "f32", 64, 4)])
@pytest.mark.parametrize("n", [200, 5000])
def test_attention_of_scores_of_any_size(fmt, dtype, d, hq, n):
    """Two equal rows whose scores pass all others by far, at sizes up to 2^100: the mean of their
    values.  A rounded maximum that large is off by more than every exponent of 32 bits."""
    torch = torch_cuda()
    rng = np.random.default_rng(n + d + hq)
    c = make_cache(fmt, 1, d, 16, [n], rng)
    unit = rng.standard_normal((1, 1, d))
    for size in (2.0 ** 8, 2.0 ** 18, 2.0 ** 27, 2.0 ** 50):
        x = rng.standard_normal((n, 1, d)) * 0.01
        x[[n // 3, n - 2]] = unit
        k, v = dev(x * size, dtype), dev(rng.standard_normal((n, 1, d)), dtype)
        R.paged_append(c, ints([0] * n), ints(range(n)), k, v)
        back = [torch.empty((n, 1, d), device="cuda") for _ in range(2)] if fmt == "q4" else [k, v]
        if fmt == "q4":
            R.paged_gather(c, ints([0] * n), ints(range(n)), *back)
        q = dev(np.repeat(unit, hq, 1) * size * (1 + np.arange(hq) / 8)[:, None], dtype)
        out, lse = attend(c, [0], [n - 1], q, n)
        K, V, Q = (y.double() for y in (back[0][:, 0], back[1][:, 0], q[0]))
        s = (Q @ K.T) / math.sqrt(d)
        # the others' weights: at least 0.9 of the score's cosine away, e^-1000 at the smallest size
        assert float((s.max(1).values - s.sort(1).values[:, -3]).min()) > 1000
        want = (V[n // 3] + V[n - 2]) / 2
        # weights of 22 bits and more, a few roundings of the sums
        assert float((out[0].double() - want).abs().max()) <= 2.0 ** -18 * float(V.abs().max())
        spread = (Q.abs() @ K.abs().T).max(1).values / math.sqrt(d)
        assert bool(((lse[0].double() - s.max(1).values - math.log(2)).abs() <= 2.0 ** -19 * (1 + spread)).all())


@pytest.mark.parametrize("fmt,dtype,page", [("q4", "bf16", 32), ("bf16", "bf16", 24), ("f32", "f32", 10)])
def test_attention_pages_that_are_none(fmt, dtype, page):
    """Pages whose ids lie outside the cache are left out, at the start, inside a chunk, whole
    chunks and the end; a sequence with no page at all is empty."""
    torch = torch_cuda()
    rng = np.random.default_rng(8)
    torch.manual_seed(1)
    lens, hq, hkv, d = [1500, 400, 200], 8, 2, 128
    c = make_cache(fmt, hkv, d, page, lens, rng)
    rows = fill(c, fmt, dtype, lens, rng)
    table = c.table.cpu().numpy()
    gone = {}
    for s, drop in ((0, [0, 3, 4] + list(range(300 // page, 1300 // page)) + [(lens[0] - 1) // page]),
                    (1, [1, 5]), (2, range(-(-lens[2] // page)))):
        at = np.zeros(lens[s], bool)
        for i, p in enumerate(drop):
            table[s, p] = (-1, c.k.shape[0], -2 ** 31, 2 ** 31 - 1)[i % 4]
            at[p * page:(p + 1) * page] = True
        gone[s] = at
    c.table.copy_(torch.from_numpy(table))
    q = dev(rng.standard_normal((3, hq, d)), dtype)
    seq, pos = [0, 1, 2], [n - 1 for n in lens]
    for window in (0, 250):
        out, lse = attend(c, seq, pos, q, max(lens), window)
        check_attention(out, lse, q, seq, pos, rows, hq, hkv, window, gone=gone)


@pytest.mark.parametrize("fmt,dtype", [("q4", "bf16"), ("q4", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("recipe", ["growing", "lowest", "huge values", "tiny values", "large scores",
                                    "wide scales", "large queries", "small queries", "zero queries"])
def test_attention_extremes(fmt, dtype, recipe):
    """Scores that grow along the rows (every tile moves the maximum), keys at the type's lowest
    value (scores of -infinity), values and queries of any size, values whose scale changes from
    row to row by powers of two up to 2^60."""
    torch = torch_cuda()
    rng = np.random.default_rng(21)
    n, hq, hkv, d, page = 1200, 8, 2, 128, 48
    c = make_cache(fmt, hkv, d, page, [n], rng)
    q = rng.standard_normal((1, hq, d))
    k, v = (rng.standard_normal((n, hkv, d)) for _ in range(2))
    if recipe == "growing":
        lead = rng.standard_normal(d)
        q = 0.5 * lead + 0.3 * q
        k = 0.3 * k + (4.0 * np.arange(n) / n)[:, None, None] * lead
    elif recipe == "lowest":
        q = np.abs(q) + 0.5
        k[200:900] = -3e38
    elif recipe == "huge values":
        v *= 1e36
    elif recipe == "tiny values":
        v *= 1e-33
    elif recipe == "large scores":
        q *= 30
    elif recipe == "wide scales":
        v *= 2.0 ** rng.integers(-60, 60, (n, 1, 1))
    elif recipe == "large queries":
        q, k = q * 1e30, k * 1e-30
    elif recipe == "small queries":
        q, k = q * 1e-30, k * 1e30
    else:
        q *= 0
    K, V, Q = dev(k, dtype), dev(v, dtype), dev(q, dtype)
    R.paged_append(c, ints([0] * n), ints(range(n)), K, V)
    rows = []
    for name in "kv":
        x = rows_in(c, fmt, name, 0, range(n))
        rows.append(ref.values4(*x) if fmt == "q4" else x)
    out, lse = attend(c, [0], [n - 1], Q, n)
    if recipe == "lowest":       # the float32 scores of those rows are -infinity
        keep = np.r_[0:200, 900:n]
        rows = [x[keep] for x in rows]
        check_attention(out, lse, Q, [0], [len(keep) - 1], [tuple(rows)], hq, hkv)
    else:
        check_attention(out, lse, Q, [0], [n - 1], [tuple(rows)], hq, hkv)


def test_attention_equals_full_attention_on_its_layout():
    """bf16 pages with page_size = max_len and table[b] = b are the layout of full_attention."""
    torch = torch_cuda()
    rng = np.random.default_rng(2)
    B, hq, hkv, d, L = 2, 28, 4, 128, 5003
    k, v = (dev(rng.standard_normal((B, hkv, L, d)), "bf16") for _ in range(2))
    c = R.PagedCache(k, v, ints([[0], [1]]))
    q = dev(rng.standard_normal((B, hq, d)), "bf16")
    h = R.Handle(batch=B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, max_len=L, k=64, cache_cap=0, r=1,
                 window=0, tau=0.8, refresh=0, dtype="bf16")
    for length in (1, 700, L):
        full = torch.empty((B, hq, d), device="cuda")
        h.full(q, k, v, length, full)
        out, _ = attend(c, [0, 1], [length - 1] * 2, q, L)
        assert float((out - full).abs().max()) <= 2e-5 * float(full.abs().max())
    h.close()


def test_appended_rows_feed_the_decode_step():
    """paged_append into the contiguous layout, then retopk_decode_step on it: keys rotated on the
    way give what rotated keys copied in by hand give, bit by bit."""
    torch = torch_cuda()
    rng = np.random.default_rng(4)
    B, hq, hkv, d, N, steps = 2, 8, 2, 64, 300, 4
    maxl, rope = N + steps, rope_of(64, False)
    cfg = dict(batch=B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, max_len=maxl, k=32, cache_cap=8, r=2,
               window=16, tau=0.5, refresh=3, dtype="bf16")
    K, V = (torch.zeros((B, hkv, maxl, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    K2, V2 = K.clone(), V.clone()
    c = R.PagedCache(K, V, ints([[0], [1]]))
    outs = [torch.empty((B, hq, d), device="cuda") for _ in range(2)]
    with R.Handle(**cfg) as h, R.Handle(**cfg) as h2:
        for first, n in [(0, N)] + [(N + i, 1) for i in range(steps)]:
            k, v = (dev(rng.standard_normal((B * n, hkv, d)), "bf16") for _ in range(2))
            q = dev(rng.standard_normal((B * n, hq, d)), "bf16")
            seq, pos = ints(np.repeat(range(B), n)), ints(np.tile(np.arange(first, first + n), B))
            qr, kr = torch.empty_like(q), torch.empty_like(k)
            R.paged_append(c, seq, pos, k, v, rope=rope, q=q, q_out=qr)
            R.rotary_embed(rope, k, pos, kr)
            K2[:, :, first:first + n] = kr.view(B, n, hkv, d).transpose(1, 2)
            V2[:, :, first:first + n] = v.view(B, n, hkv, d).transpose(1, 2)
            if n == 1:
                h.decode_step(qr, K, V, first + 1, outs[0])
                h2.decode_step(qr, K2, V2, first + 1, outs[1])
                torch.cuda.synchronize()
                assert torch.equal(outs[0], outs[1])
        assert torch.equal(K, K2) and torch.equal(V, V2)


# ---------------------------------------------------------------------------
# Streams, graphs, sizes
# ---------------------------------------------------------------------------

def step_of(c, state, ws):
    """One decoding step of every sequence: append with the rotation, then attend."""
    R.paged_append(c, state["seq"], state["pos"], state["k"], state["v"], rope=state["rope"], q=state["q"],
                   q_out=state["qr"])
    R.paged_attention(c, state["seq"], state["pos"], state["qr"], state["out"], state["max_len"],
                      workspace=ws)


@pytest.mark.parametrize("fmt,dtype", [("q4", "bf16"), ("bf16", "bf16"), ("f32", "f32")])
def test_steps_in_two_graphs(fmt, dtype):
    """A step captured for two layers, each graph with its own cache and workspace, replayed on
    two streams while positions and rows change: as the eager steps on copies, every time."""
    torch = torch_cuda()
    rng = np.random.default_rng(17)
    hq, hkv, d, page, lens, more = 8, 2, 128, 16, [900, 3, 0], 6
    rope = rope_of(128, False)
    layers, graphs = [], []
    for _ in range(2):
        pair = [make_cache(fmt, hkv, d, page, [n + more for n in lens], rng) for _ in range(2)]
        for a, b in zip(pair[0].tensors, pair[1].tensors):
            if a is not None:
                b.copy_(a)
        for c in pair:
            fill(c, fmt, dtype, lens, np.random.default_rng(5))
        st = [dict(seq=ints(range(3)), pos=ints([n - 1 for n in lens]), rope=rope, max_len=max(lens) + more,
                   k=torch.zeros((3, hkv, d), dtype=tdt(dtype), device="cuda"),
                   v=torch.zeros((3, hkv, d), dtype=tdt(dtype), device="cuda"),
                   q=torch.zeros((3, hq, d), dtype=tdt(dtype), device="cuda"),
                   qr=torch.zeros((3, hq, d), dtype=tdt(dtype), device="cuda"),
                   out=torch.zeros((3, hq, d), device="cuda")) for _ in range(2)]
        ws = [c.workspace(3, hq, max(lens) + more) for c in pair]
        layers.append((pair, st, ws))
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            step_of(pair[0], st[0], ws[0])
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(more):
        for (pair, st, ws) in layers:
            k, v, q = (dev(rng.standard_normal((3, h, d)), dtype) for h in (hkv, hkv, hq))
            for s in st:
                s["pos"].add_(1)
                s["k"].copy_(k)
                s["v"].copy_(v)
                s["q"].copy_(q)
        torch.cuda.synchronize()
        for g, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                g.replay()
        torch.cuda.synchronize()
        for (pair, st, ws) in layers:
            step_of(pair[1], st[1], ws[1])
            torch.cuda.synchronize()
            assert torch.equal(st[0]["out"], st[1]["out"]) and torch.equal(st[0]["qr"], st[1]["qr"]), i
            for a, b in zip(bytes_of(pair[0]), bytes_of(pair[1])):
                assert torch.equal(a, b), i


def test_a_step_on_another_stream():
    """The work goes to the stream that is passed, after what that stream holds."""
    torch = torch_cuda()
    rng = np.random.default_rng(23)
    hq, hkv, d, n = 4, 1, 128, 2000
    c = make_cache("q4", hkv, d, 64, [n], rng)
    k, v = (dev(rng.standard_normal((n, hkv, d)), "bf16") for _ in range(2))
    q = dev(rng.standard_normal((1, hq, d)), "bf16")
    seq, pos = ints([0] * n), ints(range(n))
    want, outs = torch.empty((1, hq, d), device="cuda"), []
    R.paged_append(c, seq, pos, k, v)
    R.paged_attention(c, seq[:1], pos[-1:], q, want, n)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    busy = torch.ones(1 << 28, device="cuda")
    for kind in (s, s.cuda_stream):
        K, V, Q = torch.zeros_like(k), torch.zeros_like(v), torch.zeros_like(q)
        out = torch.empty_like(want)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for _ in range(4):
                busy.mul_(1.0)
            for a, b in ((K, k), (V, v), (Q, q)):
                a.copy_(b)
        R.paged_append(c, seq, pos, K, V, stream=kind)
        R.paged_attention(c, seq[:1], pos[-1:], Q, out, n, stream=kind)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("fmt,dtype,d", [("f32", "f32", 128), ("q4", "bf16", 64)])
def test_offsets_past_32_bits(fmt, dtype, d):
    """Rows whose byte offset passes 2^32: the last pages of a cache of more than 4 GiB a side."""
    torch = torch_cuda()
    row = {"f32": d * 4, "q4": d // 2}[fmt]
    hkv, page = 8, 256
    n_pages = (5 << 30) // (row * hkv * page)
    c = R.PagedCache.allocate(fmt, n_pages, hkv, page, d, 1, 8)
    ids = [n_pages - 1, 0, n_pages - 2, n_pages // 2, n_pages - 3]
    c.table[0, :5] = ints(ids)
    rng = np.random.default_rng(9)
    rows = fill(c, fmt, dtype, [5 * page - 3], rng)
    q = dev(rng.standard_normal((1, 8, d)), dtype)
    out, lse = attend(c, [0], [5 * page - 4], q, 5 * page)
    check_attention(out, lse, q, [0], [5 * page - 4], rows, 8, hkv)
    k = torch.empty((1, hkv, d), dtype=tdt(dtype), device="cuda")
    R.paged_gather(c, ints([0]), ints([0]), k=k)
    want = torch.from_numpy(rows[0][0][:1].astype(np.float32)).to(tdt(dtype))
    assert torch.equal(k.cpu(), want)


def test_no_tokens_and_refusals_with_tensors():
    torch = torch_cuda()
    c = R.PagedCache.allocate("q4", 2, 1, 16, 64, 1, 2)
    z = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    none = ints([])
    R.paged_append(c, none, none, z(0, 1, 64), z(0, 1, 64))
    R.paged_gather(c, none, none, z(0, 1, 64))
    R.paged_attention(c, none, none, z(0, 2, 64), z(0, 2, 64), 8)
    R.rotary_embed(R.make_rope(64), z(0, 2, 64), none, z(0, 2, 64))
    one, i = z(1, 1, 64), ints([0])
    for bad in (lambda: R.paged_append(c, i, i, one, z(1, 1, 128)),
                lambda: R.paged_append(c, i, i, one.bfloat16(), one),
                lambda: R.paged_append(c, i.long(), i, one, one),
                lambda: R.paged_append(c, ints([0, 1]), i, one, one),
                lambda: R.paged_append(c, i, i, one, one, q=one),
                lambda: R.paged_append(c, i, i, one, one, q=one, q_out=one.clone()),   # no rope
                lambda: R.paged_append(c, i, i, one.half(), one.half()),
                lambda: R.paged_gather(c, i, i, k=one[..., ::2]),
                lambda: R.paged_attention(c, i, i, one, z(1, 1, 32), 8),
                lambda: R.paged_attention(c, i, i, one, z(1, 1, 64).int(), 8),
                lambda: R.paged_attention(c, i, i, one.cpu(), z(1, 1, 64), 8),
                lambda: R.rotary_embed(R.make_rope(64), one, i, z(1, 1, 66)[..., 1:65])):   # misaligned
        with pytest.raises(R.RetopkError):
            bad()
    torch.cuda.synchronize()
