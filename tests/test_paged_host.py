"""The rotary and paged-cache calls on the host: every refusal comes before any device work,
the frequencies follow their formulas, and the split over blocks and the division by the page
size hold over whole ranges (no GPU needed)."""
import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest

from paper_2607_27692_amd import build as B
from paper_2607_27692_amd import retopk as R

ROWS = R.retopk_rows
OK, ARG, UNSUPPORTED, TOO_LARGE = 0, -1, -2, -6


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB):
        B.build()
    return R.load()


def pages(**kw):
    base = dict(format=R.RETOPK_PAGES_Q4, n_kv_heads=2, head_dim=128, page_size=16, n_pages=8,
                n_seqs=2, table_width=4, k=16, v=16, k_par=16, v_par=16, table=16)
    base.update(kw)
    return R.retopk_pages(**base)


BAD_PAGES = [
    (dict(format=3), ARG), (dict(format=-1), ARG), (dict(n_kv_heads=0), ARG),
    (dict(head_dim=0), ARG), (dict(head_dim=96), UNSUPPORTED), (dict(page_size=0), ARG),
    (dict(page_size=24), UNSUPPORTED), (dict(n_pages=0), ARG), (dict(n_seqs=0), ARG),
    (dict(table_width=0), ARG), (dict(k=None), ARG), (dict(v=None), ARG), (dict(k=8), ARG),
    (dict(v=24), ARG), (dict(k_par=None), ARG), (dict(v_par=8), ARG), (dict(table=None), ARG),
    (dict(table=18), ARG), (dict(n_pages=1 << 26), UNSUPPORTED),
    (dict(table_width=1 << 27), UNSUPPORTED),
    (dict(format=R.RETOPK_PAGES_F32), UNSUPPORTED),        # bf16 tokens, f32 pages
]


def calls(lib, c, dtype=R.RETOPK_BF16, n=1):
    """The three calls on pages c; with n = 0 a call that passes its checks does nothing."""
    row, none = ROWS(16, 256, 128), ROWS(None, 0, 0)
    ref = C.byref(c) if c is not None else None
    return [lib.paged_append(ref, None, dtype, n, 16, 16, row, row, 0, none, none, None),
            lib.paged_gather(ref, dtype, n, 16, 16, row, row, None),
            lib.paged_attention(ref, dtype, n, 4, 16, 16, ROWS(16, 512, 128), 64, 0, 16, None, 16,
                                1 << 20, None)]


@pytest.mark.parametrize("bad, code", BAD_PAGES)
def test_pages_are_checked(lib, bad, code):
    assert calls(lib, pages(**bad)) == [code] * 3
    if bad.get("format") != R.RETOPK_PAGES_F32:
        c = pages(**bad)
        assert lib.paged_attention_workspace(C.byref(c), 1, 4, 64, 0) == code


def test_pages_null_and_dtype(lib):
    assert calls(lib, None) == [ARG] * 3
    assert calls(lib, pages(), dtype=2) == [ARG] * 3
    assert calls(lib, pages(format=R.RETOPK_PAGES_BF16), dtype=R.RETOPK_F32) == [UNSUPPORTED] * 3
    assert calls(lib, pages(), n=-1) == [ARG] * 3
    # no tokens: nothing to do, whatever the type
    assert calls(lib, pages(), n=0) == [OK] * 3
    assert calls(lib, pages(page_size=48), R.RETOPK_F32, n=0) == [OK] * 3
    assert calls(lib, pages(format=R.RETOPK_PAGES_BF16, page_size=17, k_par=None), n=0) == [OK] * 3


BAD_ROWS = [ROWS(None, 256, 128), ROWS(8, 256, 128), ROWS(16, -256, 128), ROWS(16, 256, -128),
            ROWS(16, 257, 128), ROWS(16, 256, 132)]


@pytest.mark.parametrize("i", range(len(BAD_ROWS)))
def test_rows_are_checked(lib, i):
    bad, row, none, c = BAD_ROWS[i], ROWS(16, 256, 128), ROWS(None, 0, 0), pages()
    r = R.make_rope(128)
    q = ROWS(16, 512, 128)
    bf = R.RETOPK_BF16
    for k, v in ((bad, row), (row, bad)):
        assert lib.paged_append(C.byref(c), None, bf, 3, 16, 16, k, v, 0, none, none, None) == ARG
    for a, b in ((bad, q), (q, bad)):
        assert lib.paged_append(C.byref(c), C.byref(r), bf, 3, 16, 16, row, row, 4, a, b, None) == ARG
        assert lib.rotary_embed(C.byref(r), bf, 128, 4, 3, 16, a, b, 0, None) == ARG
    if bad.p is not None:
        assert lib.paged_gather(C.byref(c), bf, 3, 16, 16, bad, row, None) == ARG
        assert lib.paged_gather(C.byref(c), bf, 3, 16, 16, row, bad, None) == ARG
    assert lib.paged_attention(C.byref(c), bf, 3, 4, 16, 16, bad, 64, 0, 16, None, 16, 1 << 20,
                               None) == ARG


def test_written_rows_must_not_lie_on_each_other(lib):
    c, r, bf, row = pages(), R.make_rope(128), R.RETOPK_BF16, ROWS(16, 256, 128)
    for bad in (ROWS(16, 0, 128), ROWS(16, 256, 64), ROWS(16, 128, 128), ROWS(16, 248, 128)):
        assert lib.paged_gather(C.byref(c), bf, 3, 16, 16, bad, row, None) == ARG
        assert lib.rotary_embed(C.byref(r), bf, 128, 2, 3, 16, row, bad, 0, None) == ARG
    # in place only with the same strides
    assert lib.rotary_embed(C.byref(r), bf, 128, 2, 3, 16, ROWS(16, 512, 128), row, 0, None) == ARG
    assert lib.paged_append(C.byref(c), C.byref(r), bf, 3, 16, 16, row, row, 2,
                            ROWS(32, 512, 128), ROWS(32, 256, 128), None) == ARG


def test_rotary_arguments(lib):
    r, row, bf = R.make_rope(64), ROWS(16, 256, 128), R.RETOPK_BF16
    fn = lib.rotary_embed
    assert fn(None, bf, 128, 2, 3, 16, row, row, 0, None) == ARG
    assert fn(C.byref(r), 2, 128, 2, 3, 16, row, row, 0, None) == ARG
    assert fn(C.byref(r), bf, 96, 2, 3, 16, row, row, 0, None) == UNSUPPORTED
    assert fn(C.byref(r), bf, 0, 2, 3, 16, row, row, 0, None) == ARG
    assert fn(C.byref(r), bf, 128, 0, 3, 16, row, row, 0, None) == ARG
    assert fn(C.byref(r), bf, 128, 70000, 3, 16, ROWS(16, 128 * 70000, 128), ROWS(32, 128 * 70000, 128),
              0, None) == UNSUPPORTED
    assert fn(C.byref(r), bf, 128, 2, -1, 16, row, row, 0, None) == ARG
    assert fn(C.byref(r), bf, 128, 2, 3, None, row, row, 0, None) == ARG
    assert fn(C.byref(r), bf, 128, 2, 3, 18, row, row, 0, None) == ARG
    assert fn(C.byref(r), bf, 128, 2, 3, 16, row, row, 2, None) == ARG
    assert fn(C.byref(r), bf, 128, 2, 0, None, row, row, 0, None) == OK
    for field, value in (("rot_dim", 0), ("rot_dim", 63), ("rot_dim", 130), ("interleaved", 2),
                         ("factor", float("nan"))):
        bad = R.make_rope(64)
        setattr(bad, field, value)
        assert fn(C.byref(bad), bf, 128, 2, 3, 16, row, row, 0, None) == ARG, field
    wide = R.make_rope(128)
    assert fn(C.byref(wide), bf, 64, 2, 3, 16, row, row, 0, None) == ARG      # rot_dim > d
    wide.freq[63] = float("inf")
    assert fn(C.byref(wide), bf, 128, 2, 3, 16, row, row, 0, None) == ARG


def test_append_and_gather_arguments(lib):
    c, r, row, none = pages(), R.make_rope(128), ROWS(16, 256, 128), ROWS(None, 0, 0)
    bf, q = R.RETOPK_BF16, ROWS(16, 512, 128)
    fn = lib.paged_append
    assert fn(C.byref(c), None, bf, 3, 16, 16, row, row, 4, q, q, None) == ARG    # q needs a rope
    assert fn(C.byref(c), None, bf, 3, 16, 16, row, row, -1, none, none, None) == ARG
    assert fn(C.byref(c), None, bf, 3, None, 16, row, row, 0, none, none, None) == ARG
    assert fn(C.byref(c), None, bf, 3, 16, None, row, row, 0, none, none, None) == ARG
    assert fn(C.byref(c), None, bf, 3, 18, 16, row, row, 0, none, none, None) == ARG
    r.rot_dim = 126 + 4
    assert fn(C.byref(c), C.byref(r), bf, 3, 16, 16, row, row, 0, none, none, None) == ARG
    fn = lib.paged_gather
    assert fn(C.byref(c), bf, 3, None, 16, row, row, None) == ARG
    assert fn(C.byref(c), bf, 3, 16, 17, row, row, None) == ARG
    assert fn(C.byref(c), bf, 3, 16, 16, none, none, None) == OK                   # nothing to write


def test_attention_arguments(lib):
    c, bf, q = pages(), R.RETOPK_BF16, ROWS(16, 512, 128)

    def fn(n=3, hq=4, seq=16, pos=16, rows=q, max_len=64, window=0, out=16, lse=None, ws=16,
           nbytes=1 << 30, cache=c):
        return lib.paged_attention(C.byref(cache), bf, n, hq, seq, pos, rows, max_len, window, out,
                                   lse, ws, nbytes, None)
    for kw in (dict(n=-1), dict(hq=0), dict(hq=3), dict(max_len=0), dict(window=-1),
               dict(seq=None), dict(pos=None), dict(out=None), dict(out=8), dict(lse=2),
               dict(pos=6)):
        assert fn(**kw) == ARG, kw
    assert fn(hq=18) == UNSUPPORTED and fn(n=1 << 31) == UNSUPPORTED
    long = pages(table_width=1 << 16)
    need = lib.paged_attention_workspace(C.byref(long), 3, 4, 1 << 20, 0)
    assert need > 0
    kw = dict(max_len=1 << 20, cache=long)
    assert fn(nbytes=need - 1, **kw) == TOO_LARGE and fn(ws=None, nbytes=0, **kw) == TOO_LARGE
    assert fn(ws=None, nbytes=need, **kw) == ARG and fn(ws=24, nbytes=need, **kw) == ARG
    # a bound past the table's own positions asks for no more than those
    assert lib.paged_attention_workspace(C.byref(c), 3, 4, 1 << 40, 1 << 40) == \
        lib.paged_attention_workspace(C.byref(c), 3, 4, 64, 0) == 0
    assert lib.paged_attention_workspace(C.byref(c), 0, 4, 64, 0) == 0
    assert lib.paged_attention_workspace(None, 1, 4, 64, 0) == ARG


def test_rope_init_refusals(lib):
    r = R.retopk_rope()
    r.rot_dim = 77
    S = R.retopk_rope_scaling

    def fn(rot=64, inter=0, theta=1e4, sc=None):
        return lib.retopk_rope_init(C.byref(r), rot, inter, theta, C.byref(sc) if sc else None)
    nan, inf = float("nan"), float("inf")
    assert lib.retopk_rope_init(None, 64, 0, 1e4, None) == ARG
    for kw in (dict(rot=0), dict(rot=1), dict(rot=130), dict(rot=63), dict(inter=2),
               dict(theta=1.0), dict(theta=nan), dict(theta=inf), dict(sc=S(5, 2, 0, 0, 0)),
               dict(sc=S(-1, 2, 0, 0, 0)), dict(sc=S(1, 0.5, 0, 0, 0)), dict(sc=S(1, nan, 0, 0, 0)),
               dict(sc=S(2, 2, 0, 0, 0), rot=2), dict(sc=S(2, 1e300, 0, 0, 0), rot=4),
               dict(sc=S(3, 2, 0, 1, 4)), dict(sc=S(3, 2, 8192, 0, 4)), dict(sc=S(3, 2, 8192, 4, 4)),
               dict(sc=S(4, 2, 8192, 1, inf)), dict(sc=S(4, 2, -1, 1, 32))):
        assert fn(**kw) == ARG, kw
        assert r.rot_dim == 77                       # left alone
    assert fn(rot=128, inter=1) == OK and r.rot_dim == 128 and r.factor == 1.0
    with pytest.raises(R.RetopkError):
        R.make_rope(64, scaling="other")


@pytest.mark.parametrize("rot", [2, 4, 10, 64, 96, 128])
@pytest.mark.parametrize("theta", [1e4, 5e5])
def test_rope_frequencies(lib, rot, theta):
    """Against scalar evaluations of the documented formulas; a few roundings of 2^-53."""
    f, n0 = 4.0, 8192.0
    plain = [theta ** (-2.0 * i / rot) for i in range(rot // 2)]
    turns = [n0 * w / (2 * math.pi) for w in plain]
    close = lambda a, b: np.testing.assert_allclose(list(a.freq)[:rot // 2], b, rtol=1e-14)  # noqa: E731
    close(R.make_rope(rot, theta), plain)
    close(R.make_rope(rot, theta, scaling="linear", factor=f), [w / f for w in plain])
    if rot > 2:
        base = theta * f ** (rot / (rot - 2))
        close(R.make_rope(rot, theta, scaling="ntk", factor=f),
              [base ** (-2.0 * i / rot) for i in range(rot // 2)])
        # what it is for: the lowest frequency divided by the factor, the highest kept
        got = R.make_rope(rot, theta, scaling="ntk", factor=f).freq
        assert got[0] == 1.0 and abs(got[rot // 2 - 1] * f / plain[-1] - 1) < 1e-12
    mix = [w if n >= 4 else w / f if n <= 1 else w * ((n - 1) / 3 + (1 - (n - 1) / 3) / f)
           for w, n in zip(plain, turns)]
    close(R.make_rope(rot, theta, scaling="bands", factor=f, original_len=n0, low=1, high=4), mix)
    index = lambda n: rot * math.log(n0 / (n * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
    first, last = max(0, math.floor(index(32))), min(rot - 1, math.ceil(index(1)))
    ramp = [min(1, max(0, (i - first) / max(last - first, 1e-3))) for i in range(rot // 2)]
    r = R.make_rope(rot, theta, scaling="ramp", factor=f, original_len=n0, low=1, high=32)
    close(r, [w * (1 - t) + w / f * t for w, t in zip(plain, ramp)])
    assert abs(r.factor - (0.1 * math.log(f) + 1)) < 1e-15
    # a factor of 1 is no scaling
    for kind in ("linear", "ntk", "bands", "ramp") if rot > 2 else ("linear",):
        one = R.make_rope(rot, theta, scaling=kind, factor=1.0, original_len=n0, low=1, high=32)
        close(one, plain)
        assert one.factor == 1.0


PLAN_PROGRAM = r"""
#include "retopk_paged_plan.h"
#include <cstdio>
#include <initializer_list>
#include <vector>
using namespace retopk;
static int bad(const char *what, long long a, long long b) { printf("%s: %lld %lld\n", what, a, b); return 1; }
int main()
{
    // the division: at the multiples of every divisor up to 4096 and of some large ones
    for (int64_t ps = 1; ps < (1 << 24); ps = ps < 4096 ? ps + 1 : ps * 2 + ps / 7) {
        const Divisor d = divisor_of((int32_t)ps);
        for (int64_t q = 0; q < 40; ++q) {
            const int64_t top = (((int64_t)1 << 31) - 1) / ps;
            for (int64_t m : {q, top - q, top / 2 + q, top / 3 - q})
                for (int64_t x : {m * ps - 1, m * ps, m * ps + ps / 2})
                    if (x >= 0 && x < ((int64_t)1 << 31) && divide((uint32_t)x, d) != (uint32_t)(x / ps))
                        return bad("divide", x, ps);
        }
    }
    for (int64_t len = 1; len < ((int64_t)1 << 31); len = len < 600 ? len + 1 : len + len / 3 + 11)
        for (int64_t tokens : {1, 2, 7, 32, 1023, 1024, 1025, 4096})
            for (int64_t hkv : {1, 4, 8, 40})
                for (int64_t w : {0, 1, 31, 32, 33, 4096, 1 << 30}) {
                    const AttendPlan p = attend_plan(tokens, hkv * 4, hkv, 128, len, w, 512, kAttendDirect);
                    // tiles of a token whose window begins as late in its tile as it can
                    int64_t worst = ceil_div(len, kAttendTile);
                    if (w > 0 && w < len) {
                        worst = 0;
                        for (int64_t first = 0; first < 64 && first + w <= len; ++first) {
                            const int64_t n = ceil_div(first + w - first / kAttendTile * kAttendTile, kAttendTile);
                            worst = n > worst ? n : worst;
                        }
                    }
                    if (p.split == ATTEND_DIRECT && (worst > (tokens * hkv * kAttendWaves >= 512 ? kAttendDirectFull : kAttendDirect) || p.waves != tokens * hkv * kAttendWaves || p.workspace))
                        return bad("direct", len, w);
                    if (p.split == ATTEND_BALANCED &&
                        (p.waves < 1 || p.waves > 512 || tokens > kAttendTokens || p.parts != p.waves + tokens * hkv))
                        return bad("balanced", len, p.waves);
                    if (p.split == ATTEND_CHUNKED && (p.chunks * kAttendChunk < worst * kAttendTile || p.waves != tokens * hkv * p.chunks))
                        return bad("chunked", len, p.chunks);
                    if (p.split != ATTEND_DIRECT && p.workspace < p.ends_bytes + p.parts * 4 * 130 * 4)
                        return bad("workspace", len, p.workspace);
                    if (p.ends_bytes % 64 || (p.split == ATTEND_BALANCED && p.ends_bytes < 4 * (tokens + 1)))
                        return bad("ends", tokens, p.ends_bytes);
                }
    // BALANCED: over random lengths, every tile in one part, no number twice, and the numbers the
    // joining kernel computes are the ones the parts were written to
    uint32_t seed = 1;
    auto rnd = [&](uint32_t n) { seed = seed * 1664525u + 1013904223u; return (seed >> 8) % n; };
    for (int round = 0; round < 4000; ++round) {
        const int tokens = 1 + rnd(round % 7 ? 12 : 1024), hkv = 1 + rnd(9), top = 1 + rnd(round % 3 ? 40 : 5000);
        std::vector<int> tiles(tokens), ends(tokens);
        int all = 0, most = 0;
        for (int t = 0; t < tokens; ++t) {
            tiles[t] = rnd(4) ? (int)rnd(top + 1) : 0;
            most = tiles[t] > most ? tiles[t] : most;
            ends[t] = all += tiles[t] * hkv;
        }
        const AttendPlan p = attend_plan(tokens, hkv, hkv, 64, (int64_t)(most <= kAttendDirectFull ? kAttendDirectFull + 1 : most) * kAttendTile, 0, 1 + rnd(512), kAttendDirect);
        if (p.split != ATTEND_BALANCED) return bad("split", tokens, p.split);
        const int per = (int)attend_part(all, (uint32_t)p.waves);
        if ((int64_t)per * p.waves < all) return bad("part", per, all);
        std::vector<int> written(p.parts, -1);
        std::vector<int> covered(tokens * hkv, 0), parts(tokens * hkv, 0);
        for (int64_t b = 0; b < p.waves; ++b)
            for (int64_t at = b * per; at < (b + 1) * per && at < all;) {
                int t = 0;
                while (ends[t] <= at) ++t;
                const int start = t ? ends[t - 1] : 0, g = (int)(at - start) / tiles[t], first = (int)(at - start) % tiles[t];
                int64_t n = tiles[t] - first, left = (b + 1) * per < all ? (b + 1) * per - at : all - at;
                if (n > left) n = left;
                const int group = t * hkv + g;
                if (covered[group] != first) return bad("order", group, first);
                covered[group] += (int)n;
                if (n != tiles[t]) {
                    // the four waves of a block inside the group have one part together
                    const int64_t block = b / kAttendWaves * kAttendWaves, base = start + (int64_t)g * tiles[t];
                    const bool joint = block * per >= base && (block + kAttendWaves) * per <= base + tiles[t];
                    const int64_t id = (joint ? block : b) + group;
                    if (id >= p.parts || (written[id] >= 0 && !(joint && written[id] == group && b != block)))
                        return bad("number", id, group);
                    if (!joint || b == block) parts[group] += 1;
                    written[id] = group;
                }
                at += n;
            }
        for (int t = 0; t < tokens; ++t)
            for (int g = 0; g < hkv; ++g) {
                const int group = t * hkv + g;
                if (covered[group] != tiles[t]) return bad("covered", group, covered[group]);
                const int from = (t ? ends[t - 1] : 0) + g * tiles[t];
                const AttendParts q = attend_parts(from, from + tiles[t], per);
                if (q.count == 1 && q.joints == 0) {   // one wave, which writes the output
                    if (parts[group]) return bad("direct", group, parts[group]);
                    continue;
                }
                if (q.count != parts[group]) return bad("count", q.count, parts[group]);
                for (int c = 0; c < q.count; ++c) {
                    const int extra = c < q.lead ? 0 : c < q.lead + q.joints ? c - q.lead : q.joints;
                    const int64_t id = q.first + group + c + extra * (kAttendWaves - 1);
                    if (id >= p.parts || written[id] != group) return bad("join", id, group);
                    written[id] = -2;
                }
            }
    }
    printf("ok\n");
    return 0;
}
"""


def test_plan_over_ranges(tmp_path):
    src = tmp_path / "plan.cc"
    src.write_text(PLAN_PROGRAM)
    exe = tmp_path / "plan"
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", B.CSRC, str(src), "-o",
                    str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout


def test_binding_refuses_before_the_library():
    """CPU tensors and wrong shapes never reach a kernel."""
    torch = pytest.importorskip("torch")
    z = torch.zeros
    with pytest.raises(R.RetopkError):
        R.PagedCache(z(2, 1, 16, 64), z(2, 1, 16, 64), z(1, 2, dtype=torch.int32))
    with pytest.raises(R.RetopkError):
        R.rotary_embed(R.make_rope(64), z(3, 2, 64), z(3, dtype=torch.int32), z(3, 2, 64))
    with pytest.raises(R.RetopkError):
        R.PagedCache(z(16, 64), z(16, 64), z(1, 2, dtype=torch.int32))


def test_cache_formats_are_checked():
    """Rows of another one-byte type are no codes; formats have three names."""
    torch = pytest.importorskip("torch")
    par, table = (torch.zeros(s, dtype=torch.int32) for s in ((2, 1, 16, 1), (1, 2)))
    for dt in (torch.int8, torch.bool, torch.float8_e4m3fn):
        k = torch.zeros((2, 1, 16, 32), dtype=dt)
        with pytest.raises(R.RetopkError, match="uint8"):
            R.PagedCache(k, k, table, par, par)
    with pytest.raises(R.RetopkError, match="bf16"):
        R.PagedCache.allocate("fp8", 2, 1, 16, 64, 1, 2, device="cpu")


STARTS_PROGRAM = r"""
#include "retopk_paged_plan.h"
#include <cstdio>
#include <vector>
using namespace retopk;
static int bad(const char *what, long long a, long long b) { printf("%s: %lld %lld\n", what, a, b); return 1; }
int main()
{
    // BALANCED with empty tiles before each group's own: as the kernels walk them
    uint32_t seed = 5;
    int most_empty = 0;
    auto rnd = [&](uint32_t n) { seed = seed * 1664525u + 1013904223u; return (seed >> 8) % n; };
    for (int round = 0; round < 6000; ++round) {
        const int tokens = 1 + rnd(round % 7 ? 12 : 1024), hkv = 1 + rnd(9), top = 1 + rnd(round % 3 ? 40 : 5000);
        std::vector<int> tiles(tokens), ends(tokens);
        int sum = 0, most = 0;
        for (int t = 0; t < tokens; ++t) {
            tiles[t] = round % 50 && rnd(4) ? (int)rnd(top + 1) : 0;
            most = tiles[t] > most ? tiles[t] : most;
            ends[t] = sum += tiles[t] * hkv;
        }
        const AttendPlan p = attend_plan(tokens, hkv, hkv, 64, (int64_t)(most <= kAttendDirectFull ? kAttendDirectFull + 1 : most) * kAttendTile, 0, 1 + rnd(2048), kAttendDirect);
        if (p.split != ATTEND_BALANCED || p.ends_bytes < 4 * (tokens + 2)) return bad("split", tokens, p.split);
        const int per = (int)attend_part(sum, (uint32_t)p.waves);
        const int empty = (int)attend_start(sum, (uint32_t)p.waves, (uint32_t)per, (uint32_t)(tokens * hkv));
        most_empty = empty > most_empty ? empty : most_empty;
        const int all = sum + empty * tokens * hkv;
        if (empty < 0 || (int64_t)per * p.waves < all) return bad("start", empty, all);
        for (int t = 0; t < tokens; ++t) ends[t] += (t + 1) * empty * hkv;
        std::vector<int> written(p.parts, -1);
        std::vector<int> covered(tokens * hkv, 0), parts(tokens * hkv, 0), alone(tokens * hkv, 0);
        for (int64_t b = 0; b < p.waves; ++b) {
            const int64_t from = b * per, last = from + per < all ? from + per : all;
            const int64_t block = b / kAttendWaves * kAttendWaves;
            const bool whole = (block + kAttendWaves) * per <= all;
            int shares = 0;
            for (int64_t at = from; at < last;) {
                int t = 0;
                while (ends[t] <= at) ++t;
                const int start = t ? ends[t - 1] : 0, n = (ends[t] - start) / hkv;
                const int first = (int)(at - start) % n, g = (int)(at - start) / n, group = t * hkv + g;
                const int step = n - first < last - at ? n - first : (int)(last - at);
                const int lo = first > empty ? first - empty : 0, hi = first + step - empty;
                const int end = start + (g + 1) * n, base = end - n + empty;
                const bool joint = whole && block * per >= base && (block + kAttendWaves) * per <= end;
                at += step;
                if (joint && (shares || at < last || lo >= hi)) return bad("joint", b, group);
                if (lo >= hi) continue;
                ++shares;
                if (covered[group] != lo) return bad("order", group, lo);
                covered[group] = hi;
                if (first <= empty && first + step == n) {
                    alone[group] = 1;
                    continue;
                }
                const int64_t id = (joint ? block : b) + group;
                if (id >= p.parts || (written[id] >= 0 && !(joint && written[id] == group && b != block)))
                    return bad("number", id, group);
                if (!joint || b == block) parts[group] += 1;
                written[id] = group;
            }
        }
        for (int t = 0; t < tokens; ++t)
            for (int g = 0; g < hkv; ++g) {
                const int group = t * hkv + g, start = t ? ends[t - 1] : 0, n = (ends[t] - start) / hkv;
                if (covered[group] != tiles[t]) return bad("covered", group, covered[group]);
                const AttendParts q = attend_parts(start + g * n + empty, start + (g + 1) * n, per);
                if (q.count == 1 && q.joints == 0) {
                    if (parts[group] || !alone[group]) return bad("direct", group, parts[group]);
                    continue;
                }
                if (alone[group] || q.count != parts[group]) return bad("count", q.count, parts[group]);
                for (int c = 0; c < q.count; ++c) {
                    const int extra = c < q.lead ? 0 : c < q.lead + q.joints ? c - q.lead : q.joints;
                    const int64_t id = q.first + group + c + extra * (kAttendWaves - 1);
                    if (id >= p.parts || written[id] != group) return bad("join", id, group);
                    written[id] = -2;
                }
            }
    }
    if (most_empty != kAttendStart) return bad("never", most_empty, kAttendStart);
    printf("ok\n");
    return 0;
}
"""


def test_plan_with_starts(tmp_path):
    src, exe = tmp_path / "starts.cc", tmp_path / "starts"
    src.write_text(STARTS_PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", B.CSRC, str(src), "-o",
                    str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout
