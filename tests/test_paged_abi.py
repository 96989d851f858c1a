"""CPU tests of the paged cache's and the draft's entry points: refusals before any work is enqueued, structure layouts,
rotary frequencies, the binding's checks, and the reference that the GPU tests use."""
import ctypes as C
import math
import os
import re
import subprocess

import numpy as np
import pytest
import torch

from tests import paged_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "wnw.h")
GOOD = dict(batch=2, layers=3, kv_heads=2, head_dim=128, page=32, pages=20, table_width=8, flags=0)
PTR = 4096


@pytest.fixture(scope="module")
def W():
    from paper_2608_22704_amd import build
    if not os.path.exists(build.LIB):
        build.build()
    from paper_2608_22704_amd import wnw
    return wnw


def cache_of(W, **over):
    return W.wnw_paged_cache(**{**dict(k=PTR, v=PTR, table=PTR), **over})


def calls(W, cfg, cache, first=0, nl=1, n=1, q_heads=4, max_len=0, ws=PTR, ws_bytes=1 << 40, rot=None, **p):
    """Status of the calls.  No pointer is read before the checks have passed, and each call here must fail."""
    c, k, r = C.byref(cfg) if cfg else None, C.byref(cache) if cache else None, C.byref(rot) if rot else None
    g = lambda name, d=PTR: p.get(name, d)    # noqa: E731
    return {"append": lambda: W.lib.wnw_paged_append(c, k, r, first, nl, q_heads, n, g("k"), g("v"), g("q"), g("q_out"), g("at"),
                                                     g("count", None), g("position", None), None),
            "attend": lambda: W.lib.wnw_paged_attend(c, k, first, nl, q_heads, n, g("q"), g("at"), g("count", None), g("mask", None),
                                                     g("out"), g("lse", None), max_len, ws, ws_bytes, None),
            "keep": lambda: W.lib.wnw_paged_keep(c, k, first, nl, n, g("at"), g("path"), g("count", None), None)}


@pytest.mark.parametrize("over,want", [
    (dict(batch=0), "INVALID"), (dict(layers=0), "INVALID"), (dict(kv_heads=0), "INVALID"), (dict(pages=0), "INVALID"),
    (dict(table_width=0), "INVALID"), (dict(head_dim=96), "UNSUPPORTED"), (dict(page=8), "UNSUPPORTED"),
    (dict(page=48), "UNSUPPORTED"), (dict(page=512), "UNSUPPORTED"), (dict(table_width=1 << 20), "UNSUPPORTED"),
    (dict(table_width=2147483647), "UNSUPPORTED"), (dict(flags=1), "INVALID"), (dict(kv_heads=1 << 30, batch=4), "UNSUPPORTED"),
    (dict(pages=2147483647, layers=2147483647, kv_heads=1 << 20), "UNSUPPORTED"),
])
def test_bad_configurations(W, over, want):
    cfg = W.wnw_paged_config(**{**GOOD, **over})
    for name, call in calls(W, cfg, cache_of(W)).items():
        assert call() == getattr(W, "WNW_ERR_" + want), name
        assert W.lib.wnw_paged_last_error()
    need = C.c_size_t(7)
    assert W.lib.wnw_paged_attend_workspace(C.byref(cfg), 1, max(4, cfg.kv_heads), 1, 0, C.byref(need)) < 0
    assert need.value == 7


@pytest.mark.parametrize("kw,names", [
    (dict(first=-1), "append attend keep"), (dict(first=3), "append attend keep"), (dict(first=2, nl=2), "append attend keep"),
    (dict(nl=0), "append attend keep"), (dict(first=1, nl=2147483647), "append attend keep"),
    (dict(n=-1), "append attend keep"), (dict(n=257), "append attend"),
    (dict(q_heads=3), "attend"), (dict(q_heads=0), "append attend"), (dict(max_len=-1), "attend"),
    (dict(k=None), "append"), (dict(v=None), "append"), (dict(q=None), "append attend"), (dict(q_out=None), "append"),
    (dict(k=None, v=None, q=None, q_out=None), "append"),
    (dict(at=None), "append attend keep"), (dict(out=None), "attend"), (dict(path=None), "keep"),
    (dict(k=4104), "append"), (dict(v=4100), "append"), (dict(q=4104), "append attend"), (dict(q_out=4097), "append"),
    (dict(out=4104), "attend"), (dict(at=4098), "append attend keep"), (dict(count=4097), "append attend keep"),
    (dict(position=4098), "append"), (dict(path=4098), "keep"), (dict(mask=4100), "attend"), (dict(lse=4098), "attend"),
    (dict(ws=None), "attend"), (dict(ws=4104), "attend"), (dict(ws_bytes=15), "attend"),
])
def test_bad_arguments(W, kw, names):
    # (for so many rows attention needs a workspace)
    cfg = W.wnw_paged_config(**{**GOOD, "table_width": 2000 if "ws" in kw or "ws_bytes" in kw else 8})
    got = calls(W, cfg, cache_of(W), **kw)
    for name in names.split():
        assert got[name]() == W.WNW_ERR_INVALID, name


def test_long_paths_are_refused(W):
    cfg = W.wnw_paged_config(**{**GOOD, "table_width": 100})
    assert calls(W, cfg, cache_of(W), n=1025)["keep"]() == W.WNW_ERR_UNSUPPORTED


@pytest.mark.parametrize("rot", [dict(dim=3), dict(dim=130), dict(dim=-2), dict(layout=2), dict(amplitude=math.nan),
                                 dict(amplitude=math.inf), dict(freq=None), dict(freq=4098)])
def test_bad_rotations(W, rot):
    r = W.wnw_rotary(**{**dict(freq=PTR, dim=64, layout=0, amplitude=1.0), **rot})
    assert calls(W, W.wnw_paged_config(**GOOD), cache_of(W), rot=r)["append"]() == W.WNW_ERR_INVALID


def test_bad_caches(W):
    cfg = W.wnw_paged_config(**GOOD)
    for cache in (None, cache_of(W, k=None), cache_of(W, v=None), cache_of(W, table=None), cache_of(W, k=4097), cache_of(W, v=4104),
                  cache_of(W, table=4098)):
        for name, call in calls(W, cfg, cache).items():
            assert call() == W.WNW_ERR_INVALID, name
    for name, call in calls(W, None, cache_of(W)).items():
        assert call() == W.WNW_ERR_INVALID, name


def test_sizes_beyond_a_launch(W):
    cfg = W.wnw_paged_config(**{**GOOD, "table_width": 1 << 19, "batch": 1 << 10, "kv_heads": 64})
    got = calls(W, cfg, cache_of(W), n=1 << 24, q_heads=64)
    assert got["append"]() == W.WNW_ERR_UNSUPPORTED
    assert got["attend"]() == W.WNW_ERR_UNSUPPORTED
    cfg = W.wnw_paged_config(**{**GOOD, "batch": 1, "layers": 1, "pages": 1, "kv_heads": (1 << 30) - 1})
    assert calls(W, cfg, cache_of(W), nl=1)["append"]() == W.WNW_ERR_UNSUPPORTED


def test_nothing_to_do(W):
    cfg = W.wnw_paged_config(**GOOD)
    for name, call in calls(W, cfg, cache_of(W), n=0).items():
        assert call() == W.WNW_OK, name
    assert W.wnw_paged_attend_workspace(cfg, 1, 4, 0) == 0


def test_workspaces(W):
    cfg = W.make_paged_config(1, 4, 2, 16, 2000, 1000)
    one = W.wnw_paged_attend_workspace(cfg, 1, 8, 1)
    assert one > 0 and W.wnw_paged_attend_workspace(cfg, 1, 8, 1, max_len=64) <= one
    for n in (1, 2, 5, 16, 100):
        W.wnw_paged_attend_workspace(cfg, 4, 8, n)
    with pytest.raises(W.WnwError) as e:
        W.wnw_paged_attend_workspace(cfg, 5, 8, 1)
    assert e.value.status == W.WNW_ERR_INVALID
    assert W.wnw_draft_verify_workspace(3, 10, 131072) > W.wnw_draft_verify_workspace(1, 10, 131072) > 0
    assert W.wnw_draft_verify_workspace(3, 10, 1000) == 0
    with pytest.raises(W.WnwError):
        W.wnw_draft_verify_workspace(3, 10, 0)


def drafts(W, B=2, n=4, V=131072, ws=PTR, ws_bytes=1 << 40, **p):
    g = lambda name, d=PTR: p.get(name, d)    # noqa: E731
    return {"tree": lambda: W.lib.wnw_draft_tree(B, n, g("parent"), g("base"), g("count", None), g("mask"), g("position"), None),
            "verify": lambda: W.lib.wnw_draft_verify(B, n, V, g("token"), g("parent", None), g("count", None), g("target"),
                                                     g("draft", None), g("uniform"), g("path"), g("accepted"), g("next"), ws, ws_bytes, None)}


@pytest.mark.parametrize("kw,want,names", [
    (dict(B=0), "INVALID", "tree verify"), (dict(n=-1), "INVALID", "tree verify"), (dict(n=1025), "UNSUPPORTED", "tree verify"),
    (dict(B=1 << 21), "UNSUPPORTED", "tree verify"), (dict(B=1 << 20, n=1024), "UNSUPPORTED", "tree"), (dict(V=0), "INVALID", "verify"), (dict(V=(1 << 24) + 1), "UNSUPPORTED", "verify"),
    (dict(parent=None), "INVALID", "tree"), (dict(base=None), "INVALID", "tree"), (dict(parent=4098), "INVALID", "tree verify"),
    (dict(mask=4100), "INVALID", "tree"), (dict(position=4098), "INVALID", "tree"), (dict(count=4097), "INVALID", "tree verify"),
    (dict(token=None), "INVALID", "verify"), (dict(target=None), "INVALID", "verify"), (dict(uniform=None), "INVALID", "verify"),
    (dict(path=None), "INVALID", "verify"), (dict(accepted=None), "INVALID", "verify"), (dict(next=None), "INVALID", "verify"),
    (dict(target=4098), "INVALID", "verify"), (dict(draft=4098), "INVALID", "verify"),
    (dict(ws=None), "INVALID", "verify"), (dict(ws=4104), "INVALID", "verify"), (dict(ws_bytes=3), "INVALID", "verify"),
])
def test_bad_drafts(W, kw, want, names):
    got = drafts(W, **kw)
    for name in names.split():
        assert got[name]() == getattr(W, "WNW_ERR_" + want), name
        assert W.lib.wnw_draft_last_error()


def test_empty_drafts(W):
    assert drafts(W, n=0)["tree"]() == W.WNW_OK
    assert drafts(W, mask=None, position=None)["tree"]() == W.WNW_OK


def test_structs_match_the_header(W, tmp_path):
    structs = (W.wnw_paged_config, W.wnw_paged_cache, W.wnw_rotary)
    lines = []
    for st in structs:
        lines.append(f'printf("{st.__name__} sizeof %zu\\n", sizeof({st.__name__}));')
        lines += [f'printf("{st.__name__} {f} %zu\\n", offsetof({st.__name__}, {f}));' for f, _ in st._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "wnw.h"\nint main(void){\n' + "\n".join(lines) +
                   "\nreturn 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    got = {tuple(line.split()[:2]): int(line.split()[2]) for line in out.splitlines()}
    for st in structs:
        assert got[(st.__name__, "sizeof")] == C.sizeof(st)
        for f, _ in st._fields_:
            assert got[(st.__name__, f)] == getattr(st, f).offset, f
    values = dict(re.findall(r"\b(WNW_ROTARY_[A-Z]+) = (\d)", open(HEADER).read()))
    assert values == {"WNW_ROTARY_HALVES": str(W.WNW_ROTARY_HALVES), "WNW_ROTARY_PAIRS": str(W.WNW_ROTARY_PAIRS)}


def test_rotary_frequencies(W):
    """Against the formula, in 64 bits, rounded once: half a step, 2^-24, and the exponential's own error."""
    for dim, base, factor, low, high, length in ((128, 1e4, 1, 0, 0, 0), (64, 5e5, 8, 1, 4, 8192), (2, 10.0, 2, 3, 3, 100),
                                                 (6, 1e6, 4, math.inf, math.inf, 1 << 40), (0, 1e4, 1, 0, 0, 0), (80, 1e4, 32, 1, 32, 4096)):
        got = W.wnw_rotary_frequencies(dim, base, factor, low, high, length)
        assert got.shape == (dim // 2,) and got.dtype == np.float32
        for i in range(dim // 2):
            f = base ** (-2 * i / dim)
            r = length * f / (2 * math.pi)
            if r < low:
                want = f / factor
            elif r > high or low == high:
                want = f
            else:
                want = (f / factor * (high - r) + f * (r - low)) / (high - low)
            assert abs(got[i] - want) <= (2 ** -24 + 2 ** -48) * want, (dim, i)
    for bad in (dict(dim=3), dict(dim=-2), dict(base=0.0), dict(base=math.nan), dict(base=math.inf), dict(factor=0.5), dict(factor=math.nan),
                dict(low=-1.0), dict(low=2.0, high=1.0), dict(high=math.nan), dict(original_len=-1)):
        with pytest.raises(W.WnwError) as e:
            W.wnw_rotary_frequencies(**{**dict(dim=64, base=1e4, factor=2.0, low=1.0, high=4.0, original_len=100), **bad})
        assert e.value.status == W.WNW_ERR_INVALID
    assert W.lib.wnw_rotary_frequencies(4, 1e4, 1.0, 0.0, 0.0, 0, None) == W.WNW_ERR_INVALID


def test_binding_refuses_buffers(W, monkeypatch):
    """On a machine without a GPU every tensor is on the host, which the binding refuses."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    cfg = W.make_paged_config(2, 1, 1, 16, 3, 2, head_dim=64)
    c = W.make_paged_cache(cfg, device="cpu")
    assert c.k.shape == (3, 1, 1, 16, 64) and c.table.shape == (2, 2) and (c.table == -1).all()
    x, at = torch.zeros((2, 1, 1, 3, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    out = torch.zeros(x.shape)
    with pytest.raises(ValueError, match="cuda:0"):
        W.wnw_paged_append(cfg, c, x, x, at, stream=0)
    for bad in (lambda: W.wnw_paged_append(cfg, c, None, None, at, stream=0), lambda: W.wnw_paged_append(cfg, c, x, None, at, stream=0),
                lambda: W.wnw_paged_append(cfg, c, x, x, at, q_dev=x, stream=0), lambda: W.wnw_paged_append(cfg, c, x, x[:, :, :, :2], at, stream=0),
                lambda: W.wnw_paged_append(cfg, c, x, x, at, q_dev=x[:, :, :, :2], q_out=x[:, :, :, :2], stream=0),
                lambda: W.wnw_paged_append(cfg, c, x[0], x[0], at, stream=0), lambda: W.wnw_paged_attend(cfg, c, x, out[:, :, :, :2], at, stream=0),
                lambda: W.wnw_paged_attend(cfg, c, x[:1], out[:1], at, stream=0), lambda: W.wnw_paged_keep(cfg, c, at, at, stream=0),
                lambda: W.wnw_paged_keep(cfg, c, at, torch.zeros((3, 2), dtype=torch.int32), stream=0)):
        with pytest.raises(ValueError):
            bad()
    for name, t in (("k", x.half()), ("v", x.float()), ("table", at.long())):
        with pytest.raises(TypeError):
            setattr(c, name, t)
    with pytest.raises(ValueError):
        c.table = torch.zeros((2, 4), dtype=torch.int32)[:, ::2]
    with pytest.raises(TypeError):
        W.make_rotary(torch.zeros(32, dtype=torch.float64), 64)
    with pytest.raises(ValueError):
        W.make_rotary(torch.zeros(31), 64)
    with pytest.raises(ValueError):
        W.make_rotary(None, 64)
    token, target = torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 4, 10))
    for t, d in ((target[:, :3], None), (target, target[:, :, :5]), (target[0], None)):
        with pytest.raises(ValueError):
            W.wnw_draft_verify(token, t, torch.zeros((2, 4)), token, at, at, draft_dev=d, stream=0)


@pytest.mark.parametrize("name", ["k", "v", "table"])
def test_binding_refuses_a_buffer_that_shrank(W, name):
    cfg = W.make_paged_config(2, 1, 1, 16, 3, 2, head_dim=64)
    c = W.make_paged_cache(cfg, device="cpu")
    c._struct(cfg, -1)
    t = getattr(c, name)
    t.resize_(t.numel() - 1)
    with pytest.raises(ValueError, match=name):
        c._struct(cfg, -1)


def test_reference_verification_keeps_the_target():
    """The definition itself: over tokens drawn from the draft and all random numbers, what comes first is distributed as the target says
    (two siblings, a vocabulary of four; the uniform numbers on a fine grid)."""
    p, q = np.array([0.5, 0.25, 0.2, 0.05]), np.array([0.125, 0.375, 0.25, 0.25])
    target, draft = np.tile(p, (3, 1)), np.tile(q, (3, 1))
    m = 64
    grid = (np.arange(m) + 0.5) / m
    got = np.zeros(4)
    for x in range(4):
        for y in range(4):
            weight = q[x] * q[y]
            for u0 in grid:
                path, _ = R.verify([x, y], [-1, -1], 1, target, draft, [u0, 0.5, 0.5])
                if path:
                    got[x] += weight / m
                    continue
                for u1 in grid:
                    path, _ = R.verify([x, y], [-1, -1], 2, target, draft, [u0, u1, 0.5])
                    if path:
                        got[y] += weight / m / m
                    else:
                        for u2 in grid[::8]:
                            got[R.verify([x, y], [-1, -1], 2, target, draft, [u0, u1, u2])[1]] += weight / m / m / (m // 8)
    # a grid of m points is off by at most half a cell for each of the three numbers, of which the last has m / 8 points
    assert abs(got.sum() - 1) < 1e-12
    assert np.abs(got - p).max() < 0.5 / m + 0.5 / m + 0.5 * 8 / m * 0.5, got


def test_reference_trees():
    see = R.ancestors([-1, 0, 0, 1, 7, -1])
    assert see.astype(int).tolist() == [[1, 0, 0, 0, 0, 0], [1, 1, 0, 0, 0, 0], [1, 0, 1, 0, 0, 0], [1, 1, 0, 1, 0, 0],
                                        [0, 0, 0, 0, 1, 0], [0, 0, 0, 0, 0, 1]]
    w = R.words(np.tril(np.ones((70, 70), dtype=bool)))
    assert w.shape == (70, 2) and w[63, 0] == -1 and w[69].tolist() == [-1, 63]
