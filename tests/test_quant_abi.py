"""CPU tests of the 8-bit cache's entry points: refusals before any work is enqueued, structure layouts, and
the layout of V's tiles that the header states."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest
import torch

from tests import quant_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "wnw.h")
GOOD = dict(batch=2, layers=3, kv_heads=2, head_dim=128, capacity=256, block=32, format=0, flags=0)


@pytest.fixture(scope="module")
def W():
    from paper_2608_22704_amd import build
    if not os.path.exists(build.LIB):
        build.build()
    from paper_2608_22704_amd import wnw
    return wnw


def calls(W, cfg, cache, first=0, nl=1, n=1, q_heads=4, ptr=4096, ws=4096, ws_bytes=1 << 40, max_len=0, mass=None):
    """Status of the three calls.  No pointer is read before the checks have passed, and each call here must fail."""
    c, k = C.byref(cfg) if cfg else None, C.byref(cache) if cache else None
    return {"write": lambda: W.lib.wnw_quant_write(c, k, first, nl, n, ptr, ptr, ptr, None, None),
            "read": lambda: W.lib.wnw_quant_read(c, k, first, nl, n, ptr, ptr, ptr, None, None),
            "attend": lambda: W.lib.wnw_quant_attend(c, k, first, nl, q_heads, n, ptr, ptr, None, ptr, None, mass, max_len, ws,
                                                     ws_bytes, None)}


def cache_of(W, **over):
    kw = dict(k=4096, v=4096, k_scale=4096, v_scale=4096)
    kw.update(over)
    return W.wnw_quant_cache(**kw)


@pytest.mark.parametrize("over,want", [
    (dict(batch=0), "INVALID"), (dict(layers=0), "INVALID"), (dict(kv_heads=0), "INVALID"),
    (dict(head_dim=96), "UNSUPPORTED"), (dict(block=8), "UNSUPPORTED"), (dict(block=128), "UNSUPPORTED"),
    (dict(capacity=0), "INVALID"), (dict(capacity=100), "INVALID"), (dict(capacity=1 << 25), "UNSUPPORTED"),
    (dict(format=2), "INVALID"), (dict(flags=1), "INVALID"), (dict(kv_heads=1 << 30, batch=4), "UNSUPPORTED"),
])
def test_bad_configurations(W, over, want):
    cfg = W.wnw_quant_config(**{**GOOD, **over})
    for name, call in calls(W, cfg, cache_of(W)).items():
        assert call() == getattr(W, "WNW_ERR_" + want), name
        assert W.lib.wnw_quant_last_error()
    need = C.c_size_t(7)
    assert W.lib.wnw_quant_attend_workspace(C.byref(cfg), 1, max(4, cfg.kv_heads), 1, 0, C.byref(need)) < 0
    assert need.value == 7


@pytest.mark.parametrize("kw,names", [
    (dict(first=-1), "write read attend"), (dict(first=3), "write read attend"), (dict(first=2, nl=2), "write read attend"),
    (dict(nl=0), "write read attend"), (dict(first=1, nl=2147483647), "write read attend"),
    (dict(n=-1), "write read attend"), (dict(n=257), "write read attend"),
    (dict(q_heads=3), "attend"), (dict(q_heads=0), "attend"), (dict(max_len=-1), "attend"),
    (dict(ptr=None), "write attend"), (dict(ptr=4100), "write read attend"),
    (dict(ws=None), "attend"), (dict(ws=4104), "attend"), (dict(ws_bytes=15), "attend"),
    (dict(n=2, mass=4096), "attend"),
])
def test_bad_arguments(W, kw, names):
    cfg = W.wnw_quant_config(**GOOD)
    got = calls(W, cfg, cache_of(W), **kw)
    for name in names.split():
        assert got[name]() == W.WNW_ERR_INVALID, name


def test_bad_caches(W):
    cfg = W.wnw_quant_config(**GOOD)
    for cache in (None, cache_of(W, k=None), cache_of(W, v=None), cache_of(W, k_scale=None), cache_of(W, v_scale=None),
                  cache_of(W, k=4097), cache_of(W, v=4104), cache_of(W, k_scale=4098), cache_of(W, v_scale=4097)):
        for name, call in calls(W, cfg, cache).items():
            assert call() == W.WNW_ERR_INVALID, name
    for name, call in calls(W, None, cache_of(W)).items():
        assert call() == W.WNW_ERR_INVALID, name


def test_sizes_beyond_a_launch(W):
    cfg = W.wnw_quant_config(**{**GOOD, "capacity": 1 << 24, "batch": 1 << 10, "kv_heads": 64})
    got = calls(W, cfg, cache_of(W), n=1 << 24, q_heads=64)
    for name, call in got.items():
        assert call() == W.WNW_ERR_UNSUPPORTED, name


def test_nothing_to_do(W):
    """No rows, no tokens, or no output: nothing is enqueued."""
    cfg = W.wnw_quant_config(**GOOD)
    for name, call in calls(W, cfg, cache_of(W), n=0).items():
        assert call() == W.WNW_OK, name
    assert W.lib.wnw_quant_read(C.byref(cfg), C.byref(cache_of(W)), 0, 1, 4, None, None, 4096, None, None) == W.WNW_OK


def test_workspace_grows_with_the_call(W):
    cfg = W.make_quant_config(1, 4, 2, 16384, 32, W.WNW_QUANT_E4M3)
    one = W.wnw_quant_attend_workspace(cfg, 1, 8, 1)
    assert one > 0 and W.wnw_quant_attend_workspace(cfg, 4, 8, 1) >= one
    assert W.wnw_quant_attend_workspace(cfg, 1, 8, 1, max_len=64) <= one
    for n in (1, 2, 5, 16, 100):
        W.wnw_quant_attend_workspace(cfg, 1, 8, n)
    with pytest.raises(W.WnwError) as e:
        W.wnw_quant_attend_workspace(cfg, 5, 8, 1)
    assert e.value.status == W.WNW_ERR_INVALID


def test_structs_match_the_header(W, tmp_path):
    structs = (W.wnw_quant_config, W.wnw_quant_cache)
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
    values = dict(re.findall(r"\b(WNW_QUANT_[A-Z0-9]+) = (\d)", open(HEADER).read()))
    assert values == {"WNW_QUANT_INT8": "0", "WNW_QUANT_E4M3": "1"}
    assert (W.WNW_QUANT_INT8, W.WNW_QUANT_E4M3) == (0, 1)


def test_binding_refuses_buffers(W):
    """On a machine without a GPU every tensor is on the host, which the binding refuses."""
    cfg = W.make_quant_config(1, 1, 1, 64, 32, W.WNW_QUANT_INT8)
    c = W.make_quant_cache(cfg, device="cpu")
    assert c.v.shape == (1, 1, 1, 1, 128, 64) and c.k_scale.shape == (1, 1, 1, 2)
    x = torch.zeros((1, 1, 1, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        W._on(0, x, W._dtypes()[W._BF16], None, "x")
    with pytest.raises(TypeError):          # half precision is no bf16
        W._on(-1, x.half(), W._dtypes()[W._BF16], None, "x")
    for bad in (x[0], x[..., :64], x.expand(2, 1, 1, 2, 128)):
        with pytest.raises(ValueError):
            W._quant_shape(cfg, bad, 1, "x")
    with pytest.raises(ValueError):
        W.wnw_quant_read(cfg, c, None, None, None)


@pytest.mark.parametrize("name", ["k", "v", "k_scale", "v_scale"])
def test_binding_refuses_a_buffer_that_shrank(W, name):
    """The size is read when a call is made, not when the cache was put together."""
    cfg = W.make_quant_config(1, 2, 1, 128, 32, W.WNW_QUANT_INT8, head_dim=64)
    c = W.make_quant_cache(cfg, device="cpu")
    c._struct(cfg, -1)
    t = getattr(c, name)
    t.resize_(t.numel() - 1)
    with pytest.raises(ValueError, match=name):
        c._struct(cfg, -1)


def test_binding_refuses_a_stream_of_another_device(W, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    class Stream:
        cuda_stream = 4096

        def __init__(self, device):
            self.device = torch.device("cuda", device)
    assert W._quant_place(Stream(0)) == (0, 4096) and W._quant_place(4096) == (0, 4096)
    cfg = W.make_quant_config(1, 1, 1, 64, 32, W.WNW_QUANT_INT8)
    c = W.make_quant_cache(cfg, device="cpu")
    x, out = torch.zeros((1, 1, 1, 2, 128), dtype=torch.bfloat16), torch.zeros((1, 1, 1, 2, 128))
    at = torch.zeros(1, dtype=torch.int32)
    for call in (lambda s: W.wnw_quant_write(cfg, c, x, x, at, stream=s), lambda s: W.wnw_quant_read(cfg, c, out, out, at, stream=s),
                 lambda s: W.wnw_quant_attend(cfg, c, x, out, at, stream=s)):
        with pytest.raises(ValueError, match="stream is on cuda:1"):
            call(Stream(1))


def test_places_of_a_v_tile():
    """Row 16 b + 4 h + i at 16 h + 4 b + i: a permutation, and what the reference encodes it decodes."""
    assert sorted(R.v_place(r) for r in range(64)) == list(range(64))
    for b in range(4):
        for h in range(4):
            for i in range(4):
                assert R.v_place(16 * b + 4 * h + i) == 16 * h + 4 * b + i
    rng = np.random.default_rng(1)
    num = rng.integers(-127, 128, size=(1, 1, 2, 128, 64)).astype(np.float64)
    assert np.array_equal(R.decode_v(R.k_to_v(R.encode(num, R.INT8)), R.INT8), num)


def test_reference_rounding():
    """Ties to even, and the scale rule, on worked examples."""
    assert R.round_to([0.5, 1.5, 2.5, -2.5, -0.5], 1.0, R.INT8).tolist() == [0, 2, 2, -2, 0]
    g = R.e4m3_grid()
    assert g[-1] == 448 and g[1] == 2.0 ** -9 and len(g) == 127
    # between 16 and 18 (codes 88 and 89), and between the subnormals 2^-9 and 2^-8
    assert R.round_to([17.0, 19.0, 1.5 * 2.0 ** -9, 2.0 ** -10], 1.0, R.E4M3).tolist() == [16, 20, 2.0 ** -8, 0]
    assert R.scale_of(127.0, R.INT8) == 1.0 and R.scale_of(0.0, R.INT8) == 2.0 ** -126
    assert R.scale_of(448.0, R.E4M3) == 1.0 and R.scale_of(448.5, R.E4M3) == 2.0 and R.scale_of(0.0, R.E4M3) == 2.0 ** -126
    assert np.isnan(R.scale_of(np.inf, R.INT8))


def test_the_two_references_agree():
    rng = np.random.default_rng(3)
    k, v = (torch.from_numpy(rng.standard_normal((2, 1, 2, 64, 8))) for _ in range(2))
    q = torch.from_numpy(rng.standard_normal((2, 1, 4, 3, 8)))
    for lens, counts in (([64, 10], [3, 2]), ([0, 2], [1, 3])):
        for a, b in zip(R.attend(q, k, v, lens, counts, 16)[:3], R.attend_fast(q, k, v, lens, counts, 16)[:3]):
            assert torch.equal(torch.isnan(a), torch.isnan(b))
            assert torch.allclose(a.nan_to_num(), b.nan_to_num(), rtol=1e-12, atol=1e-12)
