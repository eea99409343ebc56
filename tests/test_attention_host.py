"""Attention operators without a GPU: argument checks of the C entry points, and the frequencies of scaled rotations."""
import json
import math
import subprocess
import sys

import pytest

import paper_2412_04964_amd as fc
import launches

P = 0x10000      # a fake, 16-byte aligned, non-NULL device address; never dereferenced


@pytest.fixture(scope="module")
def L():
    return fc.lib()


def rotary(L, x=P, xt=256, xh=64, table=P, rows=8, positions=P, tokens=4, heads=2, dim=64, turned=64, type=0, y=P, yt=256, yh=64):
    return L.fc_rotary(x, xt, xh, table, rows, positions, tokens, heads, dim, turned, 0, 0, type, y, yt, yh, None)


def test_rotary_argument_checks(L):
    assert rotary(L, type=2) == -8
    assert rotary(L, heads=0) == rotary(L, tokens=-1) == rotary(L, dim=60) == rotary(L, turned=66) == rotary(L, turned=7) == -4
    assert rotary(L, turned=0) == rotary(L, rows=-1) == -4
    assert rotary(L, x=None) == rotary(L, y=None) == rotary(L, table=None) == rotary(L, positions=None) == -1
    assert rotary(L, x=P + 2) == rotary(L, xt=257) == rotary(L, yh=60) == -5
    assert rotary(L, tokens=0, x=None, y=None, table=None, positions=None) == 0
    assert L.fc_rotary_table(P, 4, 7, 1.0, P, None) == L.fc_rotary_table(P, -1, 8, 1.0, P, None) == -4
    assert L.fc_rotary_table(None, 4, 8, 1.0, P, None) == L.fc_rotary_table(P, 4, 8, 1.0, None, None) == -1
    assert L.fc_rotary_table(None, 0, 8, 1.0, None, None) == 0


def append(L, k=P, kt=128, v=P, tokens=4, heads=2, dim=64, type=0, table=P, rows=8, turned=64, quantizer=1, cache=P, scales=P, pages=4, page=16,
           pt=P, width=2, offsets=P, held=P, sequences=2, longest=4):
    return L.fc_cache_append(k, kt, 64, v, 128, 64, tokens, heads, dim, type, table, rows, turned, 0, quantizer, cache, cache, scales, scales,
                             pages, page, pt, width, offsets, held, sequences, longest, None)


def test_append_argument_checks(L):
    assert append(L, type=3) == append(L, quantizer=0) == append(L, quantizer=3) == -8
    assert append(L, dim=96) == append(L, page=8) == append(L, page=48) == append(L, pages=0) == append(L, width=0) == -4
    assert append(L, sequences=0) == append(L, longest=0) == append(L, turned=65) == append(L, turned=66) == append(L, heads=-1) == -4
    for name in ("k", "v", "cache", "scales", "pt", "offsets", "held", "table"):
        assert append(L, **{name: None}) == -1, name
    assert append(L, kt=130) == append(L, k=P + 8) == append(L, cache=P + 4) == -5
    assert append(L, tokens=0, k=None, v=None, cache=None, scales=None, pt=None, offsets=None, held=None, sequences=0) == 0


def attend(L, q=P, qt=512, tokens=2, heads=2, group=4, dim=64, type=0, quantizer=1, cache=P, scales=P, pages=4, page=16, pt=P, width=2,
           offsets=P, held=P, sequences=2, queries=1, longest=64, out=P, ws=P, bytes=0):
    return L.fc_cache_attention(q, qt, 64, tokens, heads, group, dim, type, quantizer, cache, cache, scales, scales, pages, page, pt, width,
                                offsets, held, sequences, queries, longest, 0.1, out, 512, 64, ws, bytes, None)


def test_cache_attention_argument_checks(L):
    assert attend(L, type=-1) == attend(L, quantizer=0) == -8
    assert attend(L, dim=32) == attend(L, group=0) == attend(L, group=40000) == attend(L, queries=0) == attend(L, longest=0) == -4
    assert attend(L, page=128) == attend(L, pages=0) == attend(L, tokens=-1) == attend(L, sequences=-1) == -4
    for name in ("q", "out", "cache", "scales", "pt", "offsets", "held"):
        assert attend(L, **{name: None}) == -1, name
    assert attend(L, qt=4) == attend(L, q=P + 4) == -5
    need = L.fc_cache_attention_workspace_bytes(2, 2, 2, 4, 64, 1, 100000)
    assert need > 0 and need % 4 == 0
    assert attend(L, longest=100000, bytes=need - 1) == attend(L, longest=100000, ws=None, bytes=need) == -6
    assert attend(L, longest=100000, ws=P + 4, bytes=need) == -5
    assert attend(L, tokens=0, q=None, out=None, cache=None) == 0
    for bad in ((2, 2, 2, 4, 32, 1, 100), (2, 2, 0, 4, 64, 1, 100), (-1, 2, 2, 4, 64, 1, 100), (2, 2, 2, 4, 64, 0, 100)):
        assert L.fc_cache_attention_workspace_bytes(*bad) == 0


def test_more_announced_work_never_plans_for_less(L):
    # announced queries and tokens are bounds, up to the largest that their types hold
    most = (1 << 31) - 1
    for sequences, heads in ((256, 8), (65536, 64), (most, 8), (1, 1)):
        for longest in (1 << 20, 1 << 26, most):
            need = [L.fc_cache_attention_workspace_bytes(64, sequences, heads, 8, 128, queries, longest) for queries in (4096, 1 << 20, 1 << 28, most)]
            assert need[0] > 0 and need == [need[0]] * 4, (sequences, heads, longest, need)


def prompt(L, q=P, k=P, v=P, tokens=4, heads=2, group=2, dim=64, type=0, offsets=P, sequences=1, longest=4, out=P, vt=128):
    return L.fc_prompt_attention(q, 256, 64, k, 128, 64, v, vt, 64, tokens, heads, group, dim, type, offsets, sequences, longest, 1, 0.1, out,
                                 256, 64, None)


def test_prompt_attention_argument_checks(L):
    assert prompt(L, type=5) == -8
    assert prompt(L, dim=256) == prompt(L, heads=0) == prompt(L, group=0) == prompt(L, longest=0) == prompt(L, sequences=0) == -4
    for name in ("q", "k", "v", "out", "offsets"):
        assert prompt(L, **{name: None}) == -1, name
    assert prompt(L, vt=129) == prompt(L, out=P + 8) == -5
    assert prompt(L, tokens=0, q=None, k=None, v=None, out=None) == 0


def test_cpu_tensors_are_refused():
    torch = pytest.importorskip("torch")
    x = torch.zeros((2, 2, 64), dtype=torch.float16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        fc.rotary(x, torch.zeros((4, 64)), i)
    with pytest.raises(TypeError):
        fc.prompt_attention(x, x, x, i, 2)


def test_scaled_frequencies():
    torch = pytest.importorskip("torch")
    n, base, factor, original = 64, 10000.0, 8.0, 4096
    plain = fc.rotary_frequencies(n, base)
    want = torch.tensor([base ** (-2 * i / n) for i in range(n // 2)], dtype=torch.float64)
    assert plain.dtype == torch.float64 and torch.allclose(plain, want, rtol=1e-14)
    assert torch.allclose(fc.rotary_frequencies(n, base, "linear", factor), plain / factor, rtol=1e-15)
    moved = fc.rotary_frequencies(n, base, "base", factor) / plain
    assert abs(moved[0] - 1) < 1e-15 and abs(moved[-1] - 1 / factor) < 1e-12
    for method, low, high in (("bands", 1.0, 4.0), ("ramp", 1.0, 32.0)):
        f = fc.rotary_frequencies(n, base, method, factor, original, low, high)
        turns, ratio = original * plain / (2 * math.pi), f / plain
        assert torch.allclose(ratio[turns >= high * 1.5], torch.ones(1, dtype=torch.float64))
        assert torch.allclose(ratio[turns <= low / 1.5], torch.full((1,), 1 / factor, dtype=torch.float64))
        assert bool((ratio[1:] <= ratio[:-1] + 1e-15).all())
    with pytest.raises(ValueError):
        fc.rotary_frequencies(7)
    with pytest.raises(ValueError):
        fc.rotary_frequencies(8, method="other")
    with pytest.raises(ValueError):
        fc.rotary_frequencies(8, method="bands", factor=2.0)


_CHILD = """
import ctypes, json, sys
ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
L = ctypes.CDLL(sys.argv[2])
L.fc_cache_attention_workspace_bytes.restype = ctypes.c_size_t
for name, args in json.load(sys.stdin):
    if name == "fc_cache_attention":
        args[-2] = L.fc_cache_attention_workspace_bytes(*[ctypes.c_int64(args[i]) for i in (3, 19, 4, 5, 6, 20, 21)])
    print("R", getattr(L, name)(*[ctypes.c_float(a) if isinstance(a, float) else ctypes.c_int64(a) for a in args]), flush=True)
"""


def launched(*calls):
    """(return code, launches) of each call, where nothing runs and no address is followed (launches.py)"""
    r = subprocess.run([sys.executable, "-c", _CHILD, launches._stand_in(), launches.LIB], input=json.dumps(calls), capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    out, seen = [], []
    for line in r.stdout.splitlines():
        if line.startswith("L "):
            _, name, grid, block, _ = line.split()
            seen.append((launches._readable(name), int(grid), int(block)))
        else:
            out.append((int(line[2:]), seen))
            seen = []
    return out


def rotary_call(tokens, heads, dim, turned):
    return "fc_rotary", [P, heads * dim, dim, P, 8, P, tokens, heads, dim, turned, 0, 0, 0, P, heads * dim, dim, 0]


def append_call(tokens, heads, dim, page, sequences, longest):
    return "fc_cache_append", [P, heads * dim, dim, P, heads * dim, dim, tokens, heads, dim, 0, 0, 0, 0, 0, 1, P, P, P, P, 1000, page, P, 1000, P, P, sequences, longest, 0]


def cache_call(tokens, heads, group, dim, sequences, queries, longest, width=1000):
    n = heads * group * dim
    return "fc_cache_attention", [P, n, dim, tokens, heads, group, dim, 0, 1, P, P, P, P, 1000, 64, P, width, P, P, sequences, queries, longest, 0.1, P, n, dim, P, 0, 0]


def prompt_call(tokens, heads, group, dim, sequences, longest):
    n = heads * group * dim
    return "fc_prompt_attention", [P, n, dim, P, heads * dim, dim, P, heads * dim, dim, tokens, heads, group, dim, 0, P, sequences, longest, 1, 0.1, P, n, dim, 0]


def test_calls_are_launched_up_to_what_the_runtime_takes():
    fine = [rotary_call(1 << 20, 64, 128, 128), rotary_call((1 << 29) - 64, 1, 128, 128), rotary_call(1 << 20, 60, 80, 24),
            append_call(1 << 22, 64, 64, 16, 1, 1 << 22), append_call(1 << 16, 128, 256, 64, 1 << 16, 1),
            cache_call(1 << 18, 8, 16, 128, 1, 1 << 18, 1 << 18), cache_call(1 << 20, 8, 16, 128, 4, 1 << 18, 1 << 18),
            cache_call(1 << 19, 8, 16, 128, 1 << 19, 1, 300), cache_call(4096, 8, 8, 64, 4096, (1 << 31) - 1, 300), cache_call(1 << 20, 16, 1, 64, 1 << 20, 1, 1 << 15, 1),
            prompt_call(1 << 22, 8, 8, 128, 1, 1 << 22), prompt_call(1 << 24, 8, 8, 64, 1 << 14, 1024)]
    for call, (rc, seen) in zip(fine, launched(*fine)):
        assert rc == 0 and seen, (call, rc, seen)
    # one step more than is launched is refused before anything is
    for call, (rc, seen) in zip(fine, launched(rotary_call(1 << 29, 1, 128, 128), rotary_call(1 << 26, 1, 80, 24), append_call(1 << 30, 64, 256, 16, 1, 1 << 30),
                                               append_call(1 << 30, 16, 256, 64, 1 << 30, 1), cache_call(1 << 28, 64, 16, 64, 1 << 28, 1, 300),
                                               prompt_call((1 << 31) - 1, 1, 1, 64, 1, 1 << 30), prompt_call(1 << 30, 64, 1, 64, 1, 1 << 30))):
        assert rc == -4 and not seen, (rc, seen)
