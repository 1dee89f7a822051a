"""Host side of the operators of long contexts on a compressed cache, on a machine without a GPU: what they refuse (before anything is launched), what they
launch (kv4_recorder.cpp), rotary frequencies, and the reference of the GPU tests against pins."""
import json
import math
import os
import subprocess

import numpy as np
import pytest

import kv4_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, SHAPE, SMALL = 0, -1, -2, -3


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    from paper_2510_03283_amd import build
    objs = [os.path.join(build.BUILD_DIR, s[:-4] + ".o") for s in build.sources()]
    if not all(os.path.exists(o) for o in objs):
        build.build_library()
    d = tmp_path_factory.mktemp("kv4")
    obj, exe = str(d / "recorder.o"), str(d / "recorder")
    subprocess.run([build.HIPCC, "-x", "hip", "--offload-host-only", "-fPIE", "-std=c++17", "-O1", "-I", build.CSRC, "-c",
                    os.path.join(ROOT, "tests", "kv4_recorder.cpp"), "-o", obj], check=True)
    subprocess.run(["g++", obj, *objs, "-o", exe], check=True)

    def run(call, **opts):
        out = subprocess.run([exe, call, *(f"{k}={v}" for k, v in opts.items())], capture_output=True, text=True, check=True).stdout
        rec = [json.loads(l) for l in out.splitlines()]
        end = rec[-1]
        return end["status"], end["error"], [r for r in rec if r["op"] == "launch"], next(r["bytes"] for r in rec if r["op"] == "need")

    return run


def nulls(call, names):
    return [(call, dict(null=n), INVALID) for n in names]


REFUSED = [
    *nulls("rotary", ("handle", "x", "positions", "freq", "out")),
    ("rotary", dict(n=-1), INVALID), ("rotary", dict(rot=0), SHAPE), ("rotary", dict(rot=7), SHAPE), ("rotary", dict(rot=66), SHAPE), ("rotary", dict(n_heads=0), SHAPE),
    ("rotary", dict(n_heads=4097), SHAPE), ("rotary", dict(ld_x=383), SHAPE), ("rotary", dict(ld_out=383), SHAPE), ("rotary", dict(ld_x=1 << 31), SHAPE),
    ("rotary", dict(magnitude="nan"), INVALID), ("rotary", dict(magnitude="inf"), INVALID), ("rotary", dict(misalign="x", by=1), INVALID),
    ("rotary", dict(misalign="out", by=2, bf16=0), INVALID), ("rotary", dict(misalign="positions", by=2), INVALID), ("rotary", dict(misalign="freq", by=4), INVALID),
    ("rotary", dict(same="x,out", ld_out=392), INVALID), ("rotary", dict(same="x,out", offset=2), INVALID), ("rotary", dict(same="positions,out"), INVALID),
    ("rotary", dict(same="freq,out"), INVALID), ("rotary", dict(device=1), INVALID),
    *nulls("append", ("handle", "cache", "k", "v", "k_scale", "v_scale", "k_new", "v_new", "slots", "positions")),
    ("append", dict(n=-1), INVALID), ("append", dict(block=0), INVALID), ("append", dict(block=24), INVALID), ("append", dict(block=512), INVALID), ("append", dict(blocks=0), INVALID),
    ("append", dict(blocks=1 << 27), SHAPE), ("append", dict(blocks=1 << 26, hkv=8), SHAPE), ("append", dict(blocks=1 << 40), SHAPE), ("append", dict(heads=2), SHAPE),
    ("append", dict(heads=0), SHAPE), ("append", dict(ld_k=255), SHAPE), ("append", dict(ld_v=260), SHAPE), ("append", dict(ld_v=258, bf16=0), SHAPE), ("append", dict(n=1 << 27), SHAPE),
    ("append", dict(misalign="k", by=8), INVALID), ("append", dict(misalign="v", by=8), INVALID), ("append", dict(misalign="k_scale"), INVALID),
    ("append", dict(misalign="v_scale", by=1), INVALID), ("append", dict(misalign="weight"), INVALID), ("append", dict(misalign="position"), INVALID),
    ("append", dict(misalign="k_new", by=8), INVALID), ("append", dict(misalign="v_new", by=8), INVALID), ("append", dict(misalign="slots"), INVALID),
    ("append", dict(misalign="positions"), INVALID), ("append", dict(same="k,k_new"), INVALID), ("append", dict(same="v_scale,v_new"), INVALID), ("append", dict(same="k,v"), INVALID),
    ("append", dict(same="k_scale,weight"), INVALID), ("append", dict(same="position,slots"), INVALID), ("append", dict(same="weight,positions"), INVALID), ("append", dict(device=1), INVALID),
    *nulls("gather", ("handle", "cache", "k", "k_scale", "slots", "k_out", "v_out")),
    ("gather", dict(n=-1), INVALID), ("gather", dict(heads=3), SHAPE), ("gather", dict(n=1 << 27), SHAPE), ("gather", dict(misalign="k_out", by=8), INVALID),
    ("gather", dict(misalign="slots"), INVALID), ("gather", dict(same="k_out,v_out"), INVALID), ("gather", dict(same="v,k_out"), INVALID), ("gather", dict(same="slots,v_out"), INVALID),
    ("gather", dict(device=1), INVALID),
    *nulls("attention", ("handle", "cache", "v", "v_scale", "q", "block_tables", "lens", "out", "work")),
    ("attention", dict(null="weight", add=1), INVALID), ("attention", dict(n_req=-1), SHAPE), ("attention", dict(n_req=65536), SHAPE), ("attention", dict(max_rows=0), SHAPE),
    ("attention", dict(max_rows=65536), SHAPE), ("attention", dict(n_req=1000, max_rows=1049), SHAPE), ("attention", dict(n_req=100, max_context=1 << 23), SHAPE), ("evict", dict(n_req=100, max_context=1 << 23), SHAPE), ("attention", dict(max_context=-1), SHAPE),
    ("attention", dict(max_context=(1 << 26) + 1), SHAPE), ("attention", dict(n_rows=-1), SHAPE), ("attention", dict(tables=-1), SHAPE), ("attention", dict(n_rows=4), INVALID),
    ("attention", dict(max_rows=2, offsets=0), INVALID), ("attention", dict(heads=2), SHAPE), ("attention", dict(scale="nan"), INVALID), ("attention", dict(scale="inf"), INVALID),
    ("attention", dict(ld_q=504), SHAPE), ("attention", dict(ld_q=516), SHAPE), ("attention", dict(ld_out=511), SHAPE), ("attention", dict(misalign="q", by=8), INVALID),
    ("attention", dict(misalign="out", by=8), INVALID), ("attention", dict(misalign="lse"), INVALID), ("attention", dict(misalign="lens"), INVALID),
    ("attention", dict(misalign="block_tables"), INVALID), ("attention", dict(misalign="q_offsets", max_rows=3), INVALID), ("attention", dict(misalign="work", by=64), INVALID),
    ("attention", dict(work=0), SMALL), ("attention", dict(max_context=100000, work=4096), SMALL), ("attention", dict(same="q,out"), INVALID), ("attention", dict(same="q,lse"), INVALID),
    ("attention", dict(same="k,out"), INVALID), ("attention", dict(same="v_scale,work"), INVALID), ("attention", dict(same="lens,lse"), INVALID), ("attention", dict(same="out,work"), INVALID),
    ("attention", dict(same="block_tables,out"), INVALID), ("attention", dict(same="weight,out", add=1), INVALID), ("attention", dict(same="q_offsets,work", max_rows=2), INVALID),
    ("attention", dict(device=1), INVALID),
    *nulls("evict", ("handle", "cache", "k", "weight", "position", "block_tables", "lens", "seq", "budgets", "new_lens", "work")),
    ("evict", dict(n_req=-1), SHAPE), ("evict", dict(n_req=65536), SHAPE), ("evict", dict(max_context=-1), SHAPE), ("evict", dict(max_context=(1 << 26) + 1), SHAPE),
    ("evict", dict(tables=-1), SHAPE), ("evict", dict(heads=2), SHAPE), ("evict", dict(sink=-1), INVALID), ("evict", dict(recent=-1), INVALID), ("evict", dict(misalign="lens"), INVALID),
    ("evict", dict(misalign="new_lens"), INVALID), ("evict", dict(misalign="work", by=128), INVALID), ("evict", dict(work=0), SMALL), ("evict", dict(same="lens,new_lens"), INVALID),
    ("evict", dict(same="lens,new_lens", heads=4, offset=4), INVALID), ("evict", dict(same="budgets,new_lens"), INVALID), ("evict", dict(same="k,v_scale"), INVALID),
    ("evict", dict(same="weight,position"), INVALID), ("evict", dict(same="new_lens,work"), INVALID), ("evict", dict(same="position,work"), INVALID),
    ("evict", dict(same="position,block_tables"), INVALID), ("evict", dict(device=1), INVALID),
]


@pytest.mark.parametrize("call,opts,status", REFUSED, ids=[f"{c}-{'-'.join(f'{k}={v}' for k, v in o.items())}" for c, o, _ in REFUSED])
def test_refused_before_anything_is_launched(recorder, call, opts, status):
    got, error, launches, _ = recorder(call, **opts)
    assert got == status and error and not launches


GOOD = [("rotary", dict()), ("rotary", dict(n=1, n_heads=4096, hd=128)), ("rotary", dict(n=1 << 20, rot=2, inter=1)), ("rotary", dict(n=(1 << 25) + 3, n_heads=8, hd=128, rot=2, ld_x=1025, ld_out=1025)), ("rotary", dict(n=2**31 - 1, n_heads=1, hd=64)), ("append", dict()), ("append", dict(heads=4, bf16=0)),
        ("append", dict(n=1 << 22, null="position")), ("append", dict(null="weight")), ("gather", dict(hd=128)), ("gather", dict(heads=4, n=1)), ("attention", dict()),
        ("attention", dict(n_req=65535, max_context=100)), ("attention", dict(n_req=1, max_context=1 << 26, add=1)), ("attention", dict(n_req=2, max_rows=65535, group=8)), ("attention", dict(n_req=1000, max_rows=1048, add=1)),
        ("attention", dict(n_req=1, max_rows=33, max_context=0, hd=128, null="lse")), ("evict", dict()), ("evict", dict(n_req=65535, max_context=10)), ("evict", dict(n_req=1, max_context=1 << 26)),
        ("evict", dict(null="seq", recent=0))]


@pytest.mark.parametrize("call,opts", GOOD, ids=[f"{c}-{'-'.join(f'{k}={v}' for k, v in o.items())}" for c, o in GOOD])
def test_good_calls_launch_on_the_callers_stream(recorder, call, opts):
    got, error, launches, _ = recorder(call, **opts)
    assert got == OK, error
    assert launches and all(l["stream"] == 0 and l["block"] <= 1024 for l in launches)
    assert all(l["grid"][0] * l["block"] < 1 << 32 and l["grid"][1] < 1 << 16 and l["grid"][2] < 1 << 16 for l in launches)


def test_nothing_to_do(recorder):
    for call in ("rotary", "append", "gather"):
        assert recorder(call, n=0)[:3] == (OK, "", [])
    assert recorder("attention", n_req=0)[:3] == (OK, "", [])
    assert recorder("attention", n_req=3, max_rows=2, n_rows=0)[:3] == (OK, "", [])
    assert recorder("evict", n_req=0)[:3] == (OK, "", [])


def test_the_same_rows_in_place(recorder):
    assert recorder("rotary", same="x,out")[0] == OK
    assert recorder("rotary", same="x,out", n=1, ld_x=400)[0] == OK                                # one row has no stride
    assert recorder("evict", same="lens,new_lens", heads=4)[0] == OK


def built_kernels(source):
    from paper_2510_03283_amd import build
    lines = subprocess.run(["nm", os.path.join(build.BUILD_DIR, source + ".o")], capture_output=True, text=True, check=True).stdout.splitlines()
    return {l.split()[-1] for l in lines if "_kernel" in l and "__device_stub__" not in l}


def launched(recorder, call, every):
    return {l["kernel"] for opts in every for l in recorder(call, **opts)[2]}


def test_every_kernel_is_reached(recorder):
    """A variant that no call can take is dead code that no test can run either."""
    rot = [dict(bf16=b, inter=i, rot=r, ld_x=ld, ld_out=ld) for b in (0, 1) for i in (0, 1) for r in (64, 56, 24, 36, 62) for ld in (384,)]
    assert launched(recorder, "rotary", rot) == built_kernels("rotary")
    both = [dict(bf16=b, hd=d) for b in (0, 1) for d in (64, 128)]
    assert launched(recorder, "append", both) | launched(recorder, "gather", both) == built_kernels("kv4_cache")
    sizes = [dict(n_req=q, max_rows=r, max_context=c, group=g, add=w, block=s) for w in (0, 1) for q, r, c in ((1, 1, 100), (3, 1, 100000), (5, 3, 500), (4, 40, 300), (64, 1, 4000), (2, 300, 5000), (40, 20, 9000)) for g in (1, 2, 4, 8) for s in (1, 16)]
    assert launched(recorder, "attention", [{**s, **b} for s in sizes for b in both]) == built_kernels("kv4_attention")
    assert launched(recorder, "evict", [dict(hd=d, max_context=c) for d in (64, 128) for c in (100, 3000, 5000, 20000, 40000)]) == built_kernels("kv4_evict")


def test_rotary_frequencies():
    from paper_2510_03283_amd import binding as B
    for rot, theta in ((2, 1e4), (64, 1e4), (128, 5e5), (24, 10.0)):
        i = np.arange(rot // 2)
        f = theta ** (-2.0 * i / rot)
        assert np.allclose(B.mace_rotary_frequencies(rot, theta), f, rtol=4e-16 * 10, atol=0)
        assert np.allclose(B.mace_rotary_frequencies(rot, theta, 8.0), f / 8, rtol=1e-14, atol=0)
        got = B.mace_rotary_frequencies(rot, theta, 8.0, 4096, 1.0, 4.0)
        turns = 4096 * f / (2 * math.pi)
        assert np.allclose(got[turns >= 4], f[turns >= 4], rtol=1e-14, atol=0) and np.allclose(got[turns <= 1], f[turns <= 1] / 8, rtol=1e-14, atol=0)
        mid = (turns > 1) & (turns < 4)
        g = (turns[mid] - 1) / 3
        assert np.allclose(got[mid], f[mid] * (g + (1 - g) / 8), rtol=1e-13, atol=0)
    for bad in (dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=258), dict(theta=0.0), dict(theta=-1.0), dict(theta=float("inf")), dict(factor=0.0), dict(factor=float("nan")),
                dict(original_len=-1), dict(original_len=10, slow=3.0, fast=3.0), dict(original_len=10, slow=float("nan"))):
        with pytest.raises(B.MaceError):
            B.mace_rotary_frequencies(**{**dict(rot_dim=64, theta=1e4), **bad})


def test_reference_pins():
    """The tests' own reference, by hand: borders of the 4-bit rounding and of its scale, and what stays of a small cache."""
    x = np.zeros((1, 32))
    x[0, :9] = 7.0, 0.25, 0.75, -5.0, 2.5, 3.5, 1.25, 1.75, -0.2
    code, scale = R.encode(x)
    assert scale[0, 0] == 127 and list(R.decode(code, scale)[0, :9]) == [6, 0, 1, -4, 2, 4, 1, 2, 0] and code[0, 8] == 8
    x[0, 0] = 7.5
    code, scale = R.encode(x)
    assert scale[0, 0] == 128 and list(R.decode(code, scale)[0, :6]) == [8, 0, 1, -4, 2, 4]      # 7.5 -> 8, 0.25 -> 0 (tie), 0.75 -> 1, 2.5 -> 2 (tie), 3.5 -> 4 (tie)
    assert R.encode(np.zeros((1, 32)))[1][0, 0] == 3 and R.encode(np.full((1, 32), 3e38))[1][0, 0] == 252
    w, p = [0.5, 0.5, float("nan"), 0.1, 9.0, 0.5], [3, 4, 0, 9, 8, 5]
    assert R.kept(w, p, [True] * 6, 3, 1, 9) == [2, 3, 4]               # the sink, the newest, the heaviest
    assert R.kept(w, p, [True] * 6, 2, 0, None) == [0, 4]               # ties: the lower token
    assert R.kept(w, p, [True] * 4 + [False, True], 4, 0, None) == [0, 1, 3, 5]
