"""Single calls of dlfp_build_window_meta at the ends of what it takes, each in a process
of its own, built with AddressSanitizer and UndefinedBehaviorSanitizer."""
import json
import os
import random
import shutil
import subprocess
from types import SimpleNamespace

import numpy as np
import pytest

from oracle import window as ow

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host C++ compiler")
    out = str(tmp_path_factory.mktemp("native") / "window_call")
    csrc = os.path.join(ROOT, "paper_2609_38386_amd", "csrc")
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-D__HIP_PLATFORM_AMD__",
           "-I/opt/rocm/include", f"-I{ROOT}/include", f"-I{csrc}",
           os.path.join(ROOT, "tests", "native", "window_call.cpp"),
           os.path.join(csrc, "dlfp_cache.cpp"), os.path.join(csrc, "dlfp_host.cpp"), "-o", out]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    return out


def _call(driver, seqs, hq=1, hkv=1, window=0, sinks=0, decode_split=0, prefill_split=0, target=0,
          tile=0):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    env.pop("LD_PRELOAD", None)
    args = [hq, hkv, window, sinks, decode_split, prefill_split, target, tile,
            *(x for s in seqs for x in s)]
    r = subprocess.run([driver, *map(str, args)], capture_output=True, text=True, env=env,
                       timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    return json.loads(r.stdout)


def _covers(got, seqs, hkv, keys):
    """Every token of every KV head once, its units' ranges end to end over `keys`."""
    assert got["status"] == 0
    rows = {}
    for u in got["units"]:
        assert 0 < u[5] - u[4] <= (32768 if u[11] == 0 else 4096)
        rows.setdefault((u[0], u[1], u[2], u[3]), []).append((u[4], u[5]))
    tokens = {}
    for (s, h, t0, nt), spans in rows.items():
        spans.sort()
        assert spans[0][0] == 0 and all(a[1] == b[0] for a, b in zip(spans, spans[1:]))
        assert spans[-1][1] == keys(*seqs[s], t0, nt)
        tokens[s, h] = tokens.get((s, h), 0) + nt
    assert tokens == {(s, h): q for s, (q, _) in enumerate(seqs) for h in range(hkv)}


def _all_keys(q, kv, t0, nt):
    return kv - q + t0 + nt


# 256 units of 4096 keys are 1048576.
@pytest.mark.parametrize("seqs,hkv,window", [
    ([(1, 1048576)], 1, 0), ([(1, 1048577)], 1, 0), ([(1, 3000001), (1, 5)], 2, 0),
    ([(1, 1048577), (40, 90)], 1, 2 ** 31 - 1), ([(1, 20), (100, 1300000)], 1, 0)])
def test_contexts_past_a_million_keys(driver, seqs, hkv, window):
    _covers(_call(driver, seqs, 2 * hkv, hkv, window), seqs, hkv, _all_keys)


@pytest.mark.parametrize("target", [1, 2, 3, 4, 5, 6, 7, 8, 9, 15, 16, 64])
def test_few_target_units_beside_a_prompt(driver, target):
    seqs = [(1, 300), (40, 90), (1, 7)]
    _covers(_call(driver, seqs, 8, 8, target=target), seqs, 8, _all_keys)
    _covers(_call(driver, seqs, 8, 1, 30, 5, target=target), seqs, 1, _in_window(30, 5))
    _covers(_call(driver, [(1, 9000)], 8, 2, target=target), [(1, 9000)], 2, _all_keys)


def _in_window(window, sinks):
    """Keys that the rows of a tile read: whole pages left out of the others."""
    def keys(q, kv, t0, nt):
        first = kv - q + t0
        low = max(0, first - window + 1) // 16
        return first + nt - 16 * max(0, low - -(-min(sinks, first + nt) // 16))
    return keys


def test_partial_results_of_a_group_below_two_gib(driver):
    """The kernels address a group's partial results in 31 bits: of 128 rows 66560 bytes."""
    fits = 64 * ((2 ** 31 - 1) // 66560)
    got = _call(driver, [(16, fits)], 8, 1, prefill_split=64, tile=16)
    _covers(got, [(16, fits)], 1, _all_keys)
    assert got["groups"] == 1 and got["workspace"] < 2 ** 31 + (1 << 20)
    assert _call(driver, [(16, fits + 64)], 8, 1, prefill_split=64, tile=16)["status"] == -2
    # A group of more than 4 GiB, whose offsets would meet others'.
    assert _call(driver, [(16, 4200000)], 8, 1, prefill_split=64, tile=16)["status"] == -2
    assert _call(driver, [(16, 4200000)], 8, 1)["status"] == 0


def test_keys_up_to_the_end_of_31_bits(driver):
    """The kernels look at most 64 keys past a unit's end: those are counted in 31 bits too.
    A window's keys count without those left out."""
    most = 2 ** 31 - 65
    assert _call(driver, [(1, most + 1)])["status"] == -2
    assert _call(driver, [(2, most + 1)], tile=2)["status"] == -2
    seqs = [(1, 2 ** 31 - 1)]
    _covers(_call(driver, seqs, window=100, sinks=5), seqs, 1, _in_window(100, 5))


@pytest.mark.parametrize("seed", range(24))
def test_random_batches_with_nothing_else_in_the_table(driver, seed):
    """Entries of pages that no row sees are -1, which a builder that looked at them would
    refuse; the list against the mask's definition."""
    rng = random.Random(seed)
    g, hkv = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3])
    window, sinks = rng.choice([1, 2, 16, 17, 33, 100, 640]), rng.choice([0, 0, 1, 15, 16, 17, 70])
    seqs = []
    for _ in range(rng.randint(1, 5)):
        q = 1 if rng.random() < 0.5 else rng.randint(1, 200)
        seqs.append((q, q + rng.choice([0, rng.randint(0, 900)])))
    tuned = dict(decode_split=16 * rng.randint(0, 20), prefill_split=64 * rng.randint(0, 6),
                 target=rng.choice([0, 5, 600]), tile=rng.randint(0, 128 // g)) if seed % 2 else {}
    got = _call(driver, seqs, g * hkv, hkv, window, sinks, **tuned)
    assert got["status"] == 0
    meta = SimpleNamespace(work=np.array(got["units"], np.int32), num_prefill_units=got["prefill"],
                           num_groups=got["groups"], workspace_bytes=got["workspace"])
    q_len, kv_len = zip(*seqs)
    ow.check_window_list(meta, q_len, kv_len, g * hkv, hkv, window, sinks)
