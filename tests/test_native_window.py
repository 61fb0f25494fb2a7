"""The host half of dlfp_cache.h built with AddressSanitizer and UndefinedBehaviorSanitizer.

The metadata builder runs on seeded random batches, windows and tunings with
tables of exactly the entries it may read; every work list is checked against
the mask's definition.
"""
import json
import os
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
    out = str(tmp_path_factory.mktemp("native") / "window_driver")
    csrc = os.path.join(ROOT, "paper_2609_38386_amd", "csrc")
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-D__HIP_PLATFORM_AMD__",
           "-I/opt/rocm/include", f"-I{ROOT}/include", f"-I{csrc}",
           os.path.join(ROOT, "tests", "native", "window_driver.cpp"),
           os.path.join(csrc, "dlfp_cache.cpp"), os.path.join(csrc, "dlfp_host.cpp"), "-o", out]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    return out


@pytest.mark.parametrize("seed", [1, 2, 3])
def test_window_metadata_under_sanitizers(driver, seed):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([driver, str(seed), "25"], capture_output=True, text=True, env=env,
                       timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    *cases, last = [json.loads(x) for x in r.stdout.splitlines()]
    assert last["refused"] == [-1] * 6 + [-5]
    for c in cases:
        assert c["status"] == 0 and c["probe"] in (0, -3)
        meta = SimpleNamespace(work=np.array(c["work"], np.int32).reshape(-1, 16),
                               num_prefill_units=c["prefill"], num_groups=c["groups"],
                               workspace_bytes=c["workspace"])
        ow.check_window_list(meta, c["q_len"], c["kv_len"], c["hq"], c["hkv"],
                             c["window"] or None, c["sinks"])
        cu = np.concatenate([[0], np.cumsum(c["q_len"])]).astype(int)
        assert c["cu_q"] == cu.tolist()
        want = [(s * c["max_blocks"] + p // 16) * 16 + p % 16
                for s, (q, kv) in enumerate(zip(c["q_len"], c["kv_len"])) for p in range(kv - q, kv)]
        assert c["slots"] == want
