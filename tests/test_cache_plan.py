"""How attention over the cache splits its work, from the bounds of a batch (host only):
which batches share their groups' prefixes, and which cut the runs of their short sequences.
"""
import os
import subprocess

import pytest

from paper_2609_13804_amd import binding, build as B

HERE = os.path.dirname(os.path.abspath(__file__))
BF16 = 1


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """plan(heads, D, rows of every sequence, own tokens, groups, prefix tokens) -> dict."""
    exe = str(tmp_path_factory.mktemp("plan") / "driver")
    lib = os.path.dirname(binding.LIB_PATH)
    r = subprocess.run([B._hipcc(), "-std=c++17", "-O1", "-I", B.INCLUDE, "-I", B.CSRC, "-x", "hip", "--cuda-host-only",
                        os.path.join(HERE, "host", "plan_driver.hip"), "-o", exe, "-L", lib, "-lstepprune",
                        f"-Wl,-rpath,{lib}"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]

    def ask(heads, D, rows, own, groups, prefix):
        line = " ".join(map(str, (BF16, *heads, D, sum(rows), max(rows), len(rows), own, groups, prefix)))
        out = subprocess.run([exe], input=line + "\n", capture_output=True, text=True, check=True).stdout.split()
        return {k: int(v) for k, v in zip(out[::2], out[1::2])}
    return ask


# us shared / each sequence by itself, warm caches: at the right no more than a tenth is lost
SHARED = [((28, 4), [40, 1], 2000),                        # 21 / 30
          ((28, 4), [40, 1], 131072),                      # 198 / 1257
          ((28, 4), [512, 1], 8192),                       # 87 / 120
          ((28, 4), [512] + [1] * 16, 8192),               # 91 / 159
          ((28, 4), [512] + [1] * 16, 131072),             # 980 / 2087
          ((32, 32), [512, 1], 8192),                      # 118 / 161
          ((32, 32), [2500] + [1] * 16, 8192),             # 431 / 575
          ((28, 4), [2500] + [1] * 127, 8192),             # 416 / 469
          ((28, 4), [2500] + [1] * 127, 131072),           # 5930 / 7900
          ((8, 1), [512] + [1] * 16, 4096),                # 36 / 61
          ((40, 8), [300] * 8 + [1] * 40, 8192),           # 481 / 523
          ((16, 16), [30] * 4 + [1] * 10, 2048)]           # 18 / 26
ALONE = [((28, 4), [96, 60, 24] * 21, 2880),               # 154 / 144 at 2000
         ((28, 4), [12, 8, 3] * 21, 1024),                 # 42 / 26
         ((28, 4), [2500, 1], 2000),                       # 151 / 141
         ((28, 4), [512] + [1] * 16, 1024),                # 41 / 32
         ((32, 8), [2500] + [1] * 16, 2000),               # 165 / 165
         ((32, 8), [300] * 4 + [1], 2000),                 # 69 / 65
         ((28, 4), [900, 500, 200] * 5, 8192),             # 1142 / 1128
         ((32, 32), [60, 40, 20] * 21, 256)]               # 100 / 62


@pytest.mark.parametrize("heads,rows,prefix", SHARED)
def test_tokens_beside_prompts_share_long_prefixes(plan, heads, rows, prefix):
    """A prompt's tiles are cut over its prefix; a token that took the prefix by itself, in
    one workgroup to a key head, would still be at it when they have ended."""
    p = plan(heads, 128, rows, max(max(rows), 65), 1, prefix)
    assert p["alone"] == 0 and p["prefix_parts"] > 0, p


@pytest.mark.parametrize("heads,rows,prefix", ALONE)
def test_prompts_take_their_prefixes(plan, heads, rows, prefix):
    p = plan(heads, 128, rows, max(rows), 4, prefix)
    assert p["alone"] == 1 and p["prefix_parts"] == 0, p


@pytest.mark.parametrize("own,whole", [(500, True), (1000, True), (1024, True), (1100, False), (4000, False)])
def test_short_sequences_among_prompts_take_whole_runs(plan, own, whole):
    """us, in chunks / whole: 4 prompts of 300 to 500 rows 23.1 / 20.8, 16 of 200 to 900 68.0 / 63.5.
    Tokens by themselves are cut as before."""
    rows = [300, 400, 500, 350]
    p = plan((28, 4), 128, rows, own, 0, 0)
    assert (p["chunk_thin"] >= own) == whole, p
    assert plan((28, 4), 128, [1] * 4, max(own, 1000), 0, 0)["short_parts"] > 1
