"""The work list of the attention over the 4-bit cache (tests/probes/kv_shares, without a GPU, for 256 compute units): with a window a
sequence's last tile of rows may go through fewer steps than an earlier one, whose shares outnumbered the items that it owned."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def shares(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("kv_shares") / "kv_shares")
    subprocess.run(["hipcc", "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17",
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2411_07942_amd", "csrc"),
                    os.path.join(ROOT, "tests", "probes", "kv_shares.hip"), "-o", exe], check=True, capture_output=True, text=True)

    def run(batches, random=0):
        """batches: heads, R, D, G, page, window, sinks, max_len, table entries, [(length, new)]; returns the counts that are printed."""
        text = "".join(" ".join(map(str, (*b[:-1], len(b[-1]), *(v for s in b[-1] for v in s)))) + "\n" for b in batches)
        r = subprocess.run([exe, str(random)], input=text, check=True, capture_output=True, text=True, timeout=100)
        words = r.stdout.split()
        return dict(zip((w.strip(",") for w in words[1::2]), map(int, words[0::2]))), r.stderr
    return run


WINDOWS = [  # the last tile of rows has fewer rows than the others, or lies better on the tiles of tokens
    (1, 4, 128, 128, 16, 512, 0, 8192, 512, [(8192, 5)]),
    (8, 2, 128, 128, 16, 1000, 0, 2000, 125, [(2000, 16)]),
    (8, 2, 128, 128, 16, 512, 4, 8192, 512, [(8192, 200)] * 4),
    (8, 8, 128, 128, 16, 1024, 4, 3000, 188, [(3000, 64)] * 4),
    (2, 2, 128, 128, 16, 4096, 0, 8192, 512, [(8192, 9)]),
    (2, 2, 128, 128, 16, 4096, 0, 8192, 512, [(8192, 9)] * 4),
    (32, 1, 128, 128, 16, 1024, 0, 2050, 129, [(2050, 385)]),
    (1, 1, 64, 64, 16, 600, 0, 3000, 188, [(3000 - b, 17) for b in range(70)]),
]


@pytest.mark.parametrize("batch", WINDOWS)
def test_shares_of_windowed_tiles(shares, batch):
    counts, faults = shares([batch])
    assert counts["batches"] == counts["cut"] == 1 and counts["faults"] == 0, faults


def test_shares_of_random_batches(shares):
    counts, faults = shares([], 300000)
    assert counts["batches"] == 300000 and counts["cut"] > 50000 and counts["faults"] == 0, faults
