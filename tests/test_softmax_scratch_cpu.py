"""Every part of softmax cross-entropy's scratch holds what the passes write of it, for each piece of classes, the shorter last one too (no device needed)."""
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.fixture(scope="module")
def layouts(tmp_path_factory):
    """Lines (fp32, forward, N, I, O) to what softmax_layout.hip says of each."""
    at = tmp_path_factory.mktemp("layout")
    obj, exe = str(at / "layout.o"), str(at / "layout")
    subprocess.run([HIPCC, "-O1", "-std=c++17", "--offload-arch=gfx950", "--offload-host-only", "-Wno-unused-function", "-c", os.path.join(HERE, "softmax_layout.hip"),
                    "-o", obj], check=True, capture_output=True)
    # (the launches and the HIP runtime stay unresolved: neither is called)
    subprocess.run(["g++", obj, "-o", exe, "-no-pie", "-Wl,--unresolved-symbols=ignore-all"], check=True, capture_output=True)

    def ask(cases):
        text = "".join("%d %d %d %d %d\n" % c for c in cases)
        got = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(got) == len(cases)
        return got
    return ask


def sweep(seed, count, forward):
    g = random.Random(seed)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** g.random()))   # noqa: E731
    cases = []
    while len(cases) < count:
        N, I, O = log(1, 1 << 18), log(1, 1 << 16), log(1, 1 << 18)
        if N * I < 1 << 31 and O * I < 1 << 31:
            cases.append((g.randint(0, 1), forward, N, I, O))
    return cases


@pytest.mark.parametrize("forward", [0, 1])
def test_parts_hold_what_is_written(layouts, forward):
    cases = sweep(forward, 20000, forward)
    got = layouts(cases)
    bad = [(c, w) for c, w in zip(cases, got) if not w.startswith(("ok", "few", "refused"))]
    assert not bad, (len(bad), bad[:5])
    assert sum(w.startswith("ok") and w.split()[1] != "1" for w in got) > 1000         # several pieces


def test_a_short_last_piece_behind_a_long_one(layouts):
    """fp32 weights of 4096 classes are laid out four rows a work-group, those of a last piece of fewer one by one."""
    cases = [(1, 0, 1024, 4096, 32000), (1, 0, 512, 4096, 8000), (1, 0, 2048, 2048, 32768), (1, 0, 2048, 1024, 65536), (1, 0, 2000, 2048, 50000), (1, 0, 100, 6400, 8000),
             (1, 0, 4096, 64, 15596)]
    for c, w in zip(cases, layouts(cases)):
        assert w.startswith("ok"), (c, w)
        assert int(w.split()[2]) >= 4096 > int(w.split()[3]), (c, w)


def test_sizes_that_the_forward_pass_takes_in_pieces(layouts):
    assert layouts([(1, 1, 65, 8192, 9000), (0, 1, 65, 8193, 17000)]) == ["ok 2 4608 4392", "ok 2 8704 8296"]
