"""The barriers in the walks of softmax cross-entropy's products, as the compiler leaves them (no device).

Behind a barrier loads overwrite a tile that fragments were read from, so each wavefront has to have its reads behind it, and its loads to the
count that may stay, when it comes there."""
import importlib.util
import os
import re
import subprocess

import pytest

# (by path: the package loads its library, and the HIP runtime with it, which has to come behind torch's for the GPU tests of the same process)
PACKAGE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1404_5997_amd")
spec = importlib.util.spec_from_file_location("_owt_build", os.path.join(PACKAGE, "build.py"))
build = importlib.util.module_from_spec(spec)
spec.loader.exec_module(build)


@pytest.mark.parametrize("half,out,kernels", [(0, 0, 8), (0, 1, 15), (1, 0, 10), (1, 1, 17)])
def test_every_barrier_of_a_walk_waits_for_the_reads_before_it(tmp_path, half, out, kernels):
    path = str(tmp_path / "k.s")
    subprocess.run([build.HIPCC] + build.FLAGS + ["-DOWT_INST_HALF=%d" % half, "-DOWT_INST_OUT=%d" % out, "--cuda-device-only", "-S", "-o", path,
                                                  os.path.join(build.CSRC, "softmax_inst.hip")], check=True, capture_output=True)
    with open(path) as f:
        found = re.findall(r"^(_ZN3owt\d+sm_(?:pair_)?kernel\w+):(.*?)^\.Lfunc_end", f.read(), re.M | re.S)
    assert len(found) == kernels, [n for n, _ in found]
    for name, body in found:
        code = [l.strip() for l in body.splitlines() if l.startswith("\t") and not l.strip().startswith((";", "."))]
        assert not any(l.startswith("scratch_") for l in code), name         # nothing is spilled
        waits = []
        for i, l in enumerate(code):
            if l.startswith("s_barrier"):
                back = next(k for k in range(1, i) if code[i - k].startswith("s_waitcnt"))      # (scalar arithmetic may stand in between)
                assert not any(c.startswith(("ds_", "global_load", "buffer_load", "v_mfma")) for c in code[i - back + 1:i]), (name, code[i - back:i])
                waits.append(code[i - back])
        # (those in front of a walk and behind it, where words are handed on through LDS, count no loads)
        assert all(re.fullmatch(r"s_waitcnt (vmcnt\(\d+\) )?lgkmcnt\(0\)", w) for w in waits), (name, waits)
        assert sum("vmcnt" in w for w in waits) >= (4 if "pair_kernel" in name else 2), name
