"""How results of the 8-bit products leave, as the compiler has it (no device): a wavefront puts 32 rows of them into LDS, other lanes of it read
them, and the next 32 rows go to the same place.  Nothing but an order of the compiler's own keeps those accesses apart, so it has to be told."""
import importlib.util
import os
import re
import subprocess

# (by path: the package loads its library, and the HIP runtime with it, which has to come behind torch's for the GPU tests of the same process)
PACKAGE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1404_5997_amd")
spec = importlib.util.spec_from_file_location("_owt_build", os.path.join(PACKAGE, "build.py"))
build = importlib.util.module_from_spec(spec)
spec.loader.exec_module(build)


def test_lanes_that_read_what_others_wrote_are_told_apart_from_them(tmp_path):
    out = str(tmp_path / "k.s")
    subprocess.run([build.HIPCC] + build.FLAGS + ["--cuda-device-only", "-S", "-o", out, os.path.join(build.CSRC, "owt_q8fc.hip")], check=True, capture_output=True)
    with open(out) as f:
        kernels = re.findall(r"^(_ZN3owt1\dq8gemm_(?:pair_)?kernel\w+):(.*?)^\.Lfunc_end", f.read(), re.M | re.S)
    assert kernels
    for name, body in kernels:
        lines = [l.strip() for l in body.splitlines()]
        blocks = 0
        for walk in re.split(r"(?=global_load_lds)", "\n".join(lines)):     # (what follows a walk's last load, up to the next product's first)
            # writes of results, reads of results, and what keeps them apart
            seen = re.findall(r"^(ds_write_b128|ds_read_b128|; wave barrier|s_barrier)", walk, re.M)
            if "ds_write_b128" not in seen:
                continue
            blocks += 1
            last = None
            for s in seen[seen.index("ds_write_b128"):]:
                if s in ("ds_write_b128", "ds_read_b128"):
                    assert last in (None, s), (name, "%s straight behind %s" % (s, last))
                    last = s
                else:
                    last = None
        assert blocks, name
