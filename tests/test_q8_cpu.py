"""What the 8-bit calls refuse before they touch a device, and what they say of their scratch."""
import pytest


@pytest.fixture(scope="module")
def m():
    import paper_1404_5997_amd as mod
    return mod


def refused(m, status, fn, *args):
    with pytest.raises(m.OwtError) as e:
        fn(*args)
    assert e.value.status == status, str(e.value)


def test_pitch(m):
    assert [m.owt_q8_pitch(c) for c in (-1, 0, 1, 128, 129, 9216)] == [0, 0, 128, 128, 256, 9216]


def test_rows_refuse(m):
    ok = (2, 100, m.OWT_F32, 256, 512, 1024)
    for at, bad in ((0, -1), (1, 0), (1, -5), (2, 7), (3, None), (4, None), (5, None), (3, 260), (4, 513), (5, 1028)):
        args = list(ok)
        args[at] = bad
        refused(m, m.OWT_EINVAL, m.owt_q8_pack, *args, 0)
        refused(m, m.OWT_EINVAL, m.owt_q8_unpack, *(args[:3] + [args[4], args[5], args[3]]), 0)


def test_norm_refuses(m):
    fwd = (2, 100, m.OWT_F32, 256, 512, 1024, 1e-5, 2048, 4096, 8192, 16384)
    for at, bad in ((0, -1), (1, 0), (2, 9), (3, None), (8, None), (9, None), (3, 257), (4, 520), (6, -1.0), (6, float("nan")), (6, float("inf"))):
        args = list(fwd)
        args[at] = bad
        refused(m, m.OWT_EINVAL, m.owt_rmsnorm_q8_fwd, *args, 0)
    args = list(fwd)
    args[4] = None                      # a sum is asked for, and there is none
    refused(m, m.OWT_EINVAL, m.owt_rmsnorm_q8_fwd, *args, 0)
    args = list(fwd)
    args[1] = 32769
    refused(m, m.OWT_EUNSUPPORTED, m.owt_rmsnorm_q8_fwd, *args, 0)
    bwd = (2, 100, m.OWT_BF16, 256, 512, 1024, 2048, 4096, 1.0, 0.0, 8192, None)
    for at, bad in ((0, -1), (1, 0), (3, None), (4, None), (6, None), (10, None), (10, 8200), (8, float("inf")), (9, float("nan"))):
        args = list(bwd)
        args[at] = bad
        refused(m, m.OWT_EINVAL, m.owt_rmsnorm_q8_bwd, *args, None, 0)
    args = list(bwd)
    args[11] = 16384                    # the gain's gradient needs scratch
    refused(m, m.OWT_EWORKSPACE, m.owt_rmsnorm_q8_bwd, *args, None, 0)
    with pytest.raises(m.OwtError):
        m.owt_rmsnorm_q8_workspace_bytes(1, 40000)
    assert m.owt_rmsnorm_q8_workspace_bytes(0, 64) == 0


def test_shard_refuses(m):
    def desc(**kw):
        g = dict(N=4, I=64, O_total=32, workers=2, rank=0, dtype=m.OWT_F32, flags=0)
        g.update(kw)
        return m.fc_desc(**g)

    ptrs = [256 * k for k in range(1, 7)]
    for kw in (dict(N=-1), dict(I=0), dict(O_total=33), dict(workers=0), dict(rank=2), dict(dtype=5), dict(flags=8)):
        refused(m, m.OWT_EINVAL, m.owt_fc_shard_q8_fwd, desc(**kw), *ptrs, None, 0)
        refused(m, m.OWT_EINVAL, m.owt_fc_shard_q8_bwd, desc(**kw), *ptrs, 1.0, 0.0, 4096, 8192, 16384, None, 0)
        with pytest.raises(m.OwtError):
            m.owt_fc_shard_q8_workspace_bytes(desc(**kw), 0)
    for kw in (dict(I=131072), dict(N=(1 << 22) + 1), dict(O_total=(1 << 23) + 2)):
        refused(m, m.OWT_EUNSUPPORTED, m.owt_fc_shard_q8_fwd, desc(**kw), *ptrs, None, 0)
    for at in (0, 1, 2, 3, 5):
        args = list(ptrs)
        args[at] = None
        refused(m, m.OWT_EINVAL, m.owt_fc_shard_q8_fwd, desc(), *args, None, 0)
    args = list(ptrs)
    args[4] = None
    refused(m, m.OWT_EINVAL, m.owt_fc_shard_q8_fwd, desc(flags=m.OWT_BIAS), *args, None, 0)
    refused(m, m.OWT_EINVAL, m.owt_fc_shard_q8_bwd, desc(flags=m.OWT_RELU), *args, 1.0, 0.0, None, 8192, None, None, 0)
    refused(m, m.OWT_EINVAL, m.owt_fc_shard_q8_bwd, desc(), *args, float("nan"), 0.0, None, 8192, None, None, 0)
    refused(m, m.OWT_EINVAL, m.owt_fc_shard_q8_bwd, desc(), *args, 1.0, 0.0, None, None, None, None, 0)
    refused(m, m.OWT_EWORKSPACE, m.owt_fc_shard_q8_bwd, desc(), *args, 1.0, 0.0, None, 8192, None, None, 0)
    with pytest.raises(m.OwtError):
        m.owt_fc_shard_q8_workspace_bytes(desc(), 3)
    assert m.owt_fc_shard_q8_workspace_bytes(desc(), m.OWT_PASS_BWD_DATA) > 0


def test_int8_tensors_have_to_be_dense(m):
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        m.owt_q8_pack(4, 64, m.OWT_F32, torch.zeros((4, 128))[:, :64], 256, 512, 0)


def test_every_barrier_of_the_products_waits_for_the_reads_before_it(tmp_path):
    """As the compiler leaves them: behind a barrier in a product's walk loads overwrite a tile that fragments were read from, so each
    wavefront has to have its reads behind it (and its loads, to the count that may stay) when it comes there."""
    import importlib.util
    import os
    import re
    import subprocess
    package = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1404_5997_amd")
    spec = importlib.util.spec_from_file_location("_owt_build", os.path.join(package, "build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    out = str(tmp_path / "k.s")
    subprocess.run([build.HIPCC] + build.FLAGS + ["--cuda-device-only", "-S", "-o", out, os.path.join(build.CSRC, "owt_q8fc.hip")], check=True, capture_output=True)
    with open(out) as f:
        kernels = re.findall(r"^(_ZN3owt1\dq8gemm_(?:pair_)?kernel\w+):(.*?)^\.Lfunc_end", f.read(), re.M | re.S)
    assert len(kernels) == 9
    for name, body in kernels:
        code = [l.strip() for l in body.splitlines() if l.startswith("\t") and not l.strip().startswith((";", "."))]
        for walk in re.split(r"\n(?=ds_write)", "\n".join(code)):           # (results go through LDS behind the walk)
            walk = walk.splitlines()
            loads = [i for i, l in enumerate(walk) if l.startswith("global_load_lds")]
            barriers = [i for i, l in enumerate(walk) if l.startswith("s_barrier") and loads and loads[0] < i < loads[-1]]
            for b in barriers:
                assert re.fullmatch(r"s_waitcnt vmcnt\(\d+\) lgkmcnt\(0\)", walk[b - 1]), (name, walk[b - 3:b + 1])
            assert not loads or barriers, name
