"""The C ABI of the sequence operators on the CPU: the host layer under AddressSanitizer and
UndefinedBehaviorSanitizer with counting stubs for the launchers (every refusal launches nothing), and the
descriptor's layout in the Python binding."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2501_14490_amd", "csrc")
SAN = ["-g", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer"]


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"),
                    reason="needs g++ and the HIP headers")
def test_host_layer_under_sanitizers(tmp_path):
    exe = str(tmp_path / "seq_driver")
    cmd = ["g++", "-std=c++20", *SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}", os.path.join(CSRC, "mfpsn_api_seq.cpp"),
           os.path.join(ROOT, "tests", "sanitize", "seq_driver.cpp"), "-o", exe]
    p = subprocess.run(cmd, capture_output=True, text=True)
    assert p.returncode == 0, p.stderr[-4000:]
    p = subprocess.run([exe], capture_output=True, text=True)
    assert p.returncode == 0 and "seq driver: OK" in p.stdout, p.stdout + p.stderr


def test_descriptor_layout_matches_header():
    pytest.importorskip("torch")
    if not os.path.exists(os.path.join(ROOT, "paper_2501_14490_amd", "libmfpsn.so")):
        pytest.skip("libmfpsn.so not built")
    from paper_2501_14490_amd import mfpsn

    text = open(os.path.join(ROOT, "include", "mfpsn.h")).read()
    body = text[text.index("typedef struct mfpsn_delta_desc"):text.index("} mfpsn_delta_desc;")]
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = [n.strip() for group in re.findall(r"\b(?:int32_t|int64_t|float)\s+([A-Za-z_, 0-9]+);", body)
             for n in group.split(",")]
    assert names == [f[0] for f in mfpsn.MfpsnDeltaDesc._fields_]
    assert ctypes.sizeof(mfpsn.MfpsnDeltaDesc) == 8 * 4 + 3 * 8


def test_wrappers_refuse_before_any_gpu_call():
    torch = pytest.importorskip("torch")
    if not os.path.exists(os.path.join(ROOT, "paper_2501_14490_amd", "libmfpsn.so")):
        pytest.skip("libmfpsn.so not built")
    from paper_2501_14490_amd import mfpsn

    x = torch.zeros(2, 3, 4)
    with pytest.raises(ValueError):  # not on a GPU
        mfpsn.layer_norm_forward(x)
    with pytest.raises(TypeError):
        mfpsn.layer_norm_forward(x.half())
    with pytest.raises(ValueError):
        mfpsn.layer_norm_forward(x, torch.ones(5))
    desc = mfpsn.make_delta_desc((5, 1, 1, 4), (5, 1, 2, 6))
    q, v, g = torch.zeros(5, 1, 1, 4), torch.zeros(5, 1, 2, 6), torch.zeros(5, 1, 2)
    with pytest.raises(ValueError):  # not on a GPU
        mfpsn.delta_forward(desc, q, q, v, g, g)
    with pytest.raises(ValueError):
        mfpsn.delta_forward(desc, q, q[:4], v, g, g)
    with pytest.raises(ValueError):  # a row's heads are not dense
        mfpsn.delta_forward(desc, q, q, torch.zeros(5, 1, 6, 2).transpose(2, 3), g, g)
    with pytest.raises(TypeError):
        mfpsn.delta_forward(desc, q, q, v, g, g.bfloat16())
    # rows of a slice: the distance of the projection's rows, whatever N is
    both = torch.zeros(5, 3, 20)
    part = both[:, :, 4:12].unflatten(2, (2, 4))
    assert mfpsn._delta_row(part, torch.float32, part.device, (5, 3, 2, 4), "q") == 20
    one = torch.zeros(5, 1, 20)[:, :, 4:12].unflatten(2, (2, 4))
    assert mfpsn._delta_row(one, torch.float32, one.device, (5, 1, 2, 4), "q") == 20
    with pytest.raises(ValueError):  # every second row of N: not at equal distances over (t, n)
        mfpsn._delta_row(torch.zeros(5, 6, 8)[:, ::2].unflatten(2, (2, 4))[:, :2], torch.float32, part.device,
                         (5, 2, 2, 4), "q")
