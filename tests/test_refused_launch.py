"""A kernel launch that the runtime refuses: the launches behind it, which would work on what it has not written, are not made (no GPU:
the runtime's launch calls are fakes)."""
import os
import subprocess

from paper_2605_20022_b200 import _build

FAKES = ["cudaLaunchKernelExC", "cudaLaunchKernel", "__cudaPushCallConfiguration", "__cudaPopCallConfiguration", "cudaGetDriverEntryPoint",
         "cudaFuncSetAttribute", "cudaFuncGetAttributes"]


def test_nothing_follows_a_refused_launch(tmp_path):
    csrc, exe = os.path.join(_build.HERE, "csrc"), str(tmp_path / "refused_launch")
    wrap = [x for f in FAKES for x in ("-Xlinker", f"--wrap={f}")]
    # (no kernel runs: intermediate code is enough, and quicker)
    subprocess.run([os.environ.get("NVCC", "nvcc"), "-std=c++17", "-gencode", "arch=compute_100a,code=compute_100a", "-I", csrc,
                    "-I", os.path.join(_build.ROOT, "include"), "-o", exe, os.path.join(os.path.dirname(__file__), "refused_launch.cu"),
                    *(os.path.join(csrc, x) for x in ("fd_pages.cu", "fd_prompt_tc.cu", "fd_prompt_simt.cu")), *wrap], check=True)
    out = subprocess.run([exe], check=True, capture_output=True, text=True).stdout
    got = {line.split(":")[0]: tuple(map(int, line.split(":")[1].split())) for line in out.splitlines()}
    # refused launch (0: none) -> launches attempted, and what the call says: kernels launched (prompt: -1 - n with an error)
    want = {f"{name} {n}": (n or kernels, n - 1 if n else kernels) for name, kernels in (("compact", 2), ("compact in a cluster", 2), ("free", 4))
            for n in range(kernels + 1)}
    want.update({"prompt 0": (2, 2), "prompt 1": (1, -1), "prompt 2": (2, -2)})
    assert got == want
