"""The training-block kernels on the CPU (no GPU): compiled as host C++ against the emulation of workgroups and wavefront
builtins that the other kernels have (tests/emu), with AddressSanitizer and UndefinedBehaviorSanitizer, and run through the C
ABI with every buffer an exact-size heap block, against plain computations in double."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_1910_10929_amd", "csrc")
EMU = os.path.join(HERE, "emu")
CLANG = os.environ.get("DGS_HOST_CLANG", "/opt/rocm/llvm/bin/clang++")
FLAGS = ["-std=c++17", "-O1", "-g", f"-I{EMU}", "-ffp-contract=off", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
         "-Wno-unknown-attributes", "-Wno-unused-function", "-Wno-array-compare"]


@pytest.fixture(scope="module")
def programs(tmp_path_factory):
    """The driver with the library as it is, and with one kind of the weight gradient's large tiles taken at any size."""
    out = str(tmp_path_factory.mktemp("blocks"))
    jobs = {name: (["-x", "c++"], os.path.join(CSRC, name + ".hip")) for name in ("dgs_edge", "dgs_checkpoint", "dgs_weight_grad")}
    for tile in (0, 1):
        jobs[f"tile{tile}"] = (["-x", "c++", f"-DDGS_GRAD_TILE={tile}"], os.path.join(CSRC, "dgs_weight_grad.hip"))
    jobs["emu_core"] = ([], os.path.join(EMU, "emu_core.cpp"))
    jobs["driver"] = ([], os.path.join(EMU, "blocks_driver.cpp"))
    procs = {n: subprocess.Popen([CLANG] + lang + FLAGS + ["-c", src, "-o", os.path.join(out, n + ".o")]) for n, (lang, src) in jobs.items()}
    assert all([p.wait() == 0 for p in procs.values()]), "compiling the emulated kernels failed"
    built = {}
    for grad in ("dgs_weight_grad", "tile0", "tile1"):
        built[grad] = os.path.join(out, "run_" + grad)
        objects = [os.path.join(out, n + ".o") for n in ("dgs_edge", "dgs_checkpoint", grad, "emu_core", "driver")]
        subprocess.run([CLANG, "-fsanitize=address,undefined"] + objects + ["-o", built[grad], "-lm"], check=True)
    return built


def test_block_kernels_on_the_cpu_under_asan_ubsan(programs):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:detect_stack_use_after_return=0")
    runs = [("dgs_weight_grad", "edges"), ("dgs_weight_grad", "weights"), ("tile0", "tiles"), ("tile1", "tiles")]
    procs = [(run, subprocess.Popen([programs[run[0]], run[1]], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env)) for run in runs]
    try:
        for run, p in procs:
            text, _ = p.communicate(timeout=600)
            assert p.returncode == 0 and "values as expected" in text, f"{run}: {text[-5000:]}"
    finally:
        for _, p in procs:
            p.kill()
