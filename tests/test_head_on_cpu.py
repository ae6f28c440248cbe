"""The output layer's and the orthogonalising kernels on the CPU (no GPU): compiled as host C++ against the emulation of workgroups
and wavefront builtins that the other kernels have (tests/emu), with AddressSanitizer and UndefinedBehaviorSanitizer, and run through
the C ABI with every buffer an exact-size heap block, against plain computations in double."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_1910_10929_amd", "csrc")
EMU = os.path.join(HERE, "emu")
CLANG = os.environ.get("DGS_HOST_CLANG", "/opt/rocm/llvm/bin/clang++")
FLAGS = ["-std=c++17", "-O1", "-g", f"-I{EMU}", "-ffp-contract=off", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
         "-Wno-unknown-attributes", "-Wno-unused-function", "-Wno-array-compare", "-Wno-pass-failed"]
# the library as it is, and with one kind of tile (256 x 256, 256 x 128, 192 x 192, 128 x 128, 64 x 64: small
# products take that by themselves, small updates a launch for all their steps), small pieces of the vocabulary and split sums taken at any size: of which kernels, and what is run
BUILDS = {
    "": ([], ("dgs_head", "dgs_orthogonal"), ("head", "large", "ortho")),
    "0": (["-DDGS_PRODUCT_SPLITS=1"], ("dgs_head", "dgs_orthogonal"), ("large", "tiles")),
    "1": (["-DDGS_PRODUCT_SPLITS=2"], ("dgs_head",), ("large",)),
    "2": (["-DDGS_PRODUCT_SPLITS=3"], ("dgs_orthogonal",), ("tiles",)),
    "3": (["-DDGS_PRODUCT_SPLITS=3"], ("dgs_head", "dgs_orthogonal"), ("large", "tiles")),
    "4": (["-DDGS_PRODUCT_SPLITS=1"], ("dgs_orthogonal",), ("ortho",)),
}


@pytest.fixture(scope="module")
def programs(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("head"))
    jobs = {"emu_core": ([], os.path.join(EMU, "emu_core.cpp")), "driver": ([], os.path.join(EMU, "head_driver.cpp"))}
    for build, (flags, names, _) in BUILDS.items():
        tile = [f"-DDGS_PRODUCT_TILE={build}", "-DDGS_HEAD_PIECE=256"] if build else []
        for name in names:
            jobs[name + build] = (["-x", "c++"] + tile + flags, os.path.join(CSRC, name + ".hip"))
    procs = {n: subprocess.Popen([CLANG] + lang + FLAGS + ["-c", src, "-o", os.path.join(out, n + ".o")]) for n, (lang, src) in jobs.items()}
    assert all([p.wait() == 0 for p in procs.values()]), "compiling the emulated kernels failed"
    built = {}
    for build, (_, names, _) in BUILDS.items():
        built[build] = os.path.join(out, "run_" + build)
        # (the other kernels as they are)
        objects = [os.path.join(out, n + ".o") for n in [name + (build if name in names else "") for name in ("dgs_head", "dgs_orthogonal")] + ["emu_core", "driver"]]
        subprocess.run([CLANG, "-fsanitize=address,undefined"] + objects + ["-o", built[build], "-lm"], check=True)
    return built


def test_head_kernels_on_the_cpu_under_asan_ubsan(programs):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:detect_stack_use_after_return=0")
    runs = [(build, what) for build, (_, _, whats) in BUILDS.items() for what in whats]
    procs = [(run, subprocess.Popen([programs[run[0]], run[1]], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env)) for run in runs]
    try:
        for run, p in procs:
            text, _ = p.communicate(timeout=600)
            assert p.returncode == 0 and "values as expected" in text, f"{run}: {text[-5000:]}"
    finally:
        for _, p in procs:
            p.kill()
