"""Where numbers are hard for the orthogonalising kernels and the output layer's, on the CPU (no GPU): the emulated kernels under
AddressSanitizer and UndefinedBehaviorSanitizer, through the C ABI, against the definitions in double; see
tests/emu/step_end_driver.cpp."""
import os
import subprocess

import pytest

from test_head_on_cpu import CLANG, CSRC, EMU, FLAGS

RUNS = ["coefficients", "improbable", "unlike"]


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("step_end"))
    jobs = {name: (["-x", "c++"], os.path.join(CSRC, name + ".hip")) for name in ("dgs_head", "dgs_orthogonal")}
    jobs["emu_core"] = ([], os.path.join(EMU, "emu_core.cpp"))
    jobs["driver"] = ([], os.path.join(EMU, "step_end_driver.cpp"))
    procs = [subprocess.Popen([CLANG] + lang + FLAGS + ["-c", src, "-o", os.path.join(out, n + ".o")]) for n, (lang, src) in jobs.items()]
    assert all([p.wait() == 0 for p in procs]), "compiling the emulated kernels failed"
    built = os.path.join(out, "run")
    subprocess.run([CLANG, "-fsanitize=address,undefined"] + [os.path.join(out, n + ".o") for n in jobs] + ["-o", built, "-lm"], check=True)
    return built


@pytest.mark.parametrize("what", RUNS)
def test_hard_numbers_on_the_cpu_under_asan_ubsan(program, what):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:detect_stack_use_after_return=0")
    p = subprocess.run([program, what], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=600)
    assert p.returncode == 0 and "values as expected" in p.stdout, p.stdout[-5000:]
