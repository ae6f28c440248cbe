"""The edges' kernels for rows of twelve and sixteen wavefronts on the CPU (no GPU), in workgroups with more than one row each:
the row loop's second round, its sums' halves by turns, in exact-size heap blocks under AddressSanitizer and
UndefinedBehaviorSanitizer."""
import os
import subprocess

import pytest

from test_blocks_on_cpu import CLANG, CSRC, EMU, FLAGS


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("wide"))
    jobs = {name: (["-x", "c++"], os.path.join(CSRC, name + ".hip")) for name in ("dgs_edge", "dgs_checkpoint", "dgs_weight_grad")}
    jobs["emu_core"] = ([], os.path.join(EMU, "emu_core.cpp"))
    jobs["driver"] = ([], os.path.join(EMU, "wide_rows_driver.cpp"))
    procs = [subprocess.Popen([CLANG] + lang + FLAGS + ["-c", src, "-o", os.path.join(out, n + ".o")]) for n, (lang, src) in jobs.items()]
    assert all([p.wait() == 0 for p in procs]), "compiling the emulated kernels failed"
    built = os.path.join(out, "run")
    subprocess.run([CLANG, "-fsanitize=address,undefined"] + [os.path.join(out, n + ".o") for n in jobs] + ["-o", built, "-lm"], check=True)
    return built


def test_wide_rows_on_the_cpu_under_asan_ubsan(program):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:detect_stack_use_after_return=0")
    runs = [(what, subprocess.Popen([program, what], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env))
            for what in ("one", "many16", "many12")]
    try:
        for what, p in runs:
            text, _ = p.communicate(timeout=600)
            assert p.returncode == 0 and "values as expected" in text, f"{what}: {text[-5000:]}"
    finally:
        for _, p in runs:
            p.kill()
