"""The training-block kernels on the CPU (no GPU): compiled as host C++ against the emulation of workgroups and wavefront
builtins that the other kernels have (tests/emu), with AddressSanitizer and UndefinedBehaviorSanitizer, and run through the C
ABI with every buffer an exact-size heap block, against plain computations in double."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SOURCES = ["dgs_edge.hip", "dgs_checkpoint.hip", "dgs_weight_grad.hip"]


def test_block_kernels_on_the_cpu_under_asan_ubsan(tmp_path):
    clang = os.environ.get("DGS_HOST_CLANG", "/opt/rocm/llvm/bin/clang++")
    emu = os.path.join(HERE, "emu")
    csrc = os.path.join(ROOT, "paper_1910_10929_amd", "csrc")
    flags = ["-std=c++17", "-O1", "-g", f"-I{emu}", "-ffp-contract=off", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
             "-Wno-unknown-attributes", "-Wno-unused-function", "-Wno-array-compare"]
    jobs = [(["-x", "c++"], os.path.join(csrc, s)) for s in SOURCES]
    jobs += [([], os.path.join(emu, s)) for s in ("emu_core.cpp", "blocks_driver.cpp")]
    objects = [str(tmp_path / (os.path.basename(src) + ".o")) for _, src in jobs]
    procs = [subprocess.Popen([clang] + lang + flags + ["-c", src, "-o", o]) for (lang, src), o in zip(jobs, objects)]
    assert [p.wait() for p in procs] == [0] * len(jobs), "compiling the emulated kernels failed"
    exe = str(tmp_path / "blocks_run")
    subprocess.run([clang, "-fsanitize=address,undefined"] + objects + ["-o", exe, "-lm"], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:detect_stack_use_after_return=0")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-6000:]
    assert "values as expected" in r.stdout
