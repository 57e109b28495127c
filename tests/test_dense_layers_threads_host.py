"""The calls of the dense layers may be made by several threads at once: their messages (CPU; nothing is launched)."""
import os
import shutil
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_thread_gets_the_messages_of_its_own_failing_calls(tmp_path):
    import paper_1901_05350_b200.build as build

    library = build.build()
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    csrc = os.path.join(ROOT, "paper_1901_05350_b200", "csrc")
    exe = str(tmp_path / "failing_threads")
    subprocess.run([nvcc, "-x", "cu", "-O1", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(ROOT, "tests", "failing_threads.cpp"), "-o", exe, "-L", os.path.dirname(library), "-l:" + os.path.basename(library),
                    "-Xlinker", f"-rpath={os.path.dirname(library)}", "-lpthread"], check=True)
    done = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.strip() == "ok", (done.returncode, done.stdout, done.stderr)
