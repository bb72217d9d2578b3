"""A warning of the compiler ends the build, which prints nothing of what passes."""
import os
import subprocess

from paper_1904_12380_amd import build

FLAGS = [f for f in build.HIPCC_FLAGS if f != "-shared"]


def compile_only(path):
    return subprocess.run([build.hipcc(), *FLAGS, "-I", os.path.join(build.ROOT, "include"),
                           "-fsyntax-only", path], capture_output=True, text=True)


def test_a_warning_is_an_error(tmp_path):
    source = tmp_path / "source.hip"
    source.write_text("int f(int x) { const int y = x; return y; }\n")
    assert compile_only(str(source)).returncode == 0
    source.write_text("int f(int x) { const const int y = x; return y; }\n")
    done = compile_only(str(source))
    assert done.returncode != 0 and "duplicate 'const'" in done.stderr
