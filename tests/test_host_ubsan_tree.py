"""The host side of the drafted-token calls -- checks, ranges, limits, workspace sizes -- under the undefined-behaviour sanitizer, as
test_host_ubsan.py has it for the other calls (no GPU needed)."""
import importlib.util
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_host_tests_of_the_drafted_token_calls_pass_against_sanitized_host_code(tmp_path):
    spec = importlib.util.spec_from_file_location("lvlm_build", os.path.join(ROOT, "paper_2509_00419_amd", "build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    lib, binding = build.build_host_sanitized(str(tmp_path))
    env = dict(os.environ, LVLM_LIBRARY=lib, LVLM_TORCH_BINDING=binding)
    files = [os.path.join(ROOT, "tests", f) for f in ("test_tree_abi.py", "test_tree_ranges.py", "test_oracle_tree.py")]
    run = subprocess.run([sys.executable, "-m", "pytest", *files, "-x", "-q", "-p", "no:cacheprovider"], cwd=ROOT,
                         env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert run.returncode == 0, run.stdout[-3000:]
    assert " passed" in run.stdout
