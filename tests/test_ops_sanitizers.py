"""The host side of the operators beside the layer (ops_api.hip: validation, workspace sizes) under
AddressSanitizer and UndefinedBehaviorSanitizer, on the CPU: its host-only tests run in a child
process in which any finding aborts."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)


def test_operator_host_code_under_asan_ubsan(tmp_path):
    from paper_2608_14385_amd import build
    lib = build.build_host_sanitized(str(tmp_path))
    names = subprocess.run(["nm", str(tmp_path / "ops_api_san.o")], capture_output=True, text=True, check=True).stdout
    assert "__asan_report" in names and "__ubsan_handle" in names
    env = dict(os.environ, LD_PRELOAD=build.asan_runtime(),
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    code = ("import sys, pytest; import paper_2608_14385_amd.deamoe as D; "
            "D.LIB_PATH = sys.argv[1]; "
            "rc = pytest.main(['-q', '-x', '-p', 'no:cacheprovider', 'tests/test_ops_abi.py']); "
            "assert D.lib()._name == sys.argv[1]; sys.exit(rc)")
    r = subprocess.run([sys.executable, "-c", code, lib], cwd=ROOT, env=env, capture_output=True,
                       text=True, timeout=900)
    assert r.returncode == 0, (r.stdout[-3000:], r.stderr[-3000:])
    assert " passed" in r.stdout, r.stdout
