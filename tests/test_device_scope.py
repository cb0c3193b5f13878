"""The current device inside the library's entry points, without a GPU: the scope object over a stand-in of the two runtime
calls, and that every entry point which touches the device opens one."""
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_23725_b200", "csrc")

PROGRAM = r"""
#include <stdio.h>
#include "device_scope.h"
static int current = 0, sets = 0, broken = 0;
extern "C" cudaError_t cudaGetDevice(int* d) { if (broken == 1) return cudaErrorInitializationError; *d = current; return cudaSuccess; }
extern "C" cudaError_t cudaSetDevice(int d) { if (broken == 2) return cudaErrorInvalidDevice; current = d; ++sets; return cudaSuccess; }
#define WANT(x) if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; }
int main() {
  { muloco::DeviceScope s(0); WANT(s.error() == cudaSuccess && current == 0); }
  WANT(current == 0 && sets == 0);                       // nothing to do, nothing done
  { muloco::DeviceScope s(1); WANT(s.error() == cudaSuccess && current == 1);
    { muloco::DeviceScope t(1); WANT(current == 1); }    // a call inside a call
    WANT(current == 1);
    { muloco::DeviceScope t(2); WANT(current == 2); }
    WANT(current == 1); }
  WANT(current == 0 && sets == 4);
  broken = 1; { muloco::DeviceScope s(1); WANT(s.error() == cudaErrorInitializationError); }
  broken = 2; { muloco::DeviceScope s(1); WANT(s.error() == cudaErrorInvalidDevice && current == 0); }
  broken = 0; WANT(current == 0 && sets == 4);
  return 0;
}
"""


def test_scope_sets_and_restores(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    cuda = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, "-isystem", cuda, str(src), "-o", str(exe)])
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout


# calls that only read or write the context's host memory
HOST_ONLY = {"muloco_fragments_due", "muloco_get_state", "muloco_set_state", "muloco_set_timing", "muloco_last_error",
             "muloco_debug_set", "muloco_check_workspace", "muloco_shard_layout", "muloco_debug_ffn_forms"}
# these have no context: the device that is current is the caller's choice (and becomes that of the context made)
NO_CONTEXT = {"muloco_create", "muloco_newton_schulz_static"}


def test_every_entry_point_opens_a_scope():
    from paper_2505_23725_b200 import binding
    seen = set()
    for name in os.listdir(CSRC):
        if not name.endswith(".cu"):
            continue
        text = open(os.path.join(CSRC, name)).read()
        for part in re.split(r'(?m)^(?:extern "C" )?MULOCO_API ', text)[1:]:
            fn = re.search(r"\b(muloco_\w+)\s*\(", part).group(1)
            body = part.split("\n}\n")[0]
            seen.add(fn)
            assert bool(re.search(r"^  (ON_DEVICE\(c\);|const DeviceScope )", body, re.M)) == (fn not in HOST_ONLY | NO_CONTEXT), fn
    assert seen >= set(binding.EXPORTS)
