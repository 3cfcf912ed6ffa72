"""What the operators around the step (and the state's initialisation) ask the HIP runtime for, and what they make of its answers: the library on a runtime whose launches are
only written down (no GPU; the calls are made in a process of their own, with addresses that nothing reads)."""
import json
import os
import shutil
import subprocess
import sys

import pytest

from paper_2505_00347_amd import solo

HERE = os.path.dirname(os.path.abspath(__file__))
RUNTIME = r"""
#include <hip/hip_runtime_api.h>
#include <cstring>

// The kernels of libsolo, as it registers them when it is loaded.
static const void *handles[8192];
static char names[8192][256];
static int known;

static unsigned long long launches[64][4];      // workgroups, threads of one, bytes of LDS, stream
static const char *launched_names[64];
static int count, refused = -1;
static hipError_t error;

extern "C" {
void __hipRegisterFunction(void **, const void *handle, char *name, const char *, unsigned, void *, void *, dim3 *, dim3 *, int *)
{
    if (known == 8192 || !strstr(name, "4solo")) return;
    handles[known] = handle;
    strncpy(names[known++], name, 255);
}
const char *kernel(int i) { return i < known ? names[i] : nullptr; }

hipError_t hipLaunchKernel(const void *handle, dim3 grid, dim3 block, void **, size_t lds, hipStream_t stream)
{
    const unsigned long long groups = 1ull * grid.x * grid.y * grid.z, threads = 1ull * block.x * block.y * block.z;
    const bool fits = count != refused && 1ull * grid.x * block.x <= 0xFFFFFFFFu && grid.y * block.y < 65536 && threads <= 1024 && groups != 0 && lds <= 65536;
    if (count < 64) {
        const unsigned long long row[4] = {groups, threads, lds, (unsigned long long)stream};
        for (int k = 0; k < 4; ++k) launches[count][k] = row[k];
        for (int k = 0; k < known; ++k)
            if (handles[k] == handle) launched_names[count] = names[k];
    }
    ++count;
    if (!fits) error = hipErrorInvalidConfiguration;
    return fits ? hipSuccess : hipErrorInvalidConfiguration;
}
// (a launch by <<< >>> sets these first)
static dim3 grid_, block_;
static size_t lds_;
static hipStream_t stream_;
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream)
{
    grid_ = grid; block_ = block; lds_ = lds; stream_ = stream;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream)
{
    *grid = grid_; *block = block_; *lds = lds_; *stream = stream_;
    return hipSuccess;
}
hipError_t hipGetLastError(void) { const hipError_t e = error; error = hipSuccess; return e; }
hipError_t hipPeekAtLastError(void) { return error; }

// Forgets the launches; the `refuse`-th from here on fails; `left`: an error of a call before that nobody has asked for.
void expect(int refuse, int left) { count = 0; refused = refuse; error = (hipError_t)left; }
int launched(void) { return count; }
unsigned long long launch(int i, int what) { return launches[i][what]; }
const char *launched_name(int i) { return launched_names[i]; }
}
"""
PROLOGUE = r"""
import ctypes as C, json, sys
runtime = C.CDLL(sys.argv[1], C.RTLD_GLOBAL)               # (in front of the real one)
runtime.launch.restype = C.c_ulonglong
runtime.kernel.restype = runtime.launched_name.restype = C.c_char_p
from paper_2505_00347_amd import solo
solo.lib()

def call(name, *args, refuse=-1, left=0):
    "The return code and the launches: [workgroups, threads, LDS, stream] each."
    runtime.expect(refuse, left)
    code = getattr(solo, name)(*args, stream=5, check=False)
    return code, [[runtime.launch(i, k) for k in range(4)] for i in range(runtime.launched())]

results = []
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    if shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("needs g++ and HIP's headers")
    folder = tmp_path_factory.mktemp("runtime")
    (folder / "runtime.cpp").write_text(RUNTIME)
    subprocess.check_call(["g++", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-Wno-deprecated-declarations",
                           str(folder / "runtime.cpp"), "-o", str(folder / "runtime.so")])

    def run(script):
        out = subprocess.run([sys.executable, "-c", PROLOGUE + script + "\nprint('RESULTS ' + json.dumps(results))", str(folder / "runtime.so")],
                             cwd=os.path.dirname(HERE), capture_output=True, text=True, timeout=300)
        assert out.returncode == 0, out.stderr[-2000:]
        return json.loads(out.stdout.split("RESULTS ")[1])
    return run


LARGEST = r"""
few, most, rows = 257, (1 << 28) - 1, (1 << 30) - 1
for types in (0, 0), (0, 1), (1, 0), (1, 1):
    for dim in 1, 3, 100, 512, 513, 1024, 1025, 4099, (1 << 24) - 1:
        for n in 0, 1, 256, few, most:
            for vocab in 1, 1 << 20, (1 << 26) + 1, rows:
                for flags in 0, 1:
                    s = solo.solo_embedding_shape(vocab, dim, n, dim, dim, *types, 64, flags, 1.0, 0)
                    results.append(["gradient", vocab, dim, n, types, flags, *call("solo_embedding_grad", 16, 16, 16, 16, 1 << 62, s)])
            s = solo.solo_embedding_shape(rows, dim, n, dim, dim, *types, 32, 0, 1.0, 0)
            results.append(["lookup", rows, dim, n, types, 0, *call("solo_embedding", 16, 16, 16, s)])
for units in 1, 4, 5, (1 << 24) - 1:
    for count in 1, (1 << 32) - 1:
        for name in "solo_grad_norm", "solo_grad_clip":
            results.append([name, units, count, *call(name, 16, count, units, None, 1.0, 16, 16, 16, 16)])
for dtype in 0, 1:
    for cols in 1, 2048, 2049, 20000, 65536, 65537, (1 << 29) - 1:
        for n in 1, 127, 128, 4096, (1 << 40) - 1:
            for top in 0, 20:
                s = solo.solo_logits(n, cols, cols, cols, dtype, 64, top, 0, 1.0, 0)
                results.append(["forward", n, cols, top, *call("solo_logprob", 16, 16, 16, 16, 16, 16, 16, 16, s)])
            results.append(["grad", n, cols, *call("solo_logprob_grad", 16, 16, 16, 16, 16, 16, 16, s)])
            results.append(["both", n, cols, *call("solo_logprob_with_grad", 16, 16, 16, 16, 16, 16, 16, s)])
"""


def test_the_largest_shapes_that_are_taken_can_be_launched(run):
    """One launch has fewer than 2^32 threads: a shape that the library takes asks for no more."""
    for *shape, code, launches in run(LARGEST):
        assert code == 0, (shape, launches)
        assert launches or shape[0] in ("gradient", "lookup") and shape[3] == 0, shape
        assert all(stream == 5 for *_, stream in launches)


EACH = r"""
embed = lambda n: solo.solo_embedding_shape(1000, 520, n, 520, 520, 1, 1, 64, 0, 1.0, 0)
x = solo.solo_logits(700, 3000, 3000, 3000, 1, 64, 5, 0, 1.0, 0)
calls = [("solo_state_init", 16, 16, 16, 16, 16, 1000, solo.make_config()), ("solo_grad_norm", 16, 2, 3, None, 1.0, 16, 16, 16, 16), ("solo_grad_norm", 16, 2, 9, None, 1.0, 16, 16, 16, 16),
         ("solo_grad_clip", 16, 2, 3, None, 1.0, 16, 16, 16, 16), ("solo_grad_clip", 16, 2, 9, None, 1.0, 16, 16, 16, 16),
         ("solo_embedding", 16, 16, 16, embed(700)), ("solo_embedding_grad", 16, 16, 16, 16, 1 << 40, embed(70)),
         ("solo_embedding_grad", 16, 16, 16, 16, 1 << 40, embed(0)), ("solo_embedding_grad", 16, 16, 16, 16, 1 << 40, embed(700)),
         ("solo_logprob", 16, 16, 16, 16, 16, 16, 16, 16, x), ("solo_logprob_grad", 16, 16, 16, 16, 16, 16, 16, x),
         ("solo_logprob_with_grad", 16, 16, 16, 16, 16, 16, 16, x)]
"""


def test_an_error_of_another_call_is_not_one_of_these(run):
    """HIP keeps the last error until someone asks: the launches have succeeded all the same."""
    for name, code, launches, left in run(EACH + "for c in calls: results.append([c[0], *call(*c, left=1), runtime.hipGetLastError()])"):
        assert code == 0 and launches, name
        assert left == 1, name                             # (whose it is finds it)


def test_a_launch_that_fails_is_reported_and_nothing_follows_it(run):
    results = run(EACH + "for c in calls:\n for k in range(len(call(*c)[1])): results.append([c[0], k, *call(*c, refuse=k), runtime.hipGetLastError()])")
    assert len(results) > 11
    for name, k, code, launches, left in results:
        assert code == solo.SOLO_E_HIP and len(launches) == k + 1, (name, k)
        assert left == 0, name                             # (reported here, not by the caller's next call)
