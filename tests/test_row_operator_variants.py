"""The GPU tests of layer norm, distillation and sampling reach every kernel that the library has for them (no GPU: which kernel a call launches is a matter
of its shape), and no launch is larger than the runtime takes."""
import subprocess

import test_gpu_distill as distill
import test_gpu_layernorm as layer
import test_gpu_sample as sample
from test_launches import run  # noqa: F401  (a fixture)
from test_operator_variants import constant

CALLS = r"""
seen = set()
def launch(name, *args):
    code, launches = call(name, *args)
    assert code == 0 and all(stream == 5 for _, _, _, stream in launches), (name, code, args)
    seen.update(runtime.launched_name(i).decode() for i in range(len(launches)))
    return launches

for name, args in CASES:
    if name == "layer":
        s = solo.solo_layernorm_shape(args[0], args[1], args[1], args[1], args[1], *args[2], 0, 0, 1e-5, 0)
        launch("solo_layernorm", 16, 16, 16, 16, 16, s)
        launch("solo_layernorm_grad", 16, 16, 16, 16, 16, 16, 16, 16, 1 << 50, s)
    elif name == "distill":
        s = solo.solo_distill_shape(args[0], args[1], args[1], args[1], 3, 3, 3, args[2], 0, 64, 0, 0, 1.0, 1.0)
        launch("solo_distill", 16, 16, 16, 16, 16, s)
        launch("solo_distill_grad", 16, 16, 16, 16, 16, 16, s)
        launch("solo_distill_with_grad", 16, 16, 16, 16, 16, 16, s)
    else:
        launch("solo_sample", 16, 16, None, None, None, None, 16, 16, solo.solo_sample_shape(args[0], args[1], args[1], args[2], 64, 0, 0, 1.0, 1.0, 0.0, 0))
known, i = set(), 0
while runtime.kernel(i):
    known.add(runtime.kernel(i).decode())
    i += 1
results = [sorted(seen), sorted(k for k in known if any(part in k for part in ("layer_", "distill_", "sample_")))]
"""


def cases():
    """The shapes of the GPU tests, from their own lists."""
    found = []
    for a, b in layer.PAIRS:
        found += [("layer", (rows, cols, (layer.TYPES.index(a), layer.TYPES.index(b)))) for rows, cols, _ in layer.SHAPES]
    for dtype in 0, 1:
        found += [("distill", (rows, cols, dtype)) for rows, cols, *_ in distill.SHAPES + distill.MANY]
        found += [("sample", (rows, cols, dtype)) for rows, cols, _ in sample.SHAPES]
    return found


def test_every_kernel_is_run_by_a_gpu_test(run):  # noqa: F811
    seen, known = run("CASES = %r\n%s" % (cases(), CALLS))
    names = subprocess.run(["c++filt"], input="\n".join(sorted(set(known) - set(seen))), capture_output=True, text=True).stdout
    assert len(known) > 80 and set(known) == set(seen), names


def test_the_lines_that_go_by_bytes():
    loads, stores = constant("solo_distill.hip", "kDistillPastLoads"), constant("solo_distill.hip", "kDistillPastStores")
    sizes = [rows * cols * size for rows, cols, *_ in distill.SHAPES + distill.MANY for size in (2, 4)]
    assert any(s <= stores for s in sizes) and any(stores < s <= loads for s in sizes) and any(s > loads for s in sizes)


LARGEST = r"""
big = 1 << 34
cases = [("solo_layernorm", 16, 16, 16, 16, 16, solo.solo_layernorm_shape((1 << 31) - 1, c, c, c, c, 0, 0, 0, 0, 1e-5, 0)) for c in (1, 100, 300, 700, 2000, 4000, 8000, 16000, 16385, (1 << 24) - 1)]
cases += [("solo_layernorm_grad", 16, 16, 16, 16, 16, 16, 16, 16, 1 << 60, c[-1]) for c in list(cases)]
for c in (1, 5000, 40000, 70000, (1 << 29) - 1):
    s = solo.solo_distill_shape(big, c, c, c, 128, 128, 128, 0, 0, 64, 0, 0, 1.0, 1.0)
    cases += [("solo_distill", 16, 16, 16, 16, 16, s), ("solo_distill_grad", 16, 16, 16, 16, 16, 16, s), ("solo_distill_with_grad", 16, 16, 16, 16, 16, 16, s)]
    cases += [("solo_sample", 16, 16, 16, 16, 16, 16, 16, 16, solo.solo_sample_shape(big, c, c, 0, 64, 0, 0, 1.0, 1.0, 0.0, 0))]
for name, *args in cases:
    code, launches = call(name, *args)
    results.append([name, code, len(launches)])
"""


def test_the_largest_shapes_launch(run):  # noqa: F811
    """As many workgroups and threads as a launch can have, and no more."""
    for name, code, launches in run(LARGEST):
        assert code == 0 and launches >= 1, (name, code, launches)


REFUSED = r"""
s = solo.solo_layernorm_shape(100, 700, 700, 700, 700, 0, 0, 0, 0, 1e-5, 0)
long = solo.solo_layernorm_shape(100, 20000, 20000, 20000, 20000, 0, 0, 0, 0, 1e-5, 0)
d = solo.solo_distill_shape(10, 700, 700, 700, 3, 3, 3, 0, 0, 64, 0, 0, 1.0, 1.0)
calls = [("solo_layernorm", 16, 16, 16, 16, 16, s), ("solo_layernorm_grad", 16, 16, 16, 16, 16, 16, 16, 16, 1 << 50, s),
         ("solo_layernorm_grad", 16, 16, 16, 16, 16, 16, 16, 16, 1 << 50, long), ("solo_distill", 16, 16, 16, 16, 16, d), ("solo_distill_grad", 16, 16, 16, 16, 16, 16, d),
         ("solo_distill_with_grad", 16, 16, 16, 16, 16, 16, d), ("solo_sample", 16, 16, None, None, None, None, 16, 16, solo.solo_sample_shape(10, 700, 700, 0, 64, 0, 0, 1.0, 1.0, 0.0, 0))]
for name, *args in calls:
    whole = len(call(name, *args)[1])
    for k in range(whole):
        code, launches = call(name, *args, refuse=k)
        results.append([name, code, len(launches), k, runtime.hipPeekAtLastError()])
    code, launches = call(name, *args, left=1)             # (an error of another call)
    results.append([name, code, len(launches), whole, runtime.hipGetLastError()])
"""


def test_a_launch_that_the_runtime_refuses(run):  # noqa: F811
    """The call says so, launches nothing more and leaves no error behind; an error of another call is not taken for its own."""
    for name, code, launches, k, error in run(REFUSED):
        if error == 1:
            assert code == 0 and launches == k, (name, code, launches)
        else:
            assert code == -3 and launches == k + 1 and error == 0, (name, code, launches, k, error)
