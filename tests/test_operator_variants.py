"""The GPU tests of the operators around the step reach every kernel that the library has for them (no GPU: which kernel a call launches
is a matter of its shape)."""
import os
import re
import subprocess

import pytest

import test_gpu_operators as small
import test_gpu_operators_large as large
from paper_2505_00347_amd import build as libbuild
from test_launches import run  # noqa: F401  (a fixture)

CSRC = libbuild.CSRC


def constant(source, name):
    text = open(os.path.join(CSRC, source)).read()
    value = re.search(r"\b%s = (\d+)(?:ull)?(?: << (\d+))?" % name, text)
    return int(value[1]) << int(value[2] or 0)


def test_the_lines_that_go_by_bytes():
    assert constant("solo_embed.hip", "kPastBytes") == large.PAST_BYTES
    assert constant("solo_logprob.hip", "kPastLoads") == large.PAST_LOADS and constant("solo_logprob.hip", "kPastStores") == large.PAST_STORES
    assert constant("solo_norm.hip", "kLargeBytes") == large.LARGE_BYTES
    for dtype in large.TYPES:
        for dim in large.DIMS:
            below, above = [large.rows_around(past, dim, dtype) * dim * dtype.itemsize for past in (False, True)]
            assert below <= large.PAST_BYTES < above
        for size in (large.PAST_STORES, large.PAST_LOADS):
            for rows, cols in large.logits_cases(dtype)[:-2]:
                assert abs(rows * cols * dtype.itemsize - size) > 0        # (none on a line itself)
            assert sum(0 < rows * cols * dtype.itemsize - size <= cols * dtype.itemsize for rows, cols in large.logits_cases(dtype)) >= len(large.COLUMNS)


CALLS = r"""
def embedding(types, vocab, dim, n, bits, flags=0):
    return solo.solo_embedding_shape(vocab, dim, n, dim, dim, *types, bits, flags, 1.0, 0)

def logits(dtype, rows, cols, top):
    return solo.solo_logits(rows, cols, cols, cols, dtype, 64, top, 0, 1.0, 0)

seen = set()
def launch(name, *args):
    code, launches = call(name, *args)
    assert code == 0, (name, code)
    seen.update(runtime.launched_name(i).decode() for i in range(len(launches)))

for name, args in CASES:
    if name == "norm":
        for entry in "solo_grad_norm", "solo_grad_clip":
            launch(entry, 16, 3, args, None, 1.0, 16, 16, 16, 16)
    elif name == "lookup":
        launch("solo_embedding", 16, 16, 16, embedding(*args))
    elif name == "gradient":
        launch("solo_embedding_grad", 16, 16, 16, 16, 1 << 50, embedding(*args))
    else:
        dtype, rows, cols, tops, ranks, entropies = args
        for top in tops:
            for rank in ranks:
                launch("solo_logprob", 16, 16, 16, 16, 16 if rank else None, 16, 16, 16, logits(dtype, rows, cols, top))
        for entropy in entropies:
            launch("solo_logprob_grad", 16, 16, 16, 16, 16, 16 if entropy else None, 16, logits(dtype, rows, cols, 0))
            launch("solo_logprob_with_grad", 16, 16, 16, 16 if entropy else None, 16, 16, 16, logits(dtype, rows, cols, 0))
known, i = set(), 0
while runtime.kernel(i):
    known.add(runtime.kernel(i).decode())
    i += 1
results = [sorted(seen), sorted(k for k in known if any(part in k for part in ("norm_", "clip_", "embed_", "logprob_")))]
"""


def cases():
    """The shapes of the GPU tests, from their own lists."""
    found = [("norm", units) for units in (1, 9)]
    pairs = [(small.TYPES.index(a), small.TYPES.index(b)) for a in small.TYPES for b in small.TYPES]
    for types in pairs:                                    # (the table's type, the rows')
        rows_type = small.TYPES[types[1]]
        for bits in 32, 64:
            found += [("lookup", (types, 1000, 2056, 257, bits))]
            found += [("lookup", (types, 3001, dim, large.rows_around(past, dim, rows_type), bits)) for dim in large.DIMS for past in (False, True)]
            found += [("gradient", (types, vocab, dim, n, bits, flags)) for n, vocab, dim, _, _ in small.GRADS for flags in (0, 1)]
        found += [("gradient", (types, 2003, dim, large.rows_around(past, dim, rows_type), 64)) for dim in large.DIMS for past in (False, True)]
    for dtype in 0, 1:
        found += [("logits", (dtype, rows, cols, (5, 0, 32), (1,), (1,))) for rows, cols in small.SHAPES]
        found += [("logits", (dtype, rows, cols, (20, 0), (1, 0), (1, 0))) for rows, cols in large.logits_cases(small.TYPES[dtype])]
    return found


def test_every_kernel_of_the_operators_is_run_by_a_gpu_test(run):  # noqa: F811
    seen, known = run("CASES = %r\n%s" % (cases(), CALLS))
    names = subprocess.run(["c++filt"], input="\n".join(sorted(set(known) - set(seen))), capture_output=True, text=True).stdout
    assert len(known) > 100 and set(known) == set(seen), names
