"""Operators on ragged batches and 8-bit pages, without a device: what their sources promise, and sizes at the ends of their ranges."""
import glob
import os
import re

import paper_2403_09054_b200 as kf

CSRC = os.path.join(os.path.dirname(os.path.abspath(kf.__file__)), "csrc")


def _kernels():
    """(file, name, body) of the kernels of files that launch kernels before the one in front of them has ended."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        text = open(path).read()
        if "launch_early(" not in text:
            continue
        starts = [(m.start(), m.group(1)) for m in re.finditer(r"__global__ void __launch_bounds__\([^\n]*?\) (\w+)\(", text)]
        for (at, name), end in zip(starts, [s for s, _ in starts[1:]] + [len(text)]):
            yield os.path.basename(path), name, text[at:end]


def test_kernels_that_launch_early_wait_before_they_take_anything_that_lasts():
    """A kernel that holds tensor memory while it waits for the one before could keep that one from ever getting its own; and nothing of global memory may be touched."""
    seen = 0
    for file, name, body in _kernels():
        seen += 1
        wait = body.find("after_earlier_kernels();")
        assert wait >= 0, (file, name)
        for taken in ("tmem_alloc(", "P.begin[", "a.length[", "U.length[", "U.parent", "let_next_kernel_launch();"):
            at = body.find(taken)
            assert at < 0 or at > wait, (file, name, taken)
    assert seen >= 8


def test_scratch_of_sizes_beyond_32_bits():
    """What does not fit the argument structs is not supported: no bytes, not those of another size."""
    attend = dict(sequences=3, table_width=4, n_pages=20, page_tokens=16, n_heads=4, n_kv_heads=2, head_dim=64)
    update = dict(sequences=3, table_width=4, n_pages=20, page_tokens=16, n_kv_heads=2, head_dim=64, n_layers=2)
    assert kf.kf_pages_attend_scratch_bytes(**attend) > 0 and kf.kf_pages_update_scratch_bytes(**update) > 0
    for f, base in ((kf.kf_pages_attend_scratch_bytes, attend), (kf.kf_pages_update_scratch_bytes, update)):
        for name, value in base.items():
            for far in (value + 2 ** 32, value - 2 ** 32, 2 ** 31, 2 ** 70):
                assert f(**{**base, name: far}) == 0, (name, far)
