"""The three e5m2 parts of a weight, without a GPU: how far their sum is from the weight, over all of fp16.

The arithmetic of take_apart in csrc/serve/attend_fp8_tc.cu: an fp32 weight is rounded to fp16; the first part is its
upper byte, the second the upper byte of four times what is left, the third eight times what is left then, rounded.
"""

import re
from pathlib import Path

import numpy as np
import torch

ROOT = Path(__file__).resolve().parent.parent
TOP, FIRST = 2.0**15, 2.0**3  # a weight passes TOP in no tile; a row's largest is FIRST or more


def upper(x):
    return (x.view(np.uint16) & np.uint16(0xFF00)).view(np.float16)


def parts_sum(a):
    """What the parts of fp16 numbers stand for, in float64."""
    first = upper(a)
    rest = (a - first) * np.float16(4)
    second = upper(rest)
    last = (rest - second) * np.float16(8)
    assert last.max() <= 57344  # no part is cut off
    third = torch.from_numpy(last).to(torch.float8_e5m2).double().numpy()
    return first.astype(np.float64) + second.astype(np.float64) / 4 + third / 32


def test_the_error_of_a_weight_is_what_the_header_says():
    a = np.arange(0x7800 + 1, dtype=np.uint16).view(np.float16)  # 0 to 2^15
    assert a[-1] == TOP
    exact, got = a.astype(np.float64), parts_sum(a)
    # a weight lies within half a step of its fp16 number: the ends are the worst
    half = np.diff(exact) / 2
    relative = smallest = 0.0
    for end in (exact[:-1] + half, exact[1:] - half):
        for of in (got[:-1], got[1:]):
            err = np.abs(end - of)
            large = end >= 2.0**-13
            relative = max(relative, float((err / np.maximum(end, 1e-30))[large].max()))
            smallest = max(smallest, float(err[~large].max()))
    print("of the weight: 2 ^", np.log2(relative), ", absolute: 2 ^", np.log2(smallest))
    text = " ".join((ROOT / "include" / "retrace.h").read_text().replace("*", " ").split())
    said = re.search(r"a weight the sum of three e5m2 numbers: off by at most (?:2\^-(\d+) \+ )?2\^-(\d+) of it, or by 2\^-(\d+) of the row's largest weight", text)
    of_it = 2.0 ** -int(said[2]) + (2.0 ** -int(said[1]) if said[1] else 0.0)
    assert relative <= of_it, (relative, of_it)
    assert smallest / FIRST <= 2.0 ** -int(said[3])
