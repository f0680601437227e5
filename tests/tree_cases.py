"""Shapes that reach each kernel of the tree attention: (B, n, H, KV heads, head dim, longest prompt), with the kernel
that the plan takes for a row type and a cache format (test_tree_plan_host.py holds the names to it).

few1, few2: one or two tiles of 16 rows a workgroup; many3, many4: pages staged for four waves, three or four of them a
SIMD; wide: tiles of 32 rows; +split: the keys of a prompt over several workgroups."""
import numpy as np

KINDS, FMTS = ("f32", "bf16"), ("int8", "e4m3")


class Case:
    def __init__(self, name, B, n, H, heads, hd, longest, lens, expect):
        self.name, self.B, self.n, self.H, self.heads, self.hd, self.longest = name, B, n, H, heads, hd, longest
        self._lens, self.expect = lens, expect

    def lens(self, rng):
        """Prompt lengths; the first and the last prompt are the ones that a test compares."""
        if self._lens is not None:
            return list(self._lens)
        lens = rng.integers(0, 60, self.B).tolist()
        lens[0], lens[-1] = 33, 61
        return lens

    def kernel(self, kind, fmt):
        e = self.expect
        return e if isinstance(e, str) else e(kind, fmt)


def _four(kind, fmt):
    return "many4" if kind == "bf16" or fmt == "e4m3" else "many3"


def _wide(kind, fmt):
    return "many4" if (kind, fmt) == ("f32", "e4m3") else "wide"


WHOLE = [
    Case("few1", 2, 2, 8, 2, 128, 70, [33, 70], "few1"),
    Case("few2", 2, 6, 8, 2, 128, 70, [33, 70], "few2"),
    Case("few2 hd64", 2, 3, 16, 2, 64, 70, [33, 70], "few2"),
    Case("many", 2, 20, 8, 2, 128, 70, [33, 70], "many3"),
    Case("many that fill the chip", 64, 65, 32, 8, 128, 61, None, _four),
    Case("wide", 96, 32, 32, 8, 128, 61, None, _wide),
    Case("wide once", 60, 32, 32, 8, 128, 61, None, lambda kind, fmt: "wide" if kind == "bf16" else "many3"),
]
SPLIT = [
    Case("few1 split", 1, 1, 8, 1, 128, 5000, [5000], "few1+split"),
    Case("few2 split", 2, 3, 16, 2, 128, 3000, [3000, 50], "few2+split"),
    Case("many split", 1, 40, 8, 1, 128, 1500, [1500], "many3+split"),
    Case("wide split", 8, 17, 32, 8, 128, 4200, [4200, 5, 0, 77, 64, 31, 200, 1030],
         lambda kind, fmt: "many3+split" if (kind, fmt) == ("f32", "e4m3") else "wide+split"),
    Case("wide split 30", 8, 30, 32, 8, 128, 4200, [1030, 5, 0, 77, 64, 31, 200, 4200],
         lambda kind, fmt: "many3+split" if (kind, fmt) == ("f32", "e4m3") else "wide+split"),
]
ALL = WHOLE + SPLIT


def params(cases=None):
    """(case, kind, fmt) with readable ids."""
    import pytest
    return [pytest.param(c, k, f, id=f"{c.name}-{k}-{f}".replace(" ", "_")) for c in cases or ALL for k in KINDS for f in FMTS]



def rms(x):
    return float(np.sqrt(np.mean(np.square(np.asarray(x, np.float64)))))
