"""Shapes that reach each kernel of the attention over the 4-bit cache, as tree_cases.py has them for the 8-bit one
(test_fp4_plan_host.py holds the names to the plan).

few1, few2: one or two tiles of 16 rows a workgroup; many: pages staged for four waves of 16 rows; wide: tiles of 32 rows;
paired: a tile of 32 to two waves; +split: the keys of a prompt over several workgroups."""
from tree_cases import KINDS, Case


def _bf16(name, else_):
    return lambda kind, fmt: name if kind == "bf16" else else_


LONG = [6600, 5, 0, 77, 64, 31, 200, 1030]
ALL = [
    Case("few1", 2, 2, 8, 2, 128, 70, [33, 70], "few1"),
    Case("few2", 2, 6, 8, 2, 128, 70, [33, 70], "few2"),
    Case("few2 hd64", 2, 3, 16, 2, 64, 70, [33, 70], "few2"),
    Case("few1 hd32", 3, 1, 10, 2, 32, 70, [33, 1, 70], "few1"),
    Case("many", 2, 20, 8, 2, 128, 70, [33, 70], "many"),
    Case("many hd64", 2, 33, 5, 1, 64, 70, [33, 70], "many"),
    Case("many hd32", 2, 20, 8, 2, 32, 70, [64, 31], "many"),
    Case("wide", 96, 32, 32, 8, 128, 61, None, _bf16("wide", "many")),
    Case("wide hd64", 96, 31, 32, 8, 64, 61, None, _bf16("wide", "many")),
    Case("wide hd32", 96, 32, 32, 8, 32, 61, None, _bf16("wide", "many")),
    Case("paired", 28, 32, 32, 8, 128, 1100, [1100] + [33] * 12 + list(range(14)) + [61], "paired"),
    Case("paired hd64", 28, 30, 32, 8, 64, 1100, [61] + [33] * 12 + list(range(14)) + [1100], "paired"),
    Case("paired hd32", 32, 17, 32, 8, 32, 1100, [1100] + [64] * 12 + list(range(18)) + [61], "paired"),
    Case("few1 split", 1, 1, 8, 1, 128, 5000, [5000], "few1+split"),
    Case("few2 split", 2, 3, 16, 2, 128, 3000, [3000, 50], "few2+split"),
    Case("many split", 1, 40, 8, 1, 128, 1500, [1500], "many+split"),
    Case("wide split", 8, 17, 32, 8, 128, 6600, LONG, "wide+split"),
    Case("wide split 30", 8, 30, 32, 8, 128, 6600, LONG[::-1], "wide+split"),
    Case("wide split 65", 8, 65, 32, 8, 128, 6600, LONG, _bf16("wide+split", "many+split")),
    Case("wide split hd64", 8, 17, 32, 8, 64, 6600, LONG, "wide+split"),
    Case("wide split hd32", 8, 31, 32, 8, 32, 6600, LONG[::-1], "wide+split"),
]


def params():
    import pytest
    return [pytest.param(c, k, id=f"{c.name}-{k}".replace(" ", "_")) for c in ALL for k in KINDS]


# Unsplit prompts of so many pages that a wave takes page ids more than once (64 at a time): first and last are long, the rest
# hold a token.  (B, n, H, KV heads, head dim, longest)
MANY_PAGES = [
    Case("few1 long", 70, 1, 8, 8, 32, 9000, None, "few1"),
    Case("few2 long", 70, 20, 8, 8, 64, 9000, None, "few2"),
    Case("many long", 70, 40, 8, 8, 64, 4200, None, "many"),
    Case("paired long", 28, 32, 32, 8, 64, 4400, None, "paired"),
    Case("wide long", 96, 32, 32, 8, 32, 4200, None, _bf16("wide", "many")),
]
