"""Which kernel a call of the attention over trees gets and how its walks are cut, and whose rows are whose where row_start is not in order:
pure host arithmetic."""
import torch

from span_plan import span_plan


def tree_plan(case):
    """The plan of a call of test_gpu_tree.Case."""
    return span_plan(case.T, case.dtype == torch.bfloat16, case.four, case.B, case.heads, (0, 1, case.max_nodes, 0), 0, 0, case.hint)


def kind(p):
    """"few" or "many" rows, and whether all walks are whole, some or none."""
    return ("many" if p.rows else "few") + ("" if p.splits == 1 else ", cut" if not p.rows or p.whole == 0 else ", some cut")


def owned(start, n_rows, most=256):
    """By sequence: its rows, or None where its row_start is not valid (its range is not in order, not within the arrays, of more than `most` rows, or
    has a row of an earlier range)."""
    ranges = [range(s, e) if 0 <= s <= e <= n_rows and e - s <= most else None for s, e in zip(start, start[1:])]
    return [r if r is not None and not any(set(r) & set(x or ()) for x in ranges[:b]) else None for b, r in enumerate(ranges)]
