"""Oracle: page tables and slots, one page and one row at a time.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``).  The paper does not fix a
cache layout; what the tables mean is in ``oracle/paged.py``.

Pins: ``tests/test_oracle_pages.py``.
"""
from __future__ import annotations


def resize(length, held, table, stack, P):
    """Lists length, held [B], table [B][max_pages], stack (its top last), changed
    in place; returns granted [B]."""
    B = len(length)
    need = [-(-n // P) for n in length]
    for b in range(B):
        for j in range(need[b], held[b]):
            stack.append(table[b][j])
            table[b][j] = -1
        held[b] = min(held[b], need[b])
    granted, closed = [1] * B, False
    for b in range(B):
        lack = need[b] - held[b]
        if lack <= 0:
            continue
        if closed or lack > len(stack):
            granted[b], closed = 0, True
            continue
        for j in range(held[b], need[b]):
            table[b][j] = stack.pop()
        held[b] = need[b]
    return granted


def slot_map(ctx, n_new, n_rows, P, table=None, rows_per_seq=0):
    """(slots, pos, seq, row_start) as lists."""
    slots, pos, seq, start = [-1] * n_rows, [0] * n_rows, [-1] * n_rows, [0]
    for b, n in enumerate(n_new):
        first = b * rows_per_seq if rows_per_seq else start[-1]
        start.append(start[-1] + n)
        for j in range(n):
            t = ctx[b] + j
            page = b if table is None else table[b][t // P]
            at = t if table is None else t % P
            slots[first + j], pos[first + j], seq[first + j] = page * P + at, t, b
    return slots, pos, seq, start
