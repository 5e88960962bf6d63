"""Plain oracle of the stack of free slots, one entry at a time.

TEST INFRASTRUCTURE ONLY, like ikv_oracle.py: it shares no code with the HIP library.
Pinned by tests/test_slots_oracle.py.
"""
from __future__ import annotations


def give_back(stack, lists, room):
    """The stack after the sessions' lists are pushed onto it, in order; at most `room` entries."""
    stack = list(stack)
    for entries in lists:
        for slot in entries:
            if len(stack) < room:
                stack.append(slot)
    return stack


def take(stack, wants, n_live=None, rooms=None):
    """Sessions that want so many slots each, with n_live entries in lists of so much room (None: no lists).

    Returns (the stack afterwards, the slots of each session)."""
    wants = list(wants)
    if n_live is not None:
        wants = [w if n + w <= room else 0 for w, n, room in zip(wants, n_live, rooms)]
    total, served = 0, 0
    for i, w in enumerate(wants):
        if total + w > len(stack):
            break
        total += w
        served = i + 1
    at, out = len(stack) - total, []
    for i, w in enumerate(wants):
        w = w if i < served else 0
        out.append(list(stack[at:at + w]))
        at += w
    return list(stack[:len(stack) - total]), out
