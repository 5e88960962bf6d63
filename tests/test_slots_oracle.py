"""Pins of the oracle of the stack of free slots."""
from oracle import slots_oracle as so


def test_hand_worked():
    stack = so.give_back([9, 8], [[1, 2], [], [3]], 10)
    assert stack == [9, 8, 1, 2, 3]
    assert so.give_back([9, 8], [[1, 2], [3]], 4) == [9, 8, 1, 2]
    left, got = so.take(stack, [2, 0, 1])
    assert left == [9, 8] and got == [[1, 2], [], [3]]


def test_the_first_that_does_not_fit_ends_it():
    left, got = so.take([5, 6, 7], [1, 3, 1])
    assert left == [5, 6] and got == [[7], [], []]
    assert so.take([], [0, 1]) == ([], [[], []])
    assert so.take([4], [2]) == ([4], [[]])


def test_a_list_without_room_holds_nobody_up():
    left, got = so.take([5, 6, 7], [1, 2, 2], n_live=[3, 4, 0], rooms=[4, 5, 2])
    assert left == [] and got == [[5], [], [6, 7]]


def test_back_again():
    stack = list(range(20, 40))
    left, got = so.take(stack, [3, 4, 5])
    assert so.give_back(left, got, 100) == stack
