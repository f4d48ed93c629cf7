"""Trees for the tests of generation that branches."""
import numpy as np


def chain(n):
    return [i - 1 for i in range(n)]


def star(n):
    return [-1] + [0] * (n - 1) if n else []


def random_tree(rng, n, near=None, roots=0.0):
    """Parents anywhere before their children (among the `near` nodes before), some nodes roots."""
    return [-1] + [-1 if rng.random() < roots else int(rng.integers(max(0, i - near) if near else 0, i)) for i in range(1, n)] if n else []


def ranges(trees):
    return np.cumsum([0] + [len(t) for t in trees]).tolist()
