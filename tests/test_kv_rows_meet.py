"""Whether rows of keys and of values, results of zc.read_kv in one buffer, have elements in common: worked out from strides alone, with no tensor made on
the way (under a default device it would be the GPU's, and asking it a wait, which a stream that is being recorded refuses)."""
import random

import pytest
import torch
from torch.overrides import TorchFunctionMode

from paper_2508_19263_amd import zc


class Rows:
    """What _rows_meet looks at of a tensor."""

    def __init__(self, shape, strides, at):
        self.shape, self.strides, self.at = shape, tuple(strides) + (1,), at

    def stride(self):
        return self.strides

    def data_ptr(self):
        return 2 * self.at

    def starts(self):
        return [self.at + i * self.strides[0] + j * self.strides[1] for i in range(self.shape[0]) for j in range(self.shape[1])]

    def apart(self):
        x = sorted(self.starts())
        return all(b - a >= self.shape[2] for a, b in zip(x, x[1:]))


def meet(k, v):
    """Rows of one length meet where they begin less than it apart: every pair."""
    dim = k.shape[2]
    return any(abs(a - b) < dim for a in k.starts() for b in v.starts())


@pytest.mark.parametrize("seed", range(6))
def test_layouts_of_all_kinds(seed):
    """Small rows, so that every way to lie between each other and on top of each other comes up; with the same strides and with others."""
    r, seen, done = random.Random(seed), {}, 0
    while done < 4000:
        n, heads, dim = r.choice((1, 1, 2, 3, 5, 9)), r.choice((1, 2, 3, 4)), r.choice((1, 2, 3, 5, 8))

        def strides():
            head = r.randint(dim, 4 * dim)
            token = (heads - 1) * head + dim + r.choice((0, 0, r.randint(0, 4 * dim)))
            if r.random() < 0.3:                               # head by head
                token = r.randint(dim, 4 * dim)
                head = (n - 1) * token + dim + r.choice((0, r.randint(0, 4 * dim)))
            return (r.randint(0, 99) if n == 1 else token, r.randint(0, 99) if heads == 1 else head)
        same = r.random() < 0.5
        a = strides()
        k, v = Rows((n, heads, dim), a, 1000), Rows((n, heads, dim), a if same else strides(), 0)
        if not k.apart() or not v.apart():
            continue
        room = max(k.starts()) - 1000 + max(v.starts()) + 2 * dim
        v.at = 1000 + r.randint(-room, room)
        want = meet(k, v)
        assert zc._rows_meet(k, v) == want, (k.shape, k.strides, v.strides, v.at - k.at)
        seen[same, want] = seen.get((same, want), 0) + 1
        done += 1
    assert all(seen.get((same, want), 0) > 200 for same in (True, False) for want in (True, False)), seen


@pytest.mark.parametrize("seed", range(3))
def test_the_least_multiple_in_an_interval(seed):
    r = random.Random(seed)
    for _ in range(3000):
        m = r.randint(1, 60)
        a, lo = r.randint(0, 2 * m), r.randint(0, m - 1)
        hi = r.randint(lo, m - 1)
        assert zc._least_in(a, m, lo, hi) == next((x for x in range(m + 1) if lo <= a * x % m <= hi), None)


class Counted(TorchFunctionMode):
    def __init__(self):
        super().__init__()
        self.calls = []

    def __torch_function__(self, f, types, args=(), kwargs=None):
        self.calls.append(getattr(f, "__name__", str(f)))
        return f(*args, **(kwargs or {}))


@pytest.mark.parametrize("k_strides,v_strides,off,want", [((4096, 128), (4096, 128), 1024, False), ((2048, 256), (2048, 256), 128, False), ((2048, 256), (2048, 256), 64, True),
                                                          ((128, 128 * 500), (128, 128 * 500), 64, True), ((4096, 128), (8192, 128), 1024, False),
                                                          ((4096, 128), (8192 + 8, 128), 1024, False), ((4096, 128), (8192 + 16, 128), 1024, True)])
def test_no_tensor_is_made(k_strides, v_strides, off, want):
    room = torch.zeros(1 << 23, dtype=torch.bfloat16)
    k, v = room.as_strided((500, 8, 128), k_strides + (1,), 0), room.as_strided((500, 8, 128), v_strides + (1,), off)
    with Counted() as c:
        assert zc._rows_meet(k, v) == want
    assert set(c.calls) <= {"stride", "data_ptr", "__get__"}, c.calls


def test_under_a_default_device():
    """(Tensors of "meta" have no values: asking one is an error here, as asking a GPU's is while a stream is being recorded.)"""
    room = torch.zeros(1 << 16, dtype=torch.bfloat16)
    k, v = room.as_strided((5, 2, 64), (400, 64, 1), 0), room.as_strided((5, 2, 64), (800, 64, 1), 128)
    with torch.device("meta"):
        assert zc._rows_meet(k, v) is False


def test_long_results_are_answered_at_once():
    """A million tokens: nothing is done for each of them."""
    k = Rows((1 << 20, 8, 128), (4096, 128), 0)
    # a token of V lies 1,024 (or 2,048 more) behind one of K, whose heads take 1,024 (64 less: the last of them is touched); or 8 further with each
    for v, want in ((Rows(k.shape, (6144, 128), 1024), False), (Rows(k.shape, (6144, 128), 960), True), (Rows(k.shape, (8192, 128), 1024), False),
                    (Rows(k.shape, (8200, 128), 1024), True)):
        asked = []
        v.stride = lambda v=v: asked.append(1) or v.strides
        assert zc._rows_meet(k, v) is want and len(asked) == 1
