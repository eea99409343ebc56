"""Whether two views have memory in common, as the calls that refuse it decide it, against the sets of their elements' addresses."""
import random

import pytest

torch = pytest.importorskip("torch")

from paper_2412_04964_amd import binding as b  # noqa: E402


def elements(t):
    at = torch.arange(t.untyped_storage().nbytes() // t.element_size()).as_strided(t.shape, t.stride(), t.storage_offset())
    return set(at.flatten().tolist())


def view(base, rng, axes):
    """a view of `base` of 1 to 3 axes, the last one dense, with strides of any kind"""
    shape = [rng.choice([1, 1, 2, 3, 5]) for _ in range(axes - 1)] + [rng.choice([1, 2, 4, 7])]
    strides = [rng.choice([0, 1, 2, 4, 8, 12, 13, 16, 24]) for _ in range(axes - 1)] + [1]
    room = base.numel() - sum(s * (n - 1) for s, n in zip(strides, shape)) - 1
    return base.as_strided(shape, strides, rng.randint(0, min(room, 30)))


def test_views_of_one_buffer_against_their_elements():
    rng = random.Random(1)
    base = torch.zeros(260, dtype=torch.int16)
    found = [0, 0]
    for i in range(6000):
        x, y = view(base, rng, rng.choice([1, 2, 2, 3])), view(base, rng, rng.choice([1, 2, 2, 3]))
        if i % 2 and x.dim() == y.dim() == 2:              # rows of one stride
            y = base.as_strided(y.shape, (x.stride(0), 1), rng.randint(0, 60))
        want = bool(elements(x) & elements(y))
        assert b._meet(x, y) == want == b._meet(y, x), (x.shape, x.stride(), x.storage_offset(), y.shape, y.stride(), y.storage_offset())
        found[want] += 1
    assert min(found) > 500, found


def test_views_of_different_types_and_none_at_all():
    base = torch.zeros(64, dtype=torch.uint8)
    halves, floats = base[:32].view(torch.float16), base[32:].view(torch.float32)
    assert not b._meet(halves, floats) and b._meet(base, floats) and b._meet(base[30:33], floats) and not b._meet(base[:32], floats)
    assert not b._meet(base[:0], base) and not b._meet(base, base[:0])
    assert not b._meet(torch.zeros(64), torch.zeros(64))
    # side by side in a joint buffer: rows between rows
    joint = torch.zeros((1000, 48), dtype=torch.float16)
    assert not b._meet(joint[:, :16], joint[:, 16:32]) and b._meet(joint[:, :17], joint[:, 16:32]) and b._meet(joint[:-1, :16], joint[1:, :16])
    assert not b._meet(joint[:500, :16], joint[500:, :16])
