"""The pages of examples/decode.py's sessions (no GPU needed)."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")


def session(pages, users, page_tokens=16, most_pages=4):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode.py")
    spec = importlib.util.spec_from_file_location("decode_example_cpu", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    s = object.__new__(m.Session)                         # without a model and its cache
    s.page_tokens, s.most_pages, s.free, s.lens = page_tokens, most_pages, list(range(pages)), [0] * users
    s.table = torch.full((users, most_pages), -1, dtype=torch.int32)
    return s


def test_users_take_pages_as_they_grow():
    s = session(8, 3)
    s._grow([17, 0, 1])
    s._grow([15, 16, 1])
    assert s.lens == [32, 16, 2] and len(s.free) == 4
    taken = s.table[s.table >= 0].tolist()
    assert sorted(taken + s.free) == list(range(8)) and [(r >= 0).sum().item() for r in s.table] == [2, 1, 1]


@pytest.mark.parametrize("news", [[16, 16, 33], [65, 0, 0], [1, 1, 64]])
def test_a_step_without_room_takes_nothing(news):
    s = session(5, 3)
    s._grow([16, 16, 1])
    lens, free, table = list(s.lens), list(s.free), s.table.clone()
    with pytest.raises(RuntimeError, match="no page left"):
        s._grow(news)
    assert s.lens == lens and s.free == free and torch.equal(s.table, table)
    s._grow([0, 0, 31])                                   # the session goes on
    assert s.lens == [16, 16, 32]
