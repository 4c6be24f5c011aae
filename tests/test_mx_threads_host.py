"""The microscaled calls from several threads, as far as no GPU is needed: what the binding looks up once."""
import os

import pytest

import paper_2506_03566_amd as P
from paper_2506_03566_amd import binding


def _lib():
    if not os.path.exists(P.LIB_PATH):
        pytest.skip("libposs.so not built (run __graft_entry__.build())")
    return P.load_library()


def test_what_is_looked_up_once_is_whole_before_it_is_seen():
    """A thread goes by `lib` to tell whether the rest is there."""
    _lib()
    seen = []

    class Watched(binding._MxState):
        def __setattr__(self, name, value):
            object.__setattr__(self, name, value)
            seen.append((name, self.lib is not None))
    Watched().open()
    assert {"torch", "u8", "types", "current", "device", "lib"} == {name for name, _ in seen}
    assert [name for name, there in seen if there] == ["lib"]
