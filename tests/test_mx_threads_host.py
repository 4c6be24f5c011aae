"""The microscaled calls from several threads, as far as no GPU is needed: what the binding looks up once, and messages of calls that fail."""
import os
import threading

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


def test_each_thread_has_its_own_message():
    """Threads that fail in different ways at the same time each read their own reason, and a thread that has not failed reads none of theirs."""
    lib = _lib()
    fails = [(lambda: lib.poss_mx_quantize(1, None, 32, 1, 32, 1 << 20, 1 << 20, None), b"poss_mx_quantize: null argument"),
             (lambda: lib.poss_mx_dequantize(9, 1 << 20, 1 << 20, 1, 32, 1 << 20, 32, None), b"poss_mx_dequantize: bad shape or type"),
             (lambda: lib.poss_mx_pack(1 << 20, 1 << 20, 0, 32, 1 << 20, None), b"poss_mx_pack: bad shape"),
             (lambda: lib.poss_gemm_static(7, 1 << 20, 1 << 20, 1 << 20, 1, 8, 8, 0, None), None)]
    for f, want in fails:                                  # (the last one's own words, whatever they are)
        assert f() != P.POSS_OK
    fails[3] = (fails[3][0], lib.poss_last_error(None))
    step, wrong, fresh = threading.Barrier(len(fails) + 1), [], []

    def failing(f, want):
        for _ in range(50):
            step.wait()
            rc = f()
            step.wait()                                    # (all have failed: now each reads)
            if rc == P.POSS_OK or lib.poss_last_error(None) != want:
                wrong.append((want, lib.poss_last_error(None)))

    def idle():
        for _ in range(50):
            step.wait()
            step.wait()
            fresh.append(lib.poss_last_error(None))
    threads = [threading.Thread(target=failing, args=a) for a in fails] + [threading.Thread(target=idle)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong[0]
    assert set(fresh) == {b""}
