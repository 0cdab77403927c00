"""The scratch buffer that calls share: what becomes of it when a call needs more (on the CPU; the calls themselves are GPU tests)."""
import weakref

import pytest

from paper_2509_05576_b200 import build as ptq_build


@pytest.fixture(scope="module")
def ptq():
    ptq_build.build()
    from paper_2509_05576_b200 import ptq as module
    return module


def test_a_buffer_is_kept_until_a_call_needs_more(ptq):
    ws = ptq.Workspace("cpu")
    first = ws.get(1000)
    assert first.numel() >= 1000 and ws.get(10) is first and ws.get(1000) is first and ws.buf is first
    gone = weakref.ref(first)
    del first
    assert ws.get(100000).numel() >= 100000 and gone() is None


def test_a_buffer_that_a_graph_writes_to_stays(ptq, monkeypatch):
    ws = ptq.Workspace("cpu")
    seen = [weakref.ref(ws.get(1000))]
    monkeypatch.setattr(ptq, "_is_capturing", lambda dev, stream: True)
    for n in (1000, 900, 5000, 6000):                    # captured: the first buffer, then two larger ones
        seen.append(weakref.ref(ws.get(n)))
        assert ws.get(n) is seen[-1]()
    monkeypatch.setattr(ptq, "_is_capturing", lambda dev, stream: False)
    seen.append(weakref.ref(ws.get(10 ** 5)))
    seen.append(weakref.ref(ws.get(10 ** 6)))
    assert [r() is not None for r in seen] == [True] * 5 + [False, True]
    assert seen[0]() is seen[1]() and seen[1]() is seen[2]()
    places = {r().data_ptr() for r in seen if r() is not None}
    assert len(places) == 4
    del ws
    assert all(r() is None for r in seen)
