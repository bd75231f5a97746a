"""The binding of the dense-layer and optimizer operators around the library's calls, with a library that does nothing."""
import threading

import pytest
import torch

from paper_2406_05546_amd import dense


class Tensor:
    def __init__(self):
        self.streams = []

    def record_stream(self, stream):
        self.streams.append(stream)


class Library:
    def ps_adamw_step(self, handle, options, stream):
        return 0

    def ps_adamw_destroy(self, handle):
        return 0


@pytest.fixture
def stand_in(monkeypatch):
    """One device, whose current stream is the number in `now`, and the library's place taken."""
    class Case:
        now, library = 7, Library()
    case = Case()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: f"stream {case.now}")
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: case.now)
    monkeypatch.setattr(dense, "_library", lambda: case.library)
    return case


def table(stream):
    lists = [[Tensor()] for _ in range(7)]
    opt = dense.AdamW(None, torch.device("cuda", 0), 8, *lists[:6], [None], Tensor(), 1, {stream})
    return opt, [t for lst in lists[:6] for t in lst] + [opt.workspace]


def test_a_step_on_another_stream_is_known_to_the_allocator(stand_in):
    """The table and all tensors that the handle keeps alive may be freed with it while the step runs: not for use on the stream where they were
    made before that one is done."""
    opt, kept = table(7)
    dense.ps_adamw_step(opt, 1, 0.1)
    assert all(t.streams == [] for t in kept)
    for stand_in.now in (9, 9, 7, 11):
        dense.ps_adamw_step(opt, 1, 0.1)
    assert all(t.streams == ["stream 9", "stream 11"] for t in kept)


def test_two_threads_step_one_table_each_with_its_own_options(stand_in):
    """Each call reads what its thread asked for, although the other thread calls in between."""
    both, seen = threading.Barrier(2, timeout=20), {}

    class Waits(Library):
        def ps_adamw_step(self, handle, options, stream):
            both.wait()  # both calls have written their options
            seen[threading.get_ident()] = (options._obj.lr, options._obj.step, options._obj.n_rows)
            both.wait()
            return 0
    stand_in.library = Waits()
    opt, _ = table(7)
    opt.rows, asked = 5, {}

    def step(lr, number, rows):
        asked[threading.get_ident()] = (lr, number, 5 if rows is None else rows)
        dense.ps_adamw_step(opt, number, lr, n_rows=rows)
    threads = [threading.Thread(target=step, args=a) for a in ((0.25, 3, 2), (0.5, 4, None))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert seen == asked and len(seen) == 2
