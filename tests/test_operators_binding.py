"""The binding of rotary positions, window attention and the paged cache on the CPU: what it does before a call reaches the library."""
import threading

import pytest

from paper_2604_13847_amd import binding as sb


def test_a_first_call_in_the_middle_of_another(monkeypatch):
    """While one thread looks the library's functions up, another makes its own first call."""
    monkeypatch.setattr(sb, "_calls", None)
    real, answers, started = sb.lib, [], []

    def other():
        try:
            sb._call("sb_cache_attn", None, None, 1, 0, None, None, None, None, None)
        except Exception as e:
            answers.append(str(e))

    def lib():
        if not started:
            started.append(threading.Thread(target=other))
            started[0].start()
            started[0].join()
        return real()

    monkeypatch.setattr(sb, "lib", lib)
    with pytest.raises(sb.SparseBalError, match="null rope|null problem"):
        sb._call("sb_rope_apply", None, None, None, None, 0, None, 0, None, None, 0, None)
    assert len(answers) == 1 and "null cache" in answers[0], answers


def test_what_a_call_keeps_on_another_device_is_refused(monkeypatch):
    """A batch, a cache or new tokens that were laid out on one device, in a call on another: the kernels would read its addresses there."""
    import torch
    # tensors of the CPU say that they lie on device -1, which stands for the first device here
    monkeypatch.setattr(sb, "_here", lambda: (-1, 0))
    x = torch.zeros(3, 2, 16, 64)
    table, cu, cached = (torch.zeros(s, dtype=torch.int32) for s in ((2, 4), (3,), (2,)))
    cache, chunk = sb.Cache(x, x, table), sb.Chunk(cu, cached, 4, 2, 1, 10)
    pb = sb.Problem([0, 40, 100], [1, 1], 4, 2, 64, device="cpu")
    monkeypatch.setattr(sb, "_here", lambda: (0, 0))
    q, elsewhere = torch.zeros(2, 4, 64), "the current device is cuda:0"
    with pytest.raises(sb.SparseBalError, match="cache: .*" + elsewhere):
        sb.sb_cache_attn(cache, chunk, q)
    with pytest.raises(sb.SparseBalError, match="cache: .*" + elsewhere):
        sb.sb_cache_append(cache, chunk, q[:, :2], q[:, :2])
    cache.device = 0
    with pytest.raises(sb.SparseBalError, match="chunk: .*" + elsewhere):
        sb.sb_cache_attn(cache, chunk, q)
    for call in (lambda: sb.sb_rope_apply(pb, sb.Rope(64), q, None), lambda: sb.sb_window_attn_fwd(pb, 8, 2, q, q, q),
                 lambda: sb.sb_window_attn_bwd(pb, 8, 2, q, q, q, q, q, q)):
        with pytest.raises(sb.SparseBalError, match="cu_seqlens: .*" + elsewhere):
            call()
    # positions are read in place of the batch's lengths
    with pytest.raises(sb.SparseBalError, match="^q: a GPU tensor"):
        sb.sb_rope_apply(pb, sb.Rope(64), q, None, positions=torch.zeros(100, dtype=torch.int32))


def test_the_library_is_there_for_all_threads_at_once(monkeypatch):
    """Nobody finds the library before its functions' result types are set: its messages would be numbers."""
    class Loaded:
        def __getattr__(self, name):
            assert sb._lib is None, name
            self.__dict__[name] = f = lambda: None
            return f

    monkeypatch.setattr(sb, "_lib", None)
    monkeypatch.setattr(sb.C, "CDLL", lambda path: Loaded())
    assert isinstance(sb.lib(), Loaded) and sb._lib is sb.lib()


def test_sizes_of_new_tokens_that_do_not_fit_32_bits(monkeypatch):
    """They would arrive as other numbers."""
    import torch
    monkeypatch.setattr(sb, "_here", lambda: (-1, 0))
    cu, cached = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    sb.Chunk(cu, cached, 4, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1)
    for sizes in ((2 ** 32 + 2, 1, 10), (2, 2 ** 32 + 1, 10), (2, 1, 2 ** 31), (2, 1, -(2 ** 32) + 10)):
        with pytest.raises(sb.SparseBalError, match="32 bits"):
            sb.Chunk(cu, cached, 4, *sizes)
    with pytest.raises(sb.SparseBalError, match="32 bits"):
        sb.Chunk(cu, cached, 2 ** 32 + 4, 2, 1, 10)
