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
