"""The count of ids out of range: cleared before the call returns, and not asked for in a capture (on a fake device)."""
import test_host_client as H


def test_count_and_reset(tmp_path, monkeypatch):
    monkeypatch.setattr(H, "HOST_SOURCES", H.HOST_SOURCES + ["she_clear.cpp"])
    H.run_on_fake_device("clear_counter_check.cpp", tmp_path)
