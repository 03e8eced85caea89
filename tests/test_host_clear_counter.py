"""The clear side's calls on a fake device: the count of ids out of range, and devices other than the context's."""
import test_host_client as H


def test_count_and_reset(tmp_path, monkeypatch):
    monkeypatch.setattr(H, "HOST_SOURCES", H.HOST_SOURCES + ["she_clear.cpp"])
    H.run_on_fake_device("clear_counter_check.cpp", tmp_path)


def test_another_device_is_refused(tmp_path, monkeypatch):
    monkeypatch.setattr(H, "HOST_SOURCES", H.HOST_SOURCES + ["she_clear.cpp"])
    H.run_on_fake_device("clear_device_check.cpp", tmp_path)
