"""The calls around a block in the C ABI without a GPU: their refusals on a fake device."""
import test_host_client as H


def test_refusals_and_scratch_on_the_fake_device(tmp_path, monkeypatch):
    monkeypatch.setattr(H, "HOST_SOURCES", H.HOST_SOURCES + ["she_clear.cpp", "she_clear_step.cpp"])
    H.run_on_fake_device("clear_step_check.cpp", tmp_path)
