"""The self-test of the waits without a device: refusals."""
import paper_2411_19870_b200 as demo


def test_null_context():
    assert demo.load_library().demo_muon_selftest_bounded_wait(None, 1000, None) == 1
