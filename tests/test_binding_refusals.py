"""What the binding of the calls around a frame's attention refuses, without a GPU."""
import pytest

from paper_2609_23286_amd import rv


@pytest.fixture
def on_device_0(monkeypatch):
    """Device 0 is current, and a call that reaches the library fails the test."""
    def reached(*args):
        pytest.fail("the call was made")

    monkeypatch.setattr(rv, "_where", lambda stream: (0, 0))
    monkeypatch.setattr(rv.torch.cuda, "current_device", lambda: 0)
    for name in ("prepare", "prepare_bwd"):
        monkeypatch.setattr(rv._bind, name, reached)


def test_weights_of_another_device_are_refused(on_device_0):
    prep = rv.QKVPrep(2, 2)
    assert prep.device is None  # (no weights: any device)
    prep.device = 1
    for call, n in ((rv.prepare_qkv, 7), (rv.prepare_qkv_bwd, 9), (rv.stage_qkv, 6)):
        with pytest.raises(ValueError, match="weights and biases on device 1 while device 0 is current"):
            call(prep, *[None] * n)


def test_weights_of_two_devices_are_refused(monkeypatch):
    class Weights(rv.torch.Tensor):
        def get_device(self):
            return self.number

    vectors = []
    for number in (0, 1):
        vectors.append(rv.torch.ones(64).as_subclass(Weights))
        vectors[-1].number = number
    monkeypatch.setattr(rv, "_ptr", lambda t, *args: None)
    assert rv.QKVPrep(2, 2, q_weight=vectors[1], k_bias=vectors[1]).device == 1
    with pytest.raises(ValueError, match="different devices"):
        rv.QKVPrep(2, 2, q_weight=vectors[0], k_weight=vectors[1])
