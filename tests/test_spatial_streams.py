"""A stream given to the spatial calls is the call's, by keyword or in its place among the arguments."""
import contextlib

import pytest
import torch

import paper_2506_21411_amd as dchag


@pytest.fixture
def entered(monkeypatch):
    """The streams that calls were made on."""
    seen = []

    @contextlib.contextmanager
    def on(stream):
        seen.append(stream)
        yield

    monkeypatch.setattr(torch.cuda, "stream", on)
    return seen


X, CODES, SCALES = torch.zeros(4, 32), torch.zeros((4, 32), dtype=torch.uint8), torch.zeros((4, 1), dtype=torch.uint8)
CALLS = [
    (dchag.dchag_pack8, (X, None, None)),
    (dchag.dchag_unpack8, (CODES, SCALES, torch.bfloat16, None)),
    (dchag.dchag_weight_grad8, (X, CODES, SCALES, None, None, True, None)),
]


@pytest.mark.parametrize("call,args", CALLS, ids=[c.__name__ for c, _ in CALLS])
def test_stream_in_its_place_and_by_keyword(entered, call, args):
    stream = object()
    for how in (lambda: call(*args, stream), lambda: call(*args, stream=stream)):
        entered.clear()
        with pytest.raises(ValueError):                            # not tensors of a device
            how()
        assert entered == [stream]
    entered.clear()
    for how in (lambda: call(*args), lambda: call(*args, None), lambda: call(*args, stream=None)):
        with pytest.raises(ValueError):
            how()
    assert entered == []
    with pytest.raises(TypeError):
        call(*args, stream, stream=stream)


def test_stream_of_the_attention_is_a_keyword(entered):
    q, k, s, stream = torch.zeros(6, 4, 64), torch.zeros(6, 2, 64), torch.zeros(2, dtype=torch.int32), object()
    with pytest.raises(ValueError):
        dchag.dchag_attend(q, k, k, s, s, stream=stream)
    assert entered == [stream]
    with pytest.raises(TypeError):
        dchag.dchag_attend(q, k, k, s, s, stream)
