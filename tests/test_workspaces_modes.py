"""The handle's workspaces without a GPU: what one mode of torch has made, calls in another one take."""
import itertools

import pytest
import torch

from paper_2309_06973_amd import q8, shifter as S


def handle():
    h = q8.Q8.__new__(q8.Q8)
    h.dev, h.work, h.recorded, h.joined, h.recorded_joined = torch.device("cpu"), None, [], None, []
    return h


MODES = {"none": torch.enable_grad, "no_grad": torch.no_grad, "inference": torch.inference_mode}


@pytest.mark.parametrize("first, then", itertools.product(MODES, MODES))
@pytest.mark.parametrize("recording", [False, True])
def test_workspaces_of_one_mode_serve_another(monkeypatch, first, then, recording):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: recording)
    h = handle()
    for room, bytes_ in ((h._joined, S.SHIFTER_LEARN_ZERO + 100), (h._room, 300)):
        with MODES[first]():
            work = room(bytes_)
        with MODES[then]():
            again = room(bytes_ - 50)
            more = room(bytes_ + 50)
        assert again is work and more is not work and more.numel() == bytes_ + 50
        assert room(bytes_) is more
    assert (h._joined(10)[:S.SHIFTER_LEARN_ZERO] == 0).all()
