"""What the decode step's program does around its steps: it lets the stream that
made the inputs finish first, and it does not report a run that failed."""
from unittest.mock import MagicMock

import pytest

from paper_2606_22541_gb300 import decode_step


@pytest.fixture
def program(monkeypatch):
    """decode_step.main on recorded calls; returns (torch's calls by name in order, the api)."""
    torch, api = MagicMock(), MagicMock()
    torch.cuda.Event.return_value.elapsed_time.return_value = 1.0
    torch.empty.return_value.__gt__ = lambda self, other: MagicMock()
    api.asap_moe_status.return_value = (0, 0)

    class Step:
        def __init__(self, *a):
            self.ws = None

        def __call__(self, x):
            torch.step()

    monkeypatch.setattr(decode_step, "torch", torch)
    monkeypatch.setattr(decode_step, "api", api)
    monkeypatch.setattr(decode_step, "inputs", MagicMock())
    monkeypatch.setattr(decode_step, "_dense_layer", lambda *a: MagicMock(weight_bytes=lambda: 1000))
    monkeypatch.setattr(decode_step, "DecodeStep", Step)

    def run():
        decode_step.main(["--tokens", "2,5", "--steps", "3"])
        return [c[0] for c in torch.mock_calls], api

    run.api = api
    return run


def test_the_first_step_waits_for_its_inputs(program, capsys):
    names, _ = program()
    for n in range(2):  # each token count captures a step of its own
        names = names[names.index("cuda.Stream"):]
        first = names.index("step")
        assert "cuda.Stream().wait_stream" in names[:first]
        assert names.index("cuda.current_stream") < names.index("cuda.Stream().wait_stream") < \
            names.index("cuda.stream") < first < names.index("cuda.synchronize")
        names = names[first:]
    assert capsys.readouterr().out.count("us per step") == 2


def test_a_failed_run_is_an_error(program, capsys):
    program.api.asap_moe_status.return_value = (7, 4)
    with pytest.raises(RuntimeError, match="0x4"):
        program()
    assert "us per step" not in capsys.readouterr().out
