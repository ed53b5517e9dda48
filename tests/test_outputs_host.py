"""The host side of the operators beside the decoder, without a GPU: first calls from several threads, the arguments as bytes."""
import ctypes as C
import os
import sys

import pytest

from paper_2311_04996_amd import LIB_PATH, binding, build_library, outputs


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(LIB_PATH):
        build_library()


def test_the_library_is_there_only_when_all_of_it_is(monkeypatch):
    """A second thread takes a library as the sign that the first call's preparations are over: at every line of them, either it
    is not there yet or everything else is."""
    rest = ("torch", "_codes", "_raw_stream")
    for name in ("lib", *rest):
        monkeypatch.setattr(outputs, name, None)
    early = []

    def look(frame, event, arg):
        if frame.f_code is outputs._start.__code__ and outputs.lib is not None:
            early.extend((frame.f_lineno, name) for name in rest if getattr(outputs, name) is None)
        return look if frame.f_code is outputs._start.__code__ else None

    before = sys.gettrace()
    sys.settrace(look)
    try:
        outputs._start()
    finally:
        sys.settrace(before)
    assert early == [] and outputs.lib is not None and outputs.torch is not None


@pytest.mark.parametrize("entry", ["linear", "loglikes", "token_logprobs", "token_logprobs_backward"])
def test_packed_arguments_are_a_whole_struct(entry):
    """The library is handed all of the struct, the padding behind its last field too."""
    assert outputs._packer(getattr(binding, f"wfst_{entry}_args")).size == C.sizeof(getattr(binding, f"wfst_{entry}_args"))
