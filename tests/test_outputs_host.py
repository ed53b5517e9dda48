"""The host side of the operators beside the decoder, without a GPU: first calls from several threads, the arguments as
bytes, the messages of failing calls, hidden states on
another GPU, numbers that no argument holds."""
import ctypes as C
import os
import sys
import threading

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


def elsewhere(call):
    """What `call` returns on a thread of its own."""
    got = []
    t = threading.Thread(target=lambda: got.append(call()))
    t.start()
    t.join()
    return got[0]


def test_a_failing_creation_is_told_on_any_thread():
    lib = binding.load_library()
    message = lambda: lib.wfst_last_error(None).decode()
    graph, opts, handle = binding.wfst_graph_csr(), binding.wfst_opts(), C.c_void_p()
    create = lambda: lib.wfst_decoder_create(C.byref(graph), C.byref(opts), C.byref(handle))      # all of them 0: refused before any GPU call
    refuse = lambda: lib.wfst_linear(C.byref(binding.wfst_linear_args()), None)

    assert elsewhere(create) == -1
    assert "max_channels" in message() and "max_channels" in message() and "max_channels" in elsewhere(message)
    # a call without a decoder: on its own thread only, and what a creation of another thread says does not come before it is read
    assert refuse() == -1 and elsewhere(message) == ""
    opts.max_channels = opts.max_frames_per_channel = opts.max_words = 1
    opts.loglike_dtype = 9
    assert elsewhere(create) == -1
    assert message().startswith("wfst_linear:") and "loglike_dtype" in message() and "loglike_dtype" in elsewhere(message)
    # a creation's own thread keeps its message, whatever fails elsewhere
    assert create() == -1 and elsewhere(refuse) == -1
    assert "loglike_dtype" in message() and elsewhere(message) == ""


def test_hidden_states_on_another_gpu_than_the_current_one_are_refused(monkeypatch):
    """The decoder runs on the current GPU's stream, which does not wait for one of another GPU."""
    import torch
    decoder = object.__new__(binding.Decoder)
    decoder.V, decoder.loglike_dtype = 29, "float32"

    class Elsewhere:                                       # a tensor on cuda:1
        is_cuda, shape, device = True, (2, 5, 8), "cuda:1"
        dim = staticmethod(lambda: 3)
        get_device = staticmethod(lambda: 1)

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for call in (lambda: decoder.decode_hidden(Elsewhere(), [5, 5], torch.zeros(29, 8), None, 10.0, 100),
                 lambda: decoder.advance_hidden_partial([0, 1], Elsewhere(), [5, 5], torch.zeros(29, 8), None)):
        with pytest.raises(ValueError, match="cuda:1"):
            call()


@pytest.mark.parametrize("where,value", [(10, 1 << 31), (10, -(1 << 31) - 1), (5, 1 << 63), (16, "1")])
def test_numbers_that_an_argument_does_not_hold_raise_value_error(where, value):
    fields = [0] * 17
    fields[where] = value
    with pytest.raises(ValueError, match="out of range"):
        outputs._run(None, outputs._linear, fields, 0, None)


def test_too_many_top_ones_are_refused_before_their_results_are_made(monkeypatch):
    """2^40 of them for a few rows would be more memory than there is."""
    import torch
    outputs._start()

    def make(*a, **kw):
        raise AssertionError("allocated")

    monkeypatch.setattr(outputs, "_new", make)
    for top in (1 << 40, 65, 9, -1):
        with pytest.raises(binding.WfstError, match="top must be"):
            outputs._token_logprobs(torch.zeros(4, 8), None, top, None, None)
