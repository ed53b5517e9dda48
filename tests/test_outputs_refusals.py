"""What the operators beside the decoder refuse, without a GPU: every check comes before the first HIP call, so addresses
are made up here and nothing is launched."""
import ctypes as C

import numpy as np
import pytest

from paper_2311_04996_amd import WfstError  # noqa: F401  (the package imports without a GPU)
from paper_2311_04996_amd import binding as b

OK, INVALID = 0, -1
A = 1 << 30                                       # a made-up address; arrays lie A bytes apart


@pytest.fixture(scope="module")
def lib():
    import os
    from paper_2311_04996_amd import LIB_PATH, build_library
    if not os.path.exists(LIB_PATH):
        build_library()
    return b.load_library()


def refused(lib, entry, args, word):
    assert getattr(lib, entry)(C.byref(args), None) == INVALID
    msg = lib.wfst_last_error(None).decode()
    assert msg.startswith(entry + ":") and word in msg, msg


def lin(**kw):
    d = dict(x=1 * A, w=2 * A, bias=3 * A, residual=4 * A, y=5 * A, rows=10, x_stride=64, w_stride=64, residual_stride=32, y_stride=32,
             k=64, n=32, dtype=2, bias_dtype=0, out_dtype=1, activation=2, scale=0.5)
    d.update(kw)
    return b.wfst_linear_args(**d)


@pytest.mark.parametrize("kw, word", [
    (dict(dtype=3), "type"), (dict(dtype=-1), "type"), (dict(out_dtype=7), "type"), (dict(bias_dtype=9), "type"),
    (dict(activation=4), "activation"), (dict(activation=-1), "activation"), (dict(rows=-1), "rows"), (dict(k=0), "k and n"),
    (dict(n=0), "k and n"), (dict(x=None), "null"), (dict(w=None), "null"), (dict(y=None), "null"), (dict(x_stride=-64), "stride"),
    (dict(w_stride=-1), "stride"), (dict(y_stride=31), "stride"), (dict(residual_stride=31), "stride"),
    (dict(x=A + 1), "multiple"), (dict(w=2 * A + 1), "multiple"), (dict(y=5 * A + 1), "multiple"), (dict(bias=3 * A + 2), "multiple"),
    (dict(residual=4 * A + 1), "multiple"), (dict(x_stride=1 << 60), "large"), (dict(rows=1 << 60), "large"),
    (dict(y=A + 2), "overlaps"), (dict(y=2 * A), "overlaps"), (dict(y=3 * A), "overlaps"), (dict(y=A - 2), "overlaps"),
    (dict(y=4 * A + 2), "residual"), (dict(y=4 * A, y_stride=40), "residual"),
    (dict(rows=1 << 40, x_stride=0, residual=None, y=A << 10), "too many rows"),
])
def test_linear_refuses(lib, kw, word):
    refused(lib, "wfst_linear", lin(**kw), word)


def llk(**kw):
    d = dict(x=1 * A, w=2 * A, bias=3 * A, log_prior=4 * A, lengths=5 * A, out=6 * A, x_seq_stride=640, x_stride=64, w_stride=64,
             out_seq_stride=10 * 29, out_stride=29, seqs=3, frames=10, k=64, v=29, dtype=1, bias_dtype=2, out_dtype=0)
    d.update(kw)
    return b.wfst_loglikes_args(**d)


@pytest.mark.parametrize("kw, word", [
    (dict(dtype=3), "type"), (dict(out_dtype=-2), "type"), (dict(bias_dtype=3), "type"), (dict(seqs=-1), "seqs"), (dict(frames=-1), "seqs"),
    (dict(k=0), "k >= 1"), (dict(v=0), "2048"), (dict(v=2049, out_stride=2049, out_seq_stride=20490), "2048"), (dict(x=None), "null"),
    (dict(w=None), "null"), (dict(out=None), "null"), (dict(x_stride=-1), "stride"), (dict(x_seq_stride=-1), "stride"),
    (dict(out_stride=28), "rows of out"), (dict(out_seq_stride=289), "rows of out"), (dict(out_seq_stride=0), "rows of out"),
    (dict(out_seq_stride=29, out_stride=2 * 29), "rows of out"), (dict(x=A + 1), "multiple"), (dict(out=6 * A + 2), "multiple"),
    (dict(log_prior=4 * A + 2), "multiple"), (dict(lengths=5 * A + 1), "multiple"), (dict(x_seq_stride=1 << 62), "large"),
    (dict(out=A + 4), "overlaps"), (dict(out=2 * A), "overlaps"), (dict(out=3 * A), "overlaps"), (dict(out=4 * A + 4), "overlaps"),
    (dict(out=5 * A + 4), "overlaps"),
])
def test_loglikes_refuses(lib, kw, word):
    refused(lib, "wfst_loglikes", llk(**kw), word)


def tlp(**kw):
    d = dict(scores=1 * A, tokens=2 * A, lengths=3 * A, logprobs=4 * A, lse=5 * A, entropy=6 * A, maximum=10 * A, log_sum=11 * A, top_ids=7 * A, top_logprobs=8 * A,
             workspace=9 * A, workspace_bytes=1 << 30, seq_stride=290, stride=29, seqs=3, frames=10, v=29, given=2, top=4, dtype=1)
    d.update(kw)
    return b.wfst_token_logprobs_args(**d)


@pytest.mark.parametrize("kw, word", [
    (dict(dtype=3), "type"), (dict(seqs=-1), "seqs"), (dict(frames=-1), "seqs"), (dict(v=0), "2^30"), (dict(v=(1 << 30) + 1), "2^30"),
    (dict(given=-1), "256"), (dict(given=257), "256"), (dict(top=-1), "64"), (dict(top=65), "64"), (dict(top=5, v=4), "at most v"),
    (dict(scores=None), "null"), (dict(tokens=None), "null"), (dict(stride=-1), "stride"), (dict(seq_stride=-1), "stride"),
    (dict(scores=A + 1), "multiple"), (dict(tokens=2 * A + 2), "multiple"), (dict(lse=5 * A + 2), "multiple"), (dict(top_ids=7 * A + 1), "multiple"),
    (dict(seq_stride=1 << 62), "large"), (dict(seqs=1 << 17, frames=1 << 17), "rows"),
    (dict(lse=A), "overlaps what is read"), (dict(entropy=2 * A + 4), "overlaps what is read"), (dict(logprobs=3 * A + 8), "overlaps what is read"),
    (dict(entropy=5 * A + 4), "two outputs"), (dict(maximum=6 * A), "two outputs"), (dict(log_sum=10 * A), "two outputs"), (dict(maximum=10 * A + 2), "multiple"), (dict(top_logprobs=7 * A), "two outputs"),
])
def test_token_logprobs_refuses(lib, kw, word):
    refused(lib, "wfst_token_logprobs", tlp(**kw), word)


def test_more_rows_than_a_launch_has_are_refused(lib):
    big = dict(seqs=1 << 15, frames=1 << 15, v=2, stride=0, seq_stride=0, given=0, top=0, lengths=None)      # 2^30 rows that share two scores
    refused(lib, "wfst_token_logprobs", tlp(logprobs=None, tokens=None, lse=None, entropy=A << 8, maximum=A << 9, log_sum=A << 10, **big), "too many rows")
    refused(lib, "wfst_linear", lin(rows=1 << 34, x_stride=0, residual=None, y=A << 12), "too many rows")


def test_token_logprobs_needs_its_workspace(lib):
    for rows, v, top in ((1, 128000, 8), (4, 128000, 0), (1, 1 << 30, 64), (30, 65536, 8)):
        need = lib.wfst_token_logprobs_workspace(rows, v, top)
        assert need >= 0
        if need:
            kw = dict(seqs=1, frames=rows, v=v, stride=v, top=top, given=0)
            refused(lib, "wfst_token_logprobs", tlp(workspace=None, workspace_bytes=need, **kw), "workspace")
            refused(lib, "wfst_token_logprobs", tlp(workspace_bytes=need - 1, **kw), "workspace")
            refused(lib, "wfst_token_logprobs", tlp(workspace=9 * A + 8, workspace_bytes=need, **kw), "workspace")
            refused(lib, "wfst_token_logprobs", tlp(workspace=5 * A, workspace_bytes=need, **kw), "two outputs")
    for bad in ((0, 10, 0), (-3, 10, 0), (5, 0, 0), (5, -1, 3)):
        assert lib.wfst_token_logprobs_workspace(*bad) == 0


def bwd(**kw):
    d = dict(scores=1 * A, tokens=2 * A, lengths=3 * A, maximum=4 * A, log_sum=12 * A, entropy=5 * A, top_ids=6 * A, grad_logprobs=7 * A, grad_lse=8 * A,
             grad_entropy=9 * A, grad_top=10 * A, grad_scores=11 * A, seq_stride=290, stride=29, grad_seq_stride=290, grad_stride=29,
             seqs=3, frames=10, v=29, given=2, top=4, dtype=0)
    d.update(kw)
    return b.wfst_token_logprobs_backward_args(**d)


@pytest.mark.parametrize("kw, word", [
    (dict(dtype=3), "type"), (dict(seqs=-1), "seqs"), (dict(v=0), "2^30"), (dict(given=257), "256"), (dict(top=65), "64"),
    (dict(scores=None), "null"), (dict(maximum=None), "null"), (dict(log_sum=None), "null"), (dict(grad_scores=None), "null"), (dict(tokens=None), "without tokens"),
    (dict(entropy=None), "without entropy"), (dict(top_ids=None), "without top_ids"), (dict(stride=-1), "stride"),
    (dict(grad_stride=28), "rows of grad_scores"), (dict(grad_seq_stride=100), "rows of grad_scores"), (dict(grad_scores=11 * A + 2), "multiple"),
    (dict(grad_top=10 * A + 1), "multiple"), (dict(seq_stride=1 << 62), "large"), (dict(grad_scores=A + 4), "scores without being them"),
    (dict(grad_scores=A, grad_stride=30, grad_seq_stride=300), "scores without being them"),
    (dict(grad_scores=2 * A), "overlaps what is read"), (dict(grad_scores=4 * A), "overlaps what is read"), (dict(grad_scores=12 * A - 8), "overlaps what is read"),
    (dict(grad_scores=10 * A + 8), "overlaps what is read"),
])
def test_token_logprobs_backward_refuses(lib, kw, word):
    refused(lib, "wfst_token_logprobs_backward", bwd(**kw), word)


def test_null_arguments_and_empty_calls(lib):
    for entry in ("wfst_linear", "wfst_loglikes", "wfst_token_logprobs", "wfst_token_logprobs_backward"):
        assert getattr(lib, entry)(None, None) == INVALID
        assert "null argument" in lib.wfst_last_error(None).decode()
    assert lib.wfst_linear(C.byref(lin(rows=0, x=None, y=None)), None) == OK      # nothing to do: no launch
    assert lib.wfst_loglikes(C.byref(llk(seqs=0, x=None, out=None)), None) == OK
    assert lib.wfst_loglikes(C.byref(llk(frames=0, x=None, out=None)), None) == OK
    assert lib.wfst_token_logprobs(C.byref(tlp(frames=0, scores=None, tokens=None)), None) == OK
    assert lib.wfst_token_logprobs_backward(C.byref(bwd(seqs=0, scores=None, maximum=None, grad_scores=None)), None) == OK


def test_the_message_belongs_to_the_thread_that_made_the_call(lib):
    import threading
    refused(lib, "wfst_linear", lin(k=0), "k and n")
    seen = []

    def other():
        seen.append(lib.wfst_last_error(None).decode())
        refused(lib, "wfst_loglikes", llk(v=0), "2048")

    t = threading.Thread(target=other)
    t.start()
    t.join()
    assert seen == [""]
    assert lib.wfst_last_error(None).decode().startswith("wfst_linear")


def test_argument_structs_are_laid_out_as_in_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = ("wfst_linear_args", "wfst_loglikes_args", "wfst_token_logprobs_args", "wfst_token_logprobs_backward_args")
    lines = ['#include "wfst_decoder.h"', "#include <stddef.h>", "#include <stdio.h>", "int main(void) {"]
    want = []
    for s in structs:
        t = getattr(b, s)
        lines.append(f'  printf("%zu\\n", sizeof({s}));')
        want.append(C.sizeof(t))
        for name, _ in t._fields_:
            lines.append(f'  printf("%zu\\n", offsetof({s}, {name}));')
            want.append(getattr(t, name).offset)
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text("\n".join(lines + ["  return 0;", "}"]))
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I" + os.path.join(root, "include"), str(src), "-o", str(exe)])
    assert [int(x) for x in subprocess.check_output([str(exe)]).split()] == want
    from paper_2311_04996_amd import outputs
    for s in structs:                                      # the struct as the Python functions pack it
        t = getattr(b, s)
        n = len(t._fields_)
        a = t.from_buffer_copy(outputs._packer(t).pack(*range(1, n + 1)).ljust(C.sizeof(t), b"\0"))
        assert [int(getattr(a, name)) for name, _ in t._fields_] == list(range(1, n + 1))


def test_cpu_tensors_are_refused():
    import torch
    from paper_2311_04996_amd import linear, loglikes, token_logprobs, token_logprobs_backward
    x = torch.zeros(4, 8)
    for call in (lambda: linear(x, x), lambda: loglikes(x, x), lambda: token_logprobs(x), lambda: token_logprobs_backward(x, None)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_frame_labels_of_a_path():
    from paper_2311_04996_amd.binding import LINK_DTYPE
    from paper_2311_04996_amd.lattice import Lattice
    rows = [(0, 1, 0, 11, 0.5, 0.0, 0.5, 0), (1, 2, 3, 0, 0.25, 0.75, 1.0, 1), (2, 3, 0, 12, 0.5, 0.0, 2.0, 1), (3, 4, 1, 0, 0.25, 0.5, 2.5, 2)]
    lat = Lattice(np.array([0, 2, 4, 5]), np.arange(5, dtype=np.int32), np.zeros(5, np.float32), np.array(rows, dtype=LINK_DTYPE))
    assert lat.frame_labels([0, 1, 2, 3]).tolist() == [2, 0]
    assert lat.frame_labels([0, 1]).tolist() == [2, -1]
    assert lat.frame_labels([]).tolist() == [-1, -1]
