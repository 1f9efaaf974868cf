"""One buffer as two inputs: an output in place of the one it may replace still overlaps the other, which a call reads after it has been
written.  Refused on the host, before anything is launched; plain numbers stand for buffers."""
import ctypes

import pytest

A = [(i + 1) << 28 for i in range(24)]           # distinct 16-byte-aligned addresses, 256 MiB apart


@pytest.fixture(scope="module")
def hn():
    from paper_2607_19378_b200.build import build
    build()
    from paper_2607_19378_b200 import hyenand
    return hyenand


def refused(hn, code, word):
    assert code == hn.HYENAND_ERR_INVALID_ARG and word in hn.hyenand_last_error(), (code, hn.hyenand_last_error())


def heads(**kw):
    a = dict(dims=(6, 8), B=2, Hq=4, Hk=4, D=16, dtype=1, norm=1, axes=None, base=10000.0, eps=1e-6, q=A[0], k=A[1], g_q=None, g_k=None, positions=None)
    a.update(kw)
    dims = a.pop("dims")
    return [len(dims), (ctypes.c_int * len(dims))(*dims)] + list(a.values())


@pytest.mark.parametrize("q_out,k_out,word", [(A[0], A[7], "q_out overlaps k"), (A[7], A[0], "k_out overlaps q")], ids=str)
def test_heads_forward(hn, q_out, k_out, word):
    refused(hn, hn.lib().hyenand_heads_forward(*heads(q=A[0], k=A[0]), q_out, k_out, None), word)


@pytest.mark.parametrize("dq,dk,word", [(A[5], A[7], "dq overlaps dk_out"), (A[7], A[5], "dk overlaps dq_out")], ids=str)
def test_heads_backward(hn, dq, dk, word):
    refused(hn, hn.lib().hyenand_heads_backward(*heads(), A[5], A[5], dq, dk, None, None, None, None), word)


def test_states(hn):
    """A state's buffer as another input of the same size."""
    L = hn.lib()
    # marks of one chunk of 8 x 8 are as many floats as a state
    refused(hn, L.hyenand_delta_backward(2, 3, 3, 64, 8, 8, 1, 0, *A[:5], None, A[6], A[7], A[6], A[9], A[10], A[11], A[12], A[13], A[6], A[14], None),
            "ds0 overlaps marks")
    # keys of 16 tokens of one entry, fp32, as a state of 16 x 16
    refused(hn, L.hyenand_delta_forward(2, 1, 1, 16, 16, 16, 1, 0, A[0], A[5], *A[2:5], A[5], None, A[7], A[5], None, A[9], None), "s_end overlaps k")
    refused(hn, L.hyenand_delta_step(2, 1, 1, 16, 1, 1, 0, A[0], A[5], *A[2:5], A[5], None, A[7], A[5], None), "new_state overlaps k")
    # a recurrence's states in place of another input than the states (of one token; over states and other inputs in one buffer, element by
    # element, test_gpu_operators_memory.py has it)
    refused(hn, L.hyenand_recurrence_step(2, 3, 1, 0, A[0], A[5], *A[2:5], None, A[7], A[5], None), "new_state overlaps k")
    refused(hn, L.hyenand_recurrence_forward(2, 3, 1, 1, 0, A[5], *A[1:4], None, None, A[7], A[5], None, None, None), "s_end overlaps q")
    # dropout's key of 16 bytes as its four numbers
    refused(hn, L.hyenand_dropout(4, 0, A[0], 0.5, A[0], 0, A[0], None), "y overlaps rng")
