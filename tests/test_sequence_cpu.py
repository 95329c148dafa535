"""Operators of a sequence without a GPU: the generator's published vectors, and refusals of the C entry
points that protect memory."""
import ctypes

import numpy as np
import pytest

from tests import sequence_reference as ref
from paper_2607_11985_gb300 import binding as B


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2607_11985_gb300 import build
    build.build()


A = 1 << 20    # an address that is never read: every call below is refused


def heads(data=A, batch=1024, token=64, head=8):
    return ctypes.byref(B.vqc_heads(data, batch, token, head))


def test_philox_of_the_published_vectors():
    """Known answers of the method's authors: counters and keys of zeros, and of ones."""
    assert [int(w) for w in ref.philox(np.zeros(1, np.uint64), 0, 0)[0]] == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    ones = 2 ** 64 - 1
    assert [int(w) for w in ref.philox(np.array([ones], np.uint64), ones, ones)[0]] == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


def refused(call, args, changes, status="VQC_ERR_INVALID_ARG"):
    for at, value in changes:
        given = list(args)
        given[at] = value
        with pytest.raises(B.VQCError, match=call.__name__) as e:
            call(*given)
        assert B.STATUS[e.value.status] == status, (call.__name__, at, value)


def test_dropout_refusals():
    args = [B.VQC_BF16, 4, 8, A, 8, A, 8, 0.5, 1, 2, None, A, None]
    refused(B.vqc_dropout_forward, args, [(0, 3), (1, -1), (2, 0), (3, None), (4, 7), (6, 7), (7, 1.0), (7, float("nan")), (11, None), (3, A + 1),
                                          (5, A + 1), (10, A + 4), (11, A + 8), (1, 1 << 60)])
    refused(B.vqc_dropout_backward, [B.VQC_F32, 4, 8, A, 8, 0.5, 1, 2, None, A, None], [(3, A + 2), (4, 7), (5, -0.5), (9, A + 4)])


def test_norm_rotary_refusals():
    args = [B.VQC_F16, 2, 3, 4, 2, 8, heads(), heads(), A, A, A, 4, A, 3, 1e-6, A, A, None]
    refused(B.vqc_norm_rotary_forward, args, [(0, 5), (1, -1), (2, 1 << 30), (3, 0), (3, 1 << 17), (4, 0), (5, 0), (5, 257), (6, None), (6, heads(A + 1)),
                                              (7, heads(batch=-1)), (8, A + 1), (10, None), (10, A + 4), (11, 5), (11, -1), (12, A + 2), (13, -1),
                                              (14, -1.0), (15, None), (16, A + 8)])
    args = [B.VQC_F16, 2, 3, 4, 2, 8, heads(), heads(), heads(), heads(), A, A, A, 4, A, 3, 1e-6, A, A, A, A, A, 1 << 30, None]
    refused(B.vqc_norm_rotary_backward, args, [(6, None), (7, heads(A + 1)), (17, None), (18, A + 8), (19, A + 1), (21, A + 128)])
    refused(B.vqc_norm_rotary_backward, args, [(21, None), (22, 16)], "VQC_ERR_WORKSPACE")
    args = [B.VQC_F16, 2, 3, 4, 2, 8, 9, heads(), heads(), heads(), A, A, A, 4, 1e-6, A, A, heads(), heads(), None]
    refused(B.vqc_norm_rotary_step, args, [(6, -1), (6, 1 << 30), (9, None), (15, None), (15, A + 2), (16, A + 2), (17, heads(None)), (18, heads(token=-1))])
    assert B.vqc_norm_rotary_workspace_bytes(2, 3, 4, 2, 300) == 2 ** 64 - 1
    assert 0 < B.vqc_norm_rotary_workspace_bytes(2, 3, 4, 2, 64) < 1 << 20


def test_attention_refusals():
    args = [B.VQC_BF16, 2, 3, 4, 2, 8, heads(), heads(), heads(), 0, 0, 0.5, A, A, A, A, 1 << 30, None]
    refused(B.vqc_attention_forward, args, [(0, -1), (1, 1 << 31), (2, -1), (3, 3), (4, 0), (5, 0), (5, 257), (6, heads(None)), (7, heads(A + 1)),
                                            (8, heads(head=-8)), (9, -1), (10, -1), (11, 0.0), (11, -1.0), (11, float("inf")), (11, 1e-45), (12, A + 2),
                                            (13, None), (13, A + 8), (14, A + 2), (15, A + 16)])
    args = [B.VQC_F32, 2, 3, 4, 2, 8, heads(), heads(), heads(), heads(), A, A, 0, 0, 0.5, None, A, A, A, A, 1 << 30, None]
    refused(B.vqc_attention_backward, args, [(6, heads(None)), (10, None), (10, A + 8), (11, None), (12, -1), (14, 0.0), (17, None), (18, A + 4), (19, A + 1)])
    refused(B.vqc_attention_backward, args, [(19, None), (20, 16)], "VQC_ERR_WORKSPACE")
    args = [B.VQC_F32, 2, 1, 4, 2, 8, 5000, heads(), heads(), heads(), 0, 0, 0.5, A, A, A, 1 << 30, None]
    refused(B.vqc_attention_step, args, [(0, 7), (3, 3), (5, 257), (6, -1), (6, 1 << 30), (7, heads(None)), (8, heads(A + 2)), (9, None), (10, -1), (11, -1),
                                         (12, float("nan")), (13, None), (13, A + 1), (14, None), (15, A + 2)])
    refused(B.vqc_attention_step, args, [(15, None), (16, 16)], "VQC_ERR_WORKSPACE")
    assert B.vqc_attention_workspace_bytes(2, B.VQC_F32, 2, 3, 4, 2, 8, 0, 0, 1) == 2 ** 64 - 1
    assert B.vqc_attention_workspace_bytes(0, B.VQC_F32, 2, 3, 4, 3, 8, 0, 0, 1) == 2 ** 64 - 1
    assert B.vqc_attention_step_workspace_bytes(1, 1, 4, 2, 8, -1, 0, 0) == 2 ** 64 - 1
    # no more than a window's keys are cut, whatever the capacity
    assert B.vqc_attention_step_workspace_bytes(1, 1, 4, 2, 64, 1 << 29, 64, 0) < 1 << 20
