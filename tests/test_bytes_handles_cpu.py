"""Handles of a cache held in 8 bits, without a GPU: the workspace that they take, and what calls beyond it get."""

import ctypes

import pytest
import torch

import paper_2609_08131_gb300 as J
from paper_2609_08131_gb300 import api
from test_operators_cpu import BAD, P, PASSED, passed, refused

ZEROED = J.JACAP_ATTEND_ZERO_BYTES


def empty(tokens=64, S=16, Hq=32, Hkv=8, n=2176):
    return api.Cache8.empty(S, 1, Hq, Hkv, n, device="cpu", tokens=tokens)


def test_the_workspace_is_that_of_the_queries_asked_for():
    few, many = empty(1), empty()
    assert few.tokens == 1 and few.ws.numel() == J.jacap_bytes_workspace(few._cache, 1)
    assert many.tokens == 64 and many.ws.numel() == J.jacap_bytes_workspace(many._cache, 64)
    assert few.ws.numel() < 2 << 20 and many.ws.numel() < 11 << 20
    for part, tokens in ((few.part(), 1), (many.part(tokens=2), 2), (many.part(slots=slice(0, 1)), 64)):
        assert part.tokens == tokens and part.ws.numel() == J.jacap_bytes_workspace(part._cache, tokens)
    # what starts at zero, as a first call finds it
    assert not few.ws[:ZEROED + 4 * few.S].any() and few.ws.numel() >= ZEROED + 4 * few.S


def test_more_queries_than_the_workspace_is_for():
    c = empty(4, S=2, Hq=4, Hkv=2, n=128)
    with pytest.raises(api.JacapError) as e:
        c.attend(torch.zeros(2, 1, 4, 5, 128, dtype=torch.bfloat16))
    assert e.value.status == J.JACAP_ERR_WORKSPACE


@pytest.mark.parametrize("tokens,status", [(0, 1), (-1, 1), (65, 2)])
def test_numbers_of_queries_that_no_workspace_has(tokens, status):
    with pytest.raises(api.JacapError) as e:
        empty(tokens, S=1, n=64)
    assert e.value.status == status


def store(rows, k, v):
    c = empty(S=2, Hq=4, Hkv=2, n=128)
    strides = (ctypes.c_int64 * 8)(*[512 * 128, 512 * 128, 256 * 128, 128] * 2)
    return J.jacap_bytes_store(c._cache, J.JACAP_BF16, k, v, strides, rows, P, P, P, 1 << 20, None)


@PASSED
def test_no_rows_have_no_address():
    passed(store(0, None, None))


@pytest.mark.parametrize("k,v", [(None, P), (P, None)])
def test_rows_have_one(k, v):
    refused(store(1, k, v), BAD)
