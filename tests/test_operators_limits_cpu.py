"""What the gate and the experts' operators refuse at the limits of their ranges, without a GPU."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def ep():
    from paper_2603_13606_amd import binding, build
    if not build.is_current():
        build.build()
    binding.load()
    return binding


class OnGpu:
    """Looks like a tensor of a GPU to the check of devices."""
    is_cuda, device = True, torch.device("cuda", 0)


def test_tensors_in_host_memory_among_those_of_a_gpu_are_refused(ep, monkeypatch):
    """A kernel that is handed their address would fault.  Pinned memory and empty tensors pass, and so do calls on the host alone
    (whose descriptors are checked before anything is launched)."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    host, empty = torch.zeros(4, dtype=torch.int32), torch.zeros(0, dtype=torch.int32)
    with pytest.raises(ValueError):
        ep._one_device([OnGpu(), host])
    with pytest.raises(ValueError):
        ep._one_device([host, OnGpu(), OnGpu()])
    pinned = type("Pinned", (), dict(is_cuda=False, device=torch.device("cpu"), numel=lambda self: 4, is_pinned=lambda self: True))()
    assert ep._one_device([OnGpu(), empty, pinned]) == 0
    assert ep._one_device([host, empty]) is None


@pytest.mark.parametrize("padded", [False, True])
def test_more_rows_than_blocks_can_count_are_refused(ep, padded):
    """Rounded up to blocks of 256 rows their number has to stay below 2^31.  (The descriptors are all there is: nothing of that
    size is allocated, and a call that passed the checks would fail for want of a GPU.)"""
    if torch.cuda.is_available():
        pytest.skip("the call would be made")
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)    # noqa: E731
    rows = bf(1, 4, 8) if padded else bf(4, 8)
    ins = [(rows, ep.EP_TAG_TOKENS), (bf(1, 8, 8), ep.EP_TAG_EXPERT_WEIGHTS), (i32(1), ep.EP_TAG_ROW_COUNT)] + [(i32(1), ep.EP_TAG_ROW_OFFSET)] * (not padded)
    cfg = ep._product_config(ep.EP_ACT_NONE, False)

    def call(n):
        x, out = (ep.tensor_desc(rows, ep.EP_TAG_TOKENS) for _ in range(2))
        x.shape[int(padded)] = out.shape[int(padded)] = n
        descs = (ep.ep_tensor_t * len(ins))(x, *[ep.tensor_desc(t, tag) for t, tag in ins[1:]])
        return ep.load().ep_expert_product(None, ctypes.byref(cfg), descs, len(ins), (ep.ep_tensor_t * 1)(out), 1, None)
    assert call(2 ** 31 - 1) == call(2 ** 31 - 255) == ep.EP_ERR_INVALID_ARG
    assert call(2 ** 31 - 256) != ep.EP_ERR_INVALID_ARG


def test_numbers_of_tokens_that_overflow_are_refused(ep):
    """2^61 tokens of 8 entries are 2^64, which is 0 in 64 bits; the call seemed to have worked."""
    ls, idx, w = torch.zeros(4, 16), torch.zeros((4, 8), dtype=torch.int32), torch.zeros(4, 8)

    def desc(t, tag, n):
        d = ep.tensor_desc(t, tag)
        d.shape[0] = n
        return d
    for n in (2 ** 61, 2 ** 25 + 1):
        l, i, g = desc(ls, ep.EP_TAG_LOGITS, n), desc(idx, ep.EP_TAG_TOPK_IDX, n), desc(w, ep.EP_TAG_TOPK_WEIGHTS, n)
        cfg, lib, arr = ep._route_config(ep.EP_SCORE_SOFTMAX, True, 1, 1, 1.0), ep.load(), ep.ep_tensor_t
        assert lib.ep_route(ctypes.byref(cfg), (arr * 1)(l), 1, (arr * 2)(i, g), 2, None) == ep.EP_ERR_INVALID_ARG
        assert lib.ep_route_backward(ctypes.byref(cfg), (arr * 3)(l, i, g), 3, (arr * 1)(l), 1, None) == ep.EP_ERR_INVALID_ARG
