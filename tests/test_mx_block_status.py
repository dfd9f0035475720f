"""The status of a layer and a stack: every part's word is read and cleared, whichever is set."""
import types

import pytest
import torch


class Part:
    def __init__(self, code):
        self.code, self.reads = code, 0

    def device_status(self):
        self.reads += 1
        code, self.code = self.code, 0
        return code


@pytest.mark.parametrize("codes", [(0, 0, 0), (9, 0, 0), (0, 1, 0), (9, 1, 9), (0, 1, 9)])
def test_all_parts_are_read(codes):
    from paper_2608_21614_b200.mx_block import MxAttention, MxMoEStack
    parts = [Part(c) for c in codes]
    layer = types.SimpleNamespace(qkv=parts[0], attention=parts[1], out=parts[2])
    assert MxAttention.device_status(layer) == next((c for c in codes if c), 0)
    assert MxAttention.device_status(layer) == 0 and [p.reads for p in parts] == [2, 2, 2]
    parts = [Part(c) for c in codes]
    stack = types.SimpleNamespace(layer=parts[0], head=parts[1], attention=[parts[2]])
    assert MxMoEStack.device_status(stack) == next((c for c in codes if c), 0)
    assert MxMoEStack.device_status(stack) == 0 and [p.reads for p in parts] == [2, 2, 2]
    assert MxMoEStack.device_status(types.SimpleNamespace(layer=Part(0), head=Part(7), attention=None)) == 7


@pytest.mark.gpu
def test_words_and_counters_are_cleared():
    """After a wait has run out in several parts, one call of device_status() leaves none of them and no counter of a call that did not end."""
    from paper_2608_21614_b200 import binding as B
    from paper_2608_21614_b200.mx_block import random_stack
    s = random_stack(256, 256, 8, 2, 2, 384, 4, heads=(8, 2, 64), pages=4, page_size=16)
    word = lambda t: t[:4].view(torch.int32)                                                                    # noqa: E731
    a = s.attention
    linears = [s.head, *(x for l in a for x in (l.qkv, l.out))]
    for x in linears:
        word(x.workspace).fill_(B.SAEM_ERR_TIMEOUT)
    word(a[0].attention.workspace).fill_(B.SAEM_ERR_TIMEOUT)
    a[0].attention.workspace[256:260].fill_(1)
    assert s.device_status() == B.SAEM_ERR_TIMEOUT and s.device_status() == 0
    assert all(int(word(x.workspace)) == 0 for x in linears)
    assert bool((a[0].attention.workspace[:8192] == 0).all())
    s.close()
