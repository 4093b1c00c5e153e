"""What the bindings take for an address: None, any int, or a tensor (host)."""
import enum

import torch

from paper_2608_13966_gb300 import quasar as Q


class Buffer(enum.IntEnum):
    LOGITS = 0x10000000


class Address(int):
    pass


def test_addresses():
    t = torch.zeros(4)
    assert Q._ptr(None) is None and Q._ptr(t) == t.data_ptr()
    for x in (0, 0x10000000, True, Buffer.LOGITS, Address(77)):
        assert Q._ptr(x) == int(x)


def test_a_call_takes_them():
    """An invalid row stride is refused on the host: the address got that far."""
    st = Q.quasar_top_logits(Buffer.LOGITS, Q.F32, 9, 4, 10, 2, 1.0, Address(0x20000000),
                             Address(0x30000000), None, stream=0)
    assert st == Q.QuasarStatus.ERR_INVALID_ARG
