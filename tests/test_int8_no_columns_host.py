"""CPU-only checks of the quantiser to 8-bit integers for operands without a column."""
P = 0x10000                                            # stands for a device address; never dereferenced on the host


def test_quantiser_refuses_and_ignores(lgn):
    """Scales at an odd address are refused before anything is enqueued; without scales there is nothing to do."""
    raw = lgn.raw()
    assert raw.lgn_int8_quantize(None, 5, 0, 0, 0, None, P + 2, None) == 1
    assert raw.lgn_int8_quantize(None, 5, 0, 0, 0, None, None, None) == 0
    assert raw.lgn_int8_quantize(None, 0, 0, 0, 0, None, None, None) == 0
