"""The generator of dropout's mask, with the rounds that entries are drawn with, against known answers."""
from heads_ref import threefry


def test_threefry_known_answers_of_13_rounds():
    """The published vectors of the 13-round form: of nothing but zeros, of nothing but ones, of digits of pi."""
    F = 0xFFFFFFFF
    assert threefry((0, 0), 0, 0, 13) == (0x9D1C5EC6, 0x8BD50731)
    assert threefry((F, F), F, F, 13) == (0xFD36D048, 0x2D17272C)
    assert threefry((0x13198A2E, 0x03707344), 0x243F6A88, 0x85A308D3, 13) == (0xBA3E4725, 0xF27D669E)
