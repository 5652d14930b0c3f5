"""Sizes of log probabilities from hidden states by which kernels' shapes take
them (not collected by pytest)."""

# bytes of an element, rows, vocabulary, width; an odd width goes by way of registers
SIZES = [
    (2, 5522, 16, 16), (2, 5862, 16, 17), (4, 9867, 16, 16), (4, 9401, 21, 363), (2, 66, 13854, 80),
    (2, 99, 19314, 145), (2, 2314, 1601, 80), (2, 5327, 2698, 16), (4, 35, 30611, 72), (4, 66, 32123, 480),
    (4, 68, 31086, 77), (4, 7754, 1566, 80), (4, 7440, 16, 1840), (2, 33, 25693, 448), (2, 9767, 76, 645),
    (4, 16, 665, 1576), (2, 16, 56628, 152), (2, 6502, 16, 2208), (4, 4432, 67, 1681), (2, 148, 111413, 1328),
    (4, 1216, 75166, 96), (2, 722, 111248, 448), (2, 5860, 17012, 208), (2, 1233, 78763, 232), (4, 35, 85801, 1984),
    (4, 650, 126149, 320), (4, 29, 125650, 2200), (2, 65, 77284, 2024), (2, 114, 98347, 984), (4, 91, 78116, 2048),
    (2, 6630, 15642, 136), (4, 7920, 4790, 648), (4, 16, 32768, 1024),
    # several pieces of the vocabulary, the last of another shape
    (2, 2600, 80021, 136), (4, 2500, 100003, 136),
]
# rows are summed one after the other by tiles that keep a sum in eight parts
LONG_SUM = (4, 9531, 5313, 176)


def direct(element, width):
    return width % (16 // element) == 0
