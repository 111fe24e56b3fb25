"""Calls of the linear layers that between them take every kernel the library holds, each with the kernel that it has to take."""
from __future__ import annotations

import numpy as np

import paper_1802_10280_amd as esc

# How inputs lie: rows on 16 bytes, or two elements further.
WIDE, ANY = 0, 2

# Whole weights: type of 4 or 2 bytes, how inputs lie, K, weight rows, T, and the kernel's (rows, tokens, steps, step_bytes).  Some ten steps along K or
# more, the last of them not whole; last blocks of rows and tokens that are not whole.
MANY = [(size, place, 520 if place == WIDE else 509, rows, T, kernel) for size, place, rows, T, kernel in [
    (2, WIDE, 300, 301, (64, 32, 3, 256)), (2, WIDE, 16468, 27, (64, 32, 4, 128)), (2, WIDE, 1980, 300, (64, 64, 3, 256)),
    (2, WIDE, 4076, 300, (64, 64, 3, 128)), (2, WIDE, 4076, 1000, (128, 128, 4, 128)), (2, WIDE, 2420, 3311, (128, 128, 2, 128)),
    (2, WIDE, 4076, 2041, (256, 128, 3, 128)), (2, WIDE, 8148, 2041, (256, 256, 2, 128)),
    (2, ANY, 300, 301, (64, 32, 3, 256)), (2, ANY, 16468, 27, (64, 32, 4, 128)), (2, ANY, 1980, 300, (64, 64, 3, 256)),
    (2, ANY, 4076, 300, (64, 64, 3, 128)), (2, ANY, 4076, 1000, (128, 128, 4, 128)),
    (4, WIDE, 1500, 100, (64, 32, 3, 256)), (4, WIDE, 2036, 600, (64, 32, 4, 128)), (4, WIDE, 2036, 2041, (128, 128, 2, 128)),
    (4, ANY, 1500, 100, (64, 32, 3, 256)), (4, ANY, 2036, 600, (64, 32, 4, 128)), (4, ANY, 2036, 2041, (128, 128, 4, 128))]]

# Kept weights: the kernel's (inputs, tokens) and K, weight rows and T that take it; each with every number of pieces.
FEW = [(size, place, K, rows, T, kernel) for size, place, K, rows, T, kernel in [
    (2, WIDE, 776, 300, 3, (1, 16)), (2, WIDE, 776, 300, 13, (2, 16)), (2, WIDE, 1032, 2124, 29, (2, 32)), (2, WIDE, 2328, 522, 239, (2, 64)),
    (2, ANY, 771, 300, 13, (0, 16)), (2, ANY, 1029, 2124, 29, (0, 32)),
    (4, WIDE, 772, 300, 3, (1, 16)), (4, WIDE, 772, 300, 13, (2, 16)), (4, WIDE, 772, 2124, 29, (2, 32)),
    (4, ANY, 771, 300, 13, (0, 16)), (4, ANY, 773, 2124, 29, (0, 32))]]
# The share of zeros at which a lane's values (a word each in fp32, two to a word in 16 bits) are so many pieces of 16 bytes at the most.
PIECES = {2: {1: 0.97, 2: 0.87, 3: 0.67, 4: 0.35, 5: 0.01}, 4: {1: 0.995, 2: 0.96, 3: 0.9, 4: 0.84, 5: 0.78, 8: 0.4}}

TYPES = {2: (1, 2), 4: (0,)}


def kernel_of(layer_desc, plan, T, place):
    """What the library tells of a call of T tokens whose rows lie so."""
    d = layer_desc
    size = 4 if d.type == 0 else 2
    return esc.escoin_linear_kernel(esc.make_linear_desc(T, d.K, d.M, d.type, d.gated), plan, place * size)


def named(k, type, gated):
    """The kernel's name without its namespace."""
    gated = "true" if gated else "false"
    if k["kept"]:
        return f"linear_few_kernel<{type}, {gated}, {k['inputs']}, {k['tokens'] // 16}, {k['pieces']}>"
    return (f"linear_many_kernel<{type}, {gated}, {'true' if k['inputs'] == 2 else 'false'}, {k['rows']}, {k['tokens']}, {k['waves']} waves, "
            f"{k['steps']}, {k['step_bytes'] // 32}>")


def header_with(plan, **fields):
    """The header of a plan with other fields: the host reads no more of it."""
    from paper_1802_10280_amd import binding
    h = binding._LinearHeader.from_buffer_copy(plan[:256].tobytes())
    for k, v in fields.items():
        setattr(h, k, v)
    return np.frombuffer(bytes(h), dtype=np.uint8)
