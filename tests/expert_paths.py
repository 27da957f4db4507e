"""Which of its three FP32 forms a mixture's experts take for given sizes, as their workspace tells: small or large tiles on FMAs, or the tensor cores."""
import ctypes as C

import paper_1802_00130_b200 as gn


def workspace(tokens, cols, inner, experts, k, backward, type=0):
    lc, lf = -(-cols // 8) * 8, -(-inner // 8) * 8
    p = lambda i: (1 << 20) + (i << 44)        # (addresses that nothing looks at)
    words = [type | 1 << 32, tokens, cols | inner << 32, experts | k << 32, p(0), p(1), p(2), p(3), lc, p(4), lc, p(5), lf, p(6), lf, p(7), lc, p(8), lc]
    for i, (rows, ld) in enumerate(((inner, lc), (inner, lc), (cols, lf)) * 2):
        words += [p(9 + i), ld, rows * ld]
    return gn.lib().gn_experts_workspace((C.c_int64 * 37)(*words), int(backward))


def path(tokens, cols, inner, experts, k, backward):
    """"small", "large" or "tensor": the one whose pieces are what the library asks for."""
    pairs, lc, lf = tokens * k, -(-cols // 8) * 8, -(-inner // 8) * 8
    few = min(pairs, experts)
    slots = -(-(pairs + 63 * few) // 64) * 64
    up = lambda n, m: -(-n // m) * m

    def plan(height):
        chunk = max(1, -(-(-(-pairs // 1024)) // 148)) * 1024
        return 4 * (2 * up(experts, 4) + up(pairs, 4) + up(slots, 4) + 4 * (pairs // height + few) + 4 + -(-pairs // chunk) * experts)

    def fma(height, width):
        pieces = [plan(height), pairs * lf * 4]
        if backward:
            pieces += [pairs * lf * 4, pairs * lf * 4, slots * -(-inner // width) * 4]
        return pieces + [pairs * lc * 4]

    tensor = [plan(256), slots * lc * 6]
    if backward:
        tensor.append(slots * lc * 6)
    tensor += [experts * inner * lc * 6] * 2 + [experts * cols * lf * 6, slots * lf * 6]
    if backward:
        tensor += [slots * lf * 6] * 2 + [slots * -(-inner // 128) * 16]
    tensor.append(pairs * lc * 4)
    sizes = {name: sum(up(n, 256) for n in pieces) + 256 for name, pieces in (("small", fma(32, 64)), ("large", fma(64, 128)), ("tensor", tensor))}
    need = workspace(tokens, cols, inner, experts, k, backward)
    found = [name for name, n in sizes.items() if n == need]
    assert found, (need, sizes)
    return " or ".join(found)


# tokens, cols, inner, experts, k
FORWARD = {
    "small": [(300, 264, 136, 6, 2), (900, 264, 136, 6, 2), (3000, 129, 65, 40, 2)],
    "large": [(700, 265, 129, 300, 1), (4000, 120, 30, 512, 4), (3000, 520, 520, 160, 1), (30000, 20, 24, 20, 2)],
    "tensor": [(700, 200, 333, 6, 3), (400, 264, 520, 3, 2), (90, 1030, 1030, 2, 2), (20000, 40, 72, 9, 2), (1003, 333, 201, 40, 3)],
}
BACKWARD = {
    "small": [(300, 264, 136, 6, 2), (900, 264, 136, 6, 2), (3000, 129, 65, 40, 2)],
    "large": [(700, 265, 129, 300, 1), (4000, 120, 30, 512, 4), (3000, 33, 130, 512, 2)],
    "tensor": [(700, 200, 333, 6, 3), (400, 264, 520, 3, 2), (90, 1030, 1030, 2, 2), (20000, 40, 72, 9, 2), (1003, 333, 201, 40, 3)],
}
