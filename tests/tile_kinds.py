"""Which tiles csrc/moe_tiles.h's kind_of takes, for tests that have to reach one of them: a copy of its rule, so that a case whose kind changes says so.

M rows, E groups, cols columns of results (forward: of gate and up together; the gradient: hidden features), depth places of the sum."""


def kind_of(M, E, cols, depth):
    each, chunks = M // E, (depth + 63) // 64
    if each >= 192 and M // 256 * ((cols + 255) // 256) * chunks >= 12288:
        return "big"
    return "mid" if each > 64 and (M + 127) // 128 * ((cols + 127) // 128) >= 256 else "few"
