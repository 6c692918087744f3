"""The order in which the many-row linear kernel takes its steps of k and their chunks of scales, on the host (test infrastructure only)."""
STEP, CHUNK = 64, 8              # columns of a step, groups of a chunk


def chunks_of_steps(k, group, column_block, half):
    """The chunk of each step, in the order in which one half of a block's waves takes them, and the chunk asked for behind each."""
    every = -(-k // STEP)
    steps = -(-every // 2)
    first, groups, turn = half * steps, -(-k // group), column_block // 8 * 3 % steps
    chunk = lambda step: min(step * STEP // group, groups - 1) // CHUNK  # noqa: E731
    low, high = chunk(first), chunk(first + steps - 1)
    return [chunk(first + (t + turn) % steps) for t in range(steps)], lambda c: low if c == high else c + 1


def late_chunks(k, group, column_block, half, waits):
    """The steps that read a chunk whose load is still on its way: all loads have landed behind every odd step, and, with `waits`, where
    a wave enters a chunk in the step after the one that asked for it."""
    order, after = chunks_of_steps(k, group, column_block, half)
    at = [(order[0], True), (after(order[0]), True)]             # what the two places hold, and whether it has landed
    place, late, asked = 0, [], False
    for t, c in enumerate(order):
        if t % 2 == 0:
            asked = False
        if c != order[max(t - 1, 0)]:
            if asked and waits:
                at = [(chunk, True) for chunk, _ in at]
            asked = True
            place ^= 1
            at[place ^ 1] = (after(c), False)
        assert at[place][0] == c
        if not at[place][1]:
            late.append(t)
        if t % 2 == 1:
            at = [(chunk, True) for chunk, _ in at]
    return late


# (rows, columns, k, group, elements between rows of scales and zeros) of products of tiles with a chunk of one step where no barrier follows it
SHORT_CHUNKS = [(1000, 1160, 3968, 256, 0), (1000, 1160, 8000, 256, 0), (1000, 1160, 776, 32, 7), (1000, 1160, 896, 32, 4), (500, 2200, 1152, 32, 4),
                (500, 2200, 2176, 64, 6), (500, 2200, 2176, 128, 7), (500, 2200, 4224, 128, 7)]
