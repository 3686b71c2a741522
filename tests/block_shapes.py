"""Shapes that reach the products' large tiles, alone and with split sums: what the plan makes of
them is pinned on the CPU, what the kernels make of them is tested on the GPU."""

# rows, width, hidden: (large tiles, split sum) of the first product, of dx and of [dWg; dWu]
GATED = {
    (2048, 136, 4096): ((True, False), (False, True), (False, False)),
    (300, 4090, 2045): ((False, True), (False, True), (True, False)),
    (1100, 4104, 4100): ((True, False), (True, True), (False, False)),
    (700, 7201, 3000): ((True, True), (False, False), (True, False)),
    (7200, 6000, 350): ((False, False), (True, False), (True, True)),
}

# m, n, k: (large tiles, split sum)
BYTES = {
    (4001, 4090, 1100): (True, False),
    (4001, 4090, 300): (True, False),
    (700, 6000, 14401): (True, True),
    (333, 501, 8200): (False, True),
}
