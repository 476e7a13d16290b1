"""Sizes for which the rule of csrc/tile_host.cu takes each width of tile, with edges
inside the tiles and an empty language, on 152 SMs: test_tile_launches_cpu.py holds
the rule to them, test_tile_shapes_gpu.py the kernels."""


def rows(T, K):
    """Bounds of K languages of T rows, uneven ones inside the tiles of 64, the second empty."""
    first = T // 3
    return [0, first] + [first + (T - first) * k // (K - 2) for k in range(K - 2)] + [T]


# T, D, F, kernel of the forward pass
FORWARD = [(515, 136, 2571, "1x128"), (1541, 136, 2571, "1x256"), (1029, 136, 4101, "1x256"),
           (2051, 520, 4101, "2x256"), (515, 1544, 6147, "2x256")]
# T, D, F, languages, kernels of the backward pass with bf16 gradients, whole and aligned
# or at odd places, and with fp32 ones
BACKWARD = [(515, 544, 515, 3, "1x64", "1x64", "1x64"), (515, 1056, 515, 3, "1x128", "1x128", "1x64"),
            (515, 2080, 515, 3, "1x256", "1x128", "1x64"), (2051, 544, 515, 3, "1x128", "1x128", "1x128"),
            (2051, 1056, 1541, 3, "2x256", "1x128", "1x128"), (2051, 2592, 515, 3, "2x256", "1x128", "1x128")]
# T, M, N, languages, the same of a linear layer's gradients
WGRAD = [(515, 515, 288, 3, "1x64", "1x64", "1x64"), (515, 515, 544, 4, "1x128", "1x128", "1x64"),
         (515, 1541, 1056, 4, "1x256", "1x128", "1x64"), (4101, 515, 544, 4, "1x128", "1x128", "1x128"),
         (3077, 1541, 3104, 3, "2x256", "1x128", "1x128"), (3077, 2051, 2592, 3, "2x256", "1x128", "1x128")]
