"""Shapes of group norm (images, pixels, channels, groups) for the launch paths
that large maps take, with what each has to reach: for float32 and for 16 bits,
(way forward, way forward that keeps x, way backward, sums a thread holds
forward).  The GPU tests run them; a CPU test asks the launch rule itself that
each still goes its way."""

PATHS = {
    # several images, one group a vector
    (3, 20000, 64, 8): {"f32": ("large", "large", "large", 1),
                        "16": ("large", "large", "large", 1)},
    # groups of one channel; in 16 bits the writing blocks join the parts
    (8, 40000, 16, 16): {"f32": ("large", "large", "large", 4),
                         "16": ("fold", "large", "large", 8)},
    # five channels a group: a sum a channel
    (2, 30000, 40, 8): {"f32": ("large", "large", "large", 4),
                        "16": ("large", "large", "large", 8)},
    # two and four channels a group
    (9, 30000, 32, 16): {"f32": ("large", "large", "large", 2),
                         "16": ("large", "large", "large", 4)},
    (2, 24000, 48, 12): {"f32": ("large", "large", "large", 1),
                         "16": ("large", "large", "large", 2)},
    # more images than dx's first block adds up
    (70, 6000, 24, 8): {"f32": ("large", "large", "large", 4),
                        "16": ("large", "large", "large", 8)},
    # rows of several slabs; a group over two slabs
    (1, 3000, 4096, 32): {"f32": ("large", "large", "large", 1),
                          "16": ("large", "large", "large", 1)},
    (2, 2000, 2056, 8): {"f32": ("large", "large", "large", 4),
                         "16": ("large", "large", "large", 8)},
    # odd widths of two slabs, with few parts
    (1, 450, 257, 1): {"f32": ("fold", "fold", "large", 1), "16": ("fold", "fold", "large", 1)},
    (2, 450, 511, 1): {"f32": ("fold", "fold", "large", 1), "16": ("fold", "fold", "large", 1)},
    # few parts, joined by the writing blocks, forward and both ways
    (3, 9000, 32, 4): {"f32": ("fold", "fold", "large", 1), "16": ("fold", "fold", "large", 1)},
    (2, 3000, 24, 3): {"f32": ("small", "fold", "fold", 1), "16": ("small", "small", "fold", 1)},
    (1, 3000, 24, 3): {"f32": ("small", "fold", "fold", 1), "16": ("small", "small", "fold", 1)},
}
