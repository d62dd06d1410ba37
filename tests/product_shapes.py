"""Shapes of products and the form of the kernels that each of them is to reach on a card of 256 compute units: which it does is
checked on the CPU (test_product_forms.py), what the form computes on the GPU (test_gpu_product_forms.py)."""

# (form, begins at unlike steps, experts: 0 for one matrix of all rows, rows, channels (those that gate among them), bytes of a row)
SHAPES = [
    ("stream", False, 0, 16, 300, 330),
    ("stream", False, 130, 2000, 98, 130),
    ("stream", True, 8, 30, 4100, 4002),
    ("64", False, 0, 130, 514, 330),
    ("64", False, 5, 2000, 514, 330),
    ("64", False, 130, 3000, 130, 130),
    ("64", True, 8, 100, 4100, 4002),
    ("128four", False, 0, 1010, 4002, 4002),
    ("128four", False, 5, 1500, 2050, 2002),
    ("128four", False, 8, 6000, 514, 2002),
    ("128four", True, 1, 400, 8194, 13000),
    ("128two", False, 0, 1900, 3902, 2002),
    ("128two", False, 70, 30000, 514, 650),
    ("128two", True, 8, 1000, 8200, 2002),
    ("256", False, 0, 4100, 4098, 1002),
    ("256", False, 130, 30000, 2050, 130),
    ("256", True, 8, 3000, 8200, 2002),
]

# experts, rows, channels, bytes of a row: starts that are out of order
DISORDERED = [
    ("stream", 130, 2000, 98, 130),
    ("64", 5, 2000, 514, 330),
    ("64", 130, 3000, 130, 130),
    ("128four", 5, 1500, 2050, 2002),
    ("128two", 70, 30000, 514, 650),
    ("256", 130, 30000, 2050, 130),
]
