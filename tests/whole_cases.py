"""Cases of the residual step's gradients in whole numbers (oracle/train.py, whole_step):
(rows, columns, tokens of a frame), for every width of a team and every way that the sums
over rows are added."""

ALL = ("gate", "scale", "shift", "weight", "bias", "post_weight")
NAMES = [ALL, ("gate", "scale", "shift"), ("scale", "shift", "weight"), ("gate", "bias"),
         ("post_weight",), ("weight", "bias")]

SHAPES = [(1, 8, 1), (3, 128, 2), (17, 136, 4), (50, 512, 7), (33, 520, 0), (9, 1024, 3),
          (70, 1536, 32), (5, 2048, 5), (6, 2056, 4), (7, 5120, 3), (4, 8192, 2), (3, 8200, 2),
          (2, 16384, 1), (40, 16000, 15), (11, 72, 3), (300, 64, 100), (1000, 256, 130),
          # one frame, or a few, of many rows
          (1, 1536, 0), (191, 1536, 0), (192, 1536, 0), (400, 1536, 300), (1000, 520, 0),
          (900, 2056, 400), (5000, 128, 0), (9000, 64, 4100), (300, 5120, 0), (420, 9000, 0),
          (2000, 520, 450), (40000, 128, 0), (30000, 64, 29000),
          # many frames of few rows
          (3200, 128, 16), (4001, 136, 21), (800, 1536, 4), (191, 520, 1), (192, 520, 1),
          (200, 9000, 1), (7000, 64, 7), (200, 128, 1), (2100, 640, 2), (33, 16000, 1),
          (30000, 64, 2), (12345, 72, 40)]

# Rows of every width of a team, and of columns that leave threads or waves without any.
WIDTHS = [8, 72, 128, 136, 256, 264, 512, 520, 1024, 1536, 2056, 5120, 6144, 6152, 8192, 8200, 16000,
          16384]
