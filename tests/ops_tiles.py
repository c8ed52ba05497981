"""Which tile a product's launch takes, by the table and the rule of
paper_2609_25442_amd/csrc/linear.hip: the table is read from that source, the
rule is written out here again, and test_ops_cpu.py holds both against the
workspaces that the library asks for, which depend on the tile."""

import math
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_25442_amd", "csrc", "linear.hip")


def _pair(text):
    return [float(v.rstrip("f")) for v in text.split(",")] if text.strip() else [0.0, 0.0]


def _read():
    with open(SOURCE) as f:
        src = f.read()
    body = src[src.index("kChoices[] = {"):]
    rows = re.findall(r"\{(\d+), (\d+), (\d+), \{([^}]*)\}, ([\d.]+)f, \{([^}]*)\}, ([\d.]+)f, \{([^}]*)\}, \{([^}]*)\}\}",
                      body[:body.index("};")])
    table = [dict(bm=int(r[0]), bn=int(r[1]), resident=int(r[2]), us=_pair(r[3]), fixed=float(r[4]), few_us=_pair(r[5]),
                  few_fixed=float(r[6]), by_registers=_pair(r[7]), few_by_registers=_pair(r[8])) for r in rows]
    number = lambda name: float(re.search(name + r" = ([\d.e]+)", src).group(1))  # noqa: E731
    return table, number("kCodesUs"), number("kCopyUs"), number("kCopyBytesPerUs"), int(re.search(r"kMaxTiles = (0x[0-9a-f]+)", src).group(1), 16)


TABLE, CODES_US, COPY_US, COPY_BYTES_PER_US, MAX_TILES = _read()


def holds_scales(tile, gated):
    return (TABLE[tile]["bn"] // 2 if gated else TABLE[tile]["bn"]) % 128 == 0


def choose(rows, n, k, f8, gated=False, experts=0, residual=False, out="bf16", direct=True):
    """(expected us, tile), or None where no tile's count is one launch's."""
    n_out = n // 2 if gated else n
    stages, best = math.ceil(k * (1 if f8 else 2) / 128), None
    for i, c in enumerate(TABLE):
        if not direct and c["by_registers"][f8] == 0:
            continue
        step = c["bn"] // 2 if gated else c["bn"]
        tiles_n = -(-n_out // step)
        tiles_m = min(rows, rows // c["bm"] + min(experts, rows)) if experts else -(-rows // c["bm"])
        if tiles_m * tiles_n > MAX_TILES:
            continue
        if experts:
            tiles_m = min(float(rows), rows / c["bm"] + 0.5 * min(experts, rows))
        tiles, more = tiles_m * tiles_n, 2 if residual else 1
        full = c["us" if direct else "by_registers"][f8] * stages + c["fixed"] * more
        few = c["few_us" if direct else "few_by_registers"][f8] * stages + c["few_fixed"] * more
        rounds = math.floor(tiles / (256 * c["resident"]))
        left = tiles - rounds * 256 * c["resident"]
        us = rounds * full + (0.0 if left <= 0 else few if left <= 256 else full)
        if out == "f8e4m3" and not holds_scales(i, gated):
            us += CODES_US
        if best is None or us < best[0]:
            best = us, i
    return best


def form(rows, n, k, f8, gated=False, experts=0, residual=False, out="bf16", x_rows=None):
    """(tile, "direct", "registers" or "copied", bytes of the workspace) of a
    product whose operands are contiguous on the 16-byte grid, with or without
    a gather from x_rows rows of x."""
    es, n_out, xr = 1 if f8 else 2, n // 2 if gated else n, rows if x_rows is None else x_rows
    near = lambda ld: (n * ld < 2 ** 32 - 4096 and (256 if x_rows is None else x_rows) * ld < 2 ** 32 - 4096  # noqa: E731
                       and not (f8 and gated and n_out % 16))
    off_grid = k * es % 16 != 0
    direct = not off_grid and near(k * es)
    got = choose(rows, n, k, f8, gated, experts, residual, out, direct)
    how, size, pitch = "direct" if direct else "registers", 0, -(-k * es // 16) * 16
    if off_grid and near(pitch):
        other = choose(rows, n, pitch // es, f8, gated, experts, residual, out)
        bytes_ = (xr + n * max(1, experts)) * pitch
        if other and (got is None or other[0] + (COPY_US + bytes_ / COPY_BYTES_PER_US) < got[0]):
            got, how, size = other, "copied", bytes_
    if got is None:
        return None
    if out == "f8e4m3" and not holds_scales(got[1], gated):
        size += rows * n_out * 4
    return got[1], how, size


# Forms of a product: the activation, whether the weight is [gate; up], bias, residual, the result's type.
FORMS = [dict(out="bf16"), dict(activation="silu", gated=True, residual=True, out="f8e4m3"),
         dict(activation="gelu", bias=True, residual=True, out="f8e4m3"), dict(activation="gelu", gated=True, bias=True, out="f32")]

# (tile, fp8 operands, way) -> sizes that take it, (form, rows, rows of the weight, k, experts or 0); ragged rows and
# columns, and several steps through the ring where such a size is not too large.
SIZES = {
    (0, False, "direct"): [(0, 1, 1533, 2064, 0), (1, 1, 8212, 400, 0), (2, 1, 8193, 400, 0), (3, 16, 84, 2064, 0),
        (0, 1, 1533, 2064, 7), (1, 1, 1044, 4112, 7), (2, 7, 123, 4112, 7), (3, 16, 84, 2064, 7)],
    (0, True, "direct"): [(0, 1, 1533, 2064, 0), (1, 1, 1024, 4112, 0), (2, 7, 123, 4112, 0), (3, 16, 64, 2064, 0),
        (0, 1, 1533, 2064, 7), (1, 1, 1024, 4112, 7), (2, 7, 123, 4112, 7), (3, 16, 64, 2064, 7)],
    (1, False, "direct"): [(0, 31, 123, 784, 0), (1, 31, 84, 1040, 0), (2, 31, 123, 784, 0), (3, 31, 84, 1040, 0),
        (0, 31, 123, 784, 7), (1, 31, 84, 1040, 7), (2, 31, 123, 784, 7), (3, 31, 84, 1040, 7)],
    (1, False, "registers"): [(0, 31, 123, 777, 0), (1, 1, 4084, 777, 0), (2, 31, 123, 777, 0), (3, 1, 4084, 777, 0),
        (0, 31, 123, 777, 7), (1, 1, 4084, 777, 7), (2, 31, 123, 777, 7), (3, 1, 4084, 777, 7)],
    (1, True, "direct"): [(0, 31, 123, 784, 0), (1, 31, 64, 1040, 0), (2, 31, 123, 784, 0), (3, 31, 64, 1040, 0),
        (0, 31, 123, 784, 7), (1, 31, 64, 1040, 7), (2, 31, 123, 784, 7), (3, 31, 64, 1040, 7)],
    (1, True, "registers"): [(0, 31, 123, 777, 0), (1, 1, 4084, 777, 0), (2, 31, 123, 777, 0), (3, 1, 4084, 777, 0),
        (0, 31, 123, 777, 7), (1, 1, 4084, 777, 7), (2, 31, 123, 777, 7), (3, 1, 4084, 777, 7)],
    (2, False, "direct"): [(0, 4100, 33, 400, 0), (1, 4100, 84, 400, 0), (2, 4100, 33, 784, 0),
        (3, 31, 8212, 400, 0), (0, 31, 1023, 400, 40), (1, 31, 2068, 400, 40), (2, 16, 4097, 400, 7),
        (3, 31, 1044, 400, 40)],
    (2, True, "direct"): [(0, 4100, 33, 784, 0), (1, 31, 8224, 784, 0), (2, 4100, 33, 784, 0), (3, 31, 8224, 784, 0),
        (0, 31, 1023, 784, 40), (1, 31, 2080, 784, 40), (2, 31, 1023, 1552, 40), (3, 31, 1024, 784, 40)],
    (3, False, "direct"): [(0, 65, 12293, 400, 0), (1, 65, 8212, 400, 0), (2, 65, 8193, 400, 0),
        (3, 65, 12308, 400, 0), (0, 31, 4089, 400, 40), (1, 31, 1044, 400, 40), (2, 31, 1025, 400, 40),
        (3, 31, 4084, 400, 40)],
    (3, False, "registers"): [(0, 1, 8193, 401, 0), (1, 1, 12308, 1553, 0), (2, 1, 12293, 1553, 0),
        (3, 1, 8212, 401, 0), (0, 31, 523, 401, 40), (1, 31, 1044, 401, 40), (2, 31, 1025, 401, 40),
        (3, 31, 532, 401, 40)],
    (3, True, "direct"): [(0, 65, 12293, 784, 0), (1, 65, 8224, 784, 0), (2, 65, 8193, 784, 0),
        (3, 65, 12288, 784, 0), (0, 31, 4089, 784, 40), (1, 31, 1056, 784, 40), (2, 31, 1025, 784, 40),
        (3, 31, 4064, 784, 40)],
    (3, True, "registers"): [(0, 1, 8193, 777, 0), (1, 31, 12308, 1553, 0), (2, 31, 12293, 1553, 0),
        (3, 1, 8212, 777, 0), (0, 31, 523, 777, 40), (1, 31, 1044, 777, 40), (2, 31, 1025, 777, 40),
        (3, 31, 532, 777, 40)],
    (4, False, "direct"): [(0, 65, 8185, 400, 0), (1, 65, 8180, 400, 0), (2, 65, 8185, 400, 0),
        (3, 65, 8180, 400, 0), (0, 16, 4097, 2064, 7), (1, 16, 4116, 4112, 7), (2, 16, 4097, 4112, 7),
        (3, 16, 4116, 2064, 7)],
    (4, True, "direct"): [(0, 65, 8185, 784, 0), (1, 65, 8160, 784, 0), (2, 65, 8185, 784, 0), (3, 65, 8160, 784, 0),
        (0, 256, 2041, 784, 8), (1, 256, 2016, 784, 8), (2, 256, 2041, 784, 8), (3, 256, 2016, 784, 8)],
    (5, False, "direct"): [(0, 129, 8185, 400, 0), (1, 16, 532, 400, 0), (2, 31, 265, 400, 0),
        (3, 129, 8180, 400, 0), (0, 3001, 523, 400, 40), (1, 1, 8180, 400, 7), (2, 1, 8185, 400, 7),
        (3, 3001, 532, 400, 40)],
    (5, False, "registers"): [(0, 7, 8193, 77, 0), (1, 1, 8212, 401, 0), (2, 1, 8193, 401, 0), (3, 7, 8212, 77, 0),
        (0, 31, 523, 203, 40), (1, 31, 532, 401, 40), (2, 31, 523, 401, 40), (3, 31, 532, 203, 40)],
    (5, True, "direct"): [(0, 129, 8185, 8208, 0), (1, 7, 2048, 208, 0), (3, 129, 8160, 8208, 0),
        (0, 4100, 523, 784, 40), (1, 4100, 544, 784, 40), (2, 4100, 523, 1040, 40), (3, 4100, 544, 784, 40)],
    (5, True, "registers"): [(0, 65, 8193, 777, 0), (1, 1, 8212, 777, 0), (2, 1, 8193, 777, 0),
        (3, 65, 8212, 777, 0), (0, 31, 4097, 777, 7), (1, 31, 532, 777, 40), (2, 31, 523, 777, 40),
        (3, 31, 4116, 777, 7)],
    (6, False, "direct"): [(0, 333, 12293, 400, 0), (1, 500, 4116, 400, 0), (2, 129, 12293, 400, 0),
        (3, 333, 12308, 400, 0), (0, 128, 12293, 400, 7), (1, 31, 8212, 400, 7), (2, 31, 2063, 400, 40),
        (3, 128, 12308, 400, 7)],
    (6, False, "registers"): [(0, 129, 12293, 401, 0), (1, 129, 12308, 401, 0), (2, 129, 12293, 401, 0),
        (3, 129, 12308, 401, 0), (0, 31, 8193, 401, 7), (1, 31, 2068, 401, 40), (2, 31, 2063, 401, 40),
        (3, 31, 8212, 401, 7)],
    (6, True, "direct"): [(0, 129, 12293, 784, 0), (1, 129, 12288, 784, 0), (2, 129, 12293, 784, 0),
        (3, 129, 12288, 784, 0), (0, 31, 8193, 784, 7), (1, 31, 8224, 784, 7), (2, 31, 8193, 784, 7),
        (3, 31, 8224, 784, 7)],
    (7, False, "direct"): [(0, 400, 8185, 400, 0), (1, 400, 8180, 784, 0), (2, 400, 8185, 400, 0),
        (3, 400, 8180, 400, 0), (0, 1800, 1537, 4112, 7), (2, 31, 8193, 1040, 7), (3, 3001, 1044, 4112, 7)],
    (7, True, "direct"): [(0, 400, 8185, 784, 0), (1, 400, 8160, 784, 0), (2, 400, 8185, 784, 0),
        (3, 400, 8160, 784, 0), (0, 3001, 523, 1552, 40), (1, 3001, 544, 4112, 40), (2, 31, 8193, 4112, 7),
        (3, 3001, 544, 1552, 40)],
    (8, False, "direct"): [(0, 2049, 4089, 400, 0), (1, 2049, 4084, 400, 0), (2, 2049, 4089, 400, 0),
        (3, 2049, 4084, 400, 0), (0, 4100, 1537, 400, 40), (1, 1800, 2068, 400, 40), (2, 1800, 2063, 400, 40),
        (3, 1800, 4116, 400, 7)],
    (8, True, "direct"): [(0, 1500, 8193, 784, 0), (1, 2049, 4064, 784, 0), (2, 1500, 8193, 784, 0),
        (3, 1500, 8224, 784, 0), (0, 3001, 4089, 784, 7), (1, 1800, 4128, 784, 7), (2, 3001, 4089, 784, 7),
        (3, 3001, 4064, 784, 7)],
}


def form_of_size(f8, size):
    f, rows, n, k, experts = size
    f = FORMS[f]
    return form(rows, n, k, f8, f.get("gated", False), experts, f.get("residual", False), f["out"])
