"""How many waves share a row of the paged append, where a wrong line costs time and no result shows it; and the registers that the rule counts on."""
import ctypes
import struct

import pytest

from test_kernels_cpu import ELF, code_objects, sections
from test_paged_cpu import B  # noqa: F401


@pytest.fixture(scope="module")
def waves(B):  # noqa: F811
    rule = getattr(ctypes.CDLL(B.LIB_PATH), "_ZN3swa22paged_append_log_partsEbbil")
    rule.restype = ctypes.c_int
    return lambda kind, passes, rows: 1 << rule(ctypes.c_bool(kind == "f32"), ctypes.c_bool(kind == "codes"), passes, ctypes.c_int64(rows))


@pytest.mark.parametrize("kind,passes,rows,n", [
    ("16", 12, 64, 16), ("16", 12, 200, 8), ("16", 12, 400, 4), ("16", 12, 700, 4), ("16", 12, 1300, 2), ("16", 12, 2048, 2), ("16", 12, 3000, 1),
    ("16", 12, 8192, 1), ("16", 12, 16000, 1), ("16", 9, 400, 4), ("16", 9, 2048, 2), ("16", 9, 2600, 1), ("16", 20, 1800, 2), ("16", 20, 4096, 1),
    ("16", 20, 5000, 1), ("16", 20, 8100, 1), ("16", 20, 8400, 2), ("16", 20, 9000, 2), ("16", 20, 14500, 1), ("16", 20, 20000, 1),
    ("codes", 20, 3000, 2), ("codes", 20, 4096, 1), ("codes", 20, 6000, 1), ("codes", 20, 7000, 1), ("codes", 20, 7300, 2), ("codes", 20, 8191, 2),
    ("codes", 20, 8193, 2), ("codes", 20, 9000, 2), ("codes", 20, 12000, 1), ("codes", 30, 14500, 2), ("16", 20, 10000, 2), ("codes", 12, 16000, 1),
    ("f32", 12, 900, 2), ("f32", 12, 1024, 2), ("f32", 12, 2300, 1), ("f32", 20, 6000, 2), ("f32", 20, 9000, 2), ("f32", 9, 2048, 1)])
def test_as_many_waves_as_were_the_fastest_nearby(waves, kind, passes, rows, n):
    assert waves(kind, passes, rows) == n


def test_every_part_of_a_row_has_a_pass(waves):
    for kind in ("16", "codes", "f32"):
        for passes in (3, 4, 5, 9, 17, 40, 49155):
            for rows in (1, 2, 63, 1023, 8193, 1 << 24):
                assert waves(kind, passes, rows) < 2 * passes and waves(kind, passes, rows) * rows <= max(1 << 16, rows)


def test_as_many_waves_fit_as_the_rule_takes(B):  # noqa: F811
    """512 registers to a lane of a SIMD: 64 leave eight waves there (8192 on the chip), 72 seven."""
    seen = 0
    with open(B.LIB_PATH, "rb") as f:
        lib = f.read()
    for elf in code_objects(lib):
        if elf[:4] != ELF or b"swa_paged_append_kernel" not in elf:
            continue
        secs = sections(elf)
        shoff, size = struct.unpack_from("<Q", elf, 0x28)[0], struct.unpack_from("<H", elf, 0x3A)[0]
        places = [struct.unpack_from("<IIQQ", elf, shoff + i * size + 8)[2:] for i in range(len(secs))]     # address, offset
        heads = [struct.unpack_from("<IIQQQQ", elf, shoff + i * size) for i in range(len(secs))]
        assert len(places) == len(heads)
        for kind, link, data in secs:
            if kind != 2:
                continue
            for o in range(0, len(data), 24):
                name, _, _, sec, value, _ = struct.unpack_from("<IBBHQQ", data, o)
                text = secs[link][2]
                sym = text[name:text.index(b"\0", name)].decode()
                if "swa_paged_append_kernel" not in sym or not sym.endswith(".kd"):
                    continue
                _, _, _, addr, off, _ = heads[sec]
                rsrc1, = struct.unpack_from("<I", elf, off + value - addr + 48)
                registers = 8 * ((rsrc1 & 63) + 1)
                wide = "3F32" in sym
                codes = "ELb1ELb" in sym.split("ELi")[1]
                seen += 1
                assert registers <= (72 if wide or codes else 64), (sym, registers)
    assert seen == 40
