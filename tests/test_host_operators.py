"""CPU-only checks of the length predictor's operators: what the C entry points refuse before they touch
the device, and the build of their sources.

A refused call returns before the context is used, so a zeroed block of memory stands for one."""
import ctypes as C

import pytest

INVALID, ALIGN = -1, -4
I32_MAX = 2 ** 31 - 1
MOST_ROWS = I32_MAX - 512
GOOD, ODD = 4096, 4104                          # addresses that no call reads: aligned, not aligned


@pytest.fixture(scope="module")
def lib():
    from paper_2605_16867_b200.binding import load_library
    return load_library()


@pytest.fixture(scope="module")
def ctx():
    block = C.create_string_buffer(1 << 16)
    yield C.addressof(block)


def linear(lib, ctx, n_rows, x, n_x_rows=None, row_token=None):
    return lib.gs_expert_linear(ctx, 1, x, n_rows if n_x_rows is None else n_x_rows, 64, row_token, GOOD, 1, n_rows, GOOD, 64, None, 64, 64, 0,
                                GOOD, 64, None)


def linear_backward(lib, ctx, n_rows, dz):
    return lib.gs_expert_linear_backward(ctx, 1, dz, 64, GOOD, n_rows, 64, None, GOOD, 1, n_rows, GOOD, 64, 64, 64, 0, GOOD, 64, None, 0, None,
                                         None, 0, None)


def test_products_refuse_rows_that_their_indices_cannot_reach(lib, ctx):
    # A tile of 256 rows that begins inside the last expert ends, and is rounded up, up to two tiles past its
    # end; all of that is 32-bit arithmetic.  (The unaligned address is looked at after the number of rows.)
    assert linear(lib, ctx, MOST_ROWS, ODD) == ALIGN
    assert linear_backward(lib, ctx, MOST_ROWS, ODD) == ALIGN
    for rows in (MOST_ROWS + 1, I32_MAX - 255, I32_MAX - 1, I32_MAX, I32_MAX + 1):
        assert linear(lib, ctx, rows, ODD) == INVALID
        assert linear(lib, ctx, rows, ODD, n_x_rows=5, row_token=GOOD) == INVALID
        assert linear_backward(lib, ctx, rows, ODD) == INVALID
        assert lib.gs_expert_linear_backward_workspace(ctx, 1, rows, 64, 64) == INVALID


def test_outputs_without_elements_need_no_address(lib, ctx):
    # out_dx has n_rows rows, out_dy n_rows, out_d_weight n_tokens: with none of them the tensor's address is null
    def linear_back(n_rows, dx):
        return lib.gs_expert_linear_backward(ctx, 1, GOOD, 64, GOOD, n_rows, 64, None, GOOD, 1, n_rows, GOOD, 64, 64, 64, 0, dx, 64, None, 0,
                                             None, None, 0, None)

    def combine_back(n_rows, n_tokens, dy, d_weight):
        return lib.gs_expert_combine_backward(ctx, 1, 1, GOOD, 64, GOOD, n_rows, 64, GOOD, None, n_tokens, 2, 64, 0, dy, 64, d_weight, None)
    assert linear_back(0, None) == 0
    assert linear_back(1, None) == INVALID
    assert combine_back(0, 0, None, None) == 0
    assert combine_back(5, 0, None, None) == 0
    assert combine_back(5, 1, None, None) == INVALID


def test_build_follows_a_source_that_changes(tmp_path, monkeypatch):
    """Two builds in one process with an edit between them; a forced one compiles everything once, and what no
    macro reaches once for all three libraries."""
    import os
    import shutil
    from paper_2605_16867_b200 import build
    csrc, include, compiled = tmp_path / "csrc", tmp_path / "include", []
    csrc.mkdir(), include.mkdir()
    (include / "goodserve.h").write_text("")
    for name in ("macro.cu", "plain.cu"):
        (csrc / name).write_text(f"{name} 1\n")

    def stand_in(cmd, check):
        """Compiles by copying, links by joining."""
        out = cmd[cmd.index("-o") + 1]
        if "-c" in cmd:
            source = cmd[cmd.index("-c") + 1]
            compiled.append(os.path.basename(source))
            shutil.copyfile(source, out)
        else:
            with open(out, "w") as f:
                f.write("".join(open(a).read() for a in cmd if a.endswith(".o")))
    for name, value in dict(CSRC=str(csrc), INCLUDE=str(include), OBJ_DIR=str(tmp_path / "obj"), LIB_PATH=str(tmp_path / "lib.so"),
                            COUNT_LIB_PATH=str(tmp_path / "count.so"), DEBUG_LIB_PATH=str(tmp_path / "debug.so"), SOURCES=("macro.cu", "plain.cu"),
                            MACRO_SOURCES=("macro.cu",), _ROOT=str(tmp_path), _compiled=set(), _nvcc=lambda: "nvcc").items():
        monkeypatch.setattr(build, name, value)
    monkeypatch.setattr(build.subprocess, "run", stand_in)

    def built(**how):
        compiled.clear()
        return open(build.build_library(**how)).read(), sorted(compiled)

    def edit(name, text):
        (csrc / name).write_text(text)
        later = max(p.stat().st_mtime for p in tmp_path.rglob("*")) + 5
        os.utime(csrc / name, (later, later))
    assert built(force=True) == ("macro.cu 1\nplain.cu 1\n", ["macro.cu", "plain.cu"])
    assert built(force=True, counting=True) == ("macro.cu 1\nplain.cu 1\n", ["macro.cu"])
    assert built() == ("macro.cu 1\nplain.cu 1\n", [])
    edit("plain.cu", "plain.cu 2\n")
    assert built(force=True)[0] == "macro.cu 1\nplain.cu 2\n"
    edit("macro.cu", "macro.cu 3\n")
    assert built()[0] == "macro.cu 3\nplain.cu 2\n"
    assert built(checking=True)[0] == "macro.cu 3\nplain.cu 2\n"
