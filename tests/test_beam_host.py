"""Decoding several continuations, on the host: the binding's structures have the C layout, groups hold what they are given, and calls
that need no GPU to be refused are."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2609_26100_gb300 import build, native, paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    build.build()
    return native.lib()


def test_structures_have_the_c_layout(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    structs = {"tss_paged_groups": native.TssPagedGroups, "tss_beam_args": native.TssBeamArgs, "tss_paged_batch": native.TssPagedBatch,
               "tss_paged_cache": native.TssPagedCache, "tss_paged_attn": native.TssPagedAttn, "tss_rope_args": native.TssRopeArgs,
               "tss_page_tables": native.TssPageTables}
    lines = ["#include \"tss.h\"", "#include <stdio.h>", "#include <stddef.h>", "int main(void) {"]
    for name, py in structs.items():
        lines.append(f'  printf("%zu\\n", sizeof({name}));')
        lines += [f'  printf("%zu\\n", offsetof({name}, {field}));' for field, _ in py._fields_]
    (tmp_path / "x.c").write_text("\n".join(lines + ["  return 0;", "}"]))
    subprocess.run([cc, "-std=c99", "-I", os.path.join(ROOT, "include"), str(tmp_path / "x.c"), "-o", str(tmp_path / "x")], check=True)
    got = iter(subprocess.run([str(tmp_path / "x")], capture_output=True, text=True, check=True).stdout.split())
    for name, py in structs.items():
        assert int(next(got)) == ctypes.sizeof(py), name
        for field, _ in py._fields_:
            assert int(next(got)) == getattr(py, field).offset, (name, field)


def test_what_groups_hold():
    g = paged.Kv4Cache.groups([2, 1], (2 ** 31 - 1, torch.tensor(7)))
    assert g.n_groups == 2
    assert [list((ctypes.c_int32 * 2).from_address(x)) for x in (g.n_req, g.shared)] == [[2, 1], [2 ** 31 - 1, 7]]
    with pytest.raises(ValueError):
        paged.Kv4Cache.groups([1, 2], [3])
    for big in (2 ** 31, -2 ** 31 - 1, 2 ** 64):
        with pytest.raises(OverflowError):
            paged.Kv4Cache.groups([1], [big])


def test_null_arguments(lib):
    a = native.TssBeamArgs()
    for s in (lib.tss_beam_select(None, ctypes.byref(a), None), lib.tss_beam_create(1, 1, 1, None), lib.tss_beam_sync_status(None, None),
              lib.tss_paged_append_rope(None, None, 0, None, None, None, 0, None),
              lib.tss_paged_attention_shared(None, None, 0, None, None, None, None),
              lib.tss_pages_reorder(None, None, None, 1, 16, 0, None, None, None, None, None),
              lib.tss_paged_create_shared(2, 2, 64, 0, None)):
        assert s == native.TSS_ERR_INVALID_ARG
    lib.tss_beam_destroy(None)  # a no-op


@pytest.mark.parametrize("rows,vocab,keep", [(0, 5, 1), (-1, 5, 1), (2 ** 20 + 1, 5, 1), (1, 0, 1), (1, 2 ** 24 + 1, 1), (1, 5, 0), (1, 5, 129)])
def test_sizes_of_a_selector(lib, rows, vocab, keep):
    out = ctypes.c_void_p(1)
    assert lib.tss_beam_create(rows, vocab, keep, ctypes.byref(out)) == native.TSS_ERR_INVALID_ARG and not out.value


@pytest.mark.parametrize("rows", [-1, 8193])
def test_room_for_shared_rows(lib, rows):
    out = ctypes.c_void_p(1)
    assert lib.tss_paged_create_shared(4, 2, 128, rows, ctypes.byref(out)) == native.TSS_ERR_INVALID_ARG and not out.value
