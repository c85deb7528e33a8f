"""The paged store on the CPU: its host bookkeeping against plain lists (a C++
program), and what the entry points refuse without a GPU."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2608_23553_amd import ChimeraError, Index, Pages, chimera

HERE = os.path.dirname(os.path.abspath(__file__))


def test_bookkeeping_against_plain_lists(tmp_path):
    exe = str(tmp_path / "check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-D_GLIBCXX_ASSERTIONS", "-Wall", "-o", exe,
                           os.path.join(HERE, "pages_book_check.cpp")])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout


def test_null_arguments_are_rejected_without_gpu():
    L, bad = chimera.lib(), chimera.E_INVAL
    one, len1 = (ctypes.c_int64 * 1)(0), (ctypes.c_int32 * 1)(1)
    assert L.chimera_pages_create(0, 1, 1, 1, None) == bad
    assert L.chimera_pages_info_get(None, None) == bad
    assert L.chimera_pages_lengths(None, one, 1, len1, None) == bad
    assert L.chimera_pages_append(None, one, len1, 1, None, 0, 128, 128, 0, None) == bad
    assert L.chimera_pages_fork(None, one, one, len1, 1, None) == bad
    assert L.chimera_pages_copy(None, one, None, one, len1, None, 1, None) == bad
    assert L.chimera_pages_drop(None, one, 1, None) == bad
    assert L.chimera_pages_read(None, one, 1, None, 0, 0, None) == bad
    assert L.chimera_pages_score(None, None, 0, 1, 32, 128, None, 1, 0, None, None) == bad
    assert L.chimera_search_pages(None, None, None, 0, 1, 32, 128, 2, 256, 10, None, None, None) == bad
    assert b"null index" in L.chimera_last_error()
    L.chimera_pages_free(None)


@pytest.mark.parametrize("npages,ndocs,max_len,code", [
    (0, 1, 1, chimera.E_INVAL), (1, 0, 1, chimera.E_INVAL), (1, 1, 0, chimera.E_INVAL), (-1, 1, 1, chimera.E_INVAL),
    (252_645_136, 1, 1, chimera.E_UNSUPPORTED), (1, 2**31, 1, chimera.E_UNSUPPORTED),
    (1, 1, 2**20 + 1, chimera.E_UNSUPPORTED)])
def test_sizes_that_a_store_cannot_have(npages, ndocs, max_len, code):
    with pytest.raises(ChimeraError) as e:
        Pages(npages, ndocs, max_len)
    assert e.value.code == code


@pytest.mark.parametrize("bad", [[1.5], np.array([0.0, 1.0])])
def test_ids_and_lengths_are_whole_numbers(bad):
    with pytest.raises(ValueError):
        chimera._ids(bad)
    with pytest.raises(ValueError):
        chimera._counts(bad, len(bad), "lens")
    with pytest.raises(ValueError):
        chimera._counts([2**31], 1, "lens")
    with pytest.raises(ValueError):
        chimera._counts([1, 2], 1, "lens")
    assert chimera._ids([]).dtype == np.int64 and chimera._counts([], 0, "lens").dtype == np.int32


def test_lengths_of_a_copy_are_checked_before_its_positions_are_read(tmp_path):
    exe = str(tmp_path / "lengths")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-D_GLIBCXX_ASSERTIONS", "-Wall", "-o", exe,
                           os.path.join(HERE, "pages_copy_lengths.cpp")])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout


def test_read_all_refuses_null_arguments_without_gpu():
    L, one, total = chimera.lib(), (ctypes.c_int64 * 1)(0), ctypes.c_int64(7)
    assert L.chimera_pages_read_all(None, one, 1, None, -1, chimera.BF16, ctypes.byref(total), None) == chimera.E_INVAL
    assert L.chimera_pages_read_all(None, one, 1, None, -1, chimera.BF16, None, None) == chimera.E_INVAL
    assert total.value == 7


@pytest.mark.parametrize("npages,ndocs,max_len,device", [
    (2**64 + 1, 1, 1, 0), (1, 2**64 + 1, 1, 0), (1, 1, 2**32 + 1, 0), (1, 1, 1, 2**32), (1, 1, -2**32 + 1, 0),
    (2**63, 1, 1, 0), (1, 1, 2**31, 0)])
def test_sizes_that_the_library_cannot_be_told(npages, ndocs, max_len, device):
    """Not taken for what is left of them in 32 or 64 bits."""
    with pytest.raises(ValueError):
        Pages(npages, ndocs, max_len, device)
    with pytest.raises(TypeError):
        Pages(1.5, 1, 1)


@pytest.mark.parametrize("nprobe,ncand,k", [(2**32 + 2, 256, 10), (2, 2**32 + 256, 10), (2, 256, 2**32 + 10),
                                            (2, 256, 2**31), (2, 256, -2**32 + 10)])
def test_a_search_from_pages_with_sizes_that_the_library_cannot_be_told(nprobe, ncand, k):
    with pytest.raises(ValueError, match="32 bits"):
        Index.search_pages(Index.__new__(Index), None, None, nprobe, ncand, k)
