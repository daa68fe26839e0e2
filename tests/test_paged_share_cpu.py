"""Blocks held together, without a GPU: the plain model against hand-worked steps, what the library refuses before it touches a GPU,
the binding's marshalling, and what the compiler makes of the kernels."""
import ctypes
import inspect
import re
import types

import numpy as np
import pytest

import paper_2504_03661_amd as P
from oracle import paged_oracle as O
from paper_2504_03661_amd import binding as B
from tests.test_exchange_codegen_cpu import assembly, kernels
from tests.test_paged_boundary_cpu import HIGH, SAMPLES, Tensor

NAMES = ("fork", "free", "compact", "copy", "shared_decode")
MORE = {**SAMPLES, "n_groups": (2, 1, -1), "n_pairs": (9, 0, 2 ** 31 - 1), "n_from": (4, 2 ** 27 - 1, -3), "n_to": (6, 1, -2 ** 31),
        "workspace_bytes": (1 << 33, 0, -1)}


def test_a_fork_shares_whole_blocks_and_copies_the_rest():
    table = np.array([[4, 2, 7], [-1, -1, -1], [-1, -1, -1], [5, -1, -1]])
    got = O.fork([-1, 0, 3, 0], None, [40, 0, 0, 3], [0, 1, 3, 6, -1, -1, -1, -1], 4, table, np.zeros(8, int), 16)
    assert got["new_seq_len"].tolist() == [40, 40, 3, 3] and got["refused"]          # the last one is not empty
    assert got["block_table"].tolist() == [[4, 2, 7], [4, 2, 6], [3, -1, -1], [5, -1, -1]]
    assert got["holders"].tolist() == [0, 0, 1, 0, 1, 0, 0, 0]
    assert got["copy_src"].tolist() == [-1, 7, 5, -1] and got["copy_dst"].tolist() == [-1, 6, 3, -1]
    assert got["new_free_count"].tolist() == [2]
    got = O.fork([-1, 0, 0, -1], [9, 32, 33, 9], [40, 0, 0, 3], [0] * 8, 0, table, np.zeros(8, int), 16)
    assert got["new_seq_len"].tolist() == [40, 32, 0, 3] and got["refused"] and got["holders"][4] == 1


def test_a_block_goes_back_with_its_last_holder():
    table = np.array([[4, 2, 7], [4, 2, 6], [4, 3, -1]])
    holders = np.array([0, 0, 1, 0, 2, 0, 0, 0])
    got = O.free([-1, 1, -1], [40, 40, 20], [0, 1, 5, -1, -1, -1, -1, -1], 3, table, holders, 16)
    assert got["holders"].tolist() == [0] * 8 and not got["over"]
    assert got["free_list"].tolist() == [0, 1, 5, 7, 3, -1, -1, -1] and got["new_free_count"].tolist() == [5]
    got = O.free([0, -1, 0], got["new_seq_len"], got["free_list"], 5, table, got["holders"], 16)
    assert got["free_list"].tolist() == [0, 1, 5, 7, 3, 6, 4, 2] and got["new_seq_len"].tolist() == [0, 0, 0]


def test_live_blocks_move_below_the_free_ones():
    got = O.compact([40, 20], [0, 5, 2, 0, 0, 0, 0, 0], 3, np.array([[7, 3, 6], [7, 4, -1]]), np.array([0, 0, 0, 0, 0, 0, 0, 1]), 16)
    assert got["moved_to"].tolist() == [-1, 1, -1, 3, 4, -1, 2, 0]                   # five live ones: 7 to 0, 6 to 2
    assert got["copy_src"].tolist() == [7, 6] and got["copy_dst"].tolist() == [0, 2]
    assert got["new_block_table"].tolist() == [[0, 3, 2], [0, 4, -1]] and got["new_holders"].tolist() == [1, 0, 0, 0, 0, 0, 0, 0]
    assert got["new_free_list"].tolist() == [7, 6, 5] and not got["outside"]


def test_null_arguments_are_rejected_without_a_gpu():
    lib = P.load_library()
    for name in NAMES:
        f = getattr(lib, "pq_paged_" + name)
        assert f(*[1 if t in (ctypes.c_int32, ctypes.c_int64) else 1.0 if t is ctypes.c_float else None for t in f.argtypes]) == -1
    assert lib.pq_paged_shared_workspace_bytes(None, 1, 1) == -1


@pytest.mark.parametrize("module", [True, False], ids=["extension module", "ctypes"])
@pytest.mark.parametrize("name", NAMES)
def test_arguments_arrive_as_passed(monkeypatch, module, name):
    lib = B.load_library()
    if module and B._calls is None:
        pytest.skip("the extension module is not built here")
    f = getattr(B, "pq_paged_" + name)
    names = [p for p in inspect.signature(f).parameters if p not in ("ctx", "stream")]
    seen = []
    kind = ctypes.CFUNCTYPE(ctypes.c_int32, *getattr(lib, "pq_paged_" + name).argtypes)

    def through(fn):
        if module:
            monkeypatch.setitem(B._paged_at, name, ctypes.cast(fn, ctypes.c_void_p).value)
        else:
            monkeypatch.setattr(B, "_calls", None)
            monkeypatch.setattr(B, "_lib", types.SimpleNamespace(**{"pq_paged_" + name: fn, "pq_status_string": lib.pq_status_string}))

    listening = kind(lambda *a: seen.append(a) or 0)
    through(listening)
    for k in range(3):
        given = [MORE[n][k] if n in MORE else [Tensor(HIGH + 16 * i), 8 + i, None][(i + k) % 3] for i, n in enumerate(names)]
        f(HIGH, *given, stream=77)
        assert seen.pop() == (HIGH, *[x.at if isinstance(x, Tensor) else x for x in given], 77)
    with pytest.raises((TypeError, AttributeError)):
        f(HIGH, *[object() for _ in names], stream=0)
    assert not seen
    failing = kind(lambda *a: -4)
    through(failing)
    with pytest.raises(P.PQAttnError) as e:
        f(0, *[MORE[n][0] if n in MORE else None for n in names], stream=0)
    assert e.value.status == -4


@pytest.mark.parametrize("source", ["pq_paged_blocks.hip", "pq_paged_shared.hip"])
def test_no_kernel_spills(source, tmp_path):
    text = assembly(source, tmp_path)
    spills = {k: int(v) for k, v in re.findall(r"\.name:\s+(\S+)\s.*?\.vgpr_spill_count:\s+(\d+)", text, re.S) if "pq_paged" in k}
    assert spills
    for name, n in spills.items():
        assert n <= (8 if "If" in name else 0), (name, n)


def test_two_workgroups_of_shared_decode_fit_a_compute_unit(tmp_path):
    """What its grid and the cut of its work are made for: 256 of a SIMD's 512 registers a wavefront, half of 160 KB a workgroup.  And
    what is spilled to keep to that is not read in the loops over keys."""
    text = assembly("pq_paged_shared.hip", tmp_path)
    entries = {re.search(r"\.name:\s+(\S+)", e).group(1): e for e in re.findall(r"  - \.agpr_count.*?\.wavefront_size", text, re.S)}
    names = [k for k in entries if "pq_paged_shared_kernel" in k]
    assert len(names) == 3 * 2 * 3                              # types, dims, who plans
    bodies = kernels(text)
    for name, entry in entries.items():
        registers, lds, spilled = (int(re.search(rf"\.{field}:\s+(\d+)", entry).group(1))
                                   for field in ("vgpr_count", "group_segment_fixed_size", "vgpr_spill_count"))
        assert spilled <= (2 if name in names and "IfLi128" in name else 0), (name, spilled)
        if name not in names:
            continue
        assert registers <= 256 and lds <= 80 * 1024, (name, registers, lds)
        parts = re.split(r"^(?=\.LBB)", bodies[name], flags=re.M)
        products = [part for part in parts if "v_mfma" in part]
        assert products and not any("scratch_" in part for part in products), name
