"""The compiled marshalling of the operators: what it is linked to, when it is built again, and its messages."""
import shutil
import subprocess

import pytest
import torch

import paper_2407_09722_b200 as M
from paper_2407_09722_b200 import build as Bd


@pytest.fixture(scope="module", autouse=True)
def lib():
    Bd.build()
    return M.load_library()


@pytest.mark.skipif(shutil.which("nm") is None, reason="binutils")
def test_the_module_has_no_c_library_of_its_own():
    """One C++ library a process: streams that torch has made look for their number formats in the copy that made them."""
    names = subprocess.run(["nm", "-DC", "--defined-only", Bd.OPS], capture_output=True, text=True, check=True).stdout
    assert "PyInit__ops" in names and "std::locale::classic()" not in names


def test_messages_with_numbers():
    from paper_2407_09722_b200 import ops
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    table, lens = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="at least 48 slots"):
        M.paged_evict(k, k, table, lens, torch.zeros(1, 2, 40), 8, max_len=48)
    with pytest.raises(ValueError, match=r"got \[2, 3, 4, 32\]"):
        M.paged_attention(torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16)[:, :, :, ::2], k, k, table.expand(2, -1).contiguous(), lens)
    with pytest.raises(TypeError, match="expected 14 arguments, got 2"):
        ops._ops().evict(k, k)


def test_the_module_belongs_to_one_torch(monkeypatch):
    """Built against another torch it is built again, and not loaded before that."""
    from paper_2407_09722_b200 import ops
    assert ops._ops().torch_version == torch.__version__ and not Bd.ops_stale()
    with monkeypatch.context() as m:
        m.setattr(torch, "__version__", "2.0.0+other")
        assert Bd.ops_stale()
        m.setattr(ops, "_mod", None)
        with pytest.raises(RuntimeError, match="another torch"):
            ops._ops()
    assert not Bd.ops_stale()


def test_headers_come_from_the_compiler_in_use(monkeypatch):
    """NVCC names the toolkit, and the marshalling takes its headers from there too."""
    seen = []
    monkeypatch.setenv("NVCC", "/elsewhere/cuda/bin/nvcc")
    monkeypatch.setattr(Bd.subprocess, "run", lambda cmd, **kw: seen.append(cmd))
    Bd.build_ops()
    assert "/elsewhere/cuda/include" in seen[0] and "/usr/local/cuda/include" not in seen[0]
