"""The binding keeps the tables' tensors on one device, the current one (no GPU: stand-ins for tensors)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2503_01586_b200 import binding as ek


class OnDevice:
    """What make_tables asks of a tensor before it makes the outputs."""
    is_cuda, dtype = True, torch.int32

    def __init__(self, index, n=8):
        self.device, self.n = torch.device("cuda", index), n

    def is_contiguous(self):
        return True

    def numel(self):
        return self.n


@pytest.mark.parametrize("other", ["fresh", "parent", "page_table", "pages_held", "free_pages", "n_free"])
def test_tensors_of_two_devices_are_refused(other):
    args = {k: OnDevice(0) for k in ("held", "fresh", "parent", "page_table", "pages_held", "free_pages", "n_free")}
    args[other] = OnDevice(1)
    with pytest.raises(ValueError, match="one device"):
        ek.make_tables(2, 8, 4, **args)


def test_tables_of_another_device_than_the_current_one_are_refused(monkeypatch):
    calls = []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(ek, "lib", lambda: calls.append(1))
    with pytest.raises(ValueError, match="another device"):
        ek.elitekv_step_tables(ek.CacheDesc(), SimpleNamespace(device=0, desc=ek.TablesDesc(), B=1, n_slots=1, m=0))
    assert not calls


@pytest.mark.parametrize("workspace", [torch.empty(64, dtype=torch.uint8), SimpleNamespace(is_cuda=True, is_contiguous=lambda: False)])
def test_a_workspace_in_host_memory_or_with_gaps_is_refused(monkeypatch, workspace):
    """A pointer that the kernels could not read, or bytes that are not one piece."""
    monkeypatch.setattr(ek, "lib", lambda: pytest.fail("reached the library"))
    layer, bf16 = SimpleNamespace(handle=None, n_h=2, r=2, d_c=8, d_h=16, kw=8), torch.bfloat16
    with pytest.raises(ValueError, match="workspace"):
        ek.elitekv_attend_tree(layer, ek.CacheDesc(), torch.zeros(3, 4, 2, 4, dtype=bf16), torch.zeros(3, 4, 2, 8, dtype=bf16),
                               torch.zeros(3, dtype=torch.int32), None, torch.zeros(3, 4, dtype=torch.int64), workspace,
                               torch.zeros(3, 4, 2, 16, dtype=bf16))


@pytest.mark.parametrize("rows,n_free", [(7, 1), (8, 0)])
def test_a_page_table_of_too_few_rows_and_a_count_of_no_entries_are_refused(rows, n_free):
    args = {k: OnDevice(0) for k in ("held", "fresh", "parent", "page_table", "pages_held", "free_pages")} | {"n_free": OnDevice(0, n_free)}
    args["parent"].n, args["page_table"].shape = 32, (rows, 3)
    with pytest.raises(ValueError, match="a row per sequence"):
        ek.make_tables(8, 32, 4, **args)
