"""Matrices and groups that die in any order, also inside reference cycles, leave no handle behind."""
import gc
import weakref

import numpy as np
import pytest

from paper_2607_08786_amd import usp


class Handles:
    """The library's rules for handles: a matrix that a group holds is not freed."""

    def __init__(self):
        self.live, self.groups, self.next = set(), {}, 0

    def _new(self, out):
        self.next += 1
        out._obj.value = self.next
        return self.next

    def usp_encode_q(self, *args):
        self.live.add(self._new(args[-1]))
        return 0

    def usp_info(self, handle, info):
        if handle not in self.live:
            return 1
        info._obj.M, info._obj.K = 3, 7
        return 0

    def usp_group_create(self, handles, count, out):
        if any(h not in self.live for h in handles):
            return 1
        self.groups[self._new(out)] = list(handles)
        return 0

    def usp_free(self, handle):
        if handle not in self.live or any(handle in g for g in self.groups.values()):
            return 1
        self.live.remove(handle)
        return 0

    def usp_group_free(self, group):
        return 0 if self.groups.pop(group, None) is not None else 1

    def usp_last_error(self):
        return b"refused"


@pytest.fixture
def lib(monkeypatch):
    h = Handles()
    monkeypatch.setattr(usp, "_lib", h)
    monkeypatch.setattr(usp, "load_library", lambda *a: h)
    monkeypatch.setattr(usp, "_shapes", {})
    monkeypatch.setattr(usp, "_ownerless", set(), raising=False)
    gc.collect()
    yield h
    gc.collect()


def matrix():
    one = np.ones((3, 7), np.int8)
    return usp.SparseMatrixQ(one, one.astype(np.uint8), np.ones(3, np.float32))


class Owner:
    pass


@pytest.mark.parametrize("experts", [1, 3])
def test_group_in_a_cycle(lib, experts):
    """The collector finalises the experts, which are older, before the group."""
    owner = Owner()
    owner.experts = [matrix() for _ in range(experts)]
    owner.group = usp.ExpertGroup(owner.experts)
    owner.self = owner
    gone = weakref.ref(owner)
    del owner
    gc.collect()
    assert gone() is None and not lib.groups and not lib.live


def test_experts_of_two_groups(lib):
    """Each held by what is left; the last group's end frees them."""
    owner = Owner()
    a, b = matrix(), matrix()
    owner.first = usp.ExpertGroup([a, b])
    second = usp.usp_group_create([b.handle, b.handle])
    owner.self = owner
    kept = b.handle
    del a, b, owner
    gc.collect()
    assert lib.live == {kept} and len(lib.groups) == 1
    usp.usp_group_free(second)
    assert not lib.live and not lib.groups


def test_plain_order(lib):
    """Without a cycle, and with the matrices' owners gone before the group."""
    g = usp.ExpertGroup([matrix(), matrix()])
    del g
    assert not lib.live and not lib.groups
    m = matrix()
    raw = usp.usp_group_create([m.handle])
    del m
    assert len(lib.live) == 1
    usp.usp_group_free(raw)
    assert not lib.live


def test_explicit_free_is_still_refused(lib):
    m = matrix()
    g = usp.ExpertGroup([m])
    with pytest.raises(usp.UspError):
        m.free()
    assert m.handle in lib.live
    g.free()
    assert m.handle in lib.live  # its owner lives
    m.free()
    assert not lib.live


def test_freed_elsewhere(lib):
    """A handle that its owner's end finds freed is not tried again: its number may be another's then."""
    m = matrix()
    h = m.handle
    usp.usp_free(h)
    del m
    lib.live.add(h)  # a new matrix with the same number
    usp.usp_group_free(usp.usp_group_create([h]))
    assert h in lib.live


def test_freed_by_number(lib):
    """A handle that outlived its owner and is then freed by its number is forgotten."""
    m = matrix()
    h = m.handle
    group = usp.usp_group_create([h])
    del m
    del lib.groups[group]
    usp.usp_free(h)
    lib.live.add(h)  # a new matrix with the same number
    usp.usp_group_free(usp.usp_group_create([h]))
    assert h in lib.live


def test_number_taken_meanwhile(lib):
    """Between a handle's end and the return of the call another thread may get its number, and lose the owner."""
    m = matrix()
    free = lib.usp_free

    def free_and_reuse(handle):
        status = free(handle)
        usp._shapes[handle] = (5, 5)
        usp._ownerless.add(handle)
        return status

    lib.usp_free = free_and_reuse
    h = m.handle
    m.free()
    assert usp._ownerless == {h} and usp._shapes == {h: (5, 5)}


@pytest.mark.gpu
def test_device_memory_of_a_cycle():
    """An expert group that dies in a cycle gives its experts' device memory back."""
    import torch
    from paper_2607_08786_amd import linear

    def cycle():
        codes, mask = torch.ones((2048, 8192), dtype=torch.int8), torch.ones((2048, 8192), dtype=torch.bool)
        m = linear.SparseExperts([codes, codes], [mask, mask], [torch.ones(2048)] * 2)
        m.myself = [m]  # not a child module

    cycle()
    gc.collect()
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    cycle()
    gc.collect()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] >= free - (4 << 20)  # two experts take 36 MB
    assert not usp._ownerless
