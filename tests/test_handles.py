"""The handles of an 8-bit cache and of sampling rules hold the addresses of the
tensors that they are made of, so a tensor is not replaced behind their back."""
import pytest
import torch

from paper_2601_09083_amd import srt as S

NAMES = ("k_pages", "v_pages", "k_scale", "v_scale", "k_tail", "v_tail", "block_table", "ctx_len", "tensors")


@pytest.mark.parametrize("name", NAMES)
def test_a_cache_does_not_take_another_tensor(name):
    kv = S.KvQuant.__new__(S.KvQuant)  # (a whole one needs a GPU)
    kv._tensors = tuple(torch.zeros(1) for _ in range(8))
    with pytest.raises(AttributeError):
        setattr(kv, name, torch.zeros(1))


def test_a_cache_is_updated_in_place():
    kv = S.KvQuant.__new__(S.KvQuant)
    kv._tensors = tuple(torch.zeros(1) for _ in range(8))
    kv.ctx_len += 1
    assert kv._tensors[7].tolist() == [1.0] and kv.ctx_len is kv._tensors[7]


def test_rules_do_not_take_another_tensor():
    rules = S.Rules(seen=torch.zeros((1, 4), dtype=torch.int16))
    with pytest.raises(TypeError):
        rules.tensors["mask"] = torch.zeros(1)
    assert rules.tensors["mask"] is None and rules.tensors["seen"].shape == (1, 4)


@pytest.mark.gpu
def test_a_cache_gives_its_tensors():
    page = torch.zeros((3, 2, 16, 64), dtype=torch.int8, device="cuda")
    one = [page, page.clone(), torch.zeros((3, 2), device="cuda"), torch.zeros((3, 2), device="cuda"),
           *(torch.zeros((1, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)),
           torch.zeros((1, 3), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")]
    kv = S.KvQuant(*one)
    assert all(getattr(kv, name) is x for name, x in zip(NAMES, one)) and all(x is y for x, y in zip(kv.tensors, one))
