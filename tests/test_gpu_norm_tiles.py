"""GPU parity: cafeq_norm_quantize through a transform where a workgroup takes several tiles of 32 tokens, one after another, and where it forms the norms of
several rows itself.  Inputs, float64 reference and tolerances are those of tests/test_gpu_norm.py."""
import pytest

from tests.test_gpu_norm import _check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


# 2 to 5 tiles a workgroup: 256 compute units hold 1024 (k = 32, 64), 512 (128) or 256 (256) workgroups, one a tile of 128 columns
WALKS = [(32, 2600, 4640), (64, 2331, 4672), (128, 2053, 4608), (256, 1001, 4608), (128, 5003, 1152), (256, 4500, 1280)]


@pytest.mark.parametrize("k,n,d", WALKS)
@pytest.mark.parametrize("dtype,group,values,pad", [("bf16", 32, "bf16", 16), ("f32", 32, "f32", 16), ("bf16", 0, "f32", 0), ("f32", None, "f32", 0), ("bf16", None, "bf16", 16)])
def test_several_tiles_a_workgroup(env, k, n, d, dtype, group, values, pad):
    _check(env, n, d, dtype, k=k, group=group, values=values, pad=pad)


@pytest.mark.parametrize("k,n,d", WALKS[2:])
def test_several_tiles_a_workgroup_in_groups_of_128(env, k, n, d):
    _check(env, n, d, "bf16", k=k, group=128, values=None, pad=8)
    _check(env, n, d, "f32", k=k, group=128, values="bf16", residual=False)


@pytest.mark.parametrize("k,n,d", [(32, 2600, 4640), (256, 1001, 4608)])
def test_several_tiles_a_workgroup_without_a_norm(env, k, n, d):
    _check(env, n, d, "bf16", k=k, group=32, norm=False, gain=False, values="bf16")


@pytest.mark.parametrize("k,d", [(32, 96), (32, 4640), (64, 192), (64, 2880), (128, 128), (128, 4608), (256, 256), (256, 3584)])
@pytest.mark.parametrize("n", [2, 3, 4, 5, 6, 7, 8, 9, 32])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_few_rows(env, k, d, n, dtype):
    _check(env, n, d, dtype, k=k, group=32, values=dtype, pad=16)
    _check(env, n, d, dtype, k=k, group=None, values="f32", residual=False)
