"""Kernel names of the rocprofv3 summaries."""
import pytest

from paper_2608_11231_amd import rocprof_summary as R

NAMES = [
    ("_ZN3lkv15kv_write_kernelIDF16bLb1ELi64EEEvNS_6KvArgsE", "lkv::kv_write_kernel<bf16,true,64>"),
    ("_ZN3lkv16attn_join_kernelILi64EfEEvNS_8AttnArgsE.kd", "lkv::attn_join_kernel<64,float>"),
    ("_ZN3lkv16attn_tile_kernelILi128ELi0ELb0ELi1EEEvNS_8AttnArgsE", "lkv::attn_tile_kernel<128,0,false,1>"),
    ("_ZN3lkv13gather_kernelENS_10GatherArgsE", "lkv::gather_kernel"),
    ("void lkv::chunk_kernel<0, 128, 64, false, 4, true, 2>(lkv::ChunkArgs)", "lkv::chunk_kernel<0,128,64,false,4,true,2>"),
    ("__amd_rocclr_copyBuffer", "__amd_rocclr_copyBuffer"),
    ("_ZN2at6native29vectorized_elementwise_kernelILi4E", "_ZN2at6native29vectorized_elementwise_kernelILi4E")]


@pytest.mark.parametrize("name,short", NAMES)
def test_short_names(name, short):
    assert R.short_name(name) == short
