"""Arguments of the calls around whole sequences and positions that are refused on the host, without a GPU."""
import pytest
import torch


def test_calls_without_a_handle_are_refused():
    from paper_2601_07891_b200 import binding
    lib = binding.load()
    assert lib.kvzap_cache_fork(None, None, None, 0, None) == 1
    assert lib.kvzap_cache_pack(None, None, 1, None, None, 0, None, None, None, None) == 1
    assert lib.kvzap_cache_unpack(None, None, 1, None, None, 0, None, None, None, None) == 1
    assert lib.kvzap_cache_share(None, None, None, 0, 8, 0, None) == 1
    assert lib.kvzap_decode_attention_shared(None, None, 0, 1, None, 8, 1.0, None, None) == 1
    assert lib.kvzap_decode_attention_shared_fp8(None, None, 0, 1, None, 8, 1.0, None, None) == 1
    assert lib.kvzap_set_rotary(None, None) == 1
    assert lib.kvzap_rotary(None, None, 0, None, 1, 0, None) == 1


def test_rows_of_the_wrong_shape_are_refused():
    from paper_2601_07891_b200 import binding
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    for out in (x.float(), x[:3], torch.zeros(4, 2, 64, dtype=torch.uint8), torch.zeros(4, 2, 66, dtype=torch.bfloat16)):
        with pytest.raises(ValueError, match="rows must be"):
            binding.rotary_rows(x, out, True)
    with pytest.raises(ValueError, match="CUDA"):
        binding.rotary_rows(x, x, True)


def test_structures_have_the_layout_of_the_header():
    import ctypes
    from paper_2601_07891_b200 import binding
    assert ctypes.sizeof(binding.KvzapRows) == 56
    assert ctypes.sizeof(binding.KvzapRotaryConfig) == 64
    assert binding.KvzapRotaryConfig.base.offset == 16
