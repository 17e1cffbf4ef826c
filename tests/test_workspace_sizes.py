"""What users' sampling options and adapters cost a context that uses neither:
a few words a slot.  Both work in buffers of the pass that are idle at the time.
Host only; no call here touches a GPU."""
import ctypes

import pytest

from paper_2604_20919_amd import sdverify as sv

SHAPES = {"qwen3-1.7b": (28, 2048, 16, 8, 128, 6144, 151936, 1, sv.SD_BF16),
          "qwen3-32b": (64, 5120, 64, 8, 128, 25600, 151936, 1, sv.SD_BF16),
          "fp32": (2, 256, 4, 2, 64, 512, 151936, 0, sv.SD_F32)}


def workspace(shape, T, B, P):
    return sv.sd_verify_query_sizes(sv.make_config(*SHAPES[shape], 256, 64, 12, B, T, 1029, P))[1]


@pytest.mark.parametrize("shape,T,B,P,forward", [
    # bytes of the pass's own buffers, without options and adapters
    ("qwen3-1.7b", 2, 1, 1, 15782656), ("qwen3-1.7b", 80, 16, 2, 179485696), ("qwen3-1.7b", 229, 32, 2, 461975040),
    ("qwen3-1.7b", 416, 32, 8, 3265824768), ("qwen3-32b", 2, 1, 1, 58323712), ("qwen3-32b", 80, 16, 2, 343161856),
    ("qwen3-32b", 229, 32, 2, 775785984), ("qwen3-32b", 416, 32, 8, 5274765312), ("fp32", 80, 16, 2, 98908672),
    ("fp32", 229, 32, 2, 282890752), ("fp32", 416, 32, 8, 2054971392),
])
def test_contexts_pay_for_the_pass_alone(shape, T, B, P, forward):
    # six staged words a slot, each table rounded up to 256 bytes, a pending batch
    assert workspace(shape, T, B, P) <= forward + P * 6 * (4 * T + 256)


def test_small_contexts_hold_one_filtered_row():
    """Where the pass's buffers are smaller than one row's records, they grow to that."""
    assert workspace("fp32", 2, 1, 1) <= 1277696 + sv.sd_filter_query_size(1, 151936) + 6 * 264


def test_filter_records_follow_the_vocabulary():
    # a row cannot have more members of a bucket than tokens
    assert sv.sd_filter_query_size(1000, 64) < 1000 * (2048 + 64 * 8 + 512)
    assert sv.sd_filter_query_size(416, 151936) > 416 * 16384 * 8
    sizes = [sv.sd_filter_query_size(n, 40000) for n in (1, 2, 16, 255, 256, 4000)]
    assert sizes == sorted(sizes)


def test_adapter_workspace_follows_the_input():
    off = (ctypes.c_int32 * 5)(0, 64)
    size = ctypes.c_uint64()

    def need(d_in, rank, n, dtype=sv.SD_BF16):
        p = ctypes.c_void_p(4096)
        w = sv.sd_lora(3, rank, d_in, 64, 1, off, dtype, p, p, None)
        assert sv.lib().sd_lora_query_size(ctypes.byref(w), n, ctypes.byref(size)) == sv.SD_OK
        return size.value

    assert need(100, 64, 1000) < 1000 * 64 * 4 * 1.1 + 512  # one range of k
    for a, b in ((need(100, 8, 50), need(5000, 8, 50)), (need(512, 8, 50), need(512, 128, 50)),
                 (need(512, 8, 50), need(512, 8, 4000)), (need(512, 8, 50), need(512, 8, 50, sv.SD_F32))):
        assert a <= b
