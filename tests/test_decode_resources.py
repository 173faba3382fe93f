"""CPU check of what the compiler made of the decode-step kernels."""
from test_kernel_resources import _kernels


def test_decode_kernels_spill_nothing():
    # launches of a few microseconds: any scratch makes them longer, and a reload in
    # a weight stream waits on the stream's own counter
    names = ("ld_first_kernel", "ld_up_kernel", "ld_down_kernel", "ld_join_kernel", "pa_kernel",
             "pa_row_kernel", "pa_join_kernel", "beam_rows_kernel", "beam_merge_kernel", "beam_reorder_kernel")
    kernels = _kernels()
    for name in names:
        mine = {n: (k[".vgpr_spill_count"], k[".private_segment_fixed_size"])
                for n, k in kernels.items() if name in n}
        assert mine, name
        assert not {n: v for n, v in mine.items() if any(v)}
