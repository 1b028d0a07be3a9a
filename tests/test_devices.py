"""What a process does once per device, without a GPU."""
import ctypes

import paper_2603_02298_amd as lc


def test_once_on_every_device():
    """A kernel's LDS limit has to be raised on each device that it runs on, also where another device had it raised first."""
    devices = [0, 0, 1, 0, 1, 7, 63, 63, 7, 64, 64, -1, 0]
    due = ctypes.create_string_buffer(len(devices))
    lc.lib().lc_debug_due_on_devices((ctypes.c_int * len(devices))(*devices), len(devices), due)
    assert list(due.raw) == [1, 0, 1, 0, 0, 1, 1, 0, 0, 1, 1, 1, 0]   # (64 and beyond are not remembered)
