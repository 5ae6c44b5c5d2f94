"""The 8-bit pool, rotate-and-append and the window at the C ABI, as far as no device is needed."""
import ctypes as C

from paper_2609_34388_b200 import binding


def test_pool_bytes_of_an_8_bit_pool():
    lib = binding.lib()
    cfg = binding.recg_config(32, 4096, 32, 8, 128, 14336, 128256, 5e5, 1e-5, -1, 16, 16, 1024, 600, binding.FLAG_KV_8BIT)
    # per page and head: 2 x 16 x 128 bytes of codes and 8 bytes of header; layers begin at multiples of 128
    assert lib.recg_kv_pool_bytes(C.byref(cfg), 10) == 32 * (10 * 8 * (2 * 16 * 128 + 8))
    cfg.head_dim, cfg.n_layers = 64, 3
    assert lib.recg_kv_pool_bytes(C.byref(cfg), 3) == 3 * ((3 * 8 * (2 * 16 * 64 + 8) + 127) // 128 * 128)


def test_refusals_that_need_no_device():
    lib = binding.lib()
    assert lib.recg_window(None, 0, 0) == 1
    assert lib.recg_kv_append_rotary(None, None, 0, None, 0, None, None, None, 0) == 1
    cfg = binding.recg_config(1, 64, 4, 2, 64, 64, 64, 1e4, 1e-5, -1, 16, 1, 8, 4, binding.FLAG_KV_8BIT | binding.FLAG_KV_4BIT)
    h = C.c_void_p()
    assert lib.recg_init(C.byref(h), C.byref(cfg), None, None) == 1 and b"not both" in lib.recg_last_error(None)
