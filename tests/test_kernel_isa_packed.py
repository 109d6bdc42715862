"""Build-time checks of the packed attention kernels' assembly (gfx950, the library's own flags): the hazards that the compiler does not
see in their asynchronous copies, and that nothing in a tile waits for the next tile's copies."""
from test_kernel_isa import _assembly, _check_m0, _check_valu_sgpr_to_vmem, _functions


def test_packed_attention_copies():
    text = _assembly("attention_packed.hip")
    _check_m0(text, "attention_packed.hip")
    _check_valu_sgpr_to_vmem(text, "attention_packed.hip")
    seen = 0
    for name, body in _functions(text).items():
        mf = [i for i, ins in enumerate(body) if ins.startswith("v_mfma")]
        if mf:
            seen += 1
            assert not any("vmcnt" in ins for ins in body[mf[0]:mf[-1] + 1]), name
            # (a spilled register that is read back there would wait for the copies in flight)
            assert not any("scratch_" in ins for ins in body[mf[0]:mf[-1] + 1]), name + " spills"
    assert seen >= 6                     # three kernels, two head sizes
