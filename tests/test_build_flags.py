"""Compiler flags that results or speed rest on."""
from paper_2608_19920_amd import build


def test_nan_quieting_by_source():
    """The prefill kernels' maxima see no NaN and take none of the instructions that
    quiet one (mfma_lse at B4 Hq32 Hkv8 d128 M32768 T512: 593 us, 615 with them); the
    one-sweep kernels keep the NaN of an 8-bit row."""
    quiet = "-fno-honor-nans"
    assert quiet in build.flags_for("sdpa_mfma.hip")
    for src in ("flash.hip", "flash_f32.hip", "decode.hip", "quant.hip", "select.hip"):
        assert quiet not in build.flags_for(src)


def test_no_packed_float32():
    for src in ("sdpa_mfma.hip", "flash.hip", "select.hip"):
        f = build.flags_for(src)
        assert any(f[i:i + 4] == ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
                   for i in range(len(f)))
