"""CPU-only tests of the benchmark's own arithmetic."""
import bench


def test_mxfp4_block_is_priced_against_what_takes_longer():
    # one token, six experts: 28 MB of weights against 0.1 GFLOP
    r = bench.mxfp4_roofline(27.6e6, 0.104e9, 30.0)
    assert r["bound"] == "hbm" and abs(r["frac"] - 27.6e6 / 30e-6 / 8e12) < 1e-9
    # a prompt of 8192 tokens: 294 MB (37 us at 8 TB/s) against 850 GFLOP (85 us at 10 PFLOP/s)
    r = bench.mxfp4_roofline(294e6, 850e9, 500.0)
    assert r["bound"] == "mfma" and r["unit"] == "TFLOP/s" and abs(r["achieved"] - 1700.0) < 1e-6 and abs(r["frac"] - 0.17) < 1e-9
