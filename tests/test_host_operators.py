"""Host code of the block-scaled contraction's plans and of AdamW's under AddressSanitizer and UndefinedBehaviorSanitizer, on the CPU (tests/sanitize/operators_driver.hip)."""
import os
import subprocess

from tests.test_host_sanitizers import ENV, SAN, _hipcc_host


def test_plans_of_block_contractions_and_adamw_by_brute_force(tmp_path):
    exe = _hipcc_host(tmp_path, "operators_san", [os.path.join(SAN, "operators_driver.hip")], extra=("-Wl,--unresolved-symbols=ignore-all",))
    p = subprocess.run([exe], env=dict(ENV, LLMQ_TUNING="1"), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert p.returncode == 0 and "operators driver ok" in p.stdout, p.stdout[-3000:]
    assert "AddressSanitizer" not in p.stdout and "runtime error" not in p.stdout, p.stdout[-3000:]
