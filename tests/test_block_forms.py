"""The kernels of packed attention, the RMS norm and the balance loss keep their state in registers."""
import re
import subprocess

from test_built_code import READELF, objects  # noqa: F401


def test_the_kernels_stay_in_registers(objects):  # noqa: F811
    spills = {}
    for path in objects:
        r = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True, check=True)
        names = re.findall(r"^\s+\.name:\s+(_Z\w+)$", r.stdout, flags=re.M)
        counts = re.findall(r"^\s+\.vgpr_spill_count:\s+(\d+)$", r.stdout, flags=re.M)
        assert len(names) == len(counts)
        spills.update((n, int(c)) for n, c in zip(names, counts) if re.match(r"_ZN2xs(5pattn|4norm|7balance)", n))
    assert len(spills) > 60
    assert {n: c for n, c in spills.items() if c} == {}
