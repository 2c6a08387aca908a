"""The resource table says by itself what its columns are, so that writing it anew loses nothing."""
from paper_1904_05347_amd import resources

LOG = """\
csrc/pk_some.hip:10:0: remark: Function Name: _ZN2pk11some_kernelILi8EEEvPf [-Rpass-analysis=kernel-resource-usage]
csrc/pk_some.hip:10:0: remark:     TotalSGPRs: 20 [-Rpass-analysis=kernel-resource-usage]
csrc/pk_some.hip:10:0: remark:     VGPRs: 33 [-Rpass-analysis=kernel-resource-usage]
csrc/pk_some.hip:10:0: remark:     AGPRs: 4 [-Rpass-analysis=kernel-resource-usage]
csrc/pk_some.hip:10:0: remark:     ScratchSize [bytes/lane]: 16 [-Rpass-analysis=kernel-resource-usage]
csrc/pk_some.hip:10:0: remark:     Occupancy [waves/SIMD]: 7 [-Rpass-analysis=kernel-resource-usage]
csrc/pk_some.hip:10:0: remark:     SGPRs Spill: 2 [-Rpass-analysis=kernel-resource-usage]
csrc/pk_some.hip:10:0: remark:     VGPRs Spill: 1 [-Rpass-analysis=kernel-resource-usage]
csrc/pk_some.hip:10:0: remark:     LDS Size [bytes/block]: 1024 [-Rpass-analysis=kernel-resource-usage]
"""


def test_the_table_has_its_legend(tmp_path):
    log = tmp_path / "usage.log"
    log.write_text(LOG)
    lines = resources.table(str(log)).splitlines()
    head = [l for l in lines if l.startswith("#")]
    assert head == lines[:len(head)] and any("command:" in l for l in head) and any("source:" in l for l in head)
    columns = lines[len(head)].split()
    assert columns == ["file", "kernel", "vgpr", "agpr", "sgpr", "vspill", "sspill", "scratch", "lds", "occ"]
    for name in columns[2:]:
        assert name == "sgpr" or name in " ".join(head)
    assert lines[-1].split() == ["pk_some.hip", "some_kernel<8>", "33", "4", "20", "1", "2", "16", "1024", "7"]
    assert len(lines) == len(head) + 2


def test_the_table_that_is_kept_has_it():
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "profiles", "kernel_resources.txt")
    with open(path) as fh:
        assert fh.read().startswith(resources.LEGEND)
