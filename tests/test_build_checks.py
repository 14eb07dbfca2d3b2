"""The build's look at hipcc's resource remarks: which kernels may spill, and how far (host logic; no GPU)."""
import pytest

from paper_2407_02068_amd import build

PRE = "csrc/x.hip:1:1: remark: "


def remarks(kernel, scratch):
    return [PRE + "Function Name: " + kernel + " [-Rpass-analysis=kernel-resource-usage]",
            PRE + "    VGPRs: 256 [-Rpass-analysis=kernel-resource-usage]",
            PRE + "    ScratchSize [bytes/lane]: %d [-Rpass-analysis=kernel-resource-usage]" % scratch]


ROWS = "_ZN3lpv12_GLOBAL__N_112k_quant_rowsILi%dELi%dELi%dELi%dELi%dELb1EEEvNS0_9QuantDimsEPKcS4_S4_S4_PcPaPf"
PANEL = "_ZN3lpv12_GLOBAL__N_113k_quant_panelILi0ELb1ELi4ELi8ELi4EEEvNS0_9PanelDimsEPKcS4_S4_PK15HIP_vector_typeIjLj2EES4_S4_Pc"


@pytest.mark.parametrize("kernel,most", [
    ("_ZN3lpv12_GLOBAL__N_110k_linear16ILi2EEEv", 0), ("_ZN3lpv12_GLOBAL__N_112k_linear_f32Ev", 0), (PANEL, 32),
    (ROWS % (2, 1, 64, 3, 4), 0), (ROWS % (0, 2, 256, 4, 8), 0), (ROWS % (0, 2, 1024, 4, 8), None),
    ("_ZN3lpv12_GLOBAL__N_111k_quant_fewILi0ELb1ELi4ELi4EEEv", None)])
def test_spills(kernel, most):
    assert build.check_resources(remarks(kernel, 0)) == []
    for n in (1, 24, 32, 33, 64, 1412):
        bad = build.check_resources(remarks(kernel, n))
        assert len(bad) == (most is not None and n > most)
        assert not bad or (kernel in bad[0] and str(n) in bad[0])


def test_each_kernel_has_its_own_line():
    lines = remarks(PANEL, 28) + remarks(ROWS % (0, 2, 256, 4, 8), 8) + remarks(ROWS % (0, 2, 1024, 4, 8), 900)
    assert len(build.check_resources(lines)) == 1
