"""Kernel names of the 4-bit operators and the experts in the profile summaries."""
from paper_2607_07862_amd import profsum as P


def test_short_names():
    tile = "mlp2::PTile<128, 2, 128, 2, 2, 4, 2>"
    assert (P.short_name(f"void mlp2::k_mx_product<{tile}, mlp2::MxProblem<mlp2::StoreMx<2, unsigned short> > >(mlp2::MxProblem<mlp2::StoreMx<2, unsigned short> >)")
            == "k_mx_product StoreMx<2, unsigned short> (tile 256 x 256, stages 2, waves 8)")
    assert P.short_name("void mlp2::k_mx_quantise_down<float>(mlp2::Quantise)") == "k_mx_quantise_down<float>"
    assert P.short_name("void mlp2::k_moe_mx<2, 1, false>(mlp2::Experts)") == "k_moe_mx<2, 1, false>"
    assert P.short_name("void mlp2::k_moe_route<unsigned short, 4>(mlp2::Route)") == "k_moe_route<unsigned short, 4>"
