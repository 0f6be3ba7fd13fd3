"""Tables of more places than a 32-bit count holds are refused, on the host: the made-up device addresses are never followed."""
from paper_2511_18871_amd import binding as B

FAR = [(i + 1) << 44 for i in range(5)]


def test_fit_refuses_more_places_than_it_counts():
    lib = B.load_library()
    for n_seqs, width in ((1 << 16, 1 << 15), (1 << 15, (1 << 16) + 1), ((1 << 31) - 1, 2), (2, (1 << 31) - 1)):
        assert lib.sp_attn_pages_fit(FAR[0], 10, 16, n_seqs, FAR[1], width, FAR[2], FAR[3], FAR[4], 1 << 40, None) == B.SP_ERR_INVALID_ARG, (n_seqs, width)
        assert b"places" in lib.sp_attn_last_error()
