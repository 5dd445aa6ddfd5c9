"""Host checks of the group norm's test hook: no GPU."""


def test_most_ctas_of_a_cluster():
    from paper_2609_13716_gb300 import aht, build
    build.build()
    L = aht.load()
    for bad in (-1, 1, 4, 12, 32):
        assert L.aht_debug_group_norm_cluster(bad) == aht.AHT_EINVAL and b"most" in L.aht_last_error()
    for good in (8, 16, 0):
        assert L.aht_debug_group_norm_cluster(good) == aht.AHT_OK
