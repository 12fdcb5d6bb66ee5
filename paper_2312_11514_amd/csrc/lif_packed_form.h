// Which kernel takes a product, by the number of outputs and rows (host code).
#pragma once

namespace lif {

// Tiles of 16 outputs for up to 4, 8 or 16 rows, the inputs dealt to the waves (k_packed_few); or workgroups of so many outputs and rows (k_packed_many; _16: in
// 16 waves, where there is the same in 8).
enum class PackedForm { few4, few8, few16, outs32_rows16, outs32_rows16_16, outs32_rows32, outs32_rows32_16, outs48_rows32, outs48_rows48, outs64_rows16, outs64_rows32,
                        outs64_rows32_16, outs64_rows48, outs64_rows64, outs64_rows64_16, outs80_rows64, outs96_rows32, outs96_rows64, outs112_rows48, outs128_rows64 };

// A larger workgroup reads and unpacks less for an output, but where there are fewer of them than the 256 compute units its own time is that of the call.
// So a call is taken to last `alone` where the workgroups fit the chip at once, one to a compute unit, and `more` for every 256 beyond, three quarters of it for the
// first of them (outs128_rows64: 256 workgroups 28.4 us, 258 42.8, 512 45.0): us for 4096 inputs in fp16 with groups of 128, in fp32 with groups of 64 and zero
// points, from 17 to 1024 rows by 1024 to 50000 outputs.  More than 8 waves begin and add up half a microsecond later, whatever the inputs; but for that other
// inputs, types and groups scale the times alike.  Widths of 48, 80, 96 and 112 outputs are there for what 64 and 128 leave idle (48 rows by 18176, bytes with scales
// by groups of 64: outs80_rows64 24, the next one 26; 24 rows by 11008, fp16: outs48_rows32 9.6, 10.3; 32 by 18176, fp16: outs96_rows32 15.3, 17.2; 256 by 11008, bf16,
// groups of 32: outs96_rows64 58, 64; 48 by 22016, fp16, groups of 64: outs112_rows48 21.8, 22.8), more waves for long inputs (60 rows of 11008 by 4096, bf16, groups
// of 32: 8 waves 22.9, 16 21).
// Against the fastest of these forms the rule's choice loses 0.6 % on average and 6 % at most in fp16, 0.7 and 9 % in bf16 with groups of 32, 1.6 and 20 % in bytes
// with scales by groups of 64 (1024, 4096 and 11008 inputs), 0.3 and 3 % in fp32.
// E.g. 4096 outputs, fp16: 24 rows 5.7 (few16 6.0, outs64_rows32_16 9.3), 128 rows 10.4 (outs32_rows16 14.0, outs64_rows64 15.8), 512 rows 28.5 (outs64_rows32
// 33.0, outs64_rows64 29.6); 50000 outputs: 24 rows 31.8 (few16 51.9), 512 rows 295 (outs64_rows32 373, outs64_rows64 331).
struct PackedCost {
    PackedForm form;
    int tiles, rows, waves;      // of a workgroup
    float alone, more;
    int group;                   // the smallest it is compiled for: with less, registers go to memory
};
constexpr PackedCost kPackedCosts[] = {
    {PackedForm::few16, 1, 16, 8, 4.3f, 1.9f, 32},
    {PackedForm::outs32_rows16, 2, 16, 8, 5.5f, 3.f, 32},
    {PackedForm::outs32_rows16_16, 2, 16, 16, 5.5f, 3.4f, 32},
    {PackedForm::outs32_rows32, 2, 32, 8, 7.4f, 5.f, 32},
    {PackedForm::outs32_rows32_16, 2, 32, 16, 7.5f, 6.7f, 32},
    {PackedForm::outs48_rows32, 3, 32, 15, 9.2f, 8.7f, 32},
    {PackedForm::outs48_rows48, 3, 48, 12, 10.6f, 10.3f, 32},
    {PackedForm::outs64_rows32, 4, 32, 8, 11.5f, 7.f, 32},
    {PackedForm::outs64_rows32_16, 4, 32, 16, 9.9f, 9.3f, 32},
    {PackedForm::outs64_rows48, 4, 48, 8, 13.2f, 9.8f, 32},
    {PackedForm::outs64_rows64, 4, 64, 8, 15.5f, 12.f, 64},
    {PackedForm::outs64_rows64_16, 4, 64, 16, 14.4f, 15.8f, 64},
    {PackedForm::outs80_rows64, 5, 64, 15, 17.4f, 18.9f, 64},
    {PackedForm::outs96_rows32, 6, 32, 12, 13.7f, 10.9f, 32},
    {PackedForm::outs96_rows64, 6, 64, 12, 20.4f, 21.5f, 32},
    {PackedForm::outs112_rows48, 7, 48, 14, 19.7f, 19.8f, 32},
    {PackedForm::outs128_rows64, 8, 64, 8, 25.7f, 21.1f, 32}};
constexpr PackedCost kPackedCostsF32[] = {
    {PackedForm::few16, 1, 16, 4, 11.5f, 6.2f, 32},
    {PackedForm::outs32_rows16, 2, 16, 8, 13.4f, 12.f, 32},
    {PackedForm::outs64_rows16, 4, 16, 8, 19.5f, 13.3f, 32},
    {PackedForm::outs128_rows64, 8, 64, 8, 70.f, 75.f, 32}};

// tiles: of 16 outputs; in_tiles: of 128 inputs
inline PackedForm packed_form(int tiles, int in_tiles, int rows, bool f32, int group) {
    if (rows <= 16) return rows <= 4 ? PackedForm::few4 : rows <= 8 ? PackedForm::few8 : PackedForm::few16;
    PackedForm best = PackedForm::few16;
    float least = 0.f;
    bool none = true;
    auto look = [&](const PackedCost& c) {
        if (group < c.group) return;
        const float groups = (float)((tiles + c.tiles - 1) / c.tiles) * (float)((rows + c.rows - 1) / c.rows) / 256.f;
        const float beyond = groups > 1.f ? groups - 1.f : 0.f, begun = (float)(long long)beyond + ((float)(long long)beyond < beyond ? 1.f : 0.f);
        const float late = c.waves > 8 ? 0.5f * (32.f / (float)in_tiles - 1.f) : 0.f;
        const float time = c.alone + c.more * (0.75f * begun + 0.25f * beyond) + late;
        if (none || time < least) best = c.form, least = time, none = false;
    };
    if (f32)
        for (const PackedCost& c : kPackedCostsF32) look(c);
    else
        for (const PackedCost& c : kPackedCosts) look(c);
    return best;
}

}  // namespace lif
