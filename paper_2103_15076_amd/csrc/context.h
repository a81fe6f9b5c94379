// context.h -- what the library's other translation units may ask of a context (its layout is picasso.hip's own).
#pragma once
struct picasso_ctx;

int picasso_device_of(const picasso_ctx* c);
void picasso_note_hip_error(picasso_ctx* c, const char* text);  // for picasso_last_hip_error
